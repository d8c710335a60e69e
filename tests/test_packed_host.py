"""Refusals of attention over packed sequences, on the host: nothing is launched (no GPU is needed), the addresses are never read."""
import pytest

P = pytest.importorskip("paper_2605_23445_amd")
from paper_2605_23445_amd import binding as B  # noqa: E402

lib = B._lib
AT = 1 << 32
GOOD = dict(seqs=3, heads=8, heads_kv=2, d=128, n_q=900, n_k=900, left=-1, right=0)


def _view(i, head=1 << 20, row=128, at=None):
    return B._View(AT * i if at is None else at, 0, head, row)


def _call(back=False, dtype=1, q_start=AT * 20, k_start=None, scale=0.1, lse=AT * 21, ws=AT * 22, ws_bytes=1 << 40, geom=None, **views):
    w = None if geom == "none" else P.Packed(**dict(GOOD, **(geom or {})))
    v = {n: views.get(n, _view(i + 1)) for i, n in enumerate(("q", "k", "v", "o", "d_o", "dq", "dk", "dv"))}
    if back:
        return lib.dfs_packed_attn_bwd(w, dtype, v["q"], v["k"], v["v"], v["o"], lse, v["d_o"], q_start, k_start, scale, v["dq"], v["dk"], v["dv"], ws, ws_bytes, None)
    return lib.dfs_packed_attn_fwd(w, dtype, v["q"], v["k"], v["v"], q_start, k_start, scale, v["o"], lse, ws, ws_bytes, None)


@pytest.mark.parametrize("back", [False, True])
@pytest.mark.parametrize("geom,code", [
    ("none", -1), (dict(seqs=-1), -2), (dict(seqs=1 << 24), -2), (dict(n_q=-1), -2), (dict(n_k=(1 << 28) + 1), -2), (dict(n_q=899), -2), (dict(heads=0), -2),
    (dict(heads=65536), -2), (dict(heads_kv=3), -2), (dict(heads_kv=0), -2), (dict(d=96), -2), (dict(heads=10, heads_kv=1, n_q=1 << 27, n_k=1 << 27), -2),
    (dict(heads=60000, heads_kv=60000, n_q=1 << 20, n_k=1 << 20), -2), (dict(seqs=(1 << 23)), -2)])
def test_geometries(geom, code, back):
    assert _call(back, geom=geom) == code and lib.dfs_last_error()


@pytest.mark.parametrize("back", [False, True])
@pytest.mark.parametrize("kw,code", [
    (dict(dtype=2), -3), (dict(dtype=-1), -3), (dict(scale=0.0), -1), (dict(scale=float("inf")), -1), (dict(scale=-1.0), -1), (dict(q_start=None), -1), (dict(q_start=AT + 2), -1),
    (dict(k_start=AT + 1), -1), (dict(lse=AT + 2), -1), (dict(q=None), -1), (dict(k=_view(2, at=8)), -1), (dict(v=_view(3, row=4)), -1), (dict(o=None), -1),
    (dict(k=_view(2, head=1 << 44)), -1), (dict(q=_view(1, at=0)), -1), (dict(k=_view(2, row=(1 << 23) + 8)), -2), (dict(v=_view(3, row=(1 << 23) + 8)), -2)])
def test_arguments(kw, code, back):
    assert _call(back, **kw) == code and lib.dfs_last_error()


@pytest.mark.parametrize("kw,code", [
    (dict(lse=None), -1), (dict(ws=None), -4), (dict(ws_bytes=100), -4), (dict(ws=AT + 128), -4), (dict(dq=_view(1)), -1), (dict(dk=_view(8)), -1), (dict(dv=_view(5)), -1),
    (dict(dq=_view(6, row=64)), -1), (dict(dk=_view(7, head=0)), -1), (dict(q=_view(1, row=(1 << 23) + 8)), -2), (dict(d_o=_view(5, row=(1 << 23) + 8)), -2)])
def test_arguments_of_the_backward_pass(kw, code):
    assert _call(True, **kw) == code and lib.dfs_last_error()


@pytest.mark.parametrize("kw,code", [(dict(o=_view(1)), -1), (dict(o=_view(3)), -1), (dict(o=_view(4, row=0)), -1), (dict(ws=None, k_start=AT * 23, geom=dict(seqs=1, n_q=4)), -4)])
def test_arguments_of_the_forward_pass(kw, code):
    assert _call(False, **kw) == code and lib.dfs_last_error()


def test_workspace_sizes():
    code = {"f32": P.DFS_F32, "bf16": P.DFS_BF16}
    for dtype in code.values():
        w = P.Packed(**dict(GOOD, seqs=1))
        assert P.dfs_packed_workspace_bytes(w, dtype, True) >= 8 * 900 * 8 and P.dfs_packed_workspace_bytes(w, dtype, False) % 256 == 0
        assert P.dfs_packed_workspace_bytes(P.Packed(**dict(GOOD, d=96)), dtype, False) == 0
        assert P.dfs_packed_workspace_bytes(P.Packed(**dict(GOOD, n_q=100000, n_k=100000)), dtype, False) == 0                # enough rows: nothing is split
    assert P.dfs_packed_workspace_bytes(P.Packed(**GOOD), 7, False) == 0


def test_no_sequences():
    assert _call(geom=dict(seqs=0, n_q=0, n_k=0), q_start=None, **{n: B._View(None, 0, 0, 0) for n in ("q", "k", "v", "o")}) == 0
