"""Refusals of the calls around the sparse path, on the host: nothing is launched (no GPU is needed), the addresses are never read."""
import ctypes as C

import pytest
import torch

P = pytest.importorskip("paper_2605_23445_amd")
from paper_2605_23445_amd import binding as B  # noqa: E402

lib = B._lib
AT = 1 << 32


def _view(i, batch=1 << 20, head=1 << 14, row=128, at=None):
    return B._View(AT * i if at is None else at, batch, head, row)


QK = dict(batch=2, tokens=5, heads=4, heads_kv=2, d=128, interleaved=1, axes=3, rot0=44, rot1=42, rot2=42, theta=1e4, eps=1e-6)


def _rope(dtype=1, pos=AT * 20, pos_batch=0, w_q=None, start=None, rows=0, back=False, ws=AT * 22, ws_bytes=1 << 30, dw=AT * 21, geom=None, **views):
    g = P.QkGeom(**dict(QK, **(geom or {})))
    v = {n: views.get(n, _view(i + 1)) for i, n in enumerate(("q", "k", "v", "q_out", "k_out", "v_out", "dq", "dk", "dv"))}
    if back:
        return lib.dfs_qk_norm_rope_bwd(g, dtype, v["q"], v["k"], pos, pos_batch, w_q, None, v["q_out"], v["k_out"], v["v_out"], v["dq"], v["dk"], v["dv"],
                                        dw, None, ws, ws_bytes, None)
    return lib.dfs_qk_norm_rope(g, dtype, v["q"], v["k"], v["v"], pos, pos_batch, w_q, None, v["q_out"], v["k_out"], v["v_out"], start, rows, None)


@pytest.mark.parametrize("back", [False, True])
@pytest.mark.parametrize("geom,code", [
    (dict(d=96), -2), (dict(heads=0), -2), (dict(heads_kv=65536), -2), (dict(batch=-1), -2), (dict(tokens=-1), -2), (dict(batch=1 << 16, tokens=1 << 16), -2),
    (dict(axes=0), -2), (dict(axes=4), -2), (dict(rot0=0), -2), (dict(rot0=43), -2), (dict(rot0=46), -2), (dict(interleaved=0), -2), (dict(rot2=-2), -2),
    (dict(theta=0.0), -1), (dict(theta=float("nan")), -1), (dict(theta=float("inf")), -1), (dict(eps=-1e-6), -1), (dict(eps=float("nan")), -1)])
def test_rope_refuses_geometries(geom, code, back):
    assert _rope(geom=geom, back=back) == code and lib.dfs_last_error()


@pytest.mark.parametrize("back", [False, True])
@pytest.mark.parametrize("bad,code", [
    (dict(dtype=2), -3), (dict(pos=None), -1), (dict(pos=AT + 2), -1), (dict(w_q=AT + 1), -1), (dict(pos_batch=-1), -1), (dict(q=None), -1), (dict(k_out=None), -1),
    (dict(q=_view(1, at=None, row=100)), -1), (dict(q=_view(1, at=AT + 8)), -1), (dict(k=_view(2, head=-128)), -1), (dict(q=_view(1, row=1 << 50)), -1),
    (dict(q=_view(0)), -1), (dict(v_out=None), -1)])
def test_rope_refuses_arguments(bad, code, back):
    assert _rope(**bad, back=back) == code and lib.dfs_last_error()


def test_rope_refuses_outputs_that_overlap():
    for bad in (_view(4, row=0), _view(4, row=64), _view(4, head=0), _view(4, batch=128), _view(4, batch=640, head=128, row=256)):
        assert _rope(q_out=bad) == -1 and b"overlap" in lib.dfs_last_error()
    assert _rope(back=True, dq=_view(7, row=64)) == -1
    assert _rope(start=AT * 9, rows=64, k_out=_view(5, batch=1 << 20, head=128 * 63)) == -1        # 64 rows of the cache reach into the next head
    assert _rope(start=AT * 9 + 1, rows=64) == -1 and _rope(start=AT * 9, rows=-1) == -2


def test_rope_backward_needs_its_workspace():
    g = P.QkGeom(**QK)
    need = P.dfs_qk_workspace_bytes(g)
    assert need > 0
    for ws, n in ((None, 1 << 30), (AT * 22 + 16, 1 << 30), (AT * 22, need - 1)):
        assert _rope(back=True, ws=ws, ws_bytes=n) == -4 and b"workspace" in lib.dfs_last_error()
    assert P.dfs_qk_workspace_bytes(P.QkGeom(**dict(QK, d=32))) == 0


WIN = dict(batch=2, heads=4, heads_kv=2, d=128, n_q=5, n_k=9, left=3, right=0, sinks=1)


def _win(dtype=1, scale=0.1, lse=AT * 20, q_len=None, k_len=None, back=False, ws=AT * 21, ws_bytes=1 << 30, win=None, **views):
    w = P.Window(**dict(WIN, **(win or {})))
    v = {n: views.get(n, _view(i + 1)) for i, n in enumerate(("q", "k", "v", "o", "d_o", "dq", "dk", "dv"))}
    if back:
        return lib.dfs_window_attn_bwd(w, dtype, v["q"], v["k"], v["v"], v["o"], lse, v["d_o"], q_len, k_len, scale, v["dq"], v["dk"], v["dv"], ws, ws_bytes, None)
    return lib.dfs_window_attn_fwd(w, dtype, v["q"], v["k"], v["v"], q_len, k_len, scale, v["o"], lse, ws, ws_bytes, None)


@pytest.mark.parametrize("back", [False, True])
@pytest.mark.parametrize("win,code", [
    (dict(d=96), -2), (dict(heads=0), -2), (dict(heads=5), -2), (dict(heads_kv=0), -2), (dict(heads=65536), -2), (dict(batch=-1), -2), (dict(n_q=-1), -2),
    (dict(n_k=(1 << 28) + 1), -2), (dict(sinks=-1), -2), (dict(batch=1 << 20, heads=1 << 12, heads_kv=1 << 12), -2)])
def test_window_refuses_sizes(win, code, back):
    assert _win(win=win, back=back) == code and lib.dfs_last_error()
    assert P.dfs_window_workspace_bytes(P.Window(**dict(WIN, **win)), 1, back) == 0


@pytest.mark.parametrize("back", [False, True])
@pytest.mark.parametrize("bad,code", [
    (dict(dtype=2), -3), (dict(scale=0.0), -1), (dict(scale=float("nan")), -1), (dict(scale=float("inf")), -1), (dict(lse=AT + 2), -1), (dict(q_len=AT + 2), -1),
    (dict(k_len=AT + 1), -1), (dict(q=None), -1), (dict(o=None), -1), (dict(v=_view(3, row=100)), -1), (dict(v=_view(3, at=AT + 8)), -1), (dict(q=_view(0)), -1),
    (dict(k=_view(2, row=1 << 24)), -2)])
def test_window_refuses_arguments(bad, code, back):
    assert _win(**bad, back=back) == code and lib.dfs_last_error()


def test_window_refuses_outputs_that_overlap():
    assert _win(o=_view(4, row=64)) == -1 and b"overlap" in lib.dfs_last_error()
    for name in ("dq", "dk", "dv"):
        assert _win(back=True, **{name: _view(6, row=0)}) == -1 and b"overlap" in lib.dfs_last_error()


def test_window_backward_needs_log_sums_and_workspace():
    assert _win(back=True, lse=None) == -1
    need = P.dfs_window_workspace_bytes(P.Window(**WIN), 1, True)
    assert need > 0
    for ws, n in ((None, 1 << 30), (AT * 21 + 16, 1 << 30), (AT * 21, need - 1)):
        assert _win(back=True, ws=ws, ws_bytes=n) == -4 and b"workspace" in lib.dfs_last_error()


def test_outputs_in_the_place_of_other_tensors_are_refused():
    v = {n: _view(i + 1) for i, n in enumerate(("q", "k", "v", "q_out", "k_out", "v_out", "dq", "dk", "dv"))}
    for out, other in (("q_out", "k"), ("k_out", "q"), ("v_out", "k"), ("q_out", "k_out"), ("k_out", "v_out")):
        assert _rope(**{out: v[other]}) == -1 and b"same memory" in lib.dfs_last_error()
    assert _rope(q_out=_view(1, row=256)) == -1 and b"elsewhere" in lib.dfs_last_error()
    assert _rope(start=AT * 9, rows=64, k_out=v["k"]) == -1 and b"elsewhere" in lib.dfs_last_error()
    for out, other in (("dq", "q"), ("dk", "q"), ("dq", "k_out"), ("dv", "q_out"), ("dk", "dv")):
        assert _rope(back=True, **{out: v[other]}) == -1 and b"same memory" in lib.dfs_last_error()
    assert _rope(back=True, dq=_view(4, row=256)) == -1
    g = P.QkGeom(**QK)
    views = [_view(i + 1) for i in range(8)]
    assert lib.dfs_qk_norm_rope_bwd(g, 1, *views[:2], AT * 20, 0, None, None, *views[2:], AT * 21, AT * 21, AT * 22, 1 << 30, None) == -1
    w = {n: _view(i + 1) for i, n in enumerate(("q", "k", "v", "o", "d_o", "dq", "dk", "dv"))}
    for other in ("q", "k", "v"):
        assert _win(o=w[other]) == -1 and b"same memory" in lib.dfs_last_error()
    for out, other in (("dq", "q"), ("dk", "k"), ("dv", "o"), ("dq", "d_o"), ("dk", "dv"), ("dq", "dk")):
        assert _win(back=True, **{out: w[other]}) == -1 and b"same memory" in lib.dfs_last_error()


def test_null_structs():
    assert lib.dfs_qk_norm_rope(None, 1, *[None] * 3, None, 0, None, None, *[None] * 3, None, 0, None) == -1
    assert lib.dfs_window_attn_fwd(None, 1, *[None] * 3, None, None, 0.1, None, None, None, 0, None) == -1
    assert P.dfs_qk_workspace_bytes(None) == 0 and P.dfs_window_workspace_bytes(None, 1, False) == 0


def test_nothing_to_do_is_no_error():
    empty = B._View(None, 0, 0, 0)
    assert lib.dfs_qk_norm_rope(P.QkGeom(**dict(QK, batch=0)), 1, *[empty] * 3, None, 0, None, None, *[empty] * 3, None, 0, None) == 0
    assert lib.dfs_window_attn_fwd(P.Window(**dict(WIN, batch=0)), 1, *[empty] * 3, None, None, 0.1, empty, None, None, 0, None) == 0


def test_binding_refuses_host_tensors():
    x = torch.zeros(2, 4, 5, 128, dtype=torch.bfloat16)
    with pytest.raises(ValueError):
        P.dfs_window_attn_fwd(P.Window(2, 4, 4, 128, 5, 5, 3, 0, 1), P.DFS_BF16, x, x, x, None, None, 0.1, x.clone())
    assert C.sizeof(P.QkGeom) == 56 and C.sizeof(P.Window) == 36


@pytest.mark.parametrize("back", [False, True])
def test_sizes_that_pass_a_grid_are_refused(back):
    """A grid has fewer than 2^32 threads: 32 a token, 256 a block of 128 rows or keys or of 32 first keys."""
    assert _rope(geom=dict(batch=1 << 7, tokens=1 << 20), back=back) == -2 and _rope(geom=dict(batch=2**31 - 1, tokens=2**31 - 1), back=back) == -2
    for win in (dict(batch=1 << 23, heads=2, heads_kv=2, n_q=1, n_k=1), dict(batch=1 << 8, n_q=1 << 24), dict(batch=1 << 11, n_k=1 << 20, heads=2, heads_kv=1, left=9, sinks=1 << 20),
                dict(batch=2**31 - 1, heads=65535, heads_kv=65535), dict(batch=1, heads=1 << 15, heads_kv=1, n_q=1 << 16)):
        assert _win(win=win, back=back) == -2 and b"too large" in lib.dfs_last_error(), win
