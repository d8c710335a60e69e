"""Refusals of the calls around a cache in pages, on the host: nothing is launched (no GPU is needed), the addresses are never read."""
import ctypes as C

import pytest
import torch

P = pytest.importorskip("paper_2605_23445_amd")
from paper_2605_23445_amd import binding as B  # noqa: E402

lib = B._lib
AT = 1 << 32
QK = dict(batch=3, tokens=50, heads=4, heads_kv=2, d=128, interleaved=0, axes=1, rot0=128, rot1=0, rot2=0, theta=1e4, eps=1e-6)
READ = dict(seqs=3, heads=4, heads_kv=2, d=128, n_q=50, left=-1, sinks=0)


def _view(i, head=1 << 14, row=128, at=None, batch=1 << 20):
    return B._View(AT * i if at is None else at, batch, head, row)


def _pages(**kw):
    c = dict(k=_view(10), v=_view(11), k_scale=AT * 12, v_scale=AT * 13, table=AT * 14, pages=40, page=64, table_row=9, dtype=2)
    return B._PagesC(**dict(c, **kw))


def _append(dtype=1, q_start=AT * 20, k_len=AT * 21, pos=None, w_q=AT * 22, w_k=AT * 23, norm=1, geom=None, pages=None, **views):
    g = None if geom == "none" else P.QkGeom(**dict(QK, **(geom or {})))
    v = {n: views.get(n, _view(i + 1)) for i, n in enumerate(("q", "k", "v", "q_out"))}
    return lib.dfs_paged_append(g, dtype, v["q"], v["k"], v["v"], q_start, k_len, pos, w_q, w_k, v["q_out"], _pages() if pages is None else pages, norm, None)


def _read(dtype=1, q_start=AT * 20, k_len=AT * 21, scale=0.1, lse=AT * 22, ws=AT * 23, ws_bytes=1 << 40, geom=None, pages=None, **views):
    w = None if geom == "none" else P.Paged(**dict(READ, **(geom or {})))
    v = {n: views.get(n, _view(i + 1)) for i, n in enumerate(("q", "o"))}
    return lib.dfs_paged_attn_fwd(w, dtype, v["q"], _pages() if pages is None else pages, q_start, k_len, scale, v["o"], lse, ws, ws_bytes, None)


@pytest.mark.parametrize("call", [_append, _read])
@pytest.mark.parametrize("pages,code", [
    (dict(page=48), -2), (dict(page=8), -2), (dict(page=256), -2), (dict(page=0), -2), (dict(pages=-1), -2), (dict(table_row=-1), -2), (dict(table_row=1 << 23), -2),
    (dict(table=None), -1), (dict(table=AT + 2), -1), (dict(k_scale=None), -1), (dict(v_scale=None), -1), (dict(v_scale=AT + 1), -1), (dict(dtype=0), -3), (dict(dtype=3), -3),
    (dict(dtype=1), -1), (dict(k=_view(10, at=8)), -1), (dict(v=_view(11, row=8)), -1), (dict(k=_view(10, row=(1 << 24) + 16, head=1 << 31, batch=1 << 33)), -2), (dict(v=_view(11, at=0)), -1),
    (dict(k=_view(10, batch=-16)), -1)])
def test_pages(pages, code, call):
    assert call(pages=_pages(**pages)) == code and lib.dfs_last_error()
    if pages.get("dtype") == 3 or "table" in pages:
        none = C.POINTER(B._PagesC)()
        assert call(pages=none) == -1


@pytest.mark.parametrize("geom,code", [
    ("none", -1), (dict(batch=-1), -2), (dict(batch=1 << 24), -2), (dict(tokens=-1), -2), (dict(tokens=1 << 27), -2), (dict(heads=0), -2), (dict(heads_kv=65536), -2), (dict(d=96), -2),
    (dict(axes=4), -2), (dict(rot0=136), -2), (dict(rot0=24), -2), (dict(theta=0.0), -1), (dict(eps=-1.0), -1), (dict(axes=2, rot0=64, rot1=64), -1),
    (dict(batch=1 << 23), -2), (dict(heads=65535, tokens=1 << 20), -2)])
def test_append_geometries(geom, code):
    far = dict(q=_view(1, head=1 << 27), k=_view(2, head=1 << 27), v=_view(3, head=1 << 27), q_out=_view(4, head=1 << 27))
    assert _append(geom=geom, **far) == code and lib.dfs_last_error()


@pytest.mark.parametrize("kw,code", [
    (dict(dtype=2), -3), (dict(dtype=7), -3), (dict(q_start=None), -1), (dict(k_len=None), -1), (dict(q_start=AT + 2), -1), (dict(k_len=AT + 1), -1), (dict(pos=AT + 3), -1),
    (dict(w_q=AT + 2), -1), (dict(norm=0), -1), (dict(norm=0, w_q=None), -1), (dict(q=None), -1), (dict(q_out=None), -1), (dict(v=_view(3, row=4)), -1), (dict(q_out=_view(4, row=64)), -1),
    (dict(q_out=_view(1, row=256)), -1), (dict(q_out=_view(2)), -1), (dict(q_out=_view(3)), -1), (dict(k=_view(10)), -1), (dict(v=_view(11)), -1), (dict(q_out=_view(10)), -1),
    (dict(pages=_pages(v=_view(10))), -1), (dict(pages=_pages(k=_view(10, row=64))), -1), (dict(pages=_pages(k=_view(10, batch=0))), -1),
    (dict(dtype=0, pages=_pages(dtype=2)), -3)])
def test_append_arguments(kw, code):
    assert _append(**kw) == code and lib.dfs_last_error()


def test_scales_that_share_memory():
    """They are written by the append, each by its own values; reading may take one for both."""
    for at in (AT * 12, AT * 12 + 4, AT * 12 + 4 * (40 * 2 - 1), AT * 12 - 4):
        assert _append(pages=_pages(v_scale=at)) == -1 and b"share memory" in lib.dfs_last_error()
        assert _read(pages=_pages(v_scale=at), ws=None) == -4                # refused for the workspace alone


@pytest.mark.parametrize("geom,code", [
    ("none", -1), (dict(seqs=-1), -2), (dict(seqs=1 << 20), -2), (dict(n_q=-1), -2), (dict(n_q=(1 << 28) + 1), -2), (dict(heads=0), -2), (dict(heads=65536), -2), (dict(heads_kv=3), -2),
    (dict(heads_kv=0), -2), (dict(d=80), -2), (dict(sinks=-1), -2), (dict(n_q=1 << 28), -2)])
def test_read_geometries(geom, code):
    assert _read(geom=geom) == code and lib.dfs_last_error()


@pytest.mark.parametrize("kw,code", [
    (dict(dtype=2), -3), (dict(scale=0.0), -1), (dict(scale=float("nan")), -1), (dict(q_start=None), -1), (dict(k_len=None), -1), (dict(q_start=AT + 1), -1), (dict(lse=AT + 2), -1),
    (dict(q=None), -1), (dict(o=_view(2, at=24)), -1), (dict(o=_view(2, row=64)), -1), (dict(o=_view(1)), -1), (dict(o=_view(10)), -1), (dict(ws=None), -4), (dict(ws=AT + 64), -4),
    (dict(ws_bytes=1000), -4)])
def test_read_arguments(kw, code):
    assert _read(**kw) == code and lib.dfs_last_error()


def test_workspace():
    def need(w, dtype, p):
        return lib.dfs_paged_workspace_bytes(w, dtype, p)
    w = P.Paged(**READ)
    n = need(w, 1, _pages())
    assert n > 0 and n % 256 == 0 and need(w, 1, _pages(table_row=1 << 22)) == n
    assert need(w, 1, _pages(page=24)) == 0 and need(P.Paged(**dict(READ, d=32)), 1, _pages()) == 0 and need(w, 0, _pages()) == 0
    assert need(P.Paged(**dict(READ, seqs=0)), 1, _pages()) == 0


def test_nothing_to_do():
    none = B._View(None, 0, 0, 0)
    assert _append(geom=dict(tokens=0), q=none, k=none, v=none, q_out=none) == 0
    assert _append(geom=dict(batch=0)) == 0
    assert _read(geom=dict(n_q=0), q=none, o=none, ws=None) == 0
    assert _read(geom=dict(seqs=0), q_start=None, k_len=None, ws=None) == 0


def test_a_cache_without_pages():
    """What the binding makes of parts that are None, without a GPU: nothing of its own goes wrong."""
    assert B._pages(None, 3, 2, 128) is None and B._pages(P.Pages(None, None, None), 3, 2, 128) is None
    with pytest.raises(ValueError, match="pages.v must be"):
        B._pages(P.Pages(None, torch.zeros(4, 2, 16, 128, dtype=torch.float16), None), 3, 2, 128)
