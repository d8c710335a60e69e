"""Norm and rotation of queries and keys, and their gradients, against the fp64 oracle.

Bounds, per row of d channels: the sum of d squares, the root and two products are below (d + 8) 2^-24 relative, sine and cosine below 4 x 2^-24, so
that a turned pair is off by less than (d + 16) 2^-24 (|a| + |b|) <= (d + 16) 2^-23 of the row's largest channel; bf16 rounds by up to 2^-8 of
the value once more.  A gradient sums twice as often, and its size is the upstream gradient's, the weight's and the norm's together."""
import numpy as np
import pytest
import torch

pytestmark = pytest.mark.gpu

P = pytest.importorskip("paper_2605_23445_amd")
from oracle import layer_oracle as L  # noqa: E402

DT = {"f32": (P.DFS_F32, torch.float32, 0.0), "bf16": (P.DFS_BF16, torch.bfloat16, 2.0 ** -8)}


def _geom(batch, tokens, heads, heads_kv, d, inter, dims, eps=1e-5, theta=1e4):
    return P.QkGeom(batch, tokens, heads, heads_kv, d, int(inter), len(dims), *(list(dims) + [0, 0])[:3], theta, eps)


def _rand(gen, *s):
    return torch.randn(*s, generator=gen, device="cuda")


def _np(t):
    return t.double().cpu().numpy()


# batch, tokens, heads, heads_kv, d, interleaved, dims, positions for each sequence, far
CASES = [
    (1, 1, 1, 1, 128, False, (128,), False, 0),
    (3, 1, 8, 2, 128, False, (128,), True, 1 << 20),
    (2, 37, 6, 3, 64, True, (16, 24, 24), False, 500),
    (1, 130, 5, 5, 128, True, (44, 42, 42), False, 80),
    (2, 19, 4, 4, 64, False, (32,), True, 2 ** 31 - 100),
    (1, 65, 3, 1, 128, False, (16, 48), True, 3000),
    (1, 9, 7, 7, 64, True, (2,), False, -1000),
    (1, 300, 41, 2, 64, False, (64,), False, 10),
]


def _inputs(case, dt, seed=0):
    batch, tokens, heads, kv, d, inter, dims, each, far = case
    gen = torch.Generator(device="cuda")
    gen.manual_seed(seed)
    fused = _rand(gen, batch, tokens, (heads + 2 * kv) * d) * torch.exp(0.5 * _rand(gen, (heads + 2 * kv) * d))
    fused = fused.to(dt)
    cut = lambda x, a, n: x[..., a * d:(a + n) * d].view(batch, tokens, n, d).transpose(1, 2)  # noqa: E731
    parts = lambda x: (cut(x, 0, heads), cut(x, heads, kv), cut(x, heads + kv, kv))  # noqa: E731
    lo = min(far, 0)
    pos = torch.randint(lo, max(far, 0) + 1, (batch if each else 1, tokens, len(dims)), generator=gen, device="cuda", dtype=torch.int64).int()
    w = [1 + 0.2 * _rand(gen, d) for _ in range(2)]
    return fused, parts, pos, w, gen


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("case", CASES)
def test_forward(case, dtype):
    batch, tokens, heads, kv, d, inter, dims, each, far = case
    code, dt, u = DT[dtype]
    fused, parts, pos, w, gen = _inputs(case, dt)
    q, k, v = parts(fused)
    g = _geom(batch, tokens, heads, kv, d, inter, dims)
    out = [torch.full((batch, n, tokens, d), 9.0, dtype=dt, device="cuda") for n in (heads, kv, kv)]
    P.dfs_qk_norm_rope(g, code, q, k, v, pos if each or batch > 1 else pos[0], w[0], None, *out)
    assert torch.equal(out[2], v)
    for x, y, ww in ((q, out[0], _np(w[0])), (k, out[1], np.ones(d))):
        x, y = _np(x), _np(y)
        for b in range(batch):
            p = _np(pos[b if each else 0])
            for h in range(x.shape[1]):
                want = L.qk_norm_rope(x[b, h], p, dims, 1e4, inter, ww, 1e-5)
                bound = (d + 16) * 2.0 ** -23 * np.abs(want).max(-1, keepdims=True) * np.sqrt(2) + u * np.abs(want) * (1 + 2.0 ** -8)
                assert (np.abs(y[b, h] - want) <= bound).all()


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("case", CASES)
def test_backward(case, dtype):
    batch, tokens, heads, kv, d, inter, dims, each, far = case
    code, dt, u = DT[dtype]
    fused, parts, pos, w, gen = _inputs(case, dt, 1)
    q, k, _ = parts(fused)
    up = [_rand(gen, batch, n, tokens, d).to(dt) for n in (heads, kv, kv)]
    g = _geom(batch, tokens, heads, kv, d, inter, dims)
    grad = torch.zeros_like(fused)
    dw = [torch.full((d,), 7.0, device="cuda") for _ in range(2)]
    ws = torch.empty(P.dfs_qk_workspace_bytes(g), dtype=torch.uint8, device="cuda")
    call = lambda: P.dfs_qk_norm_rope_bwd(g, code, q, k, pos if each or batch > 1 else pos[0], w[0], w[1], *up, *parts(grad), *dw, ws)  # noqa: E731
    call()
    dq, dk, dv = parts(grad)
    assert torch.equal(dv, up[2])
    for x, y, t, ww, got_w in ((q, dq, up[0], w[0], dw[0]), (k, dk, up[1], w[1], dw[1])):
        x, y, t, ww = _np(x), _np(y), _np(t), _np(ww)
        dw_want, dw_size = np.zeros(d), np.zeros(d)
        for b in range(batch):
            p = _np(pos[b if each else 0])
            for h in range(x.shape[1]):
                want, s = L.qk_norm_rope_bwd(x[b, h], t[b, h], p, dims, 1e4, inter, ww, 1e-5)
                r = 1 / np.sqrt((x[b, h] ** 2).mean(-1, keepdims=True) + 1e-5)
                big = 2 * np.abs(t[b, h]).max(-1, keepdims=True) * np.abs(ww).max()
                size = r * big * (1 + r * np.abs(x[b, h]) * (r * np.abs(x[b, h])).mean(-1, keepdims=True))
                assert (np.abs(y[b, h] - want) <= (2 * d + 32) * 2.0 ** -24 * size + u * np.abs(want) * (1 + 2.0 ** -8)).all()
                dw_want += s
                dw_size += (2 * np.abs(t[b, h]).max(-1, keepdims=True) * r * np.abs(x[b, h])).sum(0)
        # a channel's sum over all rows: in chains of at most tokens x heads / 16 + 64 additions
        rows = batch * tokens * x.shape[1]
        assert (np.abs(_np(got_w) - dw_want) <= (d + 32 + rows / 16 + 64) * 2.0 ** -24 * dw_size).all()
    again, dws = grad.clone(), [x.clone() for x in dw]
    ws.fill_(255)
    call()
    assert torch.equal(grad, again) and all(torch.equal(a, b) for a, b in zip(dw, dws))
    # without the weights' gradients no workspace
    grad.zero_()
    P.dfs_qk_norm_rope_bwd(g, code, q, k, pos if each or batch > 1 else pos[0], w[0], w[1], *up, *parts(grad))
    assert torch.equal(grad, again)


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
def test_in_place_gives_the_same(dtype):
    case = (2, 21, 4, 2, 64, False, (64,), True, 99)
    code, dt, _ = DT[dtype]
    fused, parts, pos, w, gen = _inputs(case, dt, 2)
    g = _geom(2, 21, 4, 2, 64, False, (64,))
    out = torch.zeros_like(fused)
    P.dfs_qk_norm_rope(g, code, *parts(fused), pos, *w, *parts(out))
    mine = fused.clone()
    P.dfs_qk_norm_rope(g, code, *parts(mine), pos, *w, *parts(mine))
    assert torch.equal(mine, out)
    up = torch.randn(fused.shape, generator=gen, device="cuda").to(dt)
    grad = torch.zeros_like(up)
    P.dfs_qk_norm_rope_bwd(g, code, *parts(fused)[:2], pos, *w, *parts(up), *parts(grad))
    P.dfs_qk_norm_rope_bwd(g, code, *parts(fused)[:2], pos, *w, *parts(up), *parts(up))
    assert torch.equal(up, grad)


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
def test_rows_of_a_cache(dtype):
    """Rows outside the cache are dropped, rows that no token goes to stay as they were."""
    batch, tokens, heads, kv, d, rows = 6, 3, 4, 2, 128, 40
    case = (batch, tokens, heads, kv, d, False, (d,), True, 4000)
    code, dt, _ = DT[dtype]
    fused, parts, pos, w, gen = _inputs(case, dt, 3)
    q, k, v = parts(fused)
    g = _geom(batch, tokens, heads, kv, d, False, (d,))
    plain = [torch.empty(batch, n, tokens, d, dtype=dt, device="cuda") for n in (heads, kv, kv)]
    P.dfs_qk_norm_rope(g, code, q, k, v, pos, *w, *plain)
    start = [0, 37, 38, -1, 2 ** 31 - 1, -(2 ** 31)]
    cache = [torch.full((batch, rows, kv, d), 5.0, dtype=dt, device="cuda").transpose(1, 2) for _ in range(2)]
    q_out = torch.empty_like(plain[0])
    P.dfs_qk_norm_rope(g, code, q, k, v, pos, *w, q_out, *cache, torch.tensor(start, dtype=torch.int32, device="cuda"))
    assert torch.equal(q_out, plain[0])
    for x, new in zip(cache, plain[1:]):
        want = torch.full_like(x, 5.0)
        for b, s in enumerate(start):
            for t in range(tokens):
                if 0 <= s + t < rows:
                    want[b, :, s + t] = new[b, :, t]
        assert torch.equal(x, want)


def test_no_tokens():
    g = _geom(2, 0, 3, 1, 64, True, (64,))
    e = lambda n: torch.empty(2, n, 0, 64, device="cuda")  # noqa: E731
    pos = torch.empty(2, 0, 1, dtype=torch.int32, device="cuda")
    P.dfs_qk_norm_rope(g, P.DFS_F32, e(3), e(1), e(1), pos, None, None, e(3), e(1), e(1))
    dw = [torch.full((64,), 3.0, device="cuda") for _ in range(2)]
    ws = torch.empty(P.dfs_qk_workspace_bytes(g), dtype=torch.uint8, device="cuda")
    P.dfs_qk_norm_rope_bwd(g, P.DFS_F32, e(3), e(1), pos, None, None, e(3), e(1), e(1), e(3), e(1), e(1), *dw, ws)
    assert not dw[0].any() and not dw[1].any()


def test_broadcast_upstream_gradient():
    """One upstream gradient for all heads, by a stride of zero."""
    case = (2, 11, 4, 4, 64, True, (64,), False, 9)
    fused, parts, pos, w, gen = _inputs(case, torch.float32, 4)
    q, k, _ = parts(fused)
    g = _geom(2, 11, 4, 4, 64, True, (64,))
    one = torch.randn(2, 1, 11, 64, generator=gen, device="cuda")
    res = []
    for up in (one.expand(2, 4, 11, 64), one.expand(2, 4, 11, 64).contiguous()):
        dq, dk = torch.empty(2, 4, 11, 64, device="cuda"), torch.empty(2, 4, 11, 64, device="cuda")
        P.dfs_qk_norm_rope_bwd(g, P.DFS_F32, q, k, pos, *w, up, up, None, dq, dk, None)
        res.append((dq, dk))
    assert all(torch.equal(a, b) for a, b in zip(*res))


def test_refusals_of_the_binding():
    case = (2, 5, 4, 2, 64, True, (64,), True, 9)
    fused, parts, pos, w, gen = _inputs(case, torch.float32)
    g = _geom(2, 5, 4, 2, 64, True, (64,))
    q, k, v = parts(fused)
    out = [torch.zeros(2, n, 5, 64, device="cuda") for n in (4, 2, 2)]
    good = [g, P.DFS_F32, q, k, v, pos, *w, *out, None]
    for i, bad in ((2, k), (2, q.bfloat16()), (2, q.cpu()), (2, q[:, :, :, ::2]), (3, q), (5, pos[:, :3]), (5, pos.long()), (5, pos.float()), (6, w[0][:9]),
                   (6, w[0].double()), (8, out[1]), (9, out[0]), (11, torch.zeros(2, device="cuda"))):
        args = list(good)
        args[i] = bad
        with pytest.raises(ValueError):
            P.dfs_qk_norm_rope(*args)
    with pytest.raises(P.DfsError):
        P.dfs_qk_norm_rope(g, P.DFS_F32, q, k, None, pos, *w, *out)
    assert not any(x.any() for x in out)
