"""Norm and rotation of many rows, against the fp64 oracle: runs of several heads that go from q over k into v, whole work-groups, reads past the memory-side cache, and in
the backward pass work-groups that take several groups of tokens.  Bounds as in test_gpu_rope."""
import numpy as np
import pytest
import torch

pytestmark = pytest.mark.gpu

P = pytest.importorskip("paper_2605_23445_amd")
from oracle import layer_oracle as L  # noqa: E402
from tests.test_gpu_rope import DT, _geom, _inputs, _np  # noqa: E402

# batch, tokens, heads, heads_kv, d, interleaved, dims, positions for each sequence, far (as in test_gpu_rope); how many rows a work-group walks over, of each token
FORWARD = [
    ((1, 1003, 53, 7, 128, True, (44, 42, 42), False, 80), "bf16", 3),       # 64 threads
    ((3, 339, 29, 3, 128, False, (128,), True, 4000), "f32", 3),
    ((1, 8229, 5, 3, 128, True, (44, 42, 42), False, 80), "bf16", 3),        # 256 threads; q q q, q q k, k k v, v v
    ((2, 8230, 4, 1, 64, False, (64,), True, 1 << 20), "f32", 3),
    ((1, 16411, 3, 2, 64, True, (16, 24, 24), False, 100), "bf16", 2),
    ((1, 4133, 3, 3, 128, False, (96,), False, 9000), "f32", 3),
    ((1, 32771, 2, 1, 128, False, (128,), False, 70000), "bf16", 4),         # all of a token's rows
    ((2, 16390, 7, 1, 128, True, (128,), False, 70000), "bf16", 9),
]


def _rows(n, most):
    """Up to `most` of n rows, the first and last among them."""
    return np.unique(np.concatenate([[0, n - 1], np.linspace(0, n - 1, min(n, most)).astype(int)]))


def _per(case, dtype):
    """Rows of all heads' that a work-group of the forward kernel walks over."""
    batch, tokens, heads, kv, d = case[:5]
    waves = (batch * tokens * (d * (2 if dtype == "bf16" else 4) // 16) + 63) // 64
    n = heads + 2 * kv
    return -(-n // min(n, max(-(-8192 // waves), -(-n // 10))))


def _check_forward(case, dtype, most):
    batch, tokens, heads, kv, d, inter, dims, each, far = case
    code, dt, u = DT[dtype]
    fused, parts, pos, w, _ = _inputs(case, dt, 5)
    q, k, v = parts(fused)
    out = [torch.full((batch, n, tokens, d), float("nan"), dtype=dt, device="cuda") for n in (heads, kv, kv)]
    P.dfs_qk_norm_rope(_geom(batch, tokens, heads, kv, d, inter, dims), code, q, k, v, pos if each or batch > 1 else pos[0], *w, *out)
    assert torch.equal(out[2], v) and bool(torch.isfinite(out[0]).all()) and bool(torch.isfinite(out[1]).all())
    at = _rows(tokens, most)
    for x, y, ww in ((q, out[0], w[0]), (k, out[1], w[1])):
        x, y, ww = _np(x[:, :, at]), _np(y[:, :, at]), _np(ww)
        for b in range(batch):
            p = _np(pos[b if each else 0])[at]
            for h in range(x.shape[1]):
                want = L.qk_norm_rope(x[b, h], p, dims, 1e4, inter, ww, 1e-5)
                bound = (d + 16) * 2.0 ** -23 * np.abs(want).max(-1, keepdims=True) * np.sqrt(2) + u * np.abs(want) * (1 + 2.0 ** -8)
                assert (np.abs(y[b, h] - want) <= bound).all(), (b, h)


@pytest.mark.parametrize("case,dtype,per", FORWARD)
def test_forward(case, dtype, per):
    assert _per(case, dtype) == per
    _check_forward(case, dtype, 1500)


@pytest.mark.parametrize("case,dtype", [((1, 32773, 27, 3, 128, True, (44, 42, 42), False, 100), "bf16"), ((2, 16391, 21, 6, 64, False, (64,), True, 50000), "f32"),
                                        ((1, 33001, 60, 3, 64, True, (64,), False, 100), "bf16"), ((1, 16411, 30, 2, 128, False, (128,), False, 100), "f32")])
def test_forward_of_more_than_the_cache_holds(case, dtype):
    batch, tokens, heads, kv, d = case[:5]
    assert batch * tokens * (heads + 2 * kv) * d * (2 if dtype == "bf16" else 4) > 256 << 20
    _check_forward(case, dtype, 200)


@pytest.mark.parametrize("case,dtype", [
    ((1, 20003, 5, 2, 128, True, (44, 42, 42), False, 80), "bf16"),          # 1 251 groups of 16 tokens for 1 024 work-groups, runs of nine
    ((3, 6667, 5, 3, 64, False, (64,), True, 5000), "f32"),                  # runs of six in two
    ((1, 40009, 2, 1, 64, True, (16, 24, 24), False, 100), "bf16"),          # groups of 32
    ((2, 5003, 3, 2, 128, False, (96,), True, 9000), "f32"),                 # groups of 8
    ((1, 9001, 17, 2, 128, False, (128,), False, 9000), "bf16"),             # three runs of seven
])
def test_backward(case, dtype):
    batch, tokens, heads, kv, d, inter, dims, each, far = case
    code, dt, u = DT[dtype]
    fused, parts, pos, w, gen = _inputs(case, dt, 6)
    q, k, _ = parts(fused)
    up = [torch.randn(batch, n, tokens, d, generator=gen, device="cuda").to(dt) for n in (heads, kv, kv)]
    g = _geom(batch, tokens, heads, kv, d, inter, dims)
    slots, n = 256 // (d * (2 if dtype == "bf16" else 4) // 16), heads + 2 * kv
    assert -(-batch * tokens // slots) * -(-n // 10) > 1024                  # work-groups take several groups of tokens
    grad = torch.full_like(fused, float("nan"))
    dw = [torch.full((d,), 7.0, device="cuda") for _ in range(2)]
    ws = torch.full((P.dfs_qk_workspace_bytes(g),), 255, dtype=torch.uint8, device="cuda")
    P.dfs_qk_norm_rope_bwd(g, code, q, k, pos if each or batch > 1 else pos[0], *w, *up, *parts(grad), *dw, ws)
    dq, dk, dv = parts(grad)
    assert torch.equal(dv, up[2]) and bool(torch.isfinite(grad).all())
    for x, y, t, ww, got_w in ((q, dq, up[0], w[0], dw[0]), (k, dk, up[1], w[1], dw[1])):
        ww, dw_want, dw_size, heads_ = _np(ww), np.zeros(d), np.zeros(d), x.shape[1]
        for b in range(batch):
            p = _np(pos[b if each else 0])
            for h in range(heads_):
                xx, yy, tt = _np(x[b, h]), _np(y[b, h]), _np(t[b, h])
                want, s = L.qk_norm_rope_bwd(xx, tt, p, dims, 1e4, inter, ww, 1e-5)
                r = 1 / np.sqrt((xx ** 2).mean(-1, keepdims=True) + 1e-5)
                big = 2 * np.abs(tt).max(-1, keepdims=True) * np.abs(ww).max()
                size = r * big * (1 + r * np.abs(xx) * (r * np.abs(xx)).mean(-1, keepdims=True))
                assert (np.abs(yy - want) <= (2 * d + 32) * 2.0 ** -24 * size + u * np.abs(want) * (1 + 2.0 ** -8)).all(), (b, h)
                dw_want += s
                dw_size += (2 * np.abs(tt).max(-1, keepdims=True) * r * np.abs(xx)).sum(0)
        rows = batch * tokens * heads_
        assert (np.abs(_np(got_w) - dw_want) <= (d + 32 + rows / 16 + 64) * 2.0 ** -24 * dw_size).all()
        # rounding errors of independent signs come to some sqrt(rows) of them: a row left out or counted twice is a hundred times that
        assert (np.abs(_np(got_w) - dw_want) <= 2.0 ** -24 * (64 * np.sqrt(rows) / rows) * dw_size).all()
