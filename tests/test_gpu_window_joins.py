"""One token over long lists of keys: many splits joined, whose largest logits lie anywhere, and lists that the memory-side cache does not hold.

Bounds as in test_gpu_window: u = 2^-8 (bf16) for the rounding of a weight and of the result, a logit off by x = (d + 4) 2^-24 scale sum|q k| at most."""
import numpy as np
import pytest
import torch

pytestmark = pytest.mark.gpu

P = pytest.importorskip("paper_2605_23445_amd")
from oracle import layer_oracle as L  # noqa: E402
from tests.test_gpu_window import DT, E, _np, _within, _ws  # noqa: E402


def _check(w, dtype, q, k, v, lens, scale, heads=None):
    code, _, u = DT[dtype]
    o, lse = torch.full_like(q, 7.0), torch.full((w.batch, w.heads, w.n_q), 7.0, device="cuda")
    k_len = None if lens is None else torch.tensor(lens, dtype=torch.int32, device="cuda")
    P.dfs_window_attn_fwd(w, code, q, k, v, None, k_len, scale, o, lse, _ws(w, dtype, False))
    group = w.heads // w.heads_kv
    for b in range(w.batch):
        m = w.n_k if lens is None else lens[b]
        see = L.window_mask(w.n_q, m, w.left, w.right, w.sinks)
        for h in heads or range(w.heads):
            x, kk, vv = _np(q[b, h]), _np(k[b, h // group, :m]), _np(v[b, h // group, :m])
            want, want_lse, p = L.window_attn(x, kk, vv, see, scale)
            off = (w.d + 4) * E * np.where(see, np.abs(x) @ np.abs(kk).T * scale, 0.0).max(-1, keepdims=True)
            _within(_np(o[b, h]), want, (u + 2 * off + (m + 16) * E) * (p @ np.abs(vv)) + u * np.abs(want) + 1e-30, "o", b, h)
            assert (np.abs(_np(lse[b, h]) - want_lse) <= off[:, 0] + (m + 16) * E + 4 * E * np.abs(want_lse)).all(), ("lse", b, h)


def _splits(w, dtype):
    """Work-groups that share the keys of 32 rows, from the workspace that they leave their sums in."""
    blocks = (w.heads // w.heads_kv * w.n_q + 31) // 32 * w.batch * w.heads_kv
    return P.dfs_window_workspace_bytes(w, DT[dtype][0], False) // (blocks * 32 * (w.d * 4 + 8))


# key heads, splits
@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("d", [64, 128])
@pytest.mark.parametrize("kv,splits", [(14, 9), (12, 10), (8, 16), (7, 18), (5, 25), (4, 32)])
def test_largest_logits_anywhere(kv, splits, d, dtype):
    gen = torch.Generator(device="cuda").manual_seed(splits)
    dt, n_k, group = DT[dtype][1], 4500, 3
    q = torch.randn(1, kv * group, 1, d, generator=gen, device="cuda")
    k, v = (torch.randn(1, kv, n_k, d, generator=gen, device="cuda") for _ in range(2))
    # of each key head, one key that its heads' queries (much alike) are drawn to, further and further behind in the list; the last two head's lists fall and rise
    q = (q + 3 * q[:, ::group].repeat_interleave(group, 1)).to(dt)
    for j in range(kv):
        k[0, j, (2 * j + 1) * n_k // (2 * kv)] = q[0, j * group, 0].float()
    k[0, -2] += q[0, -2 * group].float() * torch.linspace(0.5, -0.5, n_k, device="cuda")[:, None]
    k[0, -1] += q[0, -group].float() * torch.linspace(-0.5, 0.5, n_k, device="cuda")[:, None]
    w = P.Window(1, kv * group, kv, d, 1, n_k, -1, 0, 0)
    assert _splits(w, dtype) == splits
    _check(w, dtype, q, k.to(dt), v.to(dt), None, d ** -0.5)


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("d", [64, 128])
def test_short_lists_beside_long_ones(d, dtype):
    """Splits without keys: whole rounds of them, and all but one."""
    gen = torch.Generator(device="cuda").manual_seed(2)
    dt, lens, n_k = DT[dtype][1], [4500, 150, 1, 700], 4500
    q = torch.randn(4, 4, 1, d, generator=gen, device="cuda").to(dt)
    k, v = (torch.randn(4, 2, n_k, d, generator=gen, device="cuda").to(dt) for _ in range(2))
    for left, sinks in ((-1, 0), (4200, 40)):
        w = P.Window(4, 4, 2, d, 1, n_k, left, 0, sinks)
        assert _splits(w, dtype) == 16
        _check(w, dtype, q, k, v, lens, d ** -0.5)


@pytest.mark.parametrize("dtype,d", [("bf16", 64), ("bf16", 128), ("f32", 64), ("f32", 128)])
def test_more_than_the_cache_holds(dtype, d):
    gen = torch.Generator(device="cuda").manual_seed(3)
    dt, n_k, kv = DT[dtype][1], 4111, 8
    batch = -(-(1 << 28) // (4096 * kv * d * 2 * (2 if dtype == "bf16" else 4)))
    assert batch * kv * 4111 * d * 2 * (2 if dtype == "bf16" else 4) > 256 << 20
    q = torch.randn(batch, 2 * kv, 2, d, generator=gen, device="cuda").to(dt)
    k, v = (torch.randn(batch, kv, n_k, d, generator=gen, device="cuda").to(dt) for _ in range(2))
    lens = [n_k - 113 * (i % 5) for i in range(batch)]
    w = P.Window(batch, 2 * kv, kv, d, 2, n_k, -1, 0, 0)
    _check(w, dtype, q, k, v, lens, d ** -0.5, [0, 2 * kv - 1])
