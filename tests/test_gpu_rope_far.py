"""Angles of far positions: with a norm of one and a weight that leaves one channel of every pair, a row's pairs are the cosine and sine of its angles.

Bound: the angle is rounded to fp32 in half revolutions, below 1.6 x 2^-24 rad, and a sine and a cosine are within two units of the last place, 2^-23: below 4 x 2^-24 in
all, however far the position."""
import numpy as np
import pytest
import torch

pytestmark = pytest.mark.gpu

P = pytest.importorskip("paper_2605_23445_amd")


@pytest.mark.parametrize("lo,hi", [(0, 100), (1 << 20, 1 << 21), (1 << 30, 2 ** 31 - 1), (-(2 ** 31), -(1 << 30))])
@pytest.mark.parametrize("d,dims,interleaved,theta", [(64, (64,), True, 1e4), (128, (128,), False, 5e5), (128, (44, 42, 42), True, 1e4), (64, (16, 32), False, 1.0),
                                                      (64, (64,), True, 1.05), (64, (64,), False, 1.2), (128, (64, 64), True, 2.0)])
def test_any_position_is_as_good_as_a_small_one(d, dims, interleaved, theta, lo, hi):
    gen = torch.Generator(device="cuda").manual_seed(1)
    n = 700
    pos = torch.randint(lo, hi, (n, len(dims)), generator=gen, device="cuda", dtype=torch.int64).int()
    w, pairs, at = np.zeros(d, np.float32), [], 0
    for axis, m in enumerate(dims):
        for i in range(m // 2):
            a, b = (at + 2 * i, at + 2 * i + 1) if interleaved else (at + i, at + m // 2 + i)
            pairs.append((axis, np.longdouble(theta) ** (np.longdouble(-2 * i) / m), a, b))
            w[a] = 1
        at += m
    w = torch.from_numpy(w).cuda()
    x, out, k_out = torch.ones(1, 1, n, d, device="cuda"), torch.empty(1, 1, n, d, device="cuda"), torch.empty(1, 1, n, d, device="cuda")
    g = P.QkGeom(1, n, 1, 1, d, int(interleaved), len(dims), *(list(dims) + [0, 0])[:3], theta, 0.0)
    P.dfs_qk_norm_rope(g, P.DFS_F32, x, x, None, pos, w, w, out, k_out, None)
    assert torch.equal(out, k_out)
    out, pos = out[0, 0].double().cpu().numpy(), pos.cpu().numpy().astype(np.longdouble)
    worst = 0.0
    for axis, f, a, b in pairs:
        angle = pos[:, axis] * f
        worst = max(worst, float(np.abs(out[:, a] - np.cos(angle)).max()), float(np.abs(out[:, b] - np.sin(angle)).max()))
    assert worst <= 4 * 2.0 ** -24, worst * 2 ** 24
