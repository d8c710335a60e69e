"""<do, o> in the backward pass of windowed attention, bf16: what the rounding of o does to it, and o and log-sum-exp that were joined with other keys'.

Bounds.  u = 2^-8 is what one rounding to bf16 is off by at most, e = 2^-24.  Where a block of 128 rows sees 256 keys at most, <do, o> comes from the keys and dS
has two bf16 terms, so that nothing but the result is rounded to bf16: a logit is off by x = (d + 4) e scale sum|q k|, a weight by 2 max x + (n + 16) e of itself,
<do, v> by (d + 4) e sum|do v|, <do, o> by what these make of it, dS by u^2 of itself besides.  Elsewhere dk has two roundings to bf16, of dS and of the
result; one is off by 2^-7 / sqrt(12) of its value in the mean at most, both by 3.2e-3 of the 2-norm, with 2^-8 as the bound."""
import numpy as np
import pytest
import torch

pytestmark = pytest.mark.gpu

P = pytest.importorskip("paper_2605_23445_amd")
from oracle import layer_oracle as L  # noqa: E402
from tests.test_gpu_window import _np, _run, _within, _ws  # noqa: E402

E, U = 2.0 ** -24, 2.0 ** -8


def _rand(gen, *s):
    return torch.randn(*s, generator=gen, device="cuda")


def _far(got, want):
    return np.linalg.norm(got - want) / np.linalg.norm(want)


# heads, heads_kv, d, n_q, n_k, left, right, sinks, q_len, k_len
FEW = {
    "short_window": (2, 1, 128, 300, 300, 60, 0, 0, None, None),
    "short_window_d64": (3, 3, 64, 300, 300, 30, 20, 5, None, None),
    "few_keys": (4, 2, 128, 150, 150, -1, 0, 0, None, None),
    # work-groups share rows here
    "early_rows": (1, 1, 128, 1500, 1500, -1, 0, 0, None, None),
    "early_rows_d64": (1, 1, 64, 2100, 2100, 1200, 0, 4, None, None),
    "short_sequences": (2, 2, 64, 1100, 1100, -1, 0, 0, [200, 9], [200, 9]),
    "short_sequence_both_sides": (2, 2, 128, 1100, 1100, -1, -1, 0, [256], [256]),
}


@pytest.mark.parametrize("name", list(FEW))
def test_queries_that_see_few_keys(name):
    heads, kv, d, n_q, n_k, left, right, sinks, q_len, k_len = FEW[name]
    batch, group, scale = len(k_len) if k_len else 2, heads // kv, 0.15
    gen = torch.Generator(device="cuda").manual_seed(11)
    q, k, v, d_o = (_rand(gen, batch, h, n, d).bfloat16() for h, n in ((heads, n_q), (kv, n_k), (kv, n_k), (heads, n_q)))
    w = P.Window(batch, heads, kv, d, n_q, n_k, left, right, sinks)
    i32 = lambda x: None if x is None else torch.tensor(x, dtype=torch.int32, device="cuda")  # noqa: E731
    got = _run(w, "bf16", q, k, v, d_o, i32(q_len), i32(k_len), scale)[2]
    q, k, v, d_o, got = (_np(x) for x in (q, k, v, d_o, got))
    checked = 0
    for b in range(batch):
        n, m = (q_len[b], k_len[b]) if k_len else (n_q, n_k)
        see = L.window_mask(n, m, left, right, sinks)
        for h in range(heads):
            for r0 in range(0, n * group, 128):                            # blocks of rows: query by query, all heads of a key head
                i0, i1 = r0 // group, min(n - 1, (r0 + 127) // group)
                rows = np.arange(i0, i1 + 1)
                keys = np.flatnonzero(see[rows].any(0))
                if len(keys) > (225 if sinks else 256):                    # eight pieces of 32, of first keys and of the window
                    continue
                rows = rows[[r0 <= i * group + h % group < r0 + 128 for i in rows]]
                kk, vv, g, x = k[b, h // group][keys], v[b, h // group][keys], d_o[b, h][rows], q[b, h][rows]
                p = L.window_attn(x, kk, vv, see[np.ix_(rows, keys)], scale)[2]
                off = (d + 4) * E * np.where(p > 0, np.abs(x) @ np.abs(kk).T * scale, 0).max(-1, keepdims=True)
                rel = 2 * off + (len(keys) + 16) * E
                dp, e_dp = g @ vv.T, (d + 4) * E * (np.abs(g) @ np.abs(vv).T)
                delta = (p * dp).sum(-1, keepdims=True)
                e_delta = (p * (rel * np.abs(dp) + e_dp)).sum(-1, keepdims=True) + (len(keys) + 16) * E * (p * np.abs(dp)).sum(-1, keepdims=True)
                ds = p * (dp - delta)
                e_ds = p * (rel * np.abs(dp - delta) + e_dp + e_delta) + (U * U + 4 * E) * np.abs(ds)
                want = scale * ds @ kk
                err = scale * (e_ds @ np.abs(kk) + (len(keys) + 16) * E * (np.abs(ds) @ np.abs(kk))) * 1.01 + U * np.abs(want) + 1e-30
                _within(got[b, h][rows], want, err, name, b, h, r0)
                checked += len(rows)
    assert checked >= 100


@pytest.mark.parametrize("name,heads,d,n,left", [("shared_rows", 1, 128, 1500, 900), ("shared_rows_d64", 2, 64, 1300, -1), ("rows_of_one", 48, 64, 800, 600),
                                                 ("rows_of_one_d128", 36, 128, 900, 500)])
def test_keys_gradients_do_not_see_the_rounding_of_o(name, heads, d, n, left):
    """Values that have most in common: o is large and what it is rounded by, in <do, o>, is more than a rounding of dS, which holds the differences alone."""
    gen = torch.Generator(device="cuda").manual_seed(12)
    q, k, d_o = (_rand(gen, 1, heads, n, d).bfloat16() for _ in range(3))
    v = (8 * _rand(gen, 1, heads, 1, d) + _rand(gen, 1, heads, n, d)).bfloat16()
    w = P.Window(1, heads, heads, d, n, n, left, 0, 0)
    got = _run(w, "bf16", q, k, v, d_o, None, None, 0.1)[3]
    see = L.window_mask(n, n, left, 0, 0)
    for h in range(0, heads, 11):
        want = L.window_attn_bwd(*(_np(x[0, h]) for x in (q, k, v)), see, 0.1, _np(d_o[0, h]))[1]
        assert _far(_np(got[0, h]), want) <= U, (name, h)


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("heads,kv,d,n_q,parts", [(2, 2, 64, 200, (300, 40)), (2, 1, 128, 200, (1100, 100)), (40, 40, 64, 300, (700, 300)), (40, 20, 128, 130, (280, 60, 3))])
def test_joined_with_other_keys(heads, kv, d, n_q, parts, dtype):
    """o and log-sum-exp over several sets of keys, one call each, joined: the backward pass of each set takes the joined ones.

    Bound: rounding of the result and of dS, and the rounding of the joined o (of parts that were rounded) in <do, o>, each below 2^-8 in 2-norm and of independent
    signs: 2^-7 for all; fp32 below 1e-5 by the same count."""
    gen = torch.Generator(device="cuda").manual_seed(13)
    code, dt, tol = {"f32": (P.DFS_F32, torch.float32, 1e-5), "bf16": (P.DFS_BF16, torch.bfloat16, 2.0 ** -7)}[dtype]
    q, d_o = (_rand(gen, 1, heads, n_q, d).to(dt) for _ in range(2))
    k, v = (_rand(gen, 1, kv, sum(parts), d).to(dt) for _ in range(2))
    scale, cuts = 1.5 * d ** -0.5, np.cumsum((0,) + parts)
    sets = [(P.Window(1, heads, kv, d, n_q, m, -1, -1, 0), k[:, :, a:a + m], v[:, :, a:a + m]) for a, m in zip(cuts, parts)]
    os, lses = [], []
    for w, kk, vv in sets:
        os.append(torch.empty_like(q))
        lses.append(torch.empty(1, heads, n_q, device="cuda"))
        P.dfs_window_attn_fwd(w, code, q, kk, vv, None, None, scale, os[-1], lses[-1], _ws(w, dtype, False))
    lse = torch.logsumexp(torch.stack(lses).double(), 0)
    o = sum(x.double() * (y - lse).exp()[..., None] for x, y in zip(os, lses)).to(dt)
    lse = lse.float()
    group = heads // kv
    got = []
    for w, kk, vv in sets:
        got.append([torch.empty(x.shape, dtype=dt, device="cuda") for x in (q, kk, vv)])
        P.dfs_window_attn_bwd(w, code, q, kk, vv, o, lse, d_o, None, None, scale, *got[-1], _ws(w, dtype, True))
    see = np.ones((n_q, sum(parts)), bool)
    for h in range(0, heads, 7):
        x, kk, vv, g = (_np(y) for y in (q[0, h], k[0, h // group], v[0, h // group], d_o[0, h]))
        want, _, p = L.window_attn(x, kk, vv, see, scale)
        ds = p * (g @ vv.T - (g * want).sum(-1, keepdims=True))
        for (dq, dk, dv), a, z in zip(got, cuts, cuts[1:]):
            assert _far(_np(dq[0, h]), scale * ds[:, a:z] @ kk[a:z]) <= tol, ("dq", h, a)
            if group == 1:
                assert _far(_np(dk[0, h]), scale * ds[:, a:z].T @ x) <= tol, ("dk", h, a)
                assert _far(_np(dv[0, h]), p[:, a:z].T @ g) <= tol, ("dv", h, a)


@pytest.mark.parametrize("d,parts", [(64, (100, 40)), (128, (200, 40)), (64, (900, 40))])
def test_joined_with_keys_of_little_weight_and_large_values(d, parts):
    """The other keys have a thousandth of a row's weight and values a hundred times as large, so that they make up half of o.  Bound as above."""
    gen = torch.Generator(device="cuda").manual_seed(14)
    n_q, m = 200, parts[0]
    u = torch.nn.functional.normalize(_rand(gen, d), dim=0)
    q, d_o = ((x * _rand(gen, 1, 2, n_q, d) + y * u).bfloat16() for x, y in ((0.5, 4.0), (1.0, 0.0)))
    k, v = (_rand(gen, 1, 2, sum(parts), d) for _ in range(2))
    k = 2 * d ** -0.5 * (k - u * (k @ u)[..., None])                       # logits that the common part of the queries has no share in
    k[:, :, m:] += u * (np.log(1e-3 * m / parts[1]) / 4.0)
    v[:, :, m:] *= 100
    k, v, scale = k.bfloat16(), v.bfloat16(), 1.0
    sets = [(P.Window(1, 2, 2, d, n_q, z - a, -1, -1, 0), k[:, :, a:z], v[:, :, a:z]) for a, z in ((0, m), (m, sum(parts)))]
    os, lses = [], []
    for w, kk, vv in sets:
        os.append(torch.empty_like(q))
        lses.append(torch.empty(1, 2, n_q, device="cuda"))
        P.dfs_window_attn_fwd(w, P.DFS_BF16, q, kk, vv, None, None, scale, os[-1], lses[-1], _ws(w, "bf16", False))
    lse = torch.logsumexp(torch.stack(lses).double(), 0)
    o = sum(x.double() * (y - lse).exp()[..., None] for x, y in zip(os, lses)).bfloat16()
    w, kk, vv = sets[0]
    dq, dk, dv = (torch.empty(x.shape, dtype=torch.bfloat16, device="cuda") for x in (q, kk, vv))
    P.dfs_window_attn_bwd(w, P.DFS_BF16, q, kk, vv, o, lse.float(), d_o, None, None, scale, dq, dk, dv, _ws(w, "bf16", True))
    for h in range(2):
        x, kk, vv, g = (_np(y) for y in (q[0, h], k[0, h], v[0, h], d_o[0, h]))
        want, _, p = L.window_attn(x, kk, vv, np.ones((n_q, sum(parts)), bool), scale)
        rest = p[:, m:].sum(-1)
        assert 2.0 ** -11 < np.median(rest) < 2.0 ** -9
        ds = p * (g @ vv.T - (g * want).sum(-1, keepdims=True))
        assert _far(_np(dq[0, h]), scale * ds[:, :m] @ kk[:m]) <= 2.0 ** -7, ("dq", h)
        assert _far(_np(dk[0, h]), scale * ds[:, :m].T @ x) <= 2.0 ** -7, ("dk", h)
        assert _far(_np(dv[0, h]), p[:, :m].T @ g) <= 2.0 ** -7, ("dv", h)
