"""Attention over a window and a few first keys, and its gradients, against the fp64 oracle.

Bounds, from the arithmetic and worked out per element in fp64.  u: what one rounding to the tensors' type is off by at most (bf16 2^-8, f32 0: no
further rounding); e = 2^-24.  A logit, a sum of d products, is off by x = (d + 4) e scale sum|q k| at most, a weight by u + 2 max x + (n + 16) e of
itself, and each sum of n terms by n e of their sizes.  From there the formulas pass their operands' errors on."""
import numpy as np
import pytest
import torch

pytestmark = pytest.mark.gpu

P = pytest.importorskip("paper_2605_23445_amd")
from oracle import layer_oracle as L  # noqa: E402

DT = {"f32": (P.DFS_F32, torch.float32, 0.0), "bf16": (P.DFS_BF16, torch.bfloat16, 2.0 ** -8)}
E = 2.0 ** -24

# heads, heads_kv, d, n_q, n_k, left, right, sinks, q_len, k_len
CASES = {
    "one_token_one_key": (1, 1, 128, 1, 1, 4, 0, 0, None, None),
    "one_token_ragged": (8, 2, 128, 1, 300, 70, 0, 4, None, [300, 71, 1, 0]),
    "one_token_no_window": (4, 4, 64, 1, 200, -1, 0, 0, None, [200, 64]),
    "few_tokens_group_of_3": (6, 2, 64, 5, 333, 100, 0, 7, None, [333, 4, 5, 130]),
    "causal": (4, 2, 128, 200, 200, 64, 0, 3, None, None),
    "causal_d64": (3, 3, 64, 257, 257, 31, 0, 1, None, None),
    "both_sides": (2, 2, 128, 300, 300, 65, 63, 10, None, None),
    "both_sides_d64": (2, 1, 64, 517, 517, 63, 17, 3, None, None),
    "itself_only": (2, 2, 64, 130, 130, 0, 0, 0, None, None),
    "no_limits": (2, 1, 128, 129, 190, -1, -1, 0, None, None),
    "ahead_only": (1, 1, 64, 150, 150, 0, -1, 2, None, None),
    "many_first_keys": (2, 2, 64, 400, 400, 20, 0, 130, None, None),
    "more_first_keys_than_keys": (2, 1, 128, 90, 90, 5, 0, 1000, None, None),
    "first_keys_ahead": (1, 1, 128, 260, 260, 3, 9, 200, None, None),
    "ragged": (4, 2, 64, 310, 310, 50, 0, 4, [310, 1, 0, 155], [310, 1, 0, 155]),
    "more_queries_than_keys": (2, 2, 128, 140, 60, 20, 0, 2, [140, 140, 33], [60, 0, 7]),
    "more_queries_than_keys_ahead": (2, 1, 64, 140, 60, 20, 8, 2, [140, 90], [60, 60]),
    "later_piece": (6, 2, 128, 70, 700, 129, 0, 4, None, [700, 390]),
    "lengths_cut": (1, 1, 64, 40, 40, 9, 0, 1, [1 << 30, -5], [41, 40]),
    "wide_group": (24, 2, 64, 33, 100, 40, 0, 2, None, None),
    # long lists for few work-groups: their parts are added up
    "long_one_head": (1, 1, 64, 1500, 1500, 700, 0, 4, None, None),
    "long_group_of_5": (5, 1, 128, 700, 1100, 600, 50, 40, [700, 333], [1100, 1024]),
    # enough blocks of 128 rows that keys are not split: the kernels of long calls
    "blocks_causal": (64, 64, 64, 250, 250, 100, 0, 4, None, None),
    "blocks_group_of_3": (48, 16, 128, 340, 340, 70, 0, 40, None, None),
    "blocks_both_sides": (22, 22, 128, 700, 700, 97, 33, 5, None, None),
    "blocks_both_sides_d64": (30, 15, 64, 600, 600, 64, 127, 70, None, None),
    "blocks_ragged": (66, 22, 64, 470, 470, 129, 0, 4, [470, 0, 131], [470, 0, 131]),
    "blocks_no_limits": (32, 32, 128, 480, 510, -1, -1, 0, None, None),
    "blocks_later_piece": (60, 20, 128, 300, 900, 200, 0, 33, None, [900, 555]),
    "blocks_more_queries_than_keys": (128, 128, 64, 140, 70, 30, 0, 2, None, [70, 3]),
}


def _np(t):
    return t.double().cpu().numpy()


def _make(name, dtype, seed=0, token_major=False):
    heads, kv, d, n_q, n_k, left, right, sinks, q_len, k_len = CASES[name]
    batch = len(k_len) if k_len else 2
    gen = torch.Generator(device="cuda")
    gen.manual_seed(seed)
    dt = DT[dtype][1]

    def rand(h, n):
        if token_major:
            return torch.randn(batch, n, h, d, generator=gen, device="cuda").to(dt).transpose(1, 2)
        return torch.randn(batch, h, n, d, generator=gen, device="cuda").to(dt)
    q, k, v, d_o = rand(heads, n_q), rand(kv, n_k), rand(kv, n_k), rand(heads, n_q)
    i32 = lambda x: None if x is None else torch.tensor(x, dtype=torch.int32, device="cuda")  # noqa: E731
    cut = lambda x, n: [n] * batch if x is None else [min(max(i, 0), n) for i in x]  # noqa: E731
    w = P.Window(batch, heads, kv, d, n_q, n_k, left, right, sinks)
    return w, q, k, v, d_o, i32(q_len), i32(k_len), cut(q_len, n_q), cut(k_len, n_k)


def _ws(w, dtype, back):
    n = P.dfs_window_workspace_bytes(w, DT[dtype][0], back)
    return torch.full((n,), 255, dtype=torch.uint8, device="cuda") if n else None


def _run(w, dtype, q, k, v, d_o, q_len, k_len, scale, mark=7.0, ws=None):
    """o, lse, dq, dk, dv; every element that is not written keeps `mark`."""
    code = DT[dtype][0]
    o, dq, dk, dv = (torch.full(x.shape, mark, dtype=x.dtype, device="cuda") for x in (q, q, k, v))
    lse = torch.full((w.batch, w.heads, w.n_q), mark, device="cuda")
    P.dfs_window_attn_fwd(w, code, q, k, v, q_len, k_len, scale, o, lse, _ws(w, dtype, False))
    P.dfs_window_attn_bwd(w, code, q, k, v, o, lse, d_o, q_len, k_len, scale, dq, dk, dv, _ws(w, dtype, True))
    return o, lse, dq, dk, dv


def _within(got, want, err, *what):
    off = np.abs(got - want)
    bad = ~(off <= err)
    if bad.any():
        worst = np.unravel_index(np.argmax(np.where(bad, off / err, 0)), off.shape)
        raise AssertionError(f"{what}: {int(bad.sum())} of {bad.size} off, worst at {worst}: {got[worst]} for {want[worst]}, bound {err[worst]}")


def _check(w, dtype, q, k, v, d_o, q_lens, k_lens, scale, got, mark=7.0):
    u, group = DT[dtype][2], w.heads // w.heads_kv
    q, k, v, d_o, o, lse, dq, dk, dv = (_np(x) for x in (q, k, v, d_o, *got))
    for b, (n, m) in enumerate(zip(q_lens, k_lens)):
        see = L.window_mask(n, m, w.left, w.right, w.sinks)
        for j in range(w.heads_kv):
            kk, vv = k[b, j, :m], v[b, j, :m]
            want_k, want_v, err_k, err_v = (np.zeros((m, w.d)) for _ in range(4))
            for h in range(j * group, (j + 1) * group):
                x, g = q[b, h, :n], d_o[b, h, :n]
                want, want_lse, p = L.window_attn(x, kk, vv, see, scale)
                size = np.where(see, np.abs(x) @ np.abs(kk).T * scale, 0.0)
                off = (w.d + 4) * E * (size.max(-1, keepdims=True) if m else np.zeros((n, 1)))
                rel = u + 2 * off + (m + 16) * E
                err = rel * (p @ np.abs(vv)) + u * np.abs(want) + 1e-30
                _within(o[b, h, :n], want, err, "o", b, h)
                full = ~np.isneginf(want_lse)
                assert (np.isneginf(lse[b, h, :n]) == ~full).all(), ("lse", b, h)
                with np.errstate(invalid="ignore"):
                    assert (np.abs(lse[b, h, :n] - want_lse) <= off[:, 0] + (m + 16) * E + 4 * E * np.abs(want_lse))[full].all(), ("lse", b, h)
                # gradients: a weight as above, <do, v> and <do, o> with o as it was rounded
                dp, delta = g @ vv.T, (g * want).sum(-1, keepdims=True)
                e_dp = (w.d + 4) * E * (np.abs(g) @ np.abs(vv).T)
                e_delta = (np.abs(g) * err).sum(-1, keepdims=True) + (w.d + 4) * E * (np.abs(g) * np.abs(want)).sum(-1, keepdims=True)
                ds = p * (dp - delta)
                rel_p = 2 * off + (m + 16) * E                    # before the rounding to u
                e_ds = p * (rel_p * np.abs(dp - delta) + e_dp + e_delta) * (1 + u) + (u + 4 * E) * np.abs(ds)
                want_q = scale * ds @ kk
                err_q = scale * (e_ds @ np.abs(kk) + (m + 16) * E * (np.abs(ds) @ np.abs(kk))) * 1.01 + u * np.abs(want_q) + 1e-30
                _within(dq[b, h, :n], want_q, err_q, "dq", b, h)
                want_k += scale * ds.T @ x
                want_v += p.T @ g
                terms = n * group + 16
                err_k += scale * (e_ds.T @ np.abs(x) + terms * E * (np.abs(ds).T @ np.abs(x))) * 1.01
                err_v += ((u + rel_p + terms * E) * p).T @ np.abs(g) * 1.01
            _within(dk[b, j, :m], want_k, err_k + u * np.abs(want_k) + 1e-30, "dk", b, j)
            _within(dv[b, j, :m], want_v, err_v + u * np.abs(want_v) + 1e-30, "dv", b, j)
        for x, rest in ((o, n), (lse, n), (dq, n), (dk, m), (dv, m)):
            assert (x[b, :, rest:] == mark).all(), ("rows behind the last were written", b)


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("name", list(CASES))
def test_against_the_oracle(name, dtype):
    w, q, k, v, d_o, q_len, k_len, q_lens, k_lens = _make(name, dtype)
    scale = 1 / np.sqrt(w.d)
    got = _run(w, dtype, q, k, v, d_o, q_len, k_len, scale)
    _check(w, dtype, q, k, v, d_o, q_lens, k_lens, scale, got)
    again = _run(w, dtype, q, k, v, d_o, q_len, k_len, scale)
    assert all(torch.equal(a, b) for a, b in zip(got, again))
    o = torch.full(q.shape, 7.0, dtype=q.dtype, device="cuda")
    P.dfs_window_attn_fwd(w, DT[dtype][0], q, k, v, q_len, k_len, scale, o, None, _ws(w, dtype, False))          # without log-sum-exp
    assert torch.equal(o, got[0])


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("name", ["few_tokens_group_of_3", "both_sides", "ragged", "one_token_ragged", "many_first_keys", "blocks_group_of_3", "long_group_of_5"])
def test_token_major_tensors(name, dtype):
    w, q, k, v, d_o, q_len, k_len, q_lens, k_lens = _make(name, dtype, 1, True)
    scale = 0.2
    got = _run(w, dtype, q, k, v, d_o, q_len, k_len, scale)
    dense = _run(w, dtype, *(x.contiguous() for x in (q, k, v, d_o)), q_len, k_len, scale)
    assert all(torch.equal(a, b) for a, b in zip(got, dense))
    _check(w, dtype, q, k, v, d_o, q_lens, k_lens, scale, got)


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("name", ["one_token_ragged", "ragged", "more_queries_than_keys", "later_piece", "few_tokens_group_of_3", "blocks_ragged",
                                  "blocks_later_piece", "long_group_of_5"])
def test_what_nothing_sees_may_hold_anything(name, dtype):
    """Queries behind the last, keys and values behind the last and in front of every window: NaN and infinities there change nothing."""
    w, q, k, v, d_o, q_len, k_len, q_lens, k_lens = _make(name, dtype, 2)
    want = _run(w, dtype, q, k, v, d_o, q_len, k_len, 0.1)
    q, k, v, d_o = (x.clone() for x in (q, k, v, d_o))
    for b, (n, m) in enumerate(zip(q_lens, k_lens)):
        seen = L.window_mask(n, m, w.left, w.right, w.sinks).any(0)
        for i, bad in enumerate((float("nan"), float("inf"))):
            q[b, i::2, n:], d_o[b, i::2, n:] = bad, bad
            for x in (k, v):
                x[b, i::2, m:] = bad
                x[b, i::2, np.flatnonzero(~seen)] = bad
    got = _run(w, dtype, q, k, v, d_o, q_len, k_len, 0.1)
    for a, c, name_ in zip(want, got, ("o", "lse", "dq", "dk", "dv")):
        assert torch.equal(a, c), name_


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
def test_logits_of_infinity(dtype):
    """A key of -inf logits weighs nothing, rows of nothing else are zero; values of the type's lowest at masked places do no harm."""
    w = P.Window(1, 1, 1, 64, 64, 64, 5, 0, 2)
    code, dt, _ = DT[dtype]
    q, k, v = (torch.randn(1, 1, 64, 64, device="cuda", generator=torch.Generator(device="cuda").manual_seed(5)).to(dt) for _ in range(3))
    q = q.abs()
    k[0, 0, 10:20] = -float("inf")
    k[0, 0, 40] = torch.finfo(dt).min                                  # finite: its logits run over to -inf or stay very low
    o, lse = torch.full_like(q, 7.0), torch.full((1, 1, 64), 7.0, device="cuda")
    P.dfs_window_attn_fwd(w, code, q, k, v, None, None, 0.1, o, lse, None)
    kk = k.clone()
    kk[0, 0, 10:20], kk[0, 0, 40] = -1e4, -1e4
    o2, lse2 = torch.full_like(q, 7.0), torch.full((1, 1, 64), 7.0, device="cuda")
    P.dfs_window_attn_fwd(w, code, q, kk, v, None, None, 0.1, o2, lse2, None)
    assert torch.isfinite(o).all() and torch.equal(o, o2) and torch.equal(lse, lse2)


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
def test_long_cache(dtype):
    """Rows of a cache whose offsets pass 2^32 bytes."""
    code, dt, _ = DT[dtype]
    n_k, kv, d = (1 << 22) + 77, 4 if dtype == "bf16" else 2, 128
    cache = torch.zeros(1, n_k, kv, d, dtype=dt, device="cuda").transpose(1, 2)
    gen = torch.Generator(device="cuda").manual_seed(6)
    k, v = (torch.randn(1, kv, 500, d, device="cuda", generator=gen).to(dt) for _ in range(2))
    q = torch.randn(1, 2 * kv, 3, d, device="cuda", generator=gen).to(dt)
    cache[:, :, :10], cache[:, :, -490:] = k[:, :, :10], k[:, :, 10:]
    vals = torch.zeros(1, n_k, kv, d, dtype=dt, device="cuda").transpose(1, 2)
    vals[:, :, :10], vals[:, :, -490:] = v[:, :, :10], v[:, :, 10:]
    o, lse = torch.empty_like(q), torch.empty(1, 2 * kv, 3, device="cuda")
    w = P.Window(1, 2 * kv, kv, d, 3, n_k, 450, 0, 5)
    P.dfs_window_attn_fwd(w, code, q, cache, vals, None, None, 0.09, o, lse, _ws(w, dtype, False))
    o2, lse2 = torch.empty_like(q), torch.empty(1, 2 * kv, 3, device="cuda")
    w = P.Window(1, 2 * kv, kv, d, 3, 500, 450, 0, 5)
    P.dfs_window_attn_fwd(w, code, q, k, v, None, None, 0.09, o2, lse2, _ws(w, dtype, False))
    u = 2.0 ** -8 if dtype == "bf16" else 1e-5
    assert (o.float() - o2.float()).abs().max() <= 2 * u * v.float().abs().max() and (lse - lse2).abs().max() <= 1e-4


def test_repeated_inputs():
    """Key heads that are one and the same, and queries of one row, by strides of zero."""
    gen = torch.Generator(device="cuda").manual_seed(7)
    q = torch.randn(2, 3, 1, 64, device="cuda", generator=gen).bfloat16().expand(2, 3, 70, 64)
    k, v = (torch.randn(2, 1, 70, 64, device="cuda", generator=gen).bfloat16().expand(2, 3, 70, 64) for _ in range(2))
    d_o = torch.randn(1, 1, 1, 64, device="cuda", generator=gen).bfloat16().expand(2, 3, 70, 64)
    w = P.Window(2, 3, 3, 64, 70, 70, 11, 2, 3)
    got = _run(w, "bf16", q, k, v, d_o, None, None, 0.125)
    want = _run(w, "bf16", *(x.contiguous() for x in (q, k, v, d_o)), None, None, 0.125)
    assert all(torch.equal(a, b) for a, b in zip(got, want))
    _check(w, "bf16", q, k, v, d_o, [70] * 2, [70] * 2, 0.125, got)


def test_no_rows():
    e = lambda n: torch.empty(2, 2, n, 64, device="cuda")  # noqa: E731
    w = P.Window(2, 2, 2, 64, 0, 5, 3, 0, 1)
    dk, dv = torch.full((2, 2, 5, 64), 3.0, device="cuda"), torch.full((2, 2, 5, 64), 3.0, device="cuda")
    lse = torch.empty(2, 2, 0, device="cuda")
    P.dfs_window_attn_fwd(w, P.DFS_F32, e(0), dk, dv, None, None, 0.1, e(0), lse)
    P.dfs_window_attn_bwd(w, P.DFS_F32, e(0), torch.randn(2, 2, 5, 64, device="cuda"), torch.randn(2, 2, 5, 64, device="cuda"), e(0), lse, e(0), None, None, 0.1,
                          e(0), dk, dv, _ws(w, "f32", True))
    assert not dk.any() and not dv.any()
    w = P.Window(2, 2, 2, 64, 5, 0, 3, 0, 1)
    q, o, lse = torch.randn(2, 2, 5, 64, device="cuda"), torch.full((2, 2, 5, 64), 3.0, device="cuda"), torch.full((2, 2, 5), 3.0, device="cuda")
    P.dfs_window_attn_fwd(w, P.DFS_F32, q, e(0), e(0), None, None, 0.1, o, lse, _ws(w, "f32", False))
    assert not o.any() and torch.isneginf(lse).all()
    dq = torch.full((2, 2, 5, 64), 3.0, device="cuda")
    P.dfs_window_attn_bwd(w, P.DFS_F32, q, e(0), e(0), o, lse, q, None, None, 0.1, dq, e(0), e(0), _ws(w, "f32", True))
    assert not dq.any()


def test_tensors_without_rows_may_point_anywhere():
    """One of no rows that begins where an output does is not that output."""
    from paper_2605_23445_amd import binding as B
    q, o, lse = torch.randn(2, 2, 5, 64, device="cuda"), torch.full((2, 2, 5, 64), 3.0, device="cuda"), torch.full((2, 2, 5), 3.0, device="cuda")
    w, st = P.Window(2, 2, 2, 64, 5, 0, 3, 0, 1), torch.cuda.current_stream().cuda_stream
    view = lambda t: B._View(t.data_ptr(), *t.stride()[:3])  # noqa: E731
    ws = lambda back: (lambda t: (t.data_ptr() if t is not None else None, t.numel() if t is not None else 0, t))(_ws(w, "f32", back))  # noqa: E731
    at, n, keep = ws(False)
    assert B._lib.dfs_window_attn_fwd(w, P.DFS_F32, view(q), view(o), view(o), None, None, 0.1, view(o), lse.data_ptr(), at, n, st) == 0
    dq = torch.full_like(q, 3.0)
    at, n, keep_too = ws(True)
    assert B._lib.dfs_window_attn_bwd(w, P.DFS_F32, view(q), view(dq), view(dq), view(o), lse.data_ptr(), view(q), None, None, 0.1, view(dq), view(dq), view(dq),
                                      at, n, st) == 0
    assert not o.any() and torch.isneginf(lse).all() and not dq.any()
    del keep, keep_too


def test_refusals_of_the_binding():
    w, q, k, v, d_o, q_len, k_len, _, _ = _make("ragged", "bf16")
    o, lse = torch.zeros_like(q), torch.zeros(w.batch, w.heads, w.n_q, device="cuda")
    good = [w, P.DFS_BF16, q, k, v, q_len, k_len, 0.1, o, lse, None]
    for i, bad in ((2, q.float()), (2, q.cpu()), (2, k), (3, q), (4, v[:, :, 1:]), (4, v[..., ::2]), (5, q_len[:1]), (5, q_len.long()), (6, k_len.cpu()),
                   (8, o.float()), (9, lse.double()), (9, lse[:1]), (9, lse.transpose(1, 2))):
        args = list(good)
        args[i] = bad
        with pytest.raises(ValueError):
            P.dfs_window_attn_fwd(*args)
    assert not o.any() and not lse.any()
