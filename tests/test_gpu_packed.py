"""Attention within packed sequences and its gradients against the fp64 oracle, sequence by sequence with the bounds of windowed attention, whose arithmetic
this is."""
import numpy as np
import pytest
import torch

pytestmark = pytest.mark.gpu

P = pytest.importorskip("paper_2605_23445_amd")
from tests import test_gpu_window as W  # noqa: E402

DT = W.DT

# heads, heads_kv, d, query rows of each sequence, their keys (None: as many), left, right, rows in front of the first and behind the last sequence
CASES = {
    "one_token": (1, 1, 128, [1], None, -1, 0, 0, 0),
    "one_token_each": (8, 2, 128, [1, 1, 1, 1, 1], [300, 1, 0, 64, 31], -1, 0, 0, 0),
    "causal": (4, 2, 128, [200, 1, 0, 77], None, -1, 0, 0, 0),
    "causal_d64": (6, 3, 64, [33, 0, 0, 257, 1, 128], None, -1, 0, 3, 5),
    "both_ways": (5, 5, 64, [129, 300, 2], None, -1, -1, 0, 1),
    "both_ways_window": (4, 4, 128, [100, 260, 31], None, 65, 33, 7, 0),
    "window": (8, 1, 64, [310, 64, 5, 130], None, 40, 0, 0, 0),
    "itself_only": (2, 2, 64, [70, 1, 3], None, 0, 0, 0, 0),
    "ahead_only": (2, 1, 128, [90, 61], None, 0, -1, 0, 0),
    "later_pieces": (6, 2, 128, [70, 1, 33, 5], [700, 390, 33, 200], -1, 0, 0, 0),
    "more_queries_than_keys": (2, 2, 64, [140, 50, 9], [60, 0, 200], -1, 0, 2, 9),
    "keys_without_queries": (2, 1, 128, [0, 20, 0], [100, 20, 40], -1, 0, 0, 0),
    "queries_without_keys": (2, 1, 128, [40, 3], [0, 0], -1, 0, 0, 0),
    "many_short": (4, 2, 64, [i % 5 for i in range(150)], None, -1, 0, 0, 0),
    "many_short_keys": (3, 1, 64, [i % 3 for i in range(90)], [(7 * i) % 40 for i in range(90)], -1, 0, 1, 1),
    "long_one_head": (1, 1, 64, [900, 1300], None, -1, 0, 0, 0),
    "long_group_of_5": (5, 1, 128, [700, 40], [1100, 1024], 600, 50, 0, 0),
    # enough blocks of 128 rows that keys are not split: the kernels of long calls
    "blocks_causal": (32, 32, 64, [250, 1, 300, 0, 129], None, -1, 0, 0, 0),
    "blocks_group_of_3": (48, 16, 128, [340, 128, 60], None, 70, 0, 0, 3),
    "blocks_both_ways": (22, 22, 128, [500, 33, 128], None, -1, -1, 5, 0),
    "blocks_both_ways_window": (30, 15, 64, [600, 0, 257], None, 64, 127, 0, 0),
    "blocks_later_pieces": (60, 20, 128, [100, 1, 180], [555, 640, 180], 200, 0, 0, 0),
    "blocks_many": (24, 12, 64, [(37 * i) % 90 for i in range(80)], None, -1, 0, 0, 0),
    "blocks_64_sequences": (16, 8, 128, [(29 * i) % 70 for i in range(64)], None, -1, 0, 0, 0),
    "blocks_two_groups_of_waves": (40, 40, 128, [333, 130, 200, 31], None, -1, 0, 0, 0),
    "blocks_shared_by_three": (192, 32, 64, [250, 300], None, -1, 0, 1, 0),
    "blocks_9_key_heads": (18, 9, 128, [260, 700, 130], None, -1, 0, 0, 0),
    "blocks_more_queries_than_keys": (64, 64, 64, [140, 130], [70, 3], -1, 0, 0, 0),
    "blocks_one_token_each": (32, 8, 64, [1 - i % 9 // 8 for i in range(90)], [(37 * i) % 150 for i in range(90)], -1, 0, 0, 1),
}


def _make(name, dtype, seed=0, token_major=False):
    heads, kv, d, q_lens, k_lens, left, right, front, back = CASES[name]
    same = k_lens is None
    k_lens = q_lens if same else k_lens
    n_q, n_k = (sum(x) + front + back for x in (q_lens, k_lens))
    gen = torch.Generator(device="cuda").manual_seed(seed)
    dt = DT[dtype][1]

    def rand(h, n):
        if token_major:
            return torch.randn(n, h, d, generator=gen, device="cuda").to(dt).transpose(0, 1)
        return torch.randn(h, n, d, generator=gen, device="cuda").to(dt)
    starts = lambda x: torch.tensor(front + np.concatenate([[0], np.cumsum(x)]), dtype=torch.int32, device="cuda")  # noqa: E731
    w = P.Packed(len(q_lens), heads, kv, d, n_q, n_k, left, right)
    return w, rand(heads, n_q), rand(kv, n_k), rand(kv, n_k), rand(heads, n_q), starts(q_lens), None if same else starts(k_lens), q_lens, k_lens, front


def _ws(w, dtype, back):
    n = P.dfs_packed_workspace_bytes(w, DT[dtype][0], back)
    return torch.full((n,), 255, dtype=torch.uint8, device="cuda") if n else None


def _run(w, dtype, q, k, v, d_o, q_start, k_start, scale, mark=7.0):
    """o, lse, dq, dk, dv; every element that is not written keeps `mark`."""
    code = DT[dtype][0]
    o, dq, dk, dv = (torch.full(x.shape, mark, dtype=x.dtype, device="cuda") for x in (q, q, k, v))
    lse = torch.full((w.heads, w.n_q), mark, device="cuda")
    P.dfs_packed_attn_fwd(w, code, q, k, v, q_start, k_start, scale, o, lse, _ws(w, dtype, False))
    P.dfs_packed_attn_bwd(w, code, q, k, v, o, lse, d_o, q_start, k_start, scale, dq, dk, dv, _ws(w, dtype, True))
    return o, lse, dq, dk, dv


def _check(w, dtype, q, k, v, d_o, q_lens, k_lens, front, scale, got, mark=7.0):
    o, lse, dq, dk, dv = got
    for x in got:
        n = sum(q_lens) if x is o or x is lse or x is dq else sum(k_lens)
        assert (x[:, :front] == mark).all() and (x[:, front + n:] == mark).all(), "rows outside the sequences were written"
    at_q = at_k = front
    for n, m in zip(q_lens, k_lens):
        one = P.Window(1, w.heads, w.heads_kv, w.d, n, m, w.left, w.right, 0)
        rows, keys = (lambda x: x[None, :, at_q:at_q + n]), (lambda x: x[None, :, at_k:at_k + m])
        W._check(one, dtype, rows(q), keys(k), keys(v), rows(d_o), [n], [m], scale, (rows(o), rows(lse), rows(dq), keys(dk), keys(dv)))
        at_q, at_k = at_q + n, at_k + m


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("name", list(CASES))
def test_against_the_oracle(name, dtype):
    w, q, k, v, d_o, q_start, k_start, q_lens, k_lens, front = _make(name, dtype)
    scale = 1 / np.sqrt(w.d)
    got = _run(w, dtype, q, k, v, d_o, q_start, k_start, scale)
    _check(w, dtype, q, k, v, d_o, q_lens, k_lens, front, scale, got)
    again = _run(w, dtype, q, k, v, d_o, q_start, k_start, scale)
    assert all(torch.equal(a, b) for a, b in zip(got, again))
    o = torch.full(q.shape, 7.0, dtype=q.dtype, device="cuda")
    P.dfs_packed_attn_fwd(w, DT[dtype][0], q, k, v, q_start, k_start, scale, o, None, _ws(w, dtype, False))          # without log-sum-exp
    assert torch.equal(o, got[0])


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("name", ["causal_d64", "both_ways_window", "many_short_keys", "blocks_group_of_3", "long_group_of_5"])
def test_token_major_tensors(name, dtype):
    w, q, k, v, d_o, q_start, k_start, q_lens, k_lens, front = _make(name, dtype, 1, True)
    got = _run(w, dtype, q, k, v, d_o, q_start, k_start, 0.2)
    dense = _run(w, dtype, *(x.contiguous() for x in (q, k, v, d_o)), q_start, k_start, 0.2)
    assert all(torch.equal(a, b) for a, b in zip(got, dense))
    _check(w, dtype, q, k, v, d_o, q_lens, k_lens, front, 0.2, got)


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("name", ["causal_d64", "later_pieces", "blocks_causal", "blocks_later_pieces"])
def test_other_sequences_do_not_reach_in(name, dtype):
    """NaN in one sequence and in the rows around all of them changes nothing in the others."""
    w, q, k, v, d_o, q_start, k_start, q_lens, k_lens, front = _make(name, dtype, 2)
    want = _run(w, dtype, q, k, v, d_o, q_start, k_start, 0.1)
    bad = int(np.argmax(q_lens))
    a_q, a_k = front + sum(q_lens[:bad]), front + sum(k_lens[:bad])
    q, k, v, d_o = (x.clone() for x in (q, k, v, d_o))
    for x, lens, a in ((q, q_lens, a_q), (d_o, q_lens, a_q), (k, k_lens, a_k), (v, k_lens, a_k)):
        x[:, :front] = float("nan")
        x[:, front + sum(lens):] = float("inf")
        x[:, a:a + lens[bad]] = float("nan")
    got = _run(w, dtype, q, k, v, d_o, q_start, k_start, 0.1)
    for a, c, n, m, name_ in zip(want, got, (a_q, a_q, a_q, a_k, a_k), (q_lens, q_lens, q_lens, k_lens, k_lens), ("o", "lse", "dq", "dk", "dv")):
        assert torch.equal(a[:, :n], c[:, :n]) and torch.equal(a[:, n + m[bad]:], c[:, n + m[bad]:]), name_


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("name", ["causal", "blocks_causal", "many_short"])
def test_starts_that_break_the_format(name, dtype):
    """Starts outside the tensors are cut to them; where one falls, rows around are left alone and nothing outside is touched."""
    w, q, k, v, d_o, q_start, _, q_lens, k_lens, front = _make(name, dtype, 3)
    want = _run(w, dtype, q, k, v, d_o, q_start, None, 0.1)
    wide = q_start.clone()
    wide[0], wide[-1] = -5, 1 << 30
    got = _run(w, dtype, q, k, v, d_o, wide, None, 0.1)
    assert all(torch.equal(a, b) for a, b in zip(want, got))
    for falling in (q_start.flip(0), torch.where(torch.arange(w.seqs + 1, device="cuda") % 2 == 0, q_start, -q_start)):
        room = torch.full((2, w.heads + 2, w.n_q, w.d), 7.0, dtype=q.dtype, device="cuda")
        o = room[0, 1:-1]
        P.dfs_packed_attn_fwd(w, DT[dtype][0], q, k, v, falling.int(), None, 0.1, o, None, _ws(w, dtype, False))
        torch.cuda.synchronize()
        assert (room[1] == 7).all() and (room[0, 0] == 7).all() and (room[0, -1] == 7).all()


def _guarded(shape, dtype, mark=7.0):
    """A tensor with as much room of marks in front of it and behind."""
    n = (int(np.prod(shape)) + 4096) // 256 * 256
    room = torch.full((2 * n + int(np.prod(shape)),), mark, dtype=dtype, device="cuda")
    return room[n:-n].view(shape), (room[:n], room[-n:])


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("name", ["causal", "causal_d64", "later_pieces", "many_short", "many_short_keys", "blocks_causal", "blocks_many", "blocks_64_sequences", "blocks_shared_by_three",
                                  "blocks_both_ways_window"])
def test_starts_that_fall_touch_nothing_outside(name, dtype):
    """Both passes, with starts of queries, of keys or of both that fall, up to 64 sequences and more: nothing in front of or behind o, log-sum-exp, gradients and workspaces."""
    w, q, k, v, d_o, q_start, k_start, *_ = _make(name, dtype, 14)
    code, dt = DT[dtype][:2]
    own = q_start if k_start is None else k_start
    odd = torch.arange(w.seqs + 1, device="cuda") % 2 == 1
    falls = lambda x, n: (x.flip(0), torch.where(odd, -x, x), torch.where(odd, torch.zeros_like(x), torch.full_like(x, n + 9)))  # noqa: E731
    cases = [(a, None if k_start is None else own) for a in falls(q_start, w.n_q)] + [(q_start, b) for b in falls(own, w.n_k)] + list(zip(falls(q_start, w.n_q), falls(own, w.n_k)))
    for a, b in cases:
        if b is None and w.n_k != w.n_q:
            continue
        (o, o_room), (dq, dq_room), (dk, dk_room), (dv, dv_room) = (_guarded(x.shape, dt) for x in (q, q, k, v))
        lse, lse_room = _guarded((w.heads, w.n_q), torch.float32)
        rooms = [*o_room, *dq_room, *dk_room, *dv_room, *lse_room]
        ws = [_guarded((P.dfs_packed_workspace_bytes(w, code, back),), torch.uint8, 7) for back in (False, True)]
        P.dfs_packed_attn_fwd(w, code, q, k, v, a.int(), None if b is None else b.int(), 0.1, o, lse, ws[0][0])
        P.dfs_packed_attn_bwd(w, code, q, k, v, o, lse, d_o, a.int(), None if b is None else b.int(), 0.1, dq, dk, dv, ws[1][0])
        torch.cuda.synchronize()
        assert all((x == 7).all() for x in rooms + [*ws[0][1], *ws[1][1]])


def test_same_as_window_attention():
    """Sequences of one length, packed or in a batch."""
    gen = torch.Generator(device="cuda").manual_seed(4)
    q, k, v = (torch.randn(h, 3 * 400, 64, generator=gen, device="cuda").bfloat16() for h in (32, 16, 16))
    start = torch.arange(0, 1201, 400, dtype=torch.int32, device="cuda")
    o, lse = torch.empty_like(q), torch.empty(32, 1200, device="cuda")
    w = P.Packed(3, 32, 16, 64, 1200, 1200, 90, 3)
    P.dfs_packed_attn_fwd(w, P.DFS_BF16, q, k, v, start, None, 0.125, o, lse, _ws(w, "bf16", False))
    cut = lambda x: x.view(x.shape[0], 3, 400, 64).transpose(0, 1)  # noqa: E731
    o2, lse2 = torch.empty_like(cut(q)), torch.empty(3, 32, 400, device="cuda")
    ww = P.Window(3, 32, 16, 64, 400, 400, 90, 3, 0)
    P.dfs_window_attn_fwd(ww, P.DFS_BF16, cut(q), cut(k), cut(v), None, None, 0.125, o2, lse2, W._ws(ww, "bf16", False))
    assert torch.equal(cut(o), o2) and torch.equal(lse.view(32, 3, 400).transpose(0, 1), lse2)


def test_offsets_past_32_bits():
    """A key head whose rows lie more than 2^32 bytes behind the first."""
    n, heads, d = 9000, 2, 128
    gen = torch.Generator(device="cuda").manual_seed(5)
    room = torch.zeros((1 << 31) + 3 * n * d, dtype=torch.bfloat16, device="cuda")
    far = lambda: room.as_strided((heads, n, d), (1 << 31, d, 1))  # noqa: E731
    k = far()
    k.copy_(torch.randn(heads, n, d, generator=gen, device="cuda"))
    q, v = (torch.randn(heads, n, d, generator=gen, device="cuda").bfloat16() for _ in range(2))
    start = torch.tensor([0, 4000, 9000], dtype=torch.int32, device="cuda")
    w = P.Packed(2, heads, heads, d, n, n, 300, 0)
    got = _run(w, "bf16", q, k, v, q, start, None, 0.09)
    want = _run(w, "bf16", q, k.contiguous(), v, q, start, None, 0.09)
    assert all(torch.equal(a, b) for a, b in zip(got, want))


def test_most_keys():
    """2^28 keys, all the same row, with 1 500 heads a key head: a row that sees itself alone gives its value."""
    n, heads, kv, d = 1 << 28, 10500, 7, 64
    w = P.Packed(1, heads, kv, d, 3, n, 0, 0)
    gen = torch.Generator(device="cuda").manual_seed(12)
    q, k, v = (torch.randn(h, m, d, generator=gen, device="cuda").bfloat16() for h, m in ((heads, 3), (kv, 1), (kv, 1)))
    q_start, k_start = (torch.tensor([0, x], dtype=torch.int32, device="cuda") for x in (3, n))
    assert P.dfs_packed_workspace_bytes(w, P.DFS_BF16, False) == 0
    o = torch.zeros_like(q)
    P.dfs_packed_attn_fwd(w, P.DFS_BF16, q, k.expand(kv, n, d), v.expand(kv, n, d), q_start, k_start, 0.1, o)
    assert torch.equal(o, v.expand(kv, 3, d).repeat_interleave(heads // kv, 0))


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
def test_most_sequences(dtype):
    """As many sequences as there may be, two of which have rows: blocks of 32 rows, one for each sequence at least, would pass a grid's 2^32 threads."""
    seqs, n, d, at = (1 << 24) - 2, [24, 40], 64, [5, (1 << 24) - 9]
    w = P.Packed(seqs, 1, 1, d, sum(n), sum(n), -1, 0)
    gen = torch.Generator(device="cuda").manual_seed(13)
    q, k, v, d_o = (torch.randn(1, sum(n), d, generator=gen, device="cuda").to(DT[dtype][1]) for _ in range(4))
    start = torch.zeros(seqs + 1, dtype=torch.int32, device="cuda")
    for a, m in zip(at, n):
        start[a + 1:] += m
    got = _run(w, dtype, q, k, v, d_o, start, None, 0.125)
    _check(w, dtype, q, k, v, d_o, n, n, 0, 0.125, got)


def test_captured_and_replayed():
    """Forward and backward in a graph, replayed with other lengths in the same start array, and a second graph with a workspace of its own."""
    w, q, k, v, d_o, q_start, _, q_lens, k_lens, front = _make("blocks_causal", "bf16", 6)
    small = _make("causal_d64", "f32", 6)
    want = [_run(w, "bf16", q, k, v, d_o, q_start, None, 0.1), _run(small[0], "f32", *small[1:6], None, 0.1)]
    out = [[torch.full_like(x, 7.0) for x in y] for y in want]
    ws = [[_ws(w, "bf16", b) for b in (False, True)], [_ws(small[0], "f32", b) for b in (False, True)]]

    def call(i):
        a, dt, (qq, kk, vv, gg, ss) = ((w, P.DFS_BF16, (q, k, v, d_o, q_start)), (small[0], P.DFS_F32, small[1:6]))[i]
        o, lse, dq, dk, dv = out[i]
        P.dfs_packed_attn_fwd(a, dt, qq, kk, vv, ss, None, 0.1, o, lse, ws[i][0])
        P.dfs_packed_attn_bwd(a, dt, qq, kk, vv, o, lse, gg, ss, None, 0.1, dq, dk, dv, ws[i][1])
    graphs = []
    for i in range(2):
        g = torch.cuda.CUDAGraph()
        with torch.cuda.graph(g):
            call(i)
        graphs.append(g)
    for _ in range(3):
        for i in range(2):
            for x in out[i]:
                x.fill_(7.0)
            graphs[i].replay()
        torch.cuda.synchronize()
        for i in range(2):
            assert all(torch.equal(a, b) for a, b in zip(out[i], want[i]))
    q_start.copy_(torch.tensor([0, 100, 100, 420, 500, 680], dtype=torch.int32))
    graphs[0].replay()
    again = _run(w, "bf16", q, k, v, d_o, q_start, None, 0.1)
    assert all(torch.equal(a, b) for a, b in zip(out[0], again))


@pytest.mark.parametrize("name", ["causal_d64", "later_pieces"])
def test_gradients_against_differences(name):
    """fp32: the change of <o, do> along a direction, by differences.  A difference of step e is off by e^2 of a third derivative and by what o is off by, over e; both stay below
    2e-3 of the sum of sizes at e = 2^-6, as o is good to 1e-6 and a logit moves by less than a tenth."""
    w, q, k, v, d_o, q_start, k_start, q_lens, k_lens, front = _make(name, "f32", 7)
    _, _, dq, dk, dv = _run(w, "f32", q, k, v, d_o, q_start, k_start, 0.1)
    n, m = slice(front, front + sum(q_lens)), slice(front, front + sum(k_lens))
    gen = torch.Generator(device="cuda").manual_seed(8)

    def f(*x):
        o = torch.zeros_like(q)
        P.dfs_packed_attn_fwd(w, P.DFS_F32, *x, q_start, k_start, 0.1, o, None, _ws(w, "f32", False))
        return (o[:, n].double() * d_o[:, n].double()).sum()
    for i, (x, grad, rows) in enumerate(((q, dq, n), (k, dk, m), (v, dv, m))):
        step = torch.randn(x.shape, generator=gen, device="cuda").sign() * 2.0 ** -6
        up, down = ([y + s * step if j == i else y for j, y in enumerate((q, k, v))] for s in (1, -1))
        terms = grad[:, rows].double() * step[:, rows].double()
        assert abs((f(*up) - f(*down)) / 2 - terms.sum()) <= 2e-3 * terms.abs().sum()


def test_no_rows():
    e = lambda h, n: torch.empty(h, n, 64, device="cuda")  # noqa: E731
    start = torch.zeros(3, dtype=torch.int32, device="cuda")
    keys = torch.tensor([0, 2, 5], dtype=torch.int32, device="cuda")
    w = P.Packed(2, 2, 2, 64, 0, 5, -1, 0)
    dk, dv = torch.full((2, 5, 64), 3.0, device="cuda"), torch.full((2, 5, 64), 3.0, device="cuda")
    k, lse = torch.randn(2, 5, 64, device="cuda"), torch.empty(2, 0, device="cuda")
    P.dfs_packed_attn_fwd(w, P.DFS_F32, e(2, 0), k, k, start, keys, 0.1, e(2, 0), lse, _ws(w, "f32", False))
    P.dfs_packed_attn_bwd(w, P.DFS_F32, e(2, 0), k, k, e(2, 0), lse, e(2, 0), start, keys, 0.1, e(2, 0), dk, dv, _ws(w, "f32", True))
    assert not dk.any() and not dv.any()
    w = P.Packed(0, 2, 2, 64, 5, 5, -1, 0)
    o = torch.full((2, 5, 64), 3.0, device="cuda")
    P.dfs_packed_attn_fwd(w, P.DFS_F32, k, k.clone(), k.clone(), start[:1], None, 0.1, o, None, _ws(w, "f32", False))
    assert (o == 3).all()


def test_refusals_of_the_binding():
    w, q, k, v, d_o, q_start, _, _, _, _ = _make("causal", "bf16")
    o, lse = torch.zeros_like(q), torch.zeros(w.heads, w.n_q, device="cuda")
    good = [w, P.DFS_BF16, q, k, v, q_start, None, 0.1, o, lse, _ws(w, "bf16", False)]
    for i, bad in ((2, q.float()), (2, q.cpu()), (2, k), (2, q[None]), (3, q), (4, v[:, 1:]), (4, v[..., ::2]), (5, q_start[:-1]), (5, q_start.long()),
                   (6, q_start.cpu()), (8, o.float()), (9, lse.double()), (9, lse[:1]), (9, lse.t())):
        args = list(good)
        args[i] = bad
        with pytest.raises(ValueError):
            P.dfs_packed_attn_fwd(*args)
    for i, bad in ((5, None), (8, q), (7, 0.0), (7, float("nan"))):
        args = list(good)
        args[i] = bad
        with pytest.raises(P.DfsError):
            P.dfs_packed_attn_fwd(*args)
    assert not o.any() and not lse.any()
