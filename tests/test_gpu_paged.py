"""Attention over a cache in pages against the fp64 oracle, sequence by sequence with the bounds of windowed attention: a cache's elements times their scales are exact in bf16,
and the arithmetic from there on is the same."""
import numpy as np
import pytest
import torch

pytestmark = pytest.mark.gpu

P = pytest.importorskip("paper_2605_23445_amd")
from oracle import layer_oracle as L  # noqa: E402
from tests import test_gpu_window as W  # noqa: E402

E = W.E
KINDS = {"f32": ("f32", torch.float32), "bf16": ("bf16", torch.bfloat16), "e4m3": ("bf16", torch.float8_e4m3fn)}

# heads, heads_kv, d, page, query rows of each sequence, their keys, left, sinks, rows in front of the first and behind the last sequence
CASES = {
    "one_token": (1, 1, 128, 16, [1], [1], -1, 0, 0, 0),
    "one_token_each": (8, 2, 128, 64, [1, 1, 1, 1, 1, 1], [300, 1, 64, 65, 31, 1000], -1, 0, 0, 0),
    "one_token_each_d64": (16, 4, 64, 16, [1, 1, 1, 0, 1], [300, 17, 16, 70, 1000], -1, 0, 0, 0),
    "one_token_each_small_pages": (12, 2, 128, 16, [1, 1, 2, 1, 1], [300, 16, 65, 900, 31], -1, 0, 1, 1),
    "long_stream": (8, 2, 128, 128, [1], [5000], -1, 0, 0, 0),
    "long_and_short": (4, 1, 128, 32, [1, 1, 1], [4000, 3, 900], -1, 0, 0, 0),
    "window": (8, 2, 128, 64, [1, 1, 1, 1], [700, 40, 129, 64], 100, 0, 0, 0),
    "window_and_first_keys": (8, 2, 64, 16, [1, 1, 1, 1], [700, 40, 129, 64], 100, 4, 0, 0),
    "many_first_keys": (4, 4, 128, 32, [1, 3, 2], [600, 200, 90], 33, 75, 0, 0),
    "first_keys_reach_the_window": (4, 2, 64, 64, [1, 5, 20], [150, 140, 100], 60, 70, 0, 0),
    "itself_only": (2, 2, 64, 16, [1, 4], [50, 90], 0, 0, 0, 0),
    "few_tokens_each": (12, 4, 128, 32, [4, 3, 0, 7], [333, 4, 60, 130], -1, 0, 2, 1),
    "no_keys": (4, 2, 64, 16, [1, 2, 1], [0, 0, 9], -1, 0, 0, 0),
    "more_queries_than_keys": (4, 2, 128, 16, [40, 5], [20, 3], -1, 0, 0, 3),
    "pieces": (6, 2, 128, 64, [70, 1, 33, 200], [700, 390, 33, 200], -1, 0, 5, 0),
    "pieces_d64": (4, 4, 64, 16, [130, 64, 3], [130, 500, 777], -1, 0, 0, 4),
    "pieces_with_window": (8, 2, 64, 32, [150, 90, 31], [150, 400, 300], 70, 10, 0, 0),
    "many_streams": (4, 2, 64, 16, [i % 2 for i in range(300)], [(7 * i) % 90 + 1 for i in range(300)], -1, 0, 1, 0),
    # one long list of keys, so that items come in parts: more sequences than a wave's lanes, and than a work-group's threads
    "many_streams_one_long": (4, 2, 128, 64, [1 + i % 3 % 2 for i in range(90)], [(11 * i) % 200 + 2 for i in range(70)] + [2900] + [65] * 19, -1, 0, 2, 1),
    "more_streams_one_long": (2, 1, 64, 16, [(i + 1) % 4 // 3 + (i == 333) for i in range(700)], [(5 * i) % 50 + (3000 if i == 333 else 0) for i in range(700)], -1, 0, 0, 0),
    "more_streams_with_window": (4, 1, 128, 32, [1] * 650, [(37 * i) % 3300 + 1 for i in range(650)], 2500, 40, 0, 0),
    "long_small_pages": (4, 1, 64, 16, [1, 2, 1], [3000, 1500, 40], -1, 0, 0, 0),
    "wide_group": (24, 1, 128, 64, [3, 9], [100, 300], -1, 0, 0, 0),
    # enough blocks of 128 rows: the kernel of long calls
    "blocks": (32, 32, 128, 64, [500, 129, 1], [500, 700, 300], -1, 0, 0, 0),
    "blocks_group": (32, 8, 128, 128, [300, 130, 257], [300, 1000, 511], -1, 0, 3, 2),
    "blocks_d64": (32, 16, 64, 32, [400, 1, 333], [600, 64, 333], -1, 0, 0, 0),
    "blocks_small_pages": (36, 18, 64, 16, [250, 130, 128], [250, 463, 777], -1, 0, 0, 0),
    "blocks_small_pages_d128": (40, 20, 128, 16, [300, 150], [399, 150], -1, 0, 0, 1),
    "blocks_window": (32, 8, 128, 64, [300, 260, 90], [300, 1200, 600], 130, 0, 0, 0),
    "blocks_window_and_first_keys": (26, 13, 64, 32, [300, 260, 90], [300, 900, 600], 77, 40, 0, 0),
    "blocks_many": (16, 8, 128, 32, [(29 * i) % 70 for i in range(70)], [(29 * i) % 70 + 3 * i for i in range(70)], -1, 0, 0, 0),
    "blocks_long_small_pages": (44, 44, 64, 16, [130, 260], [2600, 1800], -1, 0, 0, 0),
    "blocks_long_small_pages_window": (44, 22, 128, 16, [130, 260], [2600, 1800], 1500, 33, 0, 0),
    "blocks_more": (64, 32, 64, 32, [300, 1, 290], [300, 90, 700], -1, 0, 0, 0),
    "blocks_more_small_pages_window": (80, 40, 64, 16, [330, 200], [330, 650], 150, 10, 0, 0),
    "blocks_more_queries_than_keys": (64, 64, 64, 16, [140, 130], [70, 3], -1, 0, 0, 0),
    # a decoding step of many streams, whose blocks have few rows each
    "blocks_one_token_each": (128, 8, 128, 32, [1 - i % 9 // 8 for i in range(150)], [(37 * i) % 200 + 1 for i in range(150)], -1, 0, 1, 0),
    "blocks_one_token_each_window": (256, 4, 64, 16, [1] * 140, [(53 * i) % 300 + 1 for i in range(140)], 60, 5, 0, 0),
}


def _make(name, kind, seed=0, token_major=False):
    heads, kv, d, page, q_lens, k_lens, left, sinks, front, back = CASES[name]
    dtype, ct = KINDS[kind]
    gen = torch.Generator(device="cuda").manual_seed(seed)
    rand = lambda *s: torch.randn(*s, generator=gen, device="cuda")  # noqa: E731
    n = sum(q_lens) + front + back
    q = rand(n, heads, d).to(W.DT[dtype][1]).transpose(0, 1) if token_major else rand(heads, n, d).to(W.DT[dtype][1])
    need = [(x + page - 1) // page for x in k_lens]
    pages, row = sum(need) + 2, max(need) + 1
    order = np.random.default_rng(seed).permutation(pages)[:sum(need)]
    table, at = np.full((len(k_lens), row), 1 << 30, dtype=np.int32), 0
    for i, m in enumerate(need):
        table[i, :m] = order[at:at + m]
        at += m
    shape = (pages, page, kv, d) if token_major else (pages, kv, page, d)
    cache = [rand(*shape) for _ in range(2)]
    if token_major:
        cache = [x.transpose(1, 2) for x in cache]
    scale = [None, None]
    if kind == "e4m3":
        scale = [torch.exp2(torch.randint(-9, -5, (pages, kv), generator=gen, device="cuda").float()) for _ in range(2)]
        cache = [(x / s[:, :, None, None]).clamp_(-448, 448) for x, s in zip(cache, scale)]
    p = P.Pages(*(x.to(ct) for x in cache), torch.from_numpy(table).cuda(), *scale)
    w = P.Paged(len(q_lens), heads, kv, d, n, left, sinks)
    i32 = lambda x: torch.tensor(x, dtype=torch.int32, device="cuda")  # noqa: E731
    return w, dtype, q, p, i32(front + np.concatenate([[0], np.cumsum(q_lens)])), i32(k_lens), q_lens, k_lens, front, table


def _ws(w, dtype, p):
    return torch.full((P.dfs_paged_workspace_bytes(w, W.DT[dtype][0], p),), 255, dtype=torch.uint8, device="cuda")


def _run(w, dtype, q, p, q_start, k_len, scale, mark=7.0, lse=True):
    o, sums = torch.full(q.shape, mark, dtype=q.dtype, device="cuda"), torch.full((w.heads, w.n_q), mark, device="cuda") if lse else None
    P.dfs_paged_attn_fwd(w, W.DT[dtype][0], q, p, q_start, k_len, scale, o, sums, _ws(w, dtype, p))
    return o, sums


def _rows(p, table, s, m):
    """Keys and values [heads_kv, m, d] of a sequence in fp64."""
    page, got = p.k.shape[2], []
    ids = torch.from_numpy(table[s, :(m + page - 1) // page].astype(np.int64)).cuda()
    for x, scale in ((p.k, p.k_scale), (p.v, p.v_scale)):
        y = torch.stack([x[int(i)].float() for i in ids]).double() if len(ids) else torch.zeros(0, *x.shape[1:], dtype=torch.float64, device="cuda")
        if scale is not None:
            y = y * scale[ids].double()[:, :, None, None]
        got.append(y.permute(1, 0, 2, 3).reshape(x.shape[1], -1, x.shape[3])[:, :m].cpu().numpy())
    return got


def _check(w, dtype, q, p, q_lens, k_lens, front, table, scale, o, lse, mark=7.0):
    u, group, at = W.DT[dtype][2], w.heads // w.heads_kv, front
    n_all = sum(q_lens)
    for x in (o, lse):
        assert (x[:, :front] == mark).all() and (x[:, front + n_all:] == mark).all(), "rows outside the sequences were written"
    q, o, lse = (W._np(x) for x in (q, o, lse))
    for s, (n, m) in enumerate(zip(q_lens, k_lens)):
        k, v = _rows(p, table, s, m)
        see = L.window_mask(n, m, w.left, 0, w.sinks)
        for h in range(w.heads if n else 0):
            kk, vv, x = k[h // group], v[h // group], q[h, at:at + n]
            want, want_lse, pr = L.window_attn(x, kk, vv, see, scale)
            size = np.where(see, np.abs(x) @ np.abs(kk).T * scale, 0.0)
            off = (w.d + 4) * E * (size.max(-1, keepdims=True) if m else np.zeros((n, 1)))
            err = (u + 2 * off + (m + 16) * E) * (pr @ np.abs(vv)) + u * np.abs(want) + 1e-30
            W._within(o[h, at:at + n], want, err, "o", s, h)
            got, full = lse[h, at:at + n], ~np.isneginf(want_lse)
            assert (np.isneginf(got) == ~full).all(), ("lse", s, h)
            with np.errstate(invalid="ignore"):
                assert (np.abs(got - want_lse) <= off[:, 0] + (m + 16) * E + 4 * E * np.abs(want_lse))[full].all(), ("lse", s, h)
        at += n


@pytest.mark.parametrize("kind", list(KINDS))
@pytest.mark.parametrize("name", list(CASES))
def test_against_the_oracle(name, kind):
    w, dtype, q, p, q_start, k_len, q_lens, k_lens, front, table = _make(name, kind)
    scale = 1 / np.sqrt(w.d)
    blocks = name.startswith("blocks") and not (kind == "f32" and w.d == 64 and w.heads * w.n_q < 256 * 128)
    assert (P.dfs_paged_workspace_bytes(w, W.DT[dtype][0], p) == 0) == blocks          # which of the two ways it goes
    o, lse = _run(w, dtype, q, p, q_start, k_len, scale)
    _check(w, dtype, q, p, q_lens, k_lens, front, table, scale, o, lse)
    again, _ = _run(w, dtype, q, p, q_start, k_len, scale, lse=False)
    assert torch.equal(o, again)


@pytest.mark.parametrize("kind", list(KINDS))
@pytest.mark.parametrize("name", ["one_token_each", "window_and_first_keys", "pieces", "blocks_d64", "blocks_small_pages_d128"])
def test_token_major_pages(name, kind):
    w, dtype, q, p, q_start, k_len, q_lens, k_lens, front, table = _make(name, kind, 1, True)
    o, lse = _run(w, dtype, q, p, q_start, k_len, 0.2)
    dense = P.Pages(p.k.float().contiguous().to(p.k.dtype), p.v.float().contiguous().to(p.v.dtype), p.table, p.k_scale, p.v_scale)
    want = _run(w, dtype, q.contiguous(), dense, q_start, k_len, 0.2)
    assert torch.equal(o, want[0]) and torch.equal(lse, want[1])
    _check(w, dtype, q, p, q_lens, k_lens, front, table, 0.2, o, lse)


@pytest.mark.parametrize("kind", list(KINDS))
@pytest.mark.parametrize("name", ["one_token_each", "pieces_d64", "blocks", "blocks_d64", "blocks_small_pages"])
def test_repeated_rows(name, kind):
    """Pages of one row, and of one key head, by strides of zero."""
    w, dtype, q, p, q_start, k_len, q_lens, k_lens, front, table = _make(name, kind, 9)
    scales = [None if x is None else x[:, :1].repeat(1, w.heads_kv) for x in (p.k_scale, p.v_scale)]
    part = [p.k[:, :1, :1].expand_as(p.k), p.v[:, :1].expand_as(p.v)]
    got = _run(w, dtype, q, P.Pages(*part, p.table, *scales), q_start, k_len, 0.1)
    whole = [x.float().contiguous().to(x.dtype) for x in part]
    want = _run(w, dtype, q, P.Pages(*whole, p.table, *scales), q_start, k_len, 0.1)
    assert torch.equal(got[0], want[0]) and torch.equal(got[1], want[1])


@pytest.mark.parametrize("kind", list(KINDS))
@pytest.mark.parametrize("name", ["one_token_each", "window_and_first_keys", "many_first_keys", "first_keys_reach_the_window", "pieces_with_window", "blocks_window",
                                  "blocks_window_and_first_keys", "blocks_small_pages"])
def test_what_nothing_sees_may_hold_anything(name, kind):
    """NaN in keys and values behind the last one and in front of every window, in pages that are nobody's, and in rows outside the sequences."""
    w, dtype, q, p, q_start, k_len, q_lens, k_lens, front, table = _make(name, kind, 2)
    want = _run(w, dtype, q, p, q_start, k_len, 0.1)
    page = p.k.shape[2]
    seen = np.zeros((p.k.shape[0], page), bool)
    for s, (n, m) in enumerate(zip(q_lens, k_lens)):
        for j in np.flatnonzero(L.window_mask(n, m, w.left, 0, w.sinks).any(0)):
            seen[table[s, j // page], j % page] = True
    blind = torch.from_numpy(~seen).cuda()
    bad = []
    for x in (p.k, p.v):
        y = x.float()
        y.transpose(1, 2)[blind] = float("nan")
        bad.append(y.to(x.dtype))
    scales = [None, None]
    if kind == "e4m3":                               # and in the scales of pages of which nothing is seen
        scales = [torch.where(blind.all(1)[:, None], torch.full_like(x, float("nan")), x) for x in (p.k_scale, p.v_scale)]
    got = _run(w, dtype, q, P.Pages(*bad, p.table, *scales), q_start, k_len, 0.1)
    assert torch.equal(got[0], want[0]) and torch.equal(got[1], want[1])


@pytest.mark.parametrize("kind", list(KINDS))
@pytest.mark.parametrize("name", ["one_token_each", "pieces", "blocks", "many_streams"])
def test_starts_lengths_and_tables_that_break_the_format(name, kind):
    """Lengths are cut to the table's room and entries that name no page are page 0; starts that fall touch nothing outside."""
    w, dtype, q, p, q_start, k_len, q_lens, k_lens, front, table = _make(name, kind, 3)
    room = table.shape[1] * p.k.shape[2]
    far = k_len.clone()
    far[0], bad = 1 << 30, np.where((table < 0) | (table >= p.k.shape[0]), 0, table)
    bad[0, 0] = 0
    broken = p.table.clone()
    broken[0, 0] = -5
    got = _run(w, dtype, q, P.Pages(p.k, p.v, broken, p.k_scale, p.v_scale), q_start, far, 0.1)
    far[0] = room
    want = _run(w, dtype, q, P.Pages(p.k, p.v, torch.from_numpy(bad).cuda(), p.k_scale, p.v_scale), q_start, far, 0.1)
    assert torch.equal(got[0], want[0]) and torch.equal(got[1], want[1])
    assert far.shape == k_len.shape
    negative = torch.full_like(k_len, -3)
    o, lse = _run(w, dtype, q, p, q_start, negative, 0.1)
    n = sum(q_lens)
    assert not o[:, front:front + n].any() and torch.isneginf(lse[:, front:front + n]).all()
    for falling in (q_start.flip(0), torch.where(torch.arange(w.seqs + 1, device="cuda") % 2 == 0, q_start, -q_start)):
        around = torch.full((2, w.heads + 2, w.n_q, w.d), 7.0, dtype=q.dtype, device="cuda")
        P.dfs_paged_attn_fwd(w, W.DT[dtype][0], q, p, falling.int(), k_len, 0.1, around[0, 1:-1], None, _ws(w, dtype, p))
        torch.cuda.synchronize()
        assert (around[1] == 7).all() and (around[0, 0] == 7).all() and (around[0, -1] == 7).all()


def test_falling_starts_over_long_lists():
    """Starts that fall so often, over such long lists, that the work of all sequences passes 32 bits and two of them claim the same piece: one of rows 0 .. 1 023, one of 512 .. 1 023.
    Nothing behind the last row is touched."""
    n_q, n_k = 1024, 1 << 28
    start = torch.tensor([0, n_q] * 64 + [512, n_q] * 2, dtype=torch.int32, device="cuda")
    w = P.Paged(len(start) - 1, 1, 1, 64, n_q, -1, 0)
    gen = torch.Generator(device="cuda").manual_seed(13)
    k, v = (torch.randn(1, 1, 128, 64, generator=gen, device="cuda").bfloat16() for _ in range(2))
    p = P.Pages(k, v, torch.zeros(w.seqs, n_k // 128, dtype=torch.int32, device="cuda"))
    q, around = torch.randn(1, n_q, 64, generator=gen, device="cuda").bfloat16(), torch.full((4, n_q, 64), 7.0, dtype=torch.bfloat16, device="cuda")
    sums = torch.full((4 * n_q,), 7.0, device="cuda")
    P.dfs_paged_attn_fwd(w, P.DFS_BF16, q, p, start, torch.full((w.seqs,), n_k, dtype=torch.int32, device="cuda"), 0.1, around[1:2], sums[n_q:2 * n_q].view(1, n_q), _ws(w, "bf16", p))
    torch.cuda.synchronize()
    for x in (around, sums.view(4, n_q)):
        assert (x[0] == 7).all() and (x[2:] == 7).all()


@pytest.mark.parametrize("kind", list(KINDS))
@pytest.mark.parametrize("name", ["one_token_each", "blocks_group"])
def test_sequences_that_share_pages(name, kind):
    """A page that several sequences have, at different places: a common beginning."""
    w, dtype, q, p, q_start, k_len, q_lens, k_lens, front, table = _make(name, kind, 10)
    shared = table.copy()
    shared[1:, 0] = np.where(np.asarray(k_lens)[1:] > 0, table[0, 0], table[1:, 0])
    shared[0, 1] = table[0, 0]
    t = torch.from_numpy(shared).cuda()
    o, lse = _run(w, dtype, q, P.Pages(p.k, p.v, t, p.k_scale, p.v_scale), q_start, k_len, 0.1)
    _check(w, dtype, q, p, q_lens, k_lens, front, shared, 0.1, o, lse)


def test_pages_past_32_bits():
    """Pages more than 2^32 bytes behind the first."""
    w = P.Paged(1, 4, 1, 128, 1, -1, 0)
    pages = (1 << 19) + 900                          # of 8 KB
    gen = torch.Generator(device="cuda").manual_seed(6)
    last = [torch.randn(5, 1, 64, 128, generator=gen, device="cuda").to(torch.float8_e4m3fn) for _ in range(2)]
    k, v = (torch.zeros(pages, 1, 64, 128, dtype=torch.float8_e4m3fn, device="cuda") for _ in range(2))
    for x, y in zip((k, v), last):
        x.view(torch.uint8)[-5:] = y.view(torch.uint8)
    ones, q = torch.ones(pages, 1, device="cuda"), torch.randn(4, 1, 128, generator=gen, device="cuda").bfloat16()
    start, length = (torch.tensor(x, dtype=torch.int32, device="cuda") for x in ([0, 1], [300]))
    table = torch.arange(5, dtype=torch.int32, device="cuda")[None]
    a = _run(w, "bf16", q, P.Pages(k, v, table + (pages - 5), ones, ones), start, length, 0.1)
    b = _run(w, "bf16", q, P.Pages(*last, table, ones[:5], ones[:5]), start, length, 0.1)
    assert torch.equal(a[0], b[0]) and torch.equal(a[1], b[1]) and a[0].any()


@pytest.mark.parametrize("kind", list(KINDS))
def test_a_prompt_and_its_tokens(kind):
    """Appending and attending: a prompt whole, in two pieces, and token by token, against attention over its keys as they were; pages in 8 bits hold what was
    rounded, so there the reference reads them."""
    heads, kv, d, n = 8, 2, 64, 150
    dtype, ct = KINDS[kind]
    code, dt, u = W.DT[dtype]
    gen = torch.Generator(device="cuda").manual_seed(7)
    x = torch.randn(n, heads + 2 * kv, d, generator=gen, device="cuda").to(dt).transpose(0, 1)
    wq, wk = (1 + 0.2 * torch.randn(d, generator=gen, device="cuda") for _ in range(2))
    i32 = lambda y: torch.tensor(y, dtype=torch.int32, device="cuda")  # noqa: E731
    scales = [torch.ones(8, kv, device="cuda") if kind == "e4m3" else None for _ in range(2)]
    outs = []
    for cuts in ([n], [90, 60], [140] + [1] * 10):
        p = P.Pages(*(torch.zeros(8, kv, 32, d, device="cuda").to(ct) for _ in range(2)), i32([[6, 1, 7, 0, 3, 2]]), *(None if s is None else s.clone() for s in scales))
        at, o = 0, torch.empty(heads, n, d, dtype=dt, device="cuda")
        for m in cuts:
            g = P.QkGeom(1, m, heads, kv, d, 0, 1, d, 0, 0, 1e4, 1e-5)
            part, rows = x[:, at:at + m], torch.empty(heads, m, d, dtype=dt, device="cuda")
            start, length = i32([0, m]), i32([at + m])
            P.dfs_paged_append(g, code, part[:heads], part[heads:heads + kv], part[heads + kv:], start, length, None, wq, wk, rows, p)
            w = P.Paged(1, heads, kv, d, m, -1, 0)
            out = torch.empty_like(rows)
            P.dfs_paged_attn_fwd(w, code, rows, p, start, length, 0.125, out, None, _ws(w, dtype, p))
            o[:, at:at + m] = out
            at += m
        outs.append(o.double())
    rope = [torch.empty(1, h, n, d, dtype=dt, device="cuda") for h in (heads, kv, kv)]
    g = P.QkGeom(1, n, heads, kv, d, 0, 1, d, 0, 0, 1e4, 1e-5)
    P.dfs_qk_norm_rope(g, code, x[None, :heads], x[None, heads:heads + kv], x[None, heads + kv:], torch.arange(n, device="cuda", dtype=torch.int32)[:, None], wq, wk, *rope)
    w, o = P.Packed(1, heads, kv, d, n, n, -1, 0), torch.empty(heads, n, d, dtype=dt, device="cuda")
    ws = torch.empty(max(256, P.dfs_packed_workspace_bytes(w, code, False)), dtype=torch.uint8, device="cuda")
    P.dfs_packed_attn_fwd(w, code, rope[0][0], rope[1][0], rope[2][0], i32([0, n]), None, 0.125, o, None, ws)
    # o is a mean of values: off by the weights' and its own rounding, and in 8 bits by what keys (through the logits) and values are rounded by, 2^-4 each
    most = float(rope[2].abs().max())
    logit = float((rope[0][0].float().norm(dim=-1).max() * rope[1][0].float().norm(dim=-1).max()) * 0.125)
    near = {"f32": 1e-5 * most, "bf16": 4 * u * most, "e4m3": (4 * u + 2.0 ** -4 + 2 * 2.0 ** -4 * logit) * most}[kind]
    for y in outs:
        assert (y - o.double()).abs().max() <= near
    if kind != "e4m3":                               # pieces see the same rows: only sums' order differs
        assert all((y - outs[0]).abs().max() <= 4 * max(u, 1e-6) * most for y in outs)


def test_captured_and_replayed():
    """Decoding steps in a graph whose lengths grow, and a graph with another workspace beside it."""
    w, dtype, q, p, q_start, k_len, q_lens, k_lens, front, table = _make("one_token_each", "e4m3", 8)
    other = _make("blocks_group", "bf16", 8)
    want_other = _run(*other[:2], *other[2:6], 0.1)
    k_len[:] = torch.tensor([200, 1, 30, 64, 20, 900], dtype=torch.int32)
    lengths = k_len.clone()
    o, lse, ws = torch.empty_like(q), torch.empty(w.heads, w.n_q, device="cuda"), _ws(w, dtype, p)
    o2, lse2, ws2 = torch.empty_like(other[2]), torch.empty(other[0].heads, other[0].n_q, device="cuda"), _ws(other[0], other[1], other[3])
    graphs = [torch.cuda.CUDAGraph() for _ in range(2)]
    with torch.cuda.graph(graphs[0]):
        P.dfs_paged_attn_fwd(w, P.DFS_BF16, q, p, q_start, k_len, 0.1, o, lse, ws)
        k_len.add_(1)
    with torch.cuda.graph(graphs[1]):
        P.dfs_paged_attn_fwd(other[0], P.DFS_BF16, *other[2:6], 0.1, o2, lse2, ws2)
    n = sum(other[6])
    for _ in range(4):
        graphs[0].replay()
        graphs[1].replay()
        want = _run(w, dtype, q, p, q_start, lengths, 0.1)
        lengths += 1
        torch.cuda.synchronize()
        assert torch.equal(o, want[0]) and torch.equal(lse, want[1])
        a = slice(other[8], other[8] + n)
        assert torch.equal(o2[:, a], want_other[0][:, a]) and torch.equal(lse2[:, a], want_other[1][:, a])


def test_on_another_stream():
    """Appending and attending on a stream of their own, behind work that makes their inputs there."""
    w, dtype, q, p, q_start, k_len, q_lens, k_lens, front, table = _make("few_tokens_each", "e4m3", 11)
    g = P.QkGeom(w.seqs, w.n_q, w.heads, w.heads_kv, w.d, 0, 1, w.d, 0, 0, 1e4, 1e-5)
    k, v = (torch.randn(w.heads_kv, w.n_q, w.d, device="cuda").bfloat16() for _ in range(2))

    def step(p_):
        rows, o = torch.empty_like(q), torch.zeros_like(q)
        P.dfs_paged_append(g, P.DFS_BF16, q * 2, k, v, q_start, k_len, None, None, None, rows, p_)
        P.dfs_paged_attn_fwd(w, P.DFS_BF16, rows, p_, q_start, k_len, 0.1, o, None, _ws(w, dtype, p_))
        return o
    copy = lambda: P.Pages(p.k.clone(), p.v.clone(), p.table, p.k_scale.clone(), p.v_scale.clone())  # noqa: E731
    a, b = copy(), copy()
    want = step(a)
    torch.cuda.synchronize()
    side = torch.cuda.Stream()
    with torch.cuda.stream(side):
        torch.cuda._sleep(1000000)
        got = step(b)
    side.synchronize()
    assert torch.equal(got, want) and torch.equal(a.k.view(torch.uint8), b.k.view(torch.uint8)) and torch.equal(a.k_scale, b.k_scale)


@pytest.mark.parametrize("n_q", [1, 6])
def test_most_keys(n_q):
    """2^28 keys with 1 500 heads a key head, few rows and blocks of them: a row that sees itself alone gives its value."""
    w, n = P.Paged(1, 3000, 2, 64, n_q, 0, 0), 1 << 28
    gen = torch.Generator(device="cuda").manual_seed(12)
    k, v = (torch.randn(1, 2, 128, 64, generator=gen, device="cuda").bfloat16() for _ in range(2))
    p = P.Pages(k, v, torch.zeros(1, n // 128, dtype=torch.int32, device="cuda"))
    assert (P.dfs_paged_workspace_bytes(w, P.DFS_BF16, p) == 0) == (n_q == 6)
    q = torch.randn(3000, n_q, 64, generator=gen, device="cuda").bfloat16()
    start, length = (torch.tensor(x, dtype=torch.int32, device="cuda") for x in ([0, n_q], [n - 20]))
    o, _ = _run(w, "bf16", q, p, start, length, 0.1)
    rows = (n - 20 - n_q + torch.arange(n_q, device="cuda")) % 128
    assert torch.equal(o, v[0][:, rows].repeat_interleave(1500, 0))


def test_no_rows():
    e = torch.empty(2, 0, 64, device="cuda")
    p = P.Pages(torch.empty(0, 2, 16, 64, device="cuda"), torch.empty(0, 2, 16, 64, device="cuda"), torch.zeros(1, 0, dtype=torch.int32, device="cuda"))
    start, length = torch.zeros(2, dtype=torch.int32, device="cuda"), torch.zeros(1, dtype=torch.int32, device="cuda")
    P.dfs_paged_attn_fwd(P.Paged(1, 2, 2, 64, 0, -1, 0), P.DFS_F32, e, p, start, length, 0.1, torch.empty_like(e), None, None)
    start[1] = 3                                     # a cache without pages: nothing is seen
    length[0] = 5
    q, o, lse = torch.randn(2, 3, 64, device="cuda"), torch.full((2, 3, 64), 3.0, device="cuda"), torch.zeros(2, 3, device="cuda")
    w = P.Paged(1, 2, 2, 64, 3, -1, 0)
    P.dfs_paged_attn_fwd(w, P.DFS_F32, q, p, start, length, 0.1, o, lse, _ws(w, "f32", p))
    assert not o.any() and torch.isneginf(lse).all()


def test_refusals_of_the_binding():
    w, dtype, q, p, q_start, k_len, _, _, _, _ = _make("pieces", "e4m3")
    o, lse = torch.zeros_like(q), torch.zeros(w.heads, w.n_q, device="cuda")
    good = [w, P.DFS_BF16, q, p, q_start, k_len, 0.1, o, lse, _ws(w, dtype, p)]
    pg = lambda **kw: P.Pages(**dict(dict(k=p.k, v=p.v, table=p.table, k_scale=p.k_scale, v_scale=p.v_scale), **kw))  # noqa: E731
    for i, bad in ((2, q.float()), (2, q.cpu()), (2, q[1:]), (3, pg(k=p.k[:, 1:])), (3, pg(v=p.v[1:])), (3, pg(table=p.table[1:])), (3, pg(table=p.table.t())), (3, pg(k_scale=p.k_scale[1:])),
                   (4, q_start[:-1]), (4, q_start.long()), (5, k_len[:-1]), (5, k_len.cpu()), (7, o.float()), (8, lse.double()), (8, lse[:1])):
        args = list(good)
        args[i] = bad
        with pytest.raises(ValueError):
            P.dfs_paged_attn_fwd(*args)
    for i, bad in ((3, None), (3, pg(v_scale=None)), (3, pg(k=p.k[:, :, :48], v=p.v[:, :, :48])), (4, None), (5, None), (6, 0.0), (7, q), (9, None), (9, good[9][:-256])):
        args = list(good)
        args[i] = bad
        with pytest.raises(P.DfsError):
            P.dfs_paged_attn_fwd(*args)
    assert not o.any() and not lse.any()


@pytest.mark.parametrize("cuts", [[150], [90, 60], [140] + [1] * 10], ids=["whole", "two_pieces", "token_by_token"])
def test_a_prompt_and_its_tokens_in_8_bits(cuts):
    """Appending and attending, e4m3: each piece against attention in 64 bits over what the pages hold behind its append, whose keys and values are as near to the normed and turned
    ones (bf16, 2^-8) as 8 bits are: 2^-4 of themselves, and where a scale c has grown half a step of the smallest value at each of the scales on the way, 2^-10 (c + c/2 + ...).
    Norm and rotation are not the same bits in both calls: each is off by (d + 16) 2^-23 sqrt(2) of a row's largest channel before it is rounded (tests/test_gpu_paged_append.py)."""
    heads, kv, d, n = 8, 2, 64, 150
    near = (d + 16) * 2.0 ** -23 * np.sqrt(2) * (1 + 2.0 ** -7)
    gen = torch.Generator(device="cuda").manual_seed(7)
    x = torch.randn(n, heads + 2 * kv, d, generator=gen, device="cuda").bfloat16().transpose(0, 1)
    wq, wk = (1 + 0.2 * torch.randn(d, generator=gen, device="cuda") for _ in range(2))
    i32 = lambda y: torch.tensor(y, dtype=torch.int32, device="cuda")  # noqa: E731
    table = np.array([[6, 1, 7, 0, 3, 2]], dtype=np.int32)
    p = P.Pages(*(torch.zeros(8, kv, 32, d, device="cuda").to(torch.float8_e4m3fn) for _ in range(2)), torch.from_numpy(table).cuda(),
                *(torch.ones(8, kv, device="cuda") for _ in range(2)))
    rope = [torch.empty(1, h, n, d, dtype=torch.bfloat16, device="cuda") for h in (heads, kv, kv)]
    g = P.QkGeom(1, n, heads, kv, d, 0, 1, d, 0, 0, 1e4, 1e-5)
    P.dfs_qk_norm_rope(g, P.DFS_BF16, x[None, :heads], x[None, heads:heads + kv], x[None, heads + kv:], torch.arange(n, device="cuda", dtype=torch.int32)[:, None], wq, wk, *rope)
    at = 0
    for m in cuts:
        g = P.QkGeom(1, m, heads, kv, d, 0, 1, d, 0, 0, 1e4, 1e-5)
        part, rows = x[:, at:at + m], torch.empty(heads, m, d, dtype=torch.bfloat16, device="cuda")
        start, length = i32([0, m]), i32([at + m])
        P.dfs_paged_append(g, P.DFS_BF16, part[:heads], part[heads:heads + kv], part[heads + kv:], start, length, None, wq, wk, rows, p)
        want = W._np(rope[0][0, :, at:at + m])
        assert (np.abs(W._np(rows) - want) <= 2 * (near * np.abs(want).max(-1, keepdims=True) + 2.0 ** -8 * (1 + 2.0 ** -7) * np.abs(want))).all()
        w = P.Paged(1, heads, kv, d, m, -1, 0)
        o, lse = _run(w, "bf16", rows, p, start, length, 0.125)
        at += m
        _check(w, "bf16", rows, p, [m], [at], 0, table, 0.125, o, lse)
        with pytest.raises(AssertionError):              # the bounds tell a wrong result
            _check(w, "bf16", rows, p, [m], [at], 0, table, 0.125, torch.zeros_like(o), lse)
    of_row = table[0, np.arange(n) // 32]
    for got, want, scale in zip(_rows(p, table, 0, n), rope[1:], (p.k_scale, p.v_scale)):
        want, c = W._np(want[0]), W._np(scale)[of_row].T[:, :, None]
        off = 2 * near * np.abs(want).max(-1, keepdims=True)
        assert (np.abs(got - want) <= (2.0 ** -4 + 2.0 ** -8 + 2.0 ** -11) * np.abs(want) + (1 + 2.0 ** -4) * off + 2.0 ** -9 * c).all()
