"""New tokens on their way into a cache in pages, against the fp64 oracle.

Bounds: a row of d channels is off by (d + 16) 2^-23 sqrt(2) of its largest channel where it is worked out in fp32 (as for norm and rotation without a cache), and
by half a step of its type more: bf16 2^-8 of the value, e4m3 2^-4 of it or 2^-10 of the scale, whichever is more.  A scale is what the oracle says unless the
largest value is that near to a border; rows from before and everything else of the cache are known bit by bit."""
import numpy as np
import pytest
import torch

pytestmark = pytest.mark.gpu

P = pytest.importorskip("paper_2605_23445_amd")
from oracle import layer_oracle as L  # noqa: E402

KINDS = {"f32": (P.DFS_F32, torch.float32, torch.float32), "bf16": (P.DFS_BF16, torch.bfloat16, torch.bfloat16),
         "e4m3": (P.DFS_BF16, torch.bfloat16, torch.float8_e4m3fn)}

# heads, heads_kv, d, page, interleaved, dims, norm, positions given, (new tokens, tokens before) of each sequence
CASES = {
    "one_token": (1, 1, 128, 16, False, (128,), True, False, [(1, 0)]),
    "tokens_of_streams": (8, 2, 128, 64, False, (128,), True, False, [(1, 5), (1, 63), (1, 64), (1, 0), (1, 127), (1, 1000)]),
    "prompts": (6, 3, 128, 64, False, (128,), True, False, [(200, 0), (1, 0), (64, 0), (63, 0), (65, 0)]),
    "later_pieces": (4, 2, 64, 32, True, (16, 24, 24), True, True, [(70, 33), (0, 5), (31, 1), (32, 32), (1, 31), (90, 7)]),
    "small_pages": (5, 5, 64, 16, True, (64,), False, False, [(33, 15), (16, 0), (17, 16), (3, 14)]),
    "large_pages": (4, 1, 128, 128, False, (64, 32, 32), True, True, [(300, 100), (128, 0), (5, 126), (1, 127)]),
    "large_pages_d64": (4, 2, 64, 128, False, (32,), False, False, [(300, 100), (128, 128), (129, 127)]),
    "pages_of_32": (3, 3, 128, 32, True, (44, 42, 42), True, True, [(50, 10), (100, 0)]),
    "many_streams": (4, 2, 64, 16, False, (64,), True, False, [(i % 3, (5 * i) % 47) for i in range(150)]),
    # few tokens a sequence but for some, whose pages get many rows
    "few_but_two": (4, 2, 128, 64, False, (128,), True, False, [(1, 7 * i) for i in range(60)] + [(100, 30), (0, 3), (64, 0)]),
    "few_but_one": (3, 3, 64, 128, True, (16, 24, 24), True, True, [(i % 4, 97 + i) for i in range(40)] + [(90, 60)]),
    "many_heads": (41, 9, 64, 64, False, (64,), True, False, [(70, 3), (9, 60)]),
}


def _np(t):
    return t.double().cpu().numpy()


def _make(name, kind, seed=0, front=2, back=3):
    heads, kv, d, page, inter, dims, norm, given, lens = CASES[name]
    code, dt, ct = KINDS[kind]
    gen = torch.Generator(device="cuda").manual_seed(seed)
    rand = lambda *s: torch.randn(*s, generator=gen, device="cuda")  # noqa: E731
    n = sum(x for x, _ in lens) + front + back
    fused = (rand(n, heads + 2 * kv, d) * torch.exp(0.5 * rand(heads + 2 * kv, d))).to(dt).transpose(0, 1)
    q, k, v = fused[:heads], fused[heads:heads + kv], fused[heads + kv:]
    pos = torch.randint(0, 400, (n, len(dims)), generator=gen, device="cuda").int() if given else None
    w = [1 + 0.2 * rand(d) if norm else None for _ in range(2)]
    g = P.QkGeom(len(lens), n, heads, kv, d, int(inter), len(dims), *(list(dims) + [0, 0])[:3], 1e4, 1e-5)
    q_start = torch.tensor(front + np.concatenate([[0], np.cumsum([x for x, _ in lens])]), dtype=torch.int32, device="cuda")
    k_len = torch.tensor([x + y for x, y in lens], dtype=torch.int32, device="cuda")
    need = [(x + y + page - 1) // page for x, y in lens]
    row, pages = max(need) + 1, sum(need) + 2
    order = np.random.default_rng(seed).permutation(pages)[:sum(need)]
    table = np.full((len(lens), row), 1 << 30, dtype=np.int32)            # entries that no token is on name no page
    table[:, -1] = -3
    at = 0
    for i, m in enumerate(need):
        table[i, :m] = order[at:at + m]
        at += m
    shape = (pages, kv, page, d)
    if kind == "e4m3":
        cache = [rand(*shape).mul_(60).clamp_(-448, 448).to(ct) for _ in range(2)]
        scale = [torch.exp2(torch.randint(-9, -3, shape[:2], generator=gen, device="cuda").float()) for _ in range(2)]
    else:
        cache, scale = [rand(*shape).to(ct) for _ in range(2)], [None, None]
    p = P.Pages(*cache, torch.from_numpy(table).cuda(), *scale)
    return g, code, q, k, v, q_start, k_len, pos, w, p, norm, lens, front, table


def _copy(p):
    c = lambda t: None if t is None else t.clone()  # noqa: E731
    return P.Pages(c(p.k), c(p.v), p.table, c(p.k_scale), c(p.v_scale))


def _bits(t):
    return t.view(torch.uint8)


def _same(a, b):
    return all(x is None and y is None or torch.equal(_bits(x), _bits(y)) for x, y in ((a.k, b.k), (a.v, b.v), (a.k_scale, b.k_scale), (a.v_scale, b.v_scale)))


def _check(kind, g, q, k, v, pos, w, before, after, q_out, norm, lens, front, table, mark=9.0):
    page, d = before.k.shape[2], g.d
    dims = [x for x in (g.rot0, g.rot1, g.rot2) if x]
    near = (d + 16) * 2.0 ** -23 * np.sqrt(2)
    u = {"f32": 0.0, "bf16": 2.0 ** -8, "e4m3": 2.0 ** -8}[kind]
    q, k, v, got_q = (_np(x) for x in (q, k, v, q_out))
    n = sum(x for x, _ in lens)
    assert (got_q[:, :front] == mark).all() and (got_q[:, front + n:] == mark).all()
    used = [torch.zeros(before.k.shape[:3], dtype=torch.bool, device="cuda") for _ in range(2)]
    at = front
    for s, (new, old) in enumerate(lens):
        p = np.arange(old, old + new)[:, None] if pos is None else _np(pos[at:at + new])

        def worked(x, ww):
            if not norm:                             # the oracle's norm of weight 1, and the rows' size again
                return L.qk_norm_rope(x, p, dims, 1e4, bool(g.interleaved), np.ones(d), 0.0) * np.sqrt((x * x).mean(-1, keepdims=True))
            return L.qk_norm_rope(x, p, dims, 1e4, bool(g.interleaved), np.ones(d) if ww is None else _np(ww), 1e-5)
        for h in range(g.heads):
            want = worked(q[h, at:at + new], w[0])
            bound = near * np.abs(want).max(-1, keepdims=True, initial=0) + u * np.abs(want) * (1 + 2.0 ** -8)
            assert (np.abs(got_q[h, at:at + new] - want) <= bound).all(), ("q", s, h)
        for x, (src, ww) in enumerate(((k, w[1]), (v, None))):
            cache, was = (after.k, before.k) if x == 0 else (after.v, before.v)
            scale, was_scale = (after.k_scale, before.k_scale) if x == 0 else (after.v_scale, before.v_scale)
            for h in range(g.heads_kv):
                rows = src[h, at:at + new]
                want = rows if x else worked(rows, ww)
                off = np.zeros((new, 1)) if x else near * np.abs(want).max(-1, keepdims=True, initial=0)
                for i in range(old // page, (old + new - 1) // page + 1 if new else 0):
                    a, z, to = max(old, i * page), min(old + new, (i + 1) * page), int(table[s, i])
                    r0, part, e = a - i * page, want[a - old:z - old], off[a - old:z - old]
                    got = _np(cache[to, h, r0:r0 + z - a].float())
                    used[x][to, h, :r0 + z - a] = True
                    if kind != "e4m3":
                        if x:
                            assert (got == part).all()
                        assert (np.abs(got - part) <= e + u * np.abs(part) * (1 + 2.0 ** -8)).all(), ("cache", x, s, h, i)
                        used[x][to, h, :r0] = False                          # rows from before are as they were
                        continue
                    c = float(scale[to, h])
                    most, slack = np.abs(part).max(), 1 + 2 * near
                    least = 2.0 ** -120 if most == 0 else max(2.0 ** -120, 2.0 ** np.ceil(np.log2(most / 448 / slack)))
                    largest = 2.0 ** -120 if most == 0 else max(2.0 ** -120, 2.0 ** np.ceil(np.log2(most / 448 * slack)))
                    if r0:
                        b = float(was_scale[to, h])
                        least, largest = max(least, b), max(largest, b)
                        rest = (was[to, h, :r0].float() * (b / c)).to(torch.float8_e4m3fn)
                        assert torch.equal(_bits(cache[to, h, :r0]), _bits(rest)), ("rows from before", x, s, h, i)
                    assert least <= c <= largest and np.log2(c) % 1 == 0, ("scale", x, s, h, i)
                    assert (np.abs(got * c - part) <= np.maximum(2.0 ** -4 * np.abs(part), 2.0 ** -10 * c) + e * (1 + 2.0 ** -4)).all(), ("cache", x, s, h, i)
        at += new
    for x, (cache, was, scale, was_scale) in enumerate(((after.k, before.k, after.k_scale, before.k_scale), (after.v, before.v, after.v_scale, before.v_scale))):
        assert torch.equal(_bits(cache)[~used[x]], _bits(was)[~used[x]]), "rows that are nobody's new ones were written"
        if scale is not None:
            untouched = ~used[x].any(-1)
            assert torch.equal(scale[untouched], was_scale[untouched])


@pytest.mark.parametrize("kind", list(KINDS))
@pytest.mark.parametrize("name", list(CASES))
def test_against_the_oracle(name, kind):
    g, code, q, k, v, q_start, k_len, pos, w, p, norm, lens, front, table = _make(name, kind)
    before = _copy(p)
    out = torch.full((g.heads, g.tokens, g.d), 9.0, dtype=q.dtype, device="cuda")
    P.dfs_paged_append(g, code, q, k, v, q_start, k_len, pos, w[0], w[1], out, p, norm)
    _check(kind, g, q, k, v, pos, w, before, p, out, norm, lens, front, table)
    once, again = _copy(p), torch.full_like(out, 9.0)
    P.dfs_paged_append(g, code, q, k, v, q_start, k_len, pos, w[0], w[1], again, p, norm)            # once more changes nothing
    assert _same(once, p) and torch.equal(out, again)
    qq = q.clone(memory_format=torch.preserve_format)
    P.dfs_paged_append(g, code, qq, k, v, q_start, k_len, pos, w[0], w[1], qq, p, norm)              # in place
    n = sum(x for x, _ in lens)
    assert torch.equal(qq[:, front:front + n], out[:, front:front + n]) and torch.equal(qq[:, front + n:], q[:, front + n:]) and torch.equal(qq[:, :front], q[:, :front])
    assert _same(once, p)


@pytest.mark.parametrize("kind", list(KINDS))
@pytest.mark.parametrize("name", ["tokens_of_streams", "later_pieces", "small_pages", "large_pages"])
def test_token_by_token_holds_what_a_piece_does(name, kind):
    """A sequence's tokens one at a time: the same rows in the end, in 8 bits but for the roundings of a growing scale."""
    g, code, q, k, v, q_start, k_len, pos, w, p, norm, lens, front, table = _make(name, kind, 1)
    if kind == "e4m3":                               # no rows from before: the scale is what these tokens make it
        lens = [(x, 0) for x, _ in lens]
        k_len = torch.tensor([x for x, _ in lens], dtype=torch.int32, device="cuda")
    a, b = _copy(p), _copy(p)
    out, one = (torch.full((g.heads, g.tokens, g.d), 9.0, dtype=q.dtype, device="cuda") for _ in range(2))
    P.dfs_paged_append(g, code, q, k, v, q_start, k_len, pos, w[0], w[1], out, a, norm)
    starts = q_start.tolist()
    for step in range(max(x for x, _ in lens)):
        live = [s for s, (x, _) in enumerate(lens) if step < x]
        gg = P.QkGeom(len(live), len(live), g.heads, g.heads_kv, g.d, g.interleaved, g.axes, g.rot0, g.rot1, g.rot2, g.theta, g.eps)
        pick = torch.tensor([starts[s] + step for s in live], device="cuda")
        i32 = lambda x: torch.tensor(x, dtype=torch.int32, device="cuda")  # noqa: E731
        part = torch.empty(g.heads, len(live), g.d, dtype=q.dtype, device="cuda")
        P.dfs_paged_append(gg, code, q[:, pick], k[:, pick], v[:, pick], i32(range(len(live) + 1)), i32([lens[s][1] + step + 1 for s in live]),
                           None if pos is None else pos[pick], w[0], w[1], part, P.Pages(b.k, b.v, b.table[live], b.k_scale, b.v_scale), norm)
        one[:, pick] = part
    assert torch.equal(out, one)
    if kind != "e4m3":
        assert _same(a, b)
        return
    for s, (n, _) in enumerate(lens):
        for i in range((n + p.k.shape[2] - 1) // p.k.shape[2]):
            to = int(table[s, i])
            rows = min(p.k.shape[2], n - i * p.k.shape[2])
            for x, y, sx, sy in ((a.k, b.k, a.k_scale, b.k_scale), (a.v, b.v, a.v_scale, b.v_scale)):
                assert torch.equal(sx[to], sy[to])
                gap = (x[to, :, :rows].float() - y[to, :, :rows].float()).abs()
                # each doubling of the scale may round what lies below the smallest value once more; elsewhere e4m3 values halve exactly
                assert (gap <= 2.0 ** -9).all() and (gap[x[to, :, :rows].float().abs() >= 2.0 ** -5] == 0).all()


@pytest.mark.parametrize("kind", list(KINDS))
def test_tokens_without_a_place(kind):
    """More new tokens than the length holds, lengths past the table's room, entries that name no page: nothing but the queries is written there."""
    g, code, q, k, v, q_start, k_len, pos, w, p, norm, lens, front, table = _make("prompts", kind, 2)
    before, out = _copy(p), torch.full((g.heads, g.tokens, g.d), 9.0, dtype=q.dtype, device="cuda")
    bad = p.table.clone()
    bad[0, 1], bad[2, 0], bad[4, :] = -1, p.k.shape[0], 1 << 30
    short = k_len.clone()
    short[3] = 10                                    # 63 tokens, of which the last ten have places
    short[1] = 1 << 30                               # cut to the table's room, whose last entry is no page
    pp = P.Pages(p.k, p.v, bad, p.k_scale, p.v_scale)
    P.dfs_paged_append(g, code, q, k, v, q_start, short, pos, w[0], w[1], out, pp, norm)
    assert not (out[:, front:front + sum(x for x, _ in lens)] == 9).all(-1).any()
    touched = {(int(table[0, i])) for i in (0, 2, 3)} | {int(table[3, 0])}
    for x, y in ((p.k, before.k), (p.v, before.v)):
        changed = {i for i in range(x.shape[0]) if not torch.equal(_bits(x[i]), _bits(y[i]))}
        assert changed == touched
        assert torch.equal(_bits(x[int(table[3, 0]), :, 10:]), _bits(y[int(table[3, 0]), :, 10:]))


def _guarded(like, mark):
    """A copy of a tensor with as much room of marks in front of it and behind, as bytes."""
    bits = _bits(like.contiguous()).flatten()
    n = (bits.numel() + 4096) // 256 * 256
    room = torch.full((2 * n + bits.numel(),), mark, dtype=torch.uint8, device="cuda")
    room[n:-n] = bits
    return room[n:-n].view(like.dtype).view(like.shape), (room[:n], room[-n:])


@pytest.mark.parametrize("kind", list(KINDS))
@pytest.mark.parametrize("name", ["one_token", "tokens_of_streams", "prompts", "later_pieces", "small_pages", "large_pages", "many_streams", "few_but_two", "few_but_one"])
def test_starts_that_break_the_format(name, kind):
    """Starts outside the rows are cut to them; where one falls, nothing in front of or behind the queries' rows, the pages and their scales is touched."""
    g, code, q, k, v, q_start, k_len, pos, w, p, norm, lens, front, table = _make(name, kind, 5)
    wide, cut = q_start.clone(), q_start.clone()
    wide[0], wide[-1], cut[0], cut[-1] = -5, 1 << 30, 0, g.tokens
    outs, caches = [], []
    for start in (wide, cut):
        caches.append(_copy(p))
        outs.append(torch.full((g.heads, g.tokens, g.d), 9.0, dtype=q.dtype, device="cuda"))
        P.dfs_paged_append(g, code, q, k, v, start, k_len, pos, w[0], w[1], outs[-1], caches[-1], norm)
    assert _same(*caches) and torch.equal(*outs) and not (outs[0] == 9).all(-1).any()
    odd = torch.arange(g.batch + 1, device="cuda") % 2 == 1
    for start in (q_start.flip(0), torch.where(odd, -q_start, q_start), torch.where(odd, torch.zeros_like(q_start), torch.full_like(q_start, g.tokens + 9))):
        out, out_room = _guarded(torch.full((g.heads, g.tokens, g.d), 9.0, dtype=q.dtype, device="cuda"), 7)
        parts = [None if x is None else _guarded(x, 7) for x in (p.k, p.v, p.k_scale, p.v_scale)]
        here = [None if x is None else x[0] for x in parts]
        P.dfs_paged_append(g, code, q, k, v, start.int(), k_len, pos, w[0], w[1], out, P.Pages(here[0], here[1], p.table, here[2], here[3]), norm)
        torch.cuda.synchronize()
        assert all((x == 7).all() for x in [*out_room] + [y for x in parts if x is not None for y in x[1]])


def test_values_that_are_not_finite():
    """e4m3: infinities and NaN are stored as NaN and leave the scale to the others; a page of zeros has the smallest scale."""
    g = P.QkGeom(1, 3, 1, 1, 64, 0, 1, 64, 0, 0, 1e4, 1e-5)
    k, v = torch.zeros(1, 3, 64, device="cuda", dtype=torch.bfloat16), torch.randn(1, 3, 64, device="cuda").bfloat16()
    v[0, 0, 3], v[0, 1, 5], v[0, 2, 7] = float("inf"), float("-inf"), float("nan")
    z = lambda: torch.zeros(1, 1, 16, 64, device="cuda").to(torch.float8_e4m3fn)  # noqa: E731
    p = P.Pages(z(), z(), torch.zeros(1, 1, dtype=torch.int32, device="cuda"), torch.ones(1, 1, device="cuda"), torch.ones(1, 1, device="cuda"))
    start, length = (torch.tensor(x, dtype=torch.int32, device="cuda") for x in ([0, 3], [3]))
    P.dfs_paged_append(g, P.DFS_BF16, k, k, v, start, length, None, None, None, torch.empty_like(k), p, False)
    assert float(p.k_scale) == 2.0 ** -120 and not p.k.float().any()
    got, finite = p.v.float()[0, 0, :3], torch.isfinite(v[0].float())
    assert torch.equal(torch.isnan(got), ~finite)
    most = v[0].float()[finite].abs().max()
    c = float(p.v_scale)
    assert most <= 448 * c and most > 224 * c
    want = (v[0].float() / c).to(torch.float8_e4m3fn).float()
    assert torch.equal(got[finite], want[finite])
    far = torch.full_like(v, 3e38)                   # the largest scale
    far[0, 1:] = 1e-30
    P.dfs_paged_append(g, P.DFS_BF16, k, k, far, start, length, None, None, None, torch.empty_like(k), p, False)
    assert float(p.v_scale) == 2.0 ** 120 and torch.equal(p.v.float()[0, 0, :3], (far[0].float() / 2.0 ** 120).to(torch.float8_e4m3fn).float())


@pytest.mark.parametrize("new", [1, 3, 20])                     # a wave's page, at d = 128 a work-group's from five rows on
@pytest.mark.parametrize("size", [1.0, 2.0 ** 30])            # the rows' scale stays, or grows
def test_rows_from_before_with_a_scale_of_the_users(size, new):
    """e4m3: of a scale that is no power of two the exponent alone counts, for attention and for an append behind the rows that have it, whose new rows stand beside them."""
    g = P.QkGeom(1, new, 1, 1, 128, 0, 1, 128, 0, 0, 1e4, 1e-5)
    gen = torch.Generator(device="cuda").manual_seed(14)
    was = torch.randn(2, 1, 1, 32, 128, generator=gen, device="cuda").to(torch.float8_e4m3fn)
    k, v = (torch.randn(2, 1, new, 128, generator=gen, device="cuda") * size).bfloat16()
    start, length = (torch.tensor(x, dtype=torch.int32, device="cuda") for x in ([0, new], [7 + new]))
    table, caches = torch.zeros(1, 1, dtype=torch.int32, device="cuda"), []
    for scales in ((-3.5, 1.25 * 2.0 ** 9), (2.0, 2.0 ** 9)):
        p = P.Pages(*was.clone(), table, *(torch.full((1, 1), x, device="cuda") for x in scales))
        one = torch.tensor([0, 1], dtype=torch.int32, device="cuda")
        w, o = P.Paged(1, 1, 1, 128, 1, -1, 0), torch.empty(1, 1, 128, dtype=torch.bfloat16, device="cuda")
        ws = torch.empty(P.dfs_paged_workspace_bytes(w, P.DFS_BF16, p), dtype=torch.uint8, device="cuda")
        P.dfs_paged_attn_fwd(w, P.DFS_BF16, k[:, :1] / size, p, one, torch.full_like(length, 7), 0.01, o, None, ws)
        P.dfs_paged_append(g, P.DFS_BF16, k, k, v, start, length, None, None, None, torch.empty_like(k), p, False)
        caches.append((p, o))
    (a, o_a), (b, o_b) = caches
    assert _same(a, b) and torch.equal(o_a, o_b)
    assert (float(a.k_scale), float(a.v_scale)) == (2.0, 512.0) if size == 1 else min(float(a.k_scale), float(a.v_scale)) > 2.0 ** 20


@pytest.mark.parametrize("new", [2, 20])
def test_rows_from_before_whose_scale_is_not_finite(new):
    """e4m3: they become NaN, the new ones are as on a page of their own scale."""
    g = P.QkGeom(1, new, 1, 1, 128, 0, 1, 128, 0, 0, 1e4, 1e-5)
    gen = torch.Generator(device="cuda").manual_seed(15)
    k, v = torch.randn(2, 1, new, 128, generator=gen, device="cuda").bfloat16()
    start, length = (torch.tensor(x, dtype=torch.int32, device="cuda") for x in ([0, new], [7 + new]))
    caches = []
    for scales in ((float("nan"), float("inf")), (2.0 ** -110, 2.0 ** -110)):
        p = P.Pages(*torch.ones(2, 1, 1, 32, 128, device="cuda").to(torch.float8_e4m3fn), torch.zeros(1, 1, dtype=torch.int32, device="cuda"),
                    *(torch.full((1, 1), x, device="cuda") for x in scales))
        P.dfs_paged_append(g, P.DFS_BF16, k, k, v, start, length, None, None, None, torch.empty_like(k), p, False)
        caches.append(p)
    a, b = caches
    for x, y in ((a.k, b.k), (a.v, b.v)):
        assert torch.isnan(x[0, 0, :7].float()).all() and torch.equal(_bits(x[0, 0, 7:]), _bits(y[0, 0, 7:]))
    assert torch.equal(a.k_scale, b.k_scale) and torch.equal(a.v_scale, b.v_scale)


def test_pages_past_32_bits():
    """A page more than 2^32 bytes behind the first."""
    g = P.QkGeom(1, 5, 1, 1, 128, 0, 1, 128, 0, 0, 1e4, 1e-5)
    pages = (1 << 21) + 1000                         # of 2 KB
    k = torch.zeros(pages, 1, 16, 128, dtype=torch.float8_e4m3fn, device="cuda")
    v, ones = torch.zeros_like(k), torch.ones(pages, 1, device="cuda")
    p = P.Pages(k, v, torch.tensor([[pages - 1]], dtype=torch.int32, device="cuda"), ones.clone(), ones.clone())
    small = P.Pages(k[:1].clone(), v[:1].clone(), torch.zeros(1, 1, dtype=torch.int32, device="cuda"), ones[:1].clone(), ones[:1].clone())
    x = torch.randn(1, 5, 128, device="cuda").bfloat16()
    start, length = (torch.tensor(y, dtype=torch.int32, device="cuda") for y in ([0, 5], [5]))
    for c in (p, small):
        P.dfs_paged_append(g, P.DFS_BF16, x, x, x, start, length, None, None, None, torch.empty_like(x), c)
    assert torch.equal(_bits(p.k[-1]), _bits(small.k[0])) and torch.equal(_bits(p.v[-1]), _bits(small.v[0])) and small.k.float().any()
    assert torch.equal(p.k_scale[-1], small.k_scale[0]) and not p.k[:2].float().any()


def test_captured_and_replayed():
    """A decoding step in a graph whose lengths grow from replay to replay."""
    g, code, q, k, v, q_start, k_len, pos, w, p, norm, lens, front, table = _make("tokens_of_streams", "e4m3", 4)
    a, out = _copy(p), torch.empty(g.heads, g.tokens, g.d, dtype=q.dtype, device="cuda")
    k_len[:] = torch.tensor([5, 8, 20, 1, 30, 900], dtype=torch.int32)
    lengths = k_len.clone()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        P.dfs_paged_append(g, code, q, k, v, q_start, k_len, pos, w[0], w[1], out, a, norm)
        k_len.add_(1)
    b, want = _copy(p), torch.empty_like(out)
    for _ in range(4):
        graph.replay()
        P.dfs_paged_append(g, code, q, k, v, q_start, lengths, pos, w[0], w[1], want, b, norm)
        lengths += 1
        torch.cuda.synchronize()
        assert _same(a, b) and torch.equal(out[:, front:-3], want[:, front:-3])


def test_refusals_of_the_binding():
    g, code, q, k, v, q_start, k_len, pos, w, p, norm, lens, front, table = _make("later_pieces", "e4m3")
    out, before = torch.zeros(g.heads, g.tokens, g.d, dtype=q.dtype, device="cuda"), _copy(p)
    good = [g, code, q, k, v, q_start, k_len, pos, w[0], w[1], out, p, norm]
    pg = lambda **kw: P.Pages(**dict(dict(k=p.k, v=p.v, table=p.table, k_scale=p.k_scale, v_scale=p.v_scale), **kw))  # noqa: E731
    for i, bad in ((2, q.float()), (2, q.cpu()), (2, k), (3, q), (4, v[:, 1:]), (5, q_start[:-1]), (6, k_len.long()), (6, k_len[:-1]), (7, pos[:-1]), (7, pos[:, :1]), (7, pos.long()),
                   (8, w[0].double()), (10, out.float()), (11, pg(k=p.k.float().half())), (11, pg(k=p.k[0])), (11, pg(v=p.v[1:])),
                   (11, pg(v=p.v.float().bfloat16())), (11, pg(table=p.table[1:])), (11, pg(table=p.table.long())), (11, pg(table=p.table.cpu())), (11, pg(k_scale=p.k_scale[1:])),
                   (11, pg(k_scale=p.k_scale.double()))):
        args = list(good)
        args[i] = bad
        with pytest.raises(ValueError):
            P.dfs_paged_append(*args)
    for i, bad in ((5, None), (6, None), (7, None), (10, None), (11, None), (11, pg(k_scale=None)), (11, pg(v=p.k)), (12, False)):
        args = list(good)
        args[i] = bad
        with pytest.raises(P.DfsError):
            P.dfs_paged_append(*args)
    assert not out.any() and _same(before, p)


@pytest.mark.parametrize("kind", list(KINDS))
def test_pages_without_a_part(kind):
    """A cache that lacks its keys, its values or its table: the library's error, as for a call without a cache."""
    g, code, q, k, v, q_start, k_len, pos, w, p, norm, lens, front, table = _make("later_pieces", kind)
    out, before = torch.zeros(g.heads, g.tokens, g.d, dtype=q.dtype, device="cuda"), _copy(p)
    read = P.Paged(g.batch, g.heads, g.heads_kv, g.d, g.tokens, -1, 0)
    for part in ("k", "v", "table", "k v"):
        bad = P.Pages(**dict(dict(k=p.k, v=p.v, table=p.table, k_scale=p.k_scale, v_scale=p.v_scale), **{x: None for x in part.split()}))
        with pytest.raises(P.DfsError, match="pages" if part != "table" else "table"):
            P.dfs_paged_append(g, code, q, k, v, q_start, k_len, pos, w[0], w[1], out, bad, norm)
        with pytest.raises(P.DfsError, match="pages" if part != "table" else "table"):
            P.dfs_paged_attn_fwd(read, code, q, bad, q_start, k_len, 0.1, out, None, torch.empty(1 << 25, dtype=torch.uint8, device="cuda"))
        assert P.dfs_paged_workspace_bytes(read, code, bad) == 0
    if kind == "e4m3":
        with pytest.raises(P.DfsError, match="share memory"):
            P.dfs_paged_append(g, code, q, k, v, q_start, k_len, pos, w[0], w[1], out, P.Pages(p.k, p.v, p.table, p.k_scale, p.k_scale), norm)
    assert not out.any() and _same(before, p)
