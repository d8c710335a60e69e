"""Attention over sequences of different lengths that lie behind one another without padding, and over a cache in pages, as cases to be timed:

  append  queries and keys of new tokens normed and turned by their position, keys and values put into the pages of a cache, in bf16 or in
          8 bits (e4m3) with a scale for each page and head, which grows with what the page holds
  read    attention over such a cache: single tokens of many sequences, or pieces of prompts
  packed  attention within packed sequences, causal or both ways, with shared key heads
  train   its forward and backward pass, as a training step makes them

Where `own` is false, a pass is computed in elementary torch operations in 32 bits; where it is true, by the package's calls.
Sizes follow the package's own shapes (clips of 13 x 30 x 45 and 5 x 19 x 27 tokens, 12 to 40 heads of 64 or 128) and those of models that share key
heads between query heads.
"""
from __future__ import annotations

import math

import torch

own = False

DEV = "cuda"
_TYPES = {"bf16": torch.bfloat16, "f32": torch.float32, "e4m3": torch.float8_e4m3fn}
EPS = 1e-6
LEAST = -120                                                    # exponent of the smallest scale of a page
_APPEND = dict(op="append", seqs=1, heads=32, heads_kv=8, d=128, dtype="bf16", cache="e4m3", page=64, tokens=1, fill=0, interleaved=False, axes=1,
               theta=1e4, norm=True)
_READ = dict(op="read", seqs=1, heads=32, heads_kv=8, d=128, dtype="bf16", cache="e4m3", page=64, tokens=1, fill=0, left=-1, sinks=0)
_PACKED = dict(op="packed", seqs=1, heads=32, heads_kv=8, d=128, dtype="bf16", tokens=1, left=-1, right=0)


def _append(name, **kw):
    return dict(_APPEND, name=name, **kw)


def _read(name, **kw):
    return dict(_READ, name=name, **kw)


def _packed(name, **kw):
    return dict(_PACKED, name=name, **kw)


def listed():
    return [
        # a decoding step of 32 streams: one new token each, behind up to 8 192 others; latency counts
        _append("append_tokens", seqs=32, tokens=32, fill=8192, theta=5e5),
        # five prompts of different lengths, 16 384 tokens in all, some of them later pieces that begin inside a page
        _append("append_prompts", seqs=5, tokens=16384, fill=1000, theta=5e5),
        # the tokens of two clips of 5 x 19 x 27 with a position of three numbers, into small pages of bf16
        _append("append_clips_bf16", seqs=2, tokens=5130, heads=12, heads_kv=12, d=64, cache="bf16", page=16, interleaved=True, axes=3),
        # one token of a lone stream over 100 000 others
        _read("read_lone_stream", fill=100000),
        # one token each of 48 streams of up to 16 384
        _read("read_streams", seqs=48, tokens=48, fill=16384),
        # 16 streams with a window and a few first tokens, heads of 64, small pages of bf16
        _read("read_window_bf16", seqs=16, tokens=16, fill=8192, heads=16, heads_kv=4, d=64, cache="bf16", page=16, left=1023, sinks=4),
        # later pieces of four prompts, 4 096 tokens in all, each over what the cache holds of its prompt
        _read("read_pieces", seqs=4, tokens=4096, fill=8192),
        # six whole prompts, 16 384 tokens in all
        _packed("packed_prompts", seqs=6, tokens=16384),
        # three clips of different lengths, every token sees its whole clip
        _packed("packed_clips", seqs=3, tokens=24815, heads=30, heads_kv=30, d=64, right=-1),
        # a check in fp32 at odd sizes
        _packed("packed_small_fp32", seqs=5, tokens=701, heads=4, heads_kv=2, d=64, dtype="f32"),
        # a training step over nine texts packed into 8 192 tokens
        _packed("train_texts", op="train", seqs=9, tokens=8192),
        # a training step in fp32 over three short texts, heads of 64
        _packed("train_small_fp32", op="train", seqs=3, tokens=1000, heads=12, heads_kv=4, d=64, dtype="f32"),
    ]


# ----------------------------------------------------------------------------------------------------- drawn cases


def _log_int(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def _heads(rng, most):
    kv = _log_int(rng, 1, most)
    return dict(heads=kv * rng.choice([1, 1, 2, 3, 4, 8]), heads_kv=kv)


def _draw_append(rng):
    c = dict(_APPEND, d=rng.choice([64, 128]), cache=rng.choice(["e4m3", "e4m3", "bf16"]), page=rng.choice([16, 32, 64, 128]),
             interleaved=rng.random() < 0.4, axes=rng.choice([1, 1, 3]), theta=rng.choice([1e4, 5e5]), norm=rng.random() < 0.7, **_heads(rng, 16))
    if rng.random() < 0.1:
        c.update(dtype="f32", cache="f32")
    if rng.random() < 0.5:
        seqs = _log_int(rng, 1, 128)
        c.update(seqs=seqs, tokens=seqs * rng.choice([1, 1, 1, 3]), fill=_log_int(rng, 4, 8192))
    else:
        seqs = rng.randint(1, 12)
        c.update(seqs=seqs, tokens=seqs + _log_int(rng, 8, 20000), fill=rng.choice([0, rng.randint(1, 4000)]))
    return c


def _draw_read(rng):
    c = dict(_READ, d=rng.choice([64, 128]), cache=rng.choice(["e4m3", "e4m3", "bf16"]), page=rng.choice([16, 32, 64, 128]), **_heads(rng, 8))
    if rng.random() < 0.1:
        c.update(dtype="f32", cache="f32")
    if rng.random() < 0.3:
        c.update(left=_log_int(rng, 1, 4096), sinks=rng.choice([0, 1, 4, rng.randint(5, 200)]))
    if rng.random() < 0.65:
        seqs = _log_int(rng, 1, 64)
        c.update(seqs=seqs, tokens=seqs * rng.choice([1, 1, 1, 4]), fill=_log_int(rng, 8, 32768))
    else:
        seqs = rng.randint(1, 8)
        c.update(seqs=seqs, tokens=seqs + _log_int(rng, 16, 4096), fill=rng.choice([0, _log_int(rng, 1, 16384)]))
    return c


def _draw_packed(rng):
    seqs = _log_int(rng, 1, 40)
    c = dict(_PACKED, op=rng.choice(["packed", "packed", "train"]), seqs=seqs, tokens=seqs + _log_int(rng, 16, 20000), d=rng.choice([64, 128]),
             right=rng.choice([0, 0, 0, -1]), **_heads(rng, 12))
    if rng.random() < 0.25:
        c["left"] = _log_int(rng, 1, 4096)
    if rng.random() < 0.15:
        c.update(dtype="f32", tokens=min(c["tokens"], 2000))
    return c


def draw(rng):
    most = {key: max(work(c)[key] for c in listed()) for key in ("bytes", "flops")}
    while True:
        c = rng.choice([_draw_append, _draw_read, _draw_packed])(rng)
        w = work(c)
        # the cache that stands behind an append is not its work: kept to what the listed ones have
        if all(w[key] <= most[key] for key in most) and c["seqs"] * c.get("fill", 0) * c["heads_kv"] * c["d"] <= 1 << 30:
            return c


# --------------------------------------------------------------------------------------------------------- inputs


def _spread(n, lo, hi):
    """n lengths between lo and hi, far apart."""
    return [int(lo + (hi - lo) * ((i + 1) * 0.6180339887 % 1.0)) for i in range(n)]


def _parts(n, total):
    """n lengths of `total` in all, one at least each."""
    share = [1 + 3 * ((i + 1) * 0.6180339887 % 1.0) for i in range(n)]
    got, left, rest = [], total, sum(share)
    for i, x in enumerate(share):
        m = left if i == n - 1 else max(1, min(left - (n - 1 - i), int(round(left * x / rest))))
        got.append(m)
        left, rest = left - m, rest - x
    return got


def _lengths(c):
    """New tokens of every sequence, and how many it has with those in front of them."""
    each = c["tokens"] // c["seqs"]
    n = [each] * c["seqs"] if each * c["seqs"] == c["tokens"] and each <= 16 else _parts(c["seqs"], c["tokens"])
    before = _spread(c["seqs"], c["fill"] // 2, c["fill"]) if c.get("fill") else [0] * c["seqs"]
    return n, [x + y for x, y in zip(n, before)]


def _axes(c):
    """Channels turned by each number of a position."""
    if c["axes"] == 1:
        return [c["d"]]
    return [16, 24, 24] if c["d"] == 64 and c["interleaved"] else [32, 16, 16] if c["d"] == 64 else [44, 42, 42] if c["interleaved"] else [64, 32, 32]


def _generator(seed):
    g = torch.Generator(device=DEV)
    g.manual_seed(seed)
    return g


def _starts(lengths):
    at = [0]
    for n in lengths:
        at.append(at[-1] + n)
    return torch.tensor(at, dtype=torch.int32, device=DEV)


def _cache(c, gen, k_len):
    """Pages in no order, as they are after some time of use: keys, values, their scales and the table."""
    page, kv, d = c["page"], c["heads_kv"], c["d"]
    need = [(n + page - 1) // page for n in k_len]
    pages, row = sum(need) + 3, max(need)
    order = torch.randperm(pages, generator=gen, device=DEV).int()
    table, at = torch.zeros(c["seqs"], row, dtype=torch.int32, device=DEV), 0
    for i, n in enumerate(need):
        table[i, :n] = order[at:at + n]
        at += n
    shape = (pages, kv, page, d)
    k, v = (torch.randn(shape, generator=gen, device=DEV) for _ in range(2))
    if c["cache"] != "e4m3":
        return dict(k=k.to(_TYPES[c["cache"]]), v=v.to(_TYPES[c["cache"]]), k_scale=None, v_scale=None, table=table)
    scale = [torch.exp2(torch.randint(-8, -5, shape[:2], generator=gen, device=DEV).float()) for _ in range(2)]
    k, v = ((x / s[:, :, None, None]).clamp_(-448, 448).to(_TYPES["e4m3"]) for x, s in zip((k, v), scale))
    return dict(k=k, v=v, k_scale=scale[0], v_scale=scale[1], table=table)


def _own_cache(st):
    import paper_2605_23445_amd as P
    return P.Pages(st["k"], st["v"], st["table"], st["k_scale"], st["v_scale"])


def _code(c):
    import paper_2605_23445_amd as P
    return P.DFS_BF16 if c["dtype"] == "bf16" else P.DFS_F32


def _room(n):
    return torch.empty(max(256, n), dtype=torch.uint8, device=DEV)


def _prepare_append(c, seed):
    gen, dt, h, kv, d = _generator(seed), _TYPES[c["dtype"]], c["heads"], c["heads_kv"], c["d"]
    rand = lambda *s: torch.randn(*s, generator=gen, device=DEV)  # noqa: E731
    n, k_len = _lengths(c)
    channel = torch.exp(0.5 * rand((h + 2 * kv) * d))                                      # channels of a projection differ in size
    fused = (rand(c["tokens"], (h + 2 * kv) * d) * channel).to(dt).view(c["tokens"], h + 2 * kv, d).transpose(0, 1)
    st = dict(c=c, x=(fused[:h], fused[h:h + kv], fused[h + kv:]), w_q=1 + 0.2 * rand(d), w_k=1 + 0.2 * rand(d), lens=(n, k_len),
              q_start=_starts(n), k_len=torch.tensor(k_len, dtype=torch.int32, device=DEV), pos=None, **_cache(c, gen, k_len))
    if c["axes"] == 3:                                                                     # frames of 19 x 27 tokens
        p = torch.cat([torch.arange(a - b, a, device=DEV) for a, b in zip(k_len, n)])
        st["pos"] = torch.stack([p // 513, p // 27 % 19, p % 27], dim=-1).int().contiguous()
    st["q_out"] = torch.empty(h, c["tokens"], d, dtype=dt, device=DEV)
    if own:
        import paper_2605_23445_amd as P
        rot = _axes(c) + [0, 0]
        st["g"] = P.QkGeom(c["seqs"], c["tokens"], h, kv, d, int(c["interleaved"]), c["axes"], *rot[:3], c["theta"], EPS)
        st["dt"], st["pages"] = _code(c), _own_cache(st)
    return st


def _prepare_read(c, seed):
    gen, dt = _generator(seed), _TYPES[c["dtype"]]
    n, k_len = _lengths(c)
    q = torch.randn(c["heads"], c["tokens"], c["d"], generator=gen, device=DEV).to(dt)
    st = dict(c=c, q=q, lens=(n, k_len), q_start=_starts(n), k_len=torch.tensor(k_len, dtype=torch.int32, device=DEV), scale=1 / math.sqrt(c["d"]),
              **_cache(c, gen, k_len))
    st["o"], st["lse"] = torch.empty_like(q), torch.empty(c["heads"], c["tokens"], device=DEV)
    if own:
        import paper_2605_23445_amd as P
        st["w"] = P.Paged(c["seqs"], c["heads"], c["heads_kv"], c["d"], c["tokens"], c["left"], c["sinks"])
        st["dt"], st["pages"] = _code(c), _own_cache(st)
        st["ws"] = _room(P.dfs_paged_workspace_bytes(st["w"], st["dt"], st["pages"]))
    return st


def _prepare_packed(c, seed):
    gen, dt, d, t = _generator(seed), _TYPES[c["dtype"]], c["d"], c["tokens"]
    rand = lambda heads: torch.randn(heads, t, d, generator=gen, device=DEV).to(dt)  # noqa: E731
    n = _lengths(c)[0]
    st = dict(c=c, q=rand(c["heads"]), k=rand(c["heads_kv"]), v=rand(c["heads_kv"]), lens=(n, n), q_start=_starts(n), scale=1 / math.sqrt(d))
    st["o"], st["lse"] = torch.empty_like(st["q"]), torch.empty(c["heads"], t, device=DEV)
    if c["op"] == "train":
        st["do"] = rand(c["heads"])
        st["dq"], st["dk"], st["dv"] = (torch.empty_like(st[x]) for x in "qkv")
    if own:
        import paper_2605_23445_amd as P
        st["w"] = P.Packed(c["seqs"], c["heads"], c["heads_kv"], d, t, t, c["left"], c["right"])
        st["dt"] = _code(c)
        st["ws"] = _room(max(P.dfs_packed_workspace_bytes(st["w"], st["dt"], back) for back in {False, c["op"] == "train"}))
    return st


_KINDS = {"append": _APPEND, "read": _READ, "packed": _PACKED, "train": _PACKED}


def _whole(case):
    return dict(_KINDS[case["op"]], **case)


def prepare(case, seed):
    c = _whole(case)
    return {"append": _prepare_append, "read": _prepare_read}.get(c["op"], _prepare_packed)(c, seed)


# ----------------------------------------------------------------------------------------------------- plain forms


def _sequence_of(q_start, n):
    """The sequence of each of n rows and its place there."""
    row = torch.arange(n, device=DEV)
    s = torch.searchsorted(q_start.long(), row, right=True) - 1
    return s, row - q_start.long()[s]


def _turned(c, y, pos):
    """y [heads, n, d] turned by the positions [n, axes]; angles in 64 bits."""
    ang, first, second, at = [], [], [], 0
    for axis, m in enumerate(_axes(c)):
        i = torch.arange(m // 2, device=DEV)
        ang.append(pos[:, axis, None].double() * torch.exp(-math.log(c["theta"]) * 2.0 * i.double() / m))
        first.append(at + (2 * i if c["interleaved"] else i))
        second.append(at + (2 * i + 1 if c["interleaved"] else i + m // 2))
        at += m
    a, i, j = torch.cat(ang, dim=-1), torch.cat(first), torch.cat(second)
    cos, sin, x, z = torch.cos(a).float(), torch.sin(a).float(), y[..., i], y[..., j]
    out = y.clone()
    out[..., i], out[..., j] = x * cos - z * sin, x * sin + z * cos
    return out


def _scale_for(most):
    """The smallest power of two by which `most` becomes 448 at most."""
    m, e = torch.frexp(most)
    e = torch.where(m > 0.875, e - 8, e - 9).clamp(min=LEAST)
    return torch.where(most == 0, torch.full_like(most, 2.0 ** LEAST), torch.exp2(e.float()))


def _append_plain(st):
    c, page, kv = st["c"], st["c"]["page"], st["c"]["heads_kv"]
    n, dt = c["tokens"], st["q_out"].dtype
    seq, i = _sequence_of(st["q_start"], n)
    new, total = torch.diff(st["q_start"]).long(), st["k_len"].long()
    p = (total - new)[seq] + i
    pos = p[:, None] if st["pos"] is None else st["pos"]
    res = []
    for x, w in zip(st["x"], (st["w_q"], st["w_k"])):
        x = x.float()
        if c["norm"]:
            x = x * torch.rsqrt(x.square().mean(-1, keepdim=True) + EPS) * w
        res.append(_turned(c, x, pos))
    st["q_out"].copy_(res[0])
    at, row = st["table"].long()[seq, p // page], p % page                                 # page and row of every new token
    begin = total - new
    first, old = st["table"].long()[torch.arange(c["seqs"], device=DEV), begin // page], begin % page   # first page of every sequence, rows it has
    for cache, scale, y in ((st["k"], st["k_scale"], res[1]), (st["v"], st["v_scale"], st["x"][2].float())):
        if scale is not None:
            most = torch.full_like(scale, -1.0).index_reduce_(0, at, y.abs().amax(-1).t(), "amax")
            need = torch.where(most < 0, scale, _scale_for(most))
            keep = torch.where((old > 0)[:, None], torch.maximum(need[first], scale[first]), need[first])
            there = (torch.arange(page, device=DEV) < old[:, None])[:, None, :, None]
            was = cache[first]
            cache[first] = torch.where(there, was.float() * (scale[first] / keep)[:, :, None, None], was.float()).to(cache.dtype)
            need[first] = keep
            scale.copy_(need)
            y = y / scale[at].t()[:, :, None]
        cache[at, :, row] = y.transpose(0, 1).to(cache.dtype)
    return _append_outputs(st)


def _append_outputs(st):
    """The cache is what it is in place: values in units of their page's scale, and the scales, which are powers of two."""
    out = {"q": st["q_out"], "k": st["k"], "v": st["v"]}
    return out if st["k_scale"] is None else dict(out, k_scale=st["k_scale"], v_scale=st["v_scale"])


def _attend(st, fetch, train=False):
    """o, lse (and dq, dk, dv) of packed rows; fetch(s, key): keys and values [s, heads_kv, keys, d] at places `key` [s, keys] of the sequences `s`."""
    c, q = st["c"], st["q"]
    h, kv, d, n, sinks = c["heads"], c["heads_kv"], c["d"], c["tokens"], c.get("sinks", 0)
    group, scale, (q_lens, k_lens) = h // kv, st["scale"], st["lens"]
    o, lse = torch.empty(h, n, d, device=DEV), torch.empty(h, n, device=DEV)
    grads = [torch.empty(h, n, d, device=DEV), torch.zeros(n, kv, d, device=DEV), torch.zeros(n, kv, d, device=DEV)] if train else []
    q_start, seqs = st["q_start"].long(), c["seqs"]
    alone = n >= 256 * seqs                                                                # long sequences one by one, short ones all at once
    for s0 in range(seqs if alone else 1):
        s = torch.arange(s0, s0 + 1 if alone else seqs, device=DEV)
        n_q, n_k = (max(x[s0:s0 + 1] if alone else x) for x in (q_lens, k_lens))
        shift = [a - b for a, b in zip(k_lens, q_lens)][s0:s0 + 1 if alone else seqs]
        q_len = q_start[s + 1] - q_start[s]
        k_len = st["k_len"].long()[s] if "k_len" in st else q_len
        left, right = n_k if c["left"] < 0 else min(c["left"], n_k), n_k if c.get("right", 0) < 0 else min(c.get("right", 0), n_k)
        step = 1024
        while step > 16 and len(s) * h * step * min(n_k, left + step + right + sinks) * 4 > 1 << 30:
            step //= 2
        tiles = []
        for r0 in range(0, n_q, step):
            r1 = min(n_q, r0 + step)
            row = torch.arange(r0, r1, device=DEV)
            pos = (k_len - q_len)[:, None] + row                                           # [s, rows]
            if left + r1 - r0 + right + sinks < n_k:                                       # first keys, and the window's
                lo = (pos[:, :1] - left).clamp(min=0)
                key = torch.cat([torch.arange(sinks, device=DEV).expand(len(s), -1), lo + torch.arange(left + r1 - r0 + right, device=DEV)], dim=1)
                twice = torch.arange(key.shape[1], device=DEV) < sinks
                there = (key < k_len[:, None]) & ~(twice & (key >= lo))                    # a first key in the window counts there
            else:
                key = torch.arange(min(n_k, max(shift) + r1 + right), device=DEV).expand(len(s), -1)
                there = key < k_len[:, None]
            see = there[:, None] & (key[:, None] <= pos[..., None] + right) & ((key[:, None] >= pos[..., None] - left) | (key < sinks)[:, None])
            see = (see & (row < q_len[:, None])[..., None])[:, None, None]                 # [s, 1, 1, rows, keys]
            at = torch.minimum(q_start[s][:, None] + row, (q_start[s + 1] - 1)[:, None])   # rows of q; behind a sequence's last, that
            ks, vs = (x.float()[:, :, None] for x in fetch(s, torch.minimum(key, (k_len - 1)[:, None])))
            pick = lambda x: x[:, at].float().transpose(0, 1).reshape(len(s), kv, group, r1 - r0, d)  # noqa: E731
            qs = pick(q)
            x = torch.matmul(qs, ks.transpose(-1, -2)).mul_(scale).masked_fill_(~see, -math.inf)
            m = x.amax(-1, keepdim=True)
            m = torch.where(m == -math.inf, torch.zeros_like(m), m)
            w = x.sub_(m).exp_()
            sums = w.sum(-1, keepdim=True)
            w = w.div_(torch.where(sums == 0, torch.ones_like(sums), sums))
            y = torch.matmul(w, vs)
            got = [y, m + sums.log()]
            if train:
                do = pick(st["do"]) * (row < q_len[:, None])[:, None, None, :, None]
                ds = torch.matmul(do, vs.transpose(-1, -2)).sub_((do * y).sum(-1, keepdim=True)).mul_(w).mul_(scale)
                got.append(torch.matmul(ds, ks))
                flat = (q_start[s][:, None] + torch.minimum(key, (k_len - 1)[:, None])).reshape(-1)
                for grad, a, b in ((grads[1], ds, qs), (grads[2], w, do)):                 # keys that are not there add zeros
                    grad.index_add_(0, flat, torch.matmul(a.transpose(-1, -2), b).sum(2).permute(0, 2, 1, 3).reshape(-1, kv, d))
            tiles.append([z.reshape(len(s), h, r1 - r0, -1) for z in got])
        whole = [torch.cat(z, dim=2) for z in zip(*tiles)]                                 # [s, heads, rows, .]
        if alone:
            to = slice(sum(q_lens[:s0]), sum(q_lens[:s0 + 1]))
            whole = [z[0] for z in whole]
        else:
            to, (seq, i) = slice(None), _sequence_of(st["q_start"], n)
            whole = [z[seq, :, i].transpose(0, 1) for z in whole]
        o[:, to], lse[:, to] = whole[0], whole[1][..., 0]
        if train:
            grads[0][:, to] = whole[2]
    if not train:
        return {"o": o.to(q.dtype), "lse": lse}
    return {"o": o.to(q.dtype), "lse": lse, "dq": grads[0].to(q.dtype), "dk": grads[1].transpose(0, 1).to(q.dtype), "dv": grads[2].transpose(0, 1).to(q.dtype)}


def _read_plain(st):
    page = st["c"]["page"]

    def fetch(s, key):
        at, row = st["table"].long()[s[:, None], key // page], key % page
        got = []
        for cache, scale in ((st["k"], st["k_scale"]), (st["v"], st["v_scale"])):
            x = cache.view(torch.uint8)[at, :, row].view(cache.dtype).float() if scale is not None else cache[at, :, row].float()
            got.append((x if scale is None else x * scale[at][..., None]).transpose(1, 2))
        return got
    return _attend(st, fetch)


def _packed_plain(st):
    q_start = st["q_start"].long()

    def fetch(s, key):
        return [x[:, q_start[s][:, None] + key].transpose(0, 1) for x in (st["k"], st["v"])]
    return _attend(st, fetch, st["c"]["op"] == "train")


# ----------------------------------------------------------------------------------------------------------- a pass


def _run_own(st):
    import paper_2605_23445_amd as P
    c = st["c"]
    if c["op"] == "append":
        P.dfs_paged_append(st["g"], st["dt"], *st["x"], st["q_start"], st["k_len"], st["pos"], st["w_q"] if c["norm"] else None,
                           st["w_k"] if c["norm"] else None, st["q_out"], st["pages"], c["norm"])
        return _append_outputs(st)
    if c["op"] == "read":
        P.dfs_paged_attn_fwd(st["w"], st["dt"], st["q"], st["pages"], st["q_start"], st["k_len"], st["scale"], st["o"], st["lse"], st["ws"])
        return {"o": st["o"], "lse": st["lse"]}
    P.dfs_packed_attn_fwd(st["w"], st["dt"], st["q"], st["k"], st["v"], st["q_start"], None, st["scale"], st["o"], st["lse"], st["ws"])
    if c["op"] == "packed":
        return {"o": st["o"], "lse": st["lse"]}
    P.dfs_packed_attn_bwd(st["w"], st["dt"], st["q"], st["k"], st["v"], st["o"], st["lse"], st["do"], st["q_start"], None, st["scale"],
                          st["dq"], st["dk"], st["dv"], st["ws"])
    return {x: st[x] for x in ("o", "lse", "dq", "dk", "dv")}


def run(state):
    if own:
        return _run_own(state)
    return {"append": _append_plain, "read": _read_plain}.get(state["c"]["op"], _packed_plain)(state)


# ------------------------------------------------------------------------------------------------- work and exact values


def _pairs(c):
    """(pairs of a query and a key it sees, keys that some query sees) of one head, over the sequences."""
    pairs, keys, sinks = 0, 0, c.get("sinks", 0)
    for n, m in zip(*_lengths(c)):
        pos = torch.arange(m - n, m, dtype=torch.int64)
        lo = (pos - c["left"]).clamp(min=0) if c["left"] >= 0 else torch.zeros_like(pos)
        hi = (pos + c.get("right", 0)).clamp(max=m - 1) if c.get("right", 0) >= 0 else torch.full_like(pos, m - 1)
        pairs += int((hi - lo + 1 + lo.clamp(max=sinks)).sum())
        keys += int(hi[-1] - lo[0] + 1 + min(sinks, int(lo[0])))
    return pairs, keys


def work(case):
    c = _whole(case)
    size = {"bf16": 2.0, "f32": 4.0, "e4m3": 1.0}
    e, h, kv, d, t = size[c["dtype"]], c["heads"], c["heads_kv"], c["d"], c["tokens"]
    if c["op"] == "append":                                     # per element: square, sum, two products of the norm, three of the turn
        return {"bytes": t * d * ((2 * h + 2 * kv) * e + 2 * kv * size[c["cache"]]), "flops": 7.0 * d * t * (h + kv)}
    pairs, keys = _pairs(c)
    q = e * d * t * h
    if c["op"] == "read":
        return {"bytes": 2 * q + 4 * t * h + 2 * size[c["cache"]] * d * keys * kv, "flops": 4.0 * d * pairs * h}
    k = e * d * keys * kv
    if c["op"] == "packed":
        return {"bytes": 2 * q + 2 * k + 4 * t * h, "flops": 4.0 * d * pairs * h}
    return {"bytes": 4 * q + 4 * k + 4 * t * h, "flops": 14.0 * d * pairs * h}


def _exact_append(st):
    """From the definition, a sequence at a time: pairs as complex numbers, pages as the tokens that lie in them."""
    c, page, d = st["c"], st["c"]["page"], st["c"]["d"]
    order, freq, at = [], [], 0
    for axis, m in enumerate(_axes(c)):                          # channel order in which the pairs are neighbours
        order += [x for i in range(m // 2) for x in ((at + 2 * i, at + 2 * i + 1) if c["interleaved"] else (at + i, at + m // 2 + i))]
        freq += [(axis, c["theta"] ** (-2.0 * i / m)) for i in range(m // 2)]
        at += m
    back = sorted(range(d), key=lambda i: order[i])
    out = {"q": torch.empty(st["q_out"].shape, dtype=torch.float64, device=DEV), "k": st["k"].double(), "v": st["v"].double()}
    scales = {x: None if st[x + "_scale"] is None else st[x + "_scale"].double() for x in "kv"}
    table, a = st["table"].tolist(), 0
    for s, (n, total) in enumerate(zip(*st["lens"])):
        pos = torch.arange(total - n, total, device=DEV, dtype=torch.float64)[:, None] if st["pos"] is None else st["pos"][a:a + n].double()
        ang = torch.stack([pos[:, axis] * f for axis, f in freq], dim=-1)
        unit = torch.polar(torch.ones_like(ang), ang)

        def rows(x, w):
            y = x[:, a:a + n].double()
            if c["norm"]:
                y = y / torch.sqrt((y * y).sum(-1, keepdim=True) / d + EPS) * w.double()
            z = torch.view_as_complex(y[..., order].reshape(*y.shape[:2], d // 2, 2).contiguous()) * unit
            return torch.view_as_real(z).reshape(y.shape)[..., back]
        out["q"][:, a:a + n] = rows(st["x"][0], st["w_q"])
        for name, y in (("k", rows(st["x"][1], st["w_k"])), ("v", st["x"][2][:, a:a + n].double())):
            cache, scale = out[name], scales[name]
            for j in range((total - n) // page, (total - 1) // page + 1):
                lo, hi, to = max(total - n, j * page), min(total, (j + 1) * page), table[s][j]
                part, old = y[:, lo - (total - n):hi - (total - n)], max(0, lo - j * page)
                if scale is not None:
                    need = torch.exp2(torch.ceil(torch.log2(part.abs().amax((1, 2)) / 448)).clamp(min=LEAST))
                    if old:
                        need = torch.maximum(need, scale[to])
                        cache[to, :, :old] *= (scale[to] / need)[:, None, None]
                    scale[to] = need
                    part = part / need[:, None, None]
                cache[to, :, old:old + hi - lo] = part
        a += n
    return out if scales["k"] is None else dict(out, k_scale=scales["k"], v_scale=scales["v"])


def _exact_attend(st):
    """From the definition, a sequence and a key head at a time, in blocks of rows over the span of keys that they see."""
    c, q = st["c"], st["q"]
    group, train, left, right, sinks = c["heads"] // c["heads_kv"], c["op"] == "train", c["left"], c.get("right", 0), c.get("sinks", 0)
    f64 = dict(dtype=torch.float64, device=DEV)
    res = {"o": torch.zeros(q.shape, **f64), "lse": torch.zeros(q.shape[:2], **f64)}
    if train:
        res.update({x: torch.zeros(st[x[1]].shape, **f64) for x in ("dq", "dk", "dv")})
    a = 0
    for s, (n, m) in enumerate(zip(*st["lens"])):
        if c["op"] == "read":
            own_pages = st["table"][s, :(m + c["page"] - 1) // c["page"]].long()
        for j in range(c["heads_kv"]):
            hs = slice(j * group, (j + 1) * group)
            if c["op"] == "read":
                kk, vv = (_rows_of(st, x, own_pages, j)[:m] for x in "kv")
            else:
                kk, vv = (st[x][j, a:a + n].double() for x in "kv")
            for r in range(0, n, 1024):
                z = min(n, r + 1024)
                pos = torch.arange(m - n + r, m - n + z, device=DEV)
                lo = 0 if left < 0 else max(0, m - n + r - left)
                hi = m if right < 0 else min(m, m - n + z + right)
                at = torch.cat([torch.arange(min(sinks, lo), device=DEV), torch.arange(lo, hi, device=DEV)])
                see = torch.ones(z - r, len(at), dtype=torch.bool, device=DEV)
                if right >= 0:
                    see &= at <= pos[:, None] + right
                if left >= 0:
                    see &= (at >= pos[:, None] - left) | (at < sinks)
                x = q[hs, a + r:a + z].double()
                t = torch.where(see, x @ kk[at].t() * st["scale"], torch.tensor(-math.inf, **f64))
                lse = torch.logsumexp(t, -1, keepdim=True)
                p = torch.exp(t - lse)
                y = p @ vv[at]
                res["o"][hs, a + r:a + z], res["lse"][hs, a + r:a + z] = y, lse[..., 0]
                if train:
                    g = st["do"][hs, a + r:a + z].double()
                    ds = p * (g @ vv[at].t() - (g * y).sum(-1, keepdim=True)) * st["scale"]
                    res["dq"][hs, a + r:a + z] = ds @ kk[at]
                    res["dk"][j, a:a + n].index_add_(0, at, (ds.transpose(1, 2) @ x).sum(0))
                    res["dv"][j, a:a + n].index_add_(0, at, (p.transpose(1, 2) @ g).sum(0))
        a += n
    return res


def _rows_of(st, x, pages, head):
    """[tokens, d] of a sequence's pages, as the values they stand for."""
    rows, scale = st[x].view(torch.uint8)[pages, head].view(st[x].dtype).double(), st[x + "_scale"]
    return (rows if scale is None else rows * scale[pages, head].double()[:, None, None]).flatten(0, 1)


def exact(case, seed):
    c = _whole(case)
    st = prepare(case, seed)
    return _exact_append(st) if c["op"] == "append" else _exact_attend(st)
