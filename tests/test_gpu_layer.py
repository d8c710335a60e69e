"""Norm, rotation and attention as they are used together: a layer from its fused projection to the gradient of that, a stream of tokens over a
cache against the whole sequence at once, the sparse path behind the rotation; on other streams, captured and replayed, from plain and
other arguments."""
import numpy as np
import pytest
import torch

pytestmark = pytest.mark.gpu

P = pytest.importorskip("paper_2605_23445_amd")
from oracle import dfs_oracle as O, layer_oracle as L  # noqa: E402
from paper_2605_23445_amd import _calls  # noqa: E402
from tests import gpu_util as G  # noqa: E402

DT = {"f32": (P.DFS_F32, torch.float32), "bf16": (P.DFS_BF16, torch.bfloat16)}


class Layer:
    """One attention layer of `batch` padded sequences: fused projection in, output and gradient of the projection out."""

    def __init__(self, dtype, batch=2, n=150, heads=6, kv=2, d=64, left=40, right=0, sinks=3, lens=None, seed=0):
        self.code, self.dt = DT[dtype]
        self.shape, self.scale, self.lens = (batch, n, heads, kv, d), d ** -0.5, lens
        self.g = P.QkGeom(batch, n, heads, kv, d, 0, 1, d, 0, 0, 1e4, 1e-6)
        self.w = P.Window(batch, heads, kv, d, n, n, left, right, sinks)
        gen = torch.Generator(device="cuda").manual_seed(seed)
        self.fused = torch.randn(batch, n, (heads + 2 * kv) * d, generator=gen, device="cuda").to(self.dt)
        self.w_q, self.w_k = (1 + 0.2 * torch.randn(d, generator=gen, device="cuda") for _ in range(2))
        self.pos = torch.arange(n, dtype=torch.int32, device="cuda")[:, None].contiguous()
        self.len = None if lens is None else torch.tensor(lens, dtype=torch.int32, device="cuda")
        new = lambda *s: torch.zeros(*s, dtype=self.dt, device="cuda")  # noqa: E731
        self.qkv, self.dqkv = ([new(batch, h, n, d) for h in (heads, kv, kv)] for _ in range(2))
        # the output and its gradient as the projection behind it has them: token-major
        self.o, self.d_o = (new(batch, n, heads, d).transpose(1, 2) for _ in range(2))
        self.d_o.copy_(torch.randn(batch, heads, n, d, generator=gen, device="cuda"))
        self.lse, self.grad = torch.zeros(batch, heads, n, device="cuda"), torch.zeros_like(self.fused)
        self.dw = [torch.zeros(d, device="cuda") for _ in range(2)]
        ws = max(P.dfs_qk_workspace_bytes(self.g), *(P.dfs_window_workspace_bytes(self.w, self.code, x) for x in (False, True)))
        self.ws = torch.empty(ws, dtype=torch.uint8, device="cuda")

    def parts(self, x):
        b, n, h, kv, d = self.shape
        cut = lambda a, m: x[..., a * d:(a + m) * d].view(b, n, m, d).transpose(1, 2)  # noqa: E731
        return cut(0, h), cut(h, kv), cut(h + kv, kv)

    def step(self):
        P.dfs_qk_norm_rope(self.g, self.code, *self.parts(self.fused), self.pos, self.w_q, self.w_k, *self.qkv)
        P.dfs_window_attn_fwd(self.w, self.code, *self.qkv, self.len, self.len, self.scale, self.o, self.lse, self.ws)
        P.dfs_window_attn_bwd(self.w, self.code, *self.qkv, self.o, self.lse, self.d_o, self.len, self.len, self.scale, *self.dqkv, self.ws)
        P.dfs_qk_norm_rope_bwd(self.g, self.code, *self.parts(self.fused)[:2], self.pos, self.w_q, self.w_k, *self.dqkv, *self.parts(self.grad), *self.dw, self.ws)

    def results(self):
        return [x.clone() for x in (self.o, self.lse, self.grad, *self.dw)]


def _np(t):
    return t.double().cpu().numpy()


def test_layer_and_its_gradient_against_the_oracle():
    """fp32, padded sequences.  Bound: each of the two stages is good to some 1e-6 of its operands' size (test_gpu_rope, test_gpu_window), a weight moves by
    the logit's error, which the rows' lengths (sqrt d) magnify by at most 8: 1e-4 of the largest value is far above all of these together."""
    la = Layer("f32", lens=[150, 71])
    la.step()
    b, n, h, kv, d = la.shape
    q, k, v = (_np(x) for x in la.parts(la.fused))
    gq, gk, gv = (_np(x) for x in la.parts(la.grad))
    o, d_o, w_q, w_k = (_np(x) for x in (la.o, la.d_o, la.w_q, la.w_k))
    dw = [np.zeros(d), np.zeros(d)]
    near = lambda got, want: np.testing.assert_allclose(got, want, atol=1e-4 * np.abs(want).max(), rtol=0)  # noqa: E731
    for i, m in enumerate(la.lens):
        pos = np.arange(m)[:, None]
        see = L.window_mask(m, m, la.w.left, la.w.right, la.w.sinks)
        rope = lambda x, w: L.qk_norm_rope(x, pos, (d,), 1e4, False, w, 1e-6)  # noqa: E731
        back = lambda x, up, w: L.qk_norm_rope_bwd(x, up, pos, (d,), 1e4, False, w, 1e-6)  # noqa: E731
        for j in range(kv):
            kk = rope(k[i, j, :m], w_k)
            dk, dv = np.zeros((m, d)), np.zeros((m, d))
            for x in range(j * h // kv, (j + 1) * h // kv):
                qq = rope(q[i, x, :m], w_q)
                near(o[i, x, :m], L.window_attn(qq, kk, v[i, j, :m], see, la.scale)[0])
                dq, a, c = L.window_attn_bwd(qq, kk, v[i, j, :m], see, la.scale, d_o[i, x, :m])
                dk, dv = dk + a, dv + c
                dx, s = back(q[i, x, :m], dq, w_q)
                near(gq[i, x, :m], dx)
                dw[0] += s
            dx, s = back(k[i, j, :m], dk, w_k)
            near(gk[i, j, :m], dx)
            near(gv[i, j, :m], dv)
            dw[1] += s
        assert not gq[i, :, m:].any() and not gk[i, :, m:].any() and not gv[i, :, m:].any()       # nothing flows into padding
    near(_np(la.dw[0]), dw[0])
    near(_np(la.dw[1]), dw[1])


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
def test_tokens_one_by_one_over_a_cache_give_what_the_whole_sequence_gives(dtype):
    """Two sequences that start with prompts of 50 and 9 tokens and go on token by token.  Rows differ by the order of their sums alone: fp32 1e-5 of the values'
    size; in bf16 each weight is rounded on its own, by up to 2^-8, on both sides, and so is the row."""
    la = Layer(dtype, n=130, lens=[130, 130])
    la.step()
    b, n, h, kv, d = la.shape
    code, dt = la.code, la.dt
    cache = [torch.full((b, n, kv, d), float("nan"), dtype=dt, device="cuda").transpose(1, 2) for _ in range(2)]
    q_fused, k_fused, v_fused = la.parts(la.fused)
    first = [50, 9]
    tol = (1e-5 if dtype == "f32" else 4 * 2.0 ** -8) * float(la.qkv[2].float().abs().max())
    ws = torch.empty(1 << 22, dtype=torch.uint8, device="cuda")

    def run(rows, start):
        """`rows` tokens of each sequence from start[b] on (start on the device); returns what attention gives for them."""
        at = start.long()[:, None] + torch.arange(rows, device="cuda")
        take = lambda x: x.transpose(1, 2)[torch.arange(b, device="cuda")[:, None], at].transpose(1, 2)  # noqa: E731
        g = P.QkGeom(b, rows, h, kv, d, 0, 1, d, 0, 0, 1e4, 1e-6)
        w = P.Window(b, h, kv, d, rows, n, la.w.left, 0, la.w.sinks)
        q = torch.empty(b, h, rows, d, dtype=dt, device="cuda")
        P.dfs_qk_norm_rope(g, code, take(q_fused), take(k_fused), take(v_fused), at.int()[..., None].contiguous(), la.w_q, la.w_k, q, *cache, start)
        o = torch.empty_like(q)
        assert P.dfs_window_workspace_bytes(w, code, False) <= ws.numel()
        P.dfs_window_attn_fwd(w, code, q, *cache, None, (start + rows).int(), la.scale, o, None, ws)
        return o, at

    # prompts: as many tokens as the shorter one has, then the rest of the longer one along with new ones of the other
    start = torch.zeros(b, dtype=torch.int32, device="cuda")
    for rows in [min(first), 5, 1, 1, 32, 1, 1, 1, 40, 1]:
        o, at = run(rows, start)
        want = la.o.transpose(1, 2)[torch.arange(b, device="cuda")[:, None], at].transpose(1, 2)
        assert float((o.float() - want.float()).abs().max()) <= tol
        start += rows
    assert torch.equal(cache[0][:, :, :92], la.qkv[1][:, :, :92]) and torch.isnan(cache[0][:, :, 92:].float()).all()


def test_sparse_path_behind_the_rotation():
    """A fused projection of a video grid with text through norm and rotation into dfs_forward, against the oracle on the same tensors."""
    T, H, W, text, heads, d = 3, 7, 9, 21, 2, 64
    geo = P.Geom(T, H, W, text, heads, d, 64, 16)
    s = P.dfs_geom_sizes(geo)
    gen = torch.Generator(device="cuda").manual_seed(3)
    fused = torch.randn(1, s.N, 3 * heads * d, generator=gen, device="cuda")
    cut = lambda i: fused[..., i * heads * d:(i + 1) * heads * d].view(1, s.N, heads, d).transpose(1, 2)  # noqa: E731
    grid = np.stack(np.meshgrid(np.arange(T), np.arange(H), np.arange(W), indexing="ij"), -1).reshape(-1, 3)
    pos = np.concatenate([grid, np.zeros((text, 3), int)])
    w = 1 + 0.2 * torch.randn(2, d, generator=gen, device="cuda")
    q, k, v = (torch.empty(heads, s.N, d, device="cuda") for _ in range(3))
    g = P.QkGeom(1, s.N, heads, heads, d, 1, 3, 16, 24, 24, 1e4, 1e-6)
    P.dfs_qk_norm_rope(g, P.DFS_F32, cut(0), cut(1), cut(2), torch.from_numpy(pos).int().cuda(), w[0], w[1], q[None], k[None], v[None])
    perm_pad, inv, valid = G.gpu_perm(geo)
    st = P.MaskState(torch.zeros((heads, s.M, s.M), dtype=torch.int32, device="cuda"), torch.zeros((heads, s.M), dtype=torch.int32, device="cuda"),
                     torch.zeros((heads, s.M, s.M), dtype=torch.uint8, device="cuda"), None, s.M)
    o = torch.empty_like(q)
    ws = G.ws_tensor(P.dfs_workspace_bytes(geo, P.DFS_WS_FORWARD))
    P.dfs_forward(geo, P.DFS_F32, q, k, v, perm_pad, inv, True, P.DFS_SELECT_TOPK, 0.5, 0.0, st, d ** -0.5, o, ws)
    perm = perm_pad.cpu().numpy()
    x = [np.stack([L.qk_norm_rope(_np(cut(i))[0, h], pos, (16, 24, 24), 1e4, True, _np(w[i]), 1e-6) for h in range(heads)]) for i in range(2)]
    qp, kp, vp = (O.permute(y, perm) for y in (*x, _np(cut(2))[0]))
    want, _ = O.sparse_attn(qp, kp, vp, st.mask.cpu().numpy(), valid.cpu().numpy(), 64)
    assert np.abs(_np(o) - O.unpermute(want, inv.cpu().numpy())).max() <= 1e-4


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
def test_captured_step_replays_on_new_inputs(dtype):
    la, other = Layer(dtype, lens=[150, 33]), Layer(dtype, lens=[80, 150], seed=9)
    la.step()
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        la.step()
    gen = torch.Generator(device="cuda").manual_seed(4)
    for i in range(4):
        la.fused.copy_(torch.randn(la.fused.shape, generator=gen, device="cuda"))
        la.len.copy_(torch.tensor([[150, 33], [1, 150], [0, 149], [64, 128]][i], dtype=torch.int32))
        for x in (la.o, la.lse, la.grad, *la.dw, *la.dqkv):
            x.zero_()
        la.step()
        want = la.results()
        for x in (la.o, la.lse, la.grad, *la.dw, *la.dqkv):
            x.zero_()
        la.ws.fill_(255)
        graph.replay()
        other.step()                                                       # the program's own work in between
        torch.cuda.synchronize()
        assert all(torch.equal(a, c) for a, c in zip(la.results(), want)), i


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
def test_two_streams_at_once(dtype):
    layers = [Layer(dtype, lens=[150, 33]), Layer(dtype, n=210, left=-1, sinks=0, seed=1)]
    want = []
    for la in layers:
        la.step()
        want.append(la.results())
    streams = [torch.cuda.Stream() for _ in layers]
    torch.cuda.synchronize()
    for _ in range(5):
        for la, st in zip(layers, streams):
            with torch.cuda.stream(st):
                la.step()
    torch.cuda.synchronize()
    for la, w in zip(layers, want):
        assert all(torch.equal(a, c) for a, c in zip(la.results(), w))


class _Tensor(torch.Tensor):
    pass


def test_plain_arguments_do_not_go_through_python_and_others_give_the_same():
    la = Layer("bf16", lens=[150, 33])
    la.step()
    want = la.results()
    q, k, v = la.parts(la.fused)
    rope = [la.g, la.code, q, k, v, la.pos, la.w_q, la.w_k, *la.qkv, None]
    fwd = [la.w, la.code, *la.qkv, la.len, la.len, la.scale, la.o, la.lse, la.ws]
    bwd = [la.w, la.code, *la.qkv, la.o, la.lse, la.d_o, la.len, la.len, la.scale, *la.dqkv, la.ws]
    rope_bwd = [la.g, la.code, q, k, la.pos, la.w_q, la.w_k, *la.dqkv, *la.parts(la.grad), *la.dw, la.ws]
    for name, args in (("qk_norm_rope", rope), ("window_attn_fwd", fwd), ("window_attn_bwd", bwd), ("qk_norm_rope_bwd", rope_bwd)):
        assert getattr(_calls, name)(*args) == 0, name
    assert all(torch.equal(a, c) for a, c in zip(la.results(), want))
    for x in (la.o, la.lse, la.grad, *la.dw, *la.dqkv, *la.qkv):
        x.zero_()
    P.dfs_qk_norm_rope(la.g, np.int64(la.code), q.as_subclass(_Tensor), k, v, torch.nn.Parameter(la.pos, requires_grad=False), la.w_q, la.w_k, *la.qkv)
    P.dfs_window_attn_fwd(la.w, np.int32(la.code), *la.qkv, la.len, la.len, np.float64(la.scale), la.o.as_subclass(_Tensor), la.lse, la.ws)
    P.dfs_window_attn_bwd(la.w, np.int32(la.code), *la.qkv, la.o, la.lse, la.d_o, la.len, la.len, np.float32(la.scale), *la.dqkv, la.ws.as_subclass(_Tensor))
    P.dfs_qk_norm_rope_bwd(la.g, np.int64(la.code), q, k, la.pos, la.w_q, la.w_k, *la.dqkv, *la.parts(la.grad), *(x.as_subclass(_Tensor) for x in la.dw), la.ws)
    assert all(torch.equal(a, c) for a, c in zip(la.results(), want))


def test_workspaces_that_are_too_small_are_refused():
    la = Layer("bf16", n=20, lens=[20, 20])
    small = torch.empty(64, dtype=torch.uint8, device="cuda")
    for call, args in ((P.dfs_qk_norm_rope_bwd, [la.g, la.code, *la.parts(la.fused)[:2], la.pos, None, None, *la.dqkv, *la.parts(la.grad), *la.dw]),
                       (P.dfs_window_attn_bwd, [la.w, la.code, *la.qkv, la.o, la.lse, la.d_o, None, None, 0.1, *la.dqkv])):
        for ws in (None, small, torch.empty(1 << 22, dtype=torch.uint8, device="cuda")[16:]):
            with pytest.raises(P.DfsError) as e:
                call(*args, ws)
            assert e.value.code == -4
