"""The MLP half of a decoder layer on 8-bit operands, as the operators are used together: residual and RMSNorm to 8 bits, the
gate/up product with scales and a bias, the activation to 8 bits, the down product onto the residual stream; with a scale per row
and microscaled; alone, in batches, in a HIP graph, and with the down product split over tensor-parallel shards."""
import pytest
import torch

import eight_bit_reference as ref
from paper_2511_17826_amd import binding as tb

pytestmark = pytest.mark.gpu
H, I, LEAF = 1024, 2048, 128
EPS = 1e-6


def rnd(seed, *shape):
    return torch.randn(shape, generator=torch.Generator(device="cuda").manual_seed(seed), device="cuda")


class Layer:
    def __init__(self, micro, dtype):
        self.micro, self.dtype = micro, dtype
        self.norm1, self.norm2 = (1 + 0.1 * rnd(1, H)).to(dtype), (1 + 0.1 * rnd(2, H)).to(dtype)
        self.w_gu, self.w_down = 0.03 * rnd(3, 2 * I, H), 0.03 * rnd(4, H, I)
        self.b_gu = 0.1 * rnd(5, 2 * I)
        quantise = ref.micro_scaled if micro else ref.row_scaled
        self.q_gu, self.s_gu = (torch.from_numpy(t).cuda() for t in quantise(self.w_gu.cpu().numpy(), "e4m3"))
        self.q_down, self.s_down = (torch.from_numpy(t).cuda() for t in quantise(self.w_down.cpu().numpy(), "e4m3"))

    def first(self, x, r):
        return (tb.tbik_rmsnorm_mxfp8 if self.micro else tb.tbik_rmsnorm_fp8)(x, self.norm1, EPS, residual=r)

    def gate_up(self, q, s):
        if self.micro:
            return tb.tbik_gemm_mxfp8_epilogue(q, s, self.q_gu, self.s_gu, LEAF, 1, bias=self.b_gu, out_dtype=self.dtype)
        return tb.tbik_gemm_fp8_epilogue(q, self.q_gu, LEAF, 1, row_scale=s, col_scale=self.s_gu, bias=self.b_gu, out_dtype=self.dtype)

    def act(self, gu):
        return (tb.tbik_silu_mul_mxfp8 if self.micro else tb.tbik_silu_mul_fp8)(gu[:, :I], gu[:, I:])

    def down(self, q, s, hidden):
        if self.micro:
            return tb.tbik_gemm_mxfp8_epilogue(q, s, self.q_down, self.s_down, LEAF, 1, residual=hidden, out_dtype=self.dtype)
        return tb.tbik_gemm_fp8_epilogue(q, self.q_down, LEAF, 1, row_scale=s, col_scale=self.s_down, residual=hidden, out_dtype=self.dtype)

    def __call__(self, x, r):
        hidden, q, s = self.first(x, r)
        return self.down(*self.act(self.gate_up(q, s)), hidden)

    def exact(self, x, r):
        """In 64 bits without any 8-bit rounding."""
        hidden = x.double() + r.double()
        n = hidden / torch.sqrt((hidden ** 2).mean(dim=1, keepdim=True) + EPS) * self.norm1.double()
        gu = n @ self.w_gu.double().t() + self.b_gu.double()
        return (gu[:, :I] * torch.sigmoid(gu[:, :I]) * gu[:, I:]) @ self.w_down.double().t() + hidden, hidden


MODES = [(False, torch.bfloat16), (True, torch.bfloat16), (False, torch.float16), (True, torch.float16)]


@pytest.mark.parametrize("micro,dtype", MODES)
def test_layer(micro, dtype):
    """Against the layer without quantisation: an 8-bit rounding is off by at most 2^-4 of a value, in the mean of squares by about
    0.026 of it, so that a product of two rounded operands is about 0.037 off in norm; through the activation (whose two factors
    carry it) and the second product 0.07 .. 0.09 of the MLP's output.  Twice that is the bar.  Rows alone: the same bits."""
    layer = Layer(micro, dtype)
    x, r = rnd(6, 300, H).to(dtype), rnd(7, 300, H).to(dtype)
    y = layer(x, r)
    want, hidden = layer.exact(x, r)
    assert float((y.double() - want).norm() / (want - hidden).norm()) < 0.18
    for rows in ([0], [299, 17], list(range(40, 140))):
        assert torch.equal(layer(x[rows].contiguous(), r[rows].contiguous()), y[rows])


@pytest.mark.parametrize("micro", [False, True])
@pytest.mark.parametrize("P", [2, 8])
def test_shards(micro, P):
    """The down product over P shards: its sum with the epilogue is the whole one's; microscaled, the shards' sums also go straight
    into the next block's norm."""
    layer = Layer(micro, torch.bfloat16)
    x, r = rnd(8, 77, H).bfloat16(), rnd(9, 77, H).bfloat16()
    hidden, q, s = layer.first(x, r)
    q2, s2 = layer.act(layer.gate_up(q, s))
    whole = layer.down(q2, s2, hidden)
    if micro:
        parts = tb.tbik_gemm_shard_partials_mxfp8(q2, s2, layer.q_down, layer.s_down, LEAF, 1, P)
        assert torch.equal(tb.tbik_tree_combine_epilogue(parts, residual=hidden), whole)
        product = tb.tbik_gemm_mxfp8(q2, s2, layer.q_down, layer.s_down, LEAF, 1)
        a, b = tb.tbik_combine_residual_rmsnorm_mxfp8(parts, hidden, layer.norm2, EPS), tb.tbik_rmsnorm_mxfp8(product, layer.norm2, EPS, residual=hidden)
        assert all(torch.equal(u, v) for u, v in zip(a, b))
    else:
        parts = tb.tbik_gemm_shard_partials_fp8(q2, layer.q_down, LEAF, 1, P)
        assert torch.equal(tb.tbik_tree_combine_epilogue(parts, row_scale=s2, col_scale=layer.s_down, residual=hidden), whole)


@pytest.mark.parametrize("M", [1, 200])
@pytest.mark.parametrize("micro,dtype", MODES[:2])
def test_layer_in_a_hip_graph(micro, dtype, M):
    """Captured once, replayed with new inputs in place, eager work on the same stream's workspaces between the replays."""
    layer = Layer(micro, dtype)
    x, r = rnd(10, M, H).to(dtype), rnd(11, M, H).to(dtype)
    layer(x, r)
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        layer(x, r)                                       # the stream's workspace, before the capture
        side.synchronize()
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph, stream=side):
            out = layer(x, r)
    for rep in range(4):
        x.copy_(rnd(20 + rep, M, H).to(dtype))
        r.copy_(rnd(30 + rep, M, H).to(dtype))
        torch.cuda.synchronize()
        graph.replay()
        torch.cuda.synchronize()
        got = out.clone()
        assert torch.equal(got, layer(x, r)), rep
        torch.cuda.synchronize()


def test_two_layers_on_two_streams():
    """Two captured layers replayed at once, each with the workspace of its own stream."""
    layers, graphs, outs, wants = [], [], [], []
    for i in range(2):
        layer = Layer(bool(i), torch.bfloat16)
        x, r = rnd(40 + i, 64, H).bfloat16(), rnd(50 + i, 64, H).bfloat16()
        wants.append(layer(x, r))
        s = torch.cuda.Stream()
        s.wait_stream(torch.cuda.current_stream())
        with torch.cuda.stream(s):
            layer(x, r)
            s.synchronize()
            g = torch.cuda.CUDAGraph()
            with torch.cuda.graph(g, stream=s):
                outs.append(layer(x, r))
        layers.append((layer, x, r, s))
        graphs.append(g)
    torch.cuda.synchronize()
    for _ in range(3):
        for g, (_, _, _, s) in zip(graphs, layers):
            with torch.cuda.stream(s):
                g.replay()
        torch.cuda.synchronize()
        assert all(torch.equal(o, w) for o, w in zip(outs, wants))


@pytest.mark.parametrize("M", [1, 150, 1000])
def test_shards_and_16_bit_products_in_a_hip_graph(M):
    """The other entry points, into buffers of the caller's, with one workspace that two captured graphs share (replayed one after the
    other): products with an epilogue that split K and that do not, a residual updated in place, shards' sums to 8 bits."""
    K, N, P, leaf = 4096, 1024, 4, 256
    X, W = rnd(60, M, K).bfloat16(), (0.02 * rnd(61, K, N)).bfloat16()
    bias, w = rnd(62, N), (1 + 0.1 * rnd(63, N)).bfloat16()
    need = max(tb.gemm_16bit_workspace_bytes(M, N, K, leaf, 1), 256)
    workspace = torch.empty(need, dtype=torch.uint8, device="cuda")

    def buffers():
        e = lambda *s, t=torch.uint8: torch.empty(s, dtype=t, device="cuda")
        return dict(stream=e(M, N, t=torch.bfloat16), parts=e(P, M, N, t=torch.float32), hidden=e(M, N, t=torch.bfloat16), combined=e(M, N, t=torch.float16),
                    q=e(M, N), s=e(M, t=torch.float32), q2=e(M, N), s2=e(M, N // 32), hidden2=e(M, N, t=torch.bfloat16))

    def one_pass(b, r):
        b["stream"].copy_(r)
        tb.tbik_gemm_epilogue(X, W, leaf, 1, bias=bias, activation="gelu_tanh", residual=b["stream"], out=b["stream"], workspace=workspace)
        tb.tbik_gemm_shard_partials(X, W, leaf, 1, P, out=b["parts"], workspace=workspace)
        tb.tbik_tree_combine_epilogue(b["parts"], bias=bias, activation="silu", out=b["combined"])
        tb.tbik_combine_residual_rmsnorm_fp8(b["parts"], b["stream"], w, EPS, hidden=b["hidden"], out=b["q"], scale=b["s"])
        tb.tbik_combine_residual_rmsnorm_mxfp8(b["parts"], b["stream"], w, EPS, fmt="e5m2", hidden=b["hidden2"], out=b["q2"], scale=b["s2"])

    r = [rnd(64 + i, M, N).bfloat16() for i in range(2)]
    eager, captured = buffers(), [buffers(), buffers()]
    one_pass(eager, r[0])
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    graphs = []
    with torch.cuda.stream(side):
        for b, x in zip(captured, r):
            g = torch.cuda.CUDAGraph()
            with torch.cuda.graph(g, stream=side):
                one_pass(b, x)
            graphs.append(g)
    for rep in range(3):
        X.copy_(rnd(80 + rep, M, K).bfloat16())
        for i in range(2):
            for t in captured[i].values():
                t.zero_()
        workspace.fill_(0xFF)
        torch.cuda.synchronize()
        for g in graphs:
            g.replay()
        torch.cuda.synchronize()
        for b, x in zip(captured, r):
            one_pass(eager, x)
            torch.cuda.synchronize()
            assert all(torch.equal(b[k].view(torch.uint8), eager[k].view(torch.uint8)) for k in b), rep
