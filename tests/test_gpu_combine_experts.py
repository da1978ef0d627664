"""tbik_combine_experts against its definition in 64 bits, and the layer's path for any number of shards."""
import pytest
import torch

from paper_2511_17826_amd import binding as tb

pytestmark = pytest.mark.gpu
DEV = "cuda:0"
bits = lambda t: t.contiguous().view(torch.int32 if t.dtype == torch.float32 else torch.int16)


def inputs(T, k, R, H, dtype, seed, P=0):
    g = torch.Generator(device=DEV).manual_seed(seed)
    Y = torch.randn((P, R, H) if P else (R, H), generator=g, device=DEV).to(torch.float32 if P else dtype)
    slots = torch.randint(0, R, (T, k), generator=g, device=DEV, dtype=torch.int32)
    weights = torch.softmax(torch.randn((T, k), generator=g, device=DEV), dim=1)
    residual = torch.randn((T, H), generator=g, device=DEV).to(dtype)
    return Y, slots, weights, residual


def check(out, Y, slots, weights, residual):
    P = Y.shape[0] if Y.dim() == 3 else 0
    y = Y.double().sum(0) if P else Y.double()
    valid = (slots >= 0) & (slots < y.shape[0])
    terms = torch.where(valid, weights, torch.zeros_like(weights)).double()[:, :, None] * y[slots.clamp(0, y.shape[0] - 1).long()]
    want = terms.sum(1)
    size = terms.abs().sum(1)
    if P:                                                            # each of log2(P) additions of a row's shards rounds a sum of at most their magnitudes
        size = (weights.double().abs()[:, :, None] * Y.double().abs().sum(0)[slots.clamp(0, y.shape[0] - 1).long()]).sum(1)
    k = slots.shape[1]
    if residual is not None:
        want, size = want + residual.double(), size + residual.double().abs()
    # k fused steps, the tree over the shards, one addition, each half a step of at most `size`; then the output's rounding.
    tol = size * 2.0 ** -24 * (k + 1 + max(P, 1).bit_length()) * 1.01 + want.abs() * (torch.finfo(out.dtype).eps / 2 if out.dtype != torch.float32 else 0) * 1.01 + 2.0 ** -24 * (out.dtype == torch.float16)
    assert ((out.double() - want).abs() <= tol).all()


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float16])
@pytest.mark.parametrize("T,k,H", [(1, 1, 8), (1, 8, 4096), (3, 2, 5120), (77, 8, 2048), (5, 9, 136), (2, 32, 1000), (4, 3, 7), (9, 17, 2056)])
@pytest.mark.parametrize("with_residual", [False, True])
def test_16_bit_rows(T, k, H, dtype, with_residual):
    Y, slots, weights, residual = inputs(T, k, T * k, H, dtype, T + k + H)
    residual = residual if with_residual else None
    out = tb.tbik_combine_experts(Y, slots, weights, residual=residual)
    assert out.dtype == dtype
    check(out, Y, slots, weights, residual)
    wide = tb.tbik_combine_experts(Y, slots, weights, residual=residual.float() if with_residual else None, out_dtype=torch.float32)
    check(wide, Y, slots, weights, residual)
    assert torch.equal(bits(wide.to(dtype)), bits(out))              # one rounding


@pytest.mark.parametrize("P", [1, 2, 4, 8, 16])
@pytest.mark.parametrize("H", [4096, 200, 9])
def test_shards_sums(P, H):
    Y, slots, weights, residual = inputs(6, 5, 30, H, torch.bfloat16, P + H, P)
    out = tb.tbik_combine_experts(Y, slots, weights, residual=residual)
    check(out, Y, slots, weights, residual)
    whole = tb.tbik_tree_combine(Y, out_dtype=torch.float32)
    assert torch.equal(bits(out), bits(tb.tbik_combine_experts(whole, slots, weights, residual=residual)))
    half = tb.tbik_combine_experts(Y, slots, weights, out_dtype=torch.float16)
    check(half, Y, slots, weights, None)


def test_dropped_choices_and_a_token_without_any():
    Y, slots, weights, residual = inputs(5, 4, 20, 64, torch.bfloat16, 1)
    slots[0, 1], slots[1, 3], slots[2] = -1, 20, -1
    Y[7] = float("nan")
    slots[slots == 7] = 8                                            # nobody's row
    out = tb.tbik_combine_experts(Y, slots, weights, residual=residual)
    Y[7] = 0
    check(out, Y, slots, weights, residual)
    assert torch.equal(bits(out[2]), bits(residual[2]))
    empty = tb.tbik_combine_experts(Y[:0], slots, weights, residual=residual)
    assert torch.equal(bits(empty), bits(residual))


def test_strides_and_the_residual_in_place():
    Y, slots, weights, residual = inputs(33, 6, 100, 520, torch.float16, 2)
    want = tb.tbik_combine_experts(Y, slots, weights, residual=residual)
    Yw = torch.zeros((100, 601), dtype=torch.float16, device=DEV)
    Yw[:, 33:553] = Y
    wide = torch.full((33, 777), 7.0, dtype=torch.float16, device=DEV)
    tb.tbik_combine_experts(Yw[:, 33:553], slots, weights, residual=residual, out=wide[:, 1:521])
    assert torch.equal(bits(wide[:, 1:521]), bits(want)) and (wide[:, 0] == 7).all() and (wide[:, 521:] == 7).all()
    wide[:, 1:521] = residual
    tb.tbik_combine_experts(Y, slots, weights, residual=wide[:, 1:521], out=wide[:, 1:521])
    assert torch.equal(bits(wide[:, 1:521]), bits(want))
    own = residual.clone()
    assert tb.tbik_combine_experts(Y, slots, weights, residual=own, out=own) is own and torch.equal(bits(own), bits(want))


def test_more_tokens_than_a_launch():
    Y, slots, weights, _ = inputs(16384 * 2 + 3, 1, 50, 8, torch.bfloat16, 3)
    check(tb.tbik_combine_experts(Y, slots, weights), Y, slots, weights, None)


def test_rows_of_millions_of_columns_are_several_launches():
    """Element by element: a grid has fewer than 2^32 threads.  One choice of weight 1: the chosen row itself."""
    T, H = 2050, (1 << 21) + 1
    Y = torch.randn((3, H), generator=torch.Generator(device=DEV).manual_seed(6), device=DEV).to(torch.bfloat16)
    slots = (torch.arange(T, device=DEV, dtype=torch.int32) * 7 % 3).reshape(T, 1)
    out = torch.full((T, H), 9.0, dtype=torch.bfloat16, device=DEV)
    tb.tbik_combine_experts(Y, slots, torch.ones((T, 1), device=DEV), out=out)
    for t in range(0, T, 205):
        assert torch.equal(out[t:t + 205], Y[slots[t:t + 205, 0].long()])
    assert torch.equal(out[-1], Y[slots[-1, 0].long()])


def test_refusals():
    Y, slots, weights, residual = inputs(5, 4, 20, 64, torch.bfloat16, 4)
    for kw in (dict(slots=slots.long()), dict(weights=weights.half()), dict(weights=weights[:, :3]), dict(residual=residual.float(), out_dtype=torch.bfloat16), dict(residual=residual[:4]),
               dict(slots=slots.cpu()), dict(out=torch.empty((5, 65), dtype=torch.bfloat16, device=DEV))):
        with pytest.raises(ValueError):
            tb.tbik_combine_experts(**{**dict(Y=Y, slots=slots, weights=weights, residual=residual), **kw})
    with pytest.raises(TypeError):
        tb.tbik_combine_experts(Y[None], slots, weights)
    with pytest.raises(tb.TbikError):
        tb.tbik_combine_experts(Y, slots, weights, out_dtype=torch.float16)
    with pytest.raises(tb.TbikError):
        tb.tbik_combine_experts(torch.zeros((3, 20, 64), device=DEV), slots, weights, out_dtype=torch.bfloat16)


@pytest.mark.parametrize("T", [1, 7, 150])
def test_a_mixture_of_experts_layer(T):
    """Router, both products, weighted sum, norm: the bits of a token depend neither on the batch nor on the number of shards; the values are the
    layer's formula's."""
    g = torch.Generator(device=DEV).manual_seed(T)
    E, k, H, I, dt = 12, 3, 512, 256, torch.bfloat16
    randn = lambda *s: torch.randn(s, generator=g, device=DEV)
    x, router = randn(T, H).to(dt), randn(H, E)
    up, down = (0.05 * randn(E, H, 2 * I)).to(dt), (0.05 * randn(E, I, H)).to(dt)
    post, nxt, gate = (1 + 0.1 * randn(H)).to(dt), (1 + 0.1 * randn(H)).to(dt), torch.sigmoid(randn(H)).to(dt)
    logits = tb.tbik_gemm_f32(x.float(), router, 128, 1)

    def layer(x, logits, P):
        experts, weights, offsets, rows, slots = tb.tbik_route_topk(logits, k)
        act = tb.tbik_gemm_grouped_swiglu(x, up, offsets, 64, 1, rows=rows)
        y = tb.tbik_gemm_grouped(act, down, offsets, 64, 1, out_dtype=torch.float32) if P == 0 else tb.tbik_gemm_grouped_shard_partials(act, down, offsets, 64, 1, P)
        mixed = tb.tbik_combine_experts(y, slots, weights, out_dtype=dt)
        return tb.tbik_rmsnorm_residual_rmsnorm(mixed, x, post, nxt, residual_scale=0.5, gate=gate) + (experts, mixed)

    hidden, normed, experts, mixed = layer(x, logits, 0)
    for P in (1, 2, 4):
        assert all(torch.equal(a, b) for a, b in zip(layer(x, logits, P), (hidden, normed, experts, mixed)))
    for lo, hi in ((0, 1), (T // 2, T)):
        part = layer(x[lo:hi], logits[lo:hi].contiguous(), 2)
        assert all(torch.equal(a, b[lo:hi]) for a, b in zip(part, (hidden, normed, experts, mixed)))
    p = torch.softmax(logits.double(), 1).gather(1, experts.long())
    p = p / p.sum(1, keepdim=True)
    want = torch.zeros((T, H), dtype=torch.float64, device=DEV)
    for j in range(k):
        for t in range(T):
            e = experts[t, j]
            gu = (x[t:t + 1].double() @ up[e].double())
            act = gu[:, :I] / (1 + torch.exp(-gu[:, :I])) * gu[:, I:]
            want[t] += p[t, j] * (act @ down[e].double())[0]
    # gate and up are rounded (half a step of 2^-8 each, the gate's up to doubled by the activation's slope), act and the output once more:
    # at most 5 half steps of each term's size, and the terms of a row's sum add up in magnitude; compared by the rows' norms.
    assert ((mixed.double() - want).norm(dim=1) <= 5 * 2.0 ** -8 * want.norm(dim=1)).all()
