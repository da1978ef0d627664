"""tbik_rmsnorm_residual_rmsnorm against its definition in 64 bits and against the calls that it joins."""
import pytest
import torch

from paper_2511_17826_amd import binding as tb

pytestmark = pytest.mark.gpu
DEV = "cuda:0"
EPS = 1e-6
bits = lambda t: t.contiguous().view(torch.int16)
NORM = {torch.bfloat16: tb.tbik_rmsnorm, torch.float16: tb.tbik_rmsnorm_f16}
GATES = {"none": None, "channel": lambda M, H: (H,), "one_row": lambda M, H: (1, H), "row": lambda M, H: (M, 1), "full": lambda M, H: (M, H), "one": lambda M, H: (1, 1)}


def inputs(M, H, dtype, gate, seed, P=0):
    g = torch.Generator(device=DEV).manual_seed(seed)
    randn = lambda *s: torch.randn(s, generator=g, device=DEV)
    y = 0.6 * randn(P, M, H) if P else (2 * randn(M, H)).to(dtype)
    shape = GATES[gate] and GATES[gate](M, H)
    return y, (3 * randn(M, H)).to(dtype), (1 + 0.2 * randn(H)).to(dtype), (1 + 0.2 * randn(H)).to(dtype), torch.sigmoid(randn(*shape)).to(dtype) if shape else None


def check_hidden(hidden, y, residual, post, gate, scale, H):
    """y [M, H] of the rows' type."""
    n = y.double()
    if post is not None:
        n = n * post.double() / torch.sqrt((n * n).mean(1, keepdim=True) + EPS)
    if gate is not None:
        n = n * gate.double()
    want = residual.double() * scale + n
    # n: the sum of squares (8 additions in a leaf and the tree's, all of one sign), mean, eps, root, reciprocal and three products: at most
    # H.bit_length() + 16 half steps; the two products and the sum one half step each; then the rounding.
    tol = n.abs() * (H.bit_length() + 18) * 2.0 ** -24 + (residual.double() * scale).abs() * 2.0 ** -23 + want.abs() * torch.finfo(hidden.dtype).eps / 2 * 1.01
    tol = tol + 2.0 ** -24 * (hidden.dtype == torch.float16)
    assert ((hidden.double() - want).abs() <= tol).all()


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float16])
@pytest.mark.parametrize("gate", sorted(GATES))
@pytest.mark.parametrize("M,H", [(1, 8), (1, 4096), (5, 520), (3, 5120), (2, 6000), (9, 1024), (2, 8200), (1, 20000), (1, 40000), (2, 65536)])
def test_16_bit_rows(M, H, dtype, gate):
    y, residual, post, nxt, g = inputs(M, H, dtype, gate, M + H)
    for scale in (1.0, 0.75):
        hidden, normed = tb.tbik_rmsnorm_residual_rmsnorm(y, residual, post, nxt, EPS, residual_scale=scale, gate=g)
        check_hidden(hidden, y, residual, post, g, scale, H)
        assert torch.equal(bits(normed), bits(NORM[dtype](hidden, nxt, EPS)))


@pytest.mark.parametrize("P", [1, 2, 4, 8, 16])
@pytest.mark.parametrize("M,H", [(3, 512), (2, 5120), (1, 16384), (1, 65536)])
def test_shards_sums(P, M, H):
    for dtype in (torch.bfloat16, torch.float16):
        parts, residual, post, nxt, g = inputs(M, H, dtype, "full", P + H, P)
        y = tb.tbik_tree_combine(parts, out_dtype=dtype)
        for a, b in zip(tb.tbik_rmsnorm_residual_rmsnorm(parts, residual, post, nxt, EPS, gate=g), tb.tbik_rmsnorm_residual_rmsnorm(y, residual, post, nxt, EPS, gate=g)):
            assert torch.equal(bits(a), bits(b))


@pytest.mark.parametrize("H", [256, 4096, 12288])
def test_the_calls_that_it_joins(H):
    """The norm behind the block on its own, and no norm behind it: the tail of a row-parallel layer."""
    for dtype, tail in ((torch.bfloat16, tb.tbik_combine_residual_rmsnorm), (torch.float16, tb.tbik_combine_residual_rmsnorm_f16)):
        parts, residual, post, nxt, _ = inputs(7, H, dtype, "none", H, 2)
        for a, b in zip(tb.tbik_rmsnorm_residual_rmsnorm(parts, residual, None, nxt, EPS), tail(parts, residual, nxt, EPS)):
            assert torch.equal(bits(a), bits(b))
        y = tb.tbik_tree_combine(parts, out_dtype=dtype)
        hidden, normed = tb.tbik_rmsnorm_residual_rmsnorm(y, torch.zeros_like(residual), post, None, EPS)
        assert normed is None and torch.equal(bits(hidden), bits(NORM[dtype](y, post, EPS)))


def test_a_row_does_not_depend_on_the_batch_and_stays_in_place():
    y, residual, post, nxt, g = inputs(50, 2048, torch.bfloat16, "row", 3)
    hidden, normed = tb.tbik_rmsnorm_residual_rmsnorm(y, residual, post, nxt, EPS, gate=g)
    for lo, hi in ((0, 1), (13, 50)):
        h, n = tb.tbik_rmsnorm_residual_rmsnorm(y[lo:hi], residual[lo:hi], post, nxt, EPS, gate=g[lo:hi])
        assert torch.equal(bits(h), bits(hidden[lo:hi])) and torch.equal(bits(n), bits(normed[lo:hi]))
    stream, block = residual.clone(), y.clone()
    h, n = tb.tbik_rmsnorm_residual_rmsnorm(y, stream, post, nxt, EPS, gate=g, hidden=stream)
    assert h is stream and torch.equal(bits(stream), bits(hidden)) and torch.equal(bits(n), bits(normed))
    tb.tbik_rmsnorm_residual_rmsnorm(block, residual, post, nxt, EPS, gate=g, hidden=block)
    assert torch.equal(bits(block), bits(hidden))


def test_strides():
    y, residual, post, nxt, g = inputs(6, 520, torch.float16, "full", 4)
    want = tb.tbik_rmsnorm_residual_rmsnorm(y, residual, post, nxt, EPS, gate=g)
    def within(t, width, at):
        w = torch.full((t.shape[0], width), 7.0, dtype=t.dtype, device=DEV)
        w[:, at:at + t.shape[1]] = t
        return w, w[:, at:at + t.shape[1]]
    (_, ys), (_, rs), (_, gs), (hw, hs), (nw, ns) = within(y, 600, 8), within(residual, 640, 16), within(g, 552, 24), within(y, 560, 32), within(y, 536, 0)
    tb.tbik_rmsnorm_residual_rmsnorm(ys, rs, post, nxt, EPS, gate=gs, hidden=hs, normed=ns)
    assert torch.equal(bits(hs), bits(want[0])) and torch.equal(bits(ns), bits(want[1]))
    assert (hw[:, :32] == 7).all() and (hw[:, 552:] == 7).all() and (nw[:, 520:] == 7).all()
    column = torch.sigmoid(torch.randn((6, 9), device=DEV)).half()
    a = tb.tbik_rmsnorm_residual_rmsnorm(y, residual, post, nxt, EPS, gate=column[:, 3:4])
    b = tb.tbik_rmsnorm_residual_rmsnorm(y, residual, post, nxt, EPS, gate=column[:, 3:4].contiguous())
    assert torch.equal(bits(a[0]), bits(b[0])) and torch.equal(bits(a[1]), bits(b[1]))


def test_zeros_infinities_and_nan():
    y, residual, post, nxt, _ = inputs(4, 512, torch.bfloat16, "none", 5)
    y[0], residual[0] = 0, 0
    y[1, 3], y[2, 4] = float("inf"), float("nan")
    hidden, normed = tb.tbik_rmsnorm_residual_rmsnorm(y, residual, post, nxt, EPS)
    assert (hidden[0] == 0).all() and (normed[0] == 0).all()
    # an infinite element makes the row's scale 0: itself 0 times infinity, the others zero
    assert torch.isnan(hidden[1, 3]) and torch.equal(bits(hidden[1, 4:]), bits(residual[1, 4:])) and torch.isnan(normed[1]).all()
    assert torch.isnan(hidden[2]).all() and torch.isfinite(hidden[3]).all()


def test_no_rows_and_refusals():
    y, residual, post, nxt, g = inputs(4, 512, torch.bfloat16, "full", 6)
    hidden, normed = tb.tbik_rmsnorm_residual_rmsnorm(y[:0], residual[:0], post, nxt)
    assert hidden.shape == normed.shape == (0, 512)
    base = dict(y=y, residual=residual, post_weight=post, next_weight=nxt, gate=g)
    for kw in (dict(y=y[:3]), dict(y=y.half()), dict(post_weight=post[:8]), dict(next_weight=nxt.float()), dict(gate=g[:3]), dict(gate=g.float()), dict(gate=g[:, :5]), dict(gate=g.t()),
               dict(next_weight=None, normed=torch.empty_like(y)), dict(hidden=torch.empty((4, 520), dtype=torch.bfloat16, device=DEV)), dict(y=y.cpu()), dict(y=torch.zeros((2, 4, 512), device=DEV).half())):
        with pytest.raises(ValueError):
            tb.tbik_rmsnorm_residual_rmsnorm(**{**base, **kw})
    with pytest.raises(TypeError):
        tb.tbik_rmsnorm_residual_rmsnorm(y.float(), residual.float(), post, nxt)
    with pytest.raises(tb.TbikError):                                # 60 columns
        tb.tbik_rmsnorm_residual_rmsnorm(y[:, :60].contiguous(), residual[:, :60].contiguous(), post[:60].contiguous(), nxt[:60].contiguous())
    with pytest.raises(tb.TbikError):                                # rows at odd addresses
        tb.tbik_rmsnorm_residual_rmsnorm(y[:, 1:505], residual[:, 8:512], post[:504].contiguous(), nxt[:504].contiguous())
    with pytest.raises(tb.TbikError):
        tb.tbik_rmsnorm_residual_rmsnorm(torch.zeros((3, 4, 512), device=DEV), residual, post, nxt)
