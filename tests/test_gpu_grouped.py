"""Products grouped by expert: every row has the bits of the ungrouped product of that row and its group's weight."""
import itertools

import pytest
import torch

from paper_2511_17826_amd import binding as tb

pytestmark = pytest.mark.gpu
DEV = "cuda:0"
GEMM = {torch.bfloat16: tb.tbik_gemm, torch.float16: tb.tbik_gemm_f16}
PARTIALS = {torch.bfloat16: tb.tbik_gemm_shard_partials, torch.float16: tb.tbik_gemm_shard_partials_f16}
bits = lambda t: t.contiguous().view(torch.int32 if t.dtype == torch.float32 else torch.int16)


def operands(sizes, K, N, dtype, seed, tokens=None):
    g = torch.Generator(device=DEV).manual_seed(seed)
    R = sum(sizes)
    X = torch.randn((R if tokens is None else tokens, K), generator=g, device=DEV).to(dtype)
    W = (0.05 * torch.randn((len(sizes), K, N), generator=g, device=DEV)).to(dtype)
    offsets = torch.tensor([0] + list(itertools.accumulate(sizes)), dtype=torch.int32, device=DEV)
    rows = None if tokens is None else torch.randint(0, tokens, (R,), generator=g, device=DEV, dtype=torch.int32)
    return X, W, offsets, rows


def each_group(fn, X, W, offsets, rows):
    """fn of each group's rows and weight."""
    ends = offsets.tolist()
    for e in range(W.shape[0]):
        if ends[e + 1] > ends[e]:
            span = slice(ends[e], ends[e + 1])
            yield span, fn(X[span].contiguous() if rows is None else X[rows[span].long()], W[e])


RAGGED = [[1], [33], [0, 0, 5, 0], [1, 2, 3, 0, 31, 32, 33], [64, 65, 1], [130, 0, 7, 257], [1] * 70 + [0] * 70 + [3] * 5, [0, 500, 12]]
TREES = [(512, 64, 1), (384, 64, 3), (1024, 256, 1), (640, 16, 5), (128, 128, 1), (96, 48, 1), (2048, 32, 1)]


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float16])
@pytest.mark.parametrize("sizes", RAGGED, ids=lambda s: "x".join(map(str, s[:8])))
@pytest.mark.parametrize("gathered", [False, True])
def test_rows_of_ragged_groups(sizes, dtype, gathered):
    X, W, offsets, rows = operands(sizes, 512, 136, dtype, 7 + len(sizes), tokens=23 if gathered else None)
    y = tb.tbik_gemm_grouped(X, W, offsets, 64, 1, rows=rows)
    wide = tb.tbik_gemm_grouped(X, W, offsets, 64, 1, rows=rows, out_dtype=torch.float32)
    assert y.dtype == dtype and y.shape == wide.shape == (sum(sizes), 136)
    for span, want in each_group(lambda x, w: GEMM[dtype](x, w, 64, 1, out_dtype=torch.float32), X, W, offsets, rows):
        assert torch.equal(bits(wide[span]), bits(want))
        assert torch.equal(bits(y[span]), bits(want.to(dtype)))


@pytest.mark.parametrize("K,leaf,k_first", TREES)
@pytest.mark.parametrize("N", [8, 64, 200, 264])
def test_trees_and_columns(K, leaf, k_first, N):
    for dtype in (torch.bfloat16, torch.float16):
        X, W, offsets, rows = operands([3, 0, 40, 129], K, N, dtype, K + N, tokens=50)
        y = tb.tbik_gemm_grouped(X, W, offsets, leaf, k_first, rows=rows)
        for span, want in each_group(lambda x, w: GEMM[dtype](x, w, leaf, k_first, out_dtype=dtype), X, W, offsets, rows):
            assert torch.equal(bits(y[span]), bits(want))


@pytest.mark.parametrize("sizes", [[1], [2, 0, 40], [33, 1, 200, 0]], ids=str)
@pytest.mark.parametrize("I", [8, 64, 104, 192])
@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float16])
def test_activation_inside(sizes, I, dtype):
    X, W, offsets, rows = operands(sizes, 512, 2 * I, dtype, 31 + I, tokens=17)
    act = tb.tbik_gemm_grouped_swiglu(X, W, offsets, 64, 1, rows=rows)
    assert act.shape == (sum(sizes), I) and act.dtype == dtype
    for span, want in each_group(lambda x, w: tb.tbik_gemm_swiglu(x, w, 64, 1), X, W, offsets, rows):
        assert torch.equal(bits(act[span]), bits(want))


@pytest.mark.parametrize("P", [1, 2, 4, 8])
@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float16])
def test_shards(P, dtype):
    for sizes, K, leaf, kf in (([5, 0, 70, 33], 512, 64, 1), ([1, 1, 1], 1024, 128, 1), ([150], 1536, 64, 3)):
        X, W, offsets, rows = operands(sizes, K, 72, dtype, 11 * P, tokens=40)
        parts = tb.tbik_gemm_grouped_shard_partials(X, W, offsets, leaf, kf, P, rows=rows)
        for span, want in each_group(lambda x, w: PARTIALS[dtype](x, w, leaf, kf, P), X, W, offsets, rows):
            assert torch.equal(bits(parts[:, span]), bits(want))
        whole = tb.tbik_gemm_grouped(X, W, offsets, leaf, kf, rows=rows)
        assert torch.equal(bits(tb.tbik_tree_combine(parts, out_dtype=dtype)), bits(whole))


def test_rows_outside_the_groups_stay():
    X, W, _, _ = operands([90], 512, 72, torch.bfloat16, 5)
    W = W.expand(3, -1, -1).contiguous()
    offsets = torch.tensor([4, 9, 9, 60], dtype=torch.int32, device=DEV)
    out = torch.full((90, 72), 7.0, dtype=torch.bfloat16, device=DEV)
    tb.tbik_gemm_grouped(X, W, offsets, 64, 1, out=out)
    want = tb.tbik_gemm(X, W[0], 64, 1)
    assert torch.equal(bits(out[4:60]), bits(want[4:60])) and (out[:4] == 7).all() and (out[60:] == 7).all()
    parts = torch.full((2, 90, 72), 7.0, device=DEV)
    tb.tbik_gemm_grouped_shard_partials(X, W, offsets, 64, 1, 2, out=parts)
    assert (parts[:, :4] == 7).all() and (parts[:, 60:] == 7).all() and not (parts[:, 4:60] == 7).all()
    act = torch.full((90, 36), 7.0, dtype=torch.bfloat16, device=DEV)
    with pytest.raises(tb.TbikError):                                # 36 channels are no multiple of 8
        tb.tbik_gemm_grouped_swiglu(X, W, offsets, 64, 1, out=act)
    assert (act == 7).all()


def test_offsets_and_rows_that_are_no_division():
    """Offsets that fall or leave the output, and rows outside X: within bounds, as documented."""
    X, W, _, _ = operands([100], 512, 72, torch.bfloat16, 6)
    W = torch.cat([W, 2 * W, 4 * W])
    y = tb.tbik_gemm(X, W[0], 64, 1, out_dtype=torch.float32)
    out = torch.full((100, 72), 7.0, device=DEV)
    tb.tbik_gemm_grouped(X, W, torch.tensor([-5, 20, 10, 1 << 30], dtype=torch.int32, device=DEV), 64, 1, out=out)
    assert torch.equal(out[:20], y[:20]) and torch.equal(out[20:], 4 * y[20:])           # group 1 is empty
    rows = torch.arange(100, dtype=torch.int32, device=DEV)
    rows[3], rows[4] = -9, 1 << 30
    got = tb.tbik_gemm_grouped(X, W, torch.tensor([0, 100, 100, 100], dtype=torch.int32, device=DEV), 64, 1, rows=rows, out_dtype=torch.float32)
    assert torch.equal(got[3], y[0]) and torch.equal(got[4], y[99]) and torch.equal(got[5:], y[5:])


def test_strides():
    """Rows apart, weights apart and in a larger buffer, one weight for all groups, an output inside a wider one and at an odd place."""
    for dtype in (torch.bfloat16, torch.float16):
        X, W, offsets, _ = operands([3, 60, 0, 40], 512, 136, dtype, 8)
        want = tb.tbik_gemm_grouped(X, W, offsets, 64, 1)
        Xw = torch.zeros((103, 528), dtype=dtype, device=DEV)
        Xw[:, 8:520] = X
        Ww = torch.zeros((4, 520, 160), dtype=dtype, device=DEV)
        Ww[:, 2:514, 16:152] = W
        out = torch.full((103, 151), 7.0, dtype=dtype, device=DEV)
        tb.tbik_gemm_grouped(Xw[:, 8:520], Ww[:, 2:514, 16:152], offsets, 64, 1, out=out[:, 5:141])
        assert torch.equal(bits(out[:, 5:141]), bits(want)) and (out[:, :5] == 7).all() and (out[:, 141:] == 7).all()
        one = tb.tbik_gemm_grouped(X, W[1:2].expand(4, -1, -1), offsets, 64, 1)
        assert torch.equal(bits(one), bits(GEMM[dtype](X, W[1], 64, 1, out_dtype=dtype)))
        actw = torch.full((103, 75), 7.0, dtype=dtype, device=DEV)
        act = tb.tbik_gemm_grouped_swiglu(X, W[:, :, :128].contiguous(), offsets, 64, 1)
        tb.tbik_gemm_grouped_swiglu(Xw[:, 8:520], W[:, :, :128], offsets, 64, 1, out=actw[:, 3:67])
        assert torch.equal(bits(actw[:, 3:67]), bits(act)) and (actw[:, :3] == 7).all() and (actw[:, 67:] == 7).all()


@pytest.mark.parametrize("sizes", [[1, 0, 2], [30, 100, 20], [400, 300, 500]], ids=str)
def test_bits_do_not_depend_on_the_kernel(sizes):
    """Forced tiles, and the reference kernel."""
    X, W, offsets, rows = operands(sizes, 1024, 256, torch.bfloat16, 9, tokens=60)
    want, want_act = tb.tbik_gemm_grouped(X, W, offsets, 128, 1, rows=rows), tb.tbik_gemm_grouped_swiglu(X, W, offsets, 128, 1, rows=rows)
    want_parts = tb.tbik_gemm_grouped_shard_partials(X, W, offsets, 128, 1, 4, rows=rows)
    for variant in (tb.VARIANT_REFERENCE, tb.VARIANT_T128, tb.VARIANT_T32, tb.VARIANT_T64):
        tb.tbik_set_gemm_variant(variant)
        assert torch.equal(bits(tb.tbik_gemm_grouped(X, W, offsets, 128, 1, rows=rows)), bits(want)), variant
        assert torch.equal(bits(tb.tbik_gemm_grouped_swiglu(X, W, offsets, 128, 1, rows=rows)), bits(want_act)), variant
        assert torch.equal(bits(tb.tbik_gemm_grouped_shard_partials(X, W, offsets, 128, 1, 4, rows=rows)), bits(want_parts)), variant


@pytest.mark.parametrize("sizes", [[1153, 5, 0, 2570, 128], [129, 0, 1], [1025], [300] * 9], ids=str)
def test_groups_of_several_tiles(sizes):
    """Tiles of 128 rows: panels of up to eight, rounds that do not fill the card, shards."""
    X, W, offsets, rows = operands(sizes, 256, 384, torch.bfloat16, 5, tokens=700)
    tb.tbik_set_gemm_variant(tb.VARIANT_T128)
    y = tb.tbik_gemm_grouped(X, W, offsets, 64, 1, rows=rows)
    odd = tb.tbik_gemm_grouped(X, W[:, :, :328], offsets, 64, 1, rows=rows)
    act = tb.tbik_gemm_grouped_swiglu(X, W, offsets, 64, 1, rows=rows)
    parts = tb.tbik_gemm_grouped_shard_partials(X, W, offsets, 64, 1, 4, rows=rows)
    tb.tbik_set_gemm_variant(0)
    for span, (want, want_act, want_parts) in each_group(
            lambda x, w: (tb.tbik_gemm(x, w, 64, 1, out_dtype=torch.bfloat16), tb.tbik_gemm_swiglu(x, w, 64, 1), tb.tbik_gemm_shard_partials(x, w, 64, 1, 4)),
            X, W, offsets, rows):
        assert torch.equal(bits(y[span]), bits(want))
        assert torch.equal(bits(odd[span]), bits(want[:, :328]))
        assert torch.equal(bits(act[span]), bits(want_act))
        assert torch.equal(bits(parts[:, span]), bits(want_parts))


def test_most_groups_and_no_rows():
    sizes = [(i * 7) % 5 for i in range(512)]
    X, W, offsets, rows = operands(sizes, 128, 40, torch.bfloat16, 10, tokens=64)
    y = tb.tbik_gemm_grouped(X, W, offsets, 64, 1, rows=rows)
    for span, want in itertools.islice(each_group(lambda x, w: tb.tbik_gemm(x, w, 64, 1), X, W, offsets, rows), 0, None, 17):
        assert torch.equal(bits(y[span]), bits(want))
    none = torch.zeros(513, dtype=torch.int32, device=DEV)
    out = torch.full((sum(sizes), 40), 7.0, dtype=torch.bfloat16, device=DEV)
    tb.tbik_gemm_grouped(X, W, none, 64, 1, rows=rows, out=out)
    assert (out == 7).all()
    assert tb.tbik_gemm_grouped(X, W, none, 64, 1, rows=rows[:0]).shape == (0, 40)


def test_captured_and_replayed_with_other_offsets():
    """A graph's call reads the offsets when it runs: replays follow what is written into them."""
    X, W, offsets, rows = operands([10, 20, 30], 512, 72, torch.bfloat16, 12, tokens=25)
    out = torch.zeros((60, 72), dtype=torch.bfloat16, device=DEV)
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.stream(side):
        tb.tbik_gemm_grouped(X, W, offsets, 64, 1, rows=rows, out=out)
        with torch.cuda.graph(graph, stream=side):
            tb.tbik_gemm_grouped(X, W, offsets, 64, 1, rows=rows, out=out)
    torch.cuda.current_stream().wait_stream(side)
    for ends in ([0, 10, 30, 60], [0, 60, 60, 60], [0, 0, 1, 33], [0, 10, 30, 60]):
        offsets.copy_(torch.tensor(ends, dtype=torch.int32))
        out.fill_(7)
        want = torch.full_like(out, 7)
        tb.tbik_gemm_grouped(X, W, offsets, 64, 1, rows=rows, out=want)
        graph.replay()
        torch.cuda.synchronize()
        assert torch.equal(bits(out), bits(want))


def test_refusals():
    X, W, offsets, rows = operands([4, 4], 512, 72, torch.bfloat16, 13)
    for bad in (offsets.long(), offsets[:2], offsets.cpu(), offsets.float()):
        with pytest.raises(ValueError):
            tb.tbik_gemm_grouped(X, W, bad, 64, 1)
    with pytest.raises(ValueError):
        tb.tbik_gemm_grouped(X, W.transpose(1, 2), offsets, 64, 1)
    with pytest.raises(ValueError):
        tb.tbik_gemm_grouped(X[:, :256], W, offsets, 64, 1)
    with pytest.raises(TypeError):
        tb.tbik_gemm_grouped(X, W.half(), offsets, 64, 1)
    with pytest.raises(ValueError):
        tb.tbik_gemm_grouped(X, W, offsets, 64, 1, out=torch.empty((8, 80), dtype=torch.bfloat16, device=DEV))
    with pytest.raises(tb.TbikError):
        tb.tbik_gemm_grouped(X, W, offsets, 64, 1, out_dtype=torch.float16)
    with pytest.raises(tb.TbikError):
        tb.tbik_gemm_grouped(X, W, offsets, 60, 1)
    with pytest.raises(tb.TbikError):
        tb.tbik_gemm_grouped_shard_partials(X, W, offsets, 64, 1, 16)
