"""Products on 4-bit weights against their definition in 64 bits, and their invariance."""
import pytest
import torch

from paper_2511_17826_amd import binding as tb

pytestmark = pytest.mark.gpu
DEV = "cuda:0"
bits = lambda t: t.contiguous().view(torch.int32 if t.dtype == torch.float32 else torch.int16)


def operands(M, N, K, group, dtype, zeros, seed):
    g = torch.Generator(device=DEV).manual_seed(seed)
    X = torch.randn((M, K), generator=g, device=DEV).to(dtype)
    Wq = torch.randint(0, 256, (N, K // 2), generator=g, device=DEV, dtype=torch.uint8)
    scales = (0.01 * torch.exp(0.5 * torch.randn((N, K // group), generator=g, device=DEV))).to(dtype)
    z = torch.randint(0, 16, (N, K // group), generator=g, device=DEV, dtype=torch.uint8) if zeros else None
    return X, Wq, scales, z


def weight(Wq, scales, zeros):
    """[K, N] in 64 bits."""
    N, K = Wq.shape[0], 2 * Wq.shape[1]
    q = torch.stack([Wq & 15, Wq >> 4], dim=2).reshape(N, K).double()
    group = K // scales.shape[1]
    z = 8.0 if zeros is None else (zeros & 15).double().repeat_interleave(group, 1)
    return ((q - z) * scales.double().repeat_interleave(group, 1)).t().contiguous()


def check(y, X, W, K):
    want, size = X.double() @ W, X.double().abs() @ W.abs()
    # Every product is exact.  Each of K additions, K / group scalings and the tree's additions rounds a partial sum of at most `size`; the
    # instruction may drop what is below half a step of the largest of its 16 products, which is no more than that again for each.
    tol = size * (2 * K + 64) * 2.0 ** -24
    if y.dtype != torch.float32:
        tol = tol + want.abs() * torch.finfo(y.dtype).eps / 2 * 1.01 + 2.0 ** -24 * (y.dtype == torch.float16)
    assert ((y.double() - want).abs() <= tol).all()
    # By the norm the errors do not line up: well within 2^-17 where the bound above would allow K 2^-23 (root of K half steps at most, K <= 16384).
    err = (y.double() - want).norm() / want.norm()
    assert err <= (2.0 ** -17 if y.dtype == torch.float32 else torch.finfo(y.dtype).eps / 2)


SHAPES = [(1, 32, 64, 64, 1, 64), (1, 4096, 512, 64, 1, 64), (3, 72, 512, 64, 1, 32), (33, 200, 1024, 128, 1, 128), (32, 33, 1536, 64, 3, 96), (70, 40, 640, 128, 5, 128),
          (5, 1, 2048, 256, 1, 64), (16, 129, 4096, 32, 1, 32), (2, 64, 5120, 128, 5, 128), (130, 130, 256, 256, 1, 256), (300, 96, 512, 64, 1, 64),
          # Slices of 32 channels, and of 16 where there are very many; groups of more than one unit.
          (4, 4136, 512, 64, 1, 64), (12, 4136, 1024, 64, 1, 32), (6, 8232, 512, 128, 1, 128), (16, 8232, 2048, 64, 1, 64), (1, 8232, 512, 64, 1, 32), (7, 4200, 768, 64, 3, 192),
          (40, 100, 2048, 256, 1, 256), (9, 100, 1536, 64, 3, 192), (1, 72, 4096, 512, 1, 256), (90, 136, 1280, 64, 5, 160),
          # Tiles of 32 and 64 rows, of one superleaf and of many, K divided or not.
          (20, 8264, 128, 128, 1, 64), (50, 8264, 256, 256, 1, 128), (20, 8264, 256, 64, 1, 32), (33, 1160, 1024, 128, 1, 128), (70, 2088, 640, 128, 5, 128), (27, 1160, 2048, 64, 1, 64),
          (130, 1160, 1024, 64, 1, 64), (300, 1160, 512, 64, 1, 64), (200, 4136, 768, 64, 3, 192), (61, 1160, 8192, 256, 1, 256)]


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float16])
@pytest.mark.parametrize("zeros", [False, True])
@pytest.mark.parametrize("M,N,K,leaf,k_first,group", SHAPES)
def test_against_the_definition(M, N, K, leaf, k_first, group, dtype, zeros):
    X, Wq, scales, z = operands(M, N, K, group, dtype, zeros, M + N + K)
    W = weight(Wq, scales, z)
    y = tb.tbik_gemm_w4(X, Wq, scales, leaf, k_first, zeros=z)
    wide = tb.tbik_gemm_w4(X, Wq, scales, leaf, k_first, zeros=z, out_dtype=torch.float32)
    assert y.dtype == dtype and y.shape == (M, N)
    check(wide, X, W, K)
    assert torch.equal(bits(wide.to(dtype)), bits(y))                # one rounding


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float16])
def test_whole_numbers_are_exact(dtype):
    """Small whole numbers and powers of two as scales: every sum is exact, so the result is the definition's to the bit; all 16 levels, every zero."""
    g = torch.Generator(device=DEV).manual_seed(1)
    for zeros in (None, torch.arange(16, device=DEV, dtype=torch.uint8).repeat(4, 1).repeat(16, 1)[:64, :16].contiguous()):
        X = torch.randint(-8, 9, (40, 1024), generator=g, device=DEV).to(dtype)
        Wq = torch.randint(0, 256, (64, 512), generator=g, device=DEV, dtype=torch.uint8)
        scales = torch.exp2(torch.randint(-3, 2, (64, 16), generator=g, device=DEV).float()).to(dtype)
        y = tb.tbik_gemm_w4(X, Wq, scales, 64, 1, zeros=zeros, out_dtype=torch.float32)
        assert torch.equal(y.double(), X.double() @ weight(Wq, scales, zeros))


def test_high_bits_of_a_zero_do_not_count():
    X, Wq, scales, z = operands(3, 40, 512, 64, torch.bfloat16, True, 2)
    assert torch.equal(tb.tbik_gemm_w4(X, Wq, scales, 64, 1, zeros=z | 0xa0), tb.tbik_gemm_w4(X, Wq, scales, 64, 1, zeros=z))
    eight = torch.full_like(z, 8)
    assert torch.equal(tb.tbik_gemm_w4(X, Wq, scales, 64, 1, zeros=eight), tb.tbik_gemm_w4(X, Wq, scales, 64, 1))


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float16])
@pytest.mark.parametrize("zeros", [False, True])
@pytest.mark.parametrize("K,leaf,k_first,group", [(4096, 256, 1, 128), (2048, 128, 1, 32), (1536, 64, 3, 64), (5120, 128, 5, 128)])
def test_batch_and_shards(K, leaf, k_first, group, dtype, zeros):
    X, Wq, scales, z = operands(200, 1160, K, group, dtype, zeros, K)
    want = tb.tbik_gemm_w4(X, Wq, scales, leaf, k_first, zeros=z, out_dtype=torch.float32)
    for lo, hi in ((0, 1), (7, 9), (100, 117), (40, 73), (5, 70), (64, 200)):
        assert torch.equal(bits(tb.tbik_gemm_w4(X[lo:hi], Wq, scales, leaf, k_first, zeros=z, out_dtype=torch.float32)), bits(want[lo:hi]))
    ns = K // (leaf * k_first)
    P = 1
    while P <= min(ns, 16):
        for rows in (X, X[:5]):
            parts = tb.tbik_gemm_shard_partials_w4(rows, Wq, scales, leaf, k_first, P, zeros=z)
            assert parts.shape == (P, rows.shape[0], 1160)
            assert torch.equal(bits(tb.tbik_tree_combine(parts, out_dtype=torch.float32)), bits(want[:rows.shape[0]]))
        P *= 2
    # A real rank's own part of the operands: whole groups, its own bytes.
    if ns >= 2:
        halves = [tb.tbik_gemm_shard_partials_w4(X[:, s * K // 2:(s + 1) * K // 2].contiguous(), Wq[:, s * K // 4:(s + 1) * K // 4].contiguous(),
                                                 scales[:, s * (K // group) // 2:(s + 1) * (K // group) // 2].contiguous(), leaf, k_first, 1,
                                                 zeros=z[:, s * (K // group) // 2:(s + 1) * (K // group) // 2].contiguous() if zeros else None)[0] for s in (0, 1)]
        assert torch.equal(bits(tb.tbik_tree_combine(torch.stack(halves), out_dtype=torch.float32)), bits(want))


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float16])
@pytest.mark.parametrize("zeros", [False, True])
@pytest.mark.parametrize("K,leaf,k_first,group", [(12288, 256, 3, 32), (8192, 64, 1, 32), (6144, 64, 3, 96), (14336, 256, 7, 64), (16384, 256, 1, 256), (12288, 64, 3, 192)])
def test_more_groups_than_a_chunk_of_scales(K, leaf, k_first, group, dtype, zeros):
    """Every wavefront walks more groups than are held at once; scales and zero points at odd addresses; one row to many, one shard."""
    X, Wq, scales, z = operands(150, 1160, K, group, dtype, zeros, K + group)
    sw = torch.zeros((1160, K // group + 3), dtype=dtype, device=DEV)
    sw[:, 1:-2] = scales
    zw = torch.zeros((1160, K // group + 6), dtype=torch.uint8, device=DEV)
    if zeros:
        zw[:, 3:-3] = z
        z = zw[:, 3:-3]
    W = weight(Wq, scales, z)
    want = tb.tbik_gemm_shard_partials_w4(X, Wq, sw[:, 1:-2], leaf, k_first, 1, zeros=z)[0]
    check(want, X, W, K)
    for rows in (1, 7, 16, 20, 50, 100):
        assert torch.equal(bits(tb.tbik_gemm_shard_partials_w4(X[:rows], Wq, scales, leaf, k_first, 1, zeros=z)[0]), bits(want[:rows])), rows
        assert torch.equal(bits(tb.tbik_gemm_w4(X[:rows], Wq, sw[:, 1:-2], leaf, k_first, zeros=z, out_dtype=torch.float32)), bits(want[:rows])), rows


def test_less_workspace_and_the_general_kernel():
    """The split of K follows the room; operands too far apart for the kernels with direct loads go another way: the same bits."""
    X, Wq, scales, z = operands(40, 1160, 4096, 64, torch.bfloat16, True, 7)
    want = tb.tbik_gemm_w4(X, Wq, scales, 256, 1, zeros=z)
    need = tb.lib().tbik_gemm_w4_workspace_bytes(40, 1160, 4096, 256, 1)
    assert need > 0
    for room in (0, 256, need // 2, need // 4 + 1, need):
        assert torch.equal(bits(tb.tbik_gemm_w4(X, Wq, scales, 256, 1, zeros=z, workspace=torch.empty(room, dtype=torch.uint8, device=DEV))), bits(want))
    far = torch.empty_strided((40, 4096), (1 << 22, 1), dtype=torch.bfloat16, device=DEV)
    far.copy_(X)
    for rows in (3, 40):
        assert torch.equal(bits(tb.tbik_gemm_w4(far[:rows], Wq, scales, 256, 1, zeros=z)), bits(want[:rows]))


def test_strides():
    X, Wq, scales, z = operands(9, 70, 512, 64, torch.bfloat16, True, 4)
    want = tb.tbik_gemm_w4(X, Wq, scales, 64, 1, zeros=z)
    Xw = torch.zeros((9, 560), dtype=torch.bfloat16, device=DEV)
    Xw[:, 16:528] = X
    Ww = torch.zeros((70, 304), dtype=torch.uint8, device=DEV)
    Ww[:, 32:288] = Wq
    sw = torch.zeros((70, 11), dtype=torch.bfloat16, device=DEV)
    sw[:, 2:10] = scales
    zw = torch.zeros((70, 13), dtype=torch.uint8, device=DEV)
    zw[:, 3:11] = z
    out = torch.full((9, 77), 7.0, dtype=torch.bfloat16, device=DEV)
    tb.tbik_gemm_w4(Xw[:, 16:528], Ww[:, 32:288], sw[:, 2:10], 64, 1, zeros=zw[:, 3:11], out=out[:, 3:73])
    assert torch.equal(bits(out[:, 3:73]), bits(want)) and (out[:, :3] == 7).all() and (out[:, 73:] == 7).all()


def test_a_graph_replayed():
    X, Wq, scales, z = operands(4, 512, 1024, 128, torch.bfloat16, True, 5)
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.stream(side):
        tb.tbik_gemm_w4(X, Wq, scales, 128, 1, zeros=z)
        with torch.cuda.graph(graph, stream=side):
            out = tb.tbik_gemm_w4(X, Wq, scales, 128, 1, zeros=z)
    torch.cuda.current_stream().wait_stream(side)
    for i in range(3):
        X.copy_(torch.randn_like(X))
        want = tb.tbik_gemm_w4(X, Wq, scales, 128, 1, zeros=z)
        graph.replay()
        torch.cuda.synchronize()
        assert torch.equal(bits(out), bits(want))


def test_no_rows_and_refusals():
    X, Wq, scales, z = operands(4, 72, 512, 64, torch.bfloat16, True, 6)
    assert tb.tbik_gemm_w4(X[:0], Wq, scales, 64, 1).shape == (0, 72)
    for kw in (dict(Wq=Wq[:, :128]), dict(scales=scales[:64]), dict(zeros=z[:, :4]), dict(scales=scales[:, :7]), dict(out=torch.empty((4, 73), dtype=torch.bfloat16, device=DEV)), dict(X=X.cpu())):
        with pytest.raises(ValueError):
            tb.tbik_gemm_w4(**{**dict(X=X, Wq=Wq, scales=scales, leaf=64, zeros=z), **kw})
    for kw in (dict(X=X.half()), dict(Wq=Wq.int()), dict(zeros=z.float()), dict(X=X.float(), scales=scales.float())):
        with pytest.raises(TypeError):
            tb.tbik_gemm_w4(**{**dict(X=X, Wq=Wq, scales=scales, leaf=64, zeros=z), **kw})
    with pytest.raises(tb.TbikError):                                # a group of 64 in a leaf of 32
        tb.tbik_gemm_w4(X, Wq, scales, 32, 1)
    with pytest.raises(tb.TbikError):                                # groups of 16
        tb.tbik_gemm_w4(X, Wq, scales.repeat_interleave(4, 1), 64, 1)
