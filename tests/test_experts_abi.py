"""The calls of a mixture of experts, of 4-bit weights and of the norms around a block refuse bad arguments before anything is launched
(CPU: no kernel runs; addresses are made up and never read)."""
import pytest

A = 1 << 20                                     # an aligned address
OK, NULL, SHAPE, SHARDS, DTYPE, ALIGN, WORKSPACE, UNSUPPORTED = 0, 1, 2, 3, 4, 5, 6, 7
F32, BF16, F16 = 0, 1, 2


@pytest.fixture(scope="module")
def L():
    from paper_2511_17826_amd import binding
    return binding.lib()


def call(L, name, defaults, **changes):
    assert set(changes) <= set(defaults), changes
    return getattr(L, name)(*{**defaults, **changes}.values())


ROUTE = dict(logits=A, ldl=64, dtype=F32, T=100, E=64, k=4, renormalize=1, experts=A, weights=A, offsets=A, rows=A, slots=A, ws=A, ws_bytes=1 << 20, stream=None)
GROUPED = dict(X=A, ldx=512, tokens=10, rows=A, W=A, ldw=256, stride=512 * 256, groups=4, offsets=A, Y=A, ldy=256, y_dtype=BF16, x_dtype=BF16, R=20, N=256,
               K=512, leaf=64, k_first=1, stream=None)
SWIGLU = dict(X=A, ldx=512, tokens=10, rows=A, W=A, ldw=256, stride=512 * 256, groups=4, offsets=A, act=A, lda=128, dtype=BF16, R=20, I=128,
              K=512, leaf=64, k_first=1, stream=None)
PARTIALS = dict(X=A, ldx=512, tokens=10, rows=A, W=A, ldw=256, stride=512 * 256, groups=4, offsets=A, partials=A, x_dtype=BF16, R=20, N=256,
                K=512, leaf=64, k_first=1, P=2, stream=None)
SUM = dict(Y=A, ldy=64, y_dtype=BF16, P=1, R=20, slots=A, weights=A, residual=A, ldr=64, out=A, ldo=64, out_dtype=BF16, T=10, H=64, k=2, stream=None)
W4 = dict(X=A, ldx=512, Wq=A, ldwq=256, scales=A, lds=8, zeros=A, ldz=8, group=64, Y=A, ldy=128, y_dtype=BF16, x_dtype=BF16, M=3, N=128, K=512, leaf=64,
          k_first=1, ws=None, ws_bytes=0, stream=None)
W4P = dict(X=A, ldx=512, Wq=A, ldwq=256, scales=A, lds=8, zeros=None, ldz=0, group=64, partials=A, x_dtype=BF16, M=3, N=128, K=512, leaf=64, k_first=1, P=2,
           stream=None)
JOIN = dict(y=A, ldy=64, partials=None, P=1, residual=A, ldr=64, scale=1.0, post=A, gate=A, gate_row=0, gate_col=1, next=A, eps=1e-6, hidden=2 * A, ldh=64, normed=A,
            ldn=64, dtype=BF16, M=3, H=64, stream=None)


@pytest.mark.parametrize("changes,status", [
    (dict(T=-1), SHAPE), (dict(E=0), SHAPE), (dict(k=0), SHAPE), (dict(k=65), SHAPE), (dict(ldl=63), SHAPE), (dict(T=1 << 27, k=32), SHAPE),
    (dict(E=513, ldl=513), UNSUPPORTED), (dict(k=33), UNSUPPORTED), (dict(T=(1 << 26) + 1, k=1), UNSUPPORTED), (dict(dtype=3), DTYPE), (dict(logits=None), NULL),
    (dict(experts=None), NULL), (dict(weights=None), NULL), (dict(offsets=None), NULL), (dict(rows=None), NULL), (dict(slots=None), NULL), (dict(T=0, offsets=None), NULL),
    (dict(logits=A + 2), ALIGN), (dict(weights=A + 2), ALIGN), (dict(ws=None), WORKSPACE), (dict(ws_bytes=8), WORKSPACE), (dict(ws=A + 64), ALIGN)])
def test_route_refuses(L, changes, status):
    assert call(L, "tbik_route_topk", ROUTE, **changes) == status


def test_route_workspace(L):
    size = L.tbik_route_topk_workspace_bytes
    assert size(64, 512) == 0 and size(0, 8) == 0 and size(65, 8) > 0 and size(-1, 8) == 0 and size(100, 513) == 0 and size(100, 0) == 0


@pytest.mark.parametrize("changes,status", [
    (dict(R=-1), SHAPE), (dict(N=-1), SHAPE), (dict(K=500), SHAPE), (dict(leaf=8), SHAPE), (dict(tokens=-1), SHAPE), (dict(groups=-1), SHAPE),
    (dict(rows=None), SHAPE),                   # 10 tokens, 20 rows
    (dict(ldx=504), SHAPE), (dict(ldw=248), SHAPE), (dict(ldy=255), SHAPE), (dict(stride=-8), SHAPE), (dict(groups=513), UNSUPPORTED), (dict(R=0x7fffff01), UNSUPPORTED),
    (dict(x_dtype=F32, y_dtype=F32), DTYPE), (dict(x_dtype=5), DTYPE), (dict(y_dtype=F16), DTYPE), (dict(X=None), NULL), (dict(W=None), NULL), (dict(offsets=None), NULL),
    (dict(Y=None), NULL), (dict(X=A + 8), ALIGN), (dict(W=A + 8), ALIGN), (dict(ldx=516), ALIGN), (dict(ldw=260), ALIGN), (dict(stride=512 * 256 + 4), ALIGN),
    (dict(offsets=A + 2), ALIGN), (dict(rows=A + 2), ALIGN), (dict(Y=A + 1), ALIGN), (dict(Y=A + 2, y_dtype=F32), ALIGN),
    (dict(R=0), OK), (dict(N=0), OK), (dict(groups=0), OK), (dict(tokens=0), OK)])
def test_grouped_refuses(L, changes, status):
    assert call(L, "tbik_gemm_grouped", GROUPED, **changes) == status


@pytest.mark.parametrize("changes,status", [
    (dict(I=-8), SHAPE), (dict(I=12), SHAPE), (dict(I=1 << 30), SHAPE), (dict(lda=120), SHAPE), (dict(ldw=248), SHAPE), (dict(dtype=F32), DTYPE), (dict(act=None), NULL),
    (dict(act=A + 1), ALIGN), (dict(rows=None), SHAPE), (dict(R=0), OK), (dict(I=0), OK)])
def test_grouped_swiglu_refuses(L, changes, status):
    assert call(L, "tbik_gemm_grouped_swiglu", SWIGLU, **changes) == status


@pytest.mark.parametrize("changes,status", [
    (dict(P=0), SHARDS), (dict(P=3), SHARDS), (dict(P=16), SHARDS), (dict(partials=None), NULL), (dict(partials=A + 4), ALIGN), (dict(x_dtype=F32), DTYPE), (dict(R=0), OK)])
def test_grouped_partials_refuse(L, changes, status):
    assert call(L, "tbik_gemm_grouped_shard_partials", PARTIALS, **changes) == status


@pytest.mark.parametrize("changes,status", [
    (dict(T=-1), SHAPE), (dict(H=-1), SHAPE), (dict(k=0), SHAPE), (dict(R=-1), SHAPE), (dict(ldy=63), SHAPE), (dict(ldo=63), SHAPE), (dict(ldr=63), SHAPE),
    (dict(residual=A, out=A, ldr=72), SHAPE), (dict(P=0), SHARDS), (dict(P=3), SHARDS), (dict(P=2), SHARDS), (dict(P=32, y_dtype=F32), UNSUPPORTED), (dict(k=33), UNSUPPORTED),
    (dict(y_dtype=3), DTYPE), (dict(out_dtype=F16), DTYPE), (dict(y_dtype=F32, out_dtype=4), DTYPE), (dict(Y=None), NULL), (dict(slots=None), NULL), (dict(weights=None), NULL),
    (dict(out=None), NULL), (dict(Y=A + 1), ALIGN), (dict(out=A + 1), ALIGN), (dict(residual=A + 1), ALIGN), (dict(slots=A + 2), ALIGN), (dict(weights=A + 2), ALIGN),
    (dict(y_dtype=F32, out_dtype=BF16, Y=A + 2), ALIGN), (dict(T=0), OK), (dict(H=0), OK)])
def test_combine_refuses(L, changes, status):
    assert call(L, "tbik_combine_experts", SUM, **changes) == status


@pytest.mark.parametrize("changes,status", [
    (dict(M=-1), SHAPE), (dict(K=500), SHAPE), (dict(group=16), SHAPE), (dict(group=48), SHAPE), (dict(group=128), SHAPE), (dict(group=0), SHAPE), (dict(ldx=504), SHAPE),
    (dict(ldwq=240), SHAPE), (dict(lds=7), SHAPE), (dict(ldz=7), SHAPE), (dict(ldy=127), SHAPE), (dict(x_dtype=F32, y_dtype=F32), DTYPE), (dict(y_dtype=F16), DTYPE),
    (dict(X=None), NULL), (dict(Wq=None), NULL), (dict(scales=None), NULL), (dict(Y=None), NULL), (dict(X=A + 8), ALIGN), (dict(Wq=A + 8), ALIGN), (dict(ldwq=264), ALIGN),
    (dict(ldx=516), ALIGN), (dict(scales=A + 1), ALIGN), (dict(Y=A + 1), ALIGN), (dict(K=64 * 256, ldx=64 * 256, ldwq=32 * 256, lds=256, ldz=256), UNSUPPORTED),
    (dict(ws=A + 64, ws_bytes=1 << 20), ALIGN), (dict(M=0), OK), (dict(N=0), OK)])
def test_w4_refuses(L, changes, status):
    assert call(L, "tbik_gemm_w4", W4, **changes) == status


@pytest.mark.parametrize("changes,status", [(dict(P=0), SHARDS), (dict(P=16), SHARDS), (dict(partials=None), NULL), (dict(partials=A + 8), ALIGN), (dict(M=0), OK)])
def test_w4_partials_refuse(L, changes, status):
    assert call(L, "tbik_gemm_shard_partials_w4", W4P, **changes) == status


@pytest.mark.parametrize("changes,status", [
    (dict(M=-1), SHAPE), (dict(H=0), SHAPE), (dict(H=60), SHAPE), (dict(H=65544, ldy=65544, ldr=65544, ldh=65544, ldn=65544), SHAPE), (dict(ldy=56), SHAPE), (dict(ldr=56), SHAPE),
    (dict(ldh=56), SHAPE), (dict(ldn=56), SHAPE), (dict(gate_col=2), SHAPE), (dict(gate_row=-8), SHAPE), (dict(hidden=A, y=A, ldh=72), SHAPE),
    (dict(dtype=F32), DTYPE), (dict(y=None), NULL), (dict(partials=A), NULL), (dict(residual=None), NULL), (dict(hidden=None), NULL), (dict(normed=None), NULL), (dict(next=None), NULL),
    (dict(y=None, partials=A, P=3), SHARDS), (dict(y=None, partials=A, P=32), UNSUPPORTED), (dict(y=A + 8), ALIGN), (dict(residual=A + 8), ALIGN), (dict(hidden=A + 8), ALIGN),
    (dict(normed=A + 8), ALIGN), (dict(post=A + 8), ALIGN), (dict(next=A + 8), ALIGN), (dict(gate=A + 2), ALIGN), (dict(gate_row=4), ALIGN), (dict(ldy=68), ALIGN), (dict(ldn=68), ALIGN),
    (dict(M=0), OK)])
def test_join_refuses(L, changes, status):
    assert call(L, "tbik_rmsnorm_residual_rmsnorm", JOIN, **changes) == status
