"""The operators around a mixture of experts, 4-bit weights and the norms around a block are names of the package, like those around
8-bit rows and epilogues, and are the binding's own."""
import pytest


@pytest.mark.parametrize("name", ["tbik_route_topk", "tbik_gemm_grouped", "tbik_gemm_grouped_swiglu", "tbik_gemm_grouped_shard_partials", "tbik_combine_experts",
                                  "tbik_gemm_w4", "tbik_gemm_shard_partials_w4", "tbik_rmsnorm_residual_rmsnorm", "tbik_silu_mul_fp8", "tbik_gemm_epilogue"])
def test_the_package_has_the_call(name):
    import paper_2511_17826_amd as package
    from paper_2511_17826_amd import binding
    assert getattr(package, name) is getattr(binding, name)
