"""The plans of products that have been timed stay those that were timed (no device is needed): every row of
profiles/tile_split_plans.csv, and shapes whose plan hangs on the rule's K split, which goes on while there are fewer work items
than compute units; the gate/up product's, while there are no more."""
import csv
import os

import pytest

TABLE = os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "profiles", "tile_split_plans.csv")
KINDS = {"bf16": "bf16", "fp32": "f32", "fp8 e4m3": "fp8", "mxfp8 e4m3": "mxfp8", "mxfp4": "mxfp4", "mxfp6 e2m3": "mxfp6"}


@pytest.fixture(scope="module")
def tb():
    from paper_2511_17826_amd import binding
    if not os.path.exists(binding.LIB_PATH):
        from paper_2511_17826_amd import build
        build.build()
    binding.lib()
    return binding


def piece(p):
    return "slices" if p[1] == "slices" else "%d/%d" % (p[2], p[3])


@pytest.mark.parametrize("operands", sorted(KINDS))
def test_plans_are_the_timed_ones(tb, operands):
    with open(TABLE) as f:
        rows = [r for r in csv.DictReader(f) if r["operands"] == operands]
    assert len(rows) >= 84
    other = []
    for r in rows:
        M, N, K, ns = (int(r[c]) for c in ("M", "N", "K", "superleaves"))
        k_first = 3 if K // ns % 3 == 0 else 1
        got = tb.gemm_route(KINDS[operands], M, N, K, K // ns // k_first, k_first)
        plan = piece(got[0]) + (" + %d rows %s" % (got[1][0], piece(got[1])) if len(got) > 1 else "")
        if plan != r["plan"]:
            other.append((K, N, M, plan, r["plan"]))
    assert not other


@pytest.mark.parametrize("kind,M,N,K,plan", [
    ("f32", 2, 6144, 4096, "32/8"), ("f32", 16, 6144, 4096, "32/8"), ("f32", 32, 6144, 4096, "32/8"),
    ("mxfp8", 60, 6144, 4096, "32/2"), ("bf16", 32, 12288, 4096, "32/4"), ("bf16", 144, 6144, 4096, "32/1"), ("bf16", 320, 4096, 4096, "64/1")])
def test_plans_at_the_rules_split(tb, kind, M, N, K, plan):
    assert [piece(p) for p in tb.gemm_route(kind, M, N, K, 256, 1)] == [plan]


@pytest.mark.parametrize("M,I,K,split", [(1, 2560, 4096, 4), (128, 2560, 4096, 4), (129, 2560, 4096, 2), (192, 2560, 4096, 2), (200, 4096, 4096, 1), (1, 2048, 4096, 8)])
def test_swiglu_splits_into_one_round(tb, M, I, K, split):
    """40 tiles are split in four, 80 in two, 32 in eight: no more items than compute units.  One round of 64-row tiles is not split: gate and up
    in 16 bits."""
    assert tb.lib().tbik_gemm_swiglu_workspace_bytes(M, I, K, 256, 1) == (split * M * 2 * I * 4 if split > 1 else M * 2 * I * 2)
