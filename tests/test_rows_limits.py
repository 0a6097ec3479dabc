"""Host-only: limits on sizes together, where each alone passes."""
import pytest

from paper_2603_09983_amd import binding as B
from test_rows_refusals import GOOD, L, SHAPE

LIMITS = [
    # call, {argument: value}
    ("moe_permute", {3: 1 << 30, 4: 1, 5: 2056}),            # T * ceil(H/2048), bf16
    ("moe_permute", {1: 0, 3: 1 << 30, 4: 1, 5: 1032}),      # T * ceil(H/1024), fp32
    ("moe_permute_fp8", {3: 1 << 30, 4: 1, 5: 136}),         # T * ceil(H/128)
    ("moe_permute_fp8", {3: 1, 4: 1, 5: (1 << 24) + 8}),     # H as a row that moe_quantize_fp8 takes
    ("moe_unpermute", {4: 1 << 30, 5: 1, 6: 520}),           # T * ceil(H/512)
    ("moe_quantize_fp8", {3: 1 << 30, 4: 136}),              # M * ceil(K/128)
    ("moe_quantize_fp8", {3: 1, 4: (1 << 24) + 8}),
    ("moe_swiglu_fp8", {3: 1 << 30, 4: 136}),
    ("moe_swiglu_fp8", {3: 1, 4: (1 << 24) + 8}),
    ("moe_quantize_weights_fp8", {2: 1024, 3: 1 << 20, 4: 1 << 15}),   # E * ceil(N/128) * ceil(K/128)
    ("moe_quantize_weights_fp8", {3: (1 << 24) + 8}),
    ("moe_grouped_matmul_fp8", {5: 1 << 30, 6: 16384, 8: 1}),   # (ceil(M/128) + E) * ceil(N/128)
    ("moe_grouped_matmul_fp8", {6: (1 << 24) + 8}),
    ("moe_grouped_matmul_fp8", {7: (1 << 20) + 128}),
]


@pytest.mark.parametrize("call,sizes", LIMITS, ids=[f"{c}{i}" for i, (c, _) in enumerate(LIMITS)])
def test_sizes_beyond_the_limits(call, sizes):
    args = list(GOOD[call])
    for at, value in sizes.items():
        args[at] = value
    assert getattr(L, call)(*args) == SHAPE
    assert B.moe_status_string(SHAPE)
