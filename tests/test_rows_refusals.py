"""Host-only: the calls on rows sorted by expert refuse what they do not take before anything is launched."""
import ctypes

import pytest

from paper_2603_09983_amd import binding as B

P, BIG = 0x1000, 1 << 30   # (never dereferenced)
NULL, SHAPE, ALIGN, WS = B.ERR_NULL, B.ERR_SHAPE, B.ERR_ALIGN, B.ERR_WORKSPACE
L = B._lib

GOOD = {
    "moe_sort_assignments": [P, 9, 6, 64, P, P, P, P, BIG, None],
    "moe_permute": [P, 1, P, 9, 6, 64, 54, P, None],
    "moe_permute_fp8": [P, 1, P, 9, 6, 64, 54, P, P, None],
    "moe_unpermute": [P, 1, P, P, 9, 6, 64, 54, P, 0, 0, None],
    "moe_unpermute_backward": [P, 1, P, 1, P, P, 9, 6, 64, 54, P, P, None],
    "moe_quantize_fp8": [P, 1, None, 54, 64, P, P, None],
    "moe_swiglu_fp8": [P, 1, None, 54, 64, P, P, None],
    "moe_quantize_weights_fp8": [P, 1, 4, 64, 64, P, P, None],
    "moe_grouped_matmul_fp8": [P, P, P, P, P, 54, 64, 128, 4, P, 1, None],
}
BAD = [
    # call, argument, value, status
    *[("moe_sort_assignments", i, None, NULL) for i in (0, 4, 5, 6, 7)],
    *[("moe_sort_assignments", i, 0, SHAPE) for i in (1, 2, 3)],
    ("moe_sort_assignments", 3, 1025, SHAPE), ("moe_sort_assignments", 1, 1 << 30, SHAPE),
    ("moe_sort_assignments", 7, P + 8, ALIGN), ("moe_sort_assignments", 8, 64, WS),
    *[(f, i, None, NULL) for f, at in (("moe_permute", (0, 2, 7)), ("moe_permute_fp8", (0, 2, 7, 8)), ("moe_unpermute", (0, 2, 8)),
                                       ("moe_unpermute_backward", (0, 2, 4)), ("moe_quantize_fp8", (0, 5, 6)),
                                       ("moe_swiglu_fp8", (0, 5, 6)), ("moe_quantize_weights_fp8", (0, 5, 6)),
                                       ("moe_grouped_matmul_fp8", (0, 1, 2, 3, 4, 9))) for i in at],
    *[(f, i, v, SHAPE) for f, at in (("moe_permute", (3, 4, 5, 6)), ("moe_permute_fp8", (3, 4, 5, 6)), ("moe_unpermute", (4, 5, 6, 7)),
                                     ("moe_unpermute_backward", (6, 7, 8, 9)), ("moe_quantize_fp8", (3, 4)), ("moe_swiglu_fp8", (3, 4)),
                                     ("moe_quantize_weights_fp8", (2, 3, 4)), ("moe_grouped_matmul_fp8", (5, 6, 7, 8)))
      for i in at for v in (0, -1)],
    *[(f, i, v, ALIGN) for f, i, v in (("moe_permute", 5, 60), ("moe_permute", 0, P + 8), ("moe_permute", 7, P + 2),
                                       ("moe_permute_fp8", 5, 60), ("moe_permute_fp8", 0, P + 8), ("moe_permute_fp8", 7, P + 8),
                                       ("moe_unpermute", 6, 60), ("moe_unpermute", 0, P + 8), ("moe_unpermute", 8, P + 8),
                                       ("moe_unpermute_backward", 8, 60), ("moe_unpermute_backward", 0, P + 8),
                                       ("moe_unpermute_backward", 2, P + 8), ("moe_unpermute_backward", 10, P + 8),
                                       ("moe_quantize_fp8", 4, 60), ("moe_quantize_fp8", 0, P + 8), ("moe_quantize_fp8", 5, P + 8),
                                       ("moe_swiglu_fp8", 4, 60), ("moe_swiglu_fp8", 0, P + 4), ("moe_swiglu_fp8", 5, P + 8),
                                       ("moe_quantize_weights_fp8", 4, 60), ("moe_quantize_weights_fp8", 0, P + 8),
                                       ("moe_quantize_weights_fp8", 5, P + 8), ("moe_grouped_matmul_fp8", 7, 136),
                                       ("moe_grouped_matmul_fp8", 6, 60), ("moe_grouped_matmul_fp8", 0, P + 8),
                                       ("moe_grouped_matmul_fp8", 2, P + 8), ("moe_grouped_matmul_fp8", 9, P + 8))],
    ("moe_quantize_weights_fp8", 2, 1025, SHAPE), ("moe_grouped_matmul_fp8", 8, 1025, SHAPE),
    ("moe_permute", 3, 1 << 30, SHAPE), ("moe_unpermute", 4, 1 << 30, SHAPE), ("moe_unpermute_backward", 6, 1 << 30, SHAPE),
    # more blocks than the kernels' 32-bit counts hold
    ("moe_quantize_fp8", 3, 1 << 30, None), ("moe_quantize_weights_fp8", 3, 1 << 24, None),
]


@pytest.mark.parametrize("call,at,value,status", BAD)
def test_refused(call, at, value, status):
    args = list(GOOD[call])
    args[at] = value
    if status is None:   # (one size alone does not pass the bound)
        args[4] = 1 << 24
        status = SHAPE
    assert getattr(L, call)(*args) == status
    assert B.moe_status_string(status)


def test_gradient_needs_an_output_and_its_inputs():
    f = L.moe_unpermute_backward
    assert f(P, 1, P, 1, P, P, 9, 6, 64, 54, None, None, None) == NULL
    assert f(P, 1, None, 1, P, P, 9, 6, 64, 54, P, P, None) == NULL   # rows are what dtopk_w comes from


def test_sort_workspace_bytes():
    n = ctypes.c_size_t(0)
    assert L.moe_sort_workspace_bytes(9, 6, 64, None) == NULL
    assert L.moe_sort_workspace_bytes(9, 6, 1025, ctypes.byref(n)) == SHAPE
    for T, k, E in ((1, 1, 1), (9, 6, 64), (16384, 8, 1024), (1 << 27, 8, 512)):
        assert 0 < B.moe_sort_workspace_bytes(T, k, E) <= 1 << 20
        assert L.moe_sort_assignments(P, T, k, E, P, P, P, P, B.moe_sort_workspace_bytes(T, k, E) - 1, None) == WS
    with pytest.raises(B.MoeError):
        B.moe_sort_workspace_bytes(9, 6, 0)


@pytest.mark.parametrize("name", B.ROWS_EXPORTS)
def test_declared_and_exported(name):
    import os
    root = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
    text = open(os.path.join(root, "include", "moe_spac.h")).read()
    assert f"int {name}(" in text and name in B.EXPORTS and hasattr(L, name)
