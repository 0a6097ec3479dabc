"""Sums of the grouped product in 8 bits, whose error a rounding to bf16 hides from a test that allows for one: 32 bits for both types of
results, and the 8-bit matrix instruction's where the caller asks for them."""
import pytest
import torch

import rows_util as R
from paper_2603_09983_amd import binding as B

pytestmark = pytest.mark.gpu
F8 = R.F8

# rows to an expert, N, K: few rows (streamed), tiles of 128 x 128, of 256 x 128, of 256 x 256, one block of columns
CALLS = [([5, 0, 2], 264, 2048), ([40, 20], 136, 256), ([600, 5, 900], 1000, 512), ([100] * 20, 2056, 256), ([700, 0, 1300], 4104, 640),
         ([300, 7], 72, 128)]
IDS = [f"{sum(c)}in{len(c)}x{n}x{k}" for c, n, k in CALLS]


def _offsets(counts):
    return torch.tensor([sum(counts[:e]) for e in range(len(counts) + 1)], dtype=torch.int32, device="cuda")


def _call(a, sa, w, sw, counts, out_bf16):
    M, K = a.shape
    E, N = w.shape[:2]
    out = torch.full((M, N), 77.0, dtype=torch.bfloat16 if out_bf16 else torch.float32, device="cuda")
    B.moe_grouped_matmul_fp8(a, sa, w, sw, _offsets(counts), M, N, K, E, out, out_bf16)
    return out.double()


def _exact(a, sa, w, sw, counts):
    """(results, sums of magnitudes) in 64 bits."""
    x = a.double() * sa.double().repeat_interleave(128, dim=1)
    out, size, lo = [], [], 0
    for e, n in enumerate(counts):
        y = w[e].double() * sw[e].double().repeat_interleave(128, dim=0)[: w.shape[1]].repeat_interleave(128, dim=1)
        out.append(x[lo: lo + n] @ y.t())
        size.append(x[lo: lo + n].abs() @ y.abs().t())
        lo += n
    return torch.cat(out), torch.cat(size)


def _cancelling(counts, N, K, seed):
    """The first two columns of each eight are 448 * 448 and -448 * 448, the six others products of 1 to 6.25."""
    g = torch.Generator().manual_seed(seed)
    M, E = sum(counts), len(counts)
    a, w = 1 + 1.5 * torch.rand(M, K, generator=g), 1 + 1.5 * torch.rand(E, N, K, generator=g)
    a[:, 0::8], a[:, 1::8], w[:, :, 0::8], w[:, :, 1::8] = 448.0, -448.0, 448.0, 448.0
    ones = lambda *s: torch.ones(*s, device="cuda")
    return a.to(F8).cuda(), ones(M, R.pad(K) // 128), w.to(F8).cuda(), ones(E, R.pad(N) // 128, R.pad(K) // 128)


def _normal(counts, N, K, seed):
    g = torch.Generator().manual_seed(seed)
    a, sa = R.blocks(torch.randn(sum(counts), K, generator=g))
    w, sw = R.blocks(torch.randn(len(counts), N, K, generator=g) * 0.02, tall=True)
    return a.cuda(), sa.cuda(), w.contiguous().cuda(), sw.cuda()


@pytest.mark.parametrize("out_bf16", [False, True])
@pytest.mark.parametrize("counts,N,K", CALLS, ids=IDS)
def test_small_products_beside_large_ones_that_cancel(counts, N, K, out_bf16):
    """The results are the small products' sums, which cutting at 2^-13 of 2^8 * 2^8 = 8 takes away whole.  The bound is that of fp32
    results (128 products of a block and the blocks' sums in 32 bits) and the result's own rounding."""
    ops = _cancelling(counts, N, K, 1)
    want, size = _exact(*ops, counts)
    dtype = torch.bfloat16 if out_bf16 else torch.float32
    sums = R.matmul_bound(size, torch.zeros_like(want), K, torch.float32)
    bound = sums + R.HALF[dtype] * (want.abs() + sums)
    assert float(bound.max()) < 0.5 * float(want.min())   # (results without the small products would not pass)
    got = _call(*ops, counts, out_bf16)
    assert bool(((got - want).abs() <= bound).all()), float(((got - want).abs() - bound).max())


@pytest.mark.parametrize("counts,N,K", CALLS, ids=IDS)
def test_results_are_the_nearest_of_their_type(counts, N, K):
    """Normal values.  A sum of 128 products a block and of the blocks is off by a walk of some 144 roundings of 2^-24 of its size, 12 * 2^-24
    of the results' norm: the bound of fp32 results is 2^-20.  A bf16 result is not the nearest where the sum lies within its error of the
    middle between two: error / step, 1 / step at most 2^8 / |result|, whose mean over normal results (down to the error) is
    2^8 * 0.8 * ln(1 / (2^8 * error)): 1.2 of a thousand for an error of 12 * 2^-24.  Bound: 2^-9."""
    ops = _normal(counts, N, K, 2)
    want, _ = _exact(*ops, counts)
    assert float((_call(*ops, counts, False) - want).norm()) <= 2.0 ** -20 * float(want.norm())
    other = _call(*ops, counts, True) != want.bfloat16().double()
    assert float(other.double().mean()) <= 2.0 ** -9


@pytest.mark.parametrize("counts,N,K", CALLS, ids=IDS)
def test_short_sums(counts, N, K):
    """Where they are asked for: within their own bound on any values, and beside the rounding to bf16 within 2^-13.5 of the norm on normal
    ones (seven of eight products cut at 2^-13 of the largest, about 3 times their rms: sqrt(7 / 3) * 3 * 2^-13 / sqrt(8) = 2^-12.3 of the
    norm for a cut of any sign, if all of it were seen behind a rounding of 2^-9; seen is what passes half a step, less than half)."""
    for ops in (_cancelling(counts, N, K, 3), _normal(counts, N, K, 4)):
        want, size = _exact(*ops, counts)
        got = _call(*ops, counts, B.BF16_SHORT_SUMS)
        assert bool(((got - want).abs() <= R.matmul_bound(size, want, K, torch.bfloat16)).all())
    half = 2.0 ** -8 * torch.exp2(torch.floor(torch.log2(got.abs().clamp(min=2.0 ** -120))))
    assert float(((got - want).abs() - half).clamp(min=0).norm()) <= 2.0 ** -13.5 * float(want.norm())
