"""Products of so many tiles that every workgroup of the tile kernels walks several: the loads of a tile's first steps go out during the tile
before, its results are stored while they are under way, and which half of LDS a step has goes on from tile to tile."""
import pytest
import torch

import rows_util as R
from paper_2603_09983_amd import binding as B
from test_gpu_fp8_sums import _call, _exact, _normal

pytestmark = pytest.mark.gpu

RAGGED = [3001, 1, 0, 7000, 255, 257, 5120, 4000]
EVEN = [2560] * 8
FEW = [7 * i * i % 61 for i in range(64)]
# rows, N, K: two blocks of columns, three, four, five (no multiple of four), eight, eleven; few rows to an expert, in tiles of 128 x 128
CALLS = [(RAGGED, 4104, 256), (EVEN, 4096, 256), (RAGGED, 4104, 384), (RAGGED, 4096, 512), (RAGGED, 4104, 640), (EVEN, 4120, 1024),
         (RAGGED, 2312, 1408),
         (FEW, 1160, 640), (FEW, 2056, 512), ([24] * 60, 1288, 1152)]
IDS = [f"{sum(c)}x{n}x{k}" for c, n, k in CALLS]


@pytest.mark.parametrize("out_bf16", [0, 1, B.BF16_SHORT_SUMS], ids=["fp32", "bf16", "short"])
@pytest.mark.parametrize("counts,N,K", CALLS, ids=IDS)
def test_several_tiles_to_a_workgroup(counts, N, K, out_bf16):
    cus = torch.cuda.get_device_properties(0).multi_processor_count
    tile = 256 if sum(counts) > 100 * len(counts) else 128   # (the largest that may be taken)
    assert sum(-(-n // tile) for n in counts) * -(-N // tile) > 2 * cus
    ops = _normal(counts, N, K, N + K)
    want, size = _exact(*ops, counts)
    got = _call(*ops, counts, out_bf16)
    assert torch.equal(got, _call(*ops, counts, out_bf16))
    if out_bf16 == 0:
        assert float((got - want).norm()) <= 2.0 ** -20 * float(want.norm())
        dtype = torch.float32
    else:
        dtype = torch.bfloat16
        # one result in a thousand beside the nearest with 32-bit sums (bound as where these are tested), else what passes half a step
        if out_bf16 == 1:
            assert float((got != want.bfloat16().double()).double().mean()) <= 2.0 ** -9
        half = 2.0 ** -8 * torch.exp2(torch.floor(torch.log2(got.abs().clamp(min=2.0 ** -120))))
        assert float(((got - want).abs() - half).clamp(min=0).norm()) <= 2.0 ** -13.5 * float(want.norm())
    for lo in range(0, want.shape[0], 4096):
        rows = slice(lo, lo + 4096)
        assert bool(((got[rows] - want[rows]).abs() <= R.matmul_bound(size[rows], want[rows], K, dtype)).all())
