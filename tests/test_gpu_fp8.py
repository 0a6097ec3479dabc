"""Values in 8 bits with a scale for each block of 128, and the experts' products of them, against plain forms on the CPU: the
quantisers bit for bit (their definition in 32 bits) and within half a step (in 64), the products within 64 bits' reach."""
import pytest
import torch

import rows_util as R
from paper_2603_09983_amd import binding as B

pytestmark = pytest.mark.gpu
F8 = R.F8


def _values(M, K, seed, dtype):
    """Normal values with wide and tiny rows, zero blocks, single values."""
    g = torch.Generator().manual_seed(seed)
    x = torch.randn(M, K, generator=g) * torch.exp2(torch.randint(-120, 100, (M, 1), generator=g).float())
    x[torch.rand(M, generator=g) < 0.2] *= 0.0
    one = torch.rand(M, generator=g) < 0.1
    x[one] = 0.0
    x[one, 0] = 1.0
    return x.to(dtype)


def _within_half_a_step(q, scale, x, tall=False, slack=0.0):
    N, K = x.shape[-2:]
    s = scale.double()
    if tall:
        s = s.repeat_interleave(128, dim=-2)[..., :N, :]
    s = s.repeat_interleave(128, dim=-1)[..., :K]
    y = x.double() / s
    # three roundings in 32 bits (the scale, 448 / m, the product) move y by 2^-22 at most; below 2^-6 the step is 2^-9
    bound = torch.maximum(y.abs() * 2 ** -4, torch.tensor(2.0 ** -10, dtype=torch.float64)) * (1 + 2 ** -20) + y.abs() * (2 ** -22 + slack)
    assert bool(((q.double()[..., :K] - y).abs() <= bound).all())
    assert not q.view(torch.uint8)[..., K:].any()   # zeros behind the row


SIZES = [(1, 8), (1, 128), (3, 136), (7, 1000), (16, 2048), (130, 1408), (33, 2040), (2, 16384), (3000, 264)]


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
@pytest.mark.parametrize("M,K", SIZES)
def test_quantize_rows(M, K, dtype):
    x = _values(M, K, M + K, dtype)
    q = torch.full((M, R.pad(K)), 9, dtype=torch.uint8, device="cuda")
    scale = torch.full((M, R.pad(K) // 128), 77.0, device="cuda")
    B.moe_quantize_fp8(x.cuda(), dtype == torch.bfloat16, None, M, K, q, scale)
    q, scale = q.cpu().view(F8), scale.cpu()
    wq, ws = R.blocks(x)
    assert torch.equal(scale, ws) and torch.equal(q.view(torch.uint8), wq.view(torch.uint8))
    _within_half_a_step(q, scale, x)


@pytest.mark.parametrize("n", [-3, 0, 1, 9, 20, 99])
def test_rows_from_n_rows_on_are_left(n):
    M, K = 20, 200
    x = torch.randn(M, 2 * K, generator=torch.Generator().manual_seed(1))
    n_dev = torch.tensor([n], dtype=torch.int32, device="cuda")
    n = min(max(n, 0), M)
    for call, given in ((B.moe_quantize_fp8, x[:, :K].contiguous()), (B.moe_swiglu_fp8, x)):
        q, scale = torch.full((M, 256), 9, dtype=torch.uint8, device="cuda"), torch.full((M, 2), 77.0, device="cuda")
        all_q, all_s = torch.empty_like(q), torch.empty_like(scale)
        call(given.cuda(), False, n_dev, M, K, q, scale)
        call(given.cuda(), False, None, M, K, all_q, all_s)
        assert torch.equal(q[:n], all_q[:n]) and torch.equal(scale[:n], all_s[:n])
        assert bool((q[n:] == 9).all()) and bool((scale[n:] == 77.0).all())


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
@pytest.mark.parametrize("M,F", SIZES)
def test_swiglu(M, F, dtype):
    g = torch.Generator().manual_seed(M + F)
    x = (torch.randn(M, 2 * F, generator=g) * 2).to(dtype)
    x[0, : min(F, 8)] = torch.tensor([0.0, -0.0, 90.0, -90.0, 30.0, -30.0, 1e-30, -1e-30])[: min(F, 8)].to(dtype)
    q = torch.full((M, R.pad(F)), 9, dtype=torch.uint8, device="cuda")
    scale = torch.full((M, R.pad(F) // 128), 77.0, device="cuda")
    B.moe_swiglu_fp8(x.cuda(), dtype == torch.bfloat16, None, M, F, q, scale)
    q, scale = q.cpu().view(F8), scale.cpu()
    gate, up = x.double()[:, :F], x.double()[:, F:]
    y = gate * torch.sigmoid(gate) * up
    # e^-g in 32 bits: its argument times log2(e) is off by |g| 2^-23, its value by two steps; a quotient and two products
    slack = 100 * 2.0 ** -23 + 6 * R.U
    m = torch.nn.functional.pad(y, (0, R.pad(F) - F)).reshape(M, -1, 128).abs().amax(dim=2).clamp(min=2.0 ** -100)
    assert bool(((scale.double() - m / 448).abs() <= m / 448 * (slack + 2 * R.U)).all())
    _within_half_a_step(q, scale, y, slack=slack)


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
@pytest.mark.parametrize("E,N,K", [(1, 8, 8), (2, 128, 128), (3, 130, 200), (2, 1000, 1000), (1, 1, 4096), (5, 384, 264)])
def test_quantize_weights(E, N, K, dtype):
    w = torch.stack([_values(N, K, e + N, dtype) for e in range(E)])
    w[0, : N // 2] = 0.0
    q = torch.full((E, N, R.pad(K)), 9, dtype=torch.uint8, device="cuda")
    scale = torch.full((E, R.pad(N) // 128, R.pad(K) // 128), 77.0, device="cuda")
    B.moe_quantize_weights_fp8(w.cuda(), dtype == torch.bfloat16, E, N, K, q, scale)
    q, scale = q.cpu().view(F8), scale.cpu()
    wq, ws = R.blocks(w, tall=True)
    assert torch.equal(scale, ws) and torch.equal(q.view(torch.uint8), wq.contiguous().view(torch.uint8))
    _within_half_a_step(q, scale, w, tall=True)


def test_blocks_that_are_not_numbers():
    """NaN and infinities mark their own block and no other."""
    x = torch.randn(4, 384, generator=torch.Generator().manual_seed(1))
    clean = x.clone()
    x[1, 130], x[2, 5], x[3, 383] = float("nan"), float("inf"), float("-inf")
    got = []
    for v in (x, clean):
        q, s = torch.empty(4, 384, dtype=torch.uint8, device="cuda"), torch.empty(4, 3, device="cuda")
        B.moe_quantize_fp8(v.cuda(), False, None, 4, 384, q, s)
        got.append((q.cpu().view(F8).float(), s.cpu()))
    (q, s), (cq, cs) = got
    bad = torch.zeros(4, 3, dtype=torch.bool)
    bad[1, 1] = bad[2, 0] = bad[3, 2] = True
    assert torch.equal(s[~bad], cs[~bad]) and torch.isnan(s[1, 1]) and torch.isinf(s[2, 0]) and torch.isinf(s[3, 2])
    wide = bad.repeat_interleave(128, dim=1)
    assert torch.equal(q[~wide], cq[~wide])
    back = q * s.repeat_interleave(128, dim=1)
    assert bool(torch.isnan(back[1, 128:256]).all()) and bool(torch.isnan(back[2, :128]).all()) and bool(torch.isnan(back[3, 256:]).all())


# ---- products ----

def _operands(counts, N, K, seed, lead=0, tail=0):
    """Rows of experts with `counts` rows each, `lead` rows of no expert in front and `tail` behind."""
    g = torch.Generator().manual_seed(seed)
    E, M = len(counts), sum(counts) + lead + tail
    x, w = torch.randn(M, K, generator=g), torch.randn(E, N, K, generator=g) * 0.02
    x[:, ::37] *= 8
    a, sa = R.blocks(x)
    q, sw = R.blocks(w, tall=True)
    offsets = torch.tensor([lead] + [lead + sum(counts[: e + 1]) for e in range(E)], dtype=torch.int32)
    return a, sa, q.contiguous(), sw, offsets


def _run(a, sa, w, sw, offsets, dtype, out=None):
    M, K = a.shape
    E, N = w.shape[:2]
    if out is None:
        out = torch.full((M, N), 77.0, dtype=dtype, device="cuda")
    B.moe_grouped_matmul_fp8(a.cuda(), sa.cuda(), w.cuda(), sw.cuda(), offsets.cuda(), M, N, K, E, out, dtype == torch.bfloat16)
    return out.cpu()


def _check(a, sa, w, sw, offsets, dtype):
    got = _run(a, sa, w, sw, offsets, dtype).double()
    want, size = R.matmul(a, sa, w, sw, offsets)
    M = a.shape[0]
    row = torch.arange(M)
    mine = ((row >= int(offsets[0])) & (row < int(offsets[-1]))).unsqueeze(1)
    want = torch.where(mine, want, 77.0)
    bound = torch.where(mine, R.matmul_bound(size, want, a.shape[1], dtype), 0.0)
    assert bool(((got - want).abs() <= bound).all()), float(((got - want).abs() - bound).max())


COUNTS = [[1], [16], [17], [0, 0, 1, 0], [3, 0, 5, 1, 16, 15], [33, 0, 64, 2], [100, 1, 130], [257], [65, 300, 7], [600, 0, 40]]


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
@pytest.mark.parametrize("N,K", [(8, 128), (136, 256), (1000, 1000), (296, 2048), (520, 1408)])
@pytest.mark.parametrize("counts", COUNTS, ids=[str(sum(c)) + "in" + str(len(c)) for c in COUNTS])
def test_product(counts, N, K, dtype):
    _check(*_operands(counts, N, K, N + K + len(counts)), dtype)


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
@pytest.mark.parametrize("counts,N,K", [([5, 2], 264, 14336), ([0] * 700 + [9] + [0] * 323, 64, 256), ([2] * 300, 72, 384),
                                        ([1500, 1200], 768, 640)])
def test_product_long_sums_many_experts_many_rows(counts, N, K, dtype):
    _check(*_operands(counts, N, K, 11), dtype)


# many rows to an expert and enough of them to fill the device: rows that end anywhere in a tile of 256, widths that end inside one,
# two blocks of columns and more, scales that are whole 16-byte words and not
MANY = [([7 * i * i % 83 for i in range(40)], 1000, 1000), ([7 * i * i % 83 for i in range(40)], 1040, 1408), ([700, 0, 1300], 4104, 640),
        ([5000], 2056, 256), ([0, 3000, 1, 2049], 2312, 384), ([16, 17, 0, 15, 1, 255, 256, 257] * 4, 1032, 512), ([9] * 300, 264, 2176)]


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
@pytest.mark.parametrize("counts,N,K", MANY, ids=[f"{sum(c)}in{len(c)}x{n}x{k}" for c, n, k in MANY])
def test_product_many_rows(counts, N, K, dtype):
    _check(*_operands(counts, N, K, 12), dtype)


# rows enough for tiles, but few of them; more than one to a workgroup, whose steps are fewer than, as many as and more than are ahead
FEW = [([600, 5, 900], 1000, 512), ([700, 0, 1300], 520, 1408), ([700, 0, 1300], 136, 5120), ([700, 0, 1300], 4104, 512),
       ([1, 129, 128, 127, 0, 256] * 3, 1160, 1024), ([40] * 30, 2056, 512), ([19 * i % 61 for i in range(60)], 1032, 640)]


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
@pytest.mark.parametrize("counts,N,K", FEW, ids=[f"{sum(c)}in{len(c)}x{n}x{k}" for c, n, k in FEW])
def test_product_few_tiles(counts, N, K, dtype):
    _check(*_operands(counts, N, K, 14, lead=2, tail=3), dtype)


# few rows and among many experts one or two that have many: their later rows' workgroups are found from the counts
SKEWED = [([0] * 500 + [90] + [1] * 200 + [70] + [0] * 300, 264, 2048), ([1] * 255 + [40, 33] + [0] * 254 + [17, 100], 72, 384),
          ([0] * 600 + [49] + [0] * 300 + [33] + [1] * 20 + [0] * 100, 264, 1024), ([0, 0, 49, 0], 40, 512), ([0] * 60 + [64, 16, 17], 136, 4224)]


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
@pytest.mark.parametrize("counts,N,K", SKEWED, ids=[f"{sum(c)}in{len(c)}x{n}x{k}" for c, n, k in SKEWED])
def test_product_skewed(counts, N, K, dtype):
    _check(*_operands(counts, N, K, 20, lead=1, tail=2), dtype)


def test_product_of_one_block_and_millions_of_rows():
    M, N, K = 2200000, 8, 128
    a, sa, w, sw, _ = _operands([5000], N, K, 21)
    x, sx = a.view(torch.uint8).cuda().repeat(M // 5000, 1), sa.cuda().repeat(M // 5000, 1)
    out = torch.empty(M, N, device="cuda")
    offsets = torch.tensor([0, M], dtype=torch.int32, device="cuda")
    B.moe_grouped_matmul_fp8(x, sx, w.cuda(), sw.cuda(), offsets, M, N, K, 1, out, False)
    got = out.reshape(-1, 5000, N)
    assert torch.equal(got, got[:1].expand_as(got))
    want, size = R.matmul(a, sa, w, sw, torch.tensor([0, 5000]))
    assert bool(((got[0].cpu().double() - want).abs() <= R.matmul_bound(size, want, K, torch.float32)).all())


def test_many_rows_rows_of_no_expert_and_nan():
    a, sa, w, sw, offsets = _operands([300, 0, 700], 4104, 512, 13, lead=5, tail=30)
    _check(a, sa, w, sw, offsets, torch.bfloat16)
    clean = _run(a, sa, w, sw, offsets, torch.bfloat16)
    assert torch.equal(clean, _run(a, sa, w, sw, offsets, torch.bfloat16))
    a.view(torch.uint8)[4, 300] = 0x7f        # of no expert
    a.view(torch.uint8)[304, 300] = 0x7f      # the last row of the first
    sa[700, 1] = float("nan")
    w.view(torch.uint8)[2, 4103, 0] = 0xff
    got = _run(a, sa, w, sw, offsets, torch.bfloat16)
    bad = torch.zeros(got.shape, dtype=torch.bool)
    bad[304], bad[700], bad[305:1005, 4103] = True, True, True
    assert bool(torch.isnan(got[bad]).all()) and torch.equal(got[~bad], clean[~bad])


@pytest.mark.parametrize("lead,tail", [(0, 9), (5, 0), (3, 40)])
def test_rows_of_no_expert_are_left(lead, tail):
    for counts in ([4, 0, 19], [0, 0, 0], [90, 200]):
        _check(*_operands(counts, 264, 256, 5, lead, tail), torch.float32)


def test_offsets_are_clamped():
    """Values below 0 and beyond M count as 0 and M; a descending pair is an expert without rows."""
    a, sa, w, sw, offsets = _operands([10, 12, 14], 72, 256, 6)
    wild = torch.tensor([-5, 10, 22, 2 ** 31 - 1], dtype=torch.int32)
    assert torch.equal(_run(a, sa, w, sw, wild, torch.float32), _run(a, sa, w, sw, offsets, torch.float32))
    down = torch.tensor([22, 10, 22, 36], dtype=torch.int32)
    got = _run(a, sa, w, sw, down, torch.float32)
    assert torch.equal(got[10:], _run(a, sa, w, sw, offsets, torch.float32)[10:]) and bool((got[:10] == 77.0).all())


def test_a_row_is_the_same_whatever_else_is_there():
    """A row's bits go by its expert, not by the rows around it, as long as the call's sizes are the same."""
    a, sa, w, sw, offsets = _operands([20, 3, 41], 136, 512, 7)
    got = _run(a, sa, w, sw, offsets, torch.float32)
    again = _run(a, sa, w, sw, offsets, torch.float32)
    assert torch.equal(got, again)
    other = a.clone()
    other.view(torch.uint8)[20:23] = 0x38
    assert torch.equal(_run(other, sa, w, sw, offsets, torch.float32)[23:], got[23:])


def test_all_values_of_a_byte():
    """Every finite e4m3 value in both operands, at large and small scales."""
    g = torch.Generator().manual_seed(8)
    bits = torch.arange(256, dtype=torch.uint8)
    bits = bits[(bits & 0x7f) != 0x7f]
    a = bits[torch.randint(0, len(bits), (40, 256), generator=g)].view(F8)
    w = bits[torch.randint(0, len(bits), (2, 64, 256), generator=g)].view(F8)
    sa, sw = torch.exp2(torch.randint(-40, 20, (40, 2), generator=g).float()), torch.exp2(torch.randint(-20, 20, (2, 1, 2), generator=g).float())
    _check(a, sa, w, sw, torch.tensor([0, 17, 40], dtype=torch.int32), torch.float32)


def test_nan_stays_in_its_row_or_column():
    a, sa, w, sw, offsets = _operands([20, 30], 264, 512, 9)
    clean = _run(a, sa, w, sw, offsets, torch.float32)
    a.view(torch.uint8)[4, 300] = 0x7f
    sa[33, 1] = float("nan")
    w.view(torch.uint8)[1, 7, 0] = 0xff
    got = _run(a, sa, w, sw, offsets, torch.float32)
    bad = torch.zeros(50, 264, dtype=torch.bool)
    bad[4], bad[33], bad[20:, 7] = True, True, True
    assert bool(torch.isnan(got[bad]).all()) and torch.equal(got[~bad], clean[~bad])


def test_gradient_to_the_rows_is_the_transposed_product():
    """dx = (quantised dout) W: the same call on the transposed weights, whose blocks are the weights' own transposed."""
    g = torch.Generator().manual_seed(10)
    E, N, K, counts = 3, 256, 384, [5, 0, 30]
    w = torch.randn(E, N, K, generator=g) * 0.02
    q, sw = R.blocks(w, tall=True)
    qt, swt = R.blocks(w.transpose(1, 2).contiguous(), tall=True)
    assert torch.equal(qt.view(torch.uint8), q.view(torch.uint8).transpose(1, 2)) and torch.equal(swt, sw.transpose(1, 2))
    d, sd = R.blocks(torch.randn(35, N, generator=g))
    offsets = torch.tensor([0, 5, 5, 35], dtype=torch.int32)
    got = _run(d, sd, qt.contiguous(), swt.contiguous(), offsets, torch.float32).double()
    x = torch.zeros(35, K, dtype=torch.float64, requires_grad=True)
    weights = q.double() * sw.double().repeat_interleave(128, dim=1).repeat_interleave(128, dim=2)
    out = torch.cat([x[int(lo):int(hi)] @ weights[e].t() for e, (lo, hi) in enumerate(zip(offsets, offsets[1:]))])
    dout = d.double() * sd.double().repeat_interleave(128, dim=1)
    (out * dout).sum().backward()
    _, size = R.matmul(d, sd, qt, swt, offsets)
    assert bool(((got - x.grad).abs() <= R.matmul_bound(size, x.grad, N, torch.float32)).all())
    # and by differences: the product is linear in its rows
    step = torch.randn(35, K, generator=g, dtype=torch.float64)
    with torch.no_grad():
        at = lambda s: sum(float(((x + s * step)[int(lo):int(hi)] @ weights[e].t() * dout[int(lo):int(hi)]).sum())
                           for e, (lo, hi) in enumerate(zip(offsets, offsets[1:])))
        slope = (at(1.0) - at(-1.0)) / 2
    assert abs(slope - float((got * step).sum())) <= float((R.matmul_bound(size, x.grad, N, torch.float32) * step.abs()).sum())


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
@pytest.mark.parametrize("counts,N,K", [([i * i % 41 for i in range(1024)], 264, 512), ([i * i % 41 for i in range(1000)], 264, 256)], ids=["1024x512", "1000x256"])
def test_tiles_of_as_many_experts_as_there_can_be(counts, N, K, dtype):
    _check(*_operands(counts, N, K, 15, lead=1, tail=1), dtype)


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
def test_product_of_rows_behind_4_gib(dtype):
    """The last rows of 5 GB, results behind 4 GiB; the rows before them are no expert's."""
    K, M, N = 8192, 600000, 4096
    a, sa, w, sw, _ = _operands([70], N, K, 16)
    x, sx = torch.zeros(M, K, dtype=torch.uint8, device="cuda"), torch.zeros(M, K // 128, device="cuda")
    x[-70:], sx[-70:] = a.view(torch.uint8).cuda(), sa.cuda()
    out = torch.full((M, N), 77.0, dtype=dtype, device="cuda")
    offsets = torch.tensor([M - 70, M], dtype=torch.int32)
    B.moe_grouped_matmul_fp8(x, sx, w.cuda(), sw.cuda(), offsets.cuda(), M, N, K, 1, out, dtype == torch.bfloat16)
    assert bool((out[:-70] == 77.0).all())
    want, size = R.matmul(a, sa, w, sw, torch.tensor([0, 70]))
    assert bool(((out[-70:].cpu().double() - want).abs() <= R.matmul_bound(size, want, K, dtype)).all())


@pytest.mark.parametrize("rows", [3, 40, 200, 700])
def test_product_with_weights_behind_4_gib(rows):
    """The last of 70 experts of 8192 x 8192, whose weights begin behind 4 GiB."""
    N = K = 8192
    E, dtype = 70, torch.bfloat16
    a, sa, w, sw, _ = _operands([rows], N, K, 17)
    all_w, all_s = torch.zeros(E, N, K, dtype=torch.uint8, device="cuda"), torch.zeros(E, N // 128, K // 128, device="cuda")
    all_w[-1], all_s[-1] = w[0].view(torch.uint8).cuda(), sw[0].cuda()
    offsets = torch.zeros(E + 1, dtype=torch.int32, device="cuda")
    offsets[-1] = rows
    out = torch.full((rows, N), 77.0, dtype=dtype, device="cuda")
    B.moe_grouped_matmul_fp8(a.cuda(), sa.cuda(), all_w, all_s, offsets, rows, N, K, E, out, True)
    want, size = R.matmul(a, sa, w, sw, torch.tensor([0, rows]))
    assert bool(((out.cpu().double() - want).abs() <= R.matmul_bound(size, want, K, dtype)).all())


def test_quantisers_behind_4_gib():
    """The last rows and matrices of tensors of 5 to 10 GB."""
    M, K = 600000, 8192
    x = torch.zeros(M, K, dtype=torch.bfloat16, device="cuda")
    rows = _values(9, K, 18, torch.bfloat16)
    x[-9:] = rows.cuda()
    q, scale = torch.empty(M, K, dtype=torch.uint8, device="cuda"), torch.empty(M, K // 128, device="cuda")
    B.moe_quantize_fp8(x, True, None, M, K, q, scale)
    wq, ws = R.blocks(rows)
    assert torch.equal(q[-9:].cpu(), wq.view(torch.uint8)) and torch.equal(scale[-9:].cpu(), ws) and not q[:-9].any()
    E = 70
    w = torch.zeros(E, K, K, dtype=torch.bfloat16, device="cuda")
    last = torch.randn(K, K, generator=torch.Generator().manual_seed(19)).bfloat16()
    w[-1] = last.cuda()
    q, scale = torch.empty(E, K, K, dtype=torch.uint8, device="cuda"), torch.empty(E, K // 128, K // 128, device="cuda")
    B.moe_quantize_weights_fp8(w, True, E, K, K, q, scale)
    wq, ws = R.blocks(last, tall=True)
    assert torch.equal(q[-1].cpu(), wq.contiguous().view(torch.uint8)) and torch.equal(scale[-1].cpu(), ws) and not q[:-1].any()
