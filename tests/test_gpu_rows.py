"""Sorting assignments by expert, moving rows into that order and back with weights, and the gradient, against plain forms in
64 bits on the CPU."""
import pytest
import torch

import rows_util as R
from paper_2603_09983_amd import binding as B

pytestmark = pytest.mark.gpu
I32 = dict(dtype=torch.int32, device="cuda")


def dev_sort(ids, E, stream=None):
    T, k = ids.shape
    off, order, pos = torch.full((E + 1,), -9, **I32), torch.full((T * k,), -9, **I32), torch.full((T, k), -9, **I32)
    ws = torch.full((B.moe_sort_workspace_bytes(T, k, E),), 255, dtype=torch.uint8, device="cuda")
    B.moe_sort_assignments(ids.cuda(), T, k, E, off, order, pos, ws, stream=stream)
    return off, order, pos


KINDS = ["uniform", "misses", "one", "none", "wild"]
SORTS = [(1, 1, 1), (1, 6, 64), (9, 6, 64), (64, 1, 2), (65, 1, 3), (1024, 1, 5), (1025, 1, 1), (33, 31, 64), (1000, 4, 60),
         (1024, 4, 7), (4097, 1, 64), (1366, 6, 128), (700, 8, 1024), (5000, 8, 1000), (4096, 8, 512)]


@pytest.mark.parametrize("T,k,E,kind", [(*s, kind) for s in SORTS for kind in KINDS] +
                         [(33000, 8, 40, "wild"), (33000, 8, 40, "one"), (300000, 1, 3, "uniform"), (300000, 1, 3, "none")])
def test_sort(T, k, E, kind):
    ids = R.routing(T, k, E, T + k + E, kind)
    got = dev_sort(ids, E)
    for name, g, want in zip(("offsets", "order", "pos"), got, R.sort(ids, E)):
        assert torch.equal(g.cpu(), want), name


@pytest.mark.parametrize("T,k,E,kind", [(T, k, E, kind) for T, k, E in ((16384, 1, 64), (16385, 1, 64), (2730, 6, 1000), (2731, 6, 9), (1023, 2, 1024))
                                        for kind in ("uniform", "misses", "wild")])
def test_sort_around_the_ends_of_one_launch(T, k, E, kind):
    test_sort(T, k, E, kind)


def _pos(T, k, extra, seed, misses=True):
    """Distinct rows of T*k + extra at random for the assignments, a few of them outside (negative, beyond the end)."""
    g = torch.Generator().manual_seed(seed)
    n = T * k + extra
    pos = torch.randperm(n, generator=g)[: T * k].to(torch.int32).reshape(T, k)
    if misses:
        pos[torch.rand(T, k, generator=g) < 0.2] = -1
        pos[torch.rand(T, k, generator=g) < 0.1] = n
        pos[torch.rand(T, k, generator=g) < 0.05] = 2 ** 31 - 1
    return pos, n


ROWS = [(1, 1, 8), (1, 6, 2048), (1, 1, 16384), (3, 2, 2040), (9, 6, 64), (37, 3, 1000), (130, 8, 520), (1100, 2, 4096), (2500, 1, 24), (300, 64, 136)]


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
@pytest.mark.parametrize("T,k,H", ROWS)
def test_permute(T, k, H, dtype):
    pos, n = _pos(T, k, 5, T + H)
    x = torch.randn(T, H, generator=torch.Generator().manual_seed(1)).to(dtype)
    out = torch.full((n, H), 77.0, dtype=dtype, device="cuda")
    B.moe_permute(x.cuda(), dtype == torch.bfloat16, pos.cuda(), T, k, H, n, out)
    want = torch.full((n, H), 77.0, dtype=dtype)
    t, j = ((pos >= 0) & (pos < n)).nonzero(as_tuple=True)
    want[pos[t, j].long()] = x[t]
    assert torch.equal(out.cpu(), want)


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
@pytest.mark.parametrize("T,k,H", ROWS)
def test_permute_fp8(T, k, H, dtype):
    pos, n = _pos(T, k, 5, T + H)
    x = (torch.randn(T, H, generator=torch.Generator().manual_seed(2)) * 3).to(dtype)
    q = torch.full((n, R.pad(H)), 9, dtype=torch.uint8, device="cuda")
    scale = torch.full((n, R.pad(H) // 128), 77.0, device="cuda")
    B.moe_permute_fp8(x.cuda(), dtype == torch.bfloat16, pos.cuda(), T, k, H, n, q, scale)
    wq, ws = R.blocks(x)
    want_q, want_s = torch.full(q.shape, 9, dtype=torch.uint8), torch.full(scale.shape, 77.0)
    t, j = ((pos >= 0) & (pos < n)).nonzero(as_tuple=True)
    want_q[pos[t, j].long()], want_s[pos[t, j].long()] = wq.view(torch.uint8)[t], ws[t]
    assert torch.equal(q.cpu(), want_q) and torch.equal(scale.cpu(), want_s)


def _picked(rows, pos, n):
    here = (pos >= 0) & (pos < n)
    return torch.where(here.unsqueeze(2), rows.double()[pos.clamp(0, n - 1).long()], 0.0)


@pytest.mark.parametrize("accumulate", [False, True])
@pytest.mark.parametrize("din,dout", [(torch.bfloat16, torch.float32), (torch.bfloat16, torch.bfloat16), (torch.float32, torch.float32),
                                      (torch.float32, torch.bfloat16)])
@pytest.mark.parametrize("T,k,H", ROWS)
def test_unpermute(T, k, H, din, dout, accumulate):
    pos, n = _pos(T, k, 5, T + H)
    g = torch.Generator().manual_seed(3)
    rows, w = torch.randn(n, H, generator=g).to(din), torch.rand(T, k, generator=g)
    was = torch.randn(T, H, generator=g).to(dout)
    for weights in (w, None):
        out = was.cuda()
        B.moe_unpermute(rows.cuda(), din == torch.bfloat16, pos.cuda(), None if weights is None else w.cuda(), T, k, H, n, out,
                        dout == torch.bfloat16, accumulate)
        terms = _picked(rows, pos, n) * (1.0 if weights is None else w.double().unsqueeze(2))
        want, size = terms.sum(dim=1), terms.abs().sum(dim=1)
        if accumulate:
            want, size = want + was.double(), size + was.double().abs()
        # k products and sums in 32 bits, and the rounding of the result
        bound = (k + 1) * R.U * size + R.HALF[dout] * want.abs() * (1 + 2 ** -8)
        assert bool(((out.cpu().double() - want).abs() <= bound).all())


@pytest.mark.parametrize("drow,dout", [(torch.bfloat16, torch.float32), (torch.bfloat16, torch.bfloat16), (torch.float32, torch.float32),
                                       (torch.float32, torch.bfloat16)])
@pytest.mark.parametrize("T,k,H", ROWS)
def test_unpermute_backward(T, k, H, drow, dout):
    pos, n = _pos(T, k, 5, T + H)
    g = torch.Generator().manual_seed(4)
    rows, w, d = torch.randn(n, H, generator=g).to(drow), torch.rand(T, k, generator=g), torch.randn(T, H, generator=g).to(dout)
    drows, dw = torch.full((n, H), 77.0, dtype=drow, device="cuda"), torch.full((T, k), 77.0, device="cuda")
    args = (d.cuda(), dout == torch.bfloat16, rows.cuda(), drow == torch.bfloat16, pos.cuda())
    B.moe_unpermute_backward(*args, w.cuda(), T, k, H, n, drows, dw)
    terms = _picked(rows, pos, n) * d.double().unsqueeze(1)
    want, size = terms.sum(dim=2), terms.abs().sum(dim=2)
    assert bool(((dw.cpu().double() - want).abs() <= H * R.U * size).all())   # (H products and sums)
    t, j = ((pos >= 0) & (pos < n)).nonzero(as_tuple=True)
    want = torch.full((n, H), 77.0, dtype=torch.float64)
    want[pos[t, j].long()] = w[t, j].double().unsqueeze(1) * d[t].double()
    named = torch.zeros(n, dtype=torch.bool)
    named[pos[t, j].long()] = True
    bound = (R.U + R.HALF[drow] * (1 + 2 ** -8)) * want.abs() * named.unsqueeze(1)
    assert bool(((drows.cpu().double() - want).abs() <= bound).all())
    # one output alone, and weights of one
    only, ones = torch.full_like(drows, 77.0), torch.full_like(drows, 77.0)
    B.moe_unpermute_backward(args[0], args[1], None, args[3], args[4], w.cuda(), T, k, H, n, only, None)
    dw2 = torch.full_like(dw, 77.0)
    B.moe_unpermute_backward(*args, w.cuda(), T, k, H, n, None, dw2)
    B.moe_unpermute_backward(*args, None, T, k, H, n, ones, None)
    assert torch.equal(only, drows) and torch.equal(dw2, dw)
    want = torch.full((n, H), 77.0, dtype=drow)
    want[pos[t, j].long()] = d[t].to(drow)
    assert torch.equal(ones.cpu(), want)


def test_gradient_against_differences():
    """out is linear in rows and in w: a step along either changes <dout, out> by the gradient's product with the step."""
    T, k, H = 21, 4, 264
    pos, n = _pos(T, k, 3, 8)
    g = torch.Generator().manual_seed(5)
    rows, w, d = torch.randn(n, H, generator=g), torch.rand(T, k, generator=g), torch.randn(T, H, generator=g)
    srows, sw = torch.randn(n, H, generator=g), torch.rand(T, k, generator=g)
    drows, dw = torch.zeros(n, H, device="cuda"), torch.zeros(T, k, device="cuda")
    B.moe_unpermute_backward(d.cuda(), False, rows.cuda(), False, pos.cuda(), w.cuda(), T, k, H, n, drows, dw)

    def value(r, v):
        out = torch.empty(T, H, device="cuda")
        B.moe_unpermute(r.cuda(), False, pos.cuda(), v.cuda(), T, k, H, n, out, False, False)
        return float((out.cpu().double() * d.double()).sum())

    def size(r, v):
        return float(((_picked(r, pos, n).abs() * v.double().abs().unsqueeze(2)).sum(dim=1) * d.double().abs()).sum())
    for step, grad, at in ((srows, drows, lambda s: (rows + s * srows, w)), (sw, dw, lambda s: (rows, w + s * sw))):
        up, down = at(1.0), at(-1.0)
        slope = (value(*up) - value(*down)) / 2
        want = float((grad.cpu().double() * step.double()).sum())
        # inputs' and outputs' roundings on both sides, the gradient's own
        bound = ((k + 3) * R.U) * (size(*up) + size(*down)) + H * R.U * (size(srows, w) + size(rows, sw))
        assert abs(slope - want) <= bound


def test_gradient_of_permute_is_the_sum_back():
    T, k, H = 40, 3, 128
    pos, n = _pos(T, k, 0, 9)
    d = torch.randn(n, H, generator=torch.Generator().manual_seed(6))
    dx = torch.empty(T, H, device="cuda")
    B.moe_unpermute(d.cuda(), False, pos.cuda(), None, T, k, H, n, dx, False, False)
    x = torch.zeros(T, H, dtype=torch.float64, requires_grad=True)
    t, j = ((pos >= 0) & (pos < n)).nonzero(as_tuple=True)
    (x[t] * d.double()[pos[t, j].long()]).sum().backward()
    assert bool(((dx.cpu().double() - x.grad).abs() <= (k + 1) * R.U * _picked(d, pos, n).abs().sum(dim=1)).all())


def test_rows_behind_4_gib():
    """Rows whose byte offsets pass 32 bits: the last rows of a 5 GB tensor."""
    H, n = 8192, 330000
    rows = torch.zeros(n, H, dtype=torch.bfloat16, device="cuda")
    x = torch.randn(3, H, generator=torch.Generator().manual_seed(7)).bfloat16()
    pos = torch.tensor([[n - 1, 5], [n - 7, 262144], [262143, -1]], dtype=torch.int32)
    B.moe_permute(x.cuda(), True, pos.cuda(), 3, 2, H, n, rows)
    for t in range(3):
        for j in range(2):
            if pos[t, j] >= 0:
                assert torch.equal(rows[int(pos[t, j])].cpu(), x[t])
    assert int((rows != 0).any(dim=1).sum()) == 5
    out = torch.empty(3, H, dtype=torch.bfloat16, device="cuda")
    B.moe_unpermute(rows, True, pos.cuda(), None, 3, 2, H, n, out, True, False)
    want = torch.stack([x[0].float() * 2, x[1].float() * 2, x[2].float()]).bfloat16()
    assert torch.equal(out.cpu(), want)
    d = torch.empty(3, 2, device="cuda")
    B.moe_unpermute_backward(x.cuda(), True, rows, True, pos.cuda(), None, 3, 2, H, n, None, d)
    want = (x.double() ** 2).sum(dim=1)
    assert bool(((d.cpu().double()[:, 0] - want).abs() <= H * R.U * want).all()) and float(d[2, 1]) == 0.0
