"""Plain forms in 64 bits of the calls on rows sorted by expert, on the CPU, and the inputs that the tests of them share."""
from __future__ import annotations

import torch

F8 = torch.float8_e4m3fn
BLOCK = 128
HALF = {torch.float32: 2.0 ** -24, torch.bfloat16: 2.0 ** -8}   # half a step, relative
U = 2.0 ** -24


def pad(n):
    return (n + BLOCK - 1) // BLOCK * BLOCK


def routing(T, k, E, seed, kind="uniform"):
    """[T,k] int32 ids.  uniform: distinct experts a token; misses: about a third -1; one: all the same expert; none: all outside;
    wild: repeated experts and values far outside [0,E)."""
    g = torch.Generator().manual_seed(seed)
    if kind == "one":
        return torch.full((T, k), E - 1, dtype=torch.int32)
    if kind == "none":
        return torch.tensor([-1, E, -2 ** 31, 2 ** 31 - 1], dtype=torch.int32)[torch.randint(0, 4, (T, k), generator=g)]
    if kind == "wild":
        ids = torch.randint(0, E, (T, k), generator=g, dtype=torch.int32)
        ids[torch.rand(T, k, generator=g) < 0.2] = -2 ** 31
        ids[torch.rand(T, k, generator=g) < 0.2] = E
        return ids
    ids = torch.topk(torch.rand(T, E, generator=g), k, dim=1).indices.to(torch.int32)
    if kind == "misses":
        ids[torch.rand(T, k, generator=g) < 0.35] = -1
    return ids


def sort(ids, E):
    """(offsets, order, pos) by definition."""
    flat = ids.reshape(-1).tolist()
    valid = sorted((e, a) for a, e in enumerate(flat) if 0 <= e < E)
    offsets = [sum(1 for e, _ in valid if e < x) for x in range(E + 1)] if E <= 64 else \
        torch.searchsorted(torch.tensor([e for e, _ in valid], dtype=torch.int64), torch.arange(E + 1)).tolist()
    order = [a for _, a in valid] + [-1] * (len(flat) - len(valid))
    pos = [-1] * len(flat)
    for r, (_, a) in enumerate(valid):
        pos[a] = r
    i32 = torch.int32
    return torch.tensor(offsets, dtype=i32), torch.tensor(order, dtype=i32), torch.tensor(pos, dtype=i32).reshape(ids.shape)


def blocks(x, tall=False):
    """(q, scale) of x [..,N,K] by the definition, in 32 bits operation for operation: q [..,N,Kp] e4m3, scale [..,N or ceil(N/128),Kb]."""
    N, K = x.shape[-2:]
    h = BLOCK if tall else 1
    whole = torch.zeros(*x.shape[:-2], -(-N // h) * h, pad(K))
    whole[..., :N, :K] = x.float()
    v = whole.reshape(-1, whole.shape[-2] // h, h, pad(K) // BLOCK, BLOCK)
    m = v.abs().amax(dim=(2, 4), keepdim=True).clamp(min=2.0 ** -100)
    # (448.0 / m would be m's reciprocal times 448: two roundings)
    q = (v * (torch.full_like(m, 448.0) / m)).to(F8).reshape(whole.shape)[..., :N, :]
    return q, (m / 448.0).reshape(*x.shape[:-2], whole.shape[-2] // h, pad(K) // BLOCK)


def matmul(a, sa, w, sw, offsets):
    """(out, sum of magnitudes) in 64 bits, zero rows outside the experts'."""
    M, K = a.shape
    E, N = w.shape[:2]
    a = a.double() * sa.double().repeat_interleave(BLOCK, dim=1)
    out, size = torch.zeros(M, N, dtype=torch.float64), torch.zeros(M, N, dtype=torch.float64)
    for e in range(E):
        lo, hi = max(0, int(offsets[e])), min(M, int(offsets[e + 1]))
        if lo < hi:
            b = w[e].double() * sw[e].double().repeat_interleave(BLOCK, dim=0)[:N].repeat_interleave(BLOCK, dim=1)
            out[lo:hi], size[lo:hi] = a[lo:hi] @ b.t(), a[lo:hi].abs() @ b.abs().t()
    return out, size


def matmul_bound(size, out, K, dtype):
    """128 products of a block and the blocks' sums in 32 bits, a scale's product and its use, the rounding of the result.  bf16
    results come from the 8-bit matrix instruction: of each eight products it cuts seven at 2^-13 of the largest at most, so their sum
    is off by at most 7 * 2^-13 of the largest, and that is at most the sum of the eight magnitudes: 7 * 2^-13 * size in all."""
    cut = 7 * 2.0 ** -13 if dtype == torch.bfloat16 else 0.0
    return ((BLOCK + K // BLOCK + 3) * U + cut) * size + HALF[dtype] * (out.abs() + cut * size) * (1 + 2 ** -8)
