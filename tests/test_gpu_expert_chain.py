"""The experts of a batch in 8 bits, as a program runs them: routing, slots, sort, rows quantised into expert order, gate and up
products, SwiGLU, down product, back into token order with the gate weights; eager, on a stream of its own, captured and replayed,
and two captured chains with workspaces of their own."""
import pytest
import torch

import rows_util as R
from paper_2603_09983_amd import binding as B

pytestmark = pytest.mark.gpu
F8 = R.F8


class Chain:
    def __init__(self, T, H, E, k, F, C, seed):
        g = torch.Generator().manual_seed(seed)
        self.sizes = T, H, E, k, F, C
        bf = lambda *s, std=1.0: (torch.randn(*s, generator=g) * std).bfloat16().cuda()
        self.x, self.w1, self.w2 = bf(T, H), bf(C, 2 * F, H, std=0.05), bf(C, H, F, std=0.05)
        self.router = (torch.randn(E, H, generator=g) * 0.05).cuda()
        table = torch.full((E,), -1, dtype=torch.int32)
        table[torch.randperm(E, generator=g)[:C]] = torch.arange(C, dtype=torch.int32)
        self.table = table.cuda()
        A, i32 = T * k, dict(dtype=torch.int32, device="cuda")
        self.topk_idx, self.topk_w = torch.empty(T, k, **i32), torch.empty(T, k, device="cuda")
        self.slot_idx, self.miss, self.n_miss = torch.empty(T, k, **i32), torch.empty(A, **i32), torch.empty(1, **i32)
        self.layer_ws = B.new_workspace(B.make_shape(T, H, E, k, F, C))
        self.offsets, self.order, self.pos = torch.empty(C + 1, **i32), torch.empty(A, **i32), torch.empty(T, k, **i32)
        self.sort_ws = torch.empty(B.moe_sort_workspace_bytes(T, k, C), dtype=torch.uint8, device="cuda")
        u8 = lambda *s: torch.zeros(*s, dtype=torch.uint8, device="cuda")
        f32 = lambda *s: torch.zeros(*s, device="cuda")
        self.q1, self.s1, self.q2, self.s2 = (u8(C, 2 * F, R.pad(H)), f32(C, R.pad(2 * F) // 128, R.pad(H) // 128),
                                              u8(C, H, R.pad(F)), f32(C, R.pad(H) // 128, R.pad(F) // 128))
        B.moe_quantize_weights_fp8(self.w1, True, C, 2 * F, H, self.q1, self.s1)
        B.moe_quantize_weights_fp8(self.w2, True, C, H, F, self.q2, self.s2)
        self.a, self.sa = u8(A, R.pad(H)), f32(A, R.pad(H) // 128)
        self.h = torch.zeros(A, 2 * F, dtype=torch.bfloat16, device="cuda")
        self.b, self.sb = u8(A, R.pad(F)), f32(A, R.pad(F) // 128)
        self.o, self.out = torch.zeros(A, H, dtype=torch.bfloat16, device="cuda"), torch.zeros(T, H, device="cuda")

    def route(self):
        T, H, E, k, F, C = self.sizes
        B.moe_route_topk(self.x, self.router, None, T, H, E, k, self.topk_idx, self.topk_w, None, self.layer_ws)
        B.moe_slot_resolve(self.topk_idx, self.table, T, k, E, C, self.slot_idx, self.miss, self.n_miss, self.layer_ws)

    def experts(self, stream=None):
        T, H, E, k, F, C = self.sizes
        A, valid = T * k, self.offsets[C:]
        B.moe_sort_assignments(self.slot_idx, T, k, C, self.offsets, self.order, self.pos, self.sort_ws, stream=stream)
        B.moe_permute_fp8(self.x, True, self.pos, T, k, H, A, self.a, self.sa, stream=stream)
        B.moe_grouped_matmul_fp8(self.a, self.sa, self.q1, self.s1, self.offsets, A, 2 * F, R.pad(H), C, self.h, True, stream=stream)
        B.moe_swiglu_fp8(self.h, True, valid, A, F, self.b, self.sb, stream=stream)
        B.moe_grouped_matmul_fp8(self.b, self.sb, self.q2, self.s2, self.offsets, A, H, R.pad(F), C, self.o, True, stream=stream)
        B.moe_unpermute(self.o, True, self.pos, self.topk_w, T, k, H, A, self.out, False, False, stream=stream)

    def check(self):
        """Every call's result against the plain form of it on what the call before left."""
        T, H, E, k, F, C = self.sizes
        c = {n: v.cpu() for n, v in self.__dict__.items() if isinstance(v, torch.Tensor)}
        for n, want in zip(("offsets", "order", "pos"), R.sort(c["slot_idx"], C)):
            assert torch.equal(c[n], want), n
        n = int(c["offsets"][C])
        assert 0 < n < T * k or C == E
        token = c["order"][:n].long() // k
        q, s = R.blocks(c["x"])
        assert torch.equal(c["a"][:n], q.view(torch.uint8)[token]) and torch.equal(c["sa"][:n], s[token])
        for a, sa, w, sw, out in (("a", "sa", "q1", "s1", "h"), ("b", "sb", "q2", "s2", "o")):
            want, size = R.matmul(c[a].view(F8), c[sa], c[w].view(F8), c[sw], c["offsets"])
            bound = R.matmul_bound(size, want, c[a].shape[1], torch.bfloat16)
            assert bool(((c[out].double() - want).abs() <= bound)[:n].all()), out
        gate, up = c["h"].double()[:n, :F], c["h"].double()[:n, F:]
        y = gate * torch.sigmoid(gate) * up
        back = c["b"].view(F8).double() * c["sb"].double().repeat_interleave(128, dim=1)
        least = c["sb"].double().repeat_interleave(128, dim=1)[:n, :F] * 2.0 ** -10
        assert bool(((back[:n, :F] - y).abs() <= torch.maximum(y.abs() * 2 ** -4, least) * (1 + 2 ** -15) + y.abs() * 2 ** -15).all())
        here = (c["pos"] >= 0).unsqueeze(2)
        terms = torch.where(here, c["o"].double()[c["pos"].clamp(min=0).long()], 0.0) * c["topk_w"].double().unsqueeze(2)
        assert bool(((c["out"].double() - terms.sum(dim=1)).abs() <= (k + 1) * R.U * terms.abs().sum(dim=1)).all())


SIZES = [(1, 256, 8, 2, 128, 5), (9, 512, 64, 6, 256, 32), (61, 264, 40, 4, 200, 20), (700, 640, 16, 3, 392, 16)]


@pytest.mark.parametrize("sizes", SIZES, ids=lambda s: "x".join(map(str, s)))
def test_experts_in_8_bits(sizes):
    c = Chain(*sizes, seed=sum(sizes))
    c.route()
    c.experts()
    torch.cuda.synchronize()
    c.check()


def test_on_a_stream_of_its_own():
    c = Chain(*SIZES[1], seed=3)
    c.route()
    torch.cuda.synchronize()
    s = torch.cuda.Stream()
    c.experts(stream=s)
    s.synchronize()
    c.check()


def test_captured_and_replayed():
    """Two chains in one graph, replayed with other inputs and eager work between; each replay against the eager run."""
    chains = [Chain(*SIZES[2], seed=4), Chain(*SIZES[3], seed=5)]
    for c in chains:
        c.route()
        c.experts()
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        for c in chains:
            c.experts()
    for turn in range(4):
        for c in chains:
            c.x.copy_(torch.randn(c.x.shape, generator=torch.Generator().manual_seed(turn)).bfloat16())
            c.route()
        for c in chains:
            c.out.fill_(float("nan"))
        graph.replay()
        torch.cuda.synchronize()
        got = [c.out.clone() for c in chains]
        for c in chains:
            c.experts()
        torch.cuda.synchronize()
        for c, g in zip(chains, got):
            assert torch.equal(c.out, g)
    for c in chains:
        c.check()


def test_two_streams_at_once():
    """Chains with buffers and workspaces of their own may run at the same time."""
    chains = [Chain(*SIZES[1], seed=6), Chain(*SIZES[2], seed=7)]
    streams = [torch.cuda.Stream() for _ in chains]
    for c in chains:
        c.route()
    torch.cuda.synchronize()
    for _ in range(5):
        for c, s in zip(chains, streams):
            c.experts(stream=s)
    torch.cuda.synchronize()
    for c in chains:
        c.check()
