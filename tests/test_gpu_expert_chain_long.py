"""A batch longer than one routing call takes (T*E <= 65536): routed and resolved in pieces of unequal length on one workspace, each into its
part of the outputs, then sorted, multiplied and summed as one."""
from unittest import mock

import pytest
import torch

from paper_2603_09983_amd import binding as B
from test_gpu_expert_chain import Chain

pytestmark = pytest.mark.gpu


class LongChain(Chain):
    def __init__(self, T, H, E, k, F, C, seed):
        self.piece = 65536 // E // 64 * 64
        shape = B.make_shape
        with mock.patch.object(B, "make_shape", lambda T, *rest: shape(min(T, self.piece), *rest)):   # (the workspace is a piece's)
            super().__init__(T, H, E, k, F, C, seed)
        self.logits = torch.empty(T, E, device="cuda")

    def route(self):
        T, H, E, k, F, C = self.sizes
        for t in range(0, T, self.piece):
            n, part = min(self.piece, T - t), slice(t, t + self.piece)
            B.moe_route_topk(self.x[part], self.router, None, n, H, E, k, self.topk_idx[part], self.topk_w[part], self.logits[part],
                             self.layer_ws)
            B.moe_slot_resolve(self.topk_idx[part], self.table, n, k, E, C, self.slot_idx[part], self.miss, self.n_miss, self.layer_ws)


@pytest.mark.parametrize("sizes", [(2500, 256, 64, 6, 128, 40), (1100, 264, 128, 4, 72, 100)], ids=lambda s: "x".join(map(str, s)))
def test_routed_in_pieces(sizes):
    T, H, E, k, F, C = sizes
    c = LongChain(*sizes, seed=1)
    assert T * E > 65536 and T % c.piece
    c.route()
    c.experts()
    torch.cuda.synchronize()
    B.moe_workspace_status(c.layer_ws)
    # the routing by definition, from the logits (ties to the lower expert) and these from the inputs
    logits = c.logits.cpu()
    want = c.x.cpu().double() @ c.router.cpu().double().t()
    size = c.x.cpu().double().abs() @ c.router.cpu().double().abs().t()
    assert bool(((logits.double() - want).abs() <= H * 2.0 ** -24 * size).all())
    order = torch.sort(logits, dim=1, descending=True, stable=True).indices[:, :k]
    assert torch.equal(c.topk_idx.cpu().long(), order)
    assert torch.equal(c.slot_idx.cpu(), c.table.cpu()[order])
    gates = torch.softmax(torch.gather(logits.double(), 1, order), dim=1)
    assert bool(((c.topk_w.cpu().double() - gates).abs() <= 2.0 ** -20 * gates + 2.0 ** -40).all())
    c.check()
