"""One decode step of a mixture-of-experts layer, two ways.

    python examples/serve_layer.py [--tokens 64] [--hidden 1024] [--experts 32] [--top-k 4] [--width 512] [--ranks 8]

Rows of several requests, each with a low-rank adapter of its own, go through the shared projection (mw_project) to the hidden rows,
the router's product (mw_project with float32 outputs) and the router's choice (mw_route).  Then
  * all experts on one GPU: mw_experts, one call;
  * the experts spread over the ranks of a domain: mw_plan_dispatch brings every hidden row to the ranks of its experts, mw_experts runs
    each rank's share on the rows of its receive region, mw_combine adds what the ranks return.
Both give the layer's output; the second rounds each rank's sum to bf16 on its way back.
"""
from __future__ import annotations

import argparse
import os
import sys

import torch

sys.path.insert(0, os.path.dirname(os.path.dirname(os.path.abspath(__file__))))

from paper_2605_22428_b200 import binding as mw  # noqa: E402


class Layer:
    """Random weights of one layer and the handles a server keeps over them."""

    def __init__(self, tokens: int, hidden: int, experts: int, top_k: int, width: int, ranks: int, adapters: int = 8, rank: int = 16, seed: int = 0):
        assert experts % ranks == 0
        self.T, self.H, self.E, self.K, self.R, self.adapters = tokens, hidden, experts, top_k, ranks, adapters
        g = torch.Generator("cuda").manual_seed(seed)

        def weights(*shape):
            return torch.empty(*shape, dtype=torch.bfloat16, device="cuda").normal_(0, shape[-1] ** -0.5, generator=g)

        self.projection = mw.Projection(hidden, hidden, tokens, weights(hidden, hidden), adapters, rank, weights(adapters, rank, hidden),
                                        weights(adapters, hidden, rank), torch.ones(adapters, device="cuda"))
        self.gate = mw.Projection(hidden, experts, tokens, weights(experts, hidden))
        w_gate_up, w_down = weights(experts, 2, width, hidden), weights(experts, hidden, width)
        self.all_experts = mw.Experts(experts, top_k, tokens, hidden, width, w_gate_up, w_down)
        per = experts // ranks
        self.shares = [mw.Experts(experts, top_k, tokens, hidden, width, w_gate_up[r * per:], w_down[r * per:], expert_first=r * per, expert_count=per)
                       for r in range(ranks)]
        self.domain = mw.Context(ranks, experts, top_k, tokens, hidden * 2)
        self.expert_to_rank = (torch.arange(experts, device="cuda") // per).int()

    def route(self, rows, adapter_ids):
        """Input rows -> hidden rows, expert ids and weights."""
        hidden = torch.empty(self.T, self.H, dtype=torch.bfloat16, device="cuda")
        logits = torch.empty(self.T, self.E, device="cuda")
        ids = torch.empty(self.T, self.K, dtype=torch.int32, device="cuda")
        weights = torch.empty(self.T, self.K, device="cuda")
        self.projection.mw_project_forward(rows, adapter_ids, self.T, hidden)
        self.gate.mw_project_forward(hidden, None, self.T, logits)
        mw.mw_route(logits, None, self.T, self.E, self.K, mw.MW_ROUTE_RENORMALISE, 1.0, ids, weights)
        return hidden, ids, weights

    def on_one_gpu(self, hidden, ids, weights):
        y = torch.empty_like(hidden)
        self.all_experts.mw_experts_forward(hidden, ids, weights, self.T, y)
        return y

    def over_the_domain(self, hidden, ids, weights):
        T, H, R = self.T, self.H, self.R
        send = torch.empty(T, H, dtype=torch.bfloat16, device="cuda")
        received = torch.zeros(R, T, H, dtype=torch.bfloat16, device="cuda")         # a region per rank
        returned = torch.zeros_like(received)
        stride = T * H * 2
        self.domain.mw_plan_dispatch(ids, self.expert_to_rank, T, hidden, mw.MW_LAYOUT_MULTIWRITE, send, T, received, stride, T)
        plan = self.domain.plan_arrays(T)
        begin = plan["rank_offsets"]
        tokens = torch.from_numpy(plan["rank_tokens"]).cuda().long()
        for r in range(R):
            n = int(begin[r + 1] - begin[r])
            here = tokens[begin[r]:begin[r + 1]]
            self.shares[r].mw_experts_forward(received[r], ids[here].contiguous(), weights[here].contiguous(), n, returned[r])
        y = torch.empty_like(hidden)
        self.domain.mw_combine(returned, stride, None, y)
        return y


def main() -> float:
    p = argparse.ArgumentParser(description=__doc__.splitlines()[0])
    for name, value in (("tokens", 64), ("hidden", 1024), ("experts", 32), ("top-k", 4), ("width", 512), ("ranks", 8)):
        p.add_argument("--" + name, type=int, default=value)
    a = p.parse_args()
    layer = Layer(a.tokens, a.hidden, a.experts, a.top_k, a.width, a.ranks)
    g = torch.Generator("cuda").manual_seed(1)
    rows = torch.empty(a.tokens, a.hidden, dtype=torch.bfloat16, device="cuda").normal_(0, 1, generator=g)
    adapter_ids = torch.randint(-1, layer.adapters, (a.tokens,), device="cuda", generator=g).int()
    hidden, ids, weights = layer.route(rows, adapter_ids)
    one, many = layer.on_one_gpu(hidden, ids, weights), layer.over_the_domain(hidden, ids, weights)
    off = float((one.float() - many.float()).norm() / one.float().norm())
    print(f"{a.tokens} tokens, {a.experts} experts on {a.ranks} ranks, top-{a.top_k}: the two ways differ by {off:.2e} (relative 2-norm)")
    return off


if __name__ == "__main__":
    main()
