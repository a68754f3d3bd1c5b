"""The serving operators together with the dispatch: examples/serve_layer.py at small sizes, against the layer in float64.

Tolerance: hidden rows and ids are the operators' own (each is tested by itself); the layer's output is held as in test_gpu_experts.py to
2^-8 in the relative 2-norm.  Over the domain every rank's sum is rounded to bf16 once more, so that way is held to 2^-8 sqrt(2) + 2^-8.
"""
import importlib.util
import os

import pytest

pytestmark = pytest.mark.gpu

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))


def example():
    spec = importlib.util.spec_from_file_location("serve_layer", os.path.join(ROOT, "examples", "serve_layer.py"))
    m = importlib.util.module_from_spec(spec)
    spec.loader.exec_module(m)
    return m


@pytest.mark.parametrize("tokens,hidden,experts,top_k,width,ranks", [(1, 256, 8, 2, 64, 2), (37, 512, 32, 4, 128, 8), (256, 1024, 32, 4, 96, 8),
                                                                    (70, 256, 64, 8, 64, 64)])
def test_one_gpu_and_the_domain_give_the_layer(tokens, hidden, experts, top_k, width, ranks):
    import torch
    layer = example().Layer(tokens, hidden, experts, top_k, width, ranks, seed=tokens)
    g = torch.Generator("cuda").manual_seed(7)
    rows = torch.empty(tokens, hidden, dtype=torch.bfloat16, device="cuda").normal_(0, 1, generator=g)
    adapter_ids = torch.randint(-1, layer.adapters, (tokens,), device="cuda", generator=g).int()
    h, ids, weights = layer.route(rows, adapter_ids)
    assert bool(((ids >= 0) & (ids < experts)).all()) and torch.allclose(weights.sum(1), torch.ones(tokens, device="cuda"), atol=1e-5)
    want = torch.zeros(tokens, hidden, dtype=torch.float64, device="cuda")
    w_gate_up, w_down = layer.all_experts._weights
    for e in range(experts):
        t, k = torch.nonzero(ids == e, as_tuple=True)
        if t.numel():
            gate, up = h[t].double() @ w_gate_up[e, 0].double().t(), h[t].double() @ w_gate_up[e, 1].double().t()
            want.index_add_(0, t, (gate * torch.sigmoid(gate) * up) @ w_down[e].double().t() * weights[t, k].double().unsqueeze(1))
    for y, most in ((layer.on_one_gpu(h, ids, weights), 2.0 ** -8), (layer.over_the_domain(h, ids, weights), 2.0 ** -8 * (1 + 2 ** 0.5))):
        torch.cuda.synchronize()
        assert float((y.double() - want).norm() / want.norm()) <= most
    assert layer.domain.mw_get_totals()["status"] == 0
    assert layer.all_experts.mw_experts_get_status() == 0 and all(s.mw_experts_get_status() == 0 for s in layer.shares)
