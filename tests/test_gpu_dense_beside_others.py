"""The dense operators on streams of their own beside the experts and the projection, whose blocks hand results to one another: every call gives the bits that it gives alone, and no
wait runs out.  (A block of any of them that needs columns of TMEM holds the shared memory that goes with them, so none waits for another's to end while it runs.)"""
import pytest

from gpu_util import torch_mod
from paper_2605_22428_b200 import binding as mw

pytestmark = pytest.mark.gpu


def test_five_handles_on_five_streams():
    torch = torch_mod()
    g = torch.Generator("cuda").manual_seed(3)
    n = lambda *s, std=1.0: (torch.randn(*s, device="cuda", generator=g) * std).bfloat16()  # noqa: E731
    H, I, E, K = 1024, 512, 16, 4
    w, d = n(2, I, H, std=H ** -0.5), n(H, I, std=I ** -0.5)
    q, s = torch.empty(2 * I, H, dtype=torch.int8, device="cuda"), torch.empty(2 * I, device="cuda")
    mw.mw_quantise_rows(w.view(2 * I, H), 2 * I, H, q, s)
    many, few, some = n(2000, H), n(48, H), n(300, H)
    ids = torch.stack([torch.randperm(E, device="cuda", generator=g)[:K] for _ in range(48)]).int()
    weights = torch.rand(48, K, device="cuda", generator=g)
    with mw.Gated(H, I, 2000, w, d, train=True) as train, mw.Gated(H, I, 48, w, d) as serve, mw.Int8Projection(H, 2 * I, 300, q, s) as product, \
            mw.Experts(E, K, 48, H, I, n(E, 2, I, H, std=H ** -0.5), n(E, H, I, std=I ** -0.5)) as experts, mw.Projection(H, H, 300, n(H, H, std=H ** -0.5)) as projection:
        kept = torch.empty(2000, 2 * I, dtype=torch.bfloat16, device="cuda")

        def training(out, stream):
            train.mw_gated_forward(many, 2000, out[0], gate_up=kept, stream=stream)
            train.mw_gated_backward(many, kept, many, 2000, dx=out[1], dw_gate_up=out[2], dw_down=out[3], stream=stream)
        calls = [(training, (many.shape, many.shape, w.shape, d.shape)), (lambda out, stream: serve.mw_gated_forward(few, 48, out[0], stream=stream), (few.shape,)),
                 (lambda out, stream: product.mw_int8_forward(some, None, 300, out[0], stream=stream), ((300, 2 * I),)),
                 (lambda out, stream: experts.mw_experts_forward(few, ids, weights, 48, out[0], stream=stream), (few.shape,)),
                 (lambda out, stream: projection.mw_project_forward(some, None, 300, out[0], stream=stream), (some.shape,))]
        make = lambda shapes: [torch.zeros(*shape, dtype=torch.bfloat16, device="cuda") for shape in shapes]  # noqa: E731
        alone = []
        for call, shapes in calls:
            alone.append(make(shapes))
            call(alone[-1], None)
            torch.cuda.synchronize()
        streams = [torch.cuda.Stream() for _ in calls]
        turns = [[make(shapes) for _, shapes in calls] for _ in range(12)]
        torch.cuda.synchronize()
        for outs in turns:
            for (call, _), out, stream in zip(calls, outs, streams):
                call(out, stream)
        torch.cuda.synchronize()
        for outs in turns:
            for out, want in zip(outs, alone):
                assert all(torch.equal(a, b) for a, b in zip(out, want))
        assert train.mw_gated_get_status() == serve.mw_gated_get_status() == product.mw_int8_get_status() == mw.MW_OK
        assert experts.mw_experts_get_status() == projection.mw_project_get_status() == mw.MW_OK
