"""Cases of the dense operators beside the router, the experts and the projection: the gated feed-forward block, forward and with its
backward pass (`Gated`), and the product in 8-bit integers with a scale per token and per channel (`Int8Projection`), alone and as the
two products of a served block.

`own` false: the operators written out in elementary torch operations, in 32 bits, rounded once at the end.  `own` true: the calls of this package.  Sizes are those of the package's own workloads (hidden size 7168 or 1024, 1 ... 4096
tokens), with generic widths.
"""
import math

import torch

own = False

DEVICE = "cuda"


def listed():
    return [
        # the shared expert for one token of one sequence: its weights are read once
        dict(name="gated_one_token", op="gated", T=1, H=7168, I=2048, half=False, gelu=False),
        # the shared expert for a decode batch
        dict(name="gated_decode_64", op="gated", T=64, H=7168, I=2048, half=False, gelu=False),
        # a dense layer of the small configuration for a ragged batch, the other type and activation
        dict(name="gated_odd", op="gated", T=201, H=1024, I=2808, half=True, gelu=True),
        # the shared expert for a prefill batch
        dict(name="gated_prefill", op="gated", T=4096, H=7168, I=2048, half=False, gelu=False),
        # a training step of the shared expert on a batch of the prefill size
        dict(name="train_batch", op="train", T=4096, H=7168, I=2048, half=False, gelu=False),
        # a training step of the small configuration, ragged, the other type and activation
        dict(name="train_small", op="train", T=777, H=1024, I=688, half=True, gelu=True),
        # one token through a projection held in 8 bits
        dict(name="int8_one_token", op="int8", T=1, H=7168, O=7168, x="bf16", y="bf16"),
        # odd everything: tokens, output width; 32-bit rows in, 32-bit results out
        dict(name="int8_odd", op="int8", T=77, H=1024, O=1003, x="f32", y="f32"),
        # prompts side by side
        dict(name="int8_prompts", op="int8", T=4096, H=7168, O=7168, x="bf16", y="bf16"),
        # the shared expert in 8 bits for one token
        dict(name="int8_block_one_token", op="block", T=1, H=7168, I=2048, half=False, gelu=False),
        # the same for a decode batch
        dict(name="int8_block_64", op="block", T=64, H=7168, I=2048, half=False, gelu=False),
        # the same for a short prefill, the other type
        dict(name="int8_block_1000", op="block", T=1000, H=7168, I=2048, half=True, gelu=False),
    ]


def _log_int(rng, low, high):
    return max(low, min(high, int(round(math.exp(rng.uniform(math.log(low), math.log(high)))))))


def draw(rng):
    op = rng.choice(("gated", "gated", "train", "int8", "int8", "block"))
    T = _log_int(rng, 1, 4096)
    if op == "int8":
        return dict(op=op, T=T, H=16 * _log_int(rng, 16, 448), O=_log_int(rng, 200, 7168), x=rng.choice(("bf16", "bf16", "f16", "f32")),
                    y=rng.choice(("bf16", "f16", "f32")))
    # three products of T x H x I each; as wide as the largest listed case allows
    H = (16 if op == "block" else 8) * _log_int(rng, 32, 448 if op == "block" else 896)
    I = 16 * _log_int(rng, 12, min(640, 4096 * 7168 * 2048 // (T * H * 16)))
    return dict(op=op, T=T, H=H, I=I, half=rng.random() < 0.4, gelu=rng.random() < 0.4)


_TYPES = dict(bf16=torch.bfloat16, f16=torch.float16, f32=torch.float32)


def _type(case):
    return torch.float16 if case["half"] else torch.bfloat16


def _rows(g, T, n, dtype):
    """Hidden rows: a few channels far larger than the others, as a layer's inputs have them."""
    gain = 1 + 7 * (torch.rand(n, device=DEVICE, generator=g) < 0.005).float()
    return (torch.randn(T, n, device=DEVICE, generator=g) * gain).to(dtype)


def _int8_weights(g, O, n):
    """A matrix in 8 bits, a scale for each of its rows."""
    w = torch.randn(O, n, device=DEVICE, generator=g) * n ** -0.5
    scale = w.abs().amax(1) / 127
    return torch.round(w / scale.unsqueeze(1)).to(torch.int8), scale


def prepare(case, seed):
    g = torch.Generator(DEVICE).manual_seed(seed)
    T, H = case["T"], case["H"]
    s = dict(case=case)
    if case["op"] == "int8":
        s["x"] = _rows(g, T, H, _TYPES[case["x"]])
        s["w"], s["w_scale"] = _int8_weights(g, case["O"], H)
        s["y"] = torch.empty(T, case["O"], dtype=_TYPES[case["y"]], device=DEVICE)
    else:
        I, dtype = case["I"], _type(case)
        s["x"], s["y"] = _rows(g, T, H, dtype), torch.empty(T, H, dtype=dtype, device=DEVICE)
        if case["op"] == "block":
            s["w_gate_up"], s["gate_up_scale"] = _int8_weights(g, 2 * I, H)
            s["w_down"], s["down_scale"] = _int8_weights(g, H, I)
            s["gate_up"] = torch.empty(T, 2 * I, dtype=dtype, device=DEVICE)
        else:
            s["w_gate_up"] = (torch.randn(2, I, H, device=DEVICE, generator=g) * H ** -0.5).to(dtype)
            s["w_down"] = (torch.randn(H, I, device=DEVICE, generator=g) * I ** -0.5).to(dtype)
        if case["op"] == "train":
            s["dy"] = torch.randn(T, H, device=DEVICE, generator=g).to(dtype)
            s["gate_up"] = torch.empty(T, 2 * I, dtype=dtype, device=DEVICE)
            s["dx"] = torch.empty(T, H, dtype=dtype, device=DEVICE)
            s["dw_gate_up"] = torch.empty(2, I, H, dtype=dtype, device=DEVICE)
            s["dw_down"] = torch.empty(H, I, dtype=dtype, device=DEVICE)
    if own:      # what a user's program makes once: handles over its weights
        from paper_2605_22428_b200 import binding as mw
        if case["op"] == "int8":
            s["handle"] = mw.Int8Projection(H, case["O"], T, s["w"], s["w_scale"])
        else:
            s["activation"] = mw.MW_ACT_GELU if case["gelu"] else mw.MW_ACT_SILU
            if case["op"] == "block":
                s["first"] = mw.Int8Projection(H, 2 * case["I"], T, s["w_gate_up"], s["gate_up_scale"])
                s["second"] = mw.Int8Projection(case["I"], H, T, s["w_down"], s["down_scale"])
            else:
                s["handle"] = mw.Gated(H, case["I"], T, s["w_gate_up"], s["w_down"], activation=s["activation"], train=case["op"] == "train")
    return s


def _sigmoid(case, gate):
    """The activation is gate * sigmoid(k): the sigmoid, and k's derivative."""
    if case["gelu"]:
        c = 2 * math.sqrt(2 / math.pi)
        return 1 / (1 + torch.exp(-c * (gate + 0.044715 * gate * gate * gate))), c * (1 + 3 * 0.044715 * gate * gate)
    return 1 / (1 + torch.exp(-gate)), torch.ones_like(gate)


def _gated_plain(s):
    case, x = s["case"], s["x"].float()
    gate, up = torch.matmul(x, s["w_gate_up"][0].float().t()), torch.matmul(x, s["w_gate_up"][1].float().t())
    sig, slope = _sigmoid(case, gate)
    h = gate * sig * up
    y = torch.matmul(h, s["w_down"].float().t()).to(_type(case))
    if case["op"] == "gated":
        return y
    dy = s["dy"].float()
    dh = torch.matmul(dy, s["w_down"].float())
    d_gate, d_up = dh * up * (sig + gate * sig * (1 - sig) * slope), dh * gate * sig
    dx = torch.matmul(d_gate, s["w_gate_up"][0].float()) + torch.matmul(d_up, s["w_gate_up"][1].float())
    dw_gate_up = torch.stack((torch.matmul(d_gate.t(), x), torch.matmul(d_up.t(), x)))
    return dict(y=y, dx=dx.to(_type(case)), dw_gate_up=dw_gate_up.to(_type(case)), dw_down=torch.matmul(dy.t(), h).to(_type(case)))


def _quantise_plain(x):
    """Rows in 8 bits: integers (as float32) and a scale for each; quotients in 64 bits, as many lie next to a border
    (and a division by a number is a product with its inverse in 32 bits)."""
    scale = (x.abs().amax(1, keepdim=True).double() / 127).float()
    return torch.round(x.double() / torch.where(scale > 0, scale, 1).double()).float(), scale


def _int8_product_plain(x, w, w_scale, dtype):
    q, scale = _quantise_plain(x)
    return (torch.matmul(q, w.float().t()) * scale * w_scale).to(dtype)


def _block_plain(s):
    case = s["case"]
    gate_up = _int8_product_plain(s["x"].float(), s["w_gate_up"], s["gate_up_scale"], _type(case)).float()
    gate, up = gate_up[:, :case["I"]], gate_up[:, case["I"]:]
    return _int8_product_plain(gate * _sigmoid(case, gate)[0] * up, s["w_down"], s["down_scale"], _type(case))


def run(s):
    case = s["case"]
    op, T = case["op"], case["T"]
    if not own:
        if op == "int8":
            return _int8_product_plain(s["x"].float(), s["w"], s["w_scale"], s["y"].dtype)
        return _block_plain(s) if op == "block" else _gated_plain(s)
    if op == "int8":
        s["handle"].mw_int8_forward(s["x"], None, T, s["y"])
        return s["y"]
    if op == "block":
        s["first"].mw_int8_forward(s["x"], None, T, s["gate_up"])
        s["second"].mw_int8_forward(s["gate_up"], None, T, s["y"], activation=s["activation"])
        return s["y"]
    if op == "gated":
        s["handle"].mw_gated_forward(s["x"], T, s["y"])
        return s["y"]
    s["handle"].mw_gated_forward(s["x"], T, s["y"], gate_up=s["gate_up"])
    s["handle"].mw_gated_backward(s["x"], s["gate_up"], s["dy"], T, dx=s["dx"], dw_gate_up=s["dw_gate_up"], dw_down=s["dw_down"])
    return dict(y=s["y"], dx=s["dx"], dw_gate_up=s["dw_gate_up"], dw_down=s["dw_down"])


def work(case):
    T, H = case["T"], case["H"]
    if case["op"] == "int8":
        O, size = case["O"], dict(bf16=2, f16=2, f32=4)
        return dict(bytes=O * H + 4 * O + T * H * size[case["x"]] + T * O * size[case["y"]], flops=2 * T * H * O)
    I = case["I"]
    if case["op"] == "block":
        return dict(bytes=3 * H * I + 4 * (2 * I + H) + 4 * T * H, flops=6 * T * H * I)
    if case["op"] == "gated":
        return dict(bytes=6 * H * I + 4 * T * H, flops=6 * T * H * I)
    return dict(bytes=12 * H * I + 8 * T * H, flops=18 * T * H * I)


def _quantise_exact(x):
    """64-bit rows of exact values; the scale is a 32-bit number, the integers are nearest to what it leaves."""
    scale = (x.abs().amax(1, keepdim=True) / 127).float().double()
    return torch.round(x / torch.where(scale == 0, 1.0, scale)), scale


def _activation_exact(case, gate):
    if case["gelu"]:
        return torch.nn.functional.gelu(gate, approximate="tanh")
    return torch.nn.functional.silu(gate)


def exact(case, seed):
    s = prepare(case, seed)
    x = s["x"].double()
    if case["op"] == "int8":
        q, scale = _quantise_exact(x)
        return (q @ s["w"].double().t()) * scale * s["w_scale"].double()
    if case["op"] == "block":
        q, scale = _quantise_exact(x)
        gate_up = ((q @ s["w_gate_up"].double().t()) * scale * s["gate_up_scale"].double()).to(_type(case)).double()   # rows between the calls are of this type
        gate, up = gate_up.chunk(2, 1)
        q, scale = _quantise_exact(_activation_exact(case, gate) * up)
        return (q @ s["w_down"].double().t()) * scale * s["down_scale"].double()
    train = case["op"] == "train"
    w = s["w_gate_up"].double()
    gate, up = x @ w[0].t(), x @ w[1].t()
    if train:
        gate.requires_grad_()
    act = _activation_exact(case, gate)
    h = act.detach() * up
    y = h @ s["w_down"].double().t()
    if not train:
        return y
    dy = s["dy"].double()
    dh = dy @ s["w_down"].double()
    d_gate, = torch.autograd.grad(act, gate, dh * up)
    d_up = dh * act.detach()
    return dict(y=y.detach(), dx=d_gate @ w[0] + d_up @ w[1], dw_gate_up=torch.stack((d_gate.t() @ x, d_up.t() @ x)), dw_down=dy.t() @ h.detach())
