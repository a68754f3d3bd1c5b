"""Cases of the serving operators around the dispatch: the router's choice (`mw_route`), a rank's experts for few tokens
(`mw_experts_forward`) and the shared projection with per-request low-rank adapters (`mw_project_forward`).

`own` false: the operators written out in elementary torch operations, in 32 bits, rounded once at the end.
`own` true: the calls of this package.  Sizes are those of the package's own workloads (hidden size 7168 or 1024, 256 / 64 / 32 experts,
top-8 / top-4, 64 ... 8192 tokens), with a generic expert width.
"""
import math

import torch

own = False

DEVICE = "cuda"


def listed():
    return [
        # one token of one sequence: latency of the smallest call
        dict(name="route_one_token", op="route", T=1, E=256, K=8, bf16=False, bias=False, sigmoid=False, renorm=True, scale=1.0),
        # the prefill batch, router scores in 32 bits with a load-balancing bias
        dict(name="route_prefill", op="route", T=4096, E=256, K=8, bf16=False, bias=True, sigmoid=True, renorm=True, scale=2.5),
        # 64 experts, top-8, scores left in 16 bits by the router's product: many ties
        dict(name="route_64_experts", op="route", T=2048, E=64, K=8, bf16=True, bias=False, sigmoid=False, renorm=False, scale=1.0),
        # all 256 experts on one GPU, one sequence: eight experts' weights are read for one token
        dict(name="experts_one_token", op="experts", T=1, E=256, first=0, count=256, K=8, H=7168, I=2048, others=False),
        # the decode batch with all experts on one GPU: most experts' weights are read for two or three tokens each
        dict(name="experts_decode_64", op="experts", T=64, E=256, first=0, count=256, K=8, H=7168, I=2048, others=False),
        # one rank's share of a 64-rank domain: 4 of 256 experts, the tokens that were delivered to it
        dict(name="experts_rank_share", op="experts", T=201, E=256, first=128, count=4, K=8, H=7168, I=2048, others=True),
        # the small configuration, a handful of tokens
        dict(name="experts_small_7", op="experts", T=7, E=32, first=0, count=32, K=4, H=1024, I=512, others=False),
        # the small configuration's whole batch, expert width that is no multiple of the tile
        dict(name="experts_small_256", op="experts", T=256, E=32, first=0, count=32, K=4, H=1024, I=688, others=False),
        # one token with its request's adapter
        dict(name="project_one_token", op="project", T=1, H=7168, O=7168, n=32, r=16, segment=1, none=0.0),
        # a decode batch: one token per request, requests share 32 adapters, some have none
        dict(name="project_decode_64", op="project", T=64, H=7168, O=7168, n=32, r=16, segment=1, none=0.15),
        # prompts of several requests side by side, each with its own adapter
        dict(name="project_prompts", op="project", T=4096, H=7168, O=7168, n=12, r=64, segment=341, none=0.1),
        # odd everything: tokens, output width, rank
        dict(name="project_odd", op="project", T=77, H=1024, O=1003, n=5, r=24, segment=9, none=0.1),
    ]


def _log_int(rng, low, high):
    return max(low, min(high, int(round(math.exp(rng.uniform(math.log(low), math.log(high)))))))


def draw(rng):
    op = rng.choice(("route", "experts", "experts", "project", "project"))
    if op == "route":
        E = rng.choice((32, 64, 96, 128, 160, 256, 384))
        return dict(op="route", T=_log_int(rng, 1, 8192), E=E, K=rng.choice((1, 2, 4, 6, 8)), bf16=rng.random() < 0.3, bias=rng.random() < 0.5,
                    sigmoid=rng.random() < 0.5, renorm=rng.random() < 0.6, scale=rng.choice((1.0, 2.5)))
    if op == "experts":
        E = rng.choice((8, 32, 64, 128, 256))
        count = rng.choice((E, E, max(2, E // 8)))
        H, K = rng.choice((1024, 2048, 4096, 7168)), rng.choice((2, 4, 6, 8))
        most = min(2048, int(2e9 / (3.0 * count * H)))           # at most 4 GB of weights
        I = 16 * _log_int(rng, 16, max(17, most // 16))
        return dict(op="experts", T=_log_int(rng, 1, 400), E=E, first=rng.choice(range(0, E, count)), count=count, K=K, H=H, I=I,
                    others=count < E)
    n = _log_int(rng, 1, 64)
    return dict(op="project", T=_log_int(rng, 1, 4096), H=8 * rng.randint(64, 896), O=_log_int(rng, 200, 7168), n=n, r=8 * rng.choice((1, 2, 3, 4, 8)),
                segment=_log_int(rng, 1, 600), none=rng.choice((0.0, 0.15)))


def _route_state(case, g):
    T, E = case["T"], case["E"]
    popularity = torch.randn(E, device=DEVICE, generator=g) * 0.5
    logits = torch.randn(T, E, device=DEVICE, generator=g) + popularity
    if case["bf16"]:
        logits = logits.bfloat16()
    return dict(logits=logits, bias=torch.randn(E, device=DEVICE, generator=g) * 0.1 if case["bias"] else None,
                ids=torch.empty(T, case["K"], dtype=torch.int32, device=DEVICE), weights=torch.empty(T, case["K"], device=DEVICE))


def _experts_state(case, g):
    T, E, K, H, I, first, count = (case[k] for k in ("T", "E", "K", "H", "I", "first", "count"))
    key = torch.rand(T, E, device=DEVICE, generator=g)
    if case["others"]:       # tokens that were delivered to this rank: each has at least one of its experts
        key[torch.arange(T, device=DEVICE), torch.randint(first, first + count, (T,), device=DEVICE, generator=g)] += 1
    ids = key.argsort(dim=1, descending=True)[:, :K]
    ids = ids.gather(1, torch.rand(T, K, device=DEVICE, generator=g).argsort(dim=1)).int().contiguous()
    return dict(x=torch.empty(T, H, dtype=torch.bfloat16, device=DEVICE).normal_(0, 1, generator=g), ids=ids,
                weights=torch.softmax(torch.randn(T, K, device=DEVICE, generator=g), 1),
                w_gate_up=torch.empty(count, 2, I, H, dtype=torch.bfloat16, device=DEVICE).normal_(0, H ** -0.5, generator=g),
                w_down=torch.empty(count, H, I, dtype=torch.bfloat16, device=DEVICE).normal_(0, I ** -0.5, generator=g),
                y=torch.empty(T, H, dtype=torch.bfloat16, device=DEVICE))


def _project_state(case, g):
    T, H, O, n, r = (case[k] for k in ("T", "H", "O", "n", "r"))
    requests = -(-T // case["segment"])
    adapter = torch.randint(0, n, (requests,), device=DEVICE, generator=g)
    adapter = torch.where(torch.rand(requests, device=DEVICE, generator=g) < case["none"], -1, adapter)
    return dict(x=torch.empty(T, H, dtype=torch.bfloat16, device=DEVICE).normal_(0, 1, generator=g),
                adapter_ids=adapter.repeat_interleave(case["segment"])[:T].int().contiguous(),
                w=torch.empty(O, H, dtype=torch.bfloat16, device=DEVICE).normal_(0, H ** -0.5, generator=g),
                a=torch.empty(n, r, H, dtype=torch.bfloat16, device=DEVICE).normal_(0, H ** -0.5, generator=g),
                b=torch.empty(n, O, r, dtype=torch.bfloat16, device=DEVICE).normal_(0, r ** -0.5, generator=g),
                scale=0.25 + 1.5 * torch.rand(n, device=DEVICE, generator=g),
                y=torch.empty(T, O, dtype=torch.bfloat16, device=DEVICE))


def prepare(case, seed):
    g = torch.Generator(DEVICE).manual_seed(seed)
    s = dict(route=_route_state, experts=_experts_state, project=_project_state)[case["op"]](case, g)
    s["case"] = case
    if own:      # what a user's program makes once: handles over its weights; route needs none
        from paper_2605_22428_b200 import binding as mw
        s["mw"] = mw
        if case["op"] == "experts":
            s["handle"] = mw.Experts(case["E"], case["K"], case["T"], case["H"], case["I"], s["w_gate_up"], s["w_down"],
                                     expert_first=case["first"], expert_count=case["count"])
        elif case["op"] == "project":
            s["handle"] = mw.Projection(case["H"], case["O"], case["T"], s["w"], adapters=case["n"], rank=case["r"], a=s["a"], b=s["b"],
                                        scale=s["scale"])
        else:
            s["flags"] = (mw.MW_ROUTE_SIGMOID if case["sigmoid"] else 0) | (mw.MW_ROUTE_RENORMALISE if case["renorm"] else 0)
    return s


def _route_plain(s):
    case = s["case"]
    logits = s["logits"].float()
    key = logits if s["bias"] is None else logits + s["bias"]
    ids = torch.sort(key, dim=1, descending=True, stable=True).indices[:, :case["K"]]
    if case["sigmoid"]:
        p = 1 / (1 + torch.exp(-logits))
    else:
        p = torch.exp(logits - logits.amax(1, keepdim=True))
        p = p / p.sum(1, keepdim=True)
    w = p.gather(1, ids)
    if case["renorm"]:
        w = w / w.sum(1, keepdim=True)
    return dict(ids=ids.int(), weights=w * case["scale"])


def _experts_plain(s):
    case = s["case"]
    T, K, count = case["T"], case["K"], case["count"]
    local = s["ids"].long() - case["first"]
    here = (local >= 0) & (local < count) & (s["ids"] >= 0)
    local = torch.where(here, local, 0)
    x = s["x"].float()
    if T * K < count:        # fewer picks than experts: each pick's matrices
        e = local.reshape(-1)
        rows = x.repeat_interleave(K, 0).unsqueeze(2)
        gate_up = torch.matmul(s["w_gate_up"][e].float(), rows.unsqueeze(1)).squeeze(3)                       # [T K, 2, I]
        h = gate_up[:, 0] / (1 + torch.exp(-gate_up[:, 0])) * gate_up[:, 1]
        out = torch.matmul(s["w_down"][e].float(), h.unsqueeze(2)).reshape(T, K, -1)
        return (torch.where(here, s["weights"], 0).unsqueeze(2) * torch.where(here.unsqueeze(2), out, 0)).sum(1).bfloat16()
    gate_up = torch.matmul(x, s["w_gate_up"].float().reshape(count, -1, case["H"]).transpose(1, 2))           # [count, T, 2 I]
    gate, up = gate_up[..., :case["I"]], gate_up[..., case["I"]:]
    h = gate / (1 + torch.exp(-gate)) * up
    share = torch.zeros(T, count, device=DEVICE).scatter_add_(1, local, torch.where(here, s["weights"], 0))
    chosen = torch.zeros(T, count, device=DEVICE).scatter_add_(1, local, here.float()) > 0
    out = torch.matmul(h, s["w_down"].float().transpose(1, 2))                                                # [count, T, H]
    return torch.where(chosen.t().unsqueeze(2), out * share.t().unsqueeze(2), 0).sum(0).bfloat16()


def _project_plain(s):
    x = s["x"].float()
    y = torch.matmul(x, s["w"].float().t())
    has = s["adapter_ids"] >= 0
    a = torch.where(has, s["adapter_ids"], 0).long()
    v = torch.matmul(s["a"][a].float(), x.unsqueeze(2))                                                       # [T, r, 1]
    delta = torch.matmul(s["b"][a].float(), v).squeeze(2) * s["scale"][a].unsqueeze(1)
    return (y + torch.where(has.unsqueeze(1), delta, 0)).bfloat16()


def run(s):
    case = s["case"]
    if not own:
        return dict(route=_route_plain, experts=_experts_plain, project=_project_plain)[case["op"]](s)
    if case["op"] == "route":
        s["mw"].mw_route(s["logits"], s["bias"], case["T"], case["E"], case["K"], s["flags"], case["scale"], s["ids"], s["weights"])
        return dict(ids=s["ids"], weights=s["weights"])
    if case["op"] == "experts":
        s["handle"].mw_experts_forward(s["x"], s["ids"], s["weights"], case["T"], s["y"])
    else:
        s["handle"].mw_project_forward(s["x"], s["adapter_ids"], case["T"], s["y"])
    return s["y"]


def work(case):
    """Means over the seeds: how many experts and adapters a batch uses depends on the draw."""
    T = case["T"]
    if case["op"] == "route":
        return dict(bytes=T * case["E"] * (2 if case["bf16"] else 4) + (case["E"] * 4 if case["bias"] else 0) + T * case["K"] * 8,
                    flops=4 * T * case["E"])
    H = case["H"]
    if case["op"] == "experts":
        E, K, count, I = case["E"], case["K"], case["count"], case["I"]
        if case["others"]:   # one local expert for certain, the other K - 1 picks anywhere among the rest
            picks = T * (1 + (K - 1) * (count - 1) / (E - 1))
            used = count * (1 - (1 - picks / T / count) ** T)
        else:
            picks = T * K
            used = count * (1 - (1 - K / E) ** T)
        return dict(bytes=used * 6 * H * I + 4 * T * H + 8 * T * K, flops=picks * 6 * H * I)
    O, n, r = case["O"], case["n"], case["r"]
    requests = -(-T // case["segment"])
    used = n * (1 - (1 - (1 - case["none"]) / n) ** requests)
    return dict(bytes=2 * (O * H + T * (H + O)) + used * 2 * r * (H + O) + 4 * T, flops=2 * T * O * H + 2 * T * (1 - case["none"]) * r * (H + O))


def exact(case, seed):
    s = prepare(case, seed)
    if case["op"] == "route":
        key = s["logits"].float()
        if s["bias"] is not None:
            key = key + s["bias"]            # the choice goes by the sum in 32 bits
        ids = torch.empty(case["T"], case["K"], dtype=torch.int64, device=DEVICE)
        rest = key.clone()
        expert = torch.arange(case["E"], device=DEVICE)
        for k in range(case["K"]):
            best = rest.amax(1, keepdim=True)
            ids[:, k] = torch.where(rest == best, expert, case["E"]).amin(1)
            rest.scatter_(1, ids[:, k:k + 1], float("-inf"))
        logits = s["logits"].double()
        p = torch.sigmoid(logits) if case["sigmoid"] else torch.softmax(logits, 1)
        w = p.gather(1, ids)
        if case["renorm"]:
            w = w / w.sum(1, keepdim=True)
        return dict(ids=ids.int(), weights=w * case["scale"])
    x = s["x"].double()
    if case["op"] == "experts":
        y = torch.zeros(case["T"], case["H"], dtype=torch.float64, device=DEVICE)
        for e in range(case["count"]):
            token, slot = torch.nonzero(s["ids"] == case["first"] + e, as_tuple=True)
            if token.numel() == 0:
                continue
            rows = x[token]
            gate, up = rows @ s["w_gate_up"][e, 0].double().t(), rows @ s["w_gate_up"][e, 1].double().t()
            out = (torch.nn.functional.silu(gate) * up) @ s["w_down"][e].double().t()
            y.index_add_(0, token, out * s["weights"][token, slot].double().unsqueeze(1))
        return y
    y = x @ s["w"].double().t()
    for a in range(case["n"]):
        token = torch.nonzero(s["adapter_ids"] == a).squeeze(1)
        if token.numel():
            y[token] += s["scale"][a].double() * ((x[token] @ s["a"][a].double().t()) @ s["b"][a].double().t())
    return y
