"""The operators around the token shuffle of an MoE block, as a program calls them: the norms that stand before and after
the block, the routing to experts, the experts' products on the dispatched rows, and the gradient of the combine.

A case is a dict of plain values.  `prepare` makes what a program holds before the call, `run` is one pass through an
operator: with `own` the calls of this framework, without it the plain form in elementary 32-bit torch operations, rounded
once at the end.  `exact` is the definition in 64 bits.

kinds
  route           scores, optional bias and groups, top-k, weights; with `grad` also the gradient of the logits
  norm            norm after a block with gate and residual scale, and the norm before the next block on the sum; with
                  `grad` also all gradients
  experts         gated product and down product of the expert-major rows
  experts_grad    gradients of both products: of the pre-activations, the rows and both weights; or (not `whole`) of the down
                  product and the activation alone, with the weight gradient in fp32
  combine_grad    gradients of the weighted combine: the experts' output rows and the weights
"""
import math

import torch

own = False

_DTYPE = {"bf16": torch.bfloat16, "f32": torch.float32}
_BYTES = {"bf16": 2, "f32": 4}
_EPS = 1e-6


def listed():
    return [
        # routing of a decode batch: launches and latency only (sigmoid scores, a bias for balance, device-limited groups)
        dict(name="route_decode", kind="route", N=128, E=256, k=8, score="sigmoid", bias=True, groups=8, keep=4, best=2, renorm=True, scale=2.5, logits="f32", grad=False),
        # routing of a long prefill batch, the token count of the largest configuration
        dict(name="route_prefill", kind="route", N=32768, E=256, k=8, score="sigmoid", bias=True, groups=8, keep=4, best=2, renorm=True, scale=2.5, logits="f32", grad=False),
        # softmax routing of a training batch, forward and backward
        dict(name="route_train", kind="route", N=16384, E=128, k=8, score="softmax", bias=False, groups=1, keep=1, best=1, renorm=True, scale=1.0, logits="bf16", grad=True),
        # one boundary between blocks while a few sequences are decoded
        dict(name="norm_token", kind="norm", N=4, H=7168, stream="bf16", block="bf16", gate="channel", scale=1.0, grad=False),
        # the same for a prefill batch
        dict(name="norm_prefill", kind="norm", N=16384, H=4096, stream="bf16", block="bf16", gate="channel", scale=0.5, grad=False),
        # a training batch with its residual stream in fp32, forward and backward
        dict(name="norm_train", kind="norm", N=8192, H=7168, stream="f32", block="bf16", gate="token", scale=0.5, grad=True),
        # a single token being decoded: eight experts' weights are read once
        dict(name="experts_token", kind="experts", N=1, E=128, k=8, H=4096, I=1280, routing="normal"),
        # a decode batch: nearly every expert's weights are read for a handful of rows
        dict(name="experts_decode", kind="experts", N=128, E=128, k=8, H=4096, I=1280, routing="normal"),
        # a prefill batch
        dict(name="experts_prefill", kind="experts", N=16384, E=128, k=8, H=4096, I=1280, routing="normal"),
        # a training batch of middle size with uneven experts
        dict(name="experts_train", kind="experts_grad", N=8192, E=64, k=4, H=2048, I=1408, routing="skewed", whole=True),
        # a ragged chunk: nothing is a power of two, fp32 residual stream
        dict(name="combine_grad_ragged", kind="combine_grad", N=1537, H=2880, k=6, E=160, D=5, y="bf16", dout="f32"),
        # the benchmark batch
        dict(name="combine_grad_batch", kind="combine_grad", N=8192, H=7168, k=8, E=256, D=8, y="bf16", dout="bf16"),
    ]


def _log_uniform(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def _plain_sizes(case):
    return 3072 not in (case.get("N"), case.get("H"), case.get("I"), 2 * case.get("I", 0), case["N"] * case.get("k", 1))


def _draw(rng):
    kind = rng.choice(["route", "route", "norm", "norm", "experts", "experts", "experts_grad", "combine_grad"])
    if kind == "route":
        E, groups = rng.choice([(16, 1), (32, 4), (60, 1), (64, 1), (64, 8), (128, 1), (128, 16), (160, 5), (160, 8), (256, 1), (256, 8), (384, 8), (512, 1)])
        k = rng.choice([1, 2, 4, 6, 8, 8, 10])
        score = rng.choice(["sigmoid", "softmax"])
        keep = max(-(-k * groups // E), (groups + 1) // 2)
        return dict(kind=kind, N=_log_uniform(rng, 1, 65536), E=E, k=k, score=score, bias=score == "sigmoid" and rng.random() < 0.7, groups=groups, keep=keep,
                    best=2 if score == "sigmoid" else 1, renorm=rng.random() < 0.8, scale=rng.choice([1.0, 2.5]), logits=rng.choice(["bf16", "f32"]), grad=rng.random() < 0.4)
    if kind == "norm":
        stream, block = rng.choice([("bf16", "bf16"), ("bf16", "bf16"), ("f32", "bf16"), ("f32", "f32")])
        grad = stream == "f32" and rng.random() < 0.6
        return dict(kind=kind, N=_log_uniform(rng, 1, 32768), H=8 * rng.randint(32, 1024), stream=stream, block=block,
                    gate=rng.choice(["none", "channel", "token"]), scale=rng.choice([1.0, 0.5]), grad=grad)
    if kind == "combine_grad":
        E, D = rng.choice([(16, 4), (64, 8), (128, 16), (160, 5), (256, 8)])
        y = rng.choice(["bf16", "bf16", "f32"])
        return dict(kind=kind, N=_log_uniform(rng, 16, 16384), H=8 * rng.randint(64, 1024), k=rng.choice([1, 2, 4, 6, 8]), E=E, D=D, y=y, dout=rng.choice(["f32", y]))
    E, k = rng.choice([(8, 2), (16, 2), (32, 4), (60, 4), (64, 4), (64, 8), (128, 8)])
    case = dict(kind=kind, N=_log_uniform(rng, 1 if kind == "experts" else 64, 32768), E=E, k=k, H=8 * rng.randint(64, 640), I=8 * rng.randint(32, 256),
                routing=rng.choice(["normal", "normal", "skewed"]))
    if rng.random() < 0.5:   # half of all models have sizes of whole 128s
        case["H"], case["I"] = max(1, case["H"] // 128) * 128, max(1, case["I"] // 128) * 128
    return dict(case, whole=rng.random() < 0.5) if kind == "experts_grad" else case


def draw(rng):
    case = _draw(rng)
    while work(case)["flops"] > 2.5e12 or work(case)["bytes"] > 4e9 or not _plain_sizes(case):
        case = _draw(rng) if case["N"] < 8 else dict(case, N=case["N"] * 2 // 3)
    return case


def _expert_order(chosen, E):
    """The stable order of the (token, expert) pairs by expert: slot -> pair, rows per expert."""
    flat = chosen.flatten().long()
    return torch.sort(flat, stable=True).indices, torch.bincount(flat, minlength=E)


def _inputs(case, seed):
    """The inputs alone, from the seed: shared by prepare and exact."""
    gen = torch.Generator(device="cuda").manual_seed(seed * 7919 + 17)
    N, kind = case["N"], case["kind"]

    def normal(*shape, dtype="f32", std=1.0, mean=0.0):
        t = torch.randn(shape, generator=gen, device="cuda", dtype=_DTYPE[dtype])
        if std != 1.0:
            t.mul_(std)
        return t.add_(mean) if mean else t

    if kind == "route":
        s = dict(logits=normal(N, case["E"], dtype=case["logits"]), bias=normal(case["E"], std=0.05) if case["bias"] else None)
        if case["grad"]:
            s["dw"] = normal(N, case["k"])
        return s
    if kind == "norm":
        H, stream, block = case["H"], case["stream"], case["block"]
        s = dict(r=normal(N, H, dtype=stream, std=2.0), y=normal(N, H, dtype=block, std=0.5), gain=normal(H, std=0.1, mean=1.0), next_gain=normal(H, std=0.1, mean=1.0),
                 gate={"none": None, "channel": normal(H, std=0.2, mean=0.5), "token": torch.sigmoid(normal(N))}[case["gate"]])
        if case["grad"]:
            s["dout"], s["dnext"] = normal(N, H, dtype=stream), normal(N, H, dtype=block)
        return s
    E, k, H = case["E"], case["k"], case["H"]
    score = torch.randn((N, E), generator=gen, device="cuda")
    if case.get("routing") == "skewed":   # some experts are more popular than others
        score += 0.5 * torch.randn((E,), generator=gen, device="cuda")
    top = score.topk(k, dim=1)
    s = dict(chosen=top.indices.to(torch.int32).contiguous())
    if kind == "combine_grad":
        return dict(s, w=torch.softmax(top.values, dim=1).contiguous(), y=normal(N * k, H, dtype=case["y"]), dout=normal(N, H, dtype=case["dout"]))
    I = case["I"]
    s["w_out"] = normal(E, H, I, dtype="bf16", std=I ** -0.5)
    if kind == "experts" or case["whole"]:
        s["x"], s["w_in"] = normal(N * k, H, dtype="bf16"), normal(E, 2 * I, H, dtype="bf16", std=H ** -0.5)
    if kind == "experts":
        return s
    return dict(s, pre=normal(N * k, 2 * I, dtype="bf16"), h=normal(N * k, I, dtype="bf16", std=0.6), dy=normal(N * k, H, dtype="bf16"))


def prepare(case, seed):
    s = dict(_inputs(case, seed), case=dict(case))
    N, kind = case["N"], case["kind"]

    def empty(*shape, dtype="f32"):
        return torch.empty(shape, dtype=torch.int32 if dtype == "i32" else _DTYPE[dtype], device="cuda")

    if kind == "route":
        s["out"] = dict(chosen=empty(N, case["k"], dtype="i32"), w=empty(N, case["k"]))
        if case["grad"]:
            s["out"]["dlogits"] = empty(N, case["E"], dtype=case["logits"])
        return s
    if kind == "norm":
        H, stream, block = case["H"], case["stream"], case["block"]
        s["out"] = dict(out=empty(N, H, dtype=stream), next=empty(N, H, dtype=block))
        if case["grad"]:
            s["out"].update(dr=empty(N, H, dtype=stream), dy=empty(N, H, dtype=block), dgain=empty(H), dnext_gain=empty(H))
            if case["gate"] != "none":
                s["out"]["dgate"] = empty(H if case["gate"] == "channel" else N)
        return s
    # the plan of the shuffle: by whose order the rows lie, for the plain form in tensors of its own
    E, k, H = case["E"], case["k"], case["H"]
    P = N * k
    order, count = _expert_order(s["chosen"], E)
    begin = torch.cumsum(count, 0) - count
    s["expert"] = s["chosen"].flatten().long()[order]
    s["most"] = int(count.max())
    s["place"] = s["expert"] * s["most"] + torch.arange(P, device="cuda") - begin[s["expert"]]
    s["slot"] = torch.empty_like(order)
    s["slot"][order] = torch.arange(P, device="cuda")
    if own:
        import paper_2512_22036_amd as fusco
        s["layout"] = fusco.Layout(N, k, E, case.get("D", 1))
        fusco.fusco_plan(s["layout"], s["chosen"])
    if kind == "combine_grad":
        s["out"] = dict(dy=empty(P, H, dtype=case["y"]), dw=empty(N, k))
    elif kind == "experts":
        s["out"] = dict(h=empty(P, case["I"], dtype="bf16"), y=empty(P, H, dtype="bf16"))
    else:
        I, whole = case["I"], case["whole"]
        s["out"] = dict(dpre=empty(P, 2 * I, dtype="bf16"), dw_out=empty(E, H, I, dtype="bf16" if whole else "f32"))
        if whole:
            s["out"].update(dx=empty(P, H, dtype="bf16"), dw_in=empty(E, 2 * I, H, dtype="bf16"))
    return s


def run(s):
    return (_run_own if own else _run_plain)(s)


def _run_own(s):
    import paper_2512_22036_amd as fusco
    case, out = s["case"], s["out"]
    kind = case["kind"]
    if kind == "route":
        how = dict(score=fusco.SCORE_SIGMOID if case["score"] == "sigmoid" else fusco.SCORE_SOFTMAX, renorm=case["renorm"], scale=case["scale"])
        fusco.fusco_route(s["logits"], out["chosen"], out["w"], bias=s["bias"], groups=case["groups"], keep_groups=case["keep"], group_best=case["best"], **how)
        if case["grad"]:
            fusco.fusco_route_backward(s["logits"], out["chosen"], s["dw"], out["dlogits"], **how)
    elif kind == "norm":
        fusco.fusco_norm_after(s["r"], s["y"], s["gain"], out["out"], gate=s["gate"], scale=case["scale"], next_gain=s["next_gain"], next_out=out["next"], eps=_EPS)
        if case["grad"]:
            fusco.fusco_norm_after_backward(s["dout"], s["y"], s["gain"], out["dr"], out["dy"], out["dgain"], gate=s["gate"], dgate=out.get("dgate"), scale=case["scale"],
                                            dnext=s["dnext"], out=out["out"], next_gain=s["next_gain"], dnext_gain=out["dnext_gain"], eps=_EPS)
    elif kind == "combine_grad":
        fusco.fusco_combine_backward(s["layout"], s["y"], s["w"], s["dout"], out["dy"], out["dw"])
    elif kind == "experts":
        fusco.fusco_experts_gated(s["layout"], s["x"], s["w_in"], out["h"])
        fusco.fusco_experts_linear(s["layout"], out["h"], s["w_out"], out["y"])
    else:
        fusco.fusco_experts_input_grad(s["layout"], s["dy"], s["w_out"], out["dpre"], pre=s["pre"])
        fusco.fusco_experts_weight_grad(s["layout"], s["dy"], s["h"], out["dw_out"])
        if case["whole"]:
            fusco.fusco_experts_input_grad(s["layout"], out["dpre"], s["w_in"], out["dx"])
            fusco.fusco_experts_weight_grad(s["layout"], out["dpre"], s["x"], out["dw_in"])
    return out


def _descending(v):
    """Places of a row's values from the largest down, equal ones by ascending place."""
    return torch.sort(v, dim=-1, descending=True, stable=True).indices


def _plain_route(s):
    case = s["case"]
    l = s["logits"].float()
    N, E = l.shape
    # the softmax's denominator is the same for a whole row and changes no order: scores are compared without it
    score = 1.0 / (1.0 + torch.exp(-l)) if case["score"] == "sigmoid" else torch.exp(l - l.amax(dim=1, keepdim=True))
    by = score if s["bias"] is None else score + s["bias"]
    if case["groups"] > 1:
        best = torch.sort(by.view(N, case["groups"], -1), dim=2, descending=True).values[:, :, :case["best"]].sum(dim=2)
        kept = torch.zeros_like(best, dtype=torch.bool).scatter_(1, _descending(best)[:, :case["keep"]], True)
        by = by.masked_fill(~kept.repeat_interleave(E // case["groups"], dim=1), -math.inf)
    chosen = _descending(by)[:, :case["k"]]
    p = score.gather(1, chosen)
    total = score.sum(dim=1, keepdim=True) if case["score"] == "softmax" else 1.0
    w = case["scale"] * p / (p.sum(dim=1, keepdim=True) if case["renorm"] else total)
    got = dict(chosen=chosen.to(torch.int32), w=w)
    if case["grad"]:
        p = p / total
        if case["renorm"]:
            sum_p = p.sum(dim=1, keepdim=True)
            dp = case["scale"] / sum_p * (s["dw"] - (s["dw"] * p).sum(dim=1, keepdim=True) / sum_p)
        else:
            dp = case["scale"] * s["dw"]
        dscore = torch.zeros_like(score).scatter_(1, chosen, dp)
        if case["score"] == "sigmoid":
            dl = dscore * score * (1.0 - score)
        else:
            q = score / total
            dl = q * (dscore - (dp * p).sum(dim=1, keepdim=True))
        got["dlogits"] = dl.to(s["logits"].dtype)
    return got


def _norm_forward(s, real):
    """The norm after a block and the one before the next, in the numbers of `real`; what the gradients need of them too."""
    case = s["case"]
    r, y, gain, next_gain = (s[n].to(real) for n in ("r", "y", "gain", "next_gain"))
    gate = 1.0 if s["gate"] is None else s["gate"].to(real)[:, None] if case["gate"] == "token" else s["gate"].to(real)
    inv = torch.rsqrt(y.square().mean(dim=1, keepdim=True) + _EPS)
    out = r + case["scale"] * gate * (y * inv * gain)
    next_inv = torch.rsqrt(out.square().mean(dim=1, keepdim=True) + _EPS)
    return y, gain, gate, next_gain, inv, out, next_inv


def _plain_norm(s):
    case, real = s["case"], torch.float32
    y, gain, gate, next_gain, inv, out, next_inv = _norm_forward(s, real)
    got = dict(out=out.to(_DTYPE[case["stream"]]), next=(out * next_inv * next_gain).to(_DTYPE[case["block"]]))
    if case["grad"]:
        dnext = s["dnext"].to(real)
        unit = out * next_inv
        got["dnext_gain"] = (dnext * unit).sum(dim=0)
        g = dnext * next_gain
        dr = s["dout"].to(real) + next_inv * (g - unit * (g * unit).mean(dim=1, keepdim=True))
        got["dr"] = dr.to(_DTYPE[case["stream"]])
        unit = y * inv
        du = case["scale"] * dr * gate
        if case["gate"] != "none":
            got["dgate"] = (case["scale"] * dr * unit * gain).sum(dim=1 if case["gate"] == "token" else 0)
        got["dgain"] = (du * unit).sum(dim=0)
        g = du * gain
        got["dy"] = (inv * (g - unit * (g * unit).mean(dim=1, keepdim=True))).to(_DTYPE[case["block"]])
    return got


def _by_expert(s, rows):
    """[E, most, columns]: the rows of every expert, padded with zeros, in 32 bits."""
    E, cols = s["case"]["E"], rows.shape[1]
    padded = torch.zeros((E * s["most"], cols), dtype=torch.float32, device="cuda")
    padded[s["place"]] = rows.float()
    return padded.view(E, s["most"], cols)


def _product(s, rows, w):
    """rows times the transposed weights of their expert, in 32 bits."""
    if 2 * rows.shape[0] <= w.shape[0]:   # a few rows: their experts' weights alone
        return torch.bmm(w[s["expert"]].float(), rows.float()[:, :, None])[:, :, 0]
    got = torch.bmm(_by_expert(s, rows), w.float().transpose(1, 2))
    return got.view(-1, w.shape[1])[s["place"]]


def _plain_experts(s):
    I = s["case"]["I"]
    pre = _product(s, s["x"], s["w_in"])
    gate, up = pre[:, :I], pre[:, I:]
    h = gate / (1.0 + torch.exp(-gate)) * up
    return dict(h=h.bfloat16(), y=_product(s, h, s["w_out"]).bfloat16())


def _gated_gradient(pre, dh):
    I = dh.shape[1]
    gate, up = pre[:, :I], pre[:, I:]
    sig = 1.0 / (1.0 + torch.exp(-gate))
    return torch.cat([dh * up * sig * (1.0 + gate * (1.0 - sig)), dh * gate * sig], dim=1)


def _plain_experts_grad(s):
    I, whole = s["case"]["I"], s["case"]["whole"]
    dy = _by_expert(s, s["dy"])
    dh = torch.bmm(dy, s["w_out"].float()).view(-1, I)[s["place"]]
    dpre = _gated_gradient(s["pre"].float(), dh)
    dw_out = torch.bmm(dy.transpose(1, 2), _by_expert(s, s["h"]))
    got = dict(dpre=dpre.bfloat16(), dw_out=dw_out.bfloat16() if whole else dw_out)
    if whole:
        padded, w = _by_expert(s, dpre), s["w_in"]
        got["dx"] = torch.bmm(padded, w.float()).view(-1, w.shape[2])[s["place"]].bfloat16()
        got["dw_in"] = torch.bmm(padded.transpose(1, 2), _by_expert(s, s["x"])).bfloat16()
    return got


def _plain_combine_grad(s):
    N, k, H = s["case"]["N"], s["case"]["k"], s["case"]["H"]
    dout, w = s["dout"].float(), s["w"]
    rows = s["y"][s["slot"]].float().view(N, k, H)
    dy = torch.empty_like(s["y"])
    dy[s["slot"]] = (w[:, :, None] * dout[:, None, :]).view(N * k, H).to(dy.dtype)
    return dict(dy=dy, dw=(rows * dout[:, None, :]).sum(dim=2))


def _run_plain(s):
    return {"route": _plain_route, "norm": _plain_norm, "experts": _plain_experts, "experts_grad": _plain_experts_grad, "combine_grad": _plain_combine_grad}[s["case"]["kind"]](s)


def work(case):
    N, kind = case["N"], case["kind"]
    if kind == "route":
        E, k, b = case["E"], case["k"], _BYTES[case["logits"]]
        bytes_ = N * E * b + 8 * N * k + (4 * E if case["bias"] else 0)
        if case["grad"]:
            bytes_ += N * E * b + 4 * N * k
        return {"bytes": bytes_, "flops": 6 * N * E * (2 if case["grad"] else 1)}
    if kind == "norm":
        H, a, b = case["H"], _BYTES[case["stream"]], _BYTES[case["block"]]
        gate = {"none": 0, "channel": 4 * H, "token": 4 * N}[case["gate"]]
        bytes_ = 2 * N * H * (a + b) + 8 * H + gate
        if case["grad"]:
            bytes_ += 2 * N * H * (a + b) + 8 * H + gate
        return {"bytes": bytes_, "flops": N * H * (30 if case["grad"] else 9)}
    k, H, E = case["k"], case["H"], case["E"]
    P = N * k
    if kind == "combine_grad":
        return {"bytes": 2 * P * H * _BYTES[case["y"]] + N * H * _BYTES[case["dout"]] + 12 * P, "flops": 3 * P * H}
    I = case["I"]
    used = E * (1.0 - (1.0 - k / E) ** N)   # experts that get rows
    if kind == "experts":
        return {"bytes": int(used * 6 * I * H) + P * (4 * H + 2 * I), "flops": 6 * P * H * I}
    if case["whole"]:   # dy, h, pre, dpre, x and dx; both weights and their gradients
        return {"bytes": int(used * 6 * I * H) + E * 6 * I * H + P * (6 * H + 10 * I), "flops": 12 * P * H * I}
    return {"bytes": int(used * 2 * I * H) + E * 4 * I * H + P * (2 * H + 10 * I), "flops": 4 * P * H * I}


def exact(case, seed):
    s = _inputs(case, seed)
    kind, N = case["kind"], case["N"]
    if kind == "route":
        return _exact_route(case, s)
    if kind == "norm":
        return _exact_norm(case, s)
    E, k, H = case["E"], case["k"], case["H"]
    order, count = _expert_order(s["chosen"], E)
    count = count.tolist()
    if kind == "combine_grad":
        dout, dy = s["dout"].double(), torch.empty((N * k, H), dtype=torch.float64, device="cuda")
        dw = torch.empty((N * k,), dtype=torch.float64, device="cuda")
        for rows in torch.arange(N * k, device="cuda").split(1 << 16):   # slots, a part at a time
            pair = order[rows]
            grad = dout[pair // k]
            dy[rows] = grad * s["w"].double().view(-1)[pair][:, None]
            dw[pair] = (grad * s["y"][rows].double()).sum(dim=1)
        return dict(dy=dy, dw=dw.view(N, k))
    I, begin, parts = case["I"], 0, []
    for e in range(E):
        rows = slice(begin, begin + count[e])
        begin += count[e]
        w_out = s["w_out"][e].double()
        if kind == "experts":
            gate, up = (s["x"][rows].double() @ s["w_in"][e].double().t()).split(I, dim=1)
            h = gate * torch.sigmoid(gate) * up
            parts.append(dict(h=h, y=h @ w_out.t()))
            continue
        (gate, up), dy = s["pre"][rows].double().split(I, dim=1), s["dy"][rows].double()
        dh, sig = dy @ w_out, torch.sigmoid(gate)
        dpre = torch.cat([dh * up * (sig + gate * sig * (1 - sig)), dh * gate * sig], dim=1)
        part = dict(dpre=dpre, dw_out=(dy.t() @ s["h"][rows].double())[None])
        if case["whole"]:
            part.update(dx=dpre @ s["w_in"][e].double(), dw_in=(dpre.t() @ s["x"][rows].double())[None])
        parts.append(part)
    return {name: torch.cat([p[name] for p in parts]) for name in parts[0]}


def _exact_route(case, s):
    logits = s["logits"].double().requires_grad_(case["grad"])
    score = torch.sigmoid(logits) if case["score"] == "sigmoid" else torch.softmax(logits, dim=1)
    by = score.detach() if s["bias"] is None else score.detach() + s["bias"].double()
    if case["groups"] > 1:
        size = case["E"] // case["groups"]
        best = by.view(-1, case["groups"], size).topk(case["best"], dim=2).values.sum(dim=2)
        worst_kept = best.topk(case["keep"], dim=1).values[:, -1:]
        by = torch.where((best >= worst_kept).repeat_interleave(size, dim=1), by, -torch.inf)
    p = score.gather(1, by.sort(dim=1, descending=True, stable=True).indices[:, :case["k"]])
    w = case["scale"] * (p / p.sum(dim=1, keepdim=True) if case["renorm"] else p)
    got = dict(chosen=None, w=w.detach())
    if case["grad"]:
        got["dlogits"], = torch.autograd.grad(w, logits, s["dw"].double())
    return got


def _exact_norm(case, s):
    real = {n: s[n].double().requires_grad_(case["grad"]) for n in ("r", "y", "gain", "gate", "next_gain") if s[n] is not None}

    def unit(v):
        return v / (v.pow(2).sum(dim=1, keepdim=True) / case["H"] + _EPS).sqrt()

    branch = unit(real["y"]) * real["gain"] * case["scale"]
    if case["gate"] != "none":
        branch = branch * (real["gate"].view(-1, 1) if case["gate"] == "token" else real["gate"])
    out = real["r"] + branch
    after = unit(out) * real["next_gain"]
    got = dict(out=out.detach(), next=after.detach())
    if case["grad"]:
        names = list(real)
        grads = torch.autograd.grad([out, after], [real[n] for n in names], [s["dout"].double(), s["dnext"].double()])
        got.update({"d" + n: g for n, g in zip(names, grads)})
    return got
