"""The block of an MoE layer in 8 bits, as a program calls it: rows and weights in 8-bit floating point (e4m3) with a scale per
block of 128, the experts' products on them, the backward pass from activations that were kept in 8 bits, and the whole layer
for a few tokens in one call.

A case is a dict of plain values.  `prepare` makes what a program holds before the call, `run` is one pass through an
operator: with `own` the calls of this framework, without it the plain form in elementary 32-bit torch operations, rounded
once at the end of every tensor that the path writes.  `exact` is the definition in 64 bits.

kinds
  scale8          rows [R, C] (a scale per 128 columns) or weights [E, M, C] (a scale per 128 x 128) to e4m3 and back to bf16, which holds
                  the values exactly as the scales are powers of two
  experts8        gated product of e4m3 rows with e4m3 weights, its result to e4m3, down product; scales are any fp32 numbers
  kept_grad       backward of both products, in bf16, from the rows, the pre-activations and the activations kept in e4m3
  few             the layer for a few tokens: from the tokens and their routing to the weighted sum of their experts' outputs, weights of
                  bf16 or e4m3
"""
import math

import torch

own = False

_DTYPE = {"bf16": torch.bfloat16, "f32": torch.float32, "fp8": torch.float8_e4m3fn}
_BYTES = {"bf16": 2, "f32": 4, "fp8": 1}
_BLOCK = 128
_LARGEST = 448.0    # of e4m3


def listed():
    return [
        # the tokens of a decode batch on their way to the dispatch: launches and latency only
        dict(name="scale8_decode", kind="scale8", of="rows", R=128, C=7168, x="bf16"),
        # a prefill batch's activations between the two products
        dict(name="scale8_prefill", kind="scale8", of="rows", R=131072, C=1280, x="bf16"),
        # the experts' weights after an optimizer step, from their fp32 masters
        dict(name="scale8_weights", kind="scale8", of="weights", E=64, M=1408, C=2048, x="f32"),
        # a decode batch: nearly every expert's weights are read for a handful of rows
        dict(name="experts8_decode", kind="experts8", N=128, E=128, k=8, H=4096, I=1280, routing="normal"),
        # a ragged batch: sizes that end inside a block of 128, uneven experts
        dict(name="experts8_ragged", kind="experts8", N=1537, E=60, k=6, H=2880, I=1040, routing="skewed"),
        # a prefill batch
        dict(name="experts8_prefill", kind="experts8", N=16384, E=128, k=8, H=4096, I=1280, routing="normal"),
        # a small fine-tuning batch, nothing a power of two
        dict(name="kept_grad_ragged", kind="kept_grad", N=301, E=16, k=2, H=1040, I=528, routing="normal"),
        # a training batch of middle size with uneven experts
        dict(name="kept_grad_train", kind="kept_grad", N=8192, E=64, k=4, H=2048, I=1408, routing="skewed"),
        # a single token being decoded: eight experts' weights are read once
        dict(name="few_token", kind="few", N=1, E=128, k=8, H=4096, I=1280, weights="bf16", out="bf16"),
        # the same with weights of half the bytes
        dict(name="few_token_fp8", kind="few", N=1, E=128, k=8, H=4096, I=1280, weights="fp8", out="bf16"),
        # a few tokens, checked by a model that speculates: five rows, sizes that end inside a block
        dict(name="few_ragged", kind="few", N=5, E=60, k=6, H=2880, I=1040, weights="bf16", out="f32"),
        # a small decode batch: most experts are read for one or two tokens each
        dict(name="few_batch_fp8", kind="few", N=16, E=128, k=8, H=4096, I=1280, weights="fp8", out="bf16"),
    ]


def _log_uniform(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def _size(rng, lo, hi):
    """A row size: whole blocks of 128 in half of all models, else any multiple of 16."""
    v = 16 * rng.randint(lo // 16, hi // 16)
    return max(1, v // 128) * 128 if rng.random() < 0.5 else v


def _draw(rng):
    kind = rng.choice(["scale8", "scale8", "experts8", "experts8", "kept_grad", "few", "few", "few"])
    if kind == "scale8":
        x = rng.choice(["bf16", "bf16", "f32"])
        if rng.random() < 0.7:
            return dict(kind=kind, of="rows", R=_log_uniform(rng, 1, 262144), C=_size(rng, 256, 8192), x=x)
        return dict(kind=kind, of="weights", E=rng.choice([1, 8, 16, 60, 64, 128]), M=_size(rng, 256, 4096), C=_size(rng, 256, 7168), x=x)
    if kind == "few":
        E, k = rng.choice([(8, 2), (16, 2), (32, 4), (60, 4), (60, 6), (64, 8), (128, 8), (160, 6), (256, 8)])
        return dict(kind=kind, N=_log_uniform(rng, 1, 64), E=E, k=k, H=_size(rng, 512, 7168), I=_size(rng, 256, 2048), weights=rng.choice(["bf16", "fp8"]), out=rng.choice(["bf16", "f32"]))
    E, k = rng.choice([(8, 2), (16, 2), (32, 4), (60, 4), (64, 4), (64, 8), (128, 8)])
    return dict(kind=kind, N=_log_uniform(rng, 8 if kind == "experts8" else 64, 32768), E=E, k=k, H=_size(rng, 512, 5120), I=_size(rng, 256, 2048), routing=rng.choice(["normal", "normal", "skewed"]))


def draw(rng):
    case = _draw(rng)
    while work(case)["flops"] > 2.5e12 or work(case)["bytes"] > 4e9:
        smaller = {n: case[n] * 2 // 3 for n in ("N", "R") if case.get(n, 0) > 8}
        case = dict(case, **smaller) if smaller else _draw(rng)
    return case


def _blocks(n):
    return -(-n // _BLOCK)


def _over_columns(scale, C):
    """A value per block as a value per column."""
    return scale.repeat_interleave(_BLOCK, dim=-1)[..., :C]


def _over_both(scale, M, C):
    return _over_columns(scale, C).repeat_interleave(_BLOCK, dim=-2)[..., :M, :]


def _largest_by_block(x, of):
    """The largest absolute value of every block of the last dimension, or of the last two."""
    M, C = x.shape[-2:]
    a = torch.nn.functional.pad(x.abs(), (0, _blocks(C) * _BLOCK - C) + ((0, _blocks(M) * _BLOCK - M) if of == "weights" else ()))
    if of == "rows":
        return a.view(*a.shape[:-1], _blocks(C), _BLOCK).amax(dim=-1)
    return a.view(a.shape[0], _blocks(M), _BLOCK, _blocks(C), _BLOCK).amax(dim=(2, 4))


def _scaled(x, of):
    """e4m3 values and their scales: the smallest powers of two with which the largest of a block stays within e4m3."""
    x = x.float()
    largest = _largest_by_block(x, of)
    mantissa, exponent = torch.frexp(largest)
    exponent = (exponent - 9 + (mantissa > _LARGEST / 512).int()).clamp(min=-126)
    power = ((exponent + 127) << 23).view(torch.float32)   # 2 ^ exponent, exactly
    scale = torch.where(largest > 0, power, torch.ones_like(power))
    whole = _over_columns(scale, x.shape[-1]) if of == "rows" else _over_both(scale, *x.shape[-2:])
    return (x / whole).to(_DTYPE["fp8"]), scale


def _rows_of(q, scale, real=torch.float32):
    return q.to(real) * _over_columns(scale.to(real), q.shape[-1])


def _weights_of(q, scale, real=torch.float32):
    return q.to(real) * _over_both(scale.to(real), *q.shape[-2:])


def _expert_order(chosen, E):
    """The stable order of the (token, expert) pairs by expert: slot -> pair, rows per expert."""
    flat = chosen.flatten().long()
    return torch.sort(flat, stable=True).indices, torch.bincount(flat, minlength=E)


def _inputs(case, seed):
    """The inputs alone, from the seed: shared by prepare and exact."""
    gen = torch.Generator(device="cuda").manual_seed(seed * 7919 + 29)
    kind = case["kind"]

    def normal(*shape, dtype="f32", std=1.0):
        return torch.randn(shape, generator=gen, device="cuda", dtype=_DTYPE[dtype]).mul_(std)

    def eight(*shape, scales, std):
        """Values as a quantiser leaves them: normal ones whose largest is near the end of e4m3, scales of any size."""
        q = normal(*shape, dtype="bf16", std=130.0).clamp_(-_LARGEST, _LARGEST).to(_DTYPE["fp8"])
        return q, torch.rand(scales, generator=gen, device="cuda").mul_(0.4).add_(0.8).mul_(std / 130.0)

    if kind == "scale8":
        if case["of"] == "weights":
            return dict(x=normal(case["E"], case["M"], case["C"], dtype=case["x"], std=case["C"] ** -0.5))
        x = normal(case["R"], case["C"], dtype=case["x"])
        return dict(x=x.mul_(torch.exp(normal(case["R"], 1)).to(x.dtype)))   # tokens differ in size
    N, E, k, H, I = (case[n] for n in ("N", "E", "k", "H", "I"))
    P = N * k
    score = torch.randn((N, E), generator=gen, device="cuda")
    if case.get("routing") == "skewed":   # some experts are more popular than others
        score += 0.5 * torch.randn((E,), generator=gen, device="cuda")
    top = score.topk(k, dim=1)
    s = dict(chosen=top.indices.to(torch.int32).contiguous())
    if kind == "kept_grad":
        s.update(dy=normal(P, H, dtype="bf16"), w_in=normal(E, 2 * I, H, dtype="bf16", std=H ** -0.5), w_out=normal(E, H, I, dtype="bf16", std=I ** -0.5))
        for name, cols, std in (("x", H, 1.0), ("pre", 2 * I, 1.0), ("h", I, 0.6)):
            s[name], s[name + "_scale"] = _scaled(normal(P, cols, dtype="bf16", std=std), "rows")
        return s
    if kind == "few":
        s.update(x=normal(N, H, dtype="bf16"), w=torch.softmax(top.values, dim=1).contiguous(), w_in_scale=None, w_out_scale=None)
        if case["weights"] == "bf16":
            return dict(s, w_in=normal(E, 2 * I, H, dtype="bf16", std=H ** -0.5), w_out=normal(E, H, I, dtype="bf16", std=I ** -0.5))
    else:
        s["x"], s["x_scale"] = eight(P, H, scales=(P, _blocks(H)), std=1.0)
    # gate and up rows are blocks of their own
    s["w_in"], s["w_in_scale"] = eight(E, 2 * I, H, scales=(E, 2 * _blocks(I), _blocks(H)), std=H ** -0.5)
    s["w_out"], s["w_out_scale"] = eight(E, H, I, scales=(E, _blocks(H), _blocks(I)), std=I ** -0.5)
    return s


def prepare(case, seed):
    s = dict(_inputs(case, seed), case=dict(case))
    kind = case["kind"]

    def empty(*shape, dtype="f32"):
        return torch.empty(shape, dtype=_DTYPE[dtype], device="cuda")

    if kind == "scale8":
        shape = tuple(s["x"].shape)
        s["q"] = empty(*shape, dtype="fp8")
        scales = (shape[0], _blocks(shape[1])) if case["of"] == "rows" else (shape[0], _blocks(shape[1]), _blocks(shape[2]))
        s["out"] = dict(scale=empty(*scales), back=empty(*shape, dtype="bf16"))
        return s
    N, E, k, H, I = (case[n] for n in ("N", "E", "k", "H", "I"))
    P = N * k
    # by whose order the rows lie, for the plain form in tensors of its own
    order, count = _expert_order(s["chosen"], E)
    begin = torch.cumsum(count, 0) - count
    s["order"], s["expert"] = order, s["chosen"].flatten().long()[order]
    s["most"] = int(count.max())
    s["place"] = s["expert"] * s["most"] + torch.arange(P, device="cuda") - begin[s["expert"]]
    if kind == "few":
        s["out"] = empty(N, H, dtype=case["out"])
        if own:
            import paper_2512_22036_amd as fusco
            s["scratch"] = torch.empty(fusco.fusco_moe_few_scratch_bytes(N, k, I), dtype=torch.uint8, device="cuda")
        return s
    if own:
        import paper_2512_22036_amd as fusco
        s["layout"] = fusco.Layout(N, k, E, 1)
        fusco.fusco_plan(s["layout"], s["chosen"])
    if kind == "experts8":
        s["h8"], s["h8_scale"] = empty(P, I, dtype="fp8"), empty(P, _blocks(I))
        s["out"] = dict(h=empty(P, I, dtype="bf16"), y=empty(P, H, dtype="bf16"))
    else:
        s["out"] = dict(dpre=empty(P, 2 * I, dtype="bf16"), dx=empty(P, H, dtype="bf16"), dw_in=empty(E, 2 * I, H, dtype="bf16"), dw_out=empty(E, H, I))
    return s


def run(s):
    return (_run_own if own else _run_plain)(s)


def _run_own(s):
    import paper_2512_22036_amd as fusco
    kind, out = s["case"]["kind"], s["out"]
    if kind == "scale8":
        fusco.fusco_to_fp8(s["x"], s["q"], out["scale"])
        fusco.fusco_from_fp8(s["q"], out["scale"], out["back"])
    elif kind == "experts8":
        fusco.fusco_experts_gated_fp8(s["layout"], s["x"], s["x_scale"], s["w_in"], s["w_in_scale"], out["h"])
        fusco.fusco_to_fp8(out["h"], s["h8"], s["h8_scale"])
        fusco.fusco_experts_linear_fp8(s["layout"], s["h8"], s["h8_scale"], s["w_out"], s["w_out_scale"], out["y"])
    elif kind == "kept_grad":
        fusco.fusco_experts_input_grad(s["layout"], s["dy"], s["w_out"], out["dpre"], pre=s["pre"], pre_scale=s["pre_scale"])
        fusco.fusco_experts_weight_grad(s["layout"], s["dy"], s["h"], out["dw_out"], x_scale=s["h_scale"])
        fusco.fusco_experts_input_grad(s["layout"], out["dpre"], s["w_in"], out["dx"])
        fusco.fusco_experts_weight_grad(s["layout"], out["dpre"], s["x"], out["dw_in"], x_scale=s["x_scale"])
    else:
        fusco.fusco_moe_few(s["x"], s["chosen"], s["w"], s["w_in"], s["w_out"], out, w_in_scale=s["w_in_scale"], w_out_scale=s["w_out_scale"], scratch=s["scratch"])
    return out


def _plain_scale8(s):
    of = s["case"]["of"]
    q, scale = _scaled(s["x"], of)
    return dict(scale=scale, back=(_rows_of if of == "rows" else _weights_of)(q, scale).bfloat16())


def _by_expert(s, rows):
    """[E, most, columns]: the rows of every expert, padded with zeros, in 32 bits."""
    E, cols = s["case"]["E"], rows.shape[1]
    padded = torch.zeros((E * s["most"], cols), dtype=torch.float32, device="cuda")
    padded[s["place"]] = rows.float()
    return padded.view(E, s["most"], cols)


def _weights(s, name, experts=None):
    """An expert's weights in 32 bits, or those of some experts."""
    q, scale = s[name], s.get(name + "_scale")
    if experts is not None:
        q, scale = q[experts], None if scale is None else scale[experts]
    if scale is None:
        return q.float()
    if name == "w_out":
        return _weights_of(q, scale)
    halves = q.view(2 * q.shape[0], -1, q.shape[2])   # gate rows and up rows
    return _weights_of(halves, scale.view(halves.shape[0], -1, scale.shape[2])).view(q.shape)


def _product(s, rows, name):
    """rows times the transposed weights of their expert, in 32 bits."""
    if 2 * rows.shape[0] <= s["case"]["E"]:   # a few rows: their experts' weights alone
        return torch.bmm(_weights(s, name, s["expert"]), rows.float()[:, :, None])[:, :, 0]
    got = torch.bmm(_by_expert(s, rows), _weights(s, name).transpose(1, 2))
    return got.view(-1, got.shape[2])[s["place"]]


def _gated(pre):
    gate, up = pre.chunk(2, dim=1)
    return gate / (1.0 + torch.exp(-gate)) * up


def _plain_experts8(s):
    h = _gated(_product(s, _rows_of(s["x"], s["x_scale"]), "w_in")).bfloat16()
    return dict(h=h, y=_product(s, _rows_of(*_scaled(h, "rows")), "w_out").bfloat16())


def _plain_kept_grad(s):
    I = s["case"]["I"]
    dy = _by_expert(s, s["dy"])
    dh = torch.bmm(dy, s["w_out"].float()).view(-1, I)[s["place"]]
    gate, up = _rows_of(s["pre"], s["pre_scale"]).split(I, dim=1)
    sig = 1.0 / (1.0 + torch.exp(-gate))
    dpre = torch.cat([dh * up * sig * (1.0 + gate * (1.0 - sig)), dh * gate * sig], dim=1).bfloat16()
    dw_out = torch.bmm(dy.transpose(1, 2), _by_expert(s, _rows_of(s["h"], s["h_scale"])))
    padded, w = _by_expert(s, dpre), s["w_in"]
    dx = torch.bmm(padded, w.float()).view(-1, w.shape[2])[s["place"]]
    dw_in = torch.bmm(padded.transpose(1, 2), _by_expert(s, _rows_of(s["x"], s["x_scale"])))
    return dict(dpre=dpre, dx=dx.bfloat16(), dw_in=dw_in.bfloat16(), dw_out=dw_out)


def _plain_few(s):
    N, k, H = s["case"]["N"], s["case"]["k"], s["case"]["H"]
    rows = s["x"].float()[s["order"] // k]
    y = _product(s, _gated(_product(s, rows, "w_in")), "w_out")
    pairs = torch.empty_like(y)
    pairs[s["order"]] = y
    return (pairs.view(N, k, H) * s["w"][:, :, None]).sum(dim=1).to(_DTYPE[s["case"]["out"]])


def _run_plain(s):
    return {"scale8": _plain_scale8, "experts8": _plain_experts8, "kept_grad": _plain_kept_grad, "few": _plain_few}[s["case"]["kind"]](s)


def work(case):
    kind = case["kind"]
    if kind == "scale8":
        if case["of"] == "rows":
            n, scales = case["R"] * case["C"], case["R"] * _blocks(case["C"])
        else:
            n, scales = case["E"] * case["M"] * case["C"], case["E"] * _blocks(case["M"]) * _blocks(case["C"])
        # there: x in, e4m3 and scales out; back: those in, bf16 out
        return {"bytes": n * (_BYTES[case["x"]] + 4) + 8 * scales, "flops": 4 * n}
    N, E, k, H, I = (case[n] for n in ("N", "E", "k", "H", "I"))
    P = N * k
    used = E * (1.0 - (1.0 - k / E) ** N)   # experts that get rows
    if kind == "few":
        return {"bytes": int(used * 3 * I * H * _BYTES[case["weights"]]) + N * H * (2 + _BYTES[case["out"]]) + 8 * P, "flops": 6 * P * H * I}
    if kind == "experts8":   # rows, h out and in, h in e4m3 out and in, y
        return {"bytes": int(used * 3 * I * H) + P * (3 * H + 6 * I), "flops": 6 * P * H * I}
    # dy, dpre and dx, three kept tensors; both weights and their gradients, that of w_out in fp32
    return {"bytes": int(used * 6 * I * H) + E * 8 * I * H + P * (5 * H + 7 * I), "flops": 12 * P * H * I}


def _exact_scaled(x, of):
    """The definition once more: the values that e4m3 with the scales stands for, in 64 bits, and the scales."""
    x = x.double()
    powers = torch.tensor([2.0 ** i for i in range(-140, 129)], dtype=torch.float64, device="cuda")
    largest = _largest_by_block(x, of)
    scale = powers[14:][torch.searchsorted(powers[14:] * _LARGEST, largest)]   # the first one that is enough
    scale = torch.where(largest > 0, scale, 1.0)
    whole = _over_columns(scale, x.shape[-1]) if of == "rows" else _over_both(scale, *x.shape[-2:])
    v = x / whole
    below = torch.searchsorted(powers, v.abs().clamp(min=2.0 ** -6), right=True) - 1   # the power of two that v begins with
    step = powers[below - 3]                                                           # e4m3: four significant bits down to 2^-6
    return torch.round(v / step) * step * whole, scale


def exact(case, seed):
    s = _inputs(case, seed)
    kind = case["kind"]
    if kind == "scale8":
        back, scale = _exact_scaled(s["x"], case["of"])
        return dict(scale=scale, back=back)
    N, E, k, H, I = (case[n] for n in ("N", "E", "k", "H", "I"))
    order, count = _expert_order(s["chosen"], E)
    count = count.tolist()

    def weights(name, e):
        w = s[name][e]
        if s.get(name + "_scale") is None:
            return w.double()
        scale = s[name + "_scale"][e]
        if name == "w_out":
            return _weights_of(w, scale, torch.float64)
        n = scale.shape[0] // 2
        return torch.cat([_weights_of(w[:I], scale[:n], torch.float64), _weights_of(w[I:], scale[n:], torch.float64)])

    out = torch.zeros((N, H), dtype=torch.float64, device="cuda")
    begin, parts = 0, []
    for e in range(E):
        rows = slice(begin, begin + count[e])
        begin += count[e]
        if kind == "few":
            if count[e]:
                pair = order[rows]
                gate, up = (s["x"][pair // k].double() @ weights("w_in", e).t()).split(I, dim=1)
                out.index_add_(0, pair // k, (gate * torch.sigmoid(gate) * up) @ weights("w_out", e).t() * s["w"].double().flatten()[pair][:, None])
            continue
        if kind == "experts8":
            gate, up = (_rows_of(s["x"][rows], s["x_scale"][rows], torch.float64) @ weights("w_in", e).t()).split(I, dim=1)
            h = gate * torch.sigmoid(gate) * up
            parts.append(dict(h=h, y=_exact_scaled(h.bfloat16(), "rows")[0] @ weights("w_out", e).t()))
            continue
        kept = {n: _rows_of(s[n][rows], s[n + "_scale"][rows], torch.float64) for n in ("x", "pre", "h")}
        (gate, up), dy = kept["pre"].split(I, dim=1), s["dy"][rows].double()
        dh, sig = dy @ s["w_out"][e].double(), torch.sigmoid(gate)
        dpre = torch.cat([dh * up * (sig + gate * sig * (1 - sig)), dh * gate * sig], dim=1)
        parts.append(dict(dpre=dpre, dx=dpre @ s["w_in"][e].double(), dw_in=(dpre.t() @ kept["x"])[None], dw_out=(dy.t() @ kept["h"])[None]))
    return out if kind == "few" else {name: torch.cat([p[name] for p in parts]) for name in parts[0]}
