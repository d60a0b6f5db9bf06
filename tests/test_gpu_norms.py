"""The norms around a block and their gradients against the formulas in 64 bits.

Tolerance.  Sums over a row are at most 64 additions deep (32 values in a thread, six steps in a wave, 16 waves): 64 * 2^-24 of the
sum of their terms' sizes; sums over rows at most 160 deep at the sizes used here.  Every result is then compared in backward form: the
same formula with all terms taken by their size, times the number of roundings on the way (SUM, counted generously as 512), plus the
rounding of the result to its type."""
import pytest
import torch

pytestmark = pytest.mark.gpu

SUM = 512 * 2.0 ** -24
EPS = 1e-6
HALF = {torch.bfloat16: 2.0 ** -8, torch.float32: 2.0 ** -24}


def fusco():
    import paper_2512_22036_amd as f
    f.load_library()
    return f


TYPES = [(torch.bfloat16, torch.bfloat16), (torch.float32, torch.bfloat16), (torch.float32, torch.float32)]
SHAPES = [(1, 8), (3, 64), (2, 520), (1, 4096), (4, 7168), (5, 8200), (2, 32768), (37, 1024), (600, 264), (1100, 512), (1030, 2880), (1025, 7168), (1024, 16392)]


def inputs(N, H, stream, block, gate, params=torch.float32, seed=0):
    gen = torch.Generator(device="cuda").manual_seed(seed + N * 31 + H)

    def normal(*shape, dtype, std=1.0, mean=0.0):
        return (torch.randn(shape, generator=gen, device="cuda") * std + mean).to(dtype)

    s = dict(r=normal(N, H, dtype=stream, std=2.0), y=normal(N, H, dtype=block, std=0.5), gain=normal(H, dtype=params, std=0.1, mean=1.0),
             next_gain=normal(H, dtype=params, std=0.1, mean=1.0), dout=normal(N, H, dtype=stream), dnext=normal(N, H, dtype=block))
    s["gate"] = {"none": None, "channel": normal(H, dtype=params), "token": normal(N, dtype=params)}[gate]
    return s


def kind(f, gate):
    return {"none": None, "channel": f.GATE_CHANNEL, "token": f.GATE_TOKEN}[gate]


def gate64(s, gate):
    return 1.0 if gate == "none" else s["gate"].double()[:, None] if gate == "token" else s["gate"].double()


def inv64(x):
    return 1.0 / (x.square().mean(dim=1, keepdim=True) + EPS).sqrt()


def near(got, want, size):
    off = (got.double() - want).abs() - (SUM * size + HALF[got.dtype] * (want.abs() + SUM * size))
    assert bool((off <= 0).all()), "off by %g more than the bound" % float(off.max())


@pytest.mark.parametrize("stream,block", TYPES)
@pytest.mark.parametrize("N,H", SHAPES)
def test_before(N, H, stream, block):
    f = fusco()
    s = inputs(N, H, stream, block, "none")
    out = torch.empty((N, H), dtype=block, device="cuda")
    f.fusco_norm_before(s["r"], s["gain"], out, eps=EPS)
    x = s["r"].double()
    want = x * inv64(x) * s["gain"].double()
    near(out, want, want.abs())


@pytest.mark.parametrize("gate", ["none", "channel", "token"])
@pytest.mark.parametrize("stream,block", TYPES)
@pytest.mark.parametrize("N,H", SHAPES)
def test_after(N, H, stream, block, gate):
    f = fusco()
    s = inputs(N, H, stream, block, gate)
    out, nxt = torch.empty((N, H), dtype=stream, device="cuda"), torch.empty((N, H), dtype=block, device="cuda")
    f.fusco_norm_after(s["r"], s["y"], s["gain"], out, gate=s["gate"], gate_kind=kind(f, gate), scale=0.5, next_gain=s["next_gain"], next_out=nxt, eps=EPS)
    y, r = s["y"].double(), s["r"].double()
    u = 0.5 * gate64(s, gate) * y * inv64(y) * s["gain"].double()
    want = r + u
    size = r.abs() + u.abs()
    near(out, want, size)
    near(nxt, want * inv64(want) * s["next_gain"].double(), size * inv64(want) * s["next_gain"].double().abs() * 2)
    alone = torch.empty_like(out)
    f.fusco_norm_after(s["r"], s["y"], s["gain"], alone, gate=s["gate"], gate_kind=kind(f, gate), scale=0.5, eps=EPS)
    assert torch.equal(alone, out)
    r, y = s["r"].clone(), s["y"].clone()       # in place of its inputs
    f.fusco_norm_after(r, y, s["gain"], r, gate=s["gate"], gate_kind=kind(f, gate), scale=0.5, next_gain=s["next_gain"], next_out=y, eps=EPS)
    assert torch.equal(r, out) and torch.equal(y, nxt)


@pytest.mark.parametrize("gate", ["channel", "token"])
def test_parameters_in_bf16(gate):
    f = fusco()
    s = inputs(9, 1000, torch.bfloat16, torch.bfloat16, gate, params=torch.bfloat16)
    wide = {n: s[n].float() for n in ("gain", "next_gain", "gate")}
    outs = []
    for p in (s, wide):
        out, nxt = torch.empty_like(s["r"]), torch.empty_like(s["r"])
        f.fusco_norm_after(s["r"], s["y"], p["gain"], out, gate=p["gate"], next_gain=p["next_gain"], next_out=nxt, eps=EPS)
        dr, dy, dg, dn, dgate = (torch.empty_like(s["r"]), torch.empty_like(s["r"]), torch.empty(1000, device="cuda"), torch.empty(1000, device="cuda"),
                                 torch.empty(p["gate"].shape, device="cuda"))
        f.fusco_norm_after_backward(s["dout"], s["y"], p["gain"], dr, dy, dg, gate=p["gate"], dgate=dgate, dnext=s["dnext"], out=out, next_gain=p["next_gain"], dnext_gain=dn, eps=EPS)
        outs.append([out, nxt, dr, dy, dg, dn, dgate])
    assert all(torch.equal(a, b) for a, b in zip(*outs))


def after_gradients(s, out, gate, scale, with_next, with_dout):
    """The gradients in 64 bits and the sizes of their terms; `out` as it was written."""
    y, gain, next_gain = s["y"].double(), s["gain"].double(), s["next_gain"].double()
    g = gate64(s, gate)
    dr = s["dout"].double() if with_dout else torch.zeros_like(y)
    size = dr.abs()
    got = {}
    if with_next:
        o, dn = out.double(), s["dnext"].double()
        inv, g2 = inv64(o), s["dnext"].double() * next_gain
        dr = dr + inv * (g2 - o * inv ** 2 * (g2 * o).mean(dim=1, keepdim=True))
        size = size + inv * (g2.abs() + o.abs() * inv ** 2 * (g2 * o).abs().mean(dim=1, keepdim=True))
        got["dnext_gain"] = ((dn * o * inv).sum(dim=0), (dn * o * inv).abs().sum(dim=0))
    got["dr"] = (dr, size)
    inv = inv64(y)
    unit = y * inv
    per = scale * dr * unit * gain, abs(scale) * size * (unit * gain).abs()
    if gate != "none":
        got["dgate"] = tuple(t.sum(dim=1 if gate == "token" else 0) for t in per)
    du, du_size = scale * g * dr, abs(scale) * (g.abs() if gate != "none" else 1.0) * size
    got["dgain"] = ((du * unit).sum(dim=0), (du_size * unit.abs()).sum(dim=0))
    g1, g1_size = du * gain, du_size * gain.abs()
    got["dy"] = (inv * (g1 - y * inv ** 2 * (g1 * y).mean(dim=1, keepdim=True)), inv * (g1_size + y.abs() * inv ** 2 * (g1_size * y.abs()).mean(dim=1, keepdim=True)))
    return got


@pytest.mark.parametrize("with_next,with_dout", [(True, True), (True, False), (False, True)])
@pytest.mark.parametrize("gate", ["none", "channel", "token"])
@pytest.mark.parametrize("stream,block", TYPES)
@pytest.mark.parametrize("N,H", SHAPES)
def test_after_backward(N, H, stream, block, gate, with_next, with_dout):
    f = fusco()
    s = inputs(N, H, stream, block, gate, seed=1)
    out = s["r"]                                # any stream will do
    dr, dy = torch.empty((N, H), dtype=stream, device="cuda"), torch.empty((N, H), dtype=block, device="cuda")
    dgain, dnext_gain = torch.empty(H, device="cuda"), torch.empty(H, device="cuda")
    dgate = None if gate == "none" else torch.empty(s["gate"].shape, device="cuda")
    more = dict(dnext=s["dnext"], out=out, next_gain=s["next_gain"], dnext_gain=dnext_gain) if with_next else {}
    f.fusco_norm_after_backward(s["dout"] if with_dout else None, s["y"], s["gain"], dr, dy, dgain, gate=s["gate"], dgate=dgate, gate_kind=kind(f, gate), scale=0.5, eps=EPS, **more)
    for name, (want, size) in after_gradients(s, out, gate, 0.5, with_next, with_dout).items():
        near(dict(dr=dr, dy=dy, dgain=dgain, dgate=dgate, dnext_gain=dnext_gain)[name], want, size)


@pytest.mark.parametrize("with_dres", [False, True])
@pytest.mark.parametrize("stream,block", TYPES)
@pytest.mark.parametrize("N,H", SHAPES)
def test_before_backward(N, H, stream, block, with_dres):
    f = fusco()
    s = inputs(N, H, stream, block, "none", seed=2)
    dx, dgain = torch.empty((N, H), dtype=stream, device="cuda"), torch.empty(H, device="cuda")
    f.fusco_norm_before_backward(s["dnext"], s["r"], s["next_gain"], dx, dgain, dres=s["dout"] if with_dres else None, eps=EPS)
    want = after_gradients(s, s["r"], "none", 1.0, True, with_dres)
    near(dx, *want["dr"])
    near(dgain, *want["dnext_gain"])


@pytest.mark.parametrize("gate", ["none", "channel", "token"])
def test_gradient_by_differences(gate):
    f = fusco()
    N, H = 6, 40
    s = inputs(N, H, torch.float32, torch.float32, gate, seed=3)
    out, nxt = torch.empty((N, H), device="cuda"), torch.empty((N, H), device="cuda")
    f.fusco_norm_after(s["r"], s["y"], s["gain"], out, gate=s["gate"], scale=0.7, next_gain=s["next_gain"], next_out=nxt, eps=EPS)
    got = dict(r=torch.empty_like(out), y=torch.empty_like(out), gain=torch.empty(H, device="cuda"), next_gain=torch.empty(H, device="cuda"))
    if gate != "none":
        got["gate"] = torch.empty(s["gate"].shape, device="cuda")
    f.fusco_norm_after_backward(s["dout"], s["y"], s["gain"], got["r"], got["y"], got["gain"], gate=s["gate"], dgate=got.get("gate"), scale=0.7,
                                dnext=s["dnext"], out=out, next_gain=s["next_gain"], dnext_gain=got["next_gain"], eps=EPS)

    def loss(p):
        y, g = p["y"], 1.0 if gate == "none" else p["gate"][:, None] if gate == "token" else p["gate"]
        o = p["r"] + 0.7 * g * y * inv64(y) * p["gain"]
        return (o * s["dout"].double()).sum() + (o * inv64(o) * p["next_gain"] * s["dnext"].double()).sum()

    gen = torch.Generator(device="cuda").manual_seed(9)
    base = {n: s[n].double() for n in got}
    for name, grad in got.items():
        d = torch.randn(grad.shape, generator=gen, device="cuda", dtype=torch.float64)
        eps = 1e-5
        slope = (loss({**base, name: base[name] + eps * d}) - loss({**base, name: base[name] - eps * d})) / (2 * eps)
        # roundings of fp32 on the way, eps^2 of the third derivative
        assert abs(float(slope - (grad.double() * d).sum())) <= 4 * SUM * float((grad.double() * d).abs().sum()) + 1e-6, name


def test_rows_of_zeros_and_not_a_number():
    f = fusco()
    r, y, gain = torch.zeros((3, 64), device="cuda"), torch.zeros((3, 64), device="cuda"), torch.ones(64, device="cuda")
    y[1, 5] = float("nan")
    y[2] = 3.0
    out, nxt = torch.empty_like(r), torch.empty_like(r)
    f.fusco_norm_after(r, y, gain, out, next_gain=gain, next_out=nxt, eps=EPS)
    assert bool((out[0] == 0).all()) and bool((nxt[0] == 0).all())
    assert bool(out[1].isnan().all()) and bool(out[2].isfinite().all())         # a row's NaN stays in its row


def test_gradients_are_the_same_every_time():
    f = fusco()
    s = inputs(3000, 1024, torch.float32, torch.bfloat16, "channel", seed=4)
    seen = []
    for _ in range(3):
        res = [torch.empty_like(s["r"]), torch.empty_like(s["y"])] + [torch.empty(1024, device="cuda") for _ in range(3)]
        f.fusco_norm_after_backward(s["dout"], s["y"], s["gain"], res[0], res[1], res[2], gate=s["gate"], dgate=res[3], dnext=s["dnext"], out=s["r"], next_gain=s["next_gain"],
                                    dnext_gain=res[4], eps=EPS)
        seen.append(res)
    assert all(torch.equal(a, b) for other in seen[1:] for a, b in zip(seen[0], other))


def test_empty_batch():
    f = fusco()
    x, gain = torch.empty((0, 64), device="cuda"), torch.ones(64, device="cuda")
    f.fusco_norm_before(x, gain, x)
    f.fusco_norm_after(x, x, gain, x, next_gain=gain, next_out=x)
    dg, dn = torch.full((64,), 7.0, device="cuda"), torch.full((64,), 7.0, device="cuda")
    f.fusco_norm_after_backward(x, x, gain, x, x, dg, dnext=x, out=x, next_gain=gain, dnext_gain=dn)
    assert bool((dg == 0).all()) and bool((dn == 0).all())
    dg.fill_(7.0)
    f.fusco_norm_before_backward(x, x, gain, x, dg)
    assert bool((dg == 0).all())


def test_refusals():
    f = fusco()
    x, gain = torch.zeros((4, 64), device="cuda"), torch.ones(64, device="cuda")
    out = torch.empty_like(x)
    bad = [dict(x=x[:, :60].contiguous()), dict(gain=gain[:32]), dict(gain=gain.double()), dict(out=out.half()), dict(out=out[:3]), dict(x=x.cpu()), dict(x=x.t().contiguous().t()), dict(eps=0.0),
           dict(eps=float("nan")), dict(x=x.bfloat16())]
    for b in bad:
        with pytest.raises(f.FuscoError):
            f.fusco_norm_before(**{**dict(x=x, gain=gain, out=out), **b})
    wide = torch.zeros((1, 32776), device="cuda")
    with pytest.raises(f.FuscoError):
        f.fusco_norm_before(wide, wide[0].contiguous(), torch.empty_like(wide))
    with pytest.raises(f.FuscoError):
        f.fusco_norm_after(x, x, gain, out, next_gain=gain)
    with pytest.raises(f.FuscoError):
        f.fusco_norm_after(x, x, gain, out, gate=torch.ones(5, device="cuda"))
    square = torch.zeros((64, 64), device="cuda")
    with pytest.raises(f.FuscoError):       # which of both a gate of 64 means has to be said
        f.fusco_norm_after(square, square, gain, torch.empty_like(square), gate=gain)
    with pytest.raises(f.FuscoError):
        f.fusco_norm_after_backward(x, x, gain, out, out.clone(), gain.clone(), scratch=torch.empty(16, dtype=torch.uint8, device="cuda"))
    with pytest.raises(f.FuscoError):
        f.fusco_norm_after_backward(None, x, gain, out, out.clone(), gain.clone())
