"""The whole layer for a few tokens against the formulas in 64 bits.

Tolerance.  fp32 sums of n exact products are at most n * 2^-23 * sum |terms| off (test_gpu_experts); with weights of e4m3 two more units for the scales.  h = silu(g) u
carries the errors of g and u by its derivatives and (12 + |g|) units of its own, and is kept as three numbers of bf16: 2^-24 of it is left.
The second product and the tokens' weights, k of them, add their own sums; a result of bf16 is rounded by up to 2^-8 of itself, one of fp32 by 2^-24.

An inner product's smallest rest may be below the normal numbers of bf16, 2^-126: TINY covers it."""
import pytest
import torch

from test_gpu_experts import BF16, TINY, U23, bf16, fusco
from test_gpu_fp8 import FP8, blocks, eight, over_both

pytestmark = pytest.mark.gpu


def layer(gen, E, H, I, eights):
    if not eights:
        w_in, w_out = bf16(gen, E, 2 * I, H, std=1.5 * H ** -0.5), bf16(gen, E, H, I, std=I ** -0.5)
        return dict(w_in=w_in, w_out=w_out), w_in.double(), w_out.double()
    w_in, in_scale = eight(gen, E, 2 * I, H, scales=(E, 2 * blocks(I), blocks(H)), std=1.5 * H ** -0.5)
    w_out, out_scale = eight(gen, E, H, I, scales=(E, blocks(H), blocks(I)), std=I ** -0.5)
    w_in, w_out = (torch.where(w.float().isnan(), torch.zeros((), device="cuda"), w.float()).to(FP8) for w in (w_in, w_out))
    wide_in = (w_in.double().view(2 * E, I, H) * over_both(in_scale.double().view(2 * E, blocks(I), blocks(H)), I, H)).view(E, 2 * I, H)
    return dict(w_in=w_in, w_out=w_out, w_in_scale=in_scale, w_out_scale=out_scale), wide_in, w_out.double() * over_both(out_scale.double(), H, I)


def routing(gen, N, E, k, kind):
    chosen = torch.rand((N, E), generator=gen, device="cuda").argsort(dim=1)[:, :k] if k <= E else torch.randint(0, E, (N, k), generator=gen, device="cuda")
    if kind == "one":         # all tokens have the same experts
        chosen = chosen[:1].repeat(N, 1)
    if kind == "equal":       # a token names an expert more than once
        chosen = torch.randint(0, max(1, E // 4), (N, k), generator=gen, device="cuda")
    if kind == "invalid":     # pairs that name none; a token without any
        chosen = torch.where(torch.rand((N, k), generator=gen, device="cuda") < 0.4, torch.randint(-3, 0, (N, k), generator=gen, device="cuda"), chosen)
        chosen[:, 0] = E + 5
        chosen[N // 2] = -1
    return chosen.to(torch.int32).contiguous(), torch.rand((N, k), generator=gen, device="cuda") + 0.1


def definition(x, chosen, w, wide_in, wide_out, scaled):
    """The result in 64 bits and what the fp32 sums may be off."""
    N, H = x.shape
    E, I = wide_in.shape[0], wide_in.shape[1] // 2
    out, off = torch.zeros((N, H), dtype=torch.float64, device="cuda"), torch.zeros((N, H), dtype=torch.float64, device="cuda")
    size = torch.zeros((N, H), dtype=torch.float64, device="cuda")
    more = 3 if scaled else 0
    for e in range(E):
        t, j = (chosen == e).nonzero(as_tuple=True)
        if not len(t):
            continue
        v, wt = x[t].double(), w[t, j].double()[:, None]
        (g, u), (dg, du) = (v @ wide_in[e].t()).split(I, dim=1), ((H + more) * U23 * (v.abs() @ wide_in[e].abs().t())).split(I, dim=1)
        s = g * torch.sigmoid(g)
        h = s * u
        dh = 1.1 * dg * (u.abs() + du) + s.abs() * du + (12 + g.abs()) * U23 * h.abs()
        dh = dh + BF16 ** 3 * (h.abs() + dh) + 2.0 ** -130
        terms = (h.abs() + dh) @ wide_out[e].abs().t()
        out.index_add_(0, t, wt * (h @ wide_out[e].t()))
        off.index_add_(0, t, wt * (dh @ wide_out[e].abs().t() + 3 * (I + more) * U23 * terms))   # three parts of h are added up
        size.index_add_(0, t, wt * terms)
    return out, off + (chosen.shape[1] + 24) * U23 * size   # the tokens' weights, the waves' parts


def within(got, want, off, dtype):
    rounding = BF16 if dtype == torch.bfloat16 else U23
    far = (got.double() - want).abs() - (off + rounding * (want.abs() + off) + TINY)
    assert bool((far <= 0).all()), "off by %g more than the bound" % float(far.max())


SIZES = [(1, 1, 1, 16, 16), (1, 8, 2, 64, 48), (1, 16, 8, 512, 256), (2, 5, 3, 144, 32), (3, 4, 4, 272, 400), (5, 60, 6, 1040, 528), (8, 3, 2, 208, 1040), (15, 128, 8, 256, 128), (16, 32, 4, 640, 272),
         (17, 8, 2, 384, 208), (31, 64, 6, 528, 144), (32, 2, 1, 128, 128), (33, 16, 4, 272, 336), (64, 128, 8, 256, 192), (64, 3, 3, 400, 272), (64, 1024, 1, 64, 32), (7, 2, 8, 128, 64),
         (2, 1024, 64, 48, 16), (64, 80, 64, 32, 16), (64, 128, 8, 144, 288), (20, 128, 8, 80, 304), (64, 32, 4, 2064, 48)]


@pytest.mark.parametrize("out_dtype", [torch.bfloat16, torch.float32])
@pytest.mark.parametrize("eights", [False, True])
@pytest.mark.parametrize("kind", ["any", "one", "equal", "invalid"])
@pytest.mark.parametrize("N,E,k,H,I", SIZES)
def test_layer(N, E, k, H, I, kind, eights, out_dtype):
    f = fusco()
    gen = torch.Generator(device="cuda").manual_seed(31)
    weights, wide_in, wide_out = layer(gen, E, H, I, eights)
    x = bf16(gen, N, H)
    chosen, w = routing(gen, N, E, k, kind)
    out = torch.full((N, H), 7.0, dtype=out_dtype, device="cuda")
    f.fusco_moe_few(x, chosen, w, out=out, **weights)
    want, off = definition(x, chosen, w, wide_in, wide_out, eights)
    within(out, want, off, out_dtype)
    if kind == "invalid":
        assert bool((out[N // 2] == 0).all())


@pytest.mark.parametrize("H,I", [(8, 8), (24, 40), (200, 72)])
def test_rows_of_eights(H, I):
    """Weights of bf16 may have rows of any multiple of 8."""
    f = fusco()
    gen = torch.Generator(device="cuda").manual_seed(32)
    weights, wide_in, wide_out = layer(gen, 6, H, I, False)
    x = bf16(gen, 9, H)
    chosen, w = routing(gen, 9, 6, 3, "any")
    out = torch.empty((9, H), device="cuda")
    f.fusco_moe_few(x, chosen, w, out=out, **weights)
    want, off = definition(x, chosen, w, wide_in, wide_out, False)
    within(out, want, off, torch.float32)


@pytest.mark.parametrize("N", [4, 40])
@pytest.mark.parametrize("eights", [False, True])
def test_an_experts_values_stay_its_own(eights, N):
    """NaN and infinities in an expert's weights or a token's row reach the tokens that chose it, or that token, and no others."""
    f = fusco()
    E, k, H, I = 8, 2, 144, 80
    gen = torch.Generator(device="cuda").manual_seed(33)
    weights, _, _ = layer(gen, E, H, I, eights)
    x = bf16(gen, N, H)
    chosen, w = routing(gen, N, E, k, "any")
    chosen[0] = torch.tensor([1, 2], dtype=torch.int32)
    chosen[1] = torch.tensor([3, 4], dtype=torch.int32)
    chosen[2] = torch.tensor([1, 4], dtype=torch.int32)
    if eights:
        weights["w_in"].view(torch.uint8)[2] = 0x7f
        weights["w_out_scale"][3] = float("inf")
    else:
        weights["w_in"][2] = float("nan")
        weights["w_out"][3] = float("inf")
    x[3] = float("inf")
    out = torch.empty((N, H), device="cuda")
    f.fusco_moe_few(x, chosen, w, out=out, **weights)
    sick = ((chosen == 2) | (chosen == 3)).any(dim=1)
    sick[3] = True
    assert bool(out[~sick].isfinite().all()) and not bool(out[sick].isfinite().any())


@pytest.mark.parametrize("N,k", [(2, 1), (40, 4)])
def test_largest_activations(N, k):
    """silu(g) u at the ends of fp32: infinities stay what they are, and what is finite in fp32 but would round to an infinity of bf16 stays finite."""
    f = fusco()
    E, H, I = 4, 64, 32
    x, w_in, w_out = torch.zeros((N, H)), torch.zeros((E, 2 * I, H)), torch.zeros((E, H, I))
    x[:, :3] = 1.0
    # unit 0: g = 2^64, u = 2^64 - 2^55, and 2^128 (1 - 2^-9) is the middle between bf16's largest number and the next power
    w_in[:, 0, 0], w_in[:, I, 0], w_in[:, I, 1] = 2.0 ** 64, 2.0 ** 64, -2.0 ** 55
    w_out[:, 0, 0] = 2.0 ** -120
    chosen = torch.arange(N * k).remainder(E).int().view(N, k)
    w = torch.full((N, k), 1.0 / k)
    out = torch.empty((N, H), device="cuda")

    def run():
        f.fusco_moe_few(x.bfloat16().cuda(), chosen.cuda(), w.cuda(), w_in.bfloat16().cuda(), w_out.bfloat16().cuda(), out)

    run()
    assert bool((out[:, 0] == 255.5).all()) and not bool(out[:, 1:].any())
    w_in[:, 1, 0], w_in[:, I + 1, 0] = 2.0 ** 100, 2.0 ** 100
    w_out[:] = 1.0
    run()
    assert bool((out == float("inf")).all())
    w_in[:, 1, 1] = float("nan")
    run()
    assert bool(out.isnan().all())


def test_as_the_calls_one_by_one():
    """The same layer by plan and dispatch, products and combine: both are within their roundings of the same number."""
    f = fusco()
    N, E, k, H, I = 12, 32, 4, 512, 256
    gen = torch.Generator(device="cuda").manual_seed(34)
    weights, wide_in, wide_out = layer(gen, E, H, I, False)
    x = bf16(gen, N, H)
    logits = torch.randn((N, E), generator=gen, device="cuda")
    chosen, w = torch.empty((N, k), dtype=torch.int32, device="cuda"), torch.empty((N, k), device="cuda")
    f.fusco_route(logits, chosen, w, score=f.SCORE_SIGMOID)
    got = torch.empty((N, H), dtype=torch.bfloat16, device="cuda")
    f.fusco_moe_few(x, chosen, w, out=got, **weights)
    L = f.Layout(N, k, E, 1)
    rows, h, y, want = (torch.empty(s, dtype=torch.bfloat16, device="cuda") for s in ((L.P, H), (L.P, I), (L.P, H), (N, H)))
    f.fusco_plan_dispatch(L, chosen, x, rows)
    f.fusco_experts_gated(L, rows, weights["w_in"], h)
    f.fusco_experts_linear(L, h, weights["w_out"], y)
    f.fusco_combine(L, y, w, want)
    exact, off = definition(x, chosen, w, wide_in, wide_out, False)
    within(got, exact, off, torch.bfloat16)
    # the other way rounds h and y to bf16: 2^-8 of every |h w_out| and |y| on top
    extra = torch.zeros_like(exact)
    for e in range(E):
        t, j = (chosen == e).nonzero(as_tuple=True)
        g, u = (x[t].double() @ wide_in[e].t()).split(I, dim=1)
        h64 = g * torch.sigmoid(g) * u
        extra.index_add_(0, t, w[t, j].double()[:, None] * 1.01 * BF16 * (h64.abs() @ wide_out[e].abs().t() + (h64 @ wide_out[e].t()).abs()))
    within(want, exact, off + extra, torch.bfloat16)


@pytest.mark.parametrize("eights", [False, True])
def test_repeats_bit_by_bit_captured_and_on_another_stream(eights):
    f = fusco()
    N, E, k, H, I = 20, 16, 4, 272, 144
    gen = torch.Generator(device="cuda").manual_seed(35)
    weights, _, _ = layer(gen, E, H, I, eights)
    x = bf16(gen, N, H)
    chosen, w = routing(gen, N, E, k, "any")
    scratch = torch.empty(f.fusco_moe_few_scratch_bytes(N, k, I), dtype=torch.uint8, device="cuda")
    out = torch.empty((N, H), device="cuda")
    run = lambda o, **kw: f.fusco_moe_few(x, chosen, w, out=o, **weights, **kw)
    run(out, scratch=scratch)
    torch.cuda.synchronize()
    side, other = torch.cuda.Stream(), torch.empty_like(out)
    side.wait_stream(torch.cuda.current_stream())
    run(other, stream=side)      # with scratch memory of its own
    torch.cuda.current_stream().wait_stream(side)
    assert torch.equal(other, out)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        run(out, scratch=scratch)
    for _ in range(3):
        x.copy_(torch.randn((N, H), generator=gen, device="cuda"))
        chosen.copy_(routing(gen, N, E, k, "any")[0])
        run(other)
        out.zero_()
        scratch.fill_(0xa5)
        graph.replay()
        torch.cuda.synchronize()
        assert torch.equal(out, other)


def test_refusals():
    f = fusco()
    gen = torch.Generator(device="cuda").manual_seed(36)
    N, E, k, H, I = 4, 6, 2, 64, 32
    weights, _, _ = layer(gen, E, H, I, False)
    eights, _, _ = layer(gen, E, H, I, True)
    chosen, w = routing(gen, N, E, k, "any")
    good = dict(x=bf16(gen, N, H), topk_idx=chosen, w=w, out=torch.empty((N, H), device="cuda"), **weights)
    f.fusco_moe_few(**good)
    for bad in (dict(x=good["x"].float()), dict(x=good["x"][:3]), dict(topk_idx=chosen.long()), dict(w=w.half()), dict(w=w[:, :1].contiguous()), dict(out=torch.empty((N, H), dtype=torch.float16, device="cuda")),
                dict(out=torch.empty((N, 32), device="cuda")), dict(w_in=weights["w_in"][:5].contiguous()), dict(w_out=weights["w_out"].transpose(1, 2)), dict(w_in=eights["w_in"]),
                dict(w_in_scale=eights["w_in_scale"]), dict(w_in_scale=eights["w_in_scale"], w_out_scale=eights["w_out_scale"]), dict(x=good["x"].cpu()),
                dict(scratch=torch.empty(16, dtype=torch.uint8, device="cuda")), dict(w_in=weights["w_in"][:, :63].contiguous())):
        with pytest.raises(f.FuscoError):
            f.fusco_moe_few(**dict(good, **bad))
    good = dict(good, **eights)
    f.fusco_moe_few(**good)
    for bad in (dict(w_out_scale=None), dict(w_in_scale=eights["w_in_scale"][:, :1].contiguous()), dict(w_out=weights["w_out"])):
        with pytest.raises(f.FuscoError):
            f.fusco_moe_few(**dict(good, **bad))
    many = 65
    chosen, w = routing(gen, many, E, k, "any")
    with pytest.raises(f.FuscoError):
        f.fusco_moe_few(x=bf16(gen, many, H), topk_idx=chosen, w=w, out=torch.empty((many, H), device="cuda"), **weights, scratch=torch.empty(1 << 20, dtype=torch.uint8, device="cuda"))
    f.fusco_moe_few(x=bf16(gen, 0, H), topk_idx=chosen[:0], w=w[:0], out=torch.empty((0, H), device="cuda"), **weights)


@pytest.mark.parametrize("N,E,k,H,I", [(1, 2, 1, 256, 16), (3, 12, 2, 144, 80), (40, 4, 2, 272, 48), (64, 128, 8, 400, 272)])   # every instance of the first product
def test_infinite_scales(N, E, k, H, I):
    """An infinite scale of one block of w_in: what is multiplied there is positive, and so are infinite the results of the tokens that chose the expert, and finite all others.  Waves
    have pieces past their last one here."""
    f = fusco()
    gen = torch.Generator(device="cuda").manual_seed(37)
    ones = lambda *s: torch.ones(s, device="cuda")
    w_in_scale = ones(E, 2 * blocks(I), blocks(H))
    chosen, w = routing(gen, N, E, k, "any")
    chosen[0, 0] = 1
    chosen[0, 1:] = 0
    w_in_scale[1, 0, 0] = float("inf")
    out = torch.empty((N, H), device="cuda")
    f.fusco_moe_few(ones(N, H).bfloat16(), chosen, w, ones(E, 2 * I, H).to(FP8), ones(E, H, I).to(FP8), out, w_in_scale=w_in_scale, w_out_scale=ones(E, blocks(H), blocks(I)))
    sick = (chosen == 1).any(dim=1)
    assert bool((out[sick] == float("inf")).all()) and bool(out[~sick].isfinite().all())


@pytest.mark.parametrize("eights", [False, True])
@pytest.mark.parametrize("kind", ["any", "one", "invalid"])
@pytest.mark.parametrize("N,E,k,H,I", [(1, 16, 8, 4096, 144), (5, 12, 4, 4112, 80), (20, 24, 4, 7168, 48), (64, 8, 2, 4096, 272), (47, 64, 8, 5120, 48)])
def test_long_rows(N, E, k, H, I, kind, eights):
    """As many blocks of outputs as there are compute units and more: the list of groups is whole, a workgroup's waves alone share it."""
    test_layer(N, E, k, H, I, kind, eights, torch.float32)
