"""Gradients of the experts' products from activations that were kept in e4m3, against the formulas in 64 bits.  Tolerances as in test_gpu_experts: kept values with
scales that are powers of two are numbers of bf16, so nothing is rounded on the way; any other scale rounds x * scale to bf16 (2^-8 of it, carried through the
product) in the weight gradient and to fp32 in the input gradient."""
import pytest
import torch

from test_gpu_experts import BF16, CASES, TINY, U23, bf16, fusco, make, product, segments, within
from test_gpu_fp8 import FP8, blocks, eight, over_columns, sixteens

pytestmark = pytest.mark.gpu

CASES16 = [(N, k, E, sixteens(C), M, routing) for N, k, E, C, M, routing in CASES] + [(700, 3, 4, 1040, 264, "skewed"), (40, 1, 1, 16, 8, "normal")]


def kept(gen, rows, columns, any_scale, std=1.0):
    """Values as the forward pass keeps them: through fusco_to_fp8, or with scales of any size."""
    if any_scale:
        return eight(gen, rows, columns, scales=(rows, blocks(columns)), std=std)
    x, q = bf16(gen, rows, columns, std=std), torch.empty((rows, columns), dtype=FP8, device="cuda")
    scale = torch.zeros((rows, blocks(columns) + 2), device="cuda")
    fusco().fusco_to_fp8(x, q, scale)
    return q, scale


def value(q, scale):
    return q.double() * over_columns(scale.double(), q.shape[1])


@pytest.mark.parametrize("any_scale", [False, True])
@pytest.mark.parametrize("N,k,E,I,M,routing", CASES16)
def test_input_grad(N, k, E, I, M, routing, any_scale):
    f = fusco()
    L, gen, bounds = make(N, k, E, 21, routing)
    dy, w = bf16(gen, L.P, M), bf16(gen, E, M, I, std=M ** -0.5)
    pre, scale = kept(gen, L.P, 2 * I, any_scale, 2.0)
    scale[bounds[-1]:] = float("nan")
    dpre = torch.full((L.P, 2 * I), 7.0, dtype=torch.bfloat16, device="cuda")
    f.fusco_experts_input_grad(L, dy, w, dpre, pre=pre, pre_scale=scale)
    for e, rows in segments(bounds, dy):
        dh, err = product(dy[rows], w[e].t())
        g, u = value(pre[rows], scale[rows]).split(I, dim=1)
        sig = torch.sigmoid(g)
        slope = torch.cat([u * sig * (1 + g * (1 - sig)), g * sig], dim=1)
        # as for bf16; a scale that is no power of two rounds g and u: one more unit of fp32 each, of a slope that changes by at most |g| + 4 times as much
        own = torch.cat([u * sig, g * sig], dim=1).abs() * (1 + g.abs()).repeat(1, 2) * (20 + 2 * g.abs()).repeat(1, 2) * U23
        dh, err = dh.repeat(1, 2), err.repeat(1, 2)
        carried = err * (slope.abs() + own) + dh.abs() * own
        within(dpre[rows], dh * slope, carried + BF16 * ((dh * slope).abs() + carried) + TINY)
    assert bool((dpre[bounds[-1]:] == 7.0).all())


@pytest.mark.parametrize("any_scale", [False, True])
@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
@pytest.mark.parametrize("N,k,E,C,M,routing", CASES16)
def test_weight_grad(N, k, E, C, M, routing, dtype, any_scale):
    f = fusco()
    L, gen, bounds = make(N, k, E, 22, routing)
    dy = bf16(gen, L.P, M)
    x, scale = kept(gen, L.P, C, any_scale)
    dy[bounds[-1]:] = float("nan")
    scale[bounds[-1]:] = float("nan")
    dw = torch.full((E, M, C), 7.0, dtype=dtype, device="cuda")
    f.fusco_experts_weight_grad(L, dy, x, dw, x_scale=scale)
    rounding = BF16 if dtype == torch.bfloat16 else U23
    for e, rows in segments(bounds, dy):
        v = value(x[rows], scale[rows])
        want, err = product(dy[rows].t(), v.t())
        if any_scale:
            err = (1 + BF16) * err + BF16 * (dy[rows].double().abs().t() @ v.abs())
        within(dw[e], want, err + rounding * (want.abs() + err) + TINY)   # zeros for an expert without rows


@pytest.mark.parametrize("I", [48, 128, 192])
def test_same_as_from_bf16(I):
    """Kept values are numbers of bf16: the gradients from them are those from bf16 tensors that hold them, bit by bit."""
    f = fusco()
    L, gen, bounds = make(400, 2, 5, 23, "skewed")
    M = 144
    dy, w = bf16(gen, L.P, M), bf16(gen, 5, M, I, std=M ** -0.5)
    pre, pre_scale = kept(gen, L.P, 2 * I, False, 2.0)
    x, x_scale = kept(gen, L.P, I, False)
    wide_pre, wide_x = torch.empty((L.P, 2 * I), dtype=torch.bfloat16, device="cuda"), torch.empty((L.P, I), dtype=torch.bfloat16, device="cuda")
    f.fusco_from_fp8(pre, pre_scale, wide_pre)
    f.fusco_from_fp8(x, x_scale, wide_x)
    got, want = torch.empty_like(wide_pre), torch.empty_like(wide_pre)
    f.fusco_experts_input_grad(L, dy, w, got, pre=pre, pre_scale=pre_scale)
    f.fusco_experts_input_grad(L, dy, w, want, pre=wide_pre)
    assert torch.equal(got, want)
    for dtype in (torch.bfloat16, torch.float32):
        got, want = torch.empty((5, M, I), dtype=dtype, device="cuda"), torch.empty((5, M, I), dtype=dtype, device="cuda")
        f.fusco_experts_weight_grad(L, dy, x, got, x_scale=x_scale)
        f.fusco_experts_weight_grad(L, dy, wide_x, want)
        assert torch.equal(got, want)


def test_an_experts_values_stay_its_own():
    """NaN in one expert's kept rows or their scales reach no other expert's gradients."""
    f = fusco()
    L, gen, bounds = make(300, 2, 4, 24, "normal")
    C, M = 208, 136
    dy = bf16(gen, L.P, M)
    x, scale = kept(gen, L.P, C, False)
    rows = slice(bounds[1], bounds[2])
    x.view(torch.uint8)[rows] = 0x7f
    scale[bounds[3]] = float("inf")
    dw = torch.empty((4, M, C), dtype=torch.bfloat16, device="cuda")
    f.fusco_experts_weight_grad(L, dy, x, dw, x_scale=scale)
    assert bool(dw[[0, 2]].isfinite().all()) and not bool(dw[1].isfinite().any()) and not bool(dw[3].isfinite().all())


def test_gradient_by_differences():
    """The gradient of sum(y * dy) along a direction of the kept pre-activations, by central differences in 64 bits of the formulas."""
    f = fusco()
    L, gen, bounds = make(90, 2, 3, 25, "normal")
    I, M = 48, 56
    w, dy = bf16(gen, 3, M, I, std=I ** -0.5), bf16(gen, L.P, M)
    pre, scale = kept(gen, L.P, 2 * I, False)
    dpre = torch.empty((L.P, 2 * I), dtype=torch.bfloat16, device="cuda")
    f.fusco_experts_input_grad(L, dy, w, dpre, pre=pre, pre_scale=scale)
    at = value(pre, scale)
    direction = torch.randn(at.shape, generator=gen, device="cuda", dtype=torch.float64)

    def loss(p):
        g, u = p.split(I, dim=1)
        h = g * torch.sigmoid(g) * u
        return sum(((h[r] @ w[e].double().t()) * dy[r].double()).sum() for e, r in segments(bounds, p))

    eps = 1e-4
    slope = (loss(at + eps * direction) - loss(at - eps * direction)) / (2 * eps)
    terms = dpre.double() * direction
    # every entry of dpre carries a rounding of up to 2^-8 of itself, at random: six standard deviations of their sum are below
    assert abs(float(slope - terms.sum())) <= 6 * 2.0 ** -8 * float(terms.norm()) + 1e-4 * abs(float(slope))


def test_empty_batch():
    f = fusco()
    L = f.Layout(0, 2, 4, 1)
    f.fusco_plan(L, torch.empty((0, 2), dtype=torch.int32, device="cuda"))
    none = lambda c, t: torch.empty((0, c), dtype=t, device="cuda")
    f.fusco_experts_input_grad(L, none(64, torch.bfloat16), torch.ones((4, 64, 32), dtype=torch.bfloat16, device="cuda"), none(64, torch.bfloat16), pre=none(64, FP8),
                               pre_scale=none(1, torch.float32))
    dw = torch.ones((4, 32, 64), device="cuda")
    f.fusco_experts_weight_grad(L, none(32, torch.bfloat16), none(64, FP8), dw, x_scale=none(1, torch.float32))
    assert bool((dw == 0).all())


def test_refusals():
    f = fusco()
    L, gen, _ = make(16, 2, 4, 26, "normal")
    dy, w, dpre = bf16(gen, L.P, 64), bf16(gen, 4, 64, 32), bf16(gen, L.P, 64)
    pre, scale = kept(gen, L.P, 64, True)
    good = dict(dy=dy, w=w, dx=dpre, pre=pre, pre_scale=scale)
    for bad in (dict(pre=dpre), dict(pre=None), dict(pre_scale=None), dict(pre_scale=scale[:-1]), dict(pre_scale=scale.double()), dict(pre=pre[:, :32].contiguous()), dict(dx=bf16(gen, L.P, 32)),
                dict(dy=dy.float()), dict(pre=pre.cpu())):
        with pytest.raises(f.FuscoError):
            f.fusco_experts_input_grad(L, **dict(good, **bad))
    x, scale = kept(gen, L.P, 64, True)
    good = dict(dy=dy, x=x, dw=torch.empty((4, 64, 64), device="cuda"), x_scale=scale)
    for bad in (dict(x=dy), dict(x_scale=None), dict(x_scale=scale[:4]), dict(x_scale=scale.half()), dict(dw=torch.empty((4, 64, 64), dtype=torch.float16, device="cuda")),
                dict(dw=torch.empty((4, 64, 48), device="cuda"))):
        with pytest.raises(f.FuscoError):
            f.fusco_experts_weight_grad(L, **dict(good, **bad))
    with pytest.raises(f.FuscoError):   # rows of 8 elements
        f.fusco_experts_weight_grad(L, dy, torch.zeros((L.P, 8), device="cuda").to(FP8), torch.empty((4, 64, 8), device="cuda"), x_scale=scale)
