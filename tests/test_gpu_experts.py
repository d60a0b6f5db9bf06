"""The experts' products and their gradients against the formulas in 64 bits.

Tolerance.  A sum of n products of bf16 factors (exact in fp32) that is held in fp32 is at most n * 2^-23 * sum |terms| from
the exact one (n additions of half a unit in the last place each, doubled for the unspecified order inside a matrix
instruction); rounding to bf16 (8 significant bits) adds up to 2^-8 of the result, to fp32 2^-24.  Factors that are functions of such sums carry the
sums' errors along by their derivatives, which the tests write out, and a few units of fp32 of their own."""
import pytest
import torch

pytestmark = pytest.mark.gpu

U23, BF16 = 2.0 ** -23, 2.0 ** -8
TINY = 1e-30


def fusco():
    import paper_2512_22036_amd as f
    f.load_library()
    return f


def make(N, k, E, seed, routing):
    """A planned layout, the routing and the bounds of the experts' segments."""
    gen = torch.Generator(device="cuda").manual_seed(seed)
    if routing == "one":         # everything goes to the last experts: most of them have no rows
        chosen = (E - 1 - torch.arange(k, device="cuda")).repeat(N, 1)
    else:
        score = torch.randn((N, E), generator=gen, device="cuda")
        if routing == "skewed":
            score += 2.0 * torch.randn((E,), generator=gen, device="cuda")
        chosen = score.topk(k, dim=1).indices
    if routing == "invalid":     # some pairs name no expert: rows at the end of the tensor belong to nobody
        chosen[torch.rand((N, k), generator=gen, device="cuda") < 0.2] = E + 3
    f = fusco()
    L = f.Layout(N, k, E, 1)
    f.fusco_plan(L, chosen.to(torch.int32).contiguous())
    return L, gen, L.array("exp_off").tolist()


def bf16(gen, *shape, std=1.0):
    return torch.randn(shape, generator=gen, device="cuda").mul_(std).bfloat16()


def segments(bounds, t):
    for e in range(len(bounds) - 1):
        yield e, slice(bounds[e], bounds[e + 1])


def product(x, w):
    """x w^T in 64 bits and the bound of its fp32 sum."""
    x, w = x.double(), w.double()
    return x @ w.t(), x.shape[1] * U23 * (x.abs() @ w.abs().t())


def within(got, want, bound):
    off = (got.double() - want).abs() - bound
    assert bool((off <= 0).all()), "off by %g more than the bound" % float(off.max())


# rows per expert from none to several tiles; row sizes from one chunk to whole tiles and a chunk more
CASES = [
    (1, 1, 1, 8, 8, "normal"), (1, 8, 16, 64, 128, "normal"), (3, 2, 5, 72, 24, "normal"), (37, 2, 4, 136, 264, "normal"),
    (64, 4, 4, 256, 128, "normal"), (65, 2, 2, 520, 136, "normal"), (130, 1, 1, 128, 256, "normal"), (257, 1, 1, 200, 520, "normal"),
    (300, 6, 12, 320, 192, "skewed"), (129, 4, 160, 264, 72, "normal"), (500, 2, 3, 1032, 392, "skewed"), (100, 2, 1024, 64, 64, "normal"),
    (700, 2, 8, 512, 640, "skewed"), (513, 2, 6, 256, 256, "one"), (200, 3, 7, 192, 248, "invalid"), (1000, 4, 5, 456, 1288, "invalid"),
]


@pytest.mark.parametrize("N,k,E,C,M,routing", CASES)
def test_linear(N, k, E, C, M, routing):
    f = fusco()
    L, gen, bounds = make(N, k, E, 1, routing)
    x, w = bf16(gen, L.P, C), bf16(gen, E, M, C, std=C ** -0.5)
    x[bounds[-1]:] = float("nan")
    y = torch.full((L.P, M), 7.0, dtype=torch.bfloat16, device="cuda")
    f.fusco_experts_linear(L, x, w, y)
    for e, rows in segments(bounds, x):
        want, err = product(x[rows], w[e])
        within(y[rows], want, err + BF16 * (want.abs() + err) + TINY)
    assert bool((y[bounds[-1]:] == 7.0).all())     # rows of nobody stay as they were


@pytest.mark.parametrize("keep_pre", [False, True])
@pytest.mark.parametrize("N,k,E,H,I,routing", CASES)
def test_gated(N, k, E, H, I, routing, keep_pre):
    f = fusco()
    L, gen, bounds = make(N, k, E, 2, routing)
    x, w = bf16(gen, L.P, H), bf16(gen, E, 2 * I, H, std=2.0 * H ** -0.5)
    x[bounds[-1]:] = float("nan")
    h = torch.full((L.P, I), 7.0, dtype=torch.bfloat16, device="cuda")
    pre = torch.full((L.P, 2 * I), 7.0, dtype=torch.bfloat16, device="cuda") if keep_pre else None
    f.fusco_experts_gated(L, x, w, h, pre)
    for e, rows in segments(bounds, x):
        both, err = product(x[rows], w[e])
        (g, u), (dg, du) = both.split(I, dim=1), err.split(I, dim=1)
        s = g * torch.sigmoid(g)
        # |silu'| < 1.1; the exponential of g costs |g| + 4 units, the division and the product 4 more
        carried = 1.1 * dg * (u.abs() + du) + s.abs() * du + (12 + g.abs()) * U23 * (s * u).abs()
        within(h[rows], s * u, carried + BF16 * ((s * u).abs() + carried) + TINY)
        if keep_pre:
            within(pre[rows], both, err + BF16 * (both.abs() + err) + TINY)
    for t in (h, pre):
        assert t is None or bool((t[bounds[-1]:] == 7.0).all())


@pytest.mark.parametrize("N,k,E,C,M,routing", CASES)
def test_input_grad(N, k, E, C, M, routing):
    f = fusco()
    L, gen, bounds = make(N, k, E, 3, routing)
    dy, w = bf16(gen, L.P, M), bf16(gen, E, M, C, std=M ** -0.5)
    dy[bounds[-1]:] = float("nan")
    dx = torch.full((L.P, C), 7.0, dtype=torch.bfloat16, device="cuda")
    f.fusco_experts_input_grad(L, dy, w, dx)
    for e, rows in segments(bounds, dy):
        want, err = product(dy[rows], w[e].t())
        within(dx[rows], want, err + BF16 * (want.abs() + err) + TINY)
    assert bool((dx[bounds[-1]:] == 7.0).all())


@pytest.mark.parametrize("N,k,E,I,M,routing", CASES)
def test_input_grad_through_the_activation(N, k, E, I, M, routing):
    f = fusco()
    L, gen, bounds = make(N, k, E, 4, routing)
    dy, w, pre = bf16(gen, L.P, M), bf16(gen, E, M, I, std=M ** -0.5), bf16(gen, L.P, 2 * I, std=2.0)
    dpre = torch.full((L.P, 2 * I), 7.0, dtype=torch.bfloat16, device="cuda")
    f.fusco_experts_input_grad(L, dy, w, dpre, pre=pre)
    for e, rows in segments(bounds, dy):
        dh, err = product(dy[rows], w[e].t())
        g, u = pre[rows].double().split(I, dim=1)
        sig = torch.sigmoid(g)
        slope = torch.cat([u * sig * (1 + g * (1 - sig)), g * sig], dim=1)
        # 1 + g (1 - sig) cancels near its zero: its own error is a few units of 1 + |g|
        own = torch.cat([u * sig, g * sig], dim=1).abs() * (1 + g.abs()).repeat(1, 2) * (16 + g.abs()).repeat(1, 2) * U23
        dh, err = dh.repeat(1, 2), err.repeat(1, 2)
        carried = err * (slope.abs() + own) + dh.abs() * own
        within(dpre[rows], dh * slope, carried + BF16 * ((dh * slope).abs() + carried) + TINY)
    assert bool((dpre[bounds[-1]:] == 7.0).all())


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
@pytest.mark.parametrize("N,k,E,C,M,routing", CASES)
def test_weight_grad(N, k, E, C, M, routing, dtype):
    f = fusco()
    L, gen, bounds = make(N, k, E, 5, routing)
    dy, x = bf16(gen, L.P, M), bf16(gen, L.P, C)
    dy[bounds[-1]:] = float("nan")
    x[bounds[-1]:] = float("nan")
    dw = torch.full((E, M, C), 7.0, dtype=dtype, device="cuda")
    f.fusco_experts_weight_grad(L, dy, x, dw)
    rounding = BF16 if dtype == torch.bfloat16 else U23
    for e, rows in segments(bounds, dy):
        want, err = product(dy[rows].t(), x[rows].t())
        within(dw[e], want, err + rounding * (want.abs() + err) + TINY)   # zeros for an expert without rows


@pytest.mark.parametrize("N", [24, 300, 900])   # tiles of every height
def test_an_experts_values_stay_its_own(N):
    """Infinities and NaN in one expert's rows or weights reach no other expert's results."""
    f = fusco()
    L, gen, bounds = make(N, 2, 4, 6, "normal")
    C, M = 200, 136
    x, w, dy = bf16(gen, L.P, C), bf16(gen, 4, M, C), bf16(gen, L.P, M)
    sick = 1
    rows = slice(bounds[sick], bounds[sick + 1])
    x[rows], dy[rows], w[sick] = float("nan"), float("inf"), float("nan")
    y, dx, dw = (torch.empty(s, dtype=torch.bfloat16, device="cuda") for s in ((L.P, M), (L.P, C), (4, M, C)))
    f.fusco_experts_linear(L, x, w, y)
    f.fusco_experts_input_grad(L, dy, w, dx)
    f.fusco_experts_weight_grad(L, dy, x, dw)
    for t in (y, dx):
        assert bool(t[:rows.start].isfinite().all()) and bool(t[rows.stop:].isfinite().all())
        assert not bool(t[rows].isfinite().any())
    assert bool(dw[[0, 2, 3]].isfinite().all()) and not bool(dw[sick].isfinite().any())


def test_gradient_by_differences():
    """The gradient of sum(y * dy) along a direction of x and of w, by central differences in 64 bits of the formulas."""
    f = fusco()
    L, gen, bounds = make(90, 2, 3, 7, "normal")
    I, M = 40, 56
    pre, w, dy = bf16(gen, L.P, 2 * I), bf16(gen, 3, M, I, std=I ** -0.5), bf16(gen, L.P, M)
    dpre = torch.empty((L.P, 2 * I), dtype=torch.bfloat16, device="cuda")
    f.fusco_experts_input_grad(L, dy, w, dpre, pre=pre)
    direction = torch.randn(pre.shape, generator=gen, device="cuda", dtype=torch.float64)

    def loss(p):
        g, u = p.split(I, dim=1)
        h = g * torch.sigmoid(g) * u
        return sum(((h[r] @ w[e].double().t()) * dy[r].double()).sum() for e, r in segments(bounds, p))

    eps = 1e-4
    slope = (loss(pre.double() + eps * direction) - loss(pre.double() - eps * direction)) / (2 * eps)
    terms = dpre.double() * direction
    # every entry of dpre carries a rounding of up to 2^-8 of itself, at random: six standard deviations of their sum are below
    assert abs(float(slope - terms.sum())) <= 6 * 2.0 ** -8 * float(terms.norm()) + 1e-4 * abs(float(slope))


def test_empty_batch():
    f = fusco()
    L = f.Layout(0, 2, 4, 1)
    f.fusco_plan(L, torch.empty((0, 2), dtype=torch.int32, device="cuda"))
    x, w = torch.empty((0, 64), dtype=torch.bfloat16, device="cuda"), torch.ones((4, 32, 64), dtype=torch.bfloat16, device="cuda")
    y = torch.empty((0, 32), dtype=torch.bfloat16, device="cuda")
    dw = torch.ones((4, 32, 64), device="cuda")
    f.fusco_experts_linear(L, x, w, y)
    f.fusco_experts_gated(L, x, w, torch.empty((0, 16), dtype=torch.bfloat16, device="cuda"))
    f.fusco_experts_input_grad(L, y, w, x)
    f.fusco_experts_weight_grad(L, y, x, dw)
    assert bool((dw == 0).all())


def test_other_stream():
    """Tensors made on one stream, used on another after an event: the products run on the stream they are given."""
    f = fusco()
    L, gen, bounds = make(200, 2, 4, 8, "normal")
    x, w = bf16(gen, L.P, 256), bf16(gen, 4, 128, 256, std=1 / 16)
    want = torch.empty((L.P, 128), dtype=torch.bfloat16, device="cuda")
    f.fusco_experts_linear(L, x, w, want)
    torch.cuda.synchronize()
    side = torch.cuda.Stream()
    got = torch.zeros_like(want)
    side.wait_stream(torch.cuda.current_stream())
    f.fusco_experts_linear(L, x, w, got, stream=side)
    torch.cuda.current_stream().wait_stream(side)
    assert torch.equal(got, want)


def test_refusals():
    f = fusco()
    L, gen, _ = make(16, 2, 4, 9, "normal")
    x, w, y = bf16(gen, L.P, 64), bf16(gen, 4, 32, 64), bf16(gen, L.P, 32)
    for bad in (dict(x=x.float()), dict(x=x[:, :32].contiguous()), dict(x=x[:-1]), dict(w=w[:3].contiguous()), dict(w=w.transpose(1, 2)),
                dict(w=w.cpu()), dict(y=y.half()), dict(y=bf16(gen, L.P, 40)), dict(w=bf16(gen, 32, 64))):
        with pytest.raises(f.FuscoError):
            f.fusco_experts_linear(L, **dict(dict(x=x, w=w, y=y), **bad))
    with pytest.raises(f.FuscoError):   # rows of 12 bytes
        f.fusco_experts_linear(L, bf16(gen, L.P, 6), bf16(gen, 4, 32, 6), y)
    with pytest.raises(f.FuscoError):   # an odd number of rows cannot be gate and up
        f.fusco_experts_gated(L, x, bf16(gen, 4, 33, 64), y)
    with pytest.raises(f.FuscoError):
        f.fusco_experts_weight_grad(L, y, x, torch.empty((4, 32, 64), dtype=torch.float16, device="cuda"))
    with pytest.raises(f.FuscoError):
        f.fusco_experts_input_grad(L, y, w, x, pre=x)
