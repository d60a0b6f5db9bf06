"""Routing and its gradient against the definition in 64 bits.

Tolerance.  A score is an exponential (2 units in the last place, and |x| units for its rounded argument), an addition and a
division: relative error below (|x| + 8) * 2^-23.  Sums of up to n scores are lane sums of n / 64 terms and six additions: below
(n / 64 + 6) * 2^-24 of their (positive) terms.  Two experts whose exact b differ by less than both errors may be chosen in either
order; everything else must be as defined, and equal scores go to the lower index exactly."""
import pytest
import torch

pytestmark = pytest.mark.gpu

U = 2.0 ** -23


def fusco():
    import paper_2512_22036_amd as f
    f.load_library()
    return f


def scores64(l, score):
    l = l.double()
    if score == "sigmoid":
        return torch.sigmoid(l)
    m = l.amax(dim=1, keepdim=True)
    e = torch.exp(l - torch.where(m == -torch.inf, torch.zeros_like(m), m))
    total = e.sum(dim=1, keepdim=True)
    return torch.where(total == 0, total, e / total.clamp_min(1e-300))


def units(l):
    """Relative error of a row's scores in units of 2^-23."""
    l = l.double()
    finite = l.isfinite()
    x = torch.where(finite, l, torch.zeros_like(l))
    m = torch.where(finite, l, torch.full_like(l, -1e9)).amax(dim=1, keepdim=True).clamp(min=-1e8)
    return torch.maximum(x.abs(), (m - torch.where(finite, l, m.expand_as(l))).abs()).clamp(max=110.0) + l.shape[1] / 128 + 16


def call(l, k, bias=None, score="softmax", groups=1, keep=1, best=1, renorm=True, scale=1.0):
    f = fusco()
    N = l.shape[0]
    idx = torch.full((N, k), -7, dtype=torch.int32, device="cuda")
    w = torch.full((N, k), -7.0, device="cuda")
    f.fusco_route(l, idx, w, bias=bias, score=f.SCORE_SIGMOID if score == "sigmoid" else f.SCORE_SOFTMAX, groups=groups, keep_groups=keep,
                  group_best=best, renorm=renorm, scale=scale)
    return idx, w


def check(l, k, bias=None, score="softmax", groups=1, keep=1, best=1, renorm=True, scale=1.0):
    idx, w = call(l, k, bias, score, groups, keep, best, renorm, scale)
    N, E = l.shape
    s = scores64(l, score)
    rel = units(l)
    b = s if bias is None else s + bias.double()
    err = rel * U * s.abs() + U * b.abs()
    at = idx.long()
    assert bool(((at >= 0) & (at < E)).all())
    assert bool((torch.sort(at, dim=1).values.diff(dim=1) > 0).all())          # distinct
    allowed = torch.ones_like(b, dtype=torch.bool)
    if groups > 1:
        size = E // groups
        score_g = b.view(N, groups, size).topk(best, dim=2).values.sum(dim=2)
        err_g = 2 * err.view(N, groups, size).amax(dim=2) + U * score_g.abs()
        used = torch.zeros((N, groups), dtype=torch.bool, device="cuda").scatter_(1, at // size, True)
        assert int(used.sum(dim=1).max()) <= keep
        # a group that was surely among the best may not have been left out: fewer than `keep` groups are surely ahead of every used one
        low = torch.where(used, score_g + err_g, torch.full_like(score_g, torch.inf)).amin(dim=1, keepdim=True)
        assert bool((((score_g - err_g) > low).sum(dim=1) < keep).all())
        ahead = ((score_g - err_g)[:, None, :] > (score_g + err_g)[:, :, None]).sum(dim=2)
        behind = ((score_g + err_g)[:, None, :] < (score_g - err_g)[:, :, None]).sum(dim=2)
        allowed = (behind >= groups - keep).repeat_interleave(size, dim=1)     # surely kept: its experts compete
        assert bool((ahead.gather(1, at // size) < keep).all())
    picked, picked_err = b.gather(1, at), err.gather(1, at)
    assert bool((picked[:, :-1] - picked[:, 1:] >= -(picked_err[:, :-1] + picked_err[:, 1:])).all())
    left = torch.where(allowed, b - err, torch.full_like(b, -torch.inf)).scatter(1, at, -torch.inf).amax(dim=1)
    assert bool((left <= picked[:, -1] + picked_err[:, -1]).all())
    p = s.gather(1, at)
    of = p.sum(dim=1, keepdim=True) if renorm else torch.ones_like(p[:, :1])
    want = torch.where(of == 0, torch.zeros_like(p), scale * p / of.clamp_min(1e-300))
    tol = 2 * rel.amax(dim=1, keepdim=True) * U * want.abs() + 1e-37
    assert bool(((w.double() - want).abs() <= tol).all())
    return idx, w


SHAPES = [(1, 1, 1), (1, 8, 2), (3, 16, 2), (5, 60, 6), (64, 64, 64), (33, 65, 3), (128, 256, 8), (1000, 128, 8), (7, 160, 6), (257, 384, 10), (9, 1024, 16), (130, 513, 1)]


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
@pytest.mark.parametrize("score", ["softmax", "sigmoid"])
@pytest.mark.parametrize("N,E,k", SHAPES)
def test_choice_and_weights(N, E, k, score, dtype):
    gen = torch.Generator(device="cuda").manual_seed(N * 1000 + E)
    l = torch.randn((N, E), generator=gen, device="cuda").mul_(2).to(dtype)
    for renorm, scale in ((True, 1.0), (True, 2.5), (False, 1.0)):
        check(l, k, score=score, renorm=renorm, scale=scale)


@pytest.mark.parametrize("score", ["softmax", "sigmoid"])
@pytest.mark.parametrize("N,E,k,groups,keep,best", [(64, 256, 8, 8, 4, 2), (33, 256, 8, 8, 4, 1), (100, 128, 8, 16, 8, 2), (17, 160, 6, 5, 2, 2), (50, 160, 6, 8, 3, 1),
                                                    (9, 384, 8, 8, 4, 2), (300, 64, 4, 64, 4, 1), (40, 64, 8, 2, 1, 2), (7, 1024, 32, 32, 5, 2), (20, 12, 2, 3, 1, 2)])
@pytest.mark.parametrize("biased", [False, True])
def test_groups(N, E, k, groups, keep, best, score, biased):
    gen = torch.Generator(device="cuda").manual_seed(N * 77 + E)
    l = torch.randn((N, E), generator=gen, device="cuda")
    bias = torch.randn((E,), generator=gen, device="cuda") * (0.1 if score == "sigmoid" else 0.01) if biased else None
    check(l, k, bias=bias, score=score, groups=groups, keep=keep, best=best, scale=2.5)


@pytest.mark.parametrize("score", ["softmax", "sigmoid"])
@pytest.mark.parametrize("N,E,k", [(50, 64, 8), (30, 256, 8), (20, 100, 12)])
def test_ties_go_to_the_lower_index(N, E, k, score):
    gen = torch.Generator(device="cuda").manual_seed(5)
    l = torch.randint(-2, 3, (N, E), generator=gen, device="cuda").float()      # five values: every choice is among ties
    idx, _ = check(l, k, score=score)
    want = torch.sort(l, dim=1, descending=True, stable=True).indices[:, :k]
    assert torch.equal(idx.long(), want)
    idx, _ = call(torch.zeros_like(l), k, score=score, groups=4, keep=2)        # all groups alike: the first ones
    assert torch.equal(idx.long(), torch.arange(k, device="cuda").expand(N, k))


@pytest.mark.parametrize("score", ["softmax", "sigmoid"])
def test_masked_experts(score):
    gen = torch.Generator(device="cuda").manual_seed(6)
    l = torch.randn((40, 64), generator=gen, device="cuda")
    l[:, ::3] = -torch.inf
    idx, w = check(l, 8, score=score)
    assert bool((idx % 3 != 0).all())
    l[:] = -torch.inf                                                           # nobody is allowed
    idx, w = call(l, 8, score=score)
    assert torch.equal(idx.long(), torch.arange(8, device="cuda").expand(40, 8)) and bool((w == 0).all())
    l[:, 5] = 0.25                                                              # one is
    idx, w = call(l, 8, score=score)
    assert bool((idx[:, 0] == 5).all()) and bool((w[:, 0] == 1).all()) and bool((w[:, 1:] == 0).all())
    low = torch.full((3, 64), torch.finfo(torch.float32).min, device="cuda")    # masked with the type's lowest value
    low[:, 7] = 1.0
    idx, w = call(low, 2, score=score)
    assert bool((idx[:, 0] == 7).all()) and bool((w[:, 0] == 1).all()) and bool((w[:, 1] == 0).all())
    idx, w = call(low[:, :7].contiguous(), 2, score=score)                      # everything masked so
    assert torch.equal(idx.long(), torch.tensor([[0, 1]] * 3, device="cuda"))
    assert bool((w == (0.5 if score == "softmax" else 0.0)).all())


def test_not_a_number():
    l = torch.zeros((4, 32), device="cuda")
    l[0, 3] = l[1, :] = float("nan")
    l[2, 4] = torch.inf
    idx, w = call(l, 4, score="sigmoid")
    assert idx[0].tolist() == [0, 1, 2, 4] and bool((w[0] == 0.25).all())       # a NaN ranks last
    assert idx[1].tolist() == [0, 1, 2, 3] and bool(w[1].isnan().all())
    assert idx[2, 0] == 4 and bool(w[2].isfinite().all())
    idx, w = call(l, 4, score="softmax")
    assert bool(w[:3].isnan().all()) and bool((w[3] == 0.25).all())
    assert bool((torch.sort(idx, dim=1).values.diff(dim=1) > 0).all())


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
def test_rows_that_lie_apart(dtype):
    gen = torch.Generator(device="cuda").manual_seed(8)
    wide = torch.randn((37, 131), generator=gen, device="cuda").to(dtype)
    view = wide[:, 5:70]
    idx, w = check(view, 6, score="sigmoid")
    idx2, w2 = call(view.contiguous(), 6, score="sigmoid")
    assert torch.equal(idx, idx2) and torch.equal(w, w2)


def grad64(l, idx, dw, score, renorm, scale):
    l = l.double().requires_grad_()
    s = torch.sigmoid(l) if score == "sigmoid" else torch.softmax(l, dim=1)
    p = s.gather(1, idx.long())
    w = scale * (p / p.sum(dim=1, keepdim=True) if renorm else p)
    return torch.autograd.grad(w, l, dw.double())[0]


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
@pytest.mark.parametrize("score", ["softmax", "sigmoid"])
@pytest.mark.parametrize("renorm", [True, False])
@pytest.mark.parametrize("N,E,k", SHAPES)
def test_gradient(N, E, k, score, renorm, dtype):
    f = fusco()
    gen = torch.Generator(device="cuda").manual_seed(N + E)
    l = torch.randn((N, E), generator=gen, device="cuda").to(dtype)
    idx, _ = call(l, k, score=score, renorm=renorm, scale=2.5)
    dw = torch.randn((N, k), generator=gen, device="cuda")
    dl = torch.full((N, E), 7.0, dtype=dtype, device="cuda")
    f.fusco_route_backward(l, idx, dw, dl, score=f.SCORE_SIGMOID if score == "sigmoid" else f.SCORE_SOFTMAX, renorm=renorm, scale=2.5)
    want = grad64(l, idx, dw, score, renorm, 2.5)
    s = scores64(l, score)
    p = s.gather(1, idx.long())
    of = p.sum(dim=1, keepdim=True) if renorm else torch.ones_like(p[:, :1])
    # the terms that the gradient is a difference of, without their signs
    size = 2.5 / of * s * (torch.zeros_like(s).scatter(1, idx.long(), dw.double().abs()) + (dw.double().abs() * p).sum(dim=1, keepdim=True) / of)
    tol = 4 * units(l).amax(dim=1, keepdim=True) * U * size + (2.0 ** -8 if dtype == torch.bfloat16 else U) * want.abs() + 1e-37
    assert bool(((dl.double() - want).abs() <= tol).all())


@pytest.mark.parametrize("score", ["softmax", "sigmoid"])
@pytest.mark.parametrize("renorm", [True, False])
def test_gradient_by_differences(score, renorm):
    f = fusco()
    gen = torch.Generator(device="cuda").manual_seed(3)
    l = torch.randn((20, 48), generator=gen, device="cuda")
    idx, _ = call(l, 5, score=score, renorm=renorm)
    dw = torch.randn((20, 5), generator=gen, device="cuda")
    dl = torch.empty_like(l)
    f.fusco_route_backward(l, idx, dw, dl, score=f.SCORE_SIGMOID if score == "sigmoid" else f.SCORE_SOFTMAX, renorm=renorm)
    direction = torch.randn(l.shape, generator=gen, device="cuda", dtype=torch.float64)

    def loss(x):   # the choice is held
        s = torch.sigmoid(x) if score == "sigmoid" else torch.softmax(x, dim=1)
        p = s.gather(1, idx.long())
        return ((p / p.sum(dim=1, keepdim=True) if renorm else p) * dw.double()).sum()

    eps = 1e-5
    slope = (loss(l.double() + eps * direction) - loss(l.double() - eps * direction)) / (2 * eps)
    # third derivatives of order one times eps^2, and 2^-52 / eps of the loss
    assert abs(float(slope - (dl.double() * direction).sum())) <= 64 * U * float((dl.double() * direction).abs().sum()) + 1e-8


def test_gradient_where_nothing_is_allowed():
    f = fusco()
    l = torch.full((2, 16), -torch.inf, device="cuda")
    for score in (f.SCORE_SOFTMAX, f.SCORE_SIGMOID):
        idx, w = torch.empty((2, 4), dtype=torch.int32, device="cuda"), torch.empty((2, 4), device="cuda")
        f.fusco_route(l, idx, w, score=score)
        dl = torch.full_like(l, 7.0)
        f.fusco_route_backward(l, idx, torch.ones_like(w), dl, score=score)
        assert bool((dl == 0).all())


def test_routing_feeds_the_plan():
    f = fusco()
    gen = torch.Generator(device="cuda").manual_seed(4)
    l = torch.randn((200, 32), generator=gen, device="cuda")
    idx, w = call(l, 4)
    L = f.Layout(200, 4, 32, 4)
    f.fusco_plan(L, idx)
    assert int(L.array("status")[0]) == 0 and int(L.array("exp_off")[32]) == 800


def test_empty_and_refusals():
    f = fusco()
    call(torch.empty((0, 8), device="cuda"), 2)
    l = torch.zeros((4, 8), device="cuda")
    for kw in (dict(k=9), dict(k=2, groups=3), dict(k=2, groups=4, keep=5), dict(k=3, groups=4, keep=1), dict(k=2, groups=8, keep=8, best=2), dict(k=2, best=3), dict(k=2, groups=0),
               dict(k=2, scale=float("nan"))):
        with pytest.raises(f.FuscoError):
            call(l, **kw)
    with pytest.raises(f.FuscoError):
        call(l.double(), 2)
    with pytest.raises(f.FuscoError):
        call(l.t(), 2)
    with pytest.raises(f.FuscoError):
        call(l, 2, bias=torch.zeros((7,), device="cuda"))
    with pytest.raises(f.FuscoError):
        call(torch.zeros((4, 1025), device="cuda"), 2)
    with pytest.raises(f.FuscoError):
        call(l.cpu(), 2)
    with pytest.raises(f.FuscoError):
        f.fusco_route_backward(l, torch.zeros((4, 2), dtype=torch.int32, device="cuda"), torch.zeros((4, 2), device="cuda"), l.bfloat16())
