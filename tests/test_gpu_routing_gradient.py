"""The routing's gradient where a sigmoid saturates, where every score is tiny, and at batch sizes of every instance of the kernel, against the
formula in 64 bits.

Tolerance.  Sigmoid scores: the gradient is sums of terms scale * s / S * dw * (1 - s), or without renormalisation scale * s * dw * (1 - s).  s and 1 - s =
1 / (1 + exp(l)) are each an exponential (2 units in the last place, and |l| units for its rounded argument), an addition and a division; the sum over k
chosen scores adds k roundings of positive terms, which carry their own errors: S is off by as much as the worst of them.  The difference dw - mean is bounded by
its two terms.  In units of 2^-23 with |l| the row's largest: 4 (|l| + 8) for the four factors that carry an exponential and k + 16 for all roundings, of the
terms' sizes, with 1 - s taken in 64 bits.  Softmax scores: the same with |l - max l| and E / 64 + 16 more for the denominator, without the factor 1 - s."""
import pytest
import torch

pytestmark = pytest.mark.gpu

U = 2.0 ** -23


def chosen(l, k):
    return l.double().sort(dim=1, descending=True, stable=True).indices[:, :k].int().contiguous()


def backward(l, idx, dw, score, renorm, scale=2.5):
    import paper_2512_22036_amd as f
    dl = torch.full(l.shape, 7.0, dtype=l.dtype, device="cuda")
    f.fusco_route_backward(l, idx, dw, dl, score=f.SCORE_SIGMOID if score == "sigmoid" else f.SCORE_SOFTMAX, renorm=renorm, scale=scale)
    return dl


def exact(l, idx, dw, score, renorm, scale=2.5):
    """The gradient and the sizes of its terms, without the derivative's own cancellations."""
    l, at, dw = l.double(), idx.long(), dw.double()
    s = torch.sigmoid(l) if score == "sigmoid" else torch.softmax(l, dim=1)
    p = s.gather(1, at)
    q = p / p.sum(dim=1, keepdim=True) if renorm else p
    mean, mean_size = (dw * q).sum(dim=1, keepdim=True), (dw.abs() * q).sum(dim=1, keepdim=True)
    if score == "sigmoid":
        slope = torch.sigmoid(-l).gather(1, at)
        d, size = scale * q * slope * (dw - mean if renorm else dw), scale * q * slope * (dw.abs() + mean_size if renorm else dw.abs())
    else:
        d, size = scale * q * (dw - mean if renorm else dw), scale * q * (dw.abs() + mean_size)
    want, bound = torch.zeros_like(l).scatter(1, at, d), torch.zeros_like(l).scatter(1, at, size)
    if score == "softmax" and not renorm:
        want, bound = want - scale * s * mean, bound + scale * s * mean_size
    return want, bound


def near(dl, l, idx, want, size, score):
    k, E = idx.shape[1], l.shape[1]
    l = l.double()
    far = l.abs().amax(dim=1, keepdim=True) if score == "sigmoid" else (l.amax(dim=1, keepdim=True) - l.amin(dim=1, keepdim=True))
    units = 4 * (far + 8) + k + 16 + (E / 64 + 16 if score == "softmax" else 0)
    own = 2.0 ** -8 if dl.dtype == torch.bfloat16 else U
    off = (dl.double() - want).abs() - (units * U * size + own * (want.abs() + units * U * size) + 1e-37)
    assert bool((off <= 0).all()), "off by %g more than the bound" % float(off.max())


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
@pytest.mark.parametrize("renorm", [True, False])
@pytest.mark.parametrize("low,high", [(8, 16), (16, 40), (-40, -8), (-40, 40), (60, 80), (-84, -60)])
@pytest.mark.parametrize("N,E,k", [(40, 64, 6), (37, 256, 8), (20, 100, 12), (2100, 256, 8)])
def test_sigmoids_that_saturate(N, E, k, low, high, renorm, dtype):
    gen = torch.Generator(device="cuda").manual_seed(N + E + high)
    l = (low + (high - low) * torch.rand((N, E), generator=gen, device="cuda")).to(dtype)
    idx, dw = chosen(l, k), torch.randn((N, k), generator=gen, device="cuda")
    want, size = exact(l, idx, dw, "sigmoid", renorm)
    near(backward(l, idx, dw, "sigmoid", renorm), l, idx, want, size, "sigmoid")


@pytest.mark.parametrize("score,low,bits", [("sigmoid", -88.7, 20), ("softmax", -89.0, 20), ("softmax", -96.0, 10)])
@pytest.mark.parametrize("N,E,k", [(10, 64, 6), (9, 256, 8), (5, 100, 12), (2100, 60, 1), (7, 64, 2)])
def test_tiny_scores(N, E, k, score, low, bits):
    """Weights that are renormalised have gradients of ordinary size, however small the chosen scores are: those of experts that a caller or a
    bias chose far below the best."""
    gen = torch.Generator(device="cuda").manual_seed(N)
    l = low + torch.rand((N, E), generator=gen, device="cuda")               # scores of 3e-39 and more, or 2e-42 and more
    idx = chosen(l, k)
    if score == "softmax":
        l[:, -1] = 0.0                                                        # the best one is not among them
        idx = (torch.arange(k, device="cuda") + torch.arange(N, device="cuda")[:, None] % (E - 1 - k)).int().contiguous()
    dw = torch.randn((N, k), generator=gen, device="cuda")
    dl = backward(l, idx, dw, score, True)
    assert bool(dl.isfinite().all())
    want, size = exact(l, idx, dw, score, True)
    # what a score below the smallest normal number has left: half a unit of 2^-bits in a share, its sum, and the mean of both; and 4 (|l| + 8) + k + 16 of 2^-23
    assert bool(((dl.double() - want).abs() <= (4 * 2.0 ** -bits + 512 * U) * size + 1e-37).all())


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
@pytest.mark.parametrize("score", ["softmax", "sigmoid"])
@pytest.mark.parametrize("renorm", [True, False])
@pytest.mark.parametrize("N,E,k", [(4097, 12, 2), (4097, 60, 4), (4098, 128, 8), (5001, 256, 8), (4099, 384, 8), (4100, 512, 10), (4097, 60, 16), (4098, 128, 12), (4099, 200, 11), (4101, 512, 24),
                                   (4097, 1024, 16), (2047, 256, 8), (2049, 512, 8), (300, 512, 4)])
def test_every_instance(N, E, k, renorm, score, dtype):
    gen = torch.Generator(device="cuda").manual_seed(N + E)
    l = torch.randn((N, E), generator=gen, device="cuda").to(dtype)
    idx, dw = chosen(l, k), torch.randn((N, k), generator=gen, device="cuda")
    want, size = exact(l, idx, dw, score, renorm)
    near(backward(l, idx, dw, score, renorm), l, idx, want, size, score)


def test_undefined_logits():
    """A NaN makes a softmax row's gradient NaN; a sigmoid's stays with its expert, and with the weights that it enters."""
    l = torch.randn((3, 32), generator=torch.Generator(device="cuda").manual_seed(1), device="cuda")
    l[0, 3] = float("nan")
    l[1, 4], l[1, 5] = torch.inf, -torch.inf
    idx = torch.tensor([[0, 1, 2, 4]] * 3, dtype=torch.int32, device="cuda")
    for renorm in (True, False):
        dl = backward(l, idx, torch.ones((3, 4), device="cuda").cumsum(1), "softmax", renorm)
        assert bool(dl[:2].isnan().all()) and bool(dl[2].isfinite().all())
        dl = backward(l, idx, torch.ones((3, 4), device="cuda").cumsum(1), "sigmoid", renorm)
        assert bool(dl[0, 3].isnan()) and bool(dl[0, :3].isfinite().all()) and bool(dl[1:].isfinite().all()) and dl[1, 4] == 0
