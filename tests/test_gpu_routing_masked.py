"""Rows without any allowed expert where a bias takes part in the choice: every score is 0, so experts (and groups) compete by the bias alone, for
softmax scores as for sigmoids, and the weights are 0.  The expected choice is exact: 0 + bias is the bias."""
import pytest
import torch

pytestmark = pytest.mark.gpu


def by_bias(bias, k, groups, keep, best):
    b = bias.double()
    if groups > 1:
        of = bias.view(groups, -1).sort(dim=1, descending=True).values[:, :best]
        of = of[:, 0] + of[:, 1] if best == 2 else of[:, 0]          # one fp32 addition, as any form of it
        kept = of.sort(descending=True, stable=True).indices[:keep]
        stays = torch.zeros(groups, dtype=torch.bool, device="cuda").scatter_(0, kept, True)
        b = torch.where(stays.repeat_interleave(bias.numel() // groups), b, torch.full_like(b, -torch.inf))
    return b.sort(descending=True, stable=True).indices[:k].int()


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
@pytest.mark.parametrize("score", ["softmax", "sigmoid"])
@pytest.mark.parametrize("N,E,k,groups,keep,best", [
    (3, 16, 4, 1, 1, 1), (5, 60, 6, 1, 1, 1), (9, 64, 6, 8, 3, 2), (2100, 64, 4, 4, 2, 1), (7, 160, 6, 5, 2, 2), (33, 256, 8, 1, 1, 1), (33, 256, 8, 8, 4, 2), (2100, 256, 8, 8, 4, 2),
    (5000, 256, 8, 16, 3, 1), (6, 384, 8, 8, 4, 2), (4, 512, 10, 8, 4, 2), (5, 1024, 32, 32, 5, 2), (3, 100, 12, 1, 1, 1)])
def test_bias_decides_where_nothing_is_allowed(N, E, k, groups, keep, best, score, dtype):
    import paper_2512_22036_amd as f
    gen = torch.Generator(device="cuda").manual_seed(E + k)
    bias = torch.randn(E, generator=gen, device="cuda")
    l = torch.randn((N, E), generator=gen, device="cuda").to(dtype)
    masked = torch.arange(N, device="cuda") % 3 != 1
    l[masked] = -torch.inf
    idx, w = torch.full((N, k), -7, dtype=torch.int32, device="cuda"), torch.full((N, k), -7.0, device="cuda")
    how = dict(score=f.SCORE_SIGMOID if score == "sigmoid" else f.SCORE_SOFTMAX, scale=2.5)
    for renorm in (True, False):
        f.fusco_route(l, idx, w, bias=bias, groups=groups, keep_groups=keep, group_best=best, renorm=renorm, **how)
        assert torch.equal(idx[masked], by_bias(bias, k, groups, keep, best).expand(int(masked.sum()), k))
        assert bool((w[masked] == 0).all()) and bool((w[~masked] > 0).all())
        dl = torch.full_like(l, 7.0)
        f.fusco_route_backward(l, idx, torch.ones_like(w), dl, renorm=renorm, **how)
        assert bool((dl[masked] == 0).all()) and bool(dl.isfinite().all())
