"""Rows that the lanes hold in neighbouring columns, 16 bytes at a time, against rows that they cannot load so, and both against the choice by
definition: scores and group scores are rounded operation by operation, so the chosen experts are equal and not merely close."""
import pytest
import torch

pytestmark = pytest.mark.gpu


def route(l, k, bias, groups, keep, best):
    import paper_2512_22036_amd as f
    idx = torch.full((l.shape[0], k), -7, dtype=torch.int32, device="cuda")
    w = torch.full((l.shape[0], k), -7.0, device="cuda")
    f.fusco_route(l, idx, w, bias=bias, score=f.SCORE_SIGMOID, groups=groups, keep_groups=keep, group_best=best, scale=2.5)
    return idx, w


def by_definition(l, k, bias, groups, keep, best):
    b = 1.0 / (1.0 + torch.exp(-l.float())) + bias
    if groups > 1:
        of = b.view(l.shape[0], groups, -1).sort(dim=2, descending=True).values[:, :, :best]
        of = of[:, :, 0] + of[:, :, 1] if best == 2 else of[:, :, 0]
        kept = of.sort(dim=1, descending=True, stable=True).indices[:, :keep]
        stays = torch.zeros((l.shape[0], groups), dtype=torch.bool, device="cuda").scatter_(1, kept, True)
        b = torch.where(stays.repeat_interleave(l.shape[1] // groups, dim=1), b, torch.full_like(b, -torch.inf))
    return b.sort(dim=1, descending=True, stable=True).indices[:, :k].int()


def off(t, columns):
    """The same values in rows that begin `columns` elements past a 16-byte boundary."""
    held = torch.zeros((t.shape[0], t.shape[1] + 16), dtype=t.dtype, device="cuda")
    held[:, columns:columns + t.shape[1]] = t
    return held[:, columns:columns + t.shape[1]]


@pytest.mark.parametrize("coarse", [False, True])
@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
@pytest.mark.parametrize("N", [1, 7, 2048, 2049, 5000])
@pytest.mark.parametrize("E,groups,keep,best,k", [
    (64, 1, 1, 1, 6), (64, 8, 3, 2, 8), (64, 16, 4, 1, 10), (64, 32, 8, 2, 8), (128, 1, 1, 1, 8), (128, 4, 2, 2, 8), (128, 16, 5, 2, 10),
    (256, 1, 1, 1, 8), (256, 2, 1, 2, 8), (256, 8, 4, 2, 8), (256, 16, 1, 1, 16), (256, 64, 3, 2, 8), (256, 32, 32, 2, 9),
    (512, 1, 1, 1, 10), (512, 8, 4, 2, 8), (512, 16, 2, 1, 24), (512, 64, 2, 2, 10), (1024, 1, 1, 1, 8), (1024, 8, 4, 2, 8), (1024, 64, 9, 2, 64)])
def test_rows_of_whole_lanes(E, groups, keep, best, k, N, dtype, coarse):
    gen = torch.Generator(device="cuda").manual_seed(E * 31 + groups * 7 + N)
    l = torch.randn((N, E), generator=gen, device="cuda") * 2
    bias = torch.randn(E, generator=gen, device="cuda") * 0.1
    if coarse:   # many equal scores: ties of experts and of groups
        l, bias = l.round(), torch.zeros_like(bias)
    l = l.to(dtype)
    want = by_definition(l, k, bias, groups, keep, best)
    idx, w = route(l, k, bias, groups, keep, best)
    assert torch.equal(idx, want)
    for moved in (off(l, 1), off(l, 8)):
        idx2, w2 = route(moved, k, bias, groups, keep, best)
        assert torch.equal(idx2, want) and torch.equal(w2, w)
    held = torch.zeros(E + 1, device="cuda")
    held[1:] = bias
    idx3, w3 = route(l, k, held[1:], groups, keep, best)
    assert torch.equal(idx3, want) and torch.equal(w3, w)


def test_masked_and_undefined_logits():
    """Infinities and NaN in rows of whole lanes: a group is not worse for a NaN in it, and a NaN is chosen behind every score."""
    l = torch.randn((9, 256), generator=torch.Generator(device="cuda").manual_seed(5), device="cuda")
    l[0] = -torch.inf
    l[1, 64:] = -torch.inf
    l[2, ::3] = torch.nan
    l[3] = torch.finfo(torch.float32).min
    l[4, 17] = torch.inf
    bias = torch.zeros(256, device="cuda")
    idx, w = route(l, 8, bias, 8, 4, 2)
    idx2, w2 = route(off(l, 3), 8, bias, 8, 4, 2)
    assert torch.equal(idx, idx2) and torch.equal(w.isnan(), w2.isnan()) and torch.equal(w.nan_to_num(-1), w2.nan_to_num(-1))
    for n in (0, 1, 3, 4, 5, 6, 7, 8):
        assert torch.equal(idx[n:n + 1], by_definition(l[n:n + 1], 8, bias, 8, 4, 2))
    assert not bool((idx[2] % 3 == 0).any())   # enough other experts in the kept groups
