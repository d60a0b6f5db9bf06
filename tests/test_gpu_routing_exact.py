"""Scores that are compared are rounded operation by operation, so that a choice does not depend on how it is computed: the kernel's sigmoids
against torch's elementary operations on the same GPU, bit by bit, for every logit in bf16 and a fine sweep in fp32."""
import pytest
import torch

pytestmark = pytest.mark.gpu


def weights(l, score):
    """A single expert's weight is its score."""
    import paper_2512_22036_amd as f
    idx, w = torch.empty((l.numel(), 1), dtype=torch.int32, device="cuda"), torch.empty((l.numel(), 1), device="cuda")
    f.fusco_route(l.view(-1, 1), idx, w, score=score, renorm=False)
    return w.view(-1)


def same(got, want):
    return bool(((got == want) | (got.isnan() & want.isnan())).all())


def test_every_bf16_logit():
    import paper_2512_22036_amd as f
    l = torch.arange(65536, device="cuda").to(torch.int32).to(torch.int16).view(torch.bfloat16)
    assert same(weights(l, f.SCORE_SIGMOID), 1.0 / (1.0 + torch.exp(-l.float())))


@pytest.mark.parametrize("low,high", [(-110.0, -80.0), (-80.0, -20.0), (-20.0, -2.0), (-2.0, 2.0), (2.0, 20.0), (20.0, 120.0)])
def test_fine_sweep(low, high):
    import paper_2512_22036_amd as f
    l = torch.linspace(low, high, 1 << 22, device="cuda")
    assert same(weights(l, f.SCORE_SIGMOID), 1.0 / (1.0 + torch.exp(-l)))


def test_every_reciprocal():
    """1 + exp(-l) reaches every number from 1 to 2 on the sweep below; their reciprocals are the division's."""
    import paper_2512_22036_amd as f
    d = 1.0 + torch.arange(1, 1 << 23, device="cuda").double() * 2.0 ** -23
    l = (-torch.log(d - 1.0)).float()
    assert same(weights(l, f.SCORE_SIGMOID), 1.0 / (1.0 + torch.exp(-l)))
