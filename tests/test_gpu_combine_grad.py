"""The gradient of the combine.  dy is one product of two numbers, rounded once: bit for bit.  dw is an fp32 sum over a row, at most 64
additions deep (32 products in a thread, six steps in a wave, 16 waves) with one rounding per product: within 66 * 2^-24 of the sum of its
terms' sizes."""
import pytest
import torch

pytestmark = pytest.mark.gpu

B, F = torch.bfloat16, torch.float32


def fusco():
    import paper_2512_22036_amd as f
    f.load_library()
    return f


def inputs(N, H, k, E, D, y, dout, seed, invalid=False):
    gen = torch.Generator(device="cuda").manual_seed(seed)
    chosen = torch.rand((N, E), generator=gen, device="cuda").topk(k, dim=1).indices.to(torch.int32)
    if invalid:
        chosen[torch.rand((N, k), generator=gen, device="cuda") < 0.3] = -1
    f = fusco()
    L = f.Layout(N, k, E, D)
    f.fusco_plan(L, chosen.contiguous())
    return (L, torch.randn((N * k, H), generator=gen, device="cuda").to(y), torch.randn((N, k), generator=gen, device="cuda"),
            torch.randn((N, H), generator=gen, device="cuda").to(dout))


@pytest.mark.parametrize("y,dout", [(B, B), (B, F), (F, B), (F, F)])
@pytest.mark.parametrize("N,H,k,E,D", [(1, 8, 1, 1, 1), (1, 7168, 8, 256, 8), (5, 72, 3, 16, 4), (64, 512, 64, 64, 1), (33, 2880, 6, 160, 5), (1100, 520, 2, 16, 4), (1030, 7168, 8, 64, 8), (3, 32768, 5, 8, 2),
                                       (1025, 10248, 3, 8, 2)])
@pytest.mark.parametrize("invalid", [False, True])
def test_gradients(N, H, k, E, D, y, dout, invalid):
    f = fusco()
    L, rows, w, grad = inputs(N, H, k, E, D, y, dout, N + H, invalid)
    dy, dw = torch.full((N * k, H), 7.0, dtype=y, device="cuda"), torch.full((N, k), 7.0, device="cuda")
    f.fusco_combine_backward(L, rows, w, grad, dy, dw)
    slot = L.array("pair_slot").long()
    there = slot >= 0
    pair = torch.arange(N * k, device="cuda")[there]
    want = torch.full_like(dy, 7.0)             # rows without a pair stay as they were
    want[slot[there]] = (w.view(-1)[pair][:, None] * grad[pair // k].float()).to(y)
    assert torch.equal(dy, want)
    terms = rows[slot[there]].double() * grad[pair // k].double()
    want_w, size = torch.zeros(N * k, dtype=torch.float64, device="cuda"), torch.zeros(N * k, dtype=torch.float64, device="cuda")
    want_w[pair], size[pair] = terms.sum(dim=1), terms.abs().sum(dim=1)
    assert bool(((dw.double().view(-1) - want_w).abs() <= 66 * 2.0 ** -24 * size).all())


def test_gradient_by_differences():
    f = fusco()
    L, rows, w, grad = inputs(12, 64, 3, 8, 2, F, F, 5)
    dy, dw = torch.empty_like(rows), torch.empty_like(w)
    f.fusco_combine_backward(L, rows, w, grad, dy, dw)
    slot = L.array("pair_slot").long()
    gen = torch.Generator(device="cuda").manual_seed(6)
    dir_y, dir_w = torch.randn(rows.shape, generator=gen, device="cuda", dtype=torch.float64), torch.randn(w.shape, generator=gen, device="cuda", dtype=torch.float64)

    def loss(y, weights):
        return ((weights.view(-1)[:, None] * y[slot]).view(12, 3, 64).sum(dim=1) * grad.double()).sum()

    y, weights, eps = rows.double(), w.double(), 1e-3     # the loss is linear in each: no error of its own
    for got, d, plus, minus in ((dy, dir_y, loss(y + eps * dir_y, weights), loss(y - eps * dir_y, weights)), (dw, dir_w, loss(y, weights + eps * dir_w), loss(y, weights - eps * dir_w))):
        terms = got.double() * d
        assert abs(float((plus - minus) / (2 * eps) - terms.sum())) <= 66 * 2.0 ** -24 * float(terms.abs().sum()) * 8 + 1e-9


def test_dispatch_gradient_is_a_combine():
    """The gradient of the dispatch: every token's rows added up, by the combine with weights of 1."""
    f = fusco()
    L, rows, w, grad = inputs(50, 256, 4, 16, 4, F, F, 7)
    dx = torch.empty((50, 256), device="cuda")
    f.fusco_combine(L, rows, torch.ones_like(w), dx)
    want = rows.double()[L.array("pair_slot").long()].view(50, 4, 256).sum(dim=1)
    assert bool(((dx.double() - want).abs() <= 8 * 2.0 ** -24 * rows.abs().max() * 4).all())


def test_empty_and_refusals():
    f = fusco()
    L, rows, w, grad = inputs(4, 64, 2, 4, 1, F, F, 8)
    dy, dw = torch.empty_like(rows), torch.empty_like(w)
    good = dict(layout=L, y=rows, w=w, dout=grad, dy=dy, dw=dw)
    for bad in (dict(dy=dy.bfloat16()), dict(dy=dy[:-1]), dict(dout=grad[:, :32].contiguous()), dict(w=w.double()), dict(dw=dw[:, :1].contiguous()), dict(y=rows.half()), dict(dout=grad.cpu()),
                dict(y=rows[:, :60].contiguous(), dy=dy[:, :60].contiguous(), dout=grad[:, :60].contiguous())):
        with pytest.raises(f.FuscoError):
            f.fusco_combine_backward(**{**good, **bad})
    L0 = f.Layout(0, 2, 4, 1)
    e = lambda *s: torch.empty(s, device="cuda")
    f.fusco_combine_backward(L0, e(0, 64), e(0, 2), e(0, 64), e(0, 64), e(0, 2))
