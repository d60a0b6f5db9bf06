"""Input gradients in tiles of 64 rows and 128 outputs: where there are few tiles, the compute units have one each.  Sums keep the order that they have in tiles of
256 outputs, so results are equal bit by bit to those of the same experts' rows among the rows of many more experts; and they hold against the formulas
where segments are so uneven that workgroups take several of these tiles."""
import pytest
import torch

import test_gpu_experts as small
import test_gpu_fp8_kept as kept
from test_gpu_experts import bf16, fusco
from test_gpu_experts_many_tiles import WORKGROUPS

pytestmark = pytest.mark.gpu


def planned(counts):
    """A layout whose experts have these numbers of rows, one after the other."""
    f = fusco()
    L = f.Layout(sum(counts), 1, len(counts), 1)
    f.fusco_plan(L, torch.repeat_interleave(torch.arange(len(counts)), torch.tensor(counts)).int().cuda().view(-1, 1))
    bounds = L.array("exp_off").tolist()
    assert [b - a for a, b in zip(bounds, bounds[1:])] == list(counts)
    return L, bounds


def tiles(counts, outputs):
    return sum((n + 63) // 64 for n in counts) * ((outputs + 127) // 128)


def outputs_of(L, C, M):
    f = fusco()
    return [f.fusco_probe_experts_tile_outputs(L, which, C, M) for which in (f.PRODUCT_INPUT_GRAD, f.PRODUCT_INPUT_GRAD_ACTIVATION)]


# outputs that end inside a tile of 128, inside one of 256, at neither; sums of one stage, of odd and even numbers of halves, with a ragged end; rows from none on
@pytest.mark.parametrize("counts", [(38, 0, 64, 65, 1, 40), (7,), (130, 64, 200)])
@pytest.mark.parametrize("M", [8, 32, 72, 104, 336, 1040])
@pytest.mark.parametrize("C", [16, 144, 272, 528, 2320])
def test_same_as_among_many_experts(C, M, counts):
    f = fusco()
    gen = torch.Generator(device="cuda").manual_seed(61)
    more = (66,) * 300
    (few, few_bounds), (many, many_bounds) = planned(counts), planned(counts + more)
    assert outputs_of(few, C, M) == [128, 128] and 128 not in outputs_of(many, C, M)
    P, E = few.P, len(counts)
    dy, pre = bf16(gen, many.P, M), bf16(gen, many.P, 2 * C, std=2.0)
    w = bf16(gen, len(counts + more), M, C, std=M ** -0.5)
    kept_pre, scale = kept.kept(gen, many.P, 2 * C, True, 2.0)
    new = lambda L, columns: torch.full((L.P, columns), 7.0, dtype=torch.bfloat16, device="cuda")
    for columns, named in ((C, lambda L: {}), (2 * C, lambda L: dict(pre=pre[:L.P])), (2 * C, lambda L: dict(pre=kept_pre[:L.P], pre_scale=scale[:L.P]))):
        got, want = new(few, columns), new(many, columns)
        f.fusco_experts_input_grad(few, dy[:P], w[:E], got, **named(few))
        f.fusco_experts_input_grad(many, dy, w, want, **named(many))
        assert torch.equal(got, want[:P])


@pytest.mark.parametrize("form", ["plain", "activation", "kept"])
@pytest.mark.parametrize("counts,C,M", [((66, 14) * 60, 256, 336), ((66, 1) * 25, 528, 72), ((1, 66, 0, 130) * 10, 624, 1040)])
def test_several_tiles_per_workgroup(monkeypatch, counts, C, M, form):
    gen = torch.Generator(device="cuda").manual_seed(62)
    L, bounds = planned(counts)
    assert outputs_of(L, C, M) == [128, 128] and tiles(counts, C) > WORKGROUPS
    for module in (small, kept):
        monkeypatch.setattr(module, "make", lambda *a: (L, gen, bounds))
    N, E = L.P, len(counts)
    if form == "plain":
        small.test_input_grad(N, 1, E, C, M, "given")
    elif form == "activation":
        small.test_input_grad_through_the_activation(N, 1, E, C, M, "given")
    else:
        kept.test_input_grad(N, 1, E, C, M, "given", True)
