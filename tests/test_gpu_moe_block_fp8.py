"""The example's block in e4m3, all operators together, forward and backward, against 64 bits from the values that it kept; and a decode step and a training step of it
captured into graphs and replayed.

Tolerances.  Of results and gradients as for the block in bf16: values that are kept in e4m3 enter both sides alike, and the matrix instructions' cuts
(2^-13 of the largest of 8 products, 2^-16 of a result on the average) are far below a rounding to bf16, 2^-8.  What is kept in e4m3 is off by half a step, 2^-4 of
each value, or where it is below 2^-6 of its block's scale by 2^-10 of that scale, at most 2^-9 / 448 of the block's largest; the rest, 0.02, is for the roundings before."""
import importlib.util
import os

import pytest
import torch

pytestmark = pytest.mark.gpu
ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))


@pytest.fixture(scope="module")
def example():
    spec = importlib.util.spec_from_file_location("moe_block", os.path.join(ROOT, "examples", "moe_block.py"))
    module = importlib.util.module_from_spec(spec)
    spec.loader.exec_module(module)
    module.fusco.load_library()
    return module


@pytest.mark.parametrize("sizes", [dict(), dict(N=1), dict(N=64, H=400, I=208), dict(N=700, H=144, I=80, E=12, k=2, D=3, keep_groups=1), dict(N=520, H=512, I=256, E=8, k=4, D=2, keep_groups=2)])
def test_block(example, sizes):
    far, kept = example.check_eight(**sizes)
    assert max(far.values()) < 0.02, far
    assert max(kept.values()) < 2.0 ** -4 + 0.02, kept


@pytest.mark.parametrize("N,train", [(3, False), (64, False), (130, False), (130, True)])
def test_captured(example, N, train):
    """Each replay reads what lies in the inputs then, with eager work and synchronizations in between."""
    H, I = 272, 144
    block = example.EightBlock(H, I, 12, 3, 4, 2)
    gen = torch.Generator(device="cuda").manual_seed(7)
    normal = lambda t: torch.randn((N, H), generator=gen, device="cuda").to(t)
    r, y, ds, dout = normal(torch.float32), normal(torch.bfloat16), normal(torch.float32), normal(torch.bfloat16)

    def step():
        if not train:
            return list(block.forward(r, y))
        s, out, kept = block.forward(r, y, keep=True)
        grads = block.backward(kept, ds, dout)
        return [s, out] + [grads[n] for n in sorted(grads) if n != "router"]     # that one comes from a library's product

    stream = torch.cuda.Stream()
    stream.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(stream):
        step()
    torch.cuda.current_stream().wait_stream(stream)
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        got = step()
    for _ in range(4):
        r.copy_(normal(torch.float32))
        y.copy_(normal(torch.bfloat16))
        graph.replay()
        torch.cuda.synchronize()
        want = step()
        for a, b in zip(got, want):
            assert torch.equal(a, b)


@pytest.mark.parametrize("N,few", [(1, True), (8, True), (9, False), (64, False)])
def test_way_of_a_forward_pass(example, monkeypatch, N, few):
    """Where the products on e4m3 rows are faster than the layer for a few tokens, they are taken."""
    block = example.EightBlock(256, 128, 16, 4, 4, 2)
    calls = []
    whole = example.fusco.fusco_moe_few
    monkeypatch.setattr(example.fusco, "fusco_moe_few", lambda *a, **kw: (calls.append(1), whole(*a, **kw)))
    r, y = torch.randn((N, 256), device="cuda"), torch.randn((N, 256), device="cuda").bfloat16()
    block.forward(r, y)
    block.forward(r, y, keep=True)
    assert len(calls) == (1 if few else 0)
