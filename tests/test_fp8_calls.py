"""The calls on e4m3 and the layer for a few tokens that go through csrc/fastcall.cpp: without a GPU it leaves everything to ctypes; with one both ways
give the same bytes, and what it cannot handle is refused or accepted as ctypes does."""
import os

import pytest
import torch

FP8 = torch.float8_e4m3fn


def test_leaves_everything_else_to_the_other_path():
    from paper_2512_22036_amd import binding
    from paper_2512_22036_amd.build import FASTCALL, build_fastcall, build_library
    if not os.path.exists(binding.library_path()):
        build_library()
    if not os.path.exists(FASTCALL):
        build_fastcall()
    fast = binding._bind_fastcall(binding.load_library())
    x, q, scale = torch.zeros((2, 16)), torch.zeros((2, 16)).to(FP8), torch.zeros((2, 1))
    assert fast.to_fp8(x, q, scale) is None and fast.to_fp8(x, q) is None and fast.to_fp8(None, q, scale) is None
    assert fast.from_fp8(q, scale, x) is None and fast.from_fp8(1, "a", x) is None
    ids, w = torch.zeros((2, 1), dtype=torch.int32), torch.zeros((2, 1))
    assert fast.moe_few(x.bfloat16(), ids, w, torch.zeros((1, 32, 16)).bfloat16(), torch.zeros((1, 16, 16)).bfloat16(), x, None, None, torch.zeros(4096)) is None
    assert fast.moe_few(*[None] * 9) is None and fast.moe_few() is None


@pytest.fixture(scope="module")
def f():
    import paper_2512_22036_amd as f
    from paper_2512_22036_amd import binding
    f.load_library()
    assert binding._fast is not None
    return f


def both(f, monkeypatch, go):
    from paper_2512_22036_amd import binding
    real, codes = binding._fast, []

    class Spy:   # the fast path took the calls
        def __getattr__(self, name):
            def call(*a):
                codes.append(getattr(real, name)(*a))
                return codes[-1]
            return call

    monkeypatch.setattr(binding, "_fast", Spy())
    one = go()
    monkeypatch.setattr(binding, "_fast", None)
    other = go()
    monkeypatch.setattr(binding, "_fast", real)
    assert codes and all(c == 0 for c in codes)
    for a, b in zip(one, other):
        assert torch.equal(a.view(torch.uint8), b.view(torch.uint8))


@pytest.mark.gpu
@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
@pytest.mark.parametrize("shape,scale_shape", [((5, 272), (5, 4)), ((0, 16), (0, 1)), ((3, 136, 144), (3, 2, 2))])
def test_both_ways(f, monkeypatch, shape, scale_shape, dtype):
    g = torch.Generator(device="cuda").manual_seed(3)
    x = torch.randn(shape, generator=g, device="cuda").to(dtype)

    def go():
        q, scale, back = torch.zeros(shape, device="cuda").to(FP8), torch.zeros(scale_shape, device="cuda"), torch.zeros_like(x)
        f.fusco_to_fp8(x, q, scale)
        f.fusco_from_fp8(q, scale, back)
        return q, scale, back

    both(f, monkeypatch, go)


@pytest.mark.gpu
@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
@pytest.mark.parametrize("eight", [False, True])
def test_few_both_ways(f, monkeypatch, eight, dtype):
    g = torch.Generator(device="cuda").manual_seed(4)
    N, k, E, H, I = 3, 2, 5, 144, 80
    x = torch.randn((N, H), generator=g, device="cuda").bfloat16()
    ids, w = torch.rand((N, E), generator=g, device="cuda").topk(k).indices.int().contiguous(), torch.rand((N, k), generator=g, device="cuda")
    w_in, w_out = (torch.randn(s, generator=g, device="cuda").mul_(0.1) for s in ((E, 2 * I, H), (E, H, I)))
    scales = {}
    if eight:
        w_in, w_out = w_in.to(FP8), w_out.to(FP8)
        scales = dict(w_in_scale=torch.rand((E, 2, 2), generator=g, device="cuda"), w_out_scale=torch.rand((E, 2, 1), generator=g, device="cuda"))
    else:
        w_in, w_out = w_in.bfloat16(), w_out.bfloat16()
    scratch = torch.empty(f.fusco_moe_few_scratch_bytes(N, k, I), dtype=torch.uint8, device="cuda")

    def go():
        out = torch.zeros((N, H), dtype=dtype, device="cuda")
        f.fusco_moe_few(x, ids, w, w_in, w_out, out, scratch=scratch, **scales)
        return [out]

    both(f, monkeypatch, go)
    for wrong in (dict(scratch=scratch[:-256]), dict(out=torch.zeros((N, H + 16), device="cuda")), dict(w=w.double()), dict(ids=ids.long())):
        a = dict(ids=ids, w=w, out=torch.zeros((N, H), dtype=dtype, device="cuda"), scratch=scratch)
        a.update(wrong)
        with pytest.raises(f.FuscoError):
            f.fusco_moe_few(x, a["ids"], a["w"], w_in, w_out, a["out"], scratch=a["scratch"], **scales)


@pytest.mark.gpu
def test_what_it_leaves(f):
    """Other types, views, strides and sizes: refused as without it."""
    x = torch.zeros((4, 32), device="cuda")
    q, scale = torch.zeros((4, 32), device="cuda").to(FP8), torch.zeros((4, 1), device="cuda")
    for args in ((x.half(), q, scale), (x.t().contiguous().t(), q, scale), (x, q.view(torch.uint8), scale), (x, q, scale.double()), (x, q, scale[:3]), (x[:, :24].contiguous(), q[:, :24].contiguous(), scale),
                 (x, q, scale.expand(4, 2)), (x.view(1, 4, 32), q, scale), (x.cpu(), q, scale)):
        with pytest.raises(f.FuscoError):
            f.fusco_to_fp8(*args)
    f.fusco_to_fp8(x, q, scale)
    stream = torch.cuda.Stream()
    stream.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(stream):
        f.fusco_to_fp8(x + 1, q, scale)
    torch.cuda.current_stream().wait_stream(stream)
    assert bool((q.float() * scale == 1).all())
