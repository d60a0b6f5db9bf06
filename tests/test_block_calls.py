"""The calls around the shuffle that go through csrc/fastcall.cpp: without a GPU it leaves everything to ctypes; with one both ways give
the same bytes, and what it cannot handle is refused or accepted as ctypes does."""
import pytest
import torch


def test_leaves_everything_else_to_the_other_path():
    import os
    from paper_2512_22036_amd import binding
    from paper_2512_22036_amd.build import FASTCALL, build_fastcall, build_library
    if not os.path.exists(binding.library_path()):
        build_library()
    if not os.path.exists(FASTCALL):
        build_fastcall()
    fast = binding._bind_fastcall(binding.load_library())

    class Plain:
        c, scratch, N, k = binding._CLayout(), torch.zeros(4), 2, 2

    rows, ids, vec = torch.zeros((2, 8)), torch.zeros((2, 2), dtype=torch.int32), torch.zeros(8)
    assert fast.route(rows, ids, torch.zeros((2, 2)), None, 0, 1, 1, 1, True, 1.0) is None
    assert fast.route(rows, ids) is None and fast.route(*[None] * 10) is None
    assert fast.norm_before(rows, vec, rows, 1e-6) is None and fast.norm_before(1, 2, 3, "x") is None
    assert fast.norm_after(rows, rows, vec, rows, None, 1.0, None, None, 1e-6, None) is None
    assert fast.experts_gated(Plain(), rows, torch.zeros((1, 2, 8)), rows, None) is None
    assert fast.experts_linear(None, rows, torch.zeros((1, 2, 8)), rows) is None


@pytest.fixture(scope="module")
def f():
    import paper_2512_22036_amd as f
    from paper_2512_22036_amd import binding
    f.load_library()
    assert binding._fast is not None
    return f


def calls(f):
    g = torch.Generator(device="cuda").manual_seed(1)
    n = lambda *s, t=torch.float32: torch.randn(s, generator=g, device="cuda").to(t)
    N, E, k, H, I = 23, 16, 4, 64, 32
    B = torch.bfloat16
    L = f.Layout(N, k, E, 1)
    wide, bias = n(N, 40), n(E)
    idx, w = torch.zeros((N, k), dtype=torch.int32, device="cuda"), torch.zeros((N, k), device="cuda")
    f.fusco_route(wide[:, :E], idx, w)
    f.fusco_plan(L, idx)
    r, y, gain, ng, channel, token = n(N, H), n(N, H, t=B), n(H), n(H), n(H), n(N)
    x, w_in, w_out = n(N * k, H, t=B), n(E, 2 * I, H, t=B), n(E, H, I, t=B)
    empty = lambda *s, t=torch.float32: torch.zeros(s, dtype=t, device="cuda")

    def route(**kw):
        def go(**s):
            a, b = torch.zeros_like(idx), torch.zeros_like(w)
            f.fusco_route(wide[:, 3:3 + E], a, b, **kw, **s)
            return [a, b]
        return go

    def norm_before(**s):
        out = empty(N, H, t=B)
        f.fusco_norm_before(r, gain, out, **s)
        return [out]

    def norm_after(**kw):
        def go(**s):
            out, nxt = empty(N, H), empty(N, H, t=B)
            more = dict(next_gain=ng, next_out=nxt) if kw.get("scale") != 1 else {}
            f.fusco_norm_after(r, y, gain, out, **kw, **more, **s)
            return [out, nxt]
        return go

    def gated(keep):
        def go(**s):
            h, pre = empty(N * k, I, t=B), empty(N * k, 2 * I, t=B)
            f.fusco_experts_gated(L, x, w_in, h, pre if keep else None, **s)
            return [h, pre]
        return go

    def linear(**s):
        out = empty(N * k, H, t=B)
        f.fusco_experts_linear(L, x[:, :I].contiguous(), w_out, out, **s)
        return [out]

    return {"route": route(), "route all": route(bias=bias, score=f.SCORE_SIGMOID, groups=4, keep_groups=2, group_best=2, renorm=False, scale=2), "norm before": norm_before,
            "norm after": norm_after(), "norm channel": norm_after(gate=channel, scale=0.5), "norm token": norm_after(gate=token, scale=1), "norm kind": norm_after(gate=channel, gate_kind=f.GATE_CHANNEL),
            "gated": gated(False), "gated kept": gated(True), "linear": linear}


NAMES = ["route", "route all", "norm before", "norm after", "norm channel", "norm token", "norm kind", "gated", "gated kept", "linear"]


@pytest.mark.gpu
@pytest.mark.parametrize("name", NAMES)
def test_same_as_ctypes(f, name, monkeypatch):
    from paper_2512_22036_amd import binding
    call = calls(f)[name]
    seen = []

    class Recorder:
        def __getattr__(self, what):
            def go(*args):
                rc = getattr(module, what)(*args)
                seen.append(rc)
                return rc
            return go

    module = binding._fast
    monkeypatch.setattr(binding, "_fast", Recorder())
    quick = call()
    assert seen and seen[-1] == 0                 # made there, not left to ctypes
    asked = len(seen)
    other = call(stream=torch.cuda.current_stream())
    assert len(seen) == asked                     # a stream argument goes the other way
    assert all(torch.equal(a, b) for a, b in zip(quick, other))


@pytest.mark.gpu
def test_current_stream(f):
    side = torch.cuda.Stream()
    for name in NAMES:
        call = calls(f)[name]
        want = call()
        torch.cuda.synchronize()
        with torch.cuda.stream(side):
            got = call()
        side.synchronize()
        assert all(torch.equal(a, b) for a, b in zip(want, got)), name


@pytest.mark.gpu
def test_graph(f):
    """All of them captured and replayed, with eager work in between."""
    for name in NAMES:
        call = calls(f)[name]
        want = [t.clone() for t in call()]
        torch.cuda.synchronize()
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph):
            got = call()
        for _ in range(3):
            for t in got:
                t.zero_()
            graph.replay()
            torch.cuda.synchronize()
            assert all(torch.equal(a, b) for a, b in zip(want, got)), name
