"""The scratch that the norms' gradients make when none is given belongs to the stream that the call is launched on: the allocator gives a
freed block to the next allocation on the block's own stream, and that one alone waits for the kernels that still use it."""
import contextlib

import pytest
import torch


class Handle:
    def __init__(self, cuda_stream):
        self.cuda_stream = cuda_stream


class Device:
    """What the binding looks at of a contiguous fp32 tensor on a device."""
    is_cuda, dtype, device = True, torch.float32, "cuda"

    def __init__(self, *shape):
        self.shape = shape

    def dim(self):
        return len(self.shape)

    def is_contiguous(self):
        return True

    def data_ptr(self):
        return 1 << 28

    def numel(self):
        return 4096

    def element_size(self):
        return 1


class Library:
    """Takes every call and remembers which stream it was given."""

    def __init__(self):
        self.launched = []

    def fusco_norm_scratch_bytes(self, N, H):
        return 4096

    def fusco_norm_before_backward(self, *args):
        self.launched.append(args[-1])
        return 0

    fusco_norm_after_backward = fusco_norm_before_backward


@pytest.fixture
def calls(monkeypatch):
    from paper_2512_22036_amd import binding
    lib, current, made = Library(), [], []

    @contextlib.contextmanager
    def stream(s):
        current.append(s.cuda_stream)
        yield
        current.pop()

    def empty(*args, **kw):
        made.append(current[-1] if current else None)
        return Device(4096)

    monkeypatch.setattr(binding, "load_library", lambda: lib)
    monkeypatch.setattr(binding, "_stream", lambda s: 5 if s is None else s.cuda_stream if hasattr(s, "cuda_stream") else int(s))
    monkeypatch.setattr(torch.cuda, "stream", stream)
    monkeypatch.setattr(torch.cuda, "ExternalStream", lambda handle, device=None: Handle(handle))
    monkeypatch.setattr(torch, "empty", empty)
    rows, vec = Device(4, 64), Device(64)
    return lib, made, {"before": lambda **kw: binding.fusco_norm_before_backward(rows, rows, vec, rows, vec, **kw),
                       "after": lambda **kw: binding.fusco_norm_after_backward(rows, rows, vec, rows, rows, vec, **kw)}


@pytest.mark.parametrize("which", ["before", "after"])
@pytest.mark.parametrize("stream,handle", [(Handle(77), 77), (77, 77), (0, 0)])
def test_scratch_is_made_on_the_stream_of_the_launch(calls, which, stream, handle):
    lib, made, call = calls
    call[which](stream=stream)
    assert lib.launched == [handle] and made == [handle]


@pytest.mark.parametrize("which", ["before", "after"])
def test_current_stream_and_scratch_of_the_caller(calls, which):
    lib, made, call = calls
    call[which]()
    assert lib.launched == [5] and made == [None]          # both by the current stream
    call[which](stream=77, scratch=Device(4096))
    assert lib.launched == [5, 77] and made == [None]      # nothing made


@pytest.mark.gpu
@pytest.mark.parametrize("raw", [False, True])
@pytest.mark.parametrize("which", ["before", "after"])
def test_blocks_of_the_current_stream_are_left_alone(which, raw):
    """Calls on another stream while the current one allocates and overwrites blocks of the scratch's size."""
    import paper_2512_22036_amd as f
    N, H = 2048, 512
    gen = torch.Generator(device="cuda").manual_seed(11)
    x, dout = (torch.randn((N, H), generator=gen, device="cuda") for _ in range(2))
    gain = torch.randn(H, generator=gen, device="cuda")

    def call(res, **kw):
        dx, dy, dgain = res
        if which == "before":
            f.fusco_norm_before_backward(dout, x, gain, dx, dgain, **kw)
        else:
            f.fusco_norm_after_backward(dout, x, gain, dx, dy, dgain, **kw)

    def results():
        return torch.zeros_like(x), torch.zeros_like(x), torch.zeros(H, device="cuda")

    want, got, held = results(), [results() for _ in range(8)], []
    call(want)
    side = torch.cuda.Stream()
    slow = torch.randn((2048, 2048), generator=gen, device="cuda")
    torch.cuda.synchronize()
    for res in got:
        with torch.cuda.stream(side):                      # what the call has to wait for
            for _ in range(4):
                slow = slow @ slow * 1e-3
        call(res, stream=side.cuda_stream if raw else side)
        block = torch.empty(f.fusco_norm_scratch_bytes(N, H), dtype=torch.uint8, device="cuda")
        held.append(block.fill_(0x5a))
    torch.cuda.synchronize()
    assert all(torch.equal(a, b) for res in got for a, b in zip(res, want))
    assert all(bool((block == 0x5a).all()) for block in held)
