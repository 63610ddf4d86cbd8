"""Whose memory KV4Cache's workspaces are, on the host: torch's allocator is modelled (a pool of blocks per stream, a
freed block goes to the next request of its stream), the library's attention calls only note the workspace they get."""
import contextlib
import os
import sys
import types
import weakref

import pytest

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
LIB = os.path.join(ROOT, "paper_2607_15865_amd", "libw4layer.so")

if not os.path.exists(LIB):
    from paper_2607_15865_amd import build as _b
    _b.build()

from paper_2607_15865_amd import binding, synth  # noqa: E402

CFG = synth.replace(synth.CONFIGS["llama8b"], max_seq=4096)
MAIN, SIDE = 0x5000, 0x6000                  # stream handles


class Block:
    def __init__(self, torch, addr, nbytes, stream):
        self.addr, self.nbytes, self.stream = addr, nbytes, stream
        weakref.finalize(self, torch.free.setdefault(stream, []).append, (nbytes, addr))
        self.device = types.SimpleNamespace(index=0, type="cuda")

    def data_ptr(self):
        return self.addr

    def numel(self):
        return self.nbytes


class Stream:
    def __init__(self, handle, device=None):
        self.cuda_stream = handle


class FakeTorch(types.ModuleType):
    """What KV4Cache uses of torch."""
    uint8, bfloat16, int16, uint16, int32, float32 = "uint8", "bfloat16", "int16", "uint16", "int32", "float32"

    def __init__(self):
        super().__init__("torch")
        self.current, self.free, self.top, self.captured = 0, {}, 1 << 20, set()
        self.blocks = {}                     # address: stream
        self.cuda = types.SimpleNamespace(
            is_current_stream_capturing=lambda: self.current in self.captured,
            current_stream=lambda dev=None: Stream(self.current), default_stream=lambda dev=None: Stream(0),
            current_device=lambda: 0, stream=self.use, ExternalStream=Stream, Stream=Stream)
        self._C = types.SimpleNamespace(_cuda_getCurrentRawStream=lambda dev: self.current, _cuda_getDevice=lambda: 0)

    @contextlib.contextmanager
    def use(self, s):
        before, self.current = self.current, s.cuda_stream
        try:
            yield
        finally:
            self.current = before

    def empty(self, n, dtype=None, device=None):
        pool = self.free.setdefault(self.current, [])
        for i, (size, addr) in enumerate(pool):
            if size >= n:
                del pool[i]
                return Block(self, addr, size, self.current)
        self.top += 1 << 30
        self.blocks[self.top] = self.current
        return Block(self, self.top, n, self.current)


class Tensor:
    def __init__(self, shape, dtype, addr):
        self.shape, self.dtype, self.addr = shape, dtype, addr

    def dim(self):
        return len(self.shape)

    def get_device(self):
        return 0

    def is_contiguous(self):
        return True

    def data_ptr(self):
        return self.addr


@pytest.fixture
def fake(monkeypatch):
    torch = FakeTorch()
    monkeypatch.setitem(sys.modules, "torch", torch)
    calls = []                               # (workspace, stream) of every launch

    def attn(*args):
        ws, nbytes, stream = args[-3:]
        if nbytes < 1 << 16:
            return binding.W4_EWORKSPACE
        calls.append((ws, stream))
        return 0

    monkeypatch.setattr(binding._lib, "kv4_load", lambda: 0)
    monkeypatch.setattr(binding._lib, "kv4_attn_decode", attn)
    monkeypatch.setattr(binding._lib, "kv4_attn_prefill", attn)
    return types.SimpleNamespace(torch=torch, calls=calls, cache=binding.KV4Cache(CFG, 2))


def decode(c, stream=None):
    q, out, ctx = (Tensor((2, 32, 128), "bfloat16", a << 12) for a in (1, 2, 3))
    ctx.shape, ctx.dtype = (2,), "int32"
    c.attn_decode(q, ctx, 4000, out, stream=stream)


def prefill(c, stream=None):
    q, out = (Tensor((200, 32, 128), "bfloat16", a << 12) for a in (1, 2))
    c.attn_prefill(q, 3000, out, stream=stream)


@pytest.mark.parametrize("order", ["main first", "side first"])
@pytest.mark.parametrize("form", ["handle", "stream"])
def test_branches_of_a_capture_have_their_own(fake, order, form):
    """Two branches of a captured graph run at once: their calls may not share a workspace, in either order."""
    torch, c = fake.torch, fake.cache
    side = SIDE if form == "handle" else Stream(SIDE)
    torch.captured |= {MAIN, SIDE}
    with torch.use(Stream(MAIN)):
        steps = [lambda: decode(c), lambda: decode(c, side)]
        for step in steps if order == "main first" else reversed(steps):
            step()
        prefill(c)
        prefill(c, side)
    on = {s: {ws for ws, st in fake.calls if st == s} for s in (MAIN, SIDE)}
    assert len(fake.calls) == 4 and not on[MAIN] & on[SIDE]
    assert all(torch.blocks[ws] == st for ws, st in fake.calls)


@pytest.mark.parametrize("stream", [SIDE, 0])
def test_a_workspace_belongs_to_the_stream_that_uses_it(fake, stream):
    """A block that was just freed on the current stream may still be in use there: a call on another stream does not get
    it, neither at its first call nor when its workspace grows."""
    torch, c = fake.torch, fake.cache
    with torch.use(Stream(MAIN)):
        mine = torch.empty(1 << 28)
        addr = mine.data_ptr()
        del mine
        decode(c, stream)
        prefill(c, stream)
        decode(c, stream)
        assert len(fake.calls) == 3
        assert all(ws != addr and torch.blocks[ws] == st == stream for ws, st in fake.calls)
        decode(c)
    assert fake.calls[3] == (addr, MAIN)


def test_a_stream_keeps_its_workspace(fake):
    c = fake.cache
    for _ in range(3):
        decode(c)
        decode(c, SIDE)
    assert len(set(fake.calls)) == 2


def test_nothing_is_kept_of_captured_calls(fake):
    """Their workspaces belong to the graph: the cache holds on to none of them."""
    torch, c = fake.torch, fake.cache
    torch.captured |= {MAIN, SIDE}
    with torch.use(Stream(MAIN)):
        for _ in range(10):
            decode(c)
            decode(c, SIDE)
    assert len({ws for ws, _ in fake.calls}) == 2
    assert sum(len(torch.free[s]) for s in (MAIN, SIDE)) == 2


def test_capture_of_a_stream_that_is_not_current(fake):
    """The state that counts is that of the stream which the call runs on, whatever the current one does: a captured call
    does not take the workspace of the stream's eager calls, and an eager call beside a capture not one of the capture's."""
    torch, c = fake.torch, fake.cache
    decode(c, SIDE)
    eager = fake.calls[0][0]
    torch.captured.add(SIDE)
    decode(c, SIDE)
    prefill(c, SIDE)
    assert all(ws != eager and torch.blocks[ws] == SIDE for ws, _ in fake.calls[1:])
    torch.captured = {MAIN}
    with torch.use(Stream(MAIN)):
        decode(c, SIDE)
    assert fake.calls[3] == (eager, SIDE)
