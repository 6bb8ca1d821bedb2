"""Whose memory a call's own tensors are: made on the stream that its kernels run on, and, where they are returned, known to the stream
that is current.  Memory of the current stream's pool may still be in use there by work queued before it was freed.  (CPU: the binding
runs on a torch and a library that write down what they are asked for.)"""
import contextlib

import pytest
import torch

from paper_2410_20305_amd import binding, layer

CURRENT, SIDE = 0x100, 0x200


class Stream:
    def __init__(self, handle):
        self.cuda_stream = handle


class Tensor:
    """What the binding asks a device tensor."""
    is_cuda, device = True, torch.device("cuda", 0)
    _next = 1 << 20

    def __init__(self, shape, dtype, made_on):
        self.shape, self.dtype, self.made_on, self.seen_by = torch.Size(shape), dtype, made_on, set()
        self.ptr, Tensor._next = Tensor._next, Tensor._next + (1 << 20)

    def dim(self):
        return len(self.shape)

    def get_device(self):
        return 0

    def is_contiguous(self):
        return True

    def data_ptr(self):
        return self.ptr

    def numel(self):
        return self.shape.numel()

    def element_size(self):
        return self.dtype.itemsize

    def record_stream(self, stream):
        self.seen_by.add(stream.cuda_stream)


class Torch:
    """Of torch, what the binding uses to make tensors."""
    bfloat16, float32, int32, uint8 = torch.bfloat16, torch.float32, torch.int32, torch.uint8

    def __init__(self):
        self.now, self.made = CURRENT, []
        self.cuda = self._C = self

    def _cuda_getDevice(self):
        return 0

    def _cuda_getCurrentRawStream(self, device):
        return self.now

    def current_stream(self, device=None):
        return Stream(self.now)

    def ExternalStream(self, handle, device=None):
        return Stream(handle)

    @contextlib.contextmanager
    def stream(self, s):
        before, self.now = self.now, s.cuda_stream
        yield
        self.now = before

    def empty(self, shape, dtype, device):
        self.made.append(Tensor((shape,) if isinstance(shape, int) else shape, dtype, self.now))
        return self.made[-1]

    zeros = empty

    def empty_like(self, t):
        return self.empty(t.shape, t.dtype, t.device)


class Library:
    """Every call succeeds; workspaces are of 64 bytes; the last argument of a call is its stream."""

    def __init__(self):
        self.streams = []

    def __getattr__(self, name):
        def call(*args):
            if name.endswith("workspace_bytes"):
                return 64
            self.streams.append(args[-1])
            return 0
        return call


class Meta:
    handle, total_tokens, n_responses = 1, 6, 4


T, H, N, V, BF, F32 = 6, 16, 24, 8, torch.bfloat16, torch.float32


def _t(*shape, dtype=BF):
    return Tensor(shape, dtype, CURRENT)


def _layer():
    a = layer.Layer.__new__(layer.Layer)
    a._h, a.hidden, a.Hq, a.Hkv, a.d = None, H, 2, 1, 8  # no handle: nothing to free
    return a


def _layer_weights():
    return _t(T, H), _t(16, H), _t(8, H), _t(8, H), _t(H, 16)


def _ffn():
    return _t(T, H), _t(N, H), _t(N, H), _t(H, N)


def _kept():
    return _t(T, N, dtype=F32), _t(T, N, dtype=F32), _t(T, N)


def _q():
    return _t(T, 2, 8), _t(T, 1, 8), _t(T, 1, 8)


def _lse():
    return _t(2, T, dtype=F32)


def _ids():
    return _t(T, dtype=torch.int32)


CALLS = {
    "fwd": lambda s: binding.psattn_fwd(Meta, *_q(), 1.0, stream=s),
    "bwd": lambda s: binding.psattn_bwd(Meta, *_q(), _t(T, 2, 8), _t(T, 2, 8), _lse(), 1.0, stream=s),
    "fwd_rope": lambda s: binding.psattn_fwd_rope(Meta, Meta, *_q(), 1.0, stream=s),
    "bwd_rope": lambda s: binding.psattn_bwd_rope(Meta, Meta, *_q(), _t(T, 2, 8), _t(T, 2, 8), _lse(), 1.0, stream=s),
    "logprob_fwd": lambda s: binding.psattn_logprob_fwd(Meta, _t(T, V), _ids(), stream=s),
    "logprob_bwd": lambda s: binding.psattn_logprob_bwd(Meta, _t(T, V), _ids(), _t(T, dtype=F32), _t(4, dtype=F32), stream=s),
    "dpo_loss": lambda s: binding.psattn_dpo_loss(_t(4, dtype=F32), _t(4, dtype=F32), 0.1, stream=s),
    "layer_fwd": lambda s: _layer().forward(Meta, Meta, 1.0, *_layer_weights(), _t(64), stream=s),
    "layer_bwd": lambda s: _layer().backward(Meta, Meta, 1.0, *_layer_weights(), _t(T, H), _t(64), stream=s),
    "embed_fwd": lambda s: binding.psattn_embed_fwd(_ids(), _t(V, H), stream=s),
    "embed_bwd": lambda s: binding.psattn_embed_bwd(_ids(), _t(T, H), V, stream=s),
    "layernorm_fwd": lambda s: binding.psattn_layernorm_fwd(_t(T, H), _t(H), residual=_t(T, H), stream=s),
    "layernorm_bwd": lambda s: binding.psattn_layernorm_bwd(_t(T, H), _t(H), _t(T, dtype=F32), _t(T, dtype=F32), _t(T, H), stream=s),
    "ffn_fwd": lambda s: binding.psattn_ffn_fwd(*_ffn(), stream=s),
    "ffn_fwd_alone": lambda s: binding.psattn_ffn_fwd(*_ffn(), keep=False, stream=s),
    "ffn_bwd": lambda s: binding.psattn_ffn_bwd(*_ffn(), _kept(), _t(T, H), stream=s),
}


def _tensors(x):
    if isinstance(x, Tensor):
        return [x]
    return [t for y in x for t in _tensors(y)] if isinstance(x, (tuple, list)) else []


@pytest.fixture
def recorded(monkeypatch):
    t, lib = Torch(), Library()
    monkeypatch.setattr(binding, "_TORCH", t)
    monkeypatch.setattr(binding, "_LIB", lib)
    monkeypatch.setattr(layer, "_LIB", lib)
    return t, lib


@pytest.mark.parametrize("as_handle", [False, True])
@pytest.mark.parametrize("name", sorted(CALLS))
def test_made_on_the_stream_that_uses_it(recorded, name, as_handle):
    t, lib = recorded
    out = CALLS[name](SIDE if as_handle else Stream(SIDE))
    assert lib.streams and set(lib.streams) == {SIDE}
    assert t.made and all(x.made_on == SIDE for x in t.made), [(x.shape, hex(x.made_on)) for x in t.made]
    mine = [x for x in _tensors(out) if x in t.made]
    assert mine and all(CURRENT in x.seen_by for x in mine), "returned, and freed without a look at the current stream"


@pytest.mark.parametrize("given", [None, CURRENT])
@pytest.mark.parametrize("name", sorted(CALLS))
def test_nothing_to_record_on_the_current_stream(recorded, name, given):
    t, lib = recorded
    CALLS[name](given)
    assert set(lib.streams) == {CURRENT}
    assert all(x.made_on == CURRENT and not x.seen_by for x in t.made)
