"""Helpers of the GPU tests of embedding, layer norm and feed-forward block.  (Not collected by pytest.)

Tolerances count roundings: a result held in an element type is off by half a step, torch.finfo(t).eps / 2 relative to its
value; fp32 sums are off by at most one 2^-24 of the magnitudes' sum per addition in a chain, plus one for the product."""
import numpy as np
import torch

DTYPES = {"bf16": torch.bfloat16, "f32": torch.float32}
HALF = {"bf16": 2.0 ** -8, "f32": 2.0 ** -24}
TINY = 2.0 ** -126  # what a type's smallest normal numbers may lose


def rnd(rng, *shape, scale=1.0, shift=0.0, dtype="bf16"):
    """Random values that the element type holds exactly, as fp64."""
    x = torch.from_numpy(np.asarray(rng.standard_normal(shape) * scale + shift))
    return x.to(DTYPES[dtype]).double().numpy()


def hold(dtype):
    """Rounding to the element type (nearest, ties to even), on fp64 arrays."""
    return lambda x: torch.from_numpy(np.ascontiguousarray(x)).to(DTYPES[dtype]).double().numpy()


class Guarded:
    """Device tensors inside larger buffers whose edges must stay as they are: writes outside a tensor show.  `shift`: elements
    that a tensor starts behind a 16-byte boundary."""

    def __init__(self, dtype, shift=0):
        self.dt, self.shift, self.all = DTYPES[dtype], shift, []

    def empty(self, *shape, dtype=None):
        dt = dtype or self.dt
        n = int(np.prod(shape, dtype=np.int64))
        buf = torch.full((n + 256,), float("nan") if dt.is_floating_point else -7, dtype=dt, device="cuda")
        at = 64 + self.shift
        edge = torch.arange(1, 257, device="cuda", dtype=torch.float32)
        buf[:at] = edge[:at].to(dt)
        buf[at + n:] = edge[at:at + 256 - at].to(dt)
        self.all.append((buf, at, n, buf[:at].clone(), buf[at + n:].clone()))
        return buf[at:at + n].view(shape)

    def put(self, x, dtype=None):
        t = self.empty(*x.shape, dtype=dtype)
        t.copy_(torch.from_numpy(np.ascontiguousarray(x)))
        return t

    def check(self):
        torch.cuda.synchronize()
        for buf, at, n, lo, hi in self.all:
            assert torch.equal(buf[:at], lo) and torch.equal(buf[at + n:], hi), "written outside the tensor"


def np64(t):
    return t.detach().double().cpu().numpy()


def close(got, ref, tol, what):
    got = np64(got) if isinstance(got, torch.Tensor) else got
    assert got.shape == ref.shape, (what, got.shape, ref.shape)
    assert np.all(np.isfinite(got)), (what, "not finite")
    off = np.abs(got - ref) - tol
    if off.size:
        i = np.unravel_index(np.argmax(off), off.shape)
        assert off[i] <= 0, (what, i, got[i], ref[i], "off by %g, allowed %g" % (abs(got[i] - ref[i]), np.broadcast_to(tol, off.shape)[i]))


def same(got, ref, what):
    got = np64(got)
    assert np.array_equal(got, ref), (what, np.argwhere(got != ref)[:5], got[got != ref][:5], ref[got != ref][:5])
