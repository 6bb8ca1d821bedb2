"""ctypes marshalling for libpsattn.so.  Names mirror include/psattn.h."""
from __future__ import annotations

import ctypes as C
import os

import numpy as np

GRID_FWD, GRID_BWD = 0, 1
TILE_SKIPPED, TILE_PARTIAL, TILE_FULL = 0, 1, 2
F32, BF16 = 0, 1

_HERE = os.path.dirname(os.path.abspath(__file__))
_LIB = None

EXPORTS = [
    "psattn_build_meta", "psattn_build_meta_host", "psattn_free_meta", "psattn_meta_tiles",
    "psattn_meta_copy_csr", "psattn_meta_copy_tok_desc", "psattn_meta_copy_key_desc",
    "psattn_meta_allowed_pairs", "psattn_meta_device_bytes", "psattn_fwd", "psattn_bwd", "psattn_bwd_workspace_bytes",
    "psattn_kernel_name", "psattn_strerror", "psattn_profile_enable", "psattn_profile_read",
    "psattn_free_meta_async", "psattn_trim_pool", "psattn_uses_mfma",
    "psattn_bwd_static", "psattn_bwd_static_max_rows", "psattn_probe_dq_atomics", "psattn_probe_mfma_peak",
    "psattn_pack_ffd", "psattn_build_meta_multi", "psattn_build_meta_multi_host",
    "psattn_rope_create", "psattn_rope_free", "psattn_rope_k", "psattn_fwd_rope", "psattn_bwd_rope",
    "psattn_meta_copy_positions",
    "psattn_logprob_plan", "psattn_logprob_plan_free", "psattn_logprob_plan_info", "psattn_logprob_fwd",
    "psattn_logprob_bwd", "psattn_dpo_loss",
    "psattn_embed_fwd", "psattn_embed_bwd", "psattn_embed_bwd_workspace_bytes",
    "psattn_layernorm_fwd", "psattn_layernorm_bwd", "psattn_layernorm_bwd_workspace_bytes",
    "psattn_ffn_fwd", "psattn_ffn_bwd", "psattn_ffn_fwd_workspace_bytes", "psattn_ffn_bwd_workspace_bytes",
    "psattn_ffn_fwd_unaligned_workspace_bytes", "psattn_ffn_bwd_unaligned_workspace_bytes",
    "psattn_rope_frequencies", "psattn_rope_create_layout", "psattn_rope_apply",
    "psattn_head_logprob_fwd", "psattn_head_logprob_bwd", "psattn_head_logprob_fwd_workspace_bytes",
    "psattn_head_logprob_bwd_workspace_bytes",
    "psattn_gatednorm_fwd", "psattn_gatednorm_bwd", "psattn_gatednorm_bwd_workspace_bytes",
]

ACT_SILU, ACT_GELU = 0, 1
_ACTS = {"silu": ACT_SILU, "gelu": ACT_GELU}
_ROPE_LAYOUTS = {"half": 0, "interleaved": 1}
_ROPE_SCALINGS = {"none": 0, "linear": 1, "base": 2, "parts": 3}


class PsattnError(RuntimeError):
    def __init__(self, status, what):
        self.status = status
        super().__init__("%s failed: %s (%d)" % (what, _strerror(status), status))


def lib_path() -> str:
    # PSATTN_LIB: another build of the same library, for A/B measurements of kernel variants
    return os.environ.get("PSATTN_LIB") or os.path.join(_HERE, "libpsattn.so")


def load_library():
    """Load libpsattn.so (built by paper_2410_20305_amd/build.py).  Raises if absent."""
    global _LIB
    if _LIB is not None:
        return _LIB
    path = lib_path()
    if not os.path.exists(path):
        raise ImportError("libpsattn.so not built: run `python -m paper_2410_20305_amd.build` "
                          "(or __graft_entry__.build()); there is no fallback path")
    lib = C.CDLL(path)
    i32, i64, vp, f32 = C.c_int32, C.c_int64, C.c_void_p, C.c_float
    pi32 = C.POINTER(C.c_int32)
    lib.psattn_build_meta.argtypes = [i32, vp, vp, vp, vp, i32, i32, i32, i32, i32, vp, C.POINTER(vp)]
    lib.psattn_build_meta_host.argtypes = [i32, vp, vp, vp, vp, i32, i32, i32, i32, i32, C.POINTER(vp)]
    lib.psattn_build_meta_multi.argtypes = [i32, vp, vp, vp, vp, i32, i32, i32, i32, i32, vp, C.POINTER(vp)]
    lib.psattn_build_meta_multi_host.argtypes = [i32, vp, vp, vp, vp, i32, i32, i32, i32, i32, C.POINTER(vp)]
    lib.psattn_rope_create.argtypes = [i32, f32, i32, vp, C.POINTER(vp)]
    lib.psattn_rope_free.argtypes = [vp]
    lib.psattn_rope_k.argtypes = [vp, vp, i32, i32, i32, vp, vp, vp]
    lib.psattn_fwd_rope.argtypes = [vp, vp, i32, i32, i32, i32, f32, vp, vp, vp, vp, vp, vp, vp, vp]
    lib.psattn_bwd_rope.argtypes = [vp, vp, i32, i32, i32, i32, f32, vp, vp, vp, vp, vp, vp, vp, vp, vp, vp,
                                    C.c_size_t, vp]
    lib.psattn_meta_copy_positions.argtypes = [vp, vp, pi32]
    lib.psattn_logprob_plan.argtypes = [i32, vp, vp, vp, vp, i32, vp, C.POINTER(vp)]
    lib.psattn_logprob_plan_free.argtypes = [vp]
    lib.psattn_logprob_plan_info.argtypes = [vp, pi32, pi32, C.POINTER(i64)]
    lib.psattn_logprob_fwd.argtypes = [vp, i32, i32, vp, vp, vp, vp, vp]
    lib.psattn_logprob_bwd.argtypes = [vp, i32, i32, vp, vp, vp, vp, vp, vp]
    lib.psattn_dpo_loss.argtypes = [i32, f32, vp, vp, vp, vp, vp]
    f64 = C.c_double
    lib.psattn_rope_frequencies.argtypes = [i32, f64, i32, f64, f64, f64, f64, vp]
    lib.psattn_rope_create_layout.argtypes = [i32, i32, i32, vp, f64, i32, vp, C.POINTER(vp)]
    lib.psattn_rope_apply.argtypes = [vp, i32, i32, i32, vp, vp, i32, vp, i64, vp, i64, i32, vp, i64, vp, i64, vp]
    lib.psattn_head_logprob_fwd.argtypes = [vp, i32, i32, i32] + [vp] * 6 + [C.c_size_t, vp]
    lib.psattn_head_logprob_bwd.argtypes = [vp, i32, i32, i32] + [vp] * 8 + [C.c_size_t, vp]
    lib.psattn_gatednorm_fwd.argtypes = [i32, i32, i32, f32, f32, vp, vp, vp, vp, i32] + [vp] * 6
    lib.psattn_gatednorm_bwd.argtypes = [i32, i32, i32, f32, vp, vp, vp, i32] + [vp] * 12 + [C.c_size_t, vp]
    lib.psattn_gatednorm_bwd_workspace_bytes.argtypes = [i32, i32]
    lib.psattn_gatednorm_bwd_workspace_bytes.restype = C.c_size_t
    for name in ("psattn_head_logprob_fwd_workspace_bytes", "psattn_head_logprob_bwd_workspace_bytes"):
        getattr(lib, name).argtypes = [vp, i32, i32, i32]
        getattr(lib, name).restype = C.c_size_t
    lib.psattn_embed_fwd.argtypes = [i32, i32, i32, i32, f32, vp, vp, vp, vp]
    lib.psattn_embed_bwd.argtypes = [i32, i32, i32, i32, f32, vp, vp, vp, vp, C.c_size_t, vp]
    lib.psattn_embed_bwd_workspace_bytes.argtypes = [i32, i32, i32, i32]
    lib.psattn_layernorm_fwd.argtypes = [i32, i32, i32, f32] + [vp] * 9
    lib.psattn_layernorm_bwd.argtypes = [i32, i32, i32] + [vp] * 10 + [C.c_size_t, vp]
    lib.psattn_layernorm_bwd_workspace_bytes.argtypes = [i32, i32]
    lib.psattn_ffn_fwd.argtypes = [i32] * 5 + [vp] * 9 + [C.c_size_t, vp]
    lib.psattn_ffn_bwd.argtypes = [i32] * 5 + [vp] * 13 + [C.c_size_t, vp]
    ffn_bytes = ("psattn_ffn_fwd_workspace_bytes", "psattn_ffn_bwd_workspace_bytes", "psattn_ffn_fwd_unaligned_workspace_bytes",
                 "psattn_ffn_bwd_unaligned_workspace_bytes")
    for name in ffn_bytes:
        getattr(lib, name).argtypes = [i32] * 4
    for name in ("psattn_embed_bwd_workspace_bytes", "psattn_layernorm_bwd_workspace_bytes", *ffn_bytes):
        getattr(lib, name).restype = C.c_size_t
    lib.psattn_free_meta.argtypes = [vp]
    lib.psattn_free_meta_async.argtypes = [vp, vp]
    lib.psattn_trim_pool.argtypes = []
    lib.psattn_uses_mfma.argtypes = [vp, i32, i32, f32, i32]
    lib.psattn_meta_tiles.argtypes = [vp, i32, pi32, pi32, pi32, pi32, C.POINTER(i64)]
    lib.psattn_meta_copy_csr.argtypes = [vp, i32, vp, vp, vp]
    lib.psattn_meta_copy_tok_desc.argtypes = [vp, vp]
    lib.psattn_meta_copy_key_desc.argtypes = [vp, vp]
    lib.psattn_meta_allowed_pairs.argtypes = [vp, C.POINTER(i64)]
    lib.psattn_meta_device_bytes.argtypes = [vp, C.POINTER(C.c_size_t)]
    lib.psattn_fwd.argtypes = [vp, i32, i32, i32, i32, f32, vp, vp, vp, vp, vp, vp]
    lib.psattn_bwd.argtypes = [vp, i32, i32, i32, i32, f32, vp, vp, vp, vp, vp, vp, vp, vp, vp, vp,
                               C.c_size_t, vp]
    lib.psattn_bwd_static.argtypes = [vp, i32, i32, i32, i32, f32, vp, vp, vp, vp, vp, vp, vp, vp, vp, vp]
    lib.psattn_bwd_static_max_rows.argtypes = []
    lib.psattn_bwd_static_max_rows.restype = C.c_size_t
    lib.psattn_probe_dq_atomics.argtypes = [vp, i32, i32, vp, i32, vp]
    lib.psattn_probe_mfma_peak.argtypes = [i32, i32, i32, vp, vp]
    lib.psattn_pack_ffd.argtypes = [i32, vp, vp, vp, i32, i32, vp, vp, pi32, C.POINTER(i64)]
    lib.psattn_bwd_workspace_bytes.argtypes = [vp, i32, i32, i32]
    lib.psattn_bwd_workspace_bytes.restype = C.c_size_t
    lib.psattn_kernel_name.argtypes = [i32, i32]
    lib.psattn_kernel_name.restype = C.c_char_p
    lib.psattn_profile_enable.argtypes = [i32]
    lib.psattn_profile_read.argtypes = [vp, vp]
    lib.psattn_strerror.argtypes = [C.c_int]
    lib.psattn_strerror.restype = C.c_char_p
    for name in EXPORTS:
        fn = getattr(lib, name)
        if fn.restype is C.c_int:
            fn.restype = C.c_int
    _LIB = lib
    return lib


def _strerror(status: int) -> str:
    try:
        return load_library().psattn_strerror(int(status)).decode()
    except Exception:
        return "status"


def _check(status, what):
    if status != 0:
        raise PsattnError(status, what)


# The calls below are a few microseconds each, and so are the smallest kernels: the marshalling keeps to what it needs
# (no stream objects, no ctypes wrappers of arrays, no modules looked up again).
_INT32 = np.dtype(np.int32)
_TORCH = None


def _torch():
    """torch, imported on first use: the host-only functions work without it."""
    global _TORCH
    if _TORCH is None:
        import torch
        _TORCH = torch
    return _TORCH


def _i32(x):
    if type(x) is np.ndarray and x.dtype == _INT32 and x.flags.c_contiguous:
        return x
    return np.ascontiguousarray(np.asarray(x, dtype=np.int32))


def _addr(x):
    """Address of a NumPy array (x.ctypes.data builds a ctypes view first)."""
    return x.__array_interface__["data"][0]


def _stream_ptr(stream):
    if stream is None:
        torch = _TORCH or _torch()
        try:  # the current stream's handle without a Stream object around it (0.2 us instead of 2.9)
            return torch._C._cuda_getCurrentRawStream(torch._C._cuda_getDevice())
        except (AttributeError, RuntimeError):  # not initialised yet, or a torch without these
            return torch.cuda.current_stream().cuda_stream
    if isinstance(stream, int):
        return stream
    return stream.cuda_stream


# torch hands a freed block out again to the stream that was current when the block was first taken, in that stream's order.  What a
# call makes for itself has to be made on the stream that its kernels run on: memory of another stream may still be in use by
# work queued there before it was freed.
def _elsewhere(call, args):
    """`call` with the arguments `args` (locals() at its start) on args["stream"], which is the current stream meanwhile.  Returned
    tensors that the call has made are both streams': freed, they are handed out again when the work queued on either by then is done."""
    torch = _TORCH or _torch()
    stream, args["stream"] = args["stream"], None
    if _stream_ptr(stream) == _stream_ptr(None):
        return call(**args)
    here = torch.cuda.current_stream()
    with torch.cuda.stream(torch.cuda.ExternalStream(stream) if isinstance(stream, int) else stream):
        out = call(**args)
    given = {id(x) for a in args.values() for x in (a if isinstance(a, (tuple, list)) else (a,))}

    def record(x):
        if isinstance(x, (tuple, list)):
            for y in x:
                record(y)
        elif x is not None and id(x) not in given:
            x.record_stream(here)

    record(out)
    return out


class Meta:
    """Owner of a psattn_meta handle."""

    def __init__(self, handle, total_tokens, on_device):
        self._h = handle
        self.total_tokens = int(total_tokens)
        self.on_device = on_device

    @property
    def handle(self):
        if self._h is None:
            raise ValueError("meta already freed")
        return self._h

    def free(self):
        if self._h is not None:
            lib = load_library()
            _check(lib.psattn_free_meta(self._h), "psattn_free_meta")
            self._h = None

    def free_async(self, stream=None):
        """Stream-ordered release: the buffers are reused only after the work enqueued so
        far on `stream` (default: torch's current stream) has finished."""
        if self._h is not None:
            lib = load_library()
            _check(lib.psattn_free_meta_async(self._h, _stream_ptr(stream)), "psattn_free_meta_async")
            self._h = None

    def uses_mfma(self, dtype_code, head_dim, scale, backward=False) -> bool:
        st = load_library().psattn_uses_mfma(self.handle, int(dtype_code), int(head_dim), float(scale),
                                             1 if backward else 0)
        if st < 0:
            raise PsattnError(st, "psattn_uses_mfma")
        return bool(st)

    def __del__(self):
        try:
            self.free()
        except Exception:
            pass

    def tiles(self, grid=GRID_FWD):
        lib = load_library()
        tq, tk, nq, nk, ne = C.c_int32(), C.c_int32(), C.c_int32(), C.c_int32(), C.c_int64()
        _check(lib.psattn_meta_tiles(self.handle, grid, C.byref(tq), C.byref(tk), C.byref(nq), C.byref(nk),
                                     C.byref(ne)), "psattn_meta_tiles")
        return dict(tile_q=tq.value, tile_k=tk.value, n_q_tiles=nq.value, n_k_tiles=nk.value,
                    n_entries=ne.value)

    def csr(self, grid=GRID_FWD):
        lib = load_library()
        t = self.tiles(grid)
        n_rows = t["n_q_tiles"] if grid == GRID_FWD else t["n_k_tiles"]
        row_ptr = np.zeros(n_rows + 1, dtype=np.int32)
        idx = np.zeros(max(1, t["n_entries"]), dtype=np.int32)
        cls = np.zeros(max(1, t["n_entries"]), dtype=np.uint8)
        _check(lib.psattn_meta_copy_csr(self.handle, grid, row_ptr.ctypes.data, idx.ctypes.data,
                                        cls.ctypes.data), "psattn_meta_copy_csr")
        return row_ptr, idx[:t["n_entries"]], cls[:t["n_entries"]]

    def tok_desc(self):
        lib = load_library()
        out = np.zeros((max(1, self.total_tokens), 3), dtype=np.int32)
        _check(lib.psattn_meta_copy_tok_desc(self.handle, out.ctypes.data), "psattn_meta_copy_tok_desc")
        return out[:self.total_tokens]

    def key_desc(self):
        lib = load_library()
        out = np.zeros(max(1, self.total_tokens), dtype=np.int32)
        _check(lib.psattn_meta_copy_key_desc(self.handle, out.ctypes.data), "psattn_meta_copy_key_desc")
        return out[:self.total_tokens]

    def positions(self):
        """(position id of every token, number of positions needed)."""
        lib = load_library()
        out = np.zeros(max(1, self.total_tokens), dtype=np.int32)
        n = C.c_int32()
        _check(lib.psattn_meta_copy_positions(self.handle, out.ctypes.data, C.byref(n)), "psattn_meta_copy_positions")
        return out[:self.total_tokens], n.value

    def device_bytes(self) -> int:
        """Device memory that the mask takes up; 0: it travels with the kernels' arguments."""
        n = C.c_size_t()
        _check(load_library().psattn_meta_device_bytes(self.handle, C.byref(n)), "psattn_meta_device_bytes")
        return n.value

    def allowed_pairs(self):
        lib = load_library()
        n = C.c_int64()
        _check(lib.psattn_meta_allowed_pairs(self.handle, C.byref(n)), "psattn_meta_allowed_pairs")
        return n.value


def psattn_build_meta(offset, prefix_len, chosen_len, rejected_len, total_tokens, tile_q=0, tile_k=0,
                      bwd_tile_q=0, bwd_tile_k=0, stream=None, host_only=False) -> Meta:
    lib = load_library()
    off, p, c, r = _i32(offset), _i32(prefix_len), _i32(chosen_len), _i32(rejected_len)
    n = off.shape[0]
    if not (p.shape[0] == c.shape[0] == r.shape[0] == n):
        raise ValueError("sample arrays differ in length")
    h = C.c_void_p()
    if host_only:
        st = lib.psattn_build_meta_host(n, _addr(off), _addr(p), _addr(c), _addr(r),
                                        int(total_tokens), tile_q, tile_k, bwd_tile_q, bwd_tile_k, C.byref(h))
        _check(st, "psattn_build_meta_host")
    else:
        st = lib.psattn_build_meta(n, _addr(off), _addr(p), _addr(c), _addr(r),
                                   int(total_tokens), tile_q, tile_k, bwd_tile_q, bwd_tile_k,
                                   _stream_ptr(stream), C.byref(h))
        _check(st, "psattn_build_meta")
    return Meta(h, total_tokens, not host_only)


def psattn_build_meta_multi(offset, prefix_len, resp_ptr, resp_len, total_tokens, tile_q=0, tile_k=0,
                            bwd_tile_q=0, bwd_tile_k=0, stream=None, host_only=False) -> Meta:
    """Block mask for samples with any number of responses per prompt (CSR-style resp_ptr / resp_len)."""
    lib = load_library()
    off, p, ptr, rl = _i32(offset), _i32(prefix_len), _i32(resp_ptr), _i32(resp_len)
    n = off.shape[0]
    if p.shape[0] != n or ptr.shape[0] != n + 1 or (n and rl.shape[0] != int(ptr[-1])):
        raise ValueError("sample arrays differ in length")
    rl_ptr = _addr(rl) if rl.shape[0] else None
    h = C.c_void_p()
    if host_only:
        st = lib.psattn_build_meta_multi_host(n, _addr(off), _addr(p), _addr(ptr), rl_ptr,
                                              int(total_tokens), tile_q, tile_k, bwd_tile_q, bwd_tile_k, C.byref(h))
        _check(st, "psattn_build_meta_multi_host")
    else:
        st = lib.psattn_build_meta_multi(n, _addr(off), _addr(p), _addr(ptr), rl_ptr,
                                         int(total_tokens), tile_q, tile_k, bwd_tile_q, bwd_tile_k,
                                         _stream_ptr(stream), C.byref(h))
        _check(st, "psattn_build_meta_multi")
    return Meta(h, total_tokens, not host_only)


def psattn_pack_ffd(prefix_len, chosen_len, rejected_len, row_len, max_rows=0):
    """First-Fit-Decreasing packing.  Returns dict(offset [n] (-1 = left out), order [n], n_rows,
    padding_tokens)."""
    lib = load_library()
    p, c, r = _i32(prefix_len), _i32(chosen_len), _i32(rejected_len)
    n = p.shape[0]
    if not (c.shape[0] == r.shape[0] == n):
        raise ValueError("sample arrays differ in length")
    offset = np.zeros(max(1, n), dtype=np.int32)
    order = np.zeros(max(1, n), dtype=np.int32)
    n_rows, pad = C.c_int32(), C.c_int64()
    st = lib.psattn_pack_ffd(n, _addr(p), _addr(c), _addr(r), int(row_len), int(max_rows),
                             offset.ctypes.data, order.ctypes.data, C.byref(n_rows), C.byref(pad))
    _check(st, "psattn_pack_ffd")
    return dict(offset=offset[:n], order=order[:n], n_rows=n_rows.value, padding_tokens=pad.value)


def _dtype_code(t):
    torch = _TORCH or _torch()
    dtype = t.dtype
    if dtype == torch.bfloat16:
        return BF16
    if dtype == torch.float32:
        return F32
    raise TypeError("psattn supports float32 and bfloat16 tensors, got %s" % t.dtype)


def _check_tensor(t, name, shape, dtype):
    if t.is_cuda and t.is_contiguous() and t.shape == shape and (dtype is None or t.dtype == dtype):
        return
    if not t.is_cuda:
        raise ValueError("%s must be a device tensor" % name)
    if not t.is_contiguous():
        raise ValueError("%s must be contiguous" % name)
    if tuple(t.shape) != tuple(shape):
        raise ValueError("%s has shape %s, expected %s" % (name, tuple(t.shape), tuple(shape)))
    if dtype is not None and t.dtype != dtype:
        raise TypeError("%s has dtype %s, expected %s" % (name, t.dtype, dtype))


def psattn_fwd(meta: Meta, Q, K, V, scale, O=None, LSE=None, stream=None):
    """O, LSE = attention forward.  Q [T, Hq, d]; K, V [T, Hkv, d]; LSE [Hq, T] float32."""
    if stream is not None:
        return _elsewhere(psattn_fwd, locals())
    torch, lib = _TORCH or _torch(), _LIB or load_library()
    T, Hq, d = Q.shape
    Hkv = K.shape[1]
    _check_tensor(Q, "Q", (meta.total_tokens, Hq, d), None)
    _check_tensor(K, "K", (T, Hkv, d), Q.dtype)
    _check_tensor(V, "V", (T, Hkv, d), Q.dtype)
    if O is None:
        O = torch.empty_like(Q)
    if LSE is None:
        LSE = torch.empty((Hq, T), dtype=torch.float32, device=Q.device)
    _check_tensor(O, "O", Q.shape, Q.dtype)
    _check_tensor(LSE, "LSE", (Hq, T), torch.float32)
    st = lib.psattn_fwd(meta.handle, _dtype_code(Q), Hq, Hkv, d, float(scale), Q.data_ptr(), K.data_ptr(),
                        V.data_ptr(), O.data_ptr(), LSE.data_ptr(), _stream_ptr(stream))
    _check(st, "psattn_fwd")
    return O, LSE


def psattn_bwd_workspace_bytes(meta: Meta, n_q_heads, n_kv_heads, head_dim) -> int:
    return int(load_library().psattn_bwd_workspace_bytes(meta.handle, n_q_heads, n_kv_heads, head_dim))


def psattn_bwd(meta: Meta, Q, K, V, O, dO, LSE, scale, dQ=None, dK=None, dV=None, workspace=None,
               stream=None):
    """dQ, dK, dV = attention backward from the forward's O and LSE."""
    if stream is not None:
        return _elsewhere(psattn_bwd, locals())
    torch, lib = _TORCH or _torch(), _LIB or load_library()
    T, Hq, d = Q.shape
    Hkv = K.shape[1]
    _check_tensor(Q, "Q", (meta.total_tokens, Hq, d), None)
    _check_tensor(K, "K", (T, Hkv, d), Q.dtype)
    _check_tensor(V, "V", (T, Hkv, d), Q.dtype)
    _check_tensor(O, "O", Q.shape, Q.dtype)
    _check_tensor(dO, "dO", Q.shape, Q.dtype)
    _check_tensor(LSE, "LSE", (Hq, T), torch.float32)
    dQ = torch.empty_like(Q) if dQ is None else dQ
    dK = torch.empty_like(K) if dK is None else dK
    dV = torch.empty_like(V) if dV is None else dV
    _check_tensor(dQ, "dQ", Q.shape, Q.dtype)
    _check_tensor(dK, "dK", K.shape, Q.dtype)
    _check_tensor(dV, "dV", V.shape, Q.dtype)
    if workspace is None:
        workspace = torch.empty(psattn_bwd_workspace_bytes(meta, Hq, Hkv, d), dtype=torch.uint8, device=Q.device)
    if not workspace.is_cuda or not workspace.is_contiguous():
        raise ValueError("workspace must be a contiguous device tensor")
    ws_bytes = workspace.numel() * workspace.element_size()
    st = lib.psattn_bwd(meta.handle, _dtype_code(Q), Hq, Hkv, d, float(scale), Q.data_ptr(), K.data_ptr(),
                        V.data_ptr(), O.data_ptr(), dO.data_ptr(), LSE.data_ptr(), dQ.data_ptr(),
                        dK.data_ptr(), dV.data_ptr(), workspace.data_ptr(), ws_bytes, _stream_ptr(stream))
    _check(st, "psattn_bwd")
    return dQ, dK, dV


def psattn_bwd_static(meta: Meta, Q, K, V, O, dO, LSE, scale, dQ, dK, dV, stream=None):
    """psattn_bwd on the library's static scratch: allocates nothing, so the outputs must be given."""
    torch, lib = _TORCH or _torch(), _LIB or load_library()
    T, Hq, d = Q.shape
    Hkv = K.shape[1]
    _check_tensor(Q, "Q", (meta.total_tokens, Hq, d), None)
    for t, name, shape in ((K, "K", (T, Hkv, d)), (V, "V", (T, Hkv, d)), (O, "O", Q.shape), (dO, "dO", Q.shape),
                           (dQ, "dQ", Q.shape), (dK, "dK", K.shape), (dV, "dV", K.shape)):
        _check_tensor(t, name, shape, Q.dtype)
    _check_tensor(LSE, "LSE", (Hq, T), torch.float32)
    st = lib.psattn_bwd_static(meta.handle, _dtype_code(Q), Hq, Hkv, d, float(scale), Q.data_ptr(), K.data_ptr(),
                               V.data_ptr(), O.data_ptr(), dO.data_ptr(), LSE.data_ptr(), dQ.data_ptr(),
                               dK.data_ptr(), dV.data_ptr(), _stream_ptr(stream))
    _check(st, "psattn_bwd_static")
    return dQ, dK, dV


def psattn_bwd_static_max_rows() -> int:
    return int(load_library().psattn_bwd_static_max_rows())


def psattn_rope_frequencies(rotary_dim, theta, scaling="none", factor=1.0, original_positions=0, low=1.0, high=32.0):
    """Angle per position of each pair of the first `rotary_dim` dimensions, float64 [rotary_dim / 2] (host only)."""
    if scaling not in _ROPE_SCALINGS:
        raise ValueError("scaling must be one of %s, got %r" % (sorted(_ROPE_SCALINGS), scaling))
    out = np.zeros(max(1, int(rotary_dim) // 2), dtype=np.float64)
    st = load_library().psattn_rope_frequencies(int(rotary_dim), float(theta), _ROPE_SCALINGS[scaling], float(factor), float(original_positions),
                                                float(low), float(high), _addr(out))
    _check(st, "psattn_rope_frequencies")
    return out


class Rope:
    """Owner of a psattn_rope handle (cos/sin table on the current device).

    With any of the keywords it is a table for psattn_rope_apply: the first `rotary_dim` dimensions of a head, "half" or "interleaved"
    pairs, `frequencies` as by psattn_rope_frequencies (default: theta's), cosines and sines times `amplitude`."""

    def __init__(self, head_dim, theta, max_positions, stream=None, *, rotary_dim=None, layout=None, frequencies=None, amplitude=None):
        lib = load_library()
        h = C.c_void_p()
        self._h = None
        self.head_dim, self.max_positions = int(head_dim), int(max_positions)
        self.rotary_dim = self.head_dim if rotary_dim is None else int(rotary_dim)
        self.layout = "half" if layout is None else layout
        if rotary_dim is None and layout is None and frequencies is None and amplitude is None:
            _check(lib.psattn_rope_create(int(head_dim), float(theta), int(max_positions), _stream_ptr(stream), C.byref(h)),
                   "psattn_rope_create")
        else:
            if self.layout not in _ROPE_LAYOUTS:
                raise ValueError("layout must be one of %s, got %r" % (sorted(_ROPE_LAYOUTS), layout))
            f = psattn_rope_frequencies(self.rotary_dim, theta) if frequencies is None else np.ascontiguousarray(frequencies, dtype=np.float64)
            if f.shape != (self.rotary_dim // 2,):
                raise ValueError("frequencies has shape %s, expected %s" % (f.shape, (self.rotary_dim // 2,)))
            _check(lib.psattn_rope_create_layout(self.head_dim, self.rotary_dim, _ROPE_LAYOUTS[self.layout], _addr(f),
                                                 1.0 if amplitude is None else float(amplitude), self.max_positions, _stream_ptr(stream),
                                                 C.byref(h)), "psattn_rope_create_layout")
        self._h = h

    @property
    def handle(self):
        if self._h is None:
            raise ValueError("rope table already freed")
        return self._h

    def free(self):
        if self._h is not None:
            _check(load_library().psattn_rope_free(self._h), "psattn_rope_free")
            self._h = None

    def __del__(self):
        try:
            self.free()
        except Exception:
            pass


def psattn_fwd_rope(meta: Meta, rope: Rope, Q, K, V, scale, O=None, LSE=None, Qr=None, Kr=None, stream=None):
    """O, LSE, Qr, Kr = forward with rotary embedding applied to the unrotated Q, K inside the op."""
    if stream is not None:
        return _elsewhere(psattn_fwd_rope, locals())
    torch, lib = _TORCH or _torch(), _LIB or load_library()
    T, Hq, d = Q.shape
    Hkv = K.shape[1]
    _check_tensor(Q, "Q", (meta.total_tokens, Hq, d), None)
    _check_tensor(K, "K", (T, Hkv, d), Q.dtype)
    _check_tensor(V, "V", (T, Hkv, d), Q.dtype)
    O = torch.empty_like(Q) if O is None else O
    LSE = torch.empty((Hq, T), dtype=torch.float32, device=Q.device) if LSE is None else LSE
    Qr = torch.empty_like(Q) if Qr is None else Qr
    Kr = torch.empty_like(K) if Kr is None else Kr
    _check_tensor(O, "O", Q.shape, Q.dtype)
    _check_tensor(LSE, "LSE", (Hq, T), torch.float32)
    _check_tensor(Qr, "Qr", Q.shape, Q.dtype)
    _check_tensor(Kr, "Kr", K.shape, Q.dtype)
    st = lib.psattn_fwd_rope(meta.handle, rope.handle, _dtype_code(Q), Hq, Hkv, d, float(scale), Q.data_ptr(),
                             K.data_ptr(), V.data_ptr(), O.data_ptr(), LSE.data_ptr(), Qr.data_ptr(), Kr.data_ptr(),
                             _stream_ptr(stream))
    _check(st, "psattn_fwd_rope")
    return O, LSE, Qr, Kr


def psattn_bwd_rope(meta: Meta, rope: Rope, Qr, Kr, V, O, dO, LSE, scale, dQ=None, dK=None, dV=None, workspace=None,
                    stream=None):
    """dQ, dK, dV (w.r.t. the unrotated Q, K) from the forward's rotated Qr, Kr."""
    if stream is not None:
        return _elsewhere(psattn_bwd_rope, locals())
    torch, lib = _TORCH or _torch(), _LIB or load_library()
    T, Hq, d = Qr.shape
    Hkv = Kr.shape[1]
    _check_tensor(Qr, "Qr", (meta.total_tokens, Hq, d), None)
    for t, name, shape in ((Kr, "Kr", (T, Hkv, d)), (V, "V", (T, Hkv, d)), (O, "O", Qr.shape), (dO, "dO", Qr.shape)):
        _check_tensor(t, name, shape, Qr.dtype)
    _check_tensor(LSE, "LSE", (Hq, T), torch.float32)
    dQ = torch.empty_like(Qr) if dQ is None else dQ
    dK = torch.empty_like(Kr) if dK is None else dK
    dV = torch.empty_like(V) if dV is None else dV
    for t, name, shape in ((dQ, "dQ", Qr.shape), (dK, "dK", Kr.shape), (dV, "dV", Kr.shape)):
        _check_tensor(t, name, shape, Qr.dtype)
    if workspace is None:
        workspace = torch.empty(psattn_bwd_workspace_bytes(meta, Hq, Hkv, d), dtype=torch.uint8, device=Qr.device)
    st = lib.psattn_bwd_rope(meta.handle, rope.handle, _dtype_code(Qr), Hq, Hkv, d, float(scale), Qr.data_ptr(),
                             Kr.data_ptr(), V.data_ptr(), O.data_ptr(), dO.data_ptr(), LSE.data_ptr(), dQ.data_ptr(),
                             dK.data_ptr(), dV.data_ptr(), workspace.data_ptr(),
                             workspace.numel() * workspace.element_size(), _stream_ptr(stream))
    _check(st, "psattn_bwd_rope")
    return dQ, dK, dV


def _check_heads(dev, t, name, shape, dtype):
    """Token stride of Q or K: heads and dimensions contiguous, tokens any distance apart."""
    if t.get_device() != dev or t.shape != shape or t.dtype != dtype:
        if not t.is_cuda:
            raise ValueError("%s must be a device tensor" % name)
        if t.get_device() != dev:
            raise ValueError("%s is on %s, not on cuda:%d" % (name, t.device, dev))
        if t.shape != shape:
            raise ValueError("%s has shape %s, expected %s" % (name, tuple(t.shape), tuple(shape)))
        raise TypeError("%s has dtype %s, expected %s" % (name, t.dtype, dtype))
    T, H, d = shape
    at, head, one = t.stride()
    if T <= 1:
        at = H * d
    if (d > 1 and one != 1) or (H > 1 and head != d) or at < H * d:
        raise ValueError("the heads of a token of %s must be contiguous" % name)
    return at


def _rope_apply(what, transposed, rope, Q, K, positions, meta, Qr, Kr):
    torch, lib = _TORCH or _torch(), _LIB or load_library()
    if Q.dim() != 3 or (K is not None and K.dim() != 3):
        raise ValueError("Q and K have three dimensions: tokens, heads, head_dim")
    if (positions is None) == (meta is None):
        raise ValueError("positions or meta say where the tokens are: one of them")
    shape, dtype, dev = Q.shape, Q.dtype, Q.get_device()
    T, Hq, d = shape
    if d != rope.head_dim:
        raise ValueError("Q has heads of %d, the rotary table of %d" % (d, rope.head_dim))
    if not Q.is_cuda:
        raise ValueError("Q must be a device tensor")
    if T >= 1 << 31 or Hq >= 1 << 31:
        raise ValueError("Q has shape %s: sizes are 32-bit" % (tuple(shape),))
    if dev != torch._C._cuda_getDevice():
        raise ValueError("Q is on %s, which is not the current device" % Q.device)
    dt, q = _dtype_code(Q), _check_heads(dev, Q, "Q", shape, dtype)
    if Qr is None:
        Qr, qr = torch.empty(shape, dtype=dtype, device=Q.device), Hq * d
    else:
        qr = _check_heads(dev, Qr, "the output for Q", shape, dtype)
    Hk = k = kr = 0
    kp = krp = None
    if K is not None:
        Hk = K.shape[1]
        k = _check_heads(dev, K, "K", (T, Hk, d), dtype)
        if Kr is None:
            Kr, kr = torch.empty((T, Hk, d), dtype=dtype, device=Q.device), Hk * d
        else:
            kr = _check_heads(dev, Kr, "the output for K", K.shape, dtype)
        kp, krp = K.data_ptr(), Kr.data_ptr()
    elif Kr is not None:
        raise ValueError("an output for K is given, but no K")
    if positions is not None:
        _check_all(dev, (positions, "positions", (T,), torch.int32))
    st = lib.psattn_rope_apply(rope.handle, dt, transposed, T, None if positions is None else positions.data_ptr(), None if meta is None else meta.handle,
                               Hq, Q.data_ptr(), q, Qr.data_ptr(), qr, Hk, kp, k, krp, kr, _stream_ptr(None))
    _check(st, what)
    return Qr, Kr


def psattn_rope_apply(rope: Rope, Q, K=None, positions=None, meta=None, Qr=None, Kr=None, stream=None):
    """Qr, Kr = Q [T, Hq, d] and K [T, Hkv, d] (or None) turned by their tokens' positions: int32 [T], or those of a Meta.  Tokens
    may be any distance apart (slices of one buffer); Qr may be Q and Kr K."""
    if stream is not None:
        return _elsewhere(psattn_rope_apply, locals())
    return _rope_apply("psattn_rope_apply", 0, rope, Q, K, positions, meta, Qr, Kr)


def psattn_rope_apply_bwd(rope: Rope, dQr, dKr=None, positions=None, meta=None, dQ=None, dK=None, stream=None):
    """dQ, dK = gradients of psattn_rope_apply's Q and K from those of Qr and Kr (the transposed turn)."""
    if stream is not None:
        return _elsewhere(psattn_rope_apply_bwd, locals())
    return _rope_apply("psattn_rope_apply_bwd", 1, rope, dQr, dKr, positions, meta, dQ, dK)


class LogprobPlan:
    """Owner of a psattn_lp_plan handle."""

    def __init__(self, offset, prefix_len, resp_ptr, resp_len, total_tokens, stream=None):
        lib = load_library()
        off, p, ptr, rl = _i32(offset), _i32(prefix_len), _i32(resp_ptr), _i32(resp_len)
        h = C.c_void_p()
        _check(lib.psattn_logprob_plan(off.shape[0], _addr(off), _addr(p), _addr(ptr),
                                       _addr(rl) if rl.shape[0] else None, int(total_tokens), _stream_ptr(stream),
                                       C.byref(h)), "psattn_logprob_plan")
        self._h = h
        self.total_tokens = int(total_tokens)
        a, b, c = C.c_int32(), C.c_int32(), C.c_int64()
        _check(lib.psattn_logprob_plan_info(h, C.byref(a), C.byref(b), C.byref(c)), "psattn_logprob_plan_info")
        self.n_responses, self.n_rows, self.n_items = a.value, b.value, c.value

    @property
    def handle(self):
        if self._h is None:
            raise ValueError("plan already freed")
        return self._h

    def free(self):
        if self._h is not None:
            _check(load_library().psattn_logprob_plan_free(self._h), "psattn_logprob_plan_free")
            self._h = None

    def __del__(self):
        try:
            self.free()
        except Exception:
            pass


def psattn_logprob_fwd(plan: LogprobPlan, logits, token_ids, row_lse=None, resp_logp=None, stream=None):
    """row_lse [T], resp_logp [n_responses] from logits [T, vocab] and token_ids int32 [T]."""
    if stream is not None:
        return _elsewhere(psattn_logprob_fwd, locals())
    torch = _TORCH or _torch()
    T, V = logits.shape
    _check_tensor(logits, "logits", (plan.total_tokens, V), None)
    _check_tensor(token_ids, "token_ids", (T,), torch.int32)
    row_lse = torch.zeros(T, dtype=torch.float32, device=logits.device) if row_lse is None else row_lse
    resp_logp = torch.empty(plan.n_responses, dtype=torch.float32, device=logits.device) if resp_logp is None else resp_logp
    _check_tensor(row_lse, "row_lse", (T,), torch.float32)
    _check_tensor(resp_logp, "resp_logp", (plan.n_responses,), torch.float32)
    st = load_library().psattn_logprob_fwd(plan.handle, _dtype_code(logits), V, logits.data_ptr(), token_ids.data_ptr(),
                                           row_lse.data_ptr(), resp_logp.data_ptr(), _stream_ptr(stream))
    _check(st, "psattn_logprob_fwd")
    return row_lse, resp_logp


def psattn_logprob_bwd(plan: LogprobPlan, logits, token_ids, row_lse, d_resp_logp, dlogits=None, stream=None):
    if stream is not None:
        return _elsewhere(psattn_logprob_bwd, locals())
    torch = _TORCH or _torch()
    T, V = logits.shape
    _check_tensor(logits, "logits", (plan.total_tokens, V), None)
    _check_tensor(token_ids, "token_ids", (T,), torch.int32)
    _check_tensor(row_lse, "row_lse", (T,), torch.float32)
    _check_tensor(d_resp_logp, "d_resp_logp", (plan.n_responses,), torch.float32)
    dlogits = torch.empty_like(logits) if dlogits is None else dlogits
    _check_tensor(dlogits, "dlogits", logits.shape, logits.dtype)
    st = load_library().psattn_logprob_bwd(plan.handle, _dtype_code(logits), V, logits.data_ptr(), token_ids.data_ptr(),
                                           row_lse.data_ptr(), d_resp_logp.data_ptr(), dlogits.data_ptr(),
                                           _stream_ptr(stream))
    _check(st, "psattn_logprob_bwd")
    return dlogits


def _head_shapes(plan, X, W, token_ids):
    dev = _check_rows(X, "X")
    _check_rows(W, "W")
    (T, h), V = X.shape, W.shape[0]
    if T != plan.total_tokens:
        raise ValueError("X has shape %s, expected %s" % ((T, h), (plan.total_tokens, h)))
    _check_all(dev, (W, "W", (V, h), X.dtype), (token_ids, "token_ids", (T,), (_TORCH or _torch()).int32))
    return dev, T, h, V, _dtype_code(X)


def psattn_head_logprob_fwd(plan: LogprobPlan, X, W, token_ids, row_lse=None, resp_logp=None, workspace=None, stream=None):
    """row_lse [T], resp_logp [n_responses] from hidden rows X [T, hidden], W [vocab, hidden] and token_ids int32 [T]; the logits X W^T
    are never in memory."""
    if stream is not None:
        return _elsewhere(psattn_head_logprob_fwd, locals())
    torch, lib = _TORCH or _torch(), _LIB or load_library()
    dev, T, h, V, dt = _head_shapes(plan, X, W, token_ids)
    _check_all(dev, (row_lse, "row_lse", (T,), torch.float32), (resp_logp, "resp_logp", (plan.n_responses,), torch.float32))
    row_lse = torch.zeros(T, dtype=torch.float32, device=X.device) if row_lse is None else row_lse
    resp_logp = torch.empty(plan.n_responses, dtype=torch.float32, device=X.device) if resp_logp is None else resp_logp
    ws = _workspace(workspace, lib.psattn_head_logprob_fwd_workspace_bytes(plan.handle, dt, V, h), X)
    st = lib.psattn_head_logprob_fwd(plan.handle, dt, V, h, X.data_ptr(), W.data_ptr(), token_ids.data_ptr(), row_lse.data_ptr(), resp_logp.data_ptr(),
                                     ws.data_ptr(), ws.numel() * ws.element_size(), _stream_ptr(None))
    _check(st, "psattn_head_logprob_fwd")
    return row_lse, resp_logp


def psattn_head_logprob_bwd(plan: LogprobPlan, X, W, token_ids, row_lse, d_resp_logp, dX=None, dW=None, workspace=None, stream=None):
    """dX [T, hidden], dW [vocab, hidden] of sum_j d_resp_logp[j] * resp_logp[j], from the forward's row_lse."""
    if stream is not None:
        return _elsewhere(psattn_head_logprob_bwd, locals())
    torch, lib = _TORCH or _torch(), _LIB or load_library()
    dev, T, h, V, dt = _head_shapes(plan, X, W, token_ids)
    for t, name in ((row_lse, "row_lse"), (d_resp_logp, "d_resp_logp")):
        if t is None:
            raise ValueError("%s is missing" % name)
    _check_all(dev, (row_lse, "row_lse", (T,), torch.float32), (d_resp_logp, "d_resp_logp", (plan.n_responses,), torch.float32),
               (dX, "dX", X.shape, X.dtype), (dW, "dW", W.shape, X.dtype))
    dX = torch.empty_like(X) if dX is None else dX
    dW = torch.empty_like(W) if dW is None else dW
    ws = _workspace(workspace, lib.psattn_head_logprob_bwd_workspace_bytes(plan.handle, dt, V, h), X)
    st = lib.psattn_head_logprob_bwd(plan.handle, dt, V, h, X.data_ptr(), W.data_ptr(), token_ids.data_ptr(), row_lse.data_ptr(), d_resp_logp.data_ptr(),
                                     dX.data_ptr(), dW.data_ptr(), ws.data_ptr(), ws.numel() * ws.element_size(), _stream_ptr(None))
    _check(st, "psattn_head_logprob_bwd")
    return dX, dW


def psattn_dpo_loss(logp_policy, logp_ref, beta, stream=None):
    """loss [n_pairs], d_logp [2 n_pairs] for responses stored as (chosen, rejected) pairs."""
    if stream is not None:
        return _elsewhere(psattn_dpo_loss, locals())
    torch = _TORCH or _torch()
    n = logp_policy.shape[0]
    if n % 2 or tuple(logp_ref.shape) != (n,):
        raise ValueError("log-probabilities must come in (chosen, rejected) pairs")
    _check_tensor(logp_policy, "logp_policy", (n,), torch.float32)
    _check_tensor(logp_ref, "logp_ref", (n,), torch.float32)
    loss = torch.empty(n // 2, dtype=torch.float32, device=logp_policy.device)
    d = torch.empty(n, dtype=torch.float32, device=logp_policy.device)
    st = load_library().psattn_dpo_loss(n // 2, float(beta), logp_policy.data_ptr(), logp_ref.data_ptr(), loss.data_ptr(),
                                        d.data_ptr(), _stream_ptr(stream))
    _check(st, "psattn_dpo_loss")
    return loss, d


# ---- what stands beside attention in a model: embedding, layer norm, feed-forward block
def _check_rows(t, name):
    """Index of the device that a call runs on: that of the tensor from which it takes its sizes."""
    if t.dim() != 2:
        raise ValueError("%s must have two dimensions, got %d" % (name, t.dim()))
    if max(t.shape) >= 1 << 31:
        raise ValueError("%s has shape %s: sizes are 32-bit" % (name, tuple(t.shape)))
    _check_tensor(t, name, t.shape, None)
    dev = t.get_device()
    if dev != (_TORCH or _torch())._C._cuda_getDevice():
        raise ValueError("%s is on %s, which is not the current device" % (name, t.device))
    return dev


def _check_all(dev, *tensors):
    """(tensor, name, shape, dtype) each, on device `dev`.  None: an output that the call makes itself."""
    for t, name, shape, dtype in tensors:
        if t is None or (t.get_device() == dev and t.is_contiguous() and t.shape == shape and t.dtype == dtype):
            continue
        _check_tensor(t, name, shape, dtype)
        raise ValueError("%s is on %s, not on cuda:%d" % (name, t.device, dev))


def _workspace(given, need, like):
    """A call's workspace: the caller's, or one that goes back to torch when the call returns."""
    if given is None:
        return (_TORCH or _torch()).empty(need, dtype=(_TORCH or _torch()).uint8, device=like.device)
    if not given.is_cuda or not given.is_contiguous() or given.device != like.device:
        raise ValueError("workspace must be a contiguous device tensor on %s" % like.device)
    return given


def psattn_embed_fwd(token_ids, W, scale=1.0, X=None, stream=None):
    """X [T, hidden] = scale * rows of W [vocab, hidden] by token_ids int32 [T]; ids outside the table give rows of zeros."""
    if stream is not None:
        return _elsewhere(psattn_embed_fwd, locals())
    torch, lib = _TORCH or _torch(), _LIB or load_library()
    dev = _check_rows(W, "W")
    (V, h), T = W.shape, token_ids.numel()
    dt = _dtype_code(W)
    _check_all(dev, (token_ids, "token_ids", (T,), torch.int32), (X, "X", (T, h), W.dtype))
    X = torch.empty((T, h), dtype=W.dtype, device=W.device) if X is None else X
    st = lib.psattn_embed_fwd(dt, T, V, h, float(scale), token_ids.data_ptr(), W.data_ptr(), X.data_ptr(), _stream_ptr(stream))
    _check(st, "psattn_embed_fwd")
    return X


def psattn_embed_bwd(token_ids, dX, vocab, scale=1.0, dW=None, workspace=None, stream=None):
    """dW [vocab, hidden]: the gradient of psattn_embed_fwd's table."""
    if stream is not None:
        return _elsewhere(psattn_embed_bwd, locals())
    torch, lib = _TORCH or _torch(), _LIB or load_library()
    dev = _check_rows(dX, "dX")
    (T, h), vocab = dX.shape, int(vocab)
    dt = _dtype_code(dX)
    if not 0 < vocab < 1 << 31:
        raise ValueError("vocab must be a positive 32-bit number, got %d" % vocab)
    _check_all(dev, (token_ids, "token_ids", (T,), torch.int32), (dW, "dW", (vocab, h), dX.dtype))
    dW = torch.empty((vocab, h), dtype=dX.dtype, device=dX.device) if dW is None else dW
    ws = _workspace(workspace, lib.psattn_embed_bwd_workspace_bytes(dt, T, vocab, h), dX)
    st = lib.psattn_embed_bwd(dt, T, vocab, h, float(scale), token_ids.data_ptr(), dX.data_ptr(), dW.data_ptr(), ws.data_ptr(),
                              ws.numel() * ws.element_size(), _stream_ptr(stream))
    _check(st, "psattn_embed_bwd")
    return dW


def psattn_layernorm_fwd(X, weight, bias=None, eps=1e-5, residual=None, S=None, Y=None, mean=None, rstd=None, stream=None):
    """Y, S, mean, rstd = layer norm of the rows of S = X + residual (S is X itself without one)."""
    if stream is not None:
        return _elsewhere(psattn_layernorm_fwd, locals())
    torch, lib = _TORCH or _torch(), _LIB or load_library()
    dev = _check_rows(X, "X")
    shape, dt, dtype, f32 = X.shape, _dtype_code(X), X.dtype, torch.float32
    n, h = shape
    if S is not None and residual is None:
        raise ValueError("S is an output of the residual sum: without a residual it is X")
    _check_all(dev, (weight, "weight", (h,), dtype), (bias, "bias", (h,), dtype), (residual, "residual", shape, dtype), (S, "S", shape, dtype),
               (Y, "Y", shape, dtype), (mean, "mean", (n,), f32), (rstd, "rstd", (n,), f32))
    if residual is not None and S is None:
        S = torch.empty_like(X)
    Y = torch.empty_like(X) if Y is None else Y
    mean = torch.empty(n, dtype=f32, device=X.device) if mean is None else mean
    rstd = torch.empty(n, dtype=f32, device=X.device) if rstd is None else rstd
    st = lib.psattn_layernorm_fwd(dt, n, h, float(eps), X.data_ptr(), None if residual is None else residual.data_ptr(), weight.data_ptr(),
                                  None if bias is None else bias.data_ptr(), None if residual is None else S.data_ptr(), Y.data_ptr(),
                                  mean.data_ptr(), rstd.data_ptr(), _stream_ptr(stream))
    _check(st, "psattn_layernorm_fwd")
    return Y, X if residual is None else S, mean, rstd


def psattn_layernorm_bwd(S, weight, mean, rstd, dY, dS=None, bias=True, dX=None, dweight=None, dbias=None, workspace=None, stream=None):
    """dX, dweight, dbias (None where `bias` is false) from the forward's S, mean and rstd; dX has dS added to it."""
    if stream is not None:
        return _elsewhere(psattn_layernorm_bwd, locals())
    torch, lib = _TORCH or _torch(), _LIB or load_library()
    dev = _check_rows(S, "S")
    shape, dt, dtype, f32 = S.shape, _dtype_code(S), S.dtype, torch.float32
    n, h = shape
    if dbias is not None and not bias:
        raise ValueError("dbias is given, but there is no bias")
    for t, name in ((weight, "weight"), (mean, "mean"), (rstd, "rstd"), (dY, "dY")):
        if t is None:
            raise ValueError("%s is missing" % name)
    _check_all(dev, (weight, "weight", (h,), dtype), (mean, "mean", (n,), f32), (rstd, "rstd", (n,), f32), (dY, "dY", shape, dtype),
               (dS, "dS", shape, dtype), (dX, "dX", shape, dtype), (dweight, "dweight", (h,), dtype), (dbias, "dbias", (h,), dtype))
    dX = torch.empty_like(S) if dX is None else dX
    dweight = torch.empty_like(weight) if dweight is None else dweight
    if bias and dbias is None:
        dbias = torch.empty_like(weight)
    ws = _workspace(workspace, lib.psattn_layernorm_bwd_workspace_bytes(n, h), S)
    st = lib.psattn_layernorm_bwd(dt, n, h, S.data_ptr(), weight.data_ptr(), mean.data_ptr(), rstd.data_ptr(), dY.data_ptr(),
                                  None if dS is None else dS.data_ptr(), dX.data_ptr(), dweight.data_ptr(),
                                  dbias.data_ptr() if bias else None, ws.data_ptr(), ws.numel() * ws.element_size(), _stream_ptr(stream))
    _check(st, "psattn_layernorm_bwd")
    return dX, dweight, dbias


def _gate_rows(gate, n, h, dtype):
    """How many rows a gate has, and its check: [hidden], [1, hidden] or [n, hidden]."""
    if gate is None:
        return 0, (None, "gate", (h,), dtype)
    if gate.dim() == 2:
        return gate.shape[0], (gate, "gate", (1 if gate.shape[0] == 1 else n, h), dtype)
    return 1, (gate, "gate", (h,), dtype)


def psattn_gatednorm_fwd(X, B, w_pre, w_post=None, gate=None, res_scale=1.0, eps=1e-6, S=None, Y=None, rstd_b=None, rstd_s=None, stream=None):
    """Y, S, rstd_b, rstd_s: S = res_scale * X + gate o (B * rstd_b * w_post), Y = S * rstd_s * w_pre, RMS norms both.  gate: [hidden], [n, hidden]
    or None; without w_post B itself joins X (rstd_b is None).  B = None: Y is the norm of X, which is S."""
    if stream is not None:
        return _elsewhere(psattn_gatednorm_fwd, locals())
    torch, lib = _TORCH or _torch(), _LIB or load_library()
    dev = _check_rows(X, "X")
    shape, dt, dtype, f32 = X.shape, _dtype_code(X), X.dtype, torch.float32
    n, h = shape
    if w_pre is None:
        raise ValueError("w_pre is missing")
    if B is None and (w_post is not None or gate is not None or S is not None):
        raise ValueError("w_post, gate and S belong to B, which is None")
    if w_post is None and rstd_b is not None:
        raise ValueError("rstd_b is given, but there is no w_post")
    rows, gate_check = _gate_rows(gate, n, h, dtype)
    _check_all(dev, (B, "B", shape, dtype), (w_pre, "w_pre", (h,), dtype), (w_post, "w_post", (h,), dtype), gate_check, (S, "S", shape, dtype),
               (Y, "Y", shape, dtype), (rstd_b, "rstd_b", (n,), f32), (rstd_s, "rstd_s", (n,), f32))
    if B is not None and S is None:
        S = torch.empty_like(X)
    Y = torch.empty_like(X) if Y is None else Y
    if w_post is not None and rstd_b is None:
        rstd_b = torch.empty(n, dtype=f32, device=X.device)
    rstd_s = torch.empty(n, dtype=f32, device=X.device) if rstd_s is None else rstd_s
    ptr = lambda t: None if t is None else t.data_ptr()
    st = lib.psattn_gatednorm_fwd(dt, n, h, float(eps), float(res_scale), X.data_ptr(), ptr(B), ptr(w_post), ptr(gate), rows, w_pre.data_ptr(), ptr(S), Y.data_ptr(),
                                  ptr(rstd_b), rstd_s.data_ptr(), _stream_ptr(None))
    _check(st, "psattn_gatednorm_fwd")
    return Y, X if B is None else S, rstd_b, rstd_s


def psattn_gatednorm_bwd(B, S, w_pre, rstd_b, rstd_s, dY, dS=None, w_post=None, gate=None, res_scale=1.0, dX=None, dB=None, dw_pre=None, dw_post=None, dgate=None,
                         workspace=None, stream=None):
    """dX, dB, dw_pre, dw_post, dgate (None for what there was not) from the forward's B, S, rstd_b and rstd_s."""
    if stream is not None:
        return _elsewhere(psattn_gatednorm_bwd, locals())
    torch, lib = _TORCH or _torch(), _LIB or load_library()
    dev = _check_rows(S, "S")
    shape, dt, dtype, f32 = S.shape, _dtype_code(S), S.dtype, torch.float32
    n, h = shape
    for t, name in ((w_pre, "w_pre"), (rstd_s, "rstd_s"), (dY, "dY")):
        if t is None:
            raise ValueError("%s is missing" % name)
    if B is None and (w_post is not None or gate is not None or dB is not None):
        raise ValueError("w_post, gate and dB belong to B, which is None")
    if (w_post is None) != (rstd_b is None):
        raise ValueError("rstd_b is the forward's where it had w_post, and None elsewhere")
    if (w_post is None and dw_post is not None) or (gate is None and dgate is not None):
        raise ValueError("dw_post or dgate is given, but not w_post or gate")
    rows, gate_check = _gate_rows(gate, n, h, dtype)
    _check_all(dev, (B, "B", shape, dtype), (w_pre, "w_pre", (h,), dtype), (rstd_b, "rstd_b", (n,), f32), (rstd_s, "rstd_s", (n,), f32), (dY, "dY", shape, dtype),
               (dS, "dS", shape, dtype), (w_post, "w_post", (h,), dtype), gate_check, (dX, "dX", shape, dtype), (dB, "dB", shape, dtype), (dw_pre, "dw_pre", (h,), dtype),
               (dw_post, "dw_post", (h,), dtype), (dgate, "dgate", None if gate is None else gate.shape, dtype))
    dX = torch.empty_like(S) if dX is None else dX
    dw_pre = torch.empty_like(w_pre) if dw_pre is None else dw_pre
    if B is not None and dB is None:
        dB = torch.empty_like(B)
    if w_post is not None and dw_post is None:
        dw_post = torch.empty_like(w_post)
    if gate is not None and dgate is None:
        dgate = torch.empty_like(gate)
    ws = _workspace(workspace, lib.psattn_gatednorm_bwd_workspace_bytes(n, h), S)
    ptr = lambda t: None if t is None else t.data_ptr()
    st = lib.psattn_gatednorm_bwd(dt, n, h, float(res_scale), ptr(B), ptr(w_post), ptr(gate), rows, w_pre.data_ptr(), S.data_ptr(), ptr(rstd_b), rstd_s.data_ptr(),
                                  dY.data_ptr(), ptr(dS), dX.data_ptr(), ptr(dB), ptr(dw_post), ptr(dgate), dw_pre.data_ptr(), ws.data_ptr(),
                                  ws.numel() * ws.element_size(), _stream_ptr(None))
    _check(st, "psattn_gatednorm_bwd")
    return dX, dB, dw_pre, dw_post, dgate


def _ffn_shapes(X, Wg, Wu, Wd, act):
    dev = _check_rows(X, "X")
    if act not in _ACTS:
        raise ValueError("act must be one of %s, got %r" % (sorted(_ACTS), act))
    if Wg.dim() != 2:
        raise ValueError("Wg must have two dimensions, got %d" % Wg.dim())
    if Wu is None or Wd is None:
        raise ValueError("Wu and Wd are needed")
    (T, h), n, dtype = X.shape, Wg.shape[0], X.dtype
    return dev, T, h, n, _dtype_code(X), [(Wg, "Wg", (n, h), dtype), (Wu, "Wu", (n, h), dtype), (Wd, "Wd", (h, n), dtype)]


def psattn_ffn_fwd(X, Wg, Wu, Wd, act="silu", keep=True, Y=None, kept=None, workspace=None, stream=None):
    """Y, kept = (act(X Wg^T) o (X Wu^T)) Wd^T.  `kept` = (G, U, H), [T, inner] each, G and U float32, is what the backward takes;
    with keep=False G and U are not written and None is returned in its place (`kept` may then give H alone, as (None, None, H))."""
    if stream is not None:
        return _elsewhere(psattn_ffn_fwd, locals())
    torch, lib = _TORCH or _torch(), _LIB or load_library()
    dev, T, h, n, dt, tensors = _ffn_shapes(X, Wg, Wu, Wd, act)
    G, U, H = kept if kept is not None else (None, None, None)
    if kept is None:
        G, U = (torch.empty((T, n), dtype=torch.float32, device=X.device) for _ in range(2)) if keep else (None, None)
        H = torch.empty((T, n), dtype=X.dtype, device=X.device)
    elif H is None or (keep and (G is None or U is None)):
        raise ValueError("kept must hold G, U and H, or with keep=False H alone")
    if not keep:
        G = U = None
    if kept is not None:
        tensors += [(G, "G", (T, n), torch.float32), (U, "U", (T, n), torch.float32), (H, "H", (T, n), X.dtype)]
    _check_all(dev, *tensors, (Y, "Y", X.shape, X.dtype))
    Y = torch.empty_like(X) if Y is None else Y
    x, g, u, d, k = X.data_ptr(), Wg.data_ptr(), Wu.data_ptr(), Wd.data_ptr(), H.data_ptr()
    need = lib.psattn_ffn_fwd_unaligned_workspace_bytes if (x | g | u | d | k) & 15 else lib.psattn_ffn_fwd_workspace_bytes
    ws = _workspace(workspace, need(dt, T, h, n), X)
    st = lib.psattn_ffn_fwd(dt, _ACTS[act], T, h, n, x, g, u, d, G.data_ptr() if keep else None, U.data_ptr() if keep else None, k, Y.data_ptr(),
                            ws.data_ptr(), ws.numel() * ws.element_size(), _stream_ptr(None))
    _check(st, "psattn_ffn_fwd")
    return Y, (G, U, H) if keep else None


def psattn_ffn_bwd(X, Wg, Wu, Wd, kept, dY, act="silu", dX=None, dWg=None, dWu=None, dWd=None, workspace=None, stream=None):
    """dX, dWg, dWu, dWd from the forward's kept (G, U, H)."""
    if stream is not None:
        return _elsewhere(psattn_ffn_bwd, locals())
    torch, lib = _TORCH or _torch(), _LIB or load_library()
    dev, T, h, n, dt, tensors = _ffn_shapes(X, Wg, Wu, Wd, act)
    G, U, H = kept if kept is not None else (None, None, None)
    if any(t is None for t in (G, U, H, dY)):
        raise ValueError("kept G, U, H (psattn_ffn_fwd without them has keep=False) and dY are needed")
    _check_all(dev, *tensors, (G, "G", (T, n), torch.float32), (U, "U", (T, n), torch.float32), (H, "H", (T, n), X.dtype), (dY, "dY", X.shape, X.dtype),
               (dX, "dX", X.shape, X.dtype), (dWg, "dWg", (n, h), X.dtype), (dWu, "dWu", (n, h), X.dtype), (dWd, "dWd", (h, n), X.dtype))
    dX = torch.empty_like(X) if dX is None else dX
    dWg = torch.empty_like(Wg) if dWg is None else dWg
    dWu = torch.empty_like(Wu) if dWu is None else dWu
    dWd = torch.empty_like(Wd) if dWd is None else dWd
    x, g, u, d, k, y = X.data_ptr(), Wg.data_ptr(), Wu.data_ptr(), Wd.data_ptr(), H.data_ptr(), dY.data_ptr()
    need = lib.psattn_ffn_bwd_unaligned_workspace_bytes if (x | g | u | d | k | y) & 15 else lib.psattn_ffn_bwd_workspace_bytes
    ws = _workspace(workspace, need(dt, T, h, n), X)
    st = lib.psattn_ffn_bwd(dt, _ACTS[act], T, h, n, x, g, u, d, G.data_ptr(), U.data_ptr(), k, y, dX.data_ptr(), dWg.data_ptr(), dWu.data_ptr(), dWd.data_ptr(),
                            ws.data_ptr(), ws.numel() * ws.element_size(), _stream_ptr(None))
    _check(st, "psattn_ffn_bwd")
    return dX, dWg, dWu, dWd


def psattn_probe_dq_atomics(meta: Meta, n_q_heads, n_kv_heads, acc, mode, stream=None) -> None:
    """Measurement aid: the dQ memory operations of a one-pass backward (see include/psattn.h)."""
    if tuple(acc.shape) != (meta.total_tokens, n_q_heads, 128) or not acc.is_cuda or not acc.is_contiguous():
        raise ValueError("acc must be a contiguous float32 device tensor [T, n_q_heads, 128]")
    st = load_library().psattn_probe_dq_atomics(meta.handle, int(n_q_heads), int(n_kv_heads), acc.data_ptr(),
                                                int(mode), _stream_ptr(stream))
    _check(st, "psattn_probe_dq_atomics")


def psattn_trim_pool() -> None:
    _check(load_library().psattn_trim_pool(), "psattn_trim_pool")


def psattn_kernel_name(dt, kernel_pass) -> str:
    return load_library().psattn_kernel_name(int(dt), int(kernel_pass)).decode()


def psattn_profile_enable(on: bool) -> None:
    _check(load_library().psattn_profile_enable(1 if on else 0), "psattn_profile_enable")


def psattn_profile_read():
    """Returns (sum_ms[4], count[4]) per pass: 0 forward, 2 dQ with delta, 3 dK/dV or a backward in one launch (1: none)."""
    ms = np.zeros(4, dtype=np.float64)
    cnt = np.zeros(4, dtype=np.int64)
    _check(load_library().psattn_profile_read(ms.ctypes.data, cnt.ctypes.data), "psattn_profile_read")
    return ms, cnt
