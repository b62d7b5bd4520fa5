"""Python binding of libsepllm: argument marshalling only.

Every function has the name of the C entry point it calls (see include/sepllm.h)
and passes torch tensors' device pointers and the current CUDA stream through.
Nothing here computes: if the shared library is missing the import fails.
"""
from __future__ import annotations

import ctypes as C
import functools
import os
import struct

import numpy as np
import torch

_HERE = os.path.dirname(os.path.abspath(__file__))
LIB_PATH = os.path.join(_HERE, "libsepllm.so")

OK, INVALID_ARG, UNSUPPORTED, BUFFER_TOO_SMALL, CUDA_ERROR, CAPACITY_EXCEEDED, TIMEOUT, NOT_BUILT = range(8)


class IndexDesc(C.Structure):
    _fields_ = [(n, C.c_int32) for n in ("B", "L", "n_init", "n_neighbor", "n_sep", "BM", "BN", "side_cap")]


SIDE_READY = 1


class AttnDesc(C.Structure):
    _fields_ = [("B", C.c_int32), ("Hq", C.c_int32), ("Hkv", C.c_int32), ("d", C.c_int32),
                ("L", C.c_int32), ("scale", C.c_float), ("grad_dtype", C.c_int32),
                ("flags", C.c_int32), ("events", C.POINTER(C.c_void_p)), ("n_events", C.c_int32)]

    def set_events(self, events):
        """events: torch.cuda.Event objects (timing enabled, recorded once so their handles
        exist), or None to switch per-kernel timing off."""
        if not events:
            self.events, self.n_events, self._keep = None, 0, None
            return
        arr = (C.c_void_p * len(events))(*[e.cuda_event for e in events])
        self._keep = arr
        self.events = C.cast(arr, C.POINTER(C.c_void_p))
        self.n_events = len(events)


CACHE_FIXED_WINDOW = 1


class CacheDesc(C.Structure):
    _fields_ = [(n, C.c_int32) for n in ("B", "Hkv", "Hq", "d", "a", "s", "w", "c", "flags")]


ROPE_LAYOUTS = {"half": 0, "interleaved": 1}
ROPE_SCALINGS = {"none": 0, "linear": 1, "ntk": 2, "yarn": 3, "llama3": 4, "factors": 5}
_ROPE_DTYPES = {torch.bfloat16: 0, torch.float32: 1}


class RopeDesc(C.Structure):
    """sepllm_rope_desc.  rot_dim 0 = d; layout and scaling by name; high defaults to 32 for "yarn" and
    4 otherwise; freq_factors: a sequence of rot_dim / 2 numbers; pos_stride defaults to L (positions
    [B][L])."""
    _fields_ = ([(n, C.c_int32) for n in ("B", "L", "Hq", "Hkv", "d", "rot_dim", "layout", "scaling")]
                + [(n, C.c_double) for n in ("base", "factor", "low", "high", "orig_len", "attn_factor")]
                + [("freq_factors", C.POINTER(C.c_double)), ("pos_first", C.c_int64), ("pos_stride", C.c_int64)])

    def __init__(self, B, L, Hq, Hkv, d, rot_dim=0, layout="half", scaling="none", base=10000.0, factor=1.0,
                 low=1.0, high=None, orig_len=8192.0, attn_factor=0.0, freq_factors=None, pos_first=0,
                 pos_stride=None):
        if high is None:
            high = 32.0 if scaling in ("yarn", ROPE_SCALINGS["yarn"]) else 4.0
        self._keep = None
        if freq_factors is not None:
            n = (rot_dim or d) // 2
            if len(freq_factors) != n:
                raise ValueError(f"freq_factors has {len(freq_factors)} entries, not rot_dim / 2 = {n}")
            self._keep = (C.c_double * n)(*freq_factors)
        super().__init__(B, L, Hq, Hkv, d, rot_dim, ROPE_LAYOUTS.get(layout, layout),
                         ROPE_SCALINGS.get(scaling, scaling), base, factor, low, high, orig_len, attn_factor,
                         C.cast(self._keep, C.POINTER(C.c_double)) if self._keep else None, pos_first,
                         L if pos_stride is None else pos_stride)


class QkNorm(C.Structure):
    """sepllm_qknorm_desc.  wq, wk: bf16 or fp32 [d] tensors of one type, or None.  Every call takes the tensors as they
    are then: their address and their type (Module.to() changes both in place)."""
    _fields_ = [("wq", C.c_void_p), ("wk", C.c_void_p), ("w_dtype", C.c_int32), ("eps", C.c_float),
                ("offset", C.c_float)]

    def __init__(self, wq=None, wk=None, eps=1e-6, offset=0.0):
        self.weights = (wq, wk)     # (kept alive, and looked at by every call)
        super().__init__(None, None, self.type_now(), eps, offset)

    def type_now(self) -> int:
        types = {w.dtype for w in self.weights if w is not None}
        if len(types) > 1 or not types <= _ROPE_DTYPES.keys():
            raise ValueError(f"the weights are bf16 or fp32, both of one type, not {sorted(map(str, types))}")
        return _ROPE_DTYPES[types.pop()] if types else 0


class IndexHeader(C.Structure):
    _fields_ = [("status", C.c_int32), ("magic", C.c_uint32), ("version", C.c_uint32),
                ("desc", IndexDesc), ("n_tiles", C.c_int32),
                ("off_cnt", C.c_int64), ("off_lim", C.c_int64), ("off_side_pos", C.c_int64),
                ("off_n_side", C.c_int64), ("off_tile_meta", C.c_int64), ("total_bytes", C.c_int64),
                ("off_seq_len", C.c_int64), ("off_doc_start", C.c_int64), ("off_doc_end", C.c_int64),
                ("packed", C.c_int64), ("reserved", C.c_int64 * 16)]


class CacheHeader(C.Structure):
    _fields_ = [("status", C.c_int32), ("magic", C.c_uint32), ("version", C.c_uint32),
                ("slots", C.c_int32), ("desc", CacheDesc),
                ("off_seq", C.c_int64), ("off_slot_pos", C.c_int64), ("off_slot_is_sep", C.c_int64),
                ("total_bytes", C.c_int64), ("reserved", C.c_int64 * 21)]


EXPORTS = [
    "sepllm_index_bytes", "sepllm_build_index", "sepllm_build_index_varlen", "sepllm_build_index_packed",
    "sepllm_build_index_static",
    "sepllm_build_index_fixed_interval",
    "sepllm_attn_workspace_bytes", "sepllm_attn_fwd",
    "sepllm_attn_bwd", "sepllm_cache_bytes", "sepllm_cache_init", "sepllm_cache_update",
    "sepllm_cache_from_prompt", "sepllm_cache_update_rope",
    "sepllm_decode_workspace_bytes", "sepllm_decode", "sepllm_rope_table_bytes",
    "sepllm_rope_table_build", "sepllm_decode_rope", "sepllm_last_device_status",
    "sepllm_rope_frequencies", "sepllm_rope_fwd", "sepllm_rope_bwd",
    "sepllm_prefix_from_cache", "sepllm_decode_prefix_workspace_bytes", "sepllm_decode_prefix",
    "sepllm_attn_prefix_workspace_bytes", "sepllm_attn_prefix_fwd",
    "sepllm_qknorm_rope_fwd", "sepllm_qknorm_rope_bwd_workspace_bytes", "sepllm_qknorm_rope_bwd",
    "sepllm_cache_bytes_quant", "sepllm_cache_update_quant", "sepllm_cache_from_prompt_quant",
    "sepllm_cache_entries_quant", "sepllm_decode_quant_workspace_bytes", "sepllm_decode_quant",
    "sepllm_status_string",
]

# Calls of the per-token and per-layer kind take plain integers as addresses (ctypes converts them
# faster than it builds an object for each).
_P, _I = C.c_void_p, C.c_int32
_ARGTYPES = {
    "sepllm_rope_fwd": [_P] * 5, "sepllm_rope_bwd": [_P] * 5,
    "sepllm_prefix_from_cache": [_P] * 4 + [_I] + [_P] * 3 + [_I, _P],
    "sepllm_decode_prefix": [_P, _I, C.c_float] + [_P] * 11,
    "sepllm_attn_prefix_fwd": [_P, _P, _I] + [_P] * 11,
    "sepllm_qknorm_rope_fwd": [_P] * 6, "sepllm_qknorm_rope_bwd": [_P] * 10,
    "sepllm_cache_update_quant": [_P] * 6 + [_I] + [_P] * 3,
    "sepllm_cache_from_prompt_quant": [_P] * 10,
    "sepllm_cache_entries_quant": [_P] * 4 + [_I] + [_P] * 4,
    "sepllm_decode_quant": [_P, C.c_float] + [_P] * 8,
}

_lib = None


def lib() -> C.CDLL:
    """Loads libsepllm.so; raises if it has not been built."""
    global _lib
    if _lib is None:
        if not os.path.exists(LIB_PATH):
            raise RuntimeError(f"{LIB_PATH} is missing: run paper_2412_12094_b200/build.py "
                               "(there is no fallback path)")
        _lib = C.CDLL(LIB_PATH)
        _lib.sepllm_status_string.restype = C.c_char_p
        _lib.sepllm_status_string.argtypes = [C.c_int]
        for name in EXPORTS:
            if name != "sepllm_status_string":
                getattr(_lib, name).restype = C.c_int
        for name, types in _ARGTYPES.items():
            getattr(_lib, name).argtypes = types
    return _lib


class SepllmError(RuntimeError):
    def __init__(self, code: int, where: str):
        self.code = code
        super().__init__(f"{where}: {lib().sepllm_status_string(code).decode()} ({code})")


def _check(code: int, where: str):
    if code != OK:
        raise SepllmError(code, where)


def _ptr(t):
    if t is None:
        return C.c_void_p(0)
    if isinstance(t, torch.Tensor):
        assert t.is_cuda and t.is_contiguous(), "device, contiguous tensors only"
        return C.c_void_p(t.data_ptr())
    return C.c_void_p(int(t))


def _stream():
    return C.c_void_p(_raw_stream())


def _raw_stream() -> int:
    # the handle of torch.cuda.current_stream() without the Python object around it (3 us a call)
    return torch._C._cuda_getCurrentRawStream(torch.cuda.current_device())


def _addresses(where, tensors):
    """Device addresses (0 for None) of contiguous tensors of the current device: the calls launch on
    it and on its current stream, so memory of another device is refused here rather than read from
    there."""
    cur = torch.cuda.current_device()
    out = []
    for t in tensors:
        if t is None:
            out.append(0)
        elif t.get_device() != cur:
            raise ValueError(f"{where}: tensor on {t.device}, current device is cuda:{cur}: make the tensors' "
                             "device current for the call")
        elif not t.is_contiguous():
            raise ValueError(f"{where}: contiguous tensors only, not strides {t.stride()}")
        else:
            out.append(t.data_ptr())
    return out


def _short(t, need):
    """Whether a call would write or read past the buffer's end (None: the library's to refuse)."""
    return t is not None and t.nbytes < need


def _refuse_short(where, *buffers):
    for what, t, need in buffers:
        if _short(t, need):
            raise ValueError(f"{where}: {what} has {t.nbytes} bytes, the descriptor needs {need}")


def _sep_array(sep_ids):
    arr = np.ascontiguousarray(np.asarray(sep_ids, dtype=np.int32))
    return arr, arr.ctypes.data_as(C.c_void_p), int(arr.size)


def _sep_bytes(sep_ids):
    """Separator ids as the int32 array that a C entry point reads during the call, and their number."""
    if isinstance(sep_ids, np.ndarray) and sep_ids.dtype == np.int32 and sep_ids.ndim == 1:
        return sep_ids.tobytes(), sep_ids.size
    return struct.pack(f"={len(sep_ids)}i", *sep_ids), len(sep_ids)


def status_string(code: int) -> str:
    return lib().sepllm_status_string(code).decode()


# ---------------------------------------------------------------- index
def sepllm_index_bytes(desc: IndexDesc):
    ib, sb = C.c_size_t(0), C.c_size_t(0)
    _check(lib().sepllm_index_bytes(C.byref(desc), C.byref(ib), C.byref(sb)), "sepllm_index_bytes")
    return ib.value, sb.value


def sepllm_build_index(desc: IndexDesc, token_ids: torch.Tensor, sep_ids, index: torch.Tensor,
                       scratch: torch.Tensor):
    arr, p, n = _sep_array(sep_ids)
    assert n == desc.n_sep
    _check(lib().sepllm_build_index(C.byref(desc), _ptr(token_ids), p, _ptr(index), _ptr(scratch),
                                    _stream()), "sepllm_build_index")


def sepllm_build_index_varlen(desc: IndexDesc, token_ids: torch.Tensor, seq_len: torch.Tensor, sep_ids,
                              index: torch.Tensor, scratch: torch.Tensor):
    arr, p, n = _sep_array(sep_ids)
    assert n == desc.n_sep
    _check(lib().sepllm_build_index_varlen(C.byref(desc), _ptr(token_ids), _ptr(seq_len), p, _ptr(index),
                                           _ptr(scratch), _stream()), "sepllm_build_index_varlen")


def sepllm_build_index_packed(desc: IndexDesc, token_ids: torch.Tensor, doc_first: torch.Tensor, seq_len,
                              sep_ids, index: torch.Tensor):
    """Index of rows that pack several documents (doc_first [B][L] int32, non-zero where a document
    begins; seq_len [B] int32 or None)."""
    arr, p, n = _sep_array(sep_ids)
    assert n == desc.n_sep
    _check(lib().sepllm_build_index_packed(C.byref(desc), _ptr(token_ids), _ptr(doc_first), _ptr(seq_len), p,
                                           _ptr(index), _ptr(None), _stream()), "sepllm_build_index_packed")


def sepllm_build_index_static(desc: IndexDesc, token_ids: torch.Tensor, sep_ids, index: torch.Tensor):
    """Index build for callers that cannot allocate a scratch buffer: the library's own fixed
    array is used instead (B * (2 * ceil(L/4096) + 1) <= 65536).  Calls that may overlap on the GPU must be
    serialised by the caller; make the first call on a device outside any stream capture."""
    arr, p, n = _sep_array(sep_ids)
    assert n == desc.n_sep
    _check(lib().sepllm_build_index_static(C.byref(desc), _ptr(token_ids), p, _ptr(index), _stream()),
           "sepllm_build_index_static")


def sepllm_build_index_fixed_interval(desc: IndexDesc, interval: int, index: torch.Tensor,
                                      scratch: torch.Tensor):
    _check(lib().sepllm_build_index_fixed_interval(C.byref(desc), C.c_int32(interval), _ptr(index),
                                                   _ptr(scratch), _stream()),
           "sepllm_build_index_fixed_interval")


def read_index(index: torch.Tensor) -> dict:
    """Copies an index blob to the host and splits it into its arrays (for tests)."""
    raw = index.cpu().numpy().tobytes()
    h = IndexHeader.from_buffer_copy(raw[:256])
    d = h.desc
    T = h.n_tiles

    def arr(off, count):
        return np.frombuffer(raw, dtype=np.int32, count=count, offset=off).copy()

    return dict(
        header=h,
        cnt=arr(h.off_cnt, d.B * (d.L + 1)).reshape(d.B, d.L + 1),
        lim=arr(h.off_lim, d.B * d.L).reshape(d.B, d.L),
        side_pos=arr(h.off_side_pos, d.B * d.side_cap).reshape(d.B, d.side_cap),
        n_side=arr(h.off_n_side, d.B),
        tile_meta=arr(h.off_tile_meta, d.B * T * 8).reshape(d.B, T, 8),
        seq_len=arr(h.off_seq_len, d.B),
        doc_start=arr(h.off_doc_start, d.B * d.L).reshape(d.B, d.L),
        doc_end=arr(h.off_doc_end, d.B * d.L).reshape(d.B, d.L),
    )


# ---------------------------------------------------------------- attention
def sepllm_attn_workspace_bytes(desc: AttnDesc, idesc: IndexDesc):
    f, b = C.c_size_t(0), C.c_size_t(0)
    _check(lib().sepllm_attn_workspace_bytes(C.byref(desc), C.byref(idesc), C.byref(f), C.byref(b)),
           "sepllm_attn_workspace_bytes")
    return f.value, b.value


def sepllm_attn_fwd(desc, idesc, Q, K, V, index, O, LSE, workspace):
    _check(lib().sepllm_attn_fwd(C.byref(desc), C.byref(idesc), _ptr(Q), _ptr(K), _ptr(V), _ptr(index),
                                 _ptr(O), _ptr(LSE), _ptr(workspace), _stream()), "sepllm_attn_fwd")


def sepllm_attn_bwd(desc, idesc, dO, Q, K, V, O, LSE, index, dQ, dK, dV, workspace):
    _check(lib().sepllm_attn_bwd(C.byref(desc), C.byref(idesc), _ptr(dO), _ptr(Q), _ptr(K), _ptr(V),
                                 _ptr(O), _ptr(LSE), _ptr(index), _ptr(dQ), _ptr(dK), _ptr(dV),
                                 _ptr(workspace), _stream()), "sepllm_attn_bwd")


# ---------------------------------------------------------------- rotary positions
def sepllm_rope_frequencies(desc: RopeDesc):
    """(frequencies [rot_dim / 2] as numpy float64, factor on the rotated pair)."""
    f, m = np.zeros(64), C.c_double(0.0)
    _check(lib().sepllm_rope_frequencies(C.byref(desc), f.ctypes.data_as(C.c_void_p), C.byref(m)),
           "sepllm_rope_frequencies")
    return f[:(desc.rot_dim or desc.d) // 2].copy(), m.value


_ROPE_VIEWS = struct.Struct("=" + "Qqqqii" * 3)   # three sepllm_rope_view


def _rope_views(desc, tensors, what, device=None):
    """The views of (q, k, v), or of inputs and outputs, one bytes object per three tensors."""
    B, L, d = desc.B, desc.L, desc.d
    q_shape, k_shape = (B, desc.Hq, L, d), (B, desc.Hkv, L, d)
    vals, shapes, dtypes = [], (q_shape, k_shape, k_shape) * 3, _ROPE_DTYPES
    for t, shape in zip(tensors, shapes):
        if t is None:
            vals += (0, 0, 0, 0, 0, 0)
            continue
        sb, sh, sl, se = t.stride()
        dtype = dtypes.get(t.dtype)
        if t.shape != shape or dtype is None or se != 1 or (device is not None and t.get_device() != device):
            _refuse_view(t, shape, what, device)
        vals += (t.data_ptr(), sb, sh, sl, dtype, 0)
    return [_ROPE_VIEWS.pack(*vals[i:i + 18]) for i in range(0, len(vals), 18)]


def _refuse_view(t, shape, what, device):
    if t.shape != shape:
        raise ValueError(f"{what}: shape {tuple(t.shape)}, the descriptor says {shape}")
    if t.dtype not in _ROPE_DTYPES or t.stride(3) != 1:
        raise ValueError(f"{what}: bf16 or fp32 with contiguous head vectors, not {t.dtype} with strides {t.stride()}")
    raise ValueError(f"{what}: tensor on {t.device}, current device is cuda:{device}: make the tensors' device current "
                     "for the call")


def _positions(where, desc, positions):
    if positions is None:
        return 0
    pos, = _addresses(where, (positions,))
    if positions.dtype != torch.int64 or positions.numel() < (desc.B - 1) * desc.pos_stride + desc.L:
        raise ValueError(f"{where}: positions are contiguous int64, pos_stride elements from row to row")
    return pos


def _rope(fn, where, desc, positions, tensors):
    device = torch.cuda.current_device()
    pos = _positions(where, desc, positions)
    ins, outs = _rope_views(desc, tensors, where, device)
    _check(fn(C.byref(desc), pos, ins, outs, torch._C._cuda_getCurrentRawStream(device)), where)


def sepllm_rope_fwd(desc: RopeDesc, positions, q, k, v, q_out, k_out, v_out):
    """Rotates q and k and copies v.  Every tensor is [B][H][L][d] with any strides (the last one 1), so a
    slice of a fused projection goes in as qkv.view(B, L, Hq + 2 * Hkv, d).transpose(1, 2).split(...);
    a tensor and its output may both be None.  positions: int64 [B][L] (see desc.pos_stride) or None."""
    _rope(lib().sepllm_rope_fwd, "sepllm_rope_fwd", desc, positions, (q, k, v, q_out, k_out, v_out))


def sepllm_rope_bwd(desc: RopeDesc, positions, dq_out, dk_out, dv_out, dq, dk, dv):
    """Gradients of sepllm_rope_fwd's inputs from those of its outputs."""
    _rope(lib().sepllm_rope_bwd, "sepllm_rope_bwd", desc, positions,
          (dq_out, dk_out, dv_out, dq, dk, dv))


# ---------------------------------------------------------------- head norms with rotary positions
def _weights(where, desc, norm, device):
    """Puts the weights' type and addresses into the descriptor."""
    dtype, addresses = None, []
    for w in norm.weights:
        if w is None:
            addresses.append(None)
            continue
        if w.shape != (desc.d,) or not w.is_contiguous() or w.get_device() != device:
            raise ValueError(f"{where}: weights are contiguous [{desc.d}] tensors of the current device, not {tuple(w.shape)} "
                             f"with stride {w.stride()} on {w.device}")
        if w.dtype is not dtype:
            if dtype is not None or w.dtype not in _ROPE_DTYPES:
                norm.type_now()     # (refuses them)
            dtype = w.dtype
        addresses.append(w.data_ptr())
    norm.w_dtype = _ROPE_DTYPES.get(dtype, 0)
    norm.wq, norm.wk = addresses


def sepllm_qknorm_rope_fwd(desc: RopeDesc, norm: QkNorm, positions, q, k, v, q_out, k_out, v_out):
    """sepllm_rope_fwd with every head of q and k normalised first.  Other arguments as there."""
    where, device = "sepllm_qknorm_rope_fwd", torch.cuda.current_device()
    _weights(where, desc, norm, device)
    pos = _positions(where, desc, positions)
    ins, outs = _rope_views(desc, (q, k, v, q_out, k_out, v_out), where, device)
    _check(lib().sepllm_qknorm_rope_fwd(C.byref(desc), C.byref(norm), pos, ins, outs,
                                        torch._C._cuda_getCurrentRawStream(device)), where)


def sepllm_qknorm_rope_bwd_workspace_bytes(desc: RopeDesc):
    b = C.c_size_t(0)
    _check(lib().sepllm_qknorm_rope_bwd_workspace_bytes(C.byref(desc), C.byref(b)),
           "sepllm_qknorm_rope_bwd_workspace_bytes")
    return b.value


@functools.lru_cache(maxsize=16)
def _norm_workspace(library, d):
    return sepllm_qknorm_rope_bwd_workspace_bytes(RopeDesc(1, 1, 1, 1, d))


def sepllm_qknorm_rope_bwd(desc: RopeDesc, norm: QkNorm, positions, q, k, dq_out, dk_out, dv_out, dq, dk, dv, dwq,
                           dwk, workspace):
    """Gradients of sepllm_qknorm_rope_fwd's inputs and weights; q, k: the forward's inputs; dwq, dwk: fp32 [d]
    or None."""
    where, device = "sepllm_qknorm_rope_bwd", torch.cuda.current_device()
    _weights(where, desc, norm, device)
    pos = _positions(where, desc, positions)
    xs, ins, outs = _rope_views(desc, (q, k, None, dq_out, dk_out, dv_out, dq, dk, dv), where, device)
    _expect(where, ("dwq", dwq, (desc.d,), torch.float32), ("dwk", dwk, (desc.d,), torch.float32))
    _refuse_short(where, ("workspace", workspace, _norm_workspace(lib(), desc.d)))
    _check(lib().sepllm_qknorm_rope_bwd(C.byref(desc), C.byref(norm), pos, xs, ins, outs,
                                        *_addresses(where, (dwq, dwk, workspace)),
                                        torch._C._cuda_getCurrentRawStream(device)), where)


# ---------------------------------------------------------------- cache
def sepllm_cache_bytes(desc: CacheDesc):
    s, k = C.c_size_t(0), C.c_size_t(0)
    _check(lib().sepllm_cache_bytes(C.byref(desc), C.byref(s), C.byref(k)), "sepllm_cache_bytes")
    return s.value, k.value


def sepllm_cache_init(desc, state):
    _check(lib().sepllm_cache_init(C.byref(desc), _ptr(state), _stream()), "sepllm_cache_init")


def sepllm_cache_update(desc, state, Kc, Vc, new_token_ids, sep_ids, k_new, v_new):
    arr, p, n = _sep_array(sep_ids)
    _check(lib().sepllm_cache_update(C.byref(desc), _ptr(state), _ptr(Kc), _ptr(Vc),
                                     _ptr(new_token_ids), p, C.c_int32(n), _ptr(k_new), _ptr(v_new),
                                     _stream()), "sepllm_cache_update")


def sepllm_cache_from_prompt(desc, idesc, index, prompt_len, K, V, state, Kc, Vc, Kr=None, rope_table=None):
    _check(lib().sepllm_cache_from_prompt(C.byref(desc), C.byref(idesc), _ptr(index), _ptr(prompt_len),
                                          _ptr(K), _ptr(V), _ptr(state), _ptr(Kc), _ptr(Vc), _ptr(Kr),
                                          _ptr(rope_table), _stream()),
           "sepllm_cache_from_prompt")


def sepllm_decode_workspace_bytes(desc):
    b = C.c_size_t(0)
    _check(lib().sepllm_decode_workspace_bytes(C.byref(desc), C.byref(b)), "sepllm_decode_workspace_bytes")
    return b.value


def sepllm_decode(desc, scale, q, state, Kc, Vc, o, lse, workspace):
    _check(lib().sepllm_decode(C.byref(desc), C.c_float(scale), _ptr(q), _ptr(state), _ptr(Kc), _ptr(Vc),
                               _ptr(o), _ptr(lse), _ptr(workspace), _stream()), "sepllm_decode")


def sepllm_rope_table_bytes(desc):
    b = C.c_size_t(0)
    _check(lib().sepllm_rope_table_bytes(C.byref(desc), C.byref(b)), "sepllm_rope_table_bytes")
    return b.value


def sepllm_rope_table_build(desc, rope_base, table):
    _check(lib().sepllm_rope_table_build(C.byref(desc), C.c_float(rope_base), _ptr(table), _stream()),
           "sepllm_rope_table_build")


def sepllm_cache_update_rope(desc, state, Kc, Vc, Kr, rope_table, new_token_ids, sep_ids, k_new, v_new):
    arr, p, n = _sep_array(sep_ids)
    _check(lib().sepllm_cache_update_rope(C.byref(desc), _ptr(state), _ptr(Kc), _ptr(Vc), _ptr(Kr),
                                          _ptr(rope_table), _ptr(new_token_ids), p, C.c_int32(n),
                                          _ptr(k_new), _ptr(v_new), _stream()), "sepllm_cache_update_rope")


def sepllm_decode_rope(desc, scale, q, state, Kr, Vc, rope_table, o, lse, workspace):
    _check(lib().sepllm_decode_rope(C.byref(desc), C.c_float(scale), _ptr(q), _ptr(state), _ptr(Kr),
                                    _ptr(Vc), _ptr(rope_table), _ptr(o), _ptr(lse), _ptr(workspace),
                                    _stream()), "sepllm_decode_rope")


# ---------------------------------------------------------------- shared prefix
def _expect(where, *tensors):
    """(name, tensor or None, shape, dtype) each."""
    for name, t, shape, dtype in tensors:
        if t is not None and (t.shape != shape or t.dtype != dtype):
            raise ValueError(f"{where}: {name} is {dtype} {tuple(shape)}, not {t.dtype} {tuple(t.shape)}")


def sepllm_prefix_from_cache(desc, state, Kc, Vc, P, Kp, Vp, prefix_len=None):
    """The retained entries of a cache of one sequence become rows 0 .. Size_run-1 of Kp, Vp [Hkv][P][d];
    prefix_len: int32 of any length, every word is set to Size_run, or None."""
    where = "sepllm_prefix_from_cache"
    shape, n = (desc.Hkv, P, desc.d), 0 if prefix_len is None else prefix_len.numel()
    _expect(where, ("Kp", Kp, shape, torch.bfloat16), ("Vp", Vp, shape, torch.bfloat16),
            ("prefix_len", prefix_len, (n,), torch.int32))
    st, kc, vc, kp, vp, pl = _addresses(where, (state, Kc, Vc, Kp, Vp, prefix_len))
    _check(lib().sepllm_prefix_from_cache(C.byref(desc), st, kc, vc, P, kp, vp, pl, n, _raw_stream()), where)


def sepllm_decode_prefix_workspace_bytes(desc, P):
    b = C.c_size_t(0)
    _check(lib().sepllm_decode_prefix_workspace_bytes(C.byref(desc), C.c_int32(P), C.byref(b)),
           "sepllm_decode_prefix_workspace_bytes")
    return b.value


def sepllm_decode_prefix(desc, P, scale, q, state, Kc, Vc, Kp, Vp, prefix_len, o, lse, workspace):
    """sepllm_decode with the shared prefix Kp, Vp [Hkv][P][d] in front of every cache; prefix_len: int32 [B]
    or None (all P rows); lse may be None."""
    where, bf, B, row = "sepllm_decode_prefix", torch.bfloat16, desc.B, (desc.B, desc.Hq, desc.d)
    shape = (desc.Hkv, P, desc.d)
    _expect(where, ("q", q, row, bf), ("Kp", Kp, shape, bf), ("Vp", Vp, shape, bf),
            ("prefix_len", prefix_len, (B,), torch.int32), ("o", o, row, bf),
            ("lse", lse, row[:2], torch.float32))
    _check(lib().sepllm_decode_prefix(C.byref(desc), P, scale, *_addresses(
        where, (q, state, Kc, Vc, Kp, Vp, prefix_len, o, lse, workspace)), _raw_stream()), where)


def sepllm_attn_prefix_workspace_bytes(desc: AttnDesc, idesc: IndexDesc, P):
    b = C.c_size_t(0)
    _check(lib().sepllm_attn_prefix_workspace_bytes(C.byref(desc), C.byref(idesc), C.c_int32(P), C.byref(b)),
           "sepllm_attn_prefix_workspace_bytes")
    return b.value


def sepllm_attn_prefix_fwd(desc, idesc, P, Q, K, V, index, Kp, Vp, prefix_len, O, LSE, workspace):
    """sepllm_attn_fwd with the shared prefix Kp, Vp [Hkv][P][d] in front of every sequence; prefix_len:
    int32 [B] or None (all P rows)."""
    where, bf, B, L = "sepllm_attn_prefix_fwd", torch.bfloat16, desc.B, desc.L
    row, key, shape = (B, desc.Hq, L, desc.d), (B, desc.Hkv, L, desc.d), (desc.Hkv, P, desc.d)
    _expect(where, ("Q", Q, row, bf), ("K", K, key, bf), ("V", V, key, bf), ("Kp", Kp, shape, bf),
            ("Vp", Vp, shape, bf), ("prefix_len", prefix_len, (B,), torch.int32), ("O", O, row, bf),
            ("LSE", LSE, row[:3], torch.float32))
    _check(lib().sepllm_attn_prefix_fwd(C.byref(desc), C.byref(idesc), P, *_addresses(
        where, (Q, K, V, index, Kp, Vp, prefix_len, O, LSE, workspace)), _raw_stream()), where)


# ---------------------------------------------------------------- cache in 4 bits
# (sizes by the descriptor's bytes: short calls are bound by the host)
@functools.lru_cache(maxsize=256)
def _quant_sizes(desc):
    d = CacheDesc.from_buffer_copy(desc)
    rows = d.B * (d.c + d.s)
    n = rows * d.Hkv * d.d
    state = 256 + (64 * d.B + 255 & -256) + (8 * rows + 255 & -256) + (rows + 255 & -256)
    return state, (n // 2 + 255 & -256) + (n // 16 + 255 & -256)


@functools.lru_cache(maxsize=256)
def _decode_quant_workspace(library, desc):
    return sepllm_decode_quant_workspace_bytes(CacheDesc.from_buffer_copy(desc))


@functools.lru_cache(maxsize=256)
def _index_size(library, idesc):
    return sepllm_index_bytes(IndexDesc.from_buffer_copy(idesc))[0]


def _quant_room(where, desc, state, Kc, Vc):
    raw = bytes(desc)
    n, kv = _quant_sizes(raw)
    if _short(state, n) or _short(Kc, kv) or _short(Vc, kv):
        _refuse_short(where, ("state", state, n), ("Kc", Kc, kv), ("Vc", Vc, kv))
    return raw


def sepllm_cache_bytes_quant(desc: CacheDesc):
    s, k = C.c_size_t(0), C.c_size_t(0)
    _check(lib().sepllm_cache_bytes_quant(C.byref(desc), C.byref(s), C.byref(k)), "sepllm_cache_bytes_quant")
    return s.value, k.value


def sepllm_cache_update_quant(desc, state, Kc, Vc, new_token_ids, sep_ids, k_new, v_new):
    """sepllm_cache_update for a cache held in 4 bits (Kc, Vc: sepllm_cache_bytes_quant)."""
    where, row = "sepllm_cache_update_quant", (desc.B, desc.Hkv, desc.d)
    p, n = _sep_bytes(sep_ids)
    _expect(where, ("new_token_ids", new_token_ids, (desc.B,), torch.int32), ("k_new", k_new, row, torch.bfloat16),
            ("v_new", v_new, row, torch.bfloat16))
    _quant_room(where, desc, state, Kc, Vc)
    st, kc, vc, ids, kn, vn = _addresses(where, (state, Kc, Vc, new_token_ids, k_new, v_new))
    _check(lib().sepllm_cache_update_quant(C.byref(desc), st, kc, vc, ids, p, n, kn, vn, _raw_stream()), where)


def sepllm_cache_from_prompt_quant(desc, idesc, index, prompt_len, K, V, state, Kc, Vc):
    """sepllm_cache_from_prompt for a cache held in 4 bits; prompt_len: int32 [B] or None."""
    where, bf, rows = "sepllm_cache_from_prompt_quant", torch.bfloat16, (desc.B, desc.Hkv, idesc.L, desc.d)
    _expect(where, ("prompt_len", prompt_len, (desc.B,), torch.int32), ("K", K, rows, bf), ("V", V, rows, bf))
    _quant_room(where, desc, state, Kc, Vc)
    _refuse_short(where, ("index", index, _index_size(lib(), bytes(idesc))))
    _check(lib().sepllm_cache_from_prompt_quant(C.byref(desc), C.byref(idesc), *_addresses(
        where, (index, prompt_len, K, V, state, Kc, Vc)), _raw_stream()), where)


def sepllm_cache_entries_quant(desc, state, Kc, Vc, n, K, V, length=None):
    """The retained entries of a cache held in 4 bits, in order, as bf16 rows 0 .. Size_run-1 of K, V
    [B][Hkv][n][d]; length: int32 [B] that receives Size_run, or None."""
    where, bf, rows = "sepllm_cache_entries_quant", torch.bfloat16, (desc.B, desc.Hkv, n, desc.d)
    _expect(where, ("K", K, rows, bf), ("V", V, rows, bf), ("length", length, (desc.B,), torch.int32))
    _quant_room(where, desc, state, Kc, Vc)
    st, kc, vc, k, v, ln = _addresses(where, (state, Kc, Vc, K, V, length))
    _check(lib().sepllm_cache_entries_quant(C.byref(desc), st, kc, vc, n, k, v, ln, _raw_stream()), where)


def sepllm_decode_quant_workspace_bytes(desc):
    b = C.c_size_t(0)
    _check(lib().sepllm_decode_quant_workspace_bytes(C.byref(desc), C.byref(b)),
           "sepllm_decode_quant_workspace_bytes")
    return b.value


def sepllm_decode_quant(desc, scale, q, state, Kc, Vc, o, lse, workspace):
    """sepllm_decode over a cache held in 4 bits; lse may be None."""
    where, row = "sepllm_decode_quant", (desc.B, desc.Hq, desc.d)
    _expect(where, ("q", q, row, torch.bfloat16), ("o", o, row, torch.bfloat16), ("lse", lse, row[:2], torch.float32))
    raw, library = _quant_room(where, desc, state, Kc, Vc), lib()
    need = _decode_quant_workspace(library, raw)
    if _short(workspace, need):
        _refuse_short(where, ("workspace", workspace, need))
    _check(library.sepllm_decode_quant(C.byref(desc), scale, *_addresses(where, (q, state, Kc, Vc, o, lse, workspace)),
                                     _raw_stream()), where)


def read_cache_state(state: torch.Tensor) -> dict:
    """Copies a cache state to the host: per-sequence records and slot metadata (for tests)."""
    raw = state.cpu().numpy().tobytes()
    h = CacheHeader.from_buffer_copy(raw[:256])
    B, slots = h.desc.B, h.slots
    seq = np.frombuffer(raw, dtype=np.int32, count=B * 16, offset=h.off_seq).reshape(B, 16).copy()
    next_pos = np.frombuffer(raw, dtype=np.int64, count=B * 8, offset=h.off_seq).reshape(B, 8)[:, 3].copy()
    pos = np.frombuffer(raw, dtype=np.int64, count=B * slots, offset=h.off_slot_pos).reshape(B, slots).copy()
    flag = np.frombuffer(raw, dtype=np.uint8, count=B * slots, offset=h.off_slot_is_sep).reshape(B, slots).copy()
    return dict(header=h, size_init=seq[:, 0], sep_start=seq[:, 1], size_sep=seq[:, 2],
                win_start=seq[:, 3], size_win=seq[:, 4], compactions=seq[:, 5], next_pos=next_pos,
                slot_pos=pos, slot_is_sep=flag)


def sepllm_last_device_status(buffer) -> int:
    out = C.c_int32(0)
    _check(lib().sepllm_last_device_status(_ptr(buffer), C.byref(out), _stream()),
           "sepllm_last_device_status")
    return out.value


# ---------------------------------------------------------------- allocation helpers (torch = memory only)
def alloc_bytes(n: int, device="cuda") -> torch.Tensor:
    """A 256-byte aligned uint8 device buffer of at least n bytes."""
    t = torch.empty(n + 256, dtype=torch.uint8, device=device)
    off = (-t.data_ptr()) % 256
    return t[off:off + n]
