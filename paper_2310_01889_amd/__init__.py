"""Python binding of libringattn.so, the MI355X (gfx950) ring-attention library.

Argument marshalling only: every step of the computation runs in the library's HIP
kernels.  torch supplies device memory and the current HIP stream.  Each function has
the name of the C entry point it calls (see include/ringattn.h for layouts, ownership
and error behaviour) and takes torch tensors that live on the current GPU; shapes are
read from the tensors.  Convenience wrappers that allocate their outputs are provided
for tests and benchmarks (``attention_fwd``, ``attention_bwd``, ``ffn_fwd``...).

The library is loaded on first use.  If it has not been built, or no GPU is present,
calls raise: there is no fallback path.
"""
import ctypes
import os

import torch

__all__ = [
    "RingAttnError", "library_path", "load", "exported_symbols",
    "ring_attn_fwd", "ring_attn_bwd", "ring_attn_fwd_f32", "ring_attn_bwd_f32",
    "ring_attn_fwd_host", "ring_attn_bwd_host", "ring_attn_fwd_ordered", "ring_attn_decode",
    "ring_attn_decode_noalloc",
    "blockwise_ffn", "blockwise_ffn_bwd",
    "blockwise_linear", "blockwise_linear_bwd", "ring_layer_fwd", "ring_layer_bwd",
    "rms_norm_fwd", "rms_norm_bwd", "rope_apply", "swiglu_ffn", "swiglu_ffn_bwd",
    "llama_layer_fwd", "llama_layer_bwd", "llama_stack_train_step",
    "paged_plan", "paged_append", "paged_attn_workspace", "paged_attn_decode", "mx4_pack", "mx4_linear",
    "attention_fwd", "attention_bwd", "attention_decode", "paged_attention", "mx4_weights",
    "PLAN_PAGES", "PLAN_CAPACITY", "PLAN_ROWS", "PLAN_BAD_INPUT",
    "ACT_GELU_ERF", "ACT_RELU", "ACT_GELU_TANH",
]

ACT_GELU_ERF, ACT_RELU, ACT_GELU_TANH = 0, 1, 2
PLAN_PAGES, PLAN_CAPACITY, PLAN_ROWS, PLAN_BAD_INPUT = 1, 2, 4, 8  # flags in counts[3] of paged_plan
_HERE = os.path.dirname(os.path.abspath(__file__))
_LIB = None

_P = ctypes.c_void_p
_I = ctypes.c_int
_SIGS = {
    "ring_attn_mfma_probe": [ctypes.c_int, ctypes.c_int, ctypes.c_void_p, ctypes.c_void_p],
    "ring_attn_release_workspace": [],
    "ring_attn_fwd": [_P] * 5 + [_I] * 6 + [_P],
    "ring_attn_fwd_f32": [_P] * 5 + [_I] * 6 + [_P],
    "ring_attn_bwd": [_P] * 9 + [_I] * 6 + [_P],
    "ring_attn_bwd_f32": [_P] * 9 + [_I] * 6 + [_P],
    "ring_attn_fwd_varlen": [_P] * 5 + [_I] * 5 + [_P],
    "ring_attn_bwd_varlen": [_P] * 9 + [_I] * 5 + [_P],
    "ring_attn_fwd_host": [_P] * 5 + [_I] * 7 + [_P],
    "ring_attn_bwd_host": [_P] * 9 + [_I] * 7 + [_P],
    "ring_attn_fwd_ordered": [_P] * 5 + [_I] * 6 + [_P, _P],
    "ring_attn_decode": [_P] * 5 + [_I] * 7 + [_P],
    "ring_attn_decode_noalloc": [_P] * 5 + [_I] * 7 + [_P],
    "blockwise_ffn": [_P] * 6 + [_I] * 5 + [_P],
    "blockwise_ffn_bwd": [_P] * 10 + [_I] * 5 + [_P],
    "blockwise_linear": [_P] * 4 + [_I] * 4 + [_P],
    "blockwise_linear_bwd": [_P] * 5 + [_I] * 4 + [_P],
    "ring_layer_fwd": [_P] * 8 + [_I] * 7 + [_P],
    "ring_layer_bwd": [_P] * 15 + [_I] * 7 + [_P],
    "rms_norm_fwd": [_P] * 4 + [_I] * 2 + [_P],
    "rms_norm_bwd": [_P] * 6 + [_I] * 2 + [_P],
    "rope_apply": [_P] + [_I] * 5 + [_P],
    "swiglu_ffn": [_P] * 6 + [_I] * 4 + [_P],
    "swiglu_ffn_bwd": [_P] * 9 + [_I] * 4 + [_P],
    "llama_layer_fwd": [_P] * 3 + [_I] * 6 + [_P],
    "llama_layer_bwd": [_P] * 5 + [_I] * 6 + [_P],
    "llama_stack_train_step": [_P] * 6 + [_I] * 7 + [_P],
    "paged_plan": [_P] * 10 + [_I] * 6 + [_P],
    "paged_append": [_P] * 10 + [_I] * 11 + [_P],
    "paged_attn_workspace": [_I] * 5 + [_P],
    "paged_attn_decode": [_P] * 11 + [ctypes.c_size_t] + [_I] * 10 + [_P],
    "mx4_pack": [_P] * 3 + [_I] * 2 + [_P],
    "mx4_linear": [_P] * 5 + [_I] * 3 + [_P],
}


class RingAttnError(RuntimeError):
    """A library call returned a non-zero ra_status."""

    def __init__(self, name, code, msg):
        super().__init__("%s failed (status %d): %s" % (name, code, msg))
        self.code = code


def library_path():
    return os.path.join(_HERE, "libringattn.so")


def load():
    """Load the shared library (once).  Raises if it is missing."""
    global _LIB
    if _LIB is None:
        path = library_path()
        if not os.path.exists(path):
            raise RuntimeError("%s is not built; run __graft_entry__.build() or "
                               "python -m paper_2310_01889_amd.build" % path)
        lib = ctypes.CDLL(path)
        for name, args in _SIGS.items():
            fn = getattr(lib, name, None)
            if fn is None:  # checked by the symbol test; calling it raises AttributeError
                continue
            fn.argtypes = args
            fn.restype = ctypes.c_int
        lib.ring_attn_last_error.argtypes = []
        lib.ring_attn_last_error.restype = ctypes.c_char_p
        lib.ring_attn_timing_enable.argtypes = [ctypes.c_int]
        lib.ring_attn_timing_enable.restype = None
        lib.ring_attn_timing_read.argtypes = [ctypes.c_int, ctypes.POINTER(ctypes.c_double),
                                              ctypes.POINTER(ctypes.c_int)]
        lib.ring_attn_timing_read.restype = ctypes.c_int
        _LIB = lib
    return _LIB


def exported_symbols():
    """Names of the C entry points the binding expects the library to export."""
    return sorted(list(_SIGS) + ["ring_attn_last_error", "ring_attn_timing_enable",
                                 "ring_attn_timing_read"])


KERNEL_ATTN_FWD, KERNEL_ATTN_BWD, KERNEL_GEMM, KERNEL_DECODE = 0, 1, 2, 3


def timing_enable(on=True):
    """Bracket every later hot-kernel launch with timing events (ring_attn_timing_enable)."""
    load().ring_attn_timing_enable(1 if on else 0)


def timing_read(kind):
    """(total milliseconds, launches) of the timed launches of ``kind`` since the last read."""
    ms, n = ctypes.c_double(0.0), ctypes.c_int(0)
    lib = load()
    rc = lib.ring_attn_timing_read(int(kind), ctypes.byref(ms), ctypes.byref(n))
    if rc != 0:
        raise RingAttnError("ring_attn_timing_read", rc, lib.ring_attn_last_error().decode())
    return ms.value, n.value


def release_workspace():
    """Return the library's cached workspace on the current device to the driver."""
    _call("ring_attn_release_workspace")


MFMA_PROBE_WAVES = 2048


def mfma_probe(iters, random_operands=False, stream=None):
    """Launch the matrix-core calibration kernel (ring_attn_mfma_probe) on the current
    stream, with fixed or random operands; returns the flops it performs.  Time it with
    events around the call."""
    import torch
    sink = torch.empty(MFMA_PROBE_WAVES, dtype=torch.float32, device="cuda")
    _call("ring_attn_mfma_probe", int(iters), 1 if random_operands else 0, sink.data_ptr(), _stream(stream))
    return float(MFMA_PROBE_WAVES) * iters * 32 * 32768


def _call(name, *args):
    lib = load()
    rc = getattr(lib, name)(*args)
    if rc != 0:
        raise RingAttnError(name, rc, lib.ring_attn_last_error().decode())


def _ptr(t, dtype=None, name="tensor"):
    if t is None:
        return None
    if not t.is_cuda:
        raise ValueError("%s must be a GPU tensor" % name)
    if not t.is_contiguous():
        raise ValueError("%s must be contiguous" % name)
    if dtype is not None and t.dtype != dtype:
        raise TypeError("%s must be %s, got %s" % (name, dtype, t.dtype))
    return ctypes.c_void_p(t.data_ptr())


def _stream(stream=None):
    s = torch.cuda.current_stream() if stream is None else stream
    return ctypes.c_void_p(s.cuda_stream)


def _bshd(q):
    if q.dim() != 4:
        raise ValueError("expected a [B, S, H, D] tensor")
    return tuple(int(x) for x in q.shape)


# ----------------------------------------------------------------------------------
# C entry points (outputs passed in)
# ----------------------------------------------------------------------------------
def ring_attn_fwd(q, k, v, o, lse, n_hosts, causal, stream=None):
    B, S, H, D = _bshd(q)
    bf = torch.bfloat16
    _call("ring_attn_fwd", _ptr(q, bf, "q"), _ptr(k, bf, "k"), _ptr(v, bf, "v"), _ptr(o, bf, "o"),
          _ptr(lse, torch.float32, "lse"), B, H, S, D, int(n_hosts), int(causal), _stream(stream))


def ring_attn_fwd_f32(q, k, v, o, lse, n_hosts, causal, stream=None):
    B, S, H, D = _bshd(q)
    f = torch.float32
    _call("ring_attn_fwd_f32", _ptr(q, f, "q"), _ptr(k, f, "k"), _ptr(v, f, "v"), _ptr(o, f, "o"),
          _ptr(lse, f, "lse"), B, H, S, D, int(n_hosts), int(causal), _stream(stream))


def ring_attn_bwd(q, k, v, o, lse, dO, dq, dk, dv, n_hosts, causal, stream=None):
    B, S, H, D = _bshd(q)
    bf = torch.bfloat16
    _call("ring_attn_bwd", _ptr(q, bf, "q"), _ptr(k, bf, "k"), _ptr(v, bf, "v"), _ptr(o, bf, "o"),
          _ptr(lse, torch.float32, "lse"), _ptr(dO, bf, "dO"), _ptr(dq, bf, "dq"), _ptr(dk, bf, "dk"),
          _ptr(dv, bf, "dv"), B, H, S, D, int(n_hosts), int(causal), _stream(stream))


def ring_attn_bwd_f32(q, k, v, o, lse, dO, dq, dk, dv, n_hosts, causal, stream=None):
    B, S, H, D = _bshd(q)
    f = torch.float32
    _call("ring_attn_bwd_f32", _ptr(q, f, "q"), _ptr(k, f, "k"), _ptr(v, f, "v"), _ptr(o, f, "o"),
          _ptr(lse, f, "lse"), _ptr(dO, f, "dO"), _ptr(dq, f, "dq"), _ptr(dk, f, "dk"), _ptr(dv, f, "dv"),
          B, H, S, D, int(n_hosts), int(causal), _stream(stream))


def ring_attn_fwd_varlen(q, k, v, o, lse, n_hosts, stream=None):
    B, S, H, D = _bshd(q)
    bf = torch.bfloat16
    _call("ring_attn_fwd_varlen", _ptr(q, bf, "q"), _ptr(k, bf, "k"), _ptr(v, bf, "v"), _ptr(o, bf, "o"),
          _ptr(lse, torch.float32, "lse"), B, H, S, D, int(n_hosts), _stream(stream))


def ring_attn_bwd_varlen(q, k, v, o, lse, dO, dq, dk, dv, n_hosts, stream=None):
    B, S, H, D = _bshd(q)
    bf = torch.bfloat16
    _call("ring_attn_bwd_varlen", _ptr(q, bf, "q"), _ptr(k, bf, "k"), _ptr(v, bf, "v"), _ptr(o, bf, "o"),
          _ptr(lse, torch.float32, "lse"), _ptr(dO, bf, "dO"), _ptr(dq, bf, "dq"), _ptr(dk, bf, "dk"),
          _ptr(dv, bf, "dv"), B, H, S, D, int(n_hosts), _stream(stream))


def ring_attn_fwd_host(q_blk, k_all, v_all, o_blk, lse_blk, n_hosts, host_idx, causal, stream=None):
    B, c, H, D = _bshd(q_blk)
    S = int(k_all.shape[1])
    bf = torch.bfloat16
    _call("ring_attn_fwd_host", _ptr(q_blk, bf, "q_blk"), _ptr(k_all, bf, "k_all"), _ptr(v_all, bf, "v_all"),
          _ptr(o_blk, bf, "o_blk"), _ptr(lse_blk, torch.float32, "lse_blk"), B, H, S, D, int(n_hosts),
          int(host_idx), int(causal), _stream(stream))


def ring_attn_bwd_host(q_blk, k_all, v_all, o_blk, lse_blk, dO_blk, dq_blk, dk_acc, dv_acc, n_hosts, host_idx, causal,
                       stream=None):
    B, c, H, D = _bshd(q_blk)
    S = int(k_all.shape[1])
    bf, f = torch.bfloat16, torch.float32
    _call("ring_attn_bwd_host", _ptr(q_blk, bf, "q_blk"), _ptr(k_all, bf, "k_all"), _ptr(v_all, bf, "v_all"),
          _ptr(o_blk, bf, "o_blk"), _ptr(lse_blk, f, "lse_blk"), _ptr(dO_blk, bf, "dO_blk"), _ptr(dq_blk, bf, "dq_blk"),
          _ptr(dk_acc, f, "dk_acc"), _ptr(dv_acc, f, "dv_acc"), B, H, S, D, int(n_hosts), int(host_idx), int(causal),
          _stream(stream))


def ring_attn_fwd_ordered(q, k, v, o, lse, n_hosts, causal, kv_order, stream=None):
    B, S, H, D = _bshd(q)
    bf = torch.bfloat16
    flat = [int(x) for row in kv_order for x in row]
    arr = (ctypes.c_int * len(flat))(*flat)
    _call("ring_attn_fwd_ordered", _ptr(q, bf, "q"), _ptr(k, bf, "k"), _ptr(v, bf, "v"), _ptr(o, bf, "o"),
          _ptr(lse, torch.float32, "lse"), B, H, S, D, int(n_hosts), int(causal),
          ctypes.cast(arr, ctypes.c_void_p), _stream(stream))


def ring_attn_decode(q, k_cache, v_cache, o, lse, n_hosts, causal=True, stream=None):
    B, Tq, H, D = _bshd(q)
    S = int(k_cache.shape[1])
    bf = torch.bfloat16
    _call("ring_attn_decode", _ptr(q, bf, "q"), _ptr(k_cache, bf, "k_cache"), _ptr(v_cache, bf, "v_cache"),
          _ptr(o, bf, "o"), _ptr(lse, torch.float32, "lse"), B, H, S, D, Tq, int(n_hosts), int(causal),
          _stream(stream))


def ring_attn_decode_noalloc(q, k_cache, v_cache, o, lse, n_hosts, causal=True, stream=None):
    B, Tq, H, D = _bshd(q)
    S = int(k_cache.shape[1])
    bf = torch.bfloat16
    _call("ring_attn_decode_noalloc", _ptr(q, bf, "q"), _ptr(k_cache, bf, "k_cache"), _ptr(v_cache, bf, "v_cache"),
          _ptr(o, bf, "o"), _ptr(lse, torch.float32, "lse"), B, H, S, D, Tq, int(n_hosts), int(causal),
          _stream(stream))


def blockwise_ffn(x, w1, b1, w2, b2, y, block, act=ACT_GELU_ERF, stream=None):
    T, dm = (int(s) for s in x.shape)
    dff = int(w1.shape[1])
    bf = torch.bfloat16
    _call("blockwise_ffn", _ptr(x, bf, "x"), _ptr(w1, bf, "w1"), _ptr(b1, bf, "b1"), _ptr(w2, bf, "w2"),
          _ptr(b2, bf, "b2"), _ptr(y, bf, "y"), T, dm, dff, int(block), int(act), _stream(stream))


def blockwise_ffn_bwd(x, w1, b1, w2, dy, dx, dw1, db1, dw2, db2, block, act=ACT_GELU_ERF, stream=None):
    T, dm = (int(s) for s in x.shape)
    dff = int(w1.shape[1])
    bf, f = torch.bfloat16, torch.float32
    _call("blockwise_ffn_bwd", _ptr(x, bf, "x"), _ptr(w1, bf, "w1"), _ptr(b1, bf, "b1"), _ptr(w2, bf, "w2"),
          _ptr(dy, bf, "dy"), _ptr(dx, bf, "dx"), _ptr(dw1, f, "dw1"), _ptr(db1, f, "db1"), _ptr(dw2, f, "dw2"),
          _ptr(db2, f, "db2"), T, dm, dff, int(block), int(act), _stream(stream))


def blockwise_linear(x, w, residual, y, block, stream=None):
    T, di = (int(s) for s in x.shape)
    do = int(w.shape[1])
    bf = torch.bfloat16
    _call("blockwise_linear", _ptr(x, bf, "x"), _ptr(w, bf, "w"), _ptr(residual, bf, "residual"),
          _ptr(y, bf, "y"), T, di, do, int(block), _stream(stream))


def blockwise_linear_bwd(x, w, dy, dx, dw, block, stream=None):
    T, di = (int(s) for s in x.shape)
    do = int(w.shape[1])
    bf = torch.bfloat16
    _call("blockwise_linear_bwd", _ptr(x, bf, "x"), _ptr(w, bf, "w"), _ptr(dy, bf, "dy"), _ptr(dx, bf, "dx"),
          _ptr(dw, torch.float32, "dw"), T, di, do, int(block), _stream(stream))


def ring_layer_fwd(x, wq, wk, wv, wo, w1, w2, z, n_heads, n_hosts, causal=True, act=ACT_GELU_ERF, stream=None):
    S, dm = (int(s) for s in x.shape)
    dff = int(w1.shape[1])
    bf = torch.bfloat16
    _call("ring_layer_fwd", _ptr(x, bf, "x"), _ptr(wq, bf, "wq"), _ptr(wk, bf, "wk"), _ptr(wv, bf, "wv"),
          _ptr(wo, bf, "wo"), _ptr(w1, bf, "w1"), _ptr(w2, bf, "w2"), _ptr(z, bf, "z"), S, dm, int(n_heads), dff,
          int(n_hosts), int(causal), int(act), _stream(stream))


def ring_layer_bwd(x, wq, wk, wv, wo, w1, w2, dz, dx, dwq, dwk, dwv, dwo, dw1, dw2, n_heads, n_hosts, causal=True,
                   act=ACT_GELU_ERF, stream=None):
    S, dm = (int(s) for s in x.shape)
    dff = int(w1.shape[1])
    bf, f = torch.bfloat16, torch.float32
    _call("ring_layer_bwd", _ptr(x, bf, "x"), _ptr(wq, bf, "wq"), _ptr(wk, bf, "wk"), _ptr(wv, bf, "wv"),
          _ptr(wo, bf, "wo"), _ptr(w1, bf, "w1"), _ptr(w2, bf, "w2"), _ptr(dz, bf, "dz"), _ptr(dx, bf, "dx"),
          _ptr(dwq, f, "dwq"), _ptr(dwk, f, "dwk"), _ptr(dwv, f, "dwv"), _ptr(dwo, f, "dwo"), _ptr(dw1, f, "dw1"),
          _ptr(dw2, f, "dw2"), S, dm, int(n_heads), dff, int(n_hosts), int(causal), int(act), _stream(stream))


def rms_norm_fwd(x, g, y, rstd=None, stream=None):
    T, d = (int(s) for s in x.shape)
    bf = torch.bfloat16
    _call("rms_norm_fwd", _ptr(x, bf, "x"), _ptr(g, bf, "g"), _ptr(y, bf, "y"), _ptr(rstd, torch.float32, "rstd"),
          T, d, _stream(stream))


def rms_norm_bwd(x, g, dy, dres, dx, dg, stream=None):
    T, d = (int(s) for s in x.shape)
    bf, f = torch.bfloat16, torch.float32
    _call("rms_norm_bwd", _ptr(x, bf, "x"), _ptr(g, bf, "g"), _ptr(dy, f, "dy"), _ptr(dres, bf, "dres"),
          _ptr(dx, bf, "dx"), _ptr(dg, f, "dg"), T, d, _stream(stream))


def rope_apply(x, pos0=0, inverse=False, stream=None):
    """In place on a bf16 [S, H, D] tensor."""
    S, H, D = (int(s) for s in x.shape)
    _call("rope_apply", _ptr(x, torch.bfloat16, "x"), S, H, D, int(pos0), int(bool(inverse)), _stream(stream))


def swiglu_ffn(x, w1, w3, w2, residual, y, block, stream=None):
    T, dm = (int(s) for s in x.shape)
    dff = int(w1.shape[1])
    bf = torch.bfloat16
    _call("swiglu_ffn", _ptr(x, bf, "x"), _ptr(w1, bf, "w1"), _ptr(w3, bf, "w3"), _ptr(w2, bf, "w2"),
          _ptr(residual, bf, "residual"), _ptr(y, bf, "y"), T, dm, dff, int(block), _stream(stream))


def swiglu_ffn_bwd(x, w1, w3, w2, dy, dx, dw1, dw3, dw2, block, stream=None):
    T, dm = (int(s) for s in x.shape)
    dff = int(w1.shape[1])
    bf, f = torch.bfloat16, torch.float32
    _call("swiglu_ffn_bwd", _ptr(x, bf, "x"), _ptr(w1, bf, "w1"), _ptr(w3, bf, "w3"), _ptr(w2, bf, "w2"),
          _ptr(dy, bf, "dy"), _ptr(dx, bf, "dx"), _ptr(dw1, f, "dw1"), _ptr(dw3, f, "dw3"), _ptr(dw2, f, "dw2"),
          T, dm, dff, int(block), _stream(stream))


def _ptr_array(ts, dtype, name):
    arr = (ctypes.c_void_p * len(ts))(*[_ptr(t, dtype, name).value for t in ts])
    return arr, ctypes.cast(arr, ctypes.c_void_p)


def llama_layer_fwd(x, params, z, n_heads, n_hosts, causal=True, stream=None):
    """params: [g1, wq, wk, wv, wo, g2, w1, w3, w2] (bf16 tensors)."""
    S, dm = (int(s) for s in x.shape)
    dff = int(params[6].shape[1])
    keep, parr = _ptr_array(params, torch.bfloat16, "params")
    _call("llama_layer_fwd", _ptr(x, torch.bfloat16, "x"), parr, _ptr(z, torch.bfloat16, "z"), S, dm, int(n_heads),
          dff, int(n_hosts), int(causal), _stream(stream))


def llama_layer_bwd(x, params, dz, dx, grads, n_heads, n_hosts, causal=True, stream=None):
    """grads: [dg1, dwq, dwk, dwv, dwo, dg2, dw1, dw3, dw2] (float32 tensors, overwritten)."""
    S, dm = (int(s) for s in x.shape)
    dff = int(params[6].shape[1])
    bf = torch.bfloat16
    keep_p, parr = _ptr_array(params, bf, "params")
    keep_g, garr = _ptr_array(grads, torch.float32, "grads")
    _call("llama_layer_bwd", _ptr(x, bf, "x"), parr, _ptr(dz, bf, "dz"), _ptr(dx, bf, "dx"), garr, S, dm,
          int(n_heads), dff, int(n_hosts), int(causal), _stream(stream))


def llama_stack_train_step(x, layer_params, dz, z, dx, layer_grads, n_heads, n_hosts, causal=True, stream=None):
    """layer_params / layer_grads: one 9-element list per layer (as llama_layer_fwd / _bwd)."""
    S, dm = (int(s) for s in x.shape)
    dff = int(layer_params[0][6].shape[1])
    bf = torch.bfloat16
    keep_p, parr = _ptr_array([t for p in layer_params for t in p], bf, "params")
    keep_g, garr = _ptr_array([t for g in layer_grads for t in g], torch.float32, "grads")
    _call("llama_stack_train_step", _ptr(x, bf, "x"), parr, _ptr(dz, bf, "dz"), _ptr(z, bf, "z"), _ptr(dx, bf, "dx"),
          garr, len(layer_params), S, dm, int(n_heads), dff, int(n_hosts), int(causal), _stream(stream))


# The calls of a decode step take a few microseconds on the GPU, so their checks are kept short: one
# pass over a tensor in `_arg` (about half the host time of `_ptr`), the raw stream handle, the
# library's function called by name.
_BF16, _F32, _I32, _U8, _E4M3 = torch.bfloat16, torch.float32, torch.int32, torch.uint8, torch.float8_e4m3fn


def _arg(t, name, dtype, dev, shape=None):
    """Address of a dense tensor on the current GPU `dev` of this type and shape; None for None."""
    if t is None:
        return None
    if t.dtype is dtype and t.get_device() == dev and t.is_contiguous() and (shape is None or t.shape == shape):
        return t.data_ptr()
    _ptr(t, dtype, name)
    if t.get_device() != dev:
        raise ValueError("%s must be on the current GPU (cuda:%d), got %s" % (name, dev, t.device))
    raise ValueError("%s must be %s, got %s" % (name, list(shape), list(t.shape)))


def _ints(t, name, n, dev):
    """_arg of n int32 elements."""
    if t.dtype is _I32 and t.get_device() == dev and t.numel() == n and t.is_contiguous():
        return t.data_ptr()
    return _arg(t, name, _I32, dev, (n,))


def _done(name, rc):
    if rc:
        raise RingAttnError(name, rc, load().ring_attn_last_error().decode())


def _rows(t, name, T, H, D, dev):
    """Address and row stride of a bf16 [T, H, D] tensor whose rows are dense."""
    if t.shape != (T, H, D):
        raise ValueError("%s must be %s, got %s" % (name, [T, H, D], list(t.shape)))
    row, head, elem = t.stride()
    if (D > 1 and elem != 1) or (H > 1 and head != D):
        raise ValueError("the heads of a row of %s must be contiguous" % name)
    if t.dtype is not _BF16 or t.get_device() != dev:
        _arg(t[:1].contiguous(), name, _BF16, dev)  # says what is wrong
    if T > 1 and row >> 31:
        raise ValueError("the rows of %s lie %d elements apart: 2^31 - 1 at most" % (name, row))
    return t.data_ptr(), row if T > 1 else H * D


def _cache(k_pages, v_pages, k_scales, v_scales, dev):
    """Addresses of a cache's tensors, its kv_type and its shape."""
    shape, dt = k_pages.shape, k_pages.dtype
    if len(shape) != 4:
        raise ValueError("expected a [n_pages, page_size, Hkv, D] cache")
    if dt is not _BF16 and dt is not _E4M3:
        raise TypeError("k_pages must be torch.bfloat16 or torch.float8_e4m3fn, got %s" % dt)
    kp, vp = _arg(k_pages, "k_pages", dt, dev), _arg(v_pages, "v_pages", dt, dev, shape)
    if dt is _BF16 and k_scales is None and v_scales is None:
        return kp, vp, None, None, 0, shape
    return (kp, vp, _arg(k_scales, "k_scales", _U8, dev, shape[:3]), _arg(v_scales, "v_scales", _U8, dev, shape[:3]),
            0 if dt is _BF16 else 1, shape)


def _current(stream):
    """The current GPU and the handle of the stream a call runs on."""
    dev = torch._C._cuda_getDevice()
    return dev, torch._C._cuda_getCurrentRawStream(dev) if stream is None else stream.cuda_stream


def paged_plan(lens, n_new, free_pages, free_head, block_table, cu_rows, new_lens, slots, positions, counts, page_size,
               n_pages, stream=None):
    """int32 tensors: lens, n_new, new_lens [R], free_pages [n_free], free_head [1] or None,
    block_table [R, max_pages], cu_rows [R + 1], slots, positions [T], counts [4]."""
    R, max_pages = block_table.shape
    T, n_free, (dev, st) = slots.numel(), free_pages.numel(), _current(stream)
    _done("paged_plan", (_LIB or load()).paged_plan(
        _ints(lens, "lens", R, dev), _ints(n_new, "n_new", R, dev), _ints(free_pages, "free_pages", n_free, dev),
        None if free_head is None else _ints(free_head, "free_head", 1, dev),
        _arg(block_table, "block_table", _I32, dev), _ints(cu_rows, "cu_rows", R + 1, dev),
        _ints(new_lens, "new_lens", R, dev), _ints(slots, "slots", T, dev), _ints(positions, "positions", T, dev),
        _ints(counts, "counts", 4, dev), R, page_size, max_pages, n_pages, n_free, T, st))


def paged_append(q, k, v, q_out, k_pages, v_pages, slots, positions, k_scales=None, v_scales=None, rotate=True,
                 stream=None):
    """q [T, Hq, D] (or None, with q_out), k, v [T, Hkv, D]: rows may be strided."""
    T, (dev, st) = slots.numel(), _current(stream)
    kp, vp, ks, vs, kind, (n_pages, page_size, Hkv, D) = _cache(k_pages, v_pages, k_scales, v_scales, dev)
    Hq = 0 if q is None else q.shape[1]
    q_at, q_row = (None, 0) if q is None else _rows(q, "q", T, Hq, D, dev)
    k_at, k_row = _rows(k, "k", T, Hkv, D, dev)
    v_at, v_row = _rows(v, "v", T, Hkv, D, dev)
    _done("paged_append", (_LIB or load()).paged_append(
        q_at, k_at, v_at, _arg(q_out, "q_out", _BF16, dev, (T, Hq, D)), kp, vp, ks, vs, _ints(slots, "slots", T, dev),
        _ints(positions, "positions", T, dev), T, Hq, Hkv, D, q_row, k_row, v_row, n_pages, page_size, kind,
        1 if rotate else 0, st))


def paged_attn_workspace(R, Hq, Hkv, D, max_new):
    """Bytes of workspace a paged_attn_decode of this shape needs."""
    n = ctypes.c_size_t(0)
    _call("paged_attn_workspace", R, Hq, Hkv, D, max_new, ctypes.addressof(n))
    return n.value


def paged_attn_decode(q, k_pages, v_pages, block_table, lens, cu_rows, o, lse, max_new, k_scales=None, v_scales=None,
                      workspace=None, stream=None):
    """q, o [T, Hq, D], lse [T, Hq]; cu_rows None: row r is the one new token of request r.
    workspace: a contiguous GPU tensor of paged_attn_workspace bytes, or None."""
    T, Hq, D = q.shape
    R, max_pages = block_table.shape
    dev, st = _current(stream)
    kp, vp, ks, vs, kind, (n_pages, page_size, Hkv, Dc) = _cache(k_pages, v_pages, k_scales, v_scales, dev)
    if Dc != D:
        raise ValueError("head dim %d of q, %d of the cache" % (D, Dc))
    ws, ws_bytes = None, 0
    if workspace is not None:
        ws, ws_bytes = _arg(workspace, "workspace", workspace.dtype, dev), workspace.numel() * workspace.element_size()
    _done("paged_attn_decode", (_LIB or load()).paged_attn_decode(
        _arg(q, "q", _BF16, dev), kp, vp, ks, vs, _arg(block_table, "block_table", _I32, dev),
        _ints(lens, "lens", R, dev), None if cu_rows is None else _ints(cu_rows, "cu_rows", R + 1, dev),
        _arg(o, "o", _BF16, dev, (T, Hq, D)), _arg(lse, "lse", _F32, dev, (T, Hq)), ws, ws_bytes, T, R, Hq, Hkv, D,
        n_pages, page_size, max_pages, max_new, kind, st))


def mx4_pack(w, w4, scales, stream=None):
    (K, N), (dev, st) = w.shape, _current(stream)
    nb, kb = -(-N // 16), -(-K // 128)
    _call("mx4_pack", _arg(w, "w", _BF16, dev), _arg(w4, "w4", _U8, dev, (nb, kb, 64, 16)),
          _arg(scales, "scales", _U8, dev, (nb, kb, 16, 4)), K, N, st)


def mx4_linear(x, w4, scales, residual, y, stream=None):
    (T, K), N, (dev, st) = x.shape, y.shape[1], _current(stream)
    nb, kb = -(-N // 16), -(-K // 128)
    _done("mx4_linear", (_LIB or load()).mx4_linear(
        _arg(x, "x", _BF16, dev), _arg(w4, "w4", _U8, dev, (nb, kb, 64, 16)),
        _arg(scales, "scales", _U8, dev, (nb, kb, 16, 4)), _arg(residual, "residual", _BF16, dev, (T, N)),
        _arg(y, "y", _BF16, dev, (T, N)), T, K, N, st))


# ----------------------------------------------------------------------------------
# Allocating wrappers
# ----------------------------------------------------------------------------------
def attention_fwd(q, k, v, n_hosts, causal=True):
    """Returns (o, lse) for bf16 or float32 q, k, v of shape [B, S, H, D].  A bf16 causal
    sequence whose length does not fill n_hosts blocks of a multiple of 128 tokens goes
    through ring_attn_fwd_varlen (short or empty last blocks)."""
    B, S, H, D = _bshd(q)
    o = torch.empty_like(q)
    lse = torch.empty((B, H, S), dtype=torch.float32, device=q.device)
    if _ragged(q, S, n_hosts, causal):
        ring_attn_fwd_varlen(q, k, v, o, lse, n_hosts)
        return o, lse
    fn = ring_attn_fwd if q.dtype == torch.bfloat16 else ring_attn_fwd_f32
    fn(q, k, v, o, lse, n_hosts, causal)
    return o, lse


def _ragged(q, S, n_hosts, causal):
    return bool(causal) and q.dtype == torch.bfloat16 and int(n_hosts) > 0 and S % (128 * int(n_hosts)) != 0


def attention_bwd(q, k, v, o, lse, dO, n_hosts, causal=True):
    """Returns (dq, dk, dv); ragged bf16 causal lengths as in attention_fwd."""
    dq, dk, dv = torch.empty_like(q), torch.empty_like(k), torch.empty_like(v)
    if _ragged(q, int(q.shape[1]), n_hosts, causal):
        ring_attn_bwd_varlen(q, k, v, o, lse, dO, dq, dk, dv, n_hosts)
        return dq, dk, dv
    fn = ring_attn_bwd if q.dtype == torch.bfloat16 else ring_attn_bwd_f32
    fn(q, k, v, o, lse, dO, dq, dk, dv, n_hosts, causal)
    return dq, dk, dv


def attention_decode(q, k_cache, v_cache, n_hosts, causal=True):
    """Returns (o [B, Tq, H, D] bf16, lse [B, H, Tq] f32) of ring_attn_decode."""
    B, Tq, H, D = _bshd(q)
    o = torch.empty_like(q)
    lse = torch.empty((B, H, Tq), dtype=torch.float32, device=q.device)
    ring_attn_decode(q, k_cache, v_cache, o, lse, n_hosts, causal)
    return o, lse


def paged_attention(q, k_pages, v_pages, block_table, lens, cu_rows=None, max_new=None, k_scales=None, v_scales=None):
    """Returns (o [T, Hq, D] bf16, lse [T, Hq] f32) of paged_attn_decode, zeros in padding rows and in the
    rows of a request past its first max_new; max_new goes with cu_rows (without them it is 1)."""
    if max_new is None:
        if cu_rows is not None:
            raise ValueError("max_new, the most new tokens of a request, must be given with cu_rows")
        max_new = 1
    o = torch.zeros_like(q)
    lse = torch.zeros(q.shape[:2], dtype=torch.float32, device=q.device)
    paged_attn_decode(q, k_pages, v_pages, block_table, lens, cu_rows, o, lse, max_new, k_scales, v_scales)
    return o, lse


def mx4_weights(w):
    """Returns (w4, scales) of mx4_pack for a bf16 [d_in, d_out] weight."""
    K, N = (int(s) for s in w.shape)
    nb, kb = -(-N // 16), -(-K // 128)
    w4 = torch.empty((nb, kb, 64, 16), dtype=torch.uint8, device=w.device)
    scales = torch.empty((nb, kb, 16, 4), dtype=torch.uint8, device=w.device)
    mx4_pack(w, w4, scales)
    return w4, scales
