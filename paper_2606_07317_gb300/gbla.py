"""Thin ctypes binding of libgbla (the C ABI declared in include/gbla.h).

Argument marshalling only: every step of the GBLA core runs in the library's
CUDA kernels.  Tensors are torch tensors; device calls take CUDA tensors and
enqueue on the current torch stream (or the stream given).  There is no CPU
fallback: if the library is missing or fails to load, calls raise.
"""
from __future__ import annotations

import ctypes
import os
import threading

import torch

from . import build as _build

GBLA_OK, GBLA_ERR_INVALID_ARG, GBLA_ERR_UNSUPPORTED, GBLA_ERR_ALLOC, GBLA_ERR_CUDA = range(5)
GBLA_FP32, GBLA_BF16 = 0, 1
ALGO_AUTO, ALGO_SIMT, ALGO_TC = 0, 1, 2
# ablation flags (gbla_flags): identity Conv1D, uniform key gate, no gated RMSNorm
FLAG_NO_CONV, FLAG_NO_GATE, FLAG_NO_NORM = 1, 2, 4
FLAG_BLA = FLAG_NO_CONV | FLAG_NO_GATE | FLAG_NO_NORM
CONV_WIDTH = 4
ROTATE_INTERLEAVED = 1
MAX_TOP = 64

EXPORTED = ["gbla_forward", "gbla_forward_ex", "gbla_forward_variant", "gbla_forward_f32out",
            "gbla_backward", "gbla_backward_variant", "gbla_backward_from_state",
            "gbla_state", "gbla_state_stats", "gbla_combine_states",
            "gbla_readout",
            "gbla_forward_host", "gbla_state_floats", "gbla_rms_eps",
            "gbla_status_string", "gbla_version", "gbla_release", "gbla_launch_count",
            "gbla_state_static_scratch", "gbla_device_error", "gbla_last_cuda_error",
            "gbla_project", "gbla_layer_forward", "gbla_attention_forward",
            "gbla_qk_norm_rotate", "gbla_qk_norm_rotate_backward", "gbla_decay_attention",
            "gbla_decay_attention_backward", "gbla_decay_attention_step",
            "gbla_delta_attention", "gbla_delta_attention_backward", "gbla_delta_attention_step",
            "gbla_token_logprobs", "gbla_token_logprobs_backward"]

_lock = threading.Lock()
_lib = None

_vp = ctypes.c_void_p
_i = ctypes.c_int


class GblaError(RuntimeError):
    def __init__(self, status: int, fn: str):
        self.status = status
        msg = f"{fn}: {status_string(status)} (status {status})"
        if status == GBLA_ERR_CUDA:
            msg += f": {load().gbla_last_cuda_error().decode()}"
        super().__init__(msg)


def lib_path() -> str:
    return _build.LIB_PATH


def load(path: str | None = None):
    """Load libgbla.so (it must have been built; see __graft_entry__.build())."""
    global _lib
    with _lock:
        if _lib is not None and path is None:
            return _lib
        p = path or lib_path()
        if not os.path.exists(p):
            raise RuntimeError(f"CUDA library not built: {p} is missing "
                               "(run `python -c 'import __graft_entry__ as g; g.build()'`)")
        lib = ctypes.CDLL(p)
        fwd = [_vp] * 9 + [_i] * 5
        lib.gbla_forward.argtypes = fwd + [_vp]
        lib.gbla_forward.restype = _i
        lib.gbla_forward_ex.argtypes = fwd + [_i, _vp]
        lib.gbla_forward_ex.restype = _i
        lib.gbla_forward_variant.argtypes = fwd + [_i, ctypes.c_uint32, _vp]
        lib.gbla_forward_variant.restype = _i
        lib.gbla_forward_f32out.argtypes = fwd + [_i, _vp]
        lib.gbla_forward_f32out.restype = _i
        lib.gbla_backward.argtypes = [_vp] * 16 + [_i] * 5 + [_vp]
        lib.gbla_backward.restype = _i
        lib.gbla_backward_variant.argtypes = [_vp] * 16 + [_i] * 5 + [ctypes.c_uint32, _vp]
        lib.gbla_backward_variant.restype = _i
        lib.gbla_backward_from_state.argtypes = [_vp] * 18 + [_i] * 5 + [_vp]
        lib.gbla_backward_from_state.restype = _i
        lib.gbla_project.argtypes = [_vp] * 9 + [_i] * 6 + [_vp]
        lib.gbla_project.restype = _i
        lib.gbla_layer_forward.argtypes = [_vp] * 6 + [_i] * 6 + [_vp]
        lib.gbla_layer_forward.restype = _i
        lib.gbla_attention_forward.argtypes = [_vp] * 5 + [_i] * 5 + [_vp]
        lib.gbla_attention_forward.restype = _i
        lib.gbla_forward_host.argtypes = fwd + [_vp]
        lib.gbla_forward_host.restype = _i
        lib.gbla_state.argtypes = [_vp] * 6 + [_i] * 6 + [_vp]
        lib.gbla_state.restype = _i
        lib.gbla_state_stats.argtypes = [_vp] * 7 + [_i] * 6 + [_vp]
        lib.gbla_state_stats.restype = _i
        lib.gbla_combine_states.argtypes = [_vp, _vp, _i, _vp, _vp, _i, _i, _i, _vp]
        lib.gbla_combine_states.restype = _i
        lib.gbla_readout.argtypes = [_vp] * 7 + [_i] * 6 + [_vp]
        lib.gbla_readout.restype = _i
        lib.gbla_state_static_scratch.argtypes = [_vp] * 6 + [_i] * 5 + [_vp]
        lib.gbla_state_static_scratch.restype = _i
        f, u32 = ctypes.c_float, ctypes.c_uint32
        lib.gbla_qk_norm_rotate.argtypes = [_vp] * 10 + [_i] * 7 + [f, u32, _i, _vp]
        lib.gbla_qk_norm_rotate.restype = _i
        lib.gbla_qk_norm_rotate_backward.argtypes = [_vp] * 14 + [_i] * 7 + [f, u32, _i, _vp]
        lib.gbla_qk_norm_rotate_backward.restype = _i
        lib.gbla_decay_attention.argtypes = [_vp] * 9 + [_i] * 5 + [f, _i, _i, _vp]
        lib.gbla_decay_attention.restype = _i
        lib.gbla_decay_attention_backward.argtypes = [_vp] * 13 + [_i] * 5 + [f, _i, _i, _vp]
        lib.gbla_decay_attention_backward.restype = _i
        lib.gbla_decay_attention_step.argtypes = [_vp] * 8 + [_i] * 5 + [f, _i, _vp]
        lib.gbla_decay_attention_step.restype = _i
        lib.gbla_delta_attention.argtypes = [_vp] * 10 + [_i] * 5 + [f, _i, _vp]
        lib.gbla_delta_attention.restype = _i
        lib.gbla_delta_attention_backward.argtypes = [_vp] * 16 + [_i] * 5 + [f, _i, _vp]
        lib.gbla_delta_attention_backward.restype = _i
        lib.gbla_delta_attention_step.argtypes = [_vp] * 9 + [_i] * 5 + [f, _i, _vp]
        lib.gbla_delta_attention_step.restype = _i
        lib.gbla_token_logprobs.argtypes = [_vp] * 9 + [_i] * 4 + [f, _i, _vp]
        lib.gbla_token_logprobs.restype = _i
        lib.gbla_token_logprobs_backward.argtypes = [_vp] * 10 + [_i] * 3 + [f, _i, _vp]
        lib.gbla_token_logprobs_backward.restype = _i
        lib.gbla_state_floats.argtypes = [_i]
        lib.gbla_state_floats.restype = ctypes.c_size_t
        lib.gbla_rms_eps.argtypes = []
        lib.gbla_rms_eps.restype = ctypes.c_float
        lib.gbla_status_string.argtypes = [_i]
        lib.gbla_status_string.restype = ctypes.c_char_p
        lib.gbla_version.argtypes = []
        lib.gbla_version.restype = ctypes.c_char_p
        lib.gbla_release.argtypes = []
        lib.gbla_release.restype = None
        lib.gbla_last_cuda_error.argtypes = []
        lib.gbla_last_cuda_error.restype = ctypes.c_char_p
        lib.gbla_device_error.argtypes = [_i]
        lib.gbla_device_error.restype = ctypes.c_uint32
        lib.gbla_launch_count.argtypes = []
        lib.gbla_launch_count.restype = ctypes.c_uint64
        if path is None:
            _lib = lib
        return lib


def status_string(status: int) -> str:
    return load().gbla_status_string(int(status)).decode()


def rms_eps() -> float:
    return float(load().gbla_rms_eps())


def version() -> str:
    return load().gbla_version().decode()


def launch_count() -> int:
    """Kernels the library has enqueued so far (all devices, all threads)."""
    return int(load().gbla_launch_count())


def device_error(reset: bool = False) -> int:
    """Error bits left by a tensor-core kernel whose bounded wait ran out (0 = none)."""
    return int(load().gbla_device_error(1 if reset else 0))


def state_floats(D: int) -> int:
    return int(load().gbla_state_floats(int(D)))


def _dtype_code(t: torch.Tensor) -> int:
    if t.dtype == torch.float32:
        return GBLA_FP32
    if t.dtype == torch.bfloat16:
        return GBLA_BF16
    raise TypeError(f"unsupported dtype {t.dtype}")


def _ptr(t):
    if t is None:
        return None
    return t.data_ptr() or None


def _stream(stream):
    if stream is None:
        stream = torch.cuda.current_stream()
    return _vp(stream.cuda_stream)


def _check(status: int, fn: str):
    if status != GBLA_OK:
        raise GblaError(status, fn)


def _bhnd(q: torch.Tensor):
    if q.dim() != 4:
        raise ValueError("q must be [B, N, H, D]")
    B, N, H, D = q.shape
    return B, H, N, D


def forward(q, k, v, gate, out_gate, conv_w, norm_w, seq_lens=None, out=None,
            algo: int = ALGO_AUTO, stream=None, flags: int = 0) -> torch.Tensor:
    """o = GBLA core forward; tensors on one CUDA device, layouts of include/gbla.h.
    `flags` (FLAG_*) selects an ablation (gbla_forward_variant); 0 is the full core."""
    B, H, N, D = _bhnd(q)
    if out is None:
        out = torch.empty_like(q)
    if flags:
        st = load().gbla_forward_variant(
            _ptr(q), _ptr(k), _ptr(v), _ptr(gate), _ptr(out_gate), _ptr(conv_w),
            _ptr(norm_w), _ptr(seq_lens), _ptr(out), B, H, N, D, _dtype_code(q), int(algo),
            int(flags), _stream(stream))
        _check(st, "gbla_forward_variant")
        return out
    st = load().gbla_forward_ex(
        _ptr(q), _ptr(k), _ptr(v), _ptr(gate), _ptr(out_gate), _ptr(conv_w),
        _ptr(norm_w), _ptr(seq_lens), _ptr(out), B, H, N, D, _dtype_code(q), int(algo),
        _stream(stream))
    _check(st, "gbla_forward_ex")
    return out


def attention(q, k, v, seq_lens=None, out=None, stream=None) -> torch.Tensor:
    """Bidirectional softmax attention of Sec. 2 (gbla_attention_forward): q, k, v,
    out [B, N, H, D] bf16 (D = 64); rows past seq_lens are not written."""
    B, H, N, D = _bhnd(q)
    if out is None:
        out = torch.empty_like(q)
    st = load().gbla_attention_forward(_ptr(q), _ptr(k), _ptr(v), _ptr(seq_lens), _ptr(out),
                                       B, H, N, D, _dtype_code(q), _stream(stream))
    _check(st, "gbla_attention_forward")
    return out


def forward_f32out(q, k, v, gate, out_gate, conv_w, norm_w, seq_lens=None, out=None,
                   algo: int = ALGO_AUTO, stream=None) -> torch.Tensor:
    """Debug variant of forward (gbla_forward_f32out): the same kernels and arithmetic,
    with o stored in fp32 before the rounding to the input dtype."""
    B, H, N, D = _bhnd(q)
    if out is None:
        out = torch.empty(q.shape, dtype=torch.float32, device=q.device)
    st = load().gbla_forward_f32out(
        _ptr(q), _ptr(k), _ptr(v), _ptr(gate), _ptr(out_gate), _ptr(conv_w),
        _ptr(norm_w), _ptr(seq_lens), _ptr(out), B, H, N, D, _dtype_code(q), int(algo),
        _stream(stream))
    _check(st, "gbla_forward_f32out")
    return out


def backward(q, k, v, gate, out_gate, conv_w, norm_w, seq_lens, dy, stream=None,
             flags: int = 0, state=None, stats=None) -> dict:
    """Gradients of sum(dy * o) (gbla_backward): dq, dk, dv, dout_gate like q; dgate like
    gate; dconv_w [3, H, D, W] and dnorm_w [H, D] fp32.  Rows past seq_lens are 0.
    `flags` (FLAG_*) selects an ablation (gbla_backward_variant); 0 is the full core.
    `state` and `stats`, as state_stats returned them for this forward, skip the state
    pass (gbla_backward_from_state; full core only)."""
    B, H, N, D = _bhnd(q)
    if (state is None) != (stats is None):
        raise ValueError("state and stats go together")
    if state is not None and flags:
        raise ValueError("a saved state serves the full core only (flags 0)")
    g = dict(dq=torch.empty_like(q), dk=torch.empty_like(q), dv=torch.empty_like(q),
             dgate=torch.empty_like(gate), dout_gate=torch.empty_like(q),
             dconv_w=torch.empty_like(conv_w, dtype=torch.float32),
             dnorm_w=torch.empty_like(norm_w, dtype=torch.float32))
    args = (_ptr(q), _ptr(k), _ptr(v), _ptr(gate), _ptr(out_gate), _ptr(conv_w), _ptr(norm_w),
            _ptr(seq_lens), _ptr(dy), _ptr(g["dq"]), _ptr(g["dk"]), _ptr(g["dv"]),
            _ptr(g["dgate"]), _ptr(g["dout_gate"]), _ptr(g["dconv_w"]), _ptr(g["dnorm_w"]),
            B, H, N, D, _dtype_code(q))
    if state is not None:
        if (state.dtype != torch.float32 or stats.dtype != torch.float32
                or tuple(state.shape) != (B, H, D * D + D) or tuple(stats.shape) != (B, H, 2)
                or not state.is_contiguous() or not stats.is_contiguous()):
            raise ValueError("state must be [B, H, D*D + D] and stats [B, H, 2], contiguous fp32")
        a = list(args)
        a[8:8] = [_ptr(state), _ptr(stats)]  # after seq_lens
        st = load().gbla_backward_from_state(*a, _stream(stream))
        _check(st, "gbla_backward_from_state")
    elif flags:
        st = load().gbla_backward_variant(*args, int(flags), _stream(stream))
        _check(st, "gbla_backward_variant")
    else:
        st = load().gbla_backward(*args, _stream(stream))
        _check(st, "gbla_backward")
    return g


def project(x, conv_x, w_proj, H, D, seq_lens=None, out=None, stream=None) -> dict:
    """Layer front end (gbla_project): X~ = Conv1D(x) over the d channels of x [B, N, d],
    then the stacked projections w_proj [4 H D + H, d] (rows W_Q, W_K, W_V, W_R per head
    and dim, then w_g per head).  Returns q, k, v, out_gate [B, N, H, D] and gate
    [B, N, H] (rows past seq_lens are not written; `out` may supply the five tensors)."""
    B, N, d = x.shape
    if out is None:
        out = {n: x.new_empty((B, N, H, D)) for n in ("q", "k", "v", "out_gate")}
        out["gate"] = x.new_empty((B, N, H))
    st = load().gbla_project(
        _ptr(x), _ptr(conv_x), _ptr(w_proj), _ptr(seq_lens), _ptr(out["q"]), _ptr(out["k"]),
        _ptr(out["v"]), _ptr(out["out_gate"]), _ptr(out["gate"]), B, N, d, H, D,
        _dtype_code(x), _stream(stream))
    _check(st, "gbla_project")
    return out


def layer_forward(x, conv_x, w_proj, norm_w, H, D, seq_lens=None, out=None,
                  stream=None) -> torch.Tensor:
    """Whole GBLA layer from x [B, N, d] (gbla_layer_forward): front end, then the core
    with its Conv1D off.  Returns o [B, N, H, D]."""
    B, N, d = x.shape
    if out is None:
        out = x.new_empty((B, N, H, D))
    st = load().gbla_layer_forward(
        _ptr(x), _ptr(conv_x), _ptr(w_proj), _ptr(norm_w), _ptr(seq_lens), _ptr(out),
        B, N, d, H, D, _dtype_code(x), _stream(stream))
    _check(st, "gbla_layer_forward")
    return out


def forward_default(q, k, v, gate, out_gate, conv_w, norm_w, seq_lens, out, stream=None):
    """Direct call of gbla_forward (the AUTO entry point)."""
    B, H, N, D = _bhnd(q)
    st = load().gbla_forward(
        _ptr(q), _ptr(k), _ptr(v), _ptr(gate), _ptr(out_gate), _ptr(conv_w),
        _ptr(norm_w), _ptr(seq_lens), _ptr(out), B, H, N, D, _dtype_code(q),
        _stream(stream))
    _check(st, "gbla_forward")
    return out


def state(k, v, gate, conv_w, seq_lens=None, out=None, algo: int = ALGO_AUTO,
          stream=None) -> torch.Tensor:
    """[B, H, D*D + D] fp32: S (row-major) then z per (batch, head)."""
    B, H, N, D = _bhnd(k)
    if out is None:
        out = torch.empty((B, H, D * D + D), dtype=torch.float32, device=k.device)
    st = load().gbla_state(_ptr(k), _ptr(v), _ptr(gate), _ptr(conv_w), _ptr(seq_lens),
                           _ptr(out), B, H, N, D, _dtype_code(k), int(algo),
                           _stream(stream))
    _check(st, "gbla_state")
    return out


def state_stats(k, v, gate, conv_w, seq_lens=None, algo: int = ALGO_AUTO, stream=None):
    """gbla_state_stats: (state [B, H, D*D + D], stats [B, H, 2]) fp32, stats = (max gate
    logit, sum of exp(logit - max)) over each sequence's valid positions."""
    B, H, N, D = _bhnd(k)
    out = torch.empty((B, H, D * D + D), dtype=torch.float32, device=k.device)
    stats = torch.empty((B, H, 2), dtype=torch.float32, device=k.device)
    st = load().gbla_state_stats(_ptr(k), _ptr(v), _ptr(gate), _ptr(conv_w), _ptr(seq_lens),
                                 _ptr(out), _ptr(stats), B, H, N, D, _dtype_code(k), int(algo),
                                 _stream(stream))
    _check(st, "gbla_state_stats")
    return out, stats


def combine_states(states, stats, stream=None):
    """gbla_combine_states: states [P, B, H, D*D + D] and stats [P, B, H, 2] (fp32, one
    CUDA device) of P disjoint token segments -> (state, stats) of the whole sequences."""
    P, B, H, F = states.shape
    D = int(round((F + 0.25) ** 0.5 - 0.5))
    if D * D + D != F or tuple(stats.shape) != (P, B, H, 2):
        raise ValueError("states must be [P, B, H, D*D + D] and stats [P, B, H, 2]")
    states, stats = states.contiguous(), stats.contiguous()
    out = torch.empty((B, H, F), dtype=torch.float32, device=states.device)
    out_stats = torch.empty((B, H, 2), dtype=torch.float32, device=states.device)
    st = load().gbla_combine_states(_ptr(states), _ptr(stats), P, _ptr(out), _ptr(out_stats),
                                    B, H, D, _stream(stream))
    _check(st, "gbla_combine_states")
    return out, out_stats


def readout(q, out_gate, conv_w, norm_w, state_t, seq_lens=None, out=None,
            algo: int = ALGO_AUTO, stream=None) -> torch.Tensor:
    B, H, N, D = _bhnd(q)
    if out is None:
        out = torch.empty_like(q)
    st = load().gbla_readout(_ptr(q), _ptr(out_gate), _ptr(conv_w), _ptr(norm_w),
                             _ptr(seq_lens), _ptr(state_t), _ptr(out), B, H, N, D,
                             _dtype_code(q), int(algo), _stream(stream))
    _check(st, "gbla_readout")
    return out


def forward_host(q, k, v, gate, out_gate, conv_w, norm_w, seq_lens=None, out=None,
                 stream=None) -> torch.Tensor:
    """Host-memory entry point: CPU tensors (pinned for full copy speed) in and out."""
    B, H, N, D = _bhnd(q)
    if out is None:
        out = torch.empty_like(q)
    st = load().gbla_forward_host(
        _ptr(q), _ptr(k), _ptr(v), _ptr(gate), _ptr(out_gate), _ptr(conv_w),
        _ptr(norm_w), _ptr(seq_lens), _ptr(out), B, H, N, D, _dtype_code(q),
        _stream(stream))
    _check(st, "gbla_forward_host")
    return out


def state_static_scratch(k, v, gate, conv_w, seq_lens=None, out=None,
                         stream=None) -> torch.Tensor:
    """gbla_state without any GPU allocation: for callers that cannot allocate
    device memory (its partial sums live in a fixed array inside the library;
    see include/gbla.h for the size limit and the rule against overlapping
    calls)."""
    B, H, N, D = _bhnd(k)
    if out is None:
        out = torch.empty((B, H, D * D + D), dtype=torch.float32, device=k.device)
    st = load().gbla_state_static_scratch(_ptr(k), _ptr(v), _ptr(gate), _ptr(conv_w),
                                          _ptr(seq_lens), _ptr(out), B, H, N, D,
                                          _dtype_code(k), _stream(stream))
    _check(st, "gbla_state_static_scratch")
    return out


# --- causal decoder operators -------------------------------------------------
#
# `stream` (None: the current one) is the stream that a call's kernels run on.  Its results
# are allocated on that stream; tensors passed in must be ready there, and their memory must
# not go back to another stream's allocator before the call's work is done (record_stream).
# Tensors that a call writes to in place (`out`, the pool of states) count as changed for
# autograd.

_changed = torch.autograd.graph.increment_version
_CODES = {torch.float32: GBLA_FP32, torch.bfloat16: GBLA_BF16}


def _code(q):
    """(dtype code, device index) of q, whose type and device the other tensors share."""
    code = _CODES.get(q.dtype)
    if code is None:
        raise TypeError(f"unsupported dtype {q.dtype}")
    return code, q.get_device()


def _raw_stream(dev, stream):
    """Handle of the stream (None: the current one) that a call on device `dev` goes to."""
    if dev < 0 or dev != torch.cuda.current_device():
        raise ValueError("the tensors must be on the current CUDA device")
    return torch._C._cuda_getCurrentRawStream(dev) if stream is None else stream.cuda_stream


def _dims(q):
    if q.dim() != 4:
        raise ValueError("q must be [B, N, H, D]")
    return q.shape


def _heads(t, name, shape, dtype, dev):
    """Checks a token-major tensor whose heads are adjacent and whose head values are
    contiguous; True if it is contiguous throughout."""
    if t.shape != shape:
        raise ValueError(f"{name} must be [B, N, heads, D] = {tuple(shape)}, not {tuple(t.shape)}")
    if t.dtype is not dtype or t.get_device() != dev:
        raise ValueError(f"{name} must have the dtype and device of q")
    if t.is_contiguous():
        return True
    if (shape[3] > 1 and t.stride(3) != 1) or (shape[2] > 1 and t.stride(2) != shape[3]):
        raise ValueError(f"the heads of {name} must be adjacent and their values contiguous")
    return False


def _key_shape(shape, k):
    """Shape of a key or value tensor that goes with q's."""
    if k.dim() != 4:
        raise ValueError("k must be [B, N, heads, D]")
    return (shape[0], shape[1], k.shape[2], shape[3])


def _plain(t, name, shape, dtype, dev):
    """Checks an optional contiguous tensor and returns its address (None: NULL)."""
    if t is None:
        return None
    if t.shape == shape and t.dtype is dtype and t.is_contiguous() and t.get_device() == dev:
        return t.data_ptr()
    if t.shape != shape or t.dtype is not dtype or not t.is_contiguous():
        raise ValueError(f"{name} must be a contiguous {dtype} tensor of shape {tuple(shape)}")
    raise ValueError(f"{name} must be on the device of q")


def _empty(stream, shape, dtype, device):
    """A tensor whose memory belongs to the stream of the call."""
    if stream is None:
        return torch.empty(shape, dtype=dtype, device=device)
    with torch.cuda.stream(stream):
        return torch.empty(shape, dtype=dtype, device=device)


def _like(t, stream):
    """A contiguous tensor like t, as _empty."""
    if stream is None and t.is_contiguous():
        return torch.empty_like(t)
    return _empty(stream, t.shape, t.dtype, t.device)


def _strides(*tensors, dims=2):
    """Host array of the (batch, token) strides of each tensor (dims=1: batch alone)."""
    flat = [s for t in tensors for s in t.stride()[:dims]]
    return (ctypes.c_int64 * len(flat))(*flat)


def rotation_table(positions: int, R: int, base: float = 10000.0, device="cuda") -> torch.Tensor:
    """[positions, R] fp32: cosines, then sines, of position * base^(-2 i / R) for the R / 2
    pairs (computed in 64 bits) -- the `rot` of qk_norm_rotate."""
    f = base ** (-torch.arange(0, R, 2, dtype=torch.float64) / max(R, 1))
    a = torch.arange(positions, dtype=torch.float64)[:, None] * f
    return torch.cat([a.cos(), a.sin()], 1).to(torch.float32).to(device)


def _rotate_args(q, k, norm_q, norm_k, rot, positions, seq_lens):
    """(code, device, input addresses and strides in the ABI's order, sizes)."""
    B, N, H, D = shape = _dims(q)
    code, dev = _code(q)
    kshape = _key_shape(shape, k)
    whole = _heads(q, "q", shape, q.dtype, dev) & _heads(k, "k", kshape, q.dtype, dev)
    P, R = rot.shape if rot is not None and rot.dim() == 2 else (0, 0)
    f32, i32 = torch.float32, torch.int32
    ins = (q.data_ptr(), k.data_ptr(), _plain(norm_q, "norm_q", (H, D), f32, dev),
           _plain(norm_k, "norm_k", (kshape[2], D), f32, dev), _plain(rot, "rot", (P, R), f32, dev),
           _plain(positions, "positions", (B, N), i32, dev),
           _plain(seq_lens, "seq_lens", (B,), i32, dev), None if whole else _strides(q, k))
    return code, dev, ins, (B, N, H, kshape[2], D, R, P)


def qk_norm_rotate(q, k, norm_q, norm_k, rot=None, positions=None, seq_lens=None,
                   eps: float = 1e-6, interleaved: bool = False, out=None, stream=None):
    """Per-head RMS norm and position rotation of q [B, N, H, D] and k [B, N, Hk, D]
    (gbla_qk_norm_rotate): weights norm_q [H, D], norm_k [Hk, D]; rot [P, R] from
    rotation_table (None: norm alone); positions [B, N] int32 (None: token t has position
    t).  q and k may be slices of a packed projection.  Returns (qo, ko), or fills `out`;
    rows past seq_lens are not written."""
    code, dev, ins, dims = _rotate_args(q, k, norm_q, norm_k, rot, positions, seq_lens)
    given = out is not None
    if not given:
        out = (_like(q, stream), _like(k, stream))
    st = (_lib or load()).gbla_qk_norm_rotate(
        *ins, _plain(out[0], "out[0]", q.shape, q.dtype, dev),
        _plain(out[1], "out[1]", k.shape, q.dtype, dev), *dims, eps,
        ROTATE_INTERLEAVED if interleaved else 0, code, _raw_stream(dev, stream))
    _check(st, "gbla_qk_norm_rotate")
    if given:
        _changed(out)
    return out[0], out[1]


def qk_norm_rotate_backward(q, k, norm_q, norm_k, rot, dqo, dko, positions=None, seq_lens=None,
                            eps: float = 1e-6, interleaved: bool = False, stream=None) -> dict:
    """Gradients of qk_norm_rotate (gbla_qk_norm_rotate_backward) for the contiguous
    gradients dqo, dko of its results: dq, dk (0 past seq_lens), dnorm_q, dnorm_k."""
    code, dev, ins, dims = _rotate_args(q, k, norm_q, norm_k, rot, positions, seq_lens)
    grads = (_plain(dqo, "dqo", q.shape, q.dtype, dev), _plain(dko, "dko", k.shape, q.dtype, dev))
    g = {"d" + n: _like(t, stream)
         for n, t in (("q", q), ("k", k), ("norm_q", norm_q), ("norm_k", norm_k))}
    st = (_lib or load()).gbla_qk_norm_rotate_backward(
        *ins, *grads, *[t.data_ptr() for t in g.values()], *dims, eps,
        ROTATE_INTERLEAVED if interleaved else 0, code, _raw_stream(dev, stream))
    _check(st, "gbla_qk_norm_rotate_backward")
    return g


def _decay_args(q, k, v, log_decay, seq_lens, state):
    """(code, device, input addresses and strides in the ABI's order, sizes)."""
    B, N, H, D = shape = _dims(q)
    code, dev = _code(q)
    kshape = _key_shape(shape, k)
    whole = (_heads(q, "q", shape, q.dtype, dev) & _heads(k, "k", kshape, q.dtype, dev)
             & _heads(v, "v", kshape, q.dtype, dev))
    ins = (q.data_ptr(), k.data_ptr(), v.data_ptr(),
           _plain(log_decay, "log_decay", (H,), torch.float32, dev),
           _plain(seq_lens, "seq_lens", (B,), torch.int32, dev),
           None if whole else _strides(q, k, v),
           _plain(state, "state", (B, H, D, D), torch.float32, dev))
    return code, dev, ins, (B, N, H, kshape[2], D)


def decay_attention(q, k, v, log_decay, seq_lens=None, state=None, scale=None, out=None,
                    return_state: bool = False, algo: int = ALGO_AUTO, stream=None):
    """Causal linear attention with a decay for each head (gbla_decay_attention):
    S_t = exp(log_decay) S_{t-1} + k_t v_t^T, o_t = scale q_t^T S_t for q [B, N, H, D] and
    k, v [B, N, Hk, D]; `state` [B, H, D, D] fp32 is S before the first token, scale
    defaults to D^-1/2.  Returns o, or (o, S after each sequence's last token) with
    return_state; rows of o past seq_lens are not written."""
    code, dev, ins, dims = _decay_args(q, k, v, log_decay, seq_lens, state)
    B, N, H, Hk, D = dims
    given = out is not None
    if not given:
        out = _like(q, stream)
    fin = _empty(stream, (B, H, D, D), torch.float32, q.device) if return_state else None
    st = (_lib or load()).gbla_decay_attention(
        *ins, _plain(out, "out", q.shape, q.dtype, dev), None if fin is None else fin.data_ptr(),
        *dims, D ** -0.5 if scale is None else scale, code, algo, _raw_stream(dev, stream))
    _check(st, "gbla_decay_attention")
    if given:
        _changed((out,))
    return (out, fin) if return_state else out


def decay_attention_backward(q, k, v, log_decay, do, seq_lens=None, state=None, dstate=None,
                             scale=None, return_dstate: bool = False, algo: int = ALGO_AUTO,
                             stream=None) -> dict:
    """Gradients of decay_attention (gbla_decay_attention_backward): `do` [B, N, H, D]
    contiguous, `dstate` [B, H, D, D] the gradient of the returned state (None: zeros).
    Returns dq, dk, dv (0 past seq_lens; shared heads summed) and, with return_dstate,
    dstate, the gradient of the first state."""
    code, dev, ins, dims = _decay_args(q, k, v, log_decay, seq_lens, state)
    B, N, H, Hk, D = dims
    grads = (_plain(do, "do", q.shape, q.dtype, dev),
             _plain(dstate, "dstate", (B, H, D, D), torch.float32, dev))
    g = {"dq": _like(q, stream), "dk": _like(k, stream), "dv": _like(v, stream)}
    if return_dstate:
        g["dstate"] = _empty(stream, (B, H, D, D), torch.float32, q.device)
    out = [t.data_ptr() for t in g.values()] + ([] if return_dstate else [None])
    st = (_lib or load()).gbla_decay_attention_backward(
        *ins, *grads, *out, *dims, D ** -0.5 if scale is None else scale, code, algo,
        _raw_stream(dev, stream))
    _check(st, "gbla_decay_attention_backward")
    return g


def decay_attention_step(q, k, v, log_decay, state, slots=None, scale=None, out=None,
                         stream=None) -> torch.Tensor:
    """One token of each sequence (gbla_decay_attention_step): q [B, 1, H, D], k, v
    [B, 1, Hk, D]; `state` [n_slots, H, D, D] fp32 is updated in place at slots[b] (int32;
    None: slot b).  Rows whose slot is outside the pool are left alone.  Returns o."""
    B, N, H, D = shape = _dims(q)
    code, dev = _code(q)
    kshape = _key_shape(shape, k)
    if N != 1:
        raise ValueError("q, k and v hold one token of each sequence")
    whole = (_heads(q, "q", shape, q.dtype, dev) & _heads(k, "k", kshape, q.dtype, dev)
             & _heads(v, "v", kshape, q.dtype, dev))
    n_slots = state.shape[0]
    given = out is not None
    if not given:
        out = _like(q, stream)
    st = (_lib or load()).gbla_decay_attention_step(
        q.data_ptr(), k.data_ptr(), v.data_ptr(),
        _plain(log_decay, "log_decay", (H,), torch.float32, dev),
        _plain(slots, "slots", (B,), torch.int32, dev),
        None if whole else _strides(q, k, v, dims=1),
        _plain(state, "state", (n_slots, H, D, D), torch.float32, dev),
        _plain(out, "out", shape, q.dtype, dev), B, H, kshape[2], D, n_slots,
        D ** -0.5 if scale is None else scale, code, _raw_stream(dev, stream))
    _check(st, "gbla_decay_attention_step")
    _changed((state, out) if given else (state,))
    return out


def _gate(t, name, shape, dtype, dev):
    """Checks gates [B, N, H] whose heads are adjacent; True if they are contiguous."""
    if t.shape != shape:
        raise ValueError(f"{name} must be [B, N, H] = {tuple(shape)}, not {tuple(t.shape)}")
    if t.dtype is not dtype or t.get_device() != dev:
        raise ValueError(f"{name} must have the dtype and device of q")
    if t.is_contiguous():
        return True
    if shape[2] > 1 and t.stride(2) != 1:
        raise ValueError(f"the heads of {name} must be adjacent")
    return False


def _delta_args(q, k, v, log_decay, beta):
    """(code, device, whether all are contiguous, sizes): the inputs of the delta rule, whose
    heads and gates are those of the values."""
    B, N, Hk, D = _dims(q)
    if v.dim() != 4:
        raise ValueError("v must be [B, N, H, D]")
    code, dev = _code(q)
    H = v.shape[2]
    dt = q.dtype
    whole = (_heads(q, "q", (B, N, Hk, D), dt, dev) & _heads(k, "k", (B, N, Hk, D), dt, dev)
             & _heads(v, "v", (B, N, H, D), dt, dev)
             & _gate(log_decay, "log_decay", (B, N, H), dt, dev)
             & _gate(beta, "beta", (B, N, H), dt, dev))
    return code, dev, whole, (B, N, H, Hk, D)


def delta_attention(q, k, v, log_decay, beta, seq_lens=None, state=None, scale=None, out=None,
                    return_state: bool = False, stream=None):
    """Causal attention by the gated delta rule (gbla_delta_attention):
    kept = exp(log_decay_t) S_{t-1}, S_t = kept + k_t (beta_t (v_t - kept^T k_t))^T,
    o_t = scale S_t^T q_t for q, k [B, N, Hk, D], v [B, N, H, D] and gates log_decay, beta
    [B, N, H] (a value head reads query / key head h / (H / Hk)); `state` [B, H, D, D] fp32 is S
    before the first token, scale defaults to D^-1/2.  Keys of about unit length keep the state
    bounded (beta |k|^2 <= 2).  Returns o, or (o, S after each sequence's last token) with
    return_state; rows of o past seq_lens are not written."""
    code, dev, whole, dims = _delta_args(q, k, v, log_decay, beta)
    B, N, H, Hk, D = dims
    given = out is not None
    if not given:
        out = _like(v, stream)
    fin = _empty(stream, (B, H, D, D), torch.float32, q.device) if return_state else None
    st = (_lib or load()).gbla_delta_attention(
        q.data_ptr(), k.data_ptr(), v.data_ptr(), log_decay.data_ptr(), beta.data_ptr(),
        _plain(seq_lens, "seq_lens", (B,), torch.int32, dev),
        None if whole else _strides(q, k, v, log_decay, beta),
        _plain(state, "state", (B, H, D, D), torch.float32, dev),
        _plain(out, "out", v.shape, q.dtype, dev), None if fin is None else fin.data_ptr(),
        *dims, D ** -0.5 if scale is None else scale, code, _raw_stream(dev, stream))
    _check(st, "gbla_delta_attention")
    if given:
        _changed((out,))
    return (out, fin) if return_state else out


def delta_attention_backward(q, k, v, log_decay, beta, do, seq_lens=None, state=None, dstate=None,
                             scale=None, return_dstate: bool = False, stream=None) -> dict:
    """Gradients of delta_attention (gbla_delta_attention_backward): `do` [B, N, H, D]
    contiguous, `dstate` [B, H, D, D] the gradient of the returned state (None: zeros).
    Returns dq, dk (summed over the value heads that share a key head), dv, dlog_decay, dbeta
    (0 past seq_lens) and, with return_dstate, dstate, the gradient of the first state."""
    code, dev, whole, dims = _delta_args(q, k, v, log_decay, beta)
    B, N, H, Hk, D = dims
    f32 = torch.float32
    g = {"d" + n: _like(t, stream) for n, t in (("q", q), ("k", k), ("v", v),
                                                ("log_decay", log_decay), ("beta", beta))}
    if return_dstate:
        g["dstate"] = _empty(stream, (B, H, D, D), f32, q.device)
    out = [t.data_ptr() for t in g.values()] + ([] if return_dstate else [None])
    st = (_lib or load()).gbla_delta_attention_backward(
        q.data_ptr(), k.data_ptr(), v.data_ptr(), log_decay.data_ptr(), beta.data_ptr(),
        _plain(seq_lens, "seq_lens", (B,), torch.int32, dev),
        None if whole else _strides(q, k, v, log_decay, beta),
        _plain(state, "state", (B, H, D, D), f32, dev), _plain(do, "do", v.shape, q.dtype, dev),
        _plain(dstate, "dstate", (B, H, D, D), f32, dev), *out, *dims,
        D ** -0.5 if scale is None else scale, code, _raw_stream(dev, stream))
    _check(st, "gbla_delta_attention_backward")
    return g


def delta_attention_step(q, k, v, log_decay, beta, state, slots=None, scale=None, out=None,
                         stream=None) -> torch.Tensor:
    """One token of each sequence (gbla_delta_attention_step): q, k [B, 1, Hk, D], v
    [B, 1, H, D], log_decay, beta [B, 1, H]; `state` [n_slots, H, D, D] fp32 is updated in place
    at slots[b] (int32; None: slot b; no two the same).  Rows whose slot is outside the pool are
    left alone.  Returns o."""
    code, dev, whole, (B, N, H, Hk, D) = _delta_args(q, k, v, log_decay, beta)
    if N != 1:
        raise ValueError("q, k, v and the gates hold one token of each sequence")
    n_slots = state.shape[0]
    given = out is not None
    if not given:
        out = _like(v, stream)
    st = (_lib or load()).gbla_delta_attention_step(
        q.data_ptr(), k.data_ptr(), v.data_ptr(), log_decay.data_ptr(), beta.data_ptr(),
        _plain(slots, "slots", (B,), torch.int32, dev),
        None if whole else _strides(q, k, v, log_decay, beta, dims=1),
        _plain(state, "state", (n_slots, H, D, D), torch.float32, dev),
        _plain(out, "out", v.shape, q.dtype, dev), B, H, Hk, D, n_slots,
        D ** -0.5 if scale is None else scale, code, _raw_stream(dev, stream))
    _check(st, "gbla_delta_attention_step")
    _changed((state, out) if given else (state,))
    return out


def _logit_args(logits, tokens, seq_lens):
    """(code, device, addresses of logits, tokens, lengths and strides, sizes)."""
    if logits.dim() != 3:
        raise ValueError("logits must be [B, N, V]")
    B, N, V = logits.shape
    code, dev = _code(logits)
    whole = logits.is_contiguous()
    if not whole and V > 1 and logits.stride(2) != 1:
        raise ValueError("the values of a row of logits must be contiguous")
    return code, dev, (logits.data_ptr(), _plain(tokens, "tokens", (B, N), torch.int32, dev),
                       _plain(seq_lens, "seq_lens", (B,), torch.int32, dev),
                       None if whole else _strides(logits)), (B, N, V)


def token_logprobs(logits, tokens=None, top: int = 0, scale: float = 1.0, seq_lens=None, out=None,
                   stream=None) -> dict:
    """What rows of logits [B, N, V] say (gbla_token_logprobs), y = scale * logits: lse
    (ln sum exp y) and entropy [B, N]; with `tokens` [B, N] int32, logprob [B, N] (0 where the
    token is outside [0, V)); with `top` (at most 64), top_logprob and top_token [B, N, top] in
    descending order, equal logits by their tokens.  Logits of -inf are ruled out.  `out` may
    supply the tensors by these names; rows past seq_lens are not written."""
    code, dev, ins, (B, N, V) = _logit_args(logits, tokens, seq_lens)
    f32 = torch.float32
    shapes = {"lse": ((B, N), f32), "entropy": ((B, N), f32)}
    if tokens is not None:
        shapes["logprob"] = ((B, N), f32)
    if top:
        shapes |= {"top_logprob": ((B, N, top), f32), "top_token": ((B, N, top), torch.int32)}
    given = out is not None
    if given and out.keys() != shapes.keys():
        raise ValueError(f"out must hold {', '.join(shapes)}")
    if not given:
        out = {n: _empty(stream, shape, dt, logits.device) for n, (shape, dt) in shapes.items()}
    at = [_plain(out.get(n), n, *shapes.get(n, ((), f32)), dev)
          for n in ("lse", "entropy", "logprob", "top_logprob", "top_token")]
    st = (_lib or load()).gbla_token_logprobs(*ins, *at, B, N, V, top, scale, code,
                                              _raw_stream(dev, stream))
    _check(st, "gbla_token_logprobs")
    if given:
        _changed(tuple(out.values()))
    return out


def token_logprobs_backward(logits, lse, entropy, tokens=None, dlogprob=None, dentropy=None,
                            dlse=None, scale: float = 1.0, seq_lens=None, out=None,
                            stream=None) -> torch.Tensor:
    """Gradient of the logits (gbla_token_logprobs_backward) for the gradients dlogprob,
    dentropy and dlse [B, N] fp32 (None: zeros) of token_logprobs' results, from its lse and
    entropy.  Rows past seq_lens are 0.  `out` [B, N, V] contiguous may be the logits
    themselves, which are overwritten then."""
    code, dev, (at, tok, lens, strides), (B, N, V) = _logit_args(logits, tokens, seq_lens)
    given = out is not None
    if not given:
        out = _like(logits, stream)
    small = [_plain(t, n, (B, N), torch.float32, dev)
             for t, n in ((lse, "lse"), (entropy, "entropy"), (dlogprob, "dlogprob"),
                          (dentropy, "dentropy"), (dlse, "dlse"))]
    if lse is None or entropy is None:
        raise ValueError("lse and entropy of the forward call are needed")
    st = (_lib or load()).gbla_token_logprobs_backward(
        at, *small[:2], tok, lens, strides, *small[2:],
        _plain(out, "out", logits.shape, logits.dtype, dev), B, N, V, scale, code,
        _raw_stream(dev, stream))
    _check(st, "gbla_token_logprobs_backward")
    if given:
        _changed((out,))
    return out
