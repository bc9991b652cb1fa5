"""ctypes binding of libolive_score.so (the C ABI of include/olive_score.h and
include/olive_layers.h).

Argument marshalling only: every function has the C name and forwards plain
pointers, sizes and the HIP stream. Torch tensors are accepted wherever the C
function takes a device pointer (their data_ptr() is passed); None maps to NULL.
The layer operators' functions refuse tensors of another type or layout than the
library would read (ValueError); the sizes of the heads' views are the caller's.
The library must have been built (python -m paper_2609_36246_amd.build); loading
fails loudly otherwise -- there is no fallback path.
"""
from __future__ import annotations

import ctypes
import os
import struct
import threading
from typing import Optional

PKG = os.path.dirname(os.path.abspath(__file__))
LIB_PATH = os.path.join(PKG, "libolive_score.so")

OLIVE_OK = 0
OLIVE_E_NULL = 1
OLIVE_E_SHAPE = 2
OLIVE_E_DTYPE = 3
OLIVE_E_RANGE = 4
OLIVE_E_HIP = 5
OLIVE_E_NOMEM = 6
OLIVE_E_UNSUPPORTED = 7
OLIVE_E_LIMIT = 8
STATUS_CODES = list(range(9))

OLIVE_F32 = 0
OLIVE_BF16 = 1
OLIVE_W_DV = 0
OLIVE_W_VD = 1
OLIVE_REGION_TEACHER = 0
OLIVE_REGION_STUDENT = 1
OLIVE_REGION_ALL = 2
OLIVE_REGION_SPANS = 3
OLIVE_FLAG_SIMPLE_KERNEL = 1
OLIVE_FLAG_KERNEL_TIMING = 2
OLIVE_FLAG_TOPK = 4
OLIVE_FLAG_BACKWARD = 8
OLIVE_FLAG_NARROW_TILE = 16
OLIVE_GRAD_REUSE_FORWARD = 1
OLIVE_TOPK = 16
OLIVE_OUT_REGION_ONLY = 1
OLIVE_ROPE_HALF = 0
OLIVE_ROPE_PAIRS = 1


class olive_score_desc(ctypes.Structure):
    _fields_ = [("vocab", ctypes.c_int64), ("d_student", ctypes.c_int32),
                ("d_teacher", ctypes.c_int32), ("dtype", ctypes.c_int32),
                ("w_layout", ctypes.c_int32), ("logit_scale_student", ctypes.c_float),
                ("logit_scale_teacher", ctypes.c_float), ("max_positions", ctypes.c_int64),
                ("max_seqs", ctypes.c_int32), ("flags", ctypes.c_int32)]


class olive_batch(ctypes.Structure):
    _fields_ = [("num_seqs", ctypes.c_int32), ("region", ctypes.c_int32),
                ("total_positions", ctypes.c_int64), ("cu_seqlens", ctypes.c_void_p),
                ("cut", ctypes.c_void_p), ("valid_len", ctypes.c_void_p),
                ("targets", ctypes.c_void_p), ("h_student", ctypes.c_void_p),
                ("h_teacher", ctypes.c_void_p)]


class olive_score_outputs(ctypes.Structure):
    _fields_ = [("size", ctypes.c_int32), ("flags", ctypes.c_int32),
                ("kl", ctypes.c_void_p), ("kl_reverse", ctypes.c_void_p),
                ("counts", ctypes.c_void_p), ("logp_student", ctypes.c_void_p),
                ("logp_teacher", ctypes.c_void_p), ("argmax_student", ctypes.c_void_p),
                ("argmax_teacher", ctypes.c_void_p), ("ce_per_seq", ctypes.c_void_p),
                ("topk_overlap", ctypes.c_void_p), ("kl_topk", ctypes.c_void_p),
                ("topk_student", ctypes.c_void_p), ("topk_teacher", ctypes.c_void_p),
                ("jsd", ctypes.c_void_p)]


class olive_grad_outputs(ctypes.Structure):
    _fields_ = [("size", ctypes.c_int32), ("flags", ctypes.c_int32),
                ("w_ce", ctypes.c_float), ("w_kl", ctypes.c_float),
                ("grad_h_student", ctypes.c_void_p), ("grad_w_student", ctypes.c_void_p),
                ("counts", ctypes.c_void_p)]


class olive_spans(ctypes.Structure):
    _fields_ = [("size", ctypes.c_int32), ("num_spans", ctypes.c_int32),
                ("span_offsets", ctypes.c_void_p), ("spans", ctypes.c_void_p)]


class olive_heads(ctypes.Structure):
    _fields_ = [("data", ctypes.c_void_p), ("stride_token", ctypes.c_int64),
                ("stride_head", ctypes.c_int64)]


class olive_qk_desc(ctypes.Structure):
    _fields_ = [("size", ctypes.c_int32), ("dtype", ctypes.c_int32), ("tokens", ctypes.c_int64),
                ("heads_q", ctypes.c_int32), ("heads_k", ctypes.c_int32),
                ("head_dim", ctypes.c_int32), ("rot_dim", ctypes.c_int32),
                ("layout", ctypes.c_int32), ("eps", ctypes.c_float),
                ("positions", ctypes.c_void_p), ("num_positions", ctypes.c_int64),
                ("cos", ctypes.c_void_p), ("sin", ctypes.c_void_p),
                ("weight_q", ctypes.c_void_p), ("weight_k", ctypes.c_void_p),
                ("slots", ctypes.c_void_p), ("slot_rows", ctypes.c_int64)]


class olive_attn_desc(ctypes.Structure):
    _fields_ = [("size", ctypes.c_int32), ("dtype", ctypes.c_int32),
                ("num_groups", ctypes.c_int32), ("num_seqs", ctypes.c_int32),
                ("heads_q", ctypes.c_int32), ("heads_kv", ctypes.c_int32),
                ("head_dim", ctypes.c_int32), ("max_q", ctypes.c_int32),
                ("total_q", ctypes.c_int64), ("max_prefix", ctypes.c_int64),
                ("max_suffix", ctypes.c_int64), ("prefix_rows", ctypes.c_int64),
                ("suffix_rows", ctypes.c_int64), ("group_seqs", ctypes.c_void_p),
                ("cu_q", ctypes.c_void_p), ("prefix_start", ctypes.c_void_p),
                ("prefix_len", ctypes.c_void_p), ("suffix_len", ctypes.c_void_p),
                ("suffix_start", ctypes.c_void_p), ("page_table", ctypes.c_void_p),
                ("table_stride", ctypes.c_int64), ("page_size", ctypes.c_int32),
                ("scale", ctypes.c_float)]


class olive_grad_tensor(ctypes.Structure):
    _fields_ = [("grad", ctypes.c_void_p), ("out", ctypes.c_void_p), ("n", ctypes.c_int64),
                ("dtype", ctypes.c_int32), ("dtype_out", ctypes.c_int32)]


class OliveError(RuntimeError):
    def __init__(self, status: int, what: str):
        self.status = status
        super().__init__("%s failed: %s" % (what, olive_status_string(status)))


_lib: Optional[ctypes.CDLL] = None
_calls = {}              # the layer operators' entries with addresses for every pointer


def load() -> ctypes.CDLL:
    """Load the built library (once) and declare its signatures."""
    global _lib
    if _lib is not None:
        return _lib
    if not os.path.exists(LIB_PATH):
        raise ImportError("libolive_score.so is not built (run: python -m "
                          "paper_2609_36246_amd.build); there is no fallback")
    # torch's HIP runtime must be resident first: the library's libamdhip64.so.7 then
    # resolves to it by soname.  Loaded the other way round, torch (which asks for the
    # file libamdhip64.so) brings a second runtime into the process and the library's
    # calls see no device and cannot use torch's streams or allocations.
    import torch  # noqa: F401
    lib = ctypes.CDLL(LIB_PATH)
    vp, i32p, i64p, f32p = ctypes.c_void_p, ctypes.c_void_p, ctypes.c_void_p, ctypes.c_void_p
    st = ctypes.c_int
    lib.olive_score_init.argtypes = [ctypes.POINTER(ctypes.c_void_p),
                                     ctypes.POINTER(olive_score_desc), vp, vp, vp]
    lib.olive_score_init.restype = st
    lib.olive_token_logprobs.argtypes = [vp, ctypes.POINTER(olive_batch), f32p, f32p, i32p, i32p,
                                         vp]
    lib.olive_token_logprobs.restype = st
    lib.olive_kl_masked.argtypes = [vp, ctypes.POINTER(olive_batch), f32p, i64p, f32p, f32p,
                                    i32p, i32p, f32p, vp]
    lib.olive_kl_masked.restype = st
    lib.olive_kl_masked_static.argtypes = [ctypes.POINTER(olive_score_desc), vp, vp,
                                           ctypes.POINTER(olive_batch), f32p, i64p, f32p, f32p,
                                           i32p, i32p, f32p, vp]
    lib.olive_kl_masked_static.restype = st
    lib.olive_score_batch.argtypes = [vp, ctypes.POINTER(olive_batch),
                                      ctypes.POINTER(olive_score_outputs), vp]
    lib.olive_score_batch.restype = st
    lib.olive_score_batch_spans.argtypes = [vp, ctypes.POINTER(olive_batch),
                                            ctypes.POINTER(olive_spans),
                                            ctypes.POINTER(olive_score_outputs), vp]
    lib.olive_score_batch_spans.restype = st
    lib.olive_score_backward.argtypes = [vp, ctypes.POINTER(olive_batch),
                                         ctypes.POINTER(olive_spans),
                                         ctypes.POINTER(olive_grad_outputs), vp]
    lib.olive_score_backward.restype = st
    lib.olive_score_free.argtypes = [vp]
    lib.olive_score_free.restype = st
    lib.olive_status_string.argtypes = [st]
    lib.olive_status_string.restype = ctypes.c_char_p
    lib.olive_score_last_error.argtypes = [vp, ctypes.POINTER(ctypes.c_int32)]
    lib.olive_score_last_error.restype = st
    lib.olive_score_last_stats.argtypes = [vp, ctypes.POINTER(ctypes.c_int64)]
    lib.olive_score_last_stats.restype = st
    lib.olive_score_kernel_times.argtypes = [vp, ctypes.POINTER(ctypes.c_float), ctypes.c_int]
    lib.olive_score_kernel_times.restype = st
    for name, args in (("olive_qk_norm_rope", "p" * 8), ("olive_qk_norm_rope_backward", "p" * 10 + "lp"),
                       ("olive_prefix_attention", "p" * 9 + "lp"),
                       ("olive_prefix_attention_backward", "p" * 15 + "lp"),
                       ("olive_grad_clip", "pfpp")):
        kinds = {"p": vp, "l": ctypes.c_int64, "f": ctypes.c_float}
        _calls[name] = ctypes.CFUNCTYPE(st, *(kinds[a] for a in args))((name, lib))
    hp, qp = ctypes.POINTER(olive_heads), ctypes.POINTER(olive_qk_desc)
    ap, i64 = ctypes.POINTER(olive_attn_desc), ctypes.c_int64
    lib.olive_qk_norm_rope.argtypes = [qp] + [hp] * 6 + [vp]
    lib.olive_qk_norm_rope.restype = st
    lib.olive_qk_norm_rope_workspace.argtypes = [qp, ctypes.POINTER(i64)]
    lib.olive_qk_norm_rope_workspace.restype = st
    lib.olive_qk_norm_rope_backward.argtypes = [qp] + [hp] * 6 + [f32p, f32p, vp, i64, vp]
    lib.olive_qk_norm_rope_backward.restype = st
    lib.olive_prefix_attention_workspace.argtypes = [ap, ctypes.c_int32, ctypes.POINTER(i64)]
    lib.olive_prefix_attention_workspace.restype = st
    lib.olive_prefix_attention.argtypes = [ap] + [hp] * 6 + [f32p, vp, i64, vp]
    lib.olive_prefix_attention.restype = st
    lib.olive_prefix_attention_backward.argtypes = [ap] + [hp] * 6 + [f32p] + [hp] * 6 + \
        [vp, i64, vp]
    lib.olive_prefix_attention_backward.restype = st
    lib.olive_grad_clip_init.argtypes = [ctypes.POINTER(ctypes.c_void_p),
                                         ctypes.POINTER(olive_grad_tensor), ctypes.c_int32, vp]
    lib.olive_grad_clip_init.restype = st
    lib.olive_grad_clip.argtypes = [vp, ctypes.c_float, f32p, vp]
    lib.olive_grad_clip.restype = st
    lib.olive_grad_clip_free.argtypes = [vp]
    lib.olive_grad_clip_free.restype = st
    _lib = lib
    return lib


def _ptr(x) -> Optional[int]:
    if x is None:
        return None
    if isinstance(x, int):
        return x
    return x.data_ptr()


def _stream(stream) -> Optional[int]:
    if stream is None:
        import torch
        # torch's bare handle where this torch has it: the public call makes a Stream object each
        # time, of the same handle
        raw = getattr(torch._C, "_cuda_getCurrentRawStream", None)
        return torch.cuda.current_stream().cuda_stream if raw is None else raw(torch.cuda.current_device())
    if isinstance(stream, int):
        return stream
    return stream.cuda_stream


def _check(status: int, what: str):
    if status != OLIVE_OK:
        raise OliveError(status, what)


def olive_status_string(status: int) -> str:
    return load().olive_status_string(status).decode()


def olive_score_init(desc: olive_score_desc, w_student, w_teacher=None, stream=None,
                     check: bool = True):
    """Returns an opaque context handle (int). Raises OliveError unless check=False,
    in which case (status, handle) is returned."""
    h = ctypes.c_void_p()
    s = load().olive_score_init(ctypes.byref(h), ctypes.byref(desc), _ptr(w_student),
                                _ptr(w_teacher), _stream(stream) if check else stream)
    if not check:
        return s, h.value
    _check(s, "olive_score_init")
    return h.value


def make_batch(cu_seqlens, cut, targets, h_student, h_teacher=None, valid_len=None,
               region: int = OLIVE_REGION_TEACHER, total_positions: Optional[int] = None,
               num_seqs: Optional[int] = None) -> olive_batch:
    """An olive_batch over device tensors (the caller keeps them alive)."""
    b = olive_batch()
    b.num_seqs = int(num_seqs if num_seqs is not None else cu_seqlens.shape[0] - 1)
    b.region = int(region)
    b.total_positions = int(total_positions if total_positions is not None
                            else targets.shape[0])
    b.cu_seqlens = _ptr(cu_seqlens)
    b.cut = _ptr(cut)
    b.valid_len = _ptr(valid_len)
    b.targets = _ptr(targets)
    b.h_student = _ptr(h_student)
    b.h_teacher = _ptr(h_teacher)
    return b


def olive_token_logprobs(ctx, batch: olive_batch, logp_student, logp_teacher=None,
                         argmax_student=None, argmax_teacher=None, stream=None,
                         check: bool = True) -> int:
    s = load().olive_token_logprobs(ctx, ctypes.byref(batch), _ptr(logp_student),
                                    _ptr(logp_teacher), _ptr(argmax_student),
                                    _ptr(argmax_teacher), _stream(stream))
    if check:
        _check(s, "olive_token_logprobs")
    return s


def olive_kl_masked(ctx, batch: olive_batch, kl, counts=None, logp_student=None,
                    logp_teacher=None, argmax_student=None, argmax_teacher=None,
                    ce_per_seq=None, stream=None, check: bool = True) -> int:
    s = load().olive_kl_masked(ctx, ctypes.byref(batch), _ptr(kl), _ptr(counts),
                               _ptr(logp_student), _ptr(logp_teacher), _ptr(argmax_student),
                               _ptr(argmax_teacher), _ptr(ce_per_seq), _stream(stream))
    if check:
        _check(s, "olive_kl_masked")
    return s


def olive_kl_masked_static(desc: olive_score_desc, w_student, w_teacher, batch: olive_batch,
                           kl, counts=None, logp_student=None, logp_teacher=None,
                           argmax_student=None, argmax_teacher=None, ce_per_seq=None,
                           stream=None, check: bool = True) -> int:
    """olive_kl_masked without a context ([V][d] weights read in place; nothing is
    allocated: the library's fixed per-GPU scratch array holds the workspace)."""
    s = load().olive_kl_masked_static(ctypes.byref(desc), _ptr(w_student), _ptr(w_teacher),
                                      ctypes.byref(batch), _ptr(kl), _ptr(counts),
                                      _ptr(logp_student), _ptr(logp_teacher),
                                      _ptr(argmax_student), _ptr(argmax_teacher),
                                      _ptr(ce_per_seq), _stream(stream))
    if check:
        _check(s, "olive_kl_masked_static")
    return s


def make_outputs(kl=None, kl_reverse=None, counts=None, logp_student=None, logp_teacher=None,
                 argmax_student=None, argmax_teacher=None, ce_per_seq=None,
                 topk_overlap=None, kl_topk=None, topk_student=None, topk_teacher=None,
                 jsd=None, flags: int = 0) -> olive_score_outputs:
    o = olive_score_outputs()
    o.size = ctypes.sizeof(olive_score_outputs)
    o.flags = int(flags)
    o.kl, o.kl_reverse, o.counts = _ptr(kl), _ptr(kl_reverse), _ptr(counts)
    o.logp_student, o.logp_teacher = _ptr(logp_student), _ptr(logp_teacher)
    o.argmax_student, o.argmax_teacher = _ptr(argmax_student), _ptr(argmax_teacher)
    o.ce_per_seq = _ptr(ce_per_seq)
    o.topk_overlap, o.kl_topk = _ptr(topk_overlap), _ptr(kl_topk)
    o.topk_student, o.topk_teacher = _ptr(topk_student), _ptr(topk_teacher)
    o.jsd = _ptr(jsd)
    return o


def olive_score_batch(ctx, batch: olive_batch, outputs: olive_score_outputs, stream=None,
                      check: bool = True) -> int:
    s = load().olive_score_batch(ctx, ctypes.byref(batch), ctypes.byref(outputs),
                                 _stream(stream))
    if check:
        _check(s, "olive_score_batch")
    return s


def make_spans(span_offsets, span_pairs, num_spans: Optional[int] = None) -> olive_spans:
    """An olive_spans over device tensors: offsets [B+1] int32, pairs [S, 2] int32."""
    sp = olive_spans()
    sp.size = ctypes.sizeof(olive_spans)
    sp.num_spans = int(num_spans if num_spans is not None else span_pairs.shape[0])
    sp.span_offsets = _ptr(span_offsets)
    sp.spans = _ptr(span_pairs) if sp.num_spans > 0 else None
    return sp


def make_grad_outputs(w_ce=1.0, w_kl=0.0, grad_h=None, grad_w=None,
                      counts=None, reuse_forward=False) -> olive_grad_outputs:
    o = olive_grad_outputs()
    o.size = ctypes.sizeof(olive_grad_outputs)
    o.flags = OLIVE_GRAD_REUSE_FORWARD if reuse_forward else 0
    o.w_ce, o.w_kl = float(w_ce), float(w_kl)
    o.grad_h_student, o.grad_w_student = _ptr(grad_h), _ptr(grad_w)
    o.counts = _ptr(counts)
    return o


def olive_score_backward(ctx, batch: olive_batch, grads: olive_grad_outputs, spans=None,
                         stream=None, check: bool = True) -> int:
    s = load().olive_score_backward(ctx, ctypes.byref(batch),
                                    ctypes.byref(spans) if spans is not None else None,
                                    ctypes.byref(grads), _stream(stream))
    if check:
        _check(s, "olive_score_backward")
    return s


def olive_score_batch_spans(ctx, batch: olive_batch, spans: olive_spans,
                            outputs: olive_score_outputs, stream=None, check: bool = True) -> int:
    s = load().olive_score_batch_spans(ctx, ctypes.byref(batch), ctypes.byref(spans),
                                       ctypes.byref(outputs), _stream(stream))
    if check:
        _check(s, "olive_score_batch_spans")
    return s


def olive_score_free(ctx) -> int:
    return load().olive_score_free(ctx)


def olive_score_last_error(ctx) -> int:
    v = ctypes.c_int32(0)
    _check(load().olive_score_last_error(ctx, ctypes.byref(v)), "olive_score_last_error")
    return v.value


def olive_score_last_stats(ctx) -> dict:
    out = (ctypes.c_int64 * 6)()
    _check(load().olive_score_last_stats(ctx, out), "olive_score_last_stats")
    kid = out[2]
    return dict(splits=out[0], flagged=out[1],
                kernel={0: "mfma", 1: "generic", 2: "mfma"}.get(kid),
                tile={0: "256x128", 2: "256x256"}.get(kid), grid=out[3],
                topk_filtered=out[4], topk_scanned=out[5])


def olive_score_kernel_times(ctx, n: int) -> list:
    """Durations (ms) of the scoring kernel in the last n calls (needs the timing flag)."""
    buf = (ctypes.c_float * n)()
    _check(load().olive_score_kernel_times(ctx, buf, n), "olive_score_kernel_times")
    return list(buf)


def make_desc(vocab, d_student, d_teacher, dtype=OLIVE_BF16, w_layout=OLIVE_W_DV,
              scale_student=1.0, scale_teacher=1.0, max_positions=1, max_seqs=1,
              flags=0) -> olive_score_desc:
    d = olive_score_desc()
    d.vocab = int(vocab)
    d.d_student = int(d_student)
    d.d_teacher = int(d_teacher)
    d.dtype = int(dtype)
    d.w_layout = int(w_layout)
    d.logit_scale_student = float(scale_student)
    d.logit_scale_teacher = float(scale_teacher)
    d.max_positions = int(max_positions)
    d.max_seqs = int(max_seqs)
    d.flags = int(flags)
    return d


def make_heads(x) -> Optional[olive_heads]:
    """An olive_heads over a [tokens, heads, head_dim] tensor whose last dimension is
    contiguous (None stays None; the caller keeps the tensor alive)."""
    if x is None or isinstance(x, olive_heads):
        return x
    s = x.stride()
    if len(s) != 3 or (s[2] != 1 and x.shape[2] > 1):
        raise ValueError("expected [tokens, heads, head_dim] with contiguous heads")
    return olive_heads(x.data_ptr(), s[0], s[1])


_dtypes = {}             # torch's types by olive_dtype or name, at the first call


def _dtype(kind):
    if not _dtypes:
        import torch
        _dtypes.update({OLIVE_F32: torch.float32, OLIVE_BF16: torch.bfloat16, "int32": torch.int32,
                        "int64": torch.int64})
    return _dtypes.get(kind)


def _array(x, kind, least: int, what: str) -> Optional[int]:
    """Address of a contiguous tensor of a type (_dtype) with at least so many elements (None
    and an address are taken as they are)."""
    if x is None or isinstance(x, int):
        return x
    if x.dtype is not _dtype(kind) or not x.is_contiguous() or x.numel() < least:
        raise ValueError("%s: expected a contiguous tensor of %s, %d elements at least" % (what, _dtype(kind), least))
    return x.data_ptr()


class _Views(threading.local):
    """A thread's olive_heads of one call: written before it, read by it before it returns."""

    def __init__(self):
        self.buffer = ctypes.create_string_buffer(16 * ctypes.sizeof(olive_heads))
        self.at = [ctypes.addressof(self.buffer) + i * ctypes.sizeof(olive_heads) for i in range(16)]


_views = _Views()
_packers = [struct.Struct("=%dq" % (3 * i)) for i in range(17)]


def _heads(desc, *xs):
    """Addresses of the views' olive_heads (one object made for each would cost more time than
    a small call on the GPU)."""
    values, at, dtype = [], [], _dtype(desc.dtype)
    for x, place in zip(xs, _views.at):
        if x is None:
            values += (0, 0, 0)
            at.append(None)
            continue
        at.append(place)
        if isinstance(x, olive_heads):
            values += (x.data or 0, x.stride_token, x.stride_head)
            continue
        s = x.stride()
        if len(s) != 3 or x.dtype is not dtype or (s[2] != 1 and x.shape[2] > 1):
            raise ValueError("expected [tokens, heads, head_dim] of the descriptor's dtype (%s) with contiguous heads"
                             % dtype)
        values += (x.data_ptr(), s[0], s[1])
    _packers[len(at)].pack_into(_views.buffer, 0, *values)
    return at


def _call(name):
    if _lib is None:
        load()
    return _calls[name]


def _workspace(w):
    if w is None:
        return None, 0
    if not w.is_contiguous():
        raise ValueError("a workspace is a contiguous tensor")
    return w.data_ptr(), w.numel() * w.element_size()


def make_qk_desc(tokens, heads_q, heads_k, head_dim, positions=None, cos=None, sin=None,
                 weight_q=None, weight_k=None, dtype=OLIVE_BF16, eps=1e-6, layout=OLIVE_ROPE_HALF,
                 rot_dim=None, num_positions=None, slots=None, slot_rows=0) -> olive_qk_desc:
    """cos and sin: fp32 [num_positions, rot_dim / 2], which give the default sizes; positions
    and slots int32, the weights of the heads' dtype, all contiguous. The descriptor keeps its
    tensors alive."""
    d = olive_qk_desc()
    d.size = ctypes.sizeof(olive_qk_desc)
    d.dtype, d.tokens = int(dtype), int(tokens)
    d.heads_q, d.heads_k, d.head_dim = int(heads_q), int(heads_k), int(head_dim)
    d.rot_dim = int(rot_dim if rot_dim is not None else 0 if cos is None else 2 * cos.shape[1])
    d.num_positions = int(num_positions if num_positions is not None
                          else 0 if cos is None else cos.shape[0])
    d.layout, d.eps = int(layout), float(eps)
    for table in (cos, sin) if d.rot_dim else ():
        if not (table is None or isinstance(table, int)) and 2 * table.shape[-1] != d.rot_dim:
            raise ValueError("cos and sin have rot_dim / 2 columns")
    d.positions = _array(positions, "int32", d.tokens, "positions")
    angles = d.num_positions * d.rot_dim // 2
    d.cos, d.sin = _array(cos, OLIVE_F32, angles, "cos"), _array(sin, OLIVE_F32, angles, "sin")
    d.weight_q = _array(weight_q, d.dtype, d.head_dim, "weight_q")
    d.weight_k = _array(weight_k, d.dtype, d.head_dim, "weight_k")
    d.slots, d.slot_rows = _array(slots, "int32", d.tokens, "slots"), int(slot_rows)
    d.tensors = (positions, cos, sin, weight_q, weight_k, slots)
    return d


def olive_qk_norm_rope(desc: olive_qk_desc, q, k, q_out, k_out, v=None, v_out=None, stream=None,
                       check: bool = True) -> int:
    s = _call("olive_qk_norm_rope")(ctypes.addressof(desc), *_heads(desc, q, k, v, q_out, k_out, v_out),
                                    _stream(stream))
    if check:
        _check(s, "olive_qk_norm_rope")
    return s


def olive_qk_norm_rope_workspace(desc: olive_qk_desc) -> int:
    """Bytes of olive_qk_norm_rope_backward's workspace."""
    n = ctypes.c_int64(0)
    _check(load().olive_qk_norm_rope_workspace(ctypes.byref(desc), ctypes.byref(n)),
           "olive_qk_norm_rope_workspace")
    return n.value


def olive_qk_norm_rope_backward(desc: olive_qk_desc, q, k, grad_q_out, grad_k_out, grad_q, grad_k,
                                grad_weight_q=None, grad_weight_k=None, workspace=None,
                                stream=None, check: bool = True) -> int:
    s = _call("olive_qk_norm_rope_backward")(
        ctypes.addressof(desc), *_heads(desc, q, k, grad_q_out, grad_k_out, grad_q, grad_k),
        _array(grad_weight_q, OLIVE_F32, desc.head_dim, "grad_weight_q"),
        _array(grad_weight_k, OLIVE_F32, desc.head_dim, "grad_weight_k"), *_workspace(workspace), _stream(stream))
    if check:
        _check(s, "olive_qk_norm_rope_backward")
    return s


def make_attn_desc(heads_q, heads_kv, head_dim, group_seqs, cu_q, prefix_start, prefix_len,
                   suffix_len, total_q, max_q, max_prefix, max_suffix, prefix_rows, suffix_rows,
                   suffix_start=None, page_table=None, page_size=0, dtype=OLIVE_BF16,
                   scale=None, num_groups=None, num_seqs=None) -> olive_attn_desc:
    """Device tensors: group_seqs [G + 1], cu_q [B + 1], prefix_len [G], suffix_len [B] int32,
    prefix_start [G], suffix_start [B] int64, page_table [B, pages] int32 (its rows at any
    distance, the others contiguous). The descriptor keeps them alive."""
    d = olive_attn_desc()
    d.size = ctypes.sizeof(olive_attn_desc)
    d.dtype = int(dtype)
    d.num_groups = int(num_groups if num_groups is not None else prefix_len.shape[0])
    d.num_seqs = int(num_seqs if num_seqs is not None else suffix_len.shape[0])
    d.heads_q, d.heads_kv, d.head_dim = int(heads_q), int(heads_kv), int(head_dim)
    d.max_q, d.total_q = int(max_q), int(total_q)
    d.max_prefix, d.max_suffix = int(max_prefix), int(max_suffix)
    d.prefix_rows, d.suffix_rows = int(prefix_rows), int(suffix_rows)
    G, B = d.num_groups, d.num_seqs
    d.group_seqs, d.cu_q = _array(group_seqs, "int32", G + 1, "group_seqs"), _array(cu_q, "int32", B + 1, "cu_q")
    d.prefix_start = _array(prefix_start, "int64", G, "prefix_start")
    d.prefix_len = _array(prefix_len, "int32", G, "prefix_len")
    d.suffix_len = _array(suffix_len, "int32", B, "suffix_len")
    d.suffix_start = _array(suffix_start, "int64", B, "suffix_start")
    d.page_table, d.page_size = _ptr(page_table), int(page_size)
    if page_table is not None and not isinstance(page_table, int):
        if page_table.dtype is not _dtype("int32") or page_table.dim() != 2 or page_table.shape[0] < B or \
                (page_table.shape[1] > 1 and page_table.stride(1) != 1):
            raise ValueError("page_table: expected int32 [%d, pages] with contiguous rows" % B)
        d.table_stride = page_table.stride(0)
    d.scale = float(scale if scale is not None else head_dim ** -0.5)
    d.tensors = (group_seqs, cu_q, prefix_start, prefix_len, suffix_len, suffix_start, page_table)
    return d


def olive_prefix_attention_workspace(desc: olive_attn_desc, backward: bool = False) -> int:
    """Bytes of the workspace of olive_prefix_attention, with `backward` of its backward's
    where that is more."""
    most = 0
    for b in (0, 1) if backward else (0,):
        n = ctypes.c_int64(0)
        _check(load().olive_prefix_attention_workspace(ctypes.byref(desc), b, ctypes.byref(n)),
               "olive_prefix_attention_workspace")
        most = max(most, n.value)
    return most


def olive_prefix_attention(desc: olive_attn_desc, q, k_prefix, v_prefix, k_suffix, v_suffix, out,
                           lse=None, workspace=None, stream=None, check: bool = True) -> int:
    s = _call("olive_prefix_attention")(
        ctypes.addressof(desc), *_heads(desc, q, k_prefix, v_prefix, k_suffix, v_suffix, out),
        _array(lse, OLIVE_F32, desc.total_q * desc.heads_q, "lse"), *_workspace(workspace), _stream(stream))
    if check:
        _check(s, "olive_prefix_attention")
    return s


def olive_prefix_attention_backward(desc: olive_attn_desc, q, k_prefix, v_prefix, k_suffix,
                                    v_suffix, out, lse, grad_out, grad_q, grad_k_prefix,
                                    grad_v_prefix, grad_k_suffix, grad_v_suffix, workspace=None,
                                    stream=None, check: bool = True) -> int:
    at = _heads(desc, q, k_prefix, v_prefix, k_suffix, v_suffix, out, grad_out, grad_q, grad_k_prefix,
                grad_v_prefix, grad_k_suffix, grad_v_suffix)
    s = _call("olive_prefix_attention_backward")(
        ctypes.addressof(desc), *at[:6], _array(lse, OLIVE_F32, desc.total_q * desc.heads_q, "lse"), *at[6:],
        *_workspace(workspace), _stream(stream))
    if check:
        _check(s, "olive_prefix_attention_backward")
    return s


def _dtype_of(x) -> int:
    kinds = {"torch.bfloat16": OLIVE_BF16, "torch.float32": OLIVE_F32}
    if str(x.dtype) not in kinds or not x.is_contiguous():
        raise ValueError("a gradient is a contiguous bf16 or fp32 tensor")
    return kinds[str(x.dtype)]


def olive_grad_clip_init(grads, outs=None, stream=None) -> int:
    """A context for a list of contiguous gradients, scaled in place, or into `outs` (None
    entries: only counted). The caller keeps the tensors alive."""
    outs = grads if outs is None else outs
    if len(outs) != len(grads):
        raise ValueError("one output for each gradient")
    arr = (olive_grad_tensor * max(1, len(grads)))()
    for i, (g, o) in enumerate(zip(grads, outs)):
        if o is not None and o.numel() != g.numel():
            raise ValueError("an output has its gradient's size")
        kind = _dtype_of(g)
        arr[i] = olive_grad_tensor(_ptr(g), _ptr(o), g.numel(), kind,
                                   kind if o is None else _dtype_of(o))
    h = ctypes.c_void_p()
    _check(load().olive_grad_clip_init(ctypes.byref(h), arr, len(grads), _stream(stream)),
           "olive_grad_clip_init")
    return h.value


def olive_grad_clip(ctx, max_norm: float, norm=None, stream=None, check: bool = True) -> int:
    s = _call("olive_grad_clip")(ctx, max_norm, _array(norm, OLIVE_F32, 1, "norm"), _stream(stream))
    if check:
        _check(s, "olive_grad_clip")
    return s


def olive_grad_clip_free(ctx) -> int:
    return load().olive_grad_clip_free(ctx)
