"""ctypes binding of the operator-level entry points (include/fax_ops.h)."""
from __future__ import annotations

import ctypes as C

FAX_EPI_NONE, FAX_EPI_BIAS, FAX_EPI_BIAS_GELU, FAX_EPI_BIAS_RESID, FAX_EPI_DGELU = range(5)

_P = C.c_void_p


class GemmDesc(C.Structure):
    _fields_ = [("M", C.c_int32), ("N", C.c_int32), ("K", C.c_int32),
                ("A", _P), ("lda", C.c_int64), ("a_mn_major", C.c_int32),
                ("B", _P), ("ldb", C.c_int64), ("b_mn_major", C.c_int32),
                ("C", _P), ("ldc", C.c_int64), ("c_f32", C.c_int32), ("accumulate", C.c_int32),
                ("epilogue", C.c_int32), ("bias", _P), ("resid", _P), ("ldr", C.c_int64),
                ("aux", _P), ("ldaux", C.c_int64), ("alpha", C.c_float), ("force_simt", C.c_int32)]


FAX_FP8_E4M3, FAX_FP8_E5M2 = range(2)
FAX_FP8_BLOCK = 128


class Fp8QuantizeDesc(C.Structure):
    _fields_ = [("rows", C.c_int32), ("cols", C.c_int32), ("x", _P), ("ldx", C.c_int64),
                ("format", C.c_int32), ("tile", C.c_int32),
                ("q", _P), ("ldq", C.c_int64), ("s", _P), ("lds", C.c_int64),
                ("qt", _P), ("ldqt", C.c_int64), ("st", _P), ("ldst", C.c_int64)]


class Fp8GemmDesc(C.Structure):
    _fields_ = [("M", C.c_int32), ("N", C.c_int32), ("K", C.c_int32),
                ("A", _P), ("lda", C.c_int64), ("a_format", C.c_int32), ("a_scale", _P), ("a_scale_ld", C.c_int64),
                ("B", _P), ("ldb", C.c_int64), ("b_format", C.c_int32), ("b_scale", _P), ("b_scale_ld", C.c_int64),
                ("b_tile", C.c_int32),
                ("C", _P), ("ldc", C.c_int64), ("c_f32", C.c_int32), ("accumulate", C.c_int32), ("bias", _P)]


FAX_ROTARY_HALVES, FAX_ROTARY_PAIRS = range(2)
FAX_ROTARY_MAX_DIM = 1024
FAX_RECURRENCE_PLAIN, FAX_RECURRENCE_COMPLEMENT = range(2)
FAX_RECURRENCE_BLOCK = 16
FAX_EXPERT_MAX = 1024


class RotaryDesc(C.Structure):
    _fields_ = [("rows", C.c_int32), ("heads", C.c_int32), ("head_dim", C.c_int32), ("rot_dim", C.c_int32),
                ("layout", C.c_int32), ("x", _P), ("ldx", C.c_int64), ("y", _P), ("ldy", C.c_int64),
                ("positions", _P), ("first", C.c_int32), ("seq", C.c_int32), ("frequencies", _P),
                ("amplitude", C.c_float), ("backward", C.c_int32)]


class DropoutDesc(C.Structure):
    _fields_ = [("rows", C.c_int32), ("cols", C.c_int32), ("x", _P), ("ldx", C.c_int64), ("resid", _P), ("ldr", C.c_int64),
                ("y", _P), ("ldy", C.c_int64), ("p", C.c_float), ("seed", C.c_uint64), ("offset", C.c_uint64),
                ("offset_device", _P)]


_RECURRENCE = [("rows", C.c_int32), ("d", C.c_int32), ("n_seq", C.c_int32), ("seq", C.c_int32), ("offsets", _P),
               ("input", C.c_int32), ("f", _P), ("ldf", C.c_int64), ("x", _P), ("ldx", C.c_int64), ("g", _P),
               ("ldg", C.c_int64), ("h0", _P)]


class RecurrenceDesc(C.Structure):
    _fields_ = _RECURRENCE + [("y", _P), ("ldy", C.c_int64), ("h_last", _P), ("states", _P)]


class RecurrenceBackwardDesc(C.Structure):
    _fields_ = _RECURRENCE + [("states", _P), ("dy", _P), ("lddy", C.c_int64), ("dh_last", _P), ("df", _P), ("lddf", C.c_int64),
                              ("dx", _P), ("lddx", C.c_int64), ("dg", _P), ("lddg", C.c_int64), ("dh0", _P)]


class ExpertSortDesc(C.Structure):
    _fields_ = [("n_tokens", C.c_int32), ("top_k", C.c_int32), ("n_experts", C.c_int32), ("capacity", C.c_int32),
                ("align", C.c_int32), ("slots", C.c_int32), ("ids", _P), ("slot_of", _P), ("source", _P), ("offsets", _P),
                ("counts", _P)]


_EXPERT_ROWS = [("n_tokens", C.c_int32), ("top_k", C.c_int32), ("d", C.c_int32), ("slots", C.c_int32), ("slot_of", _P)]


class ExpertDispatchDesc(C.Structure):
    _fields_ = _EXPERT_ROWS + [("source", _P), ("x", _P), ("ldx", C.c_int64), ("out", _P), ("ldo", C.c_int64)]


class ExpertCombineDesc(C.Structure):
    _fields_ = _EXPERT_ROWS + [("weights", _P), ("z", _P), ("ldz", C.c_int64), ("resid", _P), ("ldr", C.c_int64), ("y", _P),
                               ("ldy", C.c_int64)]


class ExpertCombineBackwardDesc(C.Structure):
    _fields_ = _EXPERT_ROWS + [("source", _P), ("weights", _P), ("z", _P), ("ldz", C.c_int64), ("dy", _P), ("lddy", C.c_int64),
                               ("dz", _P), ("lddz", C.c_int64), ("dw", _P)]


_SIGNATURES = {
    "fax_op_gemm": (C.c_int32, [_P, C.c_int32, C.POINTER(GemmDesc)]),
    "fax_op_layernorm_forward": (C.c_int32, [_P, C.c_int32, C.c_int32, C.c_int32, _P, _P, _P, C.c_float,
                                             _P, _P, _P]),
    "fax_op_layernorm_backward_scratch_bytes": (C.c_int32, [C.c_int32, C.c_int32, C.POINTER(C.c_size_t)]),
    "fax_op_layernorm_backward": (C.c_int32, [_P, C.c_int32, C.c_int32, C.c_int32, _P, _P, _P, _P, _P, _P,
                                              _P, _P, _P, _P, C.c_size_t]),
    "fax_op_layernorm_backward_static": (C.c_int32, [_P, C.c_int32, C.c_int32, C.c_int32, _P, _P, _P, _P, _P, _P,
                                                     _P, _P, _P]),
    "fax_op_attention_forward": (C.c_int32, [_P, C.c_int32, C.c_int32, C.c_int32, C.c_int32, C.c_int32,
                                             _P, _P, _P]),
    "fax_op_attention_backward_scratch_bytes": (C.c_int32, [C.c_int32] * 5 + [C.POINTER(C.c_size_t)]),
    "fax_op_attention_backward": (C.c_int32, [_P, C.c_int32, C.c_int32, C.c_int32, C.c_int32, C.c_int32,
                                              _P, _P, _P, _P, _P, _P, C.c_size_t]),
    "fax_op_embedding_forward": (C.c_int32, [_P, C.c_int32, C.c_int32, C.c_int32, C.c_int32, _P, _P, C.c_float, _P]),
    "fax_op_embedding_backward_scratch_bytes": (C.c_int32, [C.c_int32] * 3 + [C.POINTER(C.c_size_t)]),
    "fax_op_embedding_backward": (C.c_int32, [_P, C.c_int32, C.c_int32, C.c_int32, C.c_int32, _P, _P, C.c_float,
                                              C.c_int32, _P, _P, C.c_size_t]),
    "fax_op_fp8_quantize": (C.c_int32, [_P, C.c_int32, C.POINTER(Fp8QuantizeDesc)]),
    "fax_op_fp8_gemm": (C.c_int32, [_P, C.POINTER(Fp8GemmDesc)]),
    "fax_op_rotary": (C.c_int32, [_P, C.c_int32, C.POINTER(RotaryDesc)]),
    "fax_rotary_frequencies": (C.c_int32, [C.c_int32, C.c_double, C.c_double, C.c_int32, C.c_double, C.c_double, _P]),
    "fax_op_dropout": (C.c_int32, [_P, C.c_int32, C.POINTER(DropoutDesc)]),
    "fax_op_recurrence_states_floats": (C.c_int32, [C.c_int32] * 3 + [C.POINTER(C.c_size_t)]),
    "fax_op_recurrence_forward": (C.c_int32, [_P, C.c_int32, C.POINTER(RecurrenceDesc)]),
    "fax_op_recurrence_backward": (C.c_int32, [_P, C.c_int32, C.POINTER(RecurrenceBackwardDesc)]),
    "fax_op_expert_slots": (C.c_int32, [C.c_int32] * 5 + [C.POINTER(C.c_int32)]),
    "fax_op_expert_sort": (C.c_int32, [_P, C.POINTER(ExpertSortDesc)]),
    "fax_op_expert_dispatch": (C.c_int32, [_P, C.c_int32, C.POINTER(ExpertDispatchDesc)]),
    "fax_op_expert_combine": (C.c_int32, [_P, C.c_int32, C.POINTER(ExpertCombineDesc)]),
    "fax_op_expert_combine_backward": (C.c_int32, [_P, C.c_int32, C.POINTER(ExpertCombineBackwardDesc)]),
    "fax_op_fp8_gemm_tile": (C.c_int32, [_P, C.c_int32, C.c_int32, C.c_int32, C.c_int32] + [C.POINTER(C.c_int32)] * 3),
}

_lib = None


def register(lib):
    global _lib
    for name, (res, args) in _SIGNATURES.items():
        fn = getattr(lib, name)
        fn.restype = res
        fn.argtypes = args
    _lib = lib


def _L():
    if _lib is None:
        from . import binding
        binding.load_library()
    return _lib


def _check(s, where):
    if s != 0:
        from .binding import FaxError
        raise FaxError(s, where)


def fax_op_gemm(ctx, prec, desc: GemmDesc):
    _check(_L().fax_op_gemm(ctx, prec, C.byref(desc)), "fax_op_gemm")


def fax_op_layernorm_forward(ctx, prec, rows, d, x, gamma, beta, eps, out, mu, rstd):
    _check(_L().fax_op_layernorm_forward(ctx, prec, rows, d, x, gamma, beta, eps, out, mu, rstd),
           "fax_op_layernorm_forward")


def fax_op_layernorm_backward_scratch_bytes(rows, d) -> int:
    b = C.c_size_t()
    _check(_L().fax_op_layernorm_backward_scratch_bytes(rows, d, C.byref(b)), "fax_op_layernorm_backward_scratch_bytes")
    return b.value


def fax_op_layernorm_backward(ctx, prec, rows, d, da, x, mu, rstd, gamma, add, dx, dgamma, dbeta, scratch,
                              scratch_bytes):
    _check(_L().fax_op_layernorm_backward(ctx, prec, rows, d, da, x, mu, rstd, gamma, add, dx, dgamma, dbeta,
                                          scratch, scratch_bytes), "fax_op_layernorm_backward")


def fax_op_layernorm_backward_static(ctx, prec, rows, d, da, x, mu, rstd, gamma, add, dx, dgamma, dbeta):
    """LayerNorm backward whose scratch is a fixed array inside the library: for callers that
    cannot allocate device memory or pass any.  Same results as fax_op_layernorm_backward."""
    _check(_L().fax_op_layernorm_backward_static(ctx, prec, rows, d, da, x, mu, rstd, gamma, add, dx, dgamma,
                                                 dbeta), "fax_op_layernorm_backward_static")


def fax_op_attention_forward(ctx, prec, batch, seq, n_heads, head_dim, qkv, o, lse):
    _check(_L().fax_op_attention_forward(ctx, prec, batch, seq, n_heads, head_dim, qkv, o, lse),
           "fax_op_attention_forward")


def fax_op_attention_backward_scratch_bytes(prec, batch, seq, n_heads, head_dim) -> int:
    b = C.c_size_t()
    _check(_L().fax_op_attention_backward_scratch_bytes(prec, batch, seq, n_heads, head_dim, C.byref(b)),
           "fax_op_attention_backward_scratch_bytes")
    return b.value


def fax_op_attention_backward(ctx, prec, batch, seq, n_heads, head_dim, qkv, o, lse, d_o, dqkv, scratch,
                              scratch_bytes):
    _check(_L().fax_op_attention_backward(ctx, prec, batch, seq, n_heads, head_dim, qkv, o, lse, d_o, dqkv,
                                          scratch, scratch_bytes), "fax_op_attention_backward")


def fax_op_embedding_forward(ctx, prec, n_tokens, vocab, d, ids, table, scale, out):
    _check(_L().fax_op_embedding_forward(ctx, prec, n_tokens, vocab, d, ids, table, scale, out),
           "fax_op_embedding_forward")


def fax_op_embedding_backward_scratch_bytes(n_tokens, vocab, d) -> int:
    b = C.c_size_t()
    _check(_L().fax_op_embedding_backward_scratch_bytes(n_tokens, vocab, d, C.byref(b)),
           "fax_op_embedding_backward_scratch_bytes")
    return b.value


def fax_op_embedding_backward(ctx, prec, n_tokens, vocab, d, ids, dout, scale, accumulate, dtable, scratch,
                              scratch_bytes):
    _check(_L().fax_op_embedding_backward(ctx, prec, n_tokens, vocab, d, ids, dout, scale, int(bool(accumulate)),
                                          dtable, scratch, scratch_bytes), "fax_op_embedding_backward")


def fax_op_fp8_quantize(ctx, prec, desc: Fp8QuantizeDesc):
    _check(_L().fax_op_fp8_quantize(ctx, prec, C.byref(desc)), "fax_op_fp8_quantize")


def fax_op_fp8_gemm(ctx, desc: Fp8GemmDesc):
    _check(_L().fax_op_fp8_gemm(ctx, C.byref(desc)), "fax_op_fp8_gemm")


def fax_op_fp8_gemm_tile(ctx, M, N, K, c_f32) -> tuple[int, int, int]:
    """(SMs that share a tile, its columns, slices of K) of such a product under the context's settings."""
    out = [C.c_int32() for _ in range(3)]
    _check(_L().fax_op_fp8_gemm_tile(ctx, M, N, K, int(bool(c_f32)), *(C.byref(o) for o in out)), "fax_op_fp8_gemm_tile")
    return tuple(o.value for o in out)


def fax_op_rotary(ctx, prec, desc: RotaryDesc):
    _check(_L().fax_op_rotary(ctx, prec, C.byref(desc)), "fax_op_rotary")


def fax_rotary_frequencies(rot_dim, base=10000.0, factor=1.0, original_seq=0, low_turns=1.0, high_turns=32.0) -> list[int]:
    """Turns a position of each pair, in units of 2^-64."""
    out = (C.c_uint64 * max(rot_dim // 2, 1))()
    _check(_L().fax_rotary_frequencies(rot_dim, base, factor, original_seq, low_turns, high_turns, out), "fax_rotary_frequencies")
    return list(out)


def fax_op_dropout(ctx, prec, desc: DropoutDesc):
    _check(_L().fax_op_dropout(ctx, prec, C.byref(desc)), "fax_op_dropout")


def fax_op_recurrence_states_floats(rows, n_seq, d) -> int:
    n = C.c_size_t()
    _check(_L().fax_op_recurrence_states_floats(rows, n_seq, d, C.byref(n)), "fax_op_recurrence_states_floats")
    return n.value


def fax_op_recurrence_forward(ctx, prec, desc: RecurrenceDesc):
    _check(_L().fax_op_recurrence_forward(ctx, prec, C.byref(desc)), "fax_op_recurrence_forward")


def fax_op_recurrence_backward(ctx, prec, desc: RecurrenceBackwardDesc):
    _check(_L().fax_op_recurrence_backward(ctx, prec, C.byref(desc)), "fax_op_recurrence_backward")


def fax_op_expert_slots(n_tokens, top_k, n_experts, capacity=0, align=1) -> int:
    n = C.c_int32()
    _check(_L().fax_op_expert_slots(n_tokens, top_k, n_experts, capacity, align, C.byref(n)), "fax_op_expert_slots")
    return n.value


def fax_op_expert_sort(ctx, desc: ExpertSortDesc):
    _check(_L().fax_op_expert_sort(ctx, C.byref(desc)), "fax_op_expert_sort")


def fax_op_expert_dispatch(ctx, prec, desc: ExpertDispatchDesc):
    _check(_L().fax_op_expert_dispatch(ctx, prec, C.byref(desc)), "fax_op_expert_dispatch")


def fax_op_expert_combine(ctx, prec, desc: ExpertCombineDesc):
    _check(_L().fax_op_expert_combine(ctx, prec, C.byref(desc)), "fax_op_expert_combine")


def fax_op_expert_combine_backward(ctx, prec, desc: ExpertCombineBackwardDesc):
    _check(_L().fax_op_expert_combine_backward(ctx, prec, C.byref(desc)), "fax_op_expert_combine_backward")
