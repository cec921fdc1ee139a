"""ctypes binding of the CO3 CUDA library (include/co3.h): argument marshalling only.

Every step of the pipeline runs in the library's CUDA kernels.  There is no CPU fallback: if the
library has not been built (python -m paper_2203_09044_b200.build, or __graft_entry__.build())
loading raises.  torch is used for device memory and streams only.
"""
import ctypes as C
import functools
import os

import numpy as np

_HERE = os.path.dirname(os.path.abspath(__file__))
LIB_PATH = os.path.join(_HERE, "csrc", "libco3.so")

OK, EINVAL, ENOMEM, ECUDA, ECAPACITY, ECORRUPT, ENONFINITE = 0, -1, -2, -3, -4, -5, -6
FLAG_CAPACITY, FLAG_CORRUPT, FLAG_NONFINITE = 1, 2, 4
BIAS_CURRENT, BIAS_LAGGED, CODE_LAGGED, CODE_EMPIRICAL = 0, 1, 2, 3
RULE_POLY, RULE_OPT = 0, 1
FLAG_TIMEOUT = 8
FLAG_INEXACT = 16
FLAG_TOKEN = 32

EXPORTS = [
    "co3_plan_create", "co3_plan_destroy", "co3_sizes", "co3_encode", "co3_decode_aggregate",
    "co3_iteration_host", "co3_status", "co3_get_fit", "co3_state_export", "co3_state_import",
    "co3_debug_symbols", "co3_debug_hist", "co3_debug_code", "co3_model_weights", "co3_partition",
    "co3_strerror", "co3_profile_enable", "co3_profile_collect", "co3_launch_count",
    "co3_moments_static", "co3_state_header", "co3_decode_aggregate_update",
    "co3_bias_opt_table", "co3_grid_distortion", "co3_encode_empirical", "co3_decode_aggregate_empirical",
    "co3_profile_stride", "co3_tiled_begin", "co3_tiled_statistics", "co3_tiled_convert", "co3_tiled_finish",
    "co3_moments_export", "co3_moments_import", "co3_set_fit_override", "co3_debug_encode_stalled",
    "co3_model_checksum", "co3_balanced_split",
    "co3_adamw_create", "co3_adamw_destroy", "co3_adamw_sizes", "co3_grad_norm", "co3_adamw_step", "co3_adamw_values",
    "co3_adamw_status", "co3_adamw_steps_export", "co3_adamw_steps_import", "co3_adamw_launch_count",
    "co3_embed_create", "co3_embed_destroy", "co3_embed_forward", "co3_embed_backward", "co3_embed_status", "co3_embed_launch_count",
    "co3_layernorm_create", "co3_layernorm_destroy", "co3_layernorm_forward", "co3_layernorm_backward", "co3_layernorm_launch_count",
    "co3_token_loss_create", "co3_token_loss_destroy", "co3_token_loss_forward", "co3_token_loss_backward", "co3_token_loss_status",
    "co3_token_loss_launch_count",
]
ELIMIT = -7
STATIC_MAX_ELEMENTS = 1 << 29

KERNEL_NAMES = ["stats", "fit", "convert", "code_enc", "reconvert", "enc_scan", "enc_pack", "code_dec",
                "decode"]


class Format(C.Structure):
    _fields_ = [("exp_bits", C.c_int32), ("mant_bits", C.c_int32)]


class Config(C.Structure):
    _fields_ = [("d", C.c_int64), ("ld", C.c_int64), ("n_users", C.c_int32), ("fmt", Format),
                ("n_segments", C.c_int32), ("seg_offsets", C.POINTER(C.c_int64)),
                ("gamma", C.c_float), ("bias_mode", C.c_int32), ("cap_words", C.c_int64),
                ("bias_rule", C.c_int32), ("reserved", C.c_int32)]


F32, BF16, F16, NONE = 0, 1, 2, -1
I32, I64 = 3, 4
STATE_BLOCK = 256          # elements of a tensor that share an exponent in 8-bit moments


class AdamwConfig(C.Structure):
    _fields_ = [("n_tensors", C.c_int32), ("sizes", C.POINTER(C.c_int64)), ("decay", C.POINTER(C.c_float)),
                ("weight_type", C.c_int32), ("grad_type", C.c_int32), ("copy_type", C.c_int32), ("state_bits", C.c_int32),
                ("beta1", C.c_double), ("beta2", C.c_double), ("eps", C.c_double), ("weight_decay", C.c_double),
                ("seed", C.c_uint32), ("reserved", C.c_int32)]


class AdamwState(C.Structure):
    _fields_ = [("m", C.c_void_p), ("v", C.c_void_p), ("m_exp", C.c_void_p), ("v_exp", C.c_void_p)]


class Array(C.Structure):
    _fields_ = [("data", C.c_void_p), ("type", C.c_int32), ("reserved", C.c_int32), ("user_stride", C.c_int64), ("token_stride", C.c_int64)]


class Tokens(C.Structure):
    _fields_ = [("data", C.c_void_p), ("type", C.c_int32), ("top", C.c_int32), ("user_stride", C.c_int64), ("token_stride", C.c_int64)]


class ParamGrad(C.Structure):
    _fields_ = [("data", C.c_void_p), ("type", C.c_int32), ("accumulate", C.c_int32), ("user_stride", C.c_int64)]


class TokenLossConfig(C.Structure):
    _fields_ = [("vocab", C.c_int64), ("dim", C.c_int64), ("max_tokens", C.c_int64), ("n_users", C.c_int32), ("type", C.c_int32),
                ("grad_type", C.c_int32), ("max_top", C.c_int32)]


HDR_DTYPE = np.dtype([("bias", np.int8), ("ibeta", np.int8), ("ir", np.int16)])

_lib = None


class Co3Error(RuntimeError):
    def __init__(self, code, where):
        self.code = code
        super().__init__(f"{where}: {lib().co3_strerror(code).decode()} ({code})")


def lib():
    """Load csrc/libco3.so; raises if it is missing (there is no other implementation)."""
    global _lib
    if _lib is not None:
        return _lib
    if not os.path.exists(LIB_PATH):
        raise ImportError(f"{LIB_PATH} not built: run `python -m paper_2203_09044_b200.build`")
    L = C.CDLL(LIB_PATH)
    vp, i64p = C.c_void_p, C.POINTER(C.c_int64)
    L.co3_plan_create.restype = C.c_int
    L.co3_plan_create.argtypes = [C.POINTER(vp), C.POINTER(Config)]
    L.co3_plan_destroy.restype = None
    L.co3_plan_destroy.argtypes = [vp]
    L.co3_sizes.restype = C.c_int
    L.co3_sizes.argtypes = [vp, i64p, i64p, i64p]
    L.co3_encode.restype = C.c_int
    L.co3_encode.argtypes = [vp] * 9
    L.co3_decode_aggregate.restype = C.c_int
    L.co3_decode_aggregate.argtypes = [vp] * 7
    L.co3_encode_empirical.restype = C.c_int
    L.co3_encode_empirical.argtypes = [vp] * 10
    L.co3_decode_aggregate_empirical.restype = C.c_int
    L.co3_decode_aggregate_empirical.argtypes = [vp] * 8
    L.co3_decode_aggregate_update.restype = C.c_int
    L.co3_decode_aggregate_update.argtypes = [vp] * 7 + [C.c_float, vp]
    L.co3_iteration_host.restype = C.c_int
    L.co3_iteration_host.argtypes = [vp] * 12
    L.co3_status.restype = C.c_int
    L.co3_status.argtypes = [vp, C.POINTER(C.c_uint32), C.POINTER(C.c_uint64), C.c_int32]
    L.co3_get_fit.restype = C.c_int
    L.co3_get_fit.argtypes = [vp, C.c_int32] + [C.POINTER(C.c_double)] * 5
    L.co3_state_export.restype = C.c_int
    L.co3_state_export.argtypes = [vp, i64p, vp]
    L.co3_state_import.restype = C.c_int
    L.co3_state_import.argtypes = [vp, C.c_int64, vp]
    L.co3_debug_symbols.restype = C.c_int
    L.co3_debug_symbols.argtypes = [vp, vp, vp]
    L.co3_debug_hist.restype = C.c_int
    L.co3_debug_hist.argtypes = [vp, vp]
    L.co3_debug_code.restype = C.c_int
    L.co3_debug_code.argtypes = [vp, vp, vp, vp]
    L.co3_model_weights.restype = C.c_int
    L.co3_model_weights.argtypes = [Format, C.c_int32, C.c_int32, vp]
    L.co3_partition.restype = C.c_int64
    L.co3_partition.argtypes = [C.c_int64, C.c_int32, vp, vp, vp, vp, vp, i64p]
    L.co3_profile_enable.restype = C.c_int
    L.co3_profile_enable.argtypes = [vp, C.c_uint32, C.c_int32]
    L.co3_tiled_begin.restype = C.c_int
    L.co3_tiled_begin.argtypes = [vp, C.POINTER(C.c_int32)]
    L.co3_tiled_statistics.restype = C.c_int
    L.co3_tiled_statistics.argtypes = [vp, vp, vp, C.c_int32, C.c_int32, vp]
    L.co3_tiled_convert.restype = C.c_int
    L.co3_tiled_convert.argtypes = [vp, vp, vp, C.c_int32, C.c_int32, vp]
    L.co3_tiled_finish.restype = C.c_int
    L.co3_tiled_finish.argtypes = [vp] * 7
    L.co3_moments_export.restype = C.c_int
    L.co3_moments_export.argtypes = [vp, vp, vp]
    L.co3_moments_import.restype = C.c_int
    L.co3_moments_import.argtypes = [vp, vp, vp]
    L.co3_profile_stride.restype = C.c_int
    L.co3_profile_stride.argtypes = [vp, C.c_int32]
    L.co3_profile_collect.restype = C.c_int
    L.co3_profile_collect.argtypes = [vp, vp, vp]
    L.co3_launch_count.restype = C.c_int64
    L.co3_launch_count.argtypes = [vp]
    L.co3_moments_static.restype = C.c_int
    L.co3_moments_static.argtypes = [vp, vp, C.c_int64, C.c_float, vp, vp]
    L.co3_state_header.restype = C.c_int
    L.co3_state_header.argtypes = [vp, C.c_int32, vp]
    L.co3_bias_opt_table.restype = C.c_int
    L.co3_bias_opt_table.argtypes = [Format, vp]
    L.co3_grid_distortion.restype = C.c_double
    L.co3_grid_distortion.argtypes = [Format, C.c_int32, C.c_int32]
    L.co3_set_fit_override.restype = C.c_int
    L.co3_set_fit_override.argtypes = [vp, vp]
    L.co3_debug_encode_stalled.restype = C.c_int
    L.co3_debug_encode_stalled.argtypes = [vp] * 6 + [C.c_int32, vp]
    L.co3_model_checksum.restype = C.c_uint64
    L.co3_model_checksum.argtypes = [Format]
    L.co3_balanced_split.restype = C.c_int
    L.co3_balanced_split.argtypes = [vp, vp, C.c_int64, C.c_int32, C.c_int32, vp]
    L.co3_adamw_create.restype = C.c_int
    L.co3_adamw_create.argtypes = [C.POINTER(vp), C.POINTER(AdamwConfig)]
    L.co3_adamw_destroy.restype = None
    L.co3_adamw_destroy.argtypes = [vp]
    L.co3_adamw_sizes.restype = C.c_int
    L.co3_adamw_sizes.argtypes = [vp, i64p, i64p]
    L.co3_grad_norm.restype = C.c_int
    L.co3_grad_norm.argtypes = [vp, vp, C.c_float, C.c_float, vp, vp, vp]
    L.co3_adamw_step.restype = C.c_int
    L.co3_adamw_step.argtypes = [vp, vp, vp, vp, vp, C.c_double, vp, vp, vp]
    L.co3_adamw_values.restype = C.c_int
    L.co3_adamw_values.argtypes = [vp, vp, vp, vp, C.c_int32, vp]
    L.co3_adamw_status.restype = C.c_int
    L.co3_adamw_status.argtypes = [vp, C.POINTER(C.c_uint32), C.POINTER(C.c_uint64), C.POINTER(C.c_uint64), C.c_int32]
    L.co3_adamw_steps_export.restype = C.c_int
    L.co3_adamw_steps_export.argtypes = [vp, i64p]
    L.co3_adamw_steps_import.restype = C.c_int
    L.co3_adamw_steps_import.argtypes = [vp, C.c_int64]
    L.co3_adamw_launch_count.restype = C.c_int64
    L.co3_adamw_launch_count.argtypes = [vp]
    arr, tok, pgrad, i64, i32, f32 = C.POINTER(Array), C.POINTER(Tokens), C.POINTER(ParamGrad), C.c_int64, C.c_int32, C.c_float
    L.co3_embed_create.argtypes = [C.POINTER(vp), i64, i64, i32, i64]
    L.co3_embed_forward.argtypes = [vp, tok, i64, vp, i32, f32, arr, vp]
    L.co3_embed_backward.argtypes = [vp, arr, tok, i64, f32, pgrad, vp]
    L.co3_layernorm_create.argtypes = [C.POINTER(vp), i64, i32, C.c_double]
    L.co3_layernorm_forward.argtypes = [vp, arr, vp, vp, i32, i64, arr, vp, vp, vp]
    L.co3_layernorm_backward.argtypes = [vp, arr, arr, vp, i32, vp, vp, i64, arr, pgrad, pgrad, vp]
    L.co3_token_loss_create.argtypes = [C.POINTER(vp), C.POINTER(TokenLossConfig)]
    L.co3_token_loss_forward.argtypes = [vp, arr, vp, i64, tok, arr, f32, i64, vp, vp, vp]
    L.co3_token_loss_backward.argtypes = [vp, arr, vp, i64, tok, arr, f32, i64, vp, vp, f32, arr, pgrad, vp]
    for name in ("embed", "token_loss"):
        getattr(L, f"co3_{name}_status").argtypes = [vp, C.POINTER(C.c_uint32), C.POINTER(C.c_uint64), i32]
    for name in ("embed", "layernorm", "token_loss"):
        getattr(L, f"co3_{name}_destroy").restype = None
        getattr(L, f"co3_{name}_destroy").argtypes = [vp]
        getattr(L, f"co3_{name}_launch_count").restype = i64
        getattr(L, f"co3_{name}_launch_count").argtypes = [vp]
    L.co3_strerror.restype = C.c_char_p
    L.co3_strerror.argtypes = [C.c_int]
    _lib = L
    return L


def model_weights(exp_bits, mant_bits, ibeta, ir):
    """Host only: integer model weights per symbol byte for header indices (ibeta, ir)."""
    w = np.zeros(1 << (1 + exp_bits + mant_bits), np.uint32)
    rc = lib().co3_model_weights(Format(exp_bits, mant_bits), ibeta, ir, w.ctypes.data)
    if rc != OK:
        raise Co3Error(rc, "co3_model_weights")
    return w


def model_checksum(exp_bits, mant_bits):
    """Host only: digest of the whole model-weight table of a format (0: unsupported format)."""
    return int(lib().co3_model_checksum(Format(exp_bits, mant_bits)))


def balanced_split(cost, seg, teams, max_blocks):
    """Host only: cuts (max_blocks + 1 int32) and the number of blocks in use (co3_balanced_split)."""
    c = np.ascontiguousarray(cost, np.float64)
    g = np.ascontiguousarray(seg, np.int32)
    part = np.zeros(max_blocks + 1, np.int32)
    nb = lib().co3_balanced_split(c.ctypes.data, g.ctypes.data, len(c), int(teams), int(max_blocks), part.ctypes.data)
    if nb < 0:
        raise Co3Error(EINVAL, "co3_balanced_split")
    return part, nb


def bias_opt_table(exp_bits, mant_bits):
    """[23][8] int16 table behind RULE_OPT (host only)."""
    tab = np.zeros((23, 8), np.int16)
    rc = lib().co3_bias_opt_table(Format(exp_bits, mant_bits), tab.ctypes.data)
    if rc != OK:
        raise Co3Error(rc, "co3_bias_opt_table")
    return tab


def grid_distortion(exp_bits, mant_bits, ibeta, ir):
    return float(lib().co3_grid_distortion(Format(exp_bits, mant_bits), int(ibeta), int(ir)))


def partition(d, seg_offsets):
    """Host only: (chunk_seg, chunk_start, chunk_end, sub_base, n_sub) of the static partition."""
    off = np.ascontiguousarray(seg_offsets, np.int64)
    ns = C.c_int64()
    nc = lib().co3_partition(d, len(off) - 1, off.ctypes.data, None, None, None, None, C.byref(ns))
    if nc < 0:
        raise Co3Error(int(nc), "co3_partition")
    seg = np.zeros(nc, np.int32)
    st, en, sb = (np.zeros(nc, np.int64) for _ in range(3))
    lib().co3_partition(d, len(off) - 1, off.ctypes.data, seg.ctypes.data, st.ctypes.data,
                        en.ctypes.data, sb.ctypes.data, C.byref(ns))
    return seg, st, en, sb, int(ns.value)


def _ptr(t):
    return C.c_void_p(t.data_ptr()) if t is not None else None


def moments_static(grad, residual, n, gamma, moments, stream=None):
    """co3_moments_static: N, sum|a|, sum a^2, non-finite count of a = g + gamma m over n elements
    into `moments` (4 float64 on the device), with no allocation inside the library.  Returns the
    C return code (0, or a negative CO3_E* value such as ELIMIT)."""
    import torch
    s = torch.cuda.current_stream() if stream is None else stream
    return int(lib().co3_moments_static(_ptr(grad), _ptr(residual), int(n), float(gamma), _ptr(moments),
                                        C.c_void_p(s.cuda_stream)))


class Plan:
    """co3_plan plus the torch buffers of one pipeline instance on the current CUDA device."""

    def __init__(self, d, n_users, exp_bits, mant_bits, seg_offsets=None, gamma=0.9,
                 bias_mode=BIAS_LAGGED, cap_words=None, ld=None, bias_rule=RULE_POLY):
        import torch
        self.torch = torch
        L = lib()
        self.d, self.U, self.E, self.M = int(d), int(n_users), int(exp_bits), int(mant_bits)
        self.ld = int(ld) if ld is not None else (self.d + 3) // 4 * 4
        self.nsym = 1 << (1 + self.E + self.M)
        self.bias_mode = int(bias_mode)
        off = np.ascontiguousarray([0, d] if seg_offsets is None else seg_offsets, np.int64)
        self.S = len(off) - 1
        self._off = off
        # worst case needs the partition; compute it on the host first
        _, st, en, _, _ = partition(self.d, off)
        worst = int(sum(4 * ((16 * int(e - s) + 127) // 128) for s, e in zip(st, en)))
        self.cap_words = int(cap_words) if cap_words is not None else worst
        cfg = Config(self.d, self.ld, self.U, Format(self.E, self.M), self.S,
                     off.ctypes.data_as(C.POINTER(C.c_int64)), float(gamma), int(bias_mode),
                     self.cap_words, int(bias_rule), 0)
        h = C.c_void_p()
        rc = L.co3_plan_create(C.byref(h), C.byref(cfg))
        if rc != OK:
            raise Co3Error(rc, "co3_plan_create")
        self.handle = h
        nc, ns, wc = C.c_int64(), C.c_int64(), C.c_int64()
        L.co3_sizes(h, C.byref(nc), C.byref(ns), C.byref(wc))
        self.n_chunks, self.n_sub, self.worst_case_words = nc.value, ns.value, wc.value

    def close(self):
        if getattr(self, "handle", None):
            lib().co3_plan_destroy(self.handle)
            self.handle = None

    def __del__(self):
        try:
            self.close()
        except Exception:
            pass

    # ---- buffers ---------------------------------------------------------------------------
    def alloc_outputs(self, device="cuda"):
        t = self.torch
        return dict(
            bitstream=t.zeros((self.U, self.cap_words), dtype=t.int32, device=device),
            sub_bits=t.zeros((self.U, max(self.n_sub, 1)), dtype=t.int16, device=device),
            chunk_off=t.zeros((self.U, self.n_chunks + 1), dtype=t.int32, device=device),
            user_bits=t.zeros((self.U,), dtype=t.int64, device=device),
            hdr=t.zeros((self.S,), dtype=t.int32, device=device),
            avg=t.zeros((self.d,), dtype=t.float32, device=device),
            code_lens=t.zeros((self.S, self.nsym), dtype=t.uint8, device=device),   # CODE_EMPIRICAL only
        )

    def _stream(self, stream):
        s = self.torch.cuda.current_stream() if stream is None else stream
        return C.c_void_p(s.cuda_stream)

    # ---- the C-ABI calls -------------------------------------------------------------------
    def encode(self, grad, residual, out, stream=None):
        if self.bias_mode == CODE_EMPIRICAL:
            rc = lib().co3_encode_empirical(self.handle, _ptr(grad), _ptr(residual), _ptr(out["bitstream"]),
                                            _ptr(out["sub_bits"]), _ptr(out["chunk_off"]), _ptr(out["user_bits"]),
                                            _ptr(out["hdr"]), _ptr(out["code_lens"]), self._stream(stream))
        else:
            rc = lib().co3_encode(self.handle, _ptr(grad), _ptr(residual), _ptr(out["bitstream"]),
                                  _ptr(out["sub_bits"]), _ptr(out["chunk_off"]), _ptr(out["user_bits"]),
                                  _ptr(out["hdr"]), self._stream(stream))
        if rc != OK:
            raise Co3Error(rc, "co3_encode")

    def encode_tiled(self, tile_users, make_tile, residual, out, stream=None, around_call=None):
        """One iteration with the gradient supplied tile by tile: make_tile(user0, n) returns the
        [n][ld] fp32 cuda gradient of users user0 .. user0 + n - 1 (it may reuse one buffer: each tile
        is consumed by kernels enqueued on the stream before the next make_tile call returns work on
        that same stream).  Bit for bit the result of encode() on the whole gradient.
        around_call(False) / around_call(True), if given, run right before / after every library call
        (a timing hook: whatever make_tile does stays outside)."""
        need = C.c_int32()
        rc = lib().co3_tiled_begin(self.handle, C.byref(need))
        if rc != OK:
            raise Co3Error(rc, "co3_tiled_begin")
        passes = (["co3_tiled_statistics"] if need.value else []) + ["co3_tiled_convert"]
        for name in passes:
            for u0 in range(0, self.U, tile_users):
                n = min(tile_users, self.U - u0)
                g = make_tile(u0, n)
                if around_call:
                    around_call(False)
                rc = getattr(lib(), name)(self.handle, _ptr(g), _ptr(residual), u0, n, self._stream(stream))
                if around_call:
                    around_call(True)
                if rc != OK:
                    raise Co3Error(rc, name)
        if around_call:
            around_call(False)
        rc = lib().co3_tiled_finish(self.handle, _ptr(out["bitstream"]), _ptr(out["sub_bits"]), _ptr(out["chunk_off"]),
                                    _ptr(out["user_bits"]), _ptr(out["hdr"]), self._stream(stream))
        if around_call:
            around_call(True)
        if rc != OK:
            raise Co3Error(rc, "co3_tiled_finish")

    # The phases of a tiled iteration one by one (encode_tiled strings them together); between them a
    # caller may pool the moments of several plans (moments_export / moments_import).
    def tiled_begin(self):
        """Start a tiled iteration; True if statistics tiles have to come before the convert tiles."""
        need = C.c_int32()
        rc = lib().co3_tiled_begin(self.handle, C.byref(need))
        if rc != OK:
            raise Co3Error(rc, "co3_tiled_begin")
        return bool(need.value)

    def tiled_statistics(self, grad_tile, residual, user0, n_users, stream=None):
        rc = lib().co3_tiled_statistics(self.handle, _ptr(grad_tile), _ptr(residual), user0, n_users, self._stream(stream))
        if rc != OK:
            raise Co3Error(rc, "co3_tiled_statistics")

    def tiled_convert(self, grad_tile, residual, user0, n_users, stream=None):
        rc = lib().co3_tiled_convert(self.handle, _ptr(grad_tile), _ptr(residual), user0, n_users, self._stream(stream))
        if rc != OK:
            raise Co3Error(rc, "co3_tiled_convert")

    def tiled_finish(self, out, stream=None):
        rc = lib().co3_tiled_finish(self.handle, _ptr(out["bitstream"]), _ptr(out["sub_bits"]), _ptr(out["chunk_off"]),
                                    _ptr(out["user_bits"]), _ptr(out["hdr"]), self._stream(stream))
        if rc != OK:
            raise Co3Error(rc, "co3_tiled_finish")

    def moments_export(self, moments=None, stream=None):
        """[S][3] fp64 cuda: (finite entries, sum |a|, sum a^2) of every segment, all users pooled."""
        import torch
        if moments is None:
            moments = torch.empty((self.S, 3), dtype=torch.float64, device="cuda")
        rc = lib().co3_moments_export(self.handle, _ptr(moments), self._stream(stream))
        if rc != OK:
            raise Co3Error(rc, "co3_moments_export")
        return moments

    def moments_import(self, moments, stream=None):
        """The sums the next fit uses instead of the plan's own ([S][3] fp64 cuda, contiguous)."""
        assert moments.is_cuda and moments.is_contiguous() and tuple(moments.shape) == (self.S, 3)
        rc = lib().co3_moments_import(self.handle, _ptr(moments), self._stream(stream))
        if rc != OK:
            raise Co3Error(rc, "co3_moments_import")

    def decode_aggregate(self, out, avg=None, stream=None):
        avg = out["avg"] if avg is None else avg
        if self.bias_mode == CODE_EMPIRICAL:
            rc = lib().co3_decode_aggregate_empirical(self.handle, _ptr(out["bitstream"]), _ptr(out["sub_bits"]),
                                                      _ptr(out["chunk_off"]), _ptr(out["hdr"]),
                                                      _ptr(out["code_lens"]), _ptr(avg), self._stream(stream))
        else:
            rc = lib().co3_decode_aggregate(self.handle, _ptr(out["bitstream"]), _ptr(out["sub_bits"]),
                                            _ptr(out["chunk_off"]), _ptr(out["hdr"]), _ptr(avg),
                                            self._stream(stream))
        if rc != OK:
            raise Co3Error(rc, "co3_decode_aggregate")
        return avg

    def decode_aggregate_update(self, out, weights, step, avg=None, stream=None):
        """decode_aggregate with w <- w + step * avg fused in (weights: [d] fp32 cuda tensor, in place)."""
        avg = out["avg"] if avg is None else avg
        rc = lib().co3_decode_aggregate_update(self.handle, _ptr(out["bitstream"]), _ptr(out["sub_bits"]),
                                               _ptr(out["chunk_off"]), _ptr(out["hdr"]), _ptr(avg),
                                               _ptr(weights), C.c_float(float(step)), self._stream(stream))
        if rc != OK:
            raise Co3Error(rc, "co3_decode_aggregate_update")
        return avg

    def iteration_host(self, h_grad, d_grad, residual, out, h_avg, stream=None):
        rc = lib().co3_iteration_host(self.handle, _ptr(h_grad), _ptr(d_grad), _ptr(residual),
                                      _ptr(out["bitstream"]), _ptr(out["sub_bits"]),
                                      _ptr(out["chunk_off"]), _ptr(out["user_bits"]), _ptr(out["hdr"]),
                                      _ptr(out["avg"]), _ptr(h_avg), self._stream(stream))
        if rc != OK:
            raise Co3Error(rc, "co3_iteration_host")

    def status(self, clear=False):
        f, n = C.c_uint32(), C.c_uint64()
        rc = lib().co3_status(self.handle, C.byref(f), C.byref(n), int(clear))
        if rc != OK:
            raise Co3Error(rc, "co3_status")
        return int(f.value), int(n.value)

    def get_fit(self, seg):
        v = [C.c_double() for _ in range(5)]
        rc = lib().co3_get_fit(self.handle, seg, *[C.byref(x) for x in v])
        if rc != OK:
            raise Co3Error(rc, "co3_get_fit")
        return tuple(x.value for x in v)        # beta, alpha, N, S1, S2

    def set_fit_override(self, fit=None):
        """Test hook: every later fit takes (beta, alpha) per segment from `fit` ([S][2] float64);
        None switches it off."""
        if fit is None:
            rc = lib().co3_set_fit_override(self.handle, None)
        else:
            f = np.ascontiguousarray(fit, np.float64)
            assert f.shape == (self.S, 2)
            rc = lib().co3_set_fit_override(self.handle, f.ctypes.data)
        if rc != OK:
            raise Co3Error(rc, "co3_set_fit_override")

    def debug_encode_stalled(self, out, spin_limit=1000, stream=None):
        """Test hook: the packing kernel once more with the block of (user 0, chunk 0) left out, so that
        the bounded waits for that chunk's size run out after spin_limit polls (FLAG_TIMEOUT)."""
        rc = lib().co3_debug_encode_stalled(self.handle, _ptr(out["bitstream"]), _ptr(out["sub_bits"]),
                                            _ptr(out["chunk_off"]), _ptr(out["user_bits"]), _ptr(out["hdr"]),
                                            int(spin_limit), self._stream(stream))
        if rc != OK:
            raise Co3Error(rc, "co3_debug_encode_stalled")

    def state_export(self):
        it = C.c_int64()
        nb = np.zeros(self.S, np.int32)
        rc = lib().co3_state_export(self.handle, C.byref(it), nb.ctypes.data)
        if rc != OK:
            raise Co3Error(rc, "co3_state_export")
        return int(it.value), nb

    def state_import(self, iteration, next_bias):
        nb = np.ascontiguousarray(next_bias, np.int32)
        rc = lib().co3_state_import(self.handle, int(iteration), nb.ctypes.data)
        if rc != OK:
            raise Co3Error(rc, "co3_state_import")

    def state_header(self, next_header=None):
        """CODE_LAGGED only: the header of the coming iteration, as an [S][3] int32 array
        (bias, ibeta, ir).  With an argument it is imported instead."""
        raw = np.zeros(self.S, np.int32)
        if next_header is not None:
            h = np.ascontiguousarray(next_header, np.int32)
            raw = ((h[:, 0] & 0xFF) | ((h[:, 1] & 0xFF) << 8) | ((h[:, 2] & 0xFFFF) << 16)).astype(np.uint32).view(np.int32)
            raw = np.ascontiguousarray(raw)
        rc = lib().co3_state_header(self.handle, 0 if next_header is None else 1, raw.ctypes.data)
        if rc != OK:
            raise Co3Error(rc, "co3_state_header")
        v = raw.view(np.uint32)
        out = np.zeros((self.S, 3), np.int32)
        out[:, 0] = (v & 0xFF).astype(np.uint8).view(np.int8)
        out[:, 1] = ((v >> 8) & 0xFF).astype(np.uint8).view(np.int8)
        out[:, 2] = ((v >> 16) & 0xFFFF).astype(np.uint16).view(np.int16)
        return out

    def profile_enable(self, kernel_names=None, max_records=4096):
        """Trace the named kernel classes (all if None; [] switches tracing off)."""
        names = KERNEL_NAMES if kernel_names is None else kernel_names
        mask = 0
        for n in names:
            mask |= 1 << KERNEL_NAMES.index(n)
        rc = lib().co3_profile_enable(self.handle, mask, max_records)
        if rc != OK:
            raise Co3Error(rc, "co3_profile_enable")

    def profile_stride(self, every):
        """Time only every `every`-th launch of each traced kernel class."""
        rc = lib().co3_profile_stride(self.handle, int(every))
        if rc != OK:
            raise Co3Error(rc, "co3_profile_stride")

    def profile_collect(self):
        """{kernel class: (total ms, launches)} since the last collect (synchronises)."""
        ms = np.zeros(len(KERNEL_NAMES), np.float64)
        n = np.zeros(len(KERNEL_NAMES), np.int64)
        rc = lib().co3_profile_collect(self.handle, ms.ctypes.data, n.ctypes.data)
        if rc != OK:
            raise Co3Error(rc, "co3_profile_collect")
        return {k: (float(ms[i]), int(n[i])) for i, k in enumerate(KERNEL_NAMES)}

    def launch_count(self):
        return int(lib().co3_launch_count(self.handle))

    def debug_symbols(self, stream=None):
        t = self.torch
        sym = t.zeros((self.U, self.d), dtype=t.uint8, device="cuda")
        rc = lib().co3_debug_symbols(self.handle, _ptr(sym), self._stream(stream))
        if rc != OK:
            raise Co3Error(rc, "co3_debug_symbols")
        return sym

    def debug_hist(self):
        h = np.zeros((self.S, self.nsym), np.uint64)
        rc = lib().co3_debug_hist(self.handle, h.ctypes.data)
        if rc != OK:
            raise Co3Error(rc, "co3_debug_hist")
        return h

    def debug_code(self, hdr):
        ln = np.zeros((self.S, self.nsym), np.uint8)
        cw = np.zeros((self.S, self.nsym), np.uint32)
        rc = lib().co3_debug_code(self.handle, _ptr(hdr), ln.ctypes.data, cw.ctypes.data)
        if rc != OK:
            raise Co3Error(rc, "co3_debug_code")
        return ln, cw


def hdr_to_numpy(hdr_tensor):
    """[S] int32 device tensor of packed headers -> [S][3] int32 (bias, ibeta, ir)."""
    raw = hdr_tensor.cpu().numpy().view(HDR_DTYPE)
    return np.stack([raw["bias"].astype(np.int32), raw["ibeta"].astype(np.int32),
                     raw["ir"].astype(np.int32)], axis=1)


def hdr_from_numpy(hdr3, device="cuda"):
    import torch
    raw = np.zeros(len(hdr3), HDR_DTYPE)
    raw["bias"], raw["ibeta"], raw["ir"] = hdr3[:, 0], hdr3[:, 1], hdr3[:, 2]
    return torch.from_numpy(raw.view(np.int32).copy()).to(device)


# ---- optimizer: gradient norm and AdamW over many tensors ---------------------------------------------------------
_type_codes = {}


def _type_code(dtype):
    if not _type_codes:
        import torch
        _type_codes.update({torch.float32: F32, torch.bfloat16: BF16, torch.float16: F16})
    code = _type_codes.get(dtype)
    if code is None:
        raise TypeError(f"float32, bfloat16 or float16 expected, got {dtype}")
    return code


def _dense(t):
    """Whether the elements of t fill one piece of memory, in whatever order of dimensions."""
    at = 1
    for stride, size in sorted((st, n) for st, n in zip(t.stride(), t.shape) if n != 1):
        if stride != at:
            return False
        at *= size
    return True


def _order(t):
    """The order in memory of t's elements: None for the usual one, else its sizes and strides."""
    return None if t.is_contiguous() else tuple((n, st) for n, st in zip(t.shape, t.stride()) if n != 1)


def _refuse_shared(arrays):
    """arrays: (name, tensor) of all that a step writes, each in one piece of memory; raises if two of them share some."""
    spans = sorted((t.data_ptr(), t.data_ptr() + t.numel() * t.element_size(), name) for name, t in arrays if t.numel())
    for (_, end, a), (begin, _, b) in zip(spans, spans[1:]):
        if begin < end:
            raise ValueError(f"{a} and {b} share memory")


class TensorList:
    """Tensors of one dtype whose pointers have been looked at and put into a host array once (GradNorm.bind_grads).  It keeps
    the tensors; bind again after giving one of them other storage."""

    def __init__(self, tensors, sizes, dtype, device, what, order=None, fits=None):
        self.tensors = list(tensors)
        if len(self.tensors) != len(sizes):
            raise ValueError(f"{len(sizes)} {what} expected, got {len(self.tensors)}")
        for i, (t, n) in enumerate(zip(self.tensors, sizes)):
            if t.dtype != dtype or t.device != device:
                raise ValueError(f"{what} {i}: {dtype} on {device} expected, got {t.dtype} on {t.device}")
            if t.numel() != n:
                raise ValueError(f"{what} {i}: {n} elements expected, got {t.numel()}")
            if n and not _dense(t):
                raise ValueError(f"{what} {i}: its elements do not fill one piece of memory (shape {tuple(t.shape)}, strides {t.stride()})")
            if order is not None and n and _order(t) != order[i]:
                raise ValueError(f"{what} {i}: its elements lie in another order than those of its weights")
        self.pointers = (C.c_void_p * len(sizes))(*[t.data_ptr() if n else None for t, n in zip(self.tensors, sizes)])
        self.address, self.fits = C.addressof(self.pointers), fits


class GradNorm:
    """Gradient norm, clipping factor and count of non-finite elements of a set of tensors (co3_grad_norm), on the current
    CUDA device.  `sizes`: elements per tensor."""

    def __init__(self, sizes, grad_dtype=None):
        import torch
        self._create([int(n) for n in sizes], torch.float32, grad_dtype or torch.float32, None, 32, (0.0, 0.0), 0.0, 0.0, 0)

    def _create(self, sizes, weight_dtype, grad_dtype, copy_dtype, state_bits, betas, eps, weight_decay, seed, device=None):
        import torch
        self.torch, self.sizes, self.grad_dtype = torch, sizes, grad_dtype
        self._increment_version = torch._C._increment_version          # torch.autograd.graph.increment_version of a list
        self._data_ptr, self._float32 = torch.Tensor.data_ptr, torch.float32
        self._order, self._fits = None, object()          # the second goes into every list that was looked at by this object, in this order
        n = np.ascontiguousarray(sizes, np.int64)
        per_tensor = None if np.ndim(weight_decay) == 0 else np.ascontiguousarray(weight_decay, np.float32)
        if per_tensor is not None and per_tensor.shape != n.shape:
            raise ValueError(f"weight_decay: one number, or one for each of the {len(n)} tensors")
        cfg = AdamwConfig(len(n), n.ctypes.data_as(C.POINTER(C.c_int64)),
                          None if per_tensor is None else per_tensor.ctypes.data_as(C.POINTER(C.c_float)),
                          _type_code(weight_dtype), _type_code(grad_dtype), NONE if copy_dtype is None else _type_code(copy_dtype),
                          int(state_bits), float(betas[0]), float(betas[1]), float(eps),
                          float(weight_decay) if per_tensor is None else 0.0, int(seed) & 0xFFFFFFFF, 0)
        h = C.c_void_p()
        rc = lib().co3_adamw_create(C.byref(h), C.byref(cfg))
        if rc != OK:
            raise Co3Error(rc, "co3_adamw_create")
        self.handle, self._lib = h, lib()
        self.device = torch.device("cuda", torch.cuda.current_device())
        self._current_stream = functools.partial(torch._C._cuda_getCurrentRawStream, self.device.index)   # torch.cuda.current_stream's handle
        nb = C.c_int64()
        lib().co3_adamw_sizes(h, C.byref(nb), None)
        self.n_blocks = nb.value

    def close(self):
        if getattr(self, "handle", None):
            lib().co3_adamw_destroy(self.handle)
            self.handle = None

    def __del__(self):
        try:
            self.close()
        except Exception:
            pass

    @staticmethod
    def _record(stream, tensors):
        """The allocator must not hand the tensors' memory on while that stream uses it."""
        for t in tensors:
            if t is not None:
                t.record_stream(stream)
        return stream.cuda_stream

    def _empty(self, shape, dtype, stream):
        """Memory for an output that `stream` writes (None: the current one), from that stream's own: memory of the current stream may
        still be in use by work that waits there.  The caller may in turn use it on the current stream when it is given back."""
        if stream is None:
            return self.torch.empty(shape, dtype=dtype, device=self.device)
        with self.torch.cuda.stream(stream):
            t = self.torch.empty(shape, dtype=dtype, device=self.device)
        t.record_stream(self.torch.cuda.current_stream(self.device))
        return t

    def bind_grads(self, grads):
        """Check the gradient tensors and keep their pointers, for programs whose gradients stay where they are.  (What another
        optimizer's bind_grads returned is checked again.)"""
        if type(grads) is TensorList:
            grads = grads.tensors
        return TensorList(grads, self.sizes, self.grad_dtype, self.device, "gradients", self._order, self._fits)

    def grad_norm(self, grads, info=None, max_norm=0.0, grad_scale=1.0, tensor_norms=None, stream=None):
        """grads: the tensors, or what bind_grads returned.  info: 4 float32 on the device, written and returned: factor, norm,
        and in the last two the count of non-finite elements as one int64 (`info[2:].view(torch.int64)`)."""
        g = grads if type(grads) is TensorList and grads.fits is self._fits else self.bind_grads(grads)
        if info is None:
            info = self._empty(4, self.torch.float32, stream)
        _check(info, self.torch.float32, 4, self.device, "info")
        if tensor_norms is not None:
            _check(tensor_norms, self.torch.float32, len(self.sizes), self.device, "tensor_norms")
        s = self._current_stream() if stream is None else self._record(stream, [info, tensor_norms, *g.tensors])
        rc = self._lib.co3_grad_norm(self.handle, g.address, grad_scale, max_norm,
                                     None if tensor_norms is None else tensor_norms.data_ptr(), info.data_ptr(), s)
        if rc != OK:
            raise Co3Error(rc, "co3_grad_norm")
        return info

    def status(self, clear=False):
        """(flags, elements left out, steps left out); synchronises."""
        f, e, s = C.c_uint32(), C.c_uint64(), C.c_uint64()
        rc = lib().co3_adamw_status(self.handle, C.byref(f), C.byref(e), C.byref(s), int(clear))
        if rc != OK:
            raise Co3Error(rc, "co3_adamw_status")
        return int(f.value), int(e.value), int(s.value)

    def launch_count(self):
        return int(lib().co3_adamw_launch_count(self.handle))


def _check(t, dtype, n, device, what):
    if t.dtype is not dtype or t.numel() != n or t.device != device or not t.is_contiguous():
        _refuse(t, dtype, n, device, what)


def _refuse(t, dtype, n, device, what):
    raise ValueError(f"{what}: {n} contiguous {dtype} on {device} expected, got {t.numel()} {t.dtype} on {t.device}")


def _moment(name):
    def get(self):
        if name not in self._moments:
            raise AttributeError(name)
        return self._moments[name].detach()               # the optimizer's own is nobody else's, to be given other storage

    def put(self, tensor):
        self._bind_own(self.params.tensors, self.copies.tensors if self.copies else None, {**self._moments, name: tensor})
    return property(get, put)


class AdamW(GradNorm):
    """AdamW over the tensors `params` (float32 or bfloat16, on the current CUDA device, updated in place; any dense order of
    dimensions, gradients and copies in the same).  copies: tensors of bfloat16 or float16 that receive the new float32 weights.  No
    two of these share memory: a tensor that a model uses in two places is given once.
    weight_decay: one number, or one per tensor.  state_bits: 32, or 8 for moments of one byte each (include/co3.h).  An eps below
    about 6e-11 makes steps slower (ditto).
    The moments are the attributes m, v (and m_exp, v_exp): [n_blocks][256]; `state` gives existing ones (set_steps then sets the
    steps that they come from).  Weights, copies and moments may be given other storage between two steps (`p.data = x`, `opt.m = x`;
    a view stands for its part of the tensor that it is a view of, whatever becomes of the view); a captured step keeps what it was
    captured with."""

    m, v, m_exp, v_exp = (_moment(k) for k in ("m", "v", "m_exp", "v_exp"))

    def __init__(self, params, grad_dtype=None, copies=None, lr=1e-3, betas=(0.9, 0.999), eps=1e-8, weight_decay=0.01, state_bits=32,
                 seed=0, state=None):
        import torch
        params = list(params)
        if not params:
            raise ValueError("no tensors")
        sizes = [p.numel() for p in params]
        dtype = params[0].dtype
        copies = None if copies is None else list(copies)
        if copies is not None and not copies:
            raise ValueError("no copies")
        self._create(sizes, dtype, grad_dtype or dtype, copies[0].dtype if copies else None, state_bits, betas, eps, weight_decay, seed)
        self.lr, self.state_bits = float(lr), int(state_bits)
        self._dtype, self._copy_dtype = dtype, copies[0].dtype if copies else None
        self._kind = torch.float32 if self.state_bits == 32 else torch.uint8
        self._shapes = dict(m=(self.n_blocks, STATE_BLOCK), v=(self.n_blocks, STATE_BLOCK))
        if self.state_bits == 8:
            self._shapes.update(m_exp=(self.n_blocks,), v_exp=(self.n_blocks,))
        if state is None:
            state = {k: torch.zeros(shape, dtype=self._kind, device=self.device) for k, shape in self._shapes.items()}
            torch.cuda.current_stream(self.device).synchronize()      # zero for a first step on any stream
        self._bind_own(params, copies, {k: state[k] for k in self._shapes})

    def _bind_own(self, params, copies, moments):
        """Look at weights, copies and moments and keep where they are; nothing changes if one does not fit."""
        weights = TensorList(params, self.sizes, self._dtype, self.device, "weights")
        order = [_order(p) for p in weights.tensors]
        if copies is not None:
            copies = TensorList(copies, self.sizes, self._copy_dtype, self.device, "copies", order)
        for k, shape in self._shapes.items():
            _check(moments[k], self._kind, int(np.prod(shape)), self.device, k)
        moments = {k: moments[k].detach() for k in self._shapes}
        _refuse_shared([*((f"weights {i}", t) for i, t in enumerate(weights.tensors)),
                        *((f"copies {i}", t) for i, t in enumerate(copies.tensors if copies else [])), *moments.items()])
        if order != self._order:
            self._fits = object()                         # gradients bound so far are looked at again
        self.params, self.copies, self._moments, self._order = weights, copies, moments, order
        self._state = AdamwState(*[moments[k].data_ptr() if k in moments else None for k in ("m", "v", "m_exp", "v_exp")])
        self._state_p = C.addressof(self._state)
        self._weights, self._copies = weights.address, None if copies is None else copies.address
        written = weights.tensors + (copies.tensors if copies else [])
        self._own = written + list(moments.values())
        # Of the views of one tensor only one is looked at before a step, and one version counter moved after it: they share both memory and
        # counter, and a row in hundreds of pieces costs no more than one tensor (290 pieces 0.3 us, 290 tensors of their own 26).
        bases = [t._base if t._is_view() else t for t in written]
        self._written = list({id(base): t for base, t in zip(bases, written)}.values())
        self._at = [t.data_ptr() for t in self._written]

    def _rebind(self):
        """A program has given a weight or copy other storage since, and what it had may be somebody else's by now."""
        self._bind_own(self.params.tensors, self.copies.tensors if self.copies else None, self._moments)

    def bind_grads(self, grads):
        if [*map(self._data_ptr, self._written)] != self._at:
            self._rebind()                                # the order of the weights is the gradients'
        return super().bind_grads(grads)

    def step(self, grads, info=None, lr=None, stream=None):
        """One step.  info: what grad_norm returned (its factor multiplies the gradients, and nothing is changed if it counted
        non-finite elements).  lr: a number, or one float32 on the device, in place of the optimizer's."""
        if [*map(self._data_ptr, self._written)] != self._at:
            self._rebind()
        g = grads if type(grads) is TensorList and grads.fits is self._fits else GradNorm.bind_grads(self, grads)
        d_lr = None
        if lr is None:
            lr = self.lr
        elif isinstance(lr, self.torch.Tensor):
            _check(lr, self._float32, 1, self.device, "lr")
            d_lr, lr = lr, 0.0
        if info is not None and (info.dtype is not self._float32 or info.numel() != 4 or info.device != self.device or not info.is_contiguous()):
            _refuse(info, self._float32, 4, self.device, "info")
        s = self._current_stream() if stream is None else self._record(stream, [info, d_lr, *g.tensors, *self._own])
        rc = self._lib.co3_adamw_step(self.handle, self._weights, g.address, self._copies, self._state_p, lr,
                                      None if d_lr is None else d_lr.data_ptr(), None if info is None else info.data_ptr(), s)
        if rc != OK:
            raise Co3Error(rc, "co3_adamw_step")
        self._increment_version(self._written)

    def state_values(self, m_out=None, v_out=None, stream=None):
        """What the 8-bit moments stand for, [n_blocks][256] each, in float32 or bfloat16 (exact in both; bfloat16 if neither is
        given)."""
        given = m_out if m_out is not None else v_out
        n, kind = self.n_blocks * STATE_BLOCK, self.torch.bfloat16 if given is None else given.dtype
        if m_out is None:
            m_out = self._empty((self.n_blocks, STATE_BLOCK), kind, stream)
        if v_out is None:
            v_out = self._empty((self.n_blocks, STATE_BLOCK), kind, stream)
        _check(m_out, kind, n, self.device, "m_out")
        _check(v_out, kind, n, self.device, "v_out")
        if stream is None:
            s = self._current_stream()
        else:
            s = self._record(stream, [m_out, v_out, *self._moments.values()])
        rc = self._lib.co3_adamw_values(self.handle, self._state_p, m_out.data_ptr(), v_out.data_ptr(), _type_code(kind), s)
        if rc != OK:
            raise Co3Error(rc, "co3_adamw_values")
        return m_out, v_out

    def moments_of(self, i):
        """Views of the two moment arrays (codes with 8 bits) of tensor i, in the order in memory of its weights."""
        b = sum((n + STATE_BLOCK - 1) // STATE_BLOCK for n in self.sizes[:i]) * STATE_BLOCK
        return tuple(t.view(-1)[b:b + self.sizes[i]] for t in (self.m, self.v))

    def steps(self):
        """Steps taken so far (synchronises)."""
        n = C.c_int64()
        rc = lib().co3_adamw_steps_export(self.handle, C.byref(n))
        if rc != OK:
            raise Co3Error(rc, "co3_adamw_steps_export")
        return n.value

    def set_steps(self, steps):
        rc = lib().co3_adamw_steps_import(self.handle, int(steps))
        if rc != OK:
            raise Co3Error(rc, "co3_adamw_steps_import")


# ---- the two ends of a language model: embedding, layer norm, losses over the vocabulary -----------------------------
_token_kinds = {}


def _token_codes(dtype):
    if not _token_kinds:
        import torch
        _token_kinds.update({torch.int32: I32, torch.int64: I64})
    return _token_kinds.get(dtype)


class _Operator:
    """A handle of the library on the current CUDA device, for batches [users][tokens] (with one user also [tokens]).  The calls only enqueue
    kernels, on the current stream or the one given, and share the handle's scratch: use one handle on one stream at a time.  They are not
    recorded by autograd; what a call writes is marked as changed."""

    _kind, _status = None, False
    _record, _empty = staticmethod(GradNorm._record), GradNorm._empty

    def _create(self, make, n_users):
        import torch
        self.torch, self._lib, self.n_users, self._float32 = torch, lib(), int(n_users), torch.float32
        self._shapes, self._empty_like = {}, torch.empty_like
        self._increment_version = torch._C._increment_version
        h = C.c_void_p()
        rc = make(C.byref(h))
        if rc != OK:
            raise Co3Error(rc, f"co3_{self._kind}_create")
        self.handle = h
        self.device = torch.device("cuda", torch.cuda.current_device())
        self._current_stream = functools.partial(torch._C._cuda_getCurrentRawStream, self.device.index)

    def close(self):
        if getattr(self, "handle", None):
            getattr(self._lib, f"co3_{self._kind}_destroy")(self.handle)
            self.handle = None

    def __del__(self):
        try:
            self.close()
        except Exception:
            pass

    def launch_count(self):
        return int(getattr(self._lib, f"co3_{self._kind}_launch_count")(self.handle))

    def _get_status(self, clear):
        f, n = C.c_uint32(), C.c_uint64()
        rc = getattr(self._lib, f"co3_{self._kind}_status")(self.handle, C.byref(f), C.byref(n), int(clear))
        if rc != OK:
            raise Co3Error(rc, f"co3_{self._kind}_status")
        return int(f.value), int(n.value)

    def _new(self, shape, dtype, stream):
        """Memory for an output, of a shape and type that this object keeps a view of one element of: asking for a tensor like that one is the
        quickest way to memory (0.9 us, 2.4 from a shape and a type)."""
        if stream is not None:
            return self._empty(shape, dtype, stream)
        like = self._shapes.get((shape, dtype))
        if like is None:
            if len(self._shapes) >= 64:
                self._shapes.clear()
            like = self._shapes[shape, dtype] = self.torch.empty(1, dtype=dtype, device=self.device).expand(shape)
        return self._empty_like(like)

    def _batch(self, t, dim, what, like=None):
        """co3_array of a tensor [users][tokens][dim] and its tokens; `like`: the leading sizes that it has to have."""
        shape, users = t.shape, self.n_users
        if len(shape) == 3 and shape[0] == users and shape[2] == dim and t.device == self.device and t.is_contiguous() and (like is None or shape[:2] == like):
            return Array(t.data_ptr(), _type_code(t.dtype), 0, shape[1] * dim, dim), shape[1]
        strides = t.stride()
        if t.device != self.device:
            raise ValueError(f"{what}: a tensor on {self.device} expected, got one on {t.device}")
        if len(shape) == 2 and users == 1:
            tokens, us, ts = shape[0], 0, strides[0]
        elif len(shape) == 3 and shape[0] == users:
            tokens, us, ts = shape[1], strides[0], strides[1]
        else:
            raise ValueError(f"{what}: [{users}, tokens, {dim}] expected, got {tuple(shape)}")
        if shape[-1] != dim or (dim > 1 and strides[-1] != 1):
            raise ValueError(f"{what}: rows of {dim} elements side by side expected, got shape {tuple(shape)}, strides {strides}")
        if like is not None and shape[:-1] != like:
            raise ValueError(f"{what}: {tuple(like)} rows expected, got {tuple(shape[:-1])}")
        return Array(t.data_ptr(), _type_code(t.dtype), 0, us, ts), tokens

    def _own_batch(self, t, dim, n):
        """... of one that was made here."""
        return Array(t.data_ptr(), _type_code(t.dtype), 0, n * dim, dim)

    def _tokens(self, t, what="tokens", like=None, top=None):
        """co3_tokens of whole numbers [users][tokens], or [users][tokens][top]."""
        kind = _token_codes(t.dtype)
        if kind is None or t.device != self.device:
            raise ValueError(f"{what}: int32 or int64 on {self.device} expected, got {t.dtype} on {t.device}")
        shape, strides = t.shape, t.stride()
        lead = shape if top is None else shape[:-1]
        if top is not None and (len(shape) < 2 or (top > 1 and strides[-1] != 1)):
            raise ValueError(f"{what}: entries of a token side by side expected, got shape {tuple(shape)}, strides {strides}")
        if len(lead) == 2 and lead[0] == self.n_users:
            us, ts = strides[0], strides[1]
        elif len(lead) == 1 and self.n_users == 1:
            us, ts = 0, strides[0]
        else:
            raise ValueError(f"{what}: [{self.n_users}, tokens] expected, got {tuple(lead)}")
        if like is not None and lead != like:
            raise ValueError(f"{what}: {tuple(like)} expected, got {tuple(lead)}")
        return Tokens(t.data_ptr(), kind, 1 if top is None else top, us, ts), lead

    def _grad(self, t, n, accumulate, what):
        """co3_param_grad of a tensor that holds n elements for each user, each user's in one piece."""
        users = self.n_users
        if t.device != self.device or t.numel() != users * n:
            raise ValueError(f"{what}: {users} times {n} elements on {self.device} expected, got {tuple(t.shape)} on {t.device}")
        if t.is_contiguous() and (users == 1 or t.shape[0] == users):
            return ParamGrad(t.data_ptr(), _type_code(t.dtype), bool(accumulate), n)
        shape, strides = t.shape, t.stride()
        if users > 1 and (not shape or shape[0] != users):
            raise ValueError(f"{what}: [{users}, ...] expected, got {tuple(shape)}")
        at = 1
        for i in range(len(shape) - 1, 0 if users > 1 else -1, -1):
            if shape[i] != 1 and strides[i] != at and n:
                raise ValueError(f"{what}: each user's part in one piece expected, got shape {tuple(shape)}, strides {strides}")
            at *= shape[i]
        return ParamGrad(t.data_ptr(), _type_code(t.dtype), bool(accumulate), strides[0] if users > 1 else n)

    def _vector(self, t, n, what):
        """Pointer and type of a weight of n elements, or (None, F32)."""
        if t is None:
            return None, F32
        if t.numel() != n or t.device != self.device or not t.is_contiguous():
            raise ValueError(f"{what}: {n} contiguous elements on {self.device} expected, got {tuple(t.shape)} on {t.device}")
        return t.data_ptr(), _type_code(t.dtype)

    def _per_token(self, t, like, what):
        if t.dtype is not self._float32 or t.shape != like or t.device != self.device or not t.is_contiguous():
            raise ValueError(f"{what}: contiguous float32 {tuple(like)} on {self.device} expected, got {t.dtype} {tuple(t.shape)} on {t.device}")
        return t.data_ptr()

    def _output(self, t, lead, what, stream):
        """A float32 output of a number a token, the one given or a new one, and its pointer."""
        if t is not None:
            return t, self._per_token(t, lead, what)
        t = self._new(lead, self._float32, stream)
        return t, t.data_ptr()

    def _on(self, stream, tensors):
        return self._current_stream() if stream is None else self._record(stream, tensors)

    def _changed(self, *given):
        """What the caller gave to be written."""
        given = [t for t in given if t is not None]
        if given:
            self._increment_version(given)


class Embedding(_Operator):
    """Embedding lookup and its gradient (co3_embed_*).  tokens: the most that a user has in a call."""

    _kind = "embed"

    def __init__(self, vocab, dim, n_users=1, *, tokens):
        self.vocab, self.dim = int(vocab), int(dim)
        self._create(lambda h: lib().co3_embed_create(h, self.vocab, self.dim, int(n_users), int(tokens)), n_users)

    def status(self, clear=False):
        """(flags, token numbers met that the vocabulary does not have); synchronises."""
        return self._get_status(clear)

    def forward(self, tokens, table, scale=1.0, out=None, out_dtype=None, stream=None):
        """scale * table[token], zeros where a token is below zero: [*tokens.shape, dim], in out_dtype (the table's if None)."""
        k, lead = self._tokens(tokens)
        if table.shape != (self.vocab, self.dim) or not table.is_contiguous() or table.device != self.device:
            raise ValueError(f"table: contiguous [{self.vocab}, {self.dim}] on {self.device} expected, got {tuple(table.shape)} on {table.device}")
        given, n = out, lead[-1]
        if out is None:
            out = self._new((*lead, self.dim), out_dtype or table.dtype, stream)
            o = self._own_batch(out, self.dim, n)
        else:
            if out_dtype not in (None, out.dtype):
                raise ValueError(f"out: {out_dtype} expected, got {out.dtype}")
            o, _ = self._batch(out, self.dim, "out", lead)
        s = self._on(stream, (tokens, table, out))
        rc = self._lib.co3_embed_forward(self.handle, k, n, table.data_ptr(), _type_code(table.dtype), scale, o, s)
        if rc != OK:
            raise Co3Error(rc, "co3_embed_forward")
        self._changed(given)
        return out

    def backward(self, dout, tokens, dtable, scale=1.0, accumulate=False, stream=None):
        """Gradient of the table for each user into dtable: [users, vocab * dim] or [users, vocab, dim], each user's part in one piece
        (a segment of gradient rows)."""
        k, lead = self._tokens(tokens)
        g, n = self._batch(dout, self.dim, "dout", lead)
        t = self._grad(dtable, self.vocab * self.dim, accumulate, "dtable")
        s = self._on(stream, (dout, tokens, dtable))
        rc = self._lib.co3_embed_backward(self.handle, g, k, n, scale, t, s)
        if rc != OK:
            raise Co3Error(rc, "co3_embed_backward")
        self._changed(dtable)
        return dtable


class LayerNorm(_Operator):
    """Layer norm over the last dimension, forward and backward (co3_layernorm_*)."""

    _kind = "layernorm"

    def __init__(self, dim, n_users=1, eps=1e-5):
        self.dim, self.eps = int(dim), float(eps)
        self._create(lambda h: lib().co3_layernorm_create(h, self.dim, int(n_users), self.eps), n_users)

    def forward(self, x, weight=None, bias=None, y=None, mean=None, rstd=None, stream=None):
        """(y, mean, rstd); y has x's type, mean and rstd are float32, one for each row."""
        dim = self.dim
        a, n = self._batch(x, dim, "x")
        lead = x.shape[:-1]
        w, wt = self._vector(weight, dim, "weight")
        b, bt = self._vector(bias, dim, "bias")
        if weight is None:
            wt = bt
        elif bias is not None and wt != bt:
            raise ValueError(f"weight and bias of one type expected, got {weight.dtype} and {bias.dtype}")
        given = y, mean, rstd
        if y is None:
            y = self._new(x.shape, x.dtype, stream)
            o = self._own_batch(y, dim, n)
        else:
            o, _ = self._batch(y, dim, "y", lead)
        mean, m = self._output(mean, lead, "mean", stream)
        rstd, r = self._output(rstd, lead, "rstd", stream)
        s = self._on(stream, (x, weight, bias, y, mean, rstd))
        rc = self._lib.co3_layernorm_forward(self.handle, a, w, b, wt, n, o, m, r, s)
        if rc != OK:
            raise Co3Error(rc, "co3_layernorm_forward")
        self._changed(*given)
        return y, mean, rstd

    def backward(self, dy, x, weight, mean, rstd, dx=None, dweight=None, dbias=None, accumulate=False, want_dx=True, stream=None):
        """dx (None if not wanted); the users' gradients of weight and bias go into dweight and dbias ([users, dim], any float type) where
        given."""
        dim, given = self.dim, dx
        a, n = self._batch(x, dim, "x")
        lead = x.shape[:-1]
        g, _ = self._batch(dy, dim, "dy", lead)
        w, wt = self._vector(weight, dim, "weight")
        m, r = self._per_token(mean, lead, "mean"), self._per_token(rstd, lead, "rstd")
        o = None
        if dx is not None:
            o, _ = self._batch(dx, dim, "dx", lead)
        elif want_dx:
            dx = self._new(x.shape, x.dtype, stream)
            o = self._own_batch(dx, dim, n)
        dw = None if dweight is None else self._grad(dweight, dim, accumulate, "dweight")
        db = None if dbias is None else self._grad(dbias, dim, accumulate, "dbias")
        s = self._on(stream, (dy, x, weight, mean, rstd, dx, dweight, dbias))
        rc = self._lib.co3_layernorm_backward(self.handle, g, a, w, wt, m, r, n, o, dw, db, s)
        if rc != OK:
            raise Co3Error(rc, "co3_layernorm_backward")
        self._changed(given, dweight, dbias)
        return dx


class TokenLoss(_Operator):
    """Losses of tokens over a large vocabulary from the last hidden states, with their gradients, without the logits being kept
    (co3_token_loss_*).  dtype: of hidden states and weight, bfloat16 or float16.  grad_dtype: of the weight's gradient, float32 or dtype.
    tokens: the most that a user has in a call; top: the most entries that a teacher gives for a token."""

    _kind = "token_loss"

    def __init__(self, vocab, dim, n_users=1, *, tokens, dtype=None, grad_dtype=None, top=1):
        import torch
        self.vocab, self.dim, self.dtype, self.grad_dtype = int(vocab), int(dim), dtype or torch.bfloat16, grad_dtype or torch.float32
        cfg = TokenLossConfig(self.vocab, self.dim, int(tokens), int(n_users), _type_code(self.dtype), _type_code(self.grad_dtype), int(top))
        self._create(lambda h: lib().co3_token_loss_create(h, C.byref(cfg)), n_users)

    def status(self, clear=False):
        """(flags, target numbers met that the vocabulary does not have); synchronises."""
        return self._get_status(clear)

    def loss(self, hidden, weight, targets, loss=None, lse=None, stream=None):
        """Cross entropy: (loss, lse), float32 like targets; 0 where a target is below zero."""
        return self._forward(hidden, weight, targets, None, 1.0, loss, lse, stream)

    def loss_grad(self, hidden, weight, targets, lse, dloss=None, scale=1.0, dhidden=None, dweight=None, accumulate=False, want_dhidden=True,
                  stream=None):
        """dhidden (None if not wanted); the users' gradients of the weight go into dweight where given ([users, vocab * dim], see
        Embedding.backward).  lse: what loss() gave.  dloss: gradient of each token's loss, 0 where none is wanted, whatever the token
        holds; None: of the mean over each user's tokens that have a target."""
        return self._backward(hidden, weight, targets, None, 1.0, lse, dloss, scale, dhidden, dweight, accumulate, want_dhidden, stream)

    def distill(self, hidden, weight, index, logits, temperature=1.0, loss=None, lse=None, stream=None):
        """Divergence from a teacher's top logits: index (whole numbers) and logits [*, tokens, top]; (loss, lse) as loss()."""
        return self._forward(hidden, weight, index, logits, temperature, loss, lse, stream)

    def distill_grad(self, hidden, weight, index, logits, lse, dloss=None, temperature=1.0, scale=1.0, dhidden=None, dweight=None, accumulate=False,
                     want_dhidden=True, stream=None):
        return self._backward(hidden, weight, index, logits, temperature, lse, dloss, scale, dhidden, dweight, accumulate, want_dhidden, stream)

    def _inputs(self, hidden, weight, targets, logits):
        h, n = self._batch(hidden, self.dim, "hidden")
        if hidden.dtype is not self.dtype or weight.dtype is not self.dtype:
            raise TypeError(f"hidden and weight in {self.dtype} expected, got {hidden.dtype} and {weight.dtype}")
        strides = weight.stride()
        if weight.shape != (self.vocab, self.dim) or weight.device != self.device or strides[1] != 1:
            raise ValueError(f"weight: rows of [{self.vocab}, {self.dim}] on {self.device} expected, got {tuple(weight.shape)}, strides {strides}, on {weight.device}")
        lead, t = hidden.shape[:-1], None
        if logits is None:
            k, _ = self._tokens(targets, "targets", lead)
        else:
            top = targets.shape[-1] if targets.dim() else 1
            k, _ = self._tokens(targets, "index", lead, top)
            t, _ = self._batch(logits, top, "logits", lead)
        return h, n, lead, k, t, weight.data_ptr(), strides[0] if self.vocab > 1 else self.dim

    def _forward(self, hidden, weight, targets, logits, temperature, loss, lse, stream):
        h, n, lead, k, t, w, stride = self._inputs(hidden, weight, targets, logits)
        given = loss, lse
        loss, p = self._output(loss, lead, "loss", stream)
        lse, q = self._output(lse, lead, "lse", stream)
        s = self._on(stream, (hidden, weight, targets, logits, loss, lse))
        rc = self._lib.co3_token_loss_forward(self.handle, h, w, stride, k, t, temperature, n, p, q, s)
        if rc != OK:
            raise Co3Error(rc, "co3_token_loss_forward")
        self._changed(*given)
        return loss, lse

    def _backward(self, hidden, weight, targets, logits, temperature, lse, dloss, scale, dhidden, dweight, accumulate, want_dhidden, stream):
        h, n, lead, k, t, w, stride = self._inputs(hidden, weight, targets, logits)
        p = self._per_token(lse, lead, "lse")
        q = None if dloss is None else self._per_token(dloss, lead, "dloss")
        given, o = dhidden, None
        if dhidden is not None:
            o, _ = self._batch(dhidden, self.dim, "dhidden", lead)
        elif want_dhidden:
            dhidden = self._new(hidden.shape, self.dtype, stream)
            o = self._own_batch(dhidden, self.dim, n)
        d = None if dweight is None else self._grad(dweight, self.vocab * self.dim, accumulate, "dweight")
        s = self._on(stream, (hidden, weight, targets, logits, lse, dloss, dhidden, dweight))
        rc = self._lib.co3_token_loss_backward(self.handle, h, w, stride, k, t, temperature, n, p, q, scale, o, d, s)
        if rc != OK:
            raise Co3Error(rc, "co3_token_loss_backward")
        self._changed(given, dweight)
        return dhidden
