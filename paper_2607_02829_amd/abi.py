"""ctypes binding of libsr (include/sr.h): the same names, argument marshalling only.

Tensor arguments are torch tensors on the GPU (their ``data_ptr()`` is passed) or
raw integer device addresses; ``stream=None`` uses torch's current stream.  A
non-OK status raises ``SrError`` carrying ``sr_last_error()``.  If libsr.so has
not been built, ``lib()`` raises ``SrLibraryMissing``: there is no fallback.
"""
from __future__ import annotations

import ctypes
import os

HERE = os.path.dirname(os.path.abspath(__file__))
LIB_PATH = os.path.join(HERE, "libsr.so")

SR_OK, SR_EINVAL, SR_ESHAPE, SR_EDTYPE, SR_EALIGN, SR_EWORKSPACE, SR_EUNSUPPORTED, SR_EHIP = range(8)
SR_F32, SR_BF16 = 0, 1
SR_BLOCK_PRELN, SR_BLOCK_ADALN = 0, 1
SR_BLOCK_SAVE8 = 16
SR_SEL_RANDOM, SR_SEL_TOPK_DIFFNORM = 0, 1
SR_Q8_ROW, SR_Q8_BLOCK = 0, 1
SR_ACT_NONE, SR_ACT_GELU = 0, 1
SR_ROT_HALVES, SR_ROT_NEIGHBOURS = 0, 1
SR_NORM_LAYER, SR_NORM_RMS = 0, 1
SR_F8_ROW, SR_F8_TILE = 0, 1

PARAM_FIELDS = ("ln1_w", "ln1_b", "w_qkv", "b_qkv", "w_o", "b_o", "ln2_w", "ln2_b",
                "w_fc1", "b_fc1", "w_fc2", "b_fc2", "w_ada", "b_ada")

EXPORTS = ("sr_last_error", "sr_version", "sr_workspace_bytes", "sr_select_scratch_bytes",
           "sr_select_indices", "sr_select_indices_noalloc", "sr_gather", "sr_scatter_delta", "sr_sparse_blocks_fwd",
           "sr_sparse_blocks_bwd", "sr_dense_blocks_fwd", "sr_dense_blocks_bwd", "sr_validate_indices",
           "sr_attention_colsums", "sr_select_topk_scores", "sr_routed_blocks_fwd", "sr_routed_blocks_bwd",
           "sr_cross_attention_fwd", "sr_cross_attention_bwd",
           "sr_edm_workspace_bytes", "sr_edm_blocks_fwd", "sr_edm_blocks_bwd",
           "sr_quantize8", "sr_dequantize8", "sr_linear8", "sr_weight_grad8", "sr_weight_grad8_scratch_bytes",
           "sr_blocks8_scratch_bytes", "sr_blocks8_fwd",
           "sr_rotary", "sr_dropout", "sr_residual_norm_fwd", "sr_residual_norm_scratch_bytes", "sr_residual_norm_bwd",
           "sr_quantize_f8", "sr_linear_f8_scratch_bytes", "sr_linear_f8",
           "sr_profile_start", "sr_profile_stop", "sr_probe_mfma_rate")


class SrLibraryMissing(RuntimeError):
    pass


class SrError(RuntimeError):
    def __init__(self, status: int, msg: str):
        super().__init__(f"libsr status {status}: {msg}")
        self.status = status


class SrConfig(ctypes.Structure):
    _fields_ = [("B", ctypes.c_int32), ("L", ctypes.c_int32), ("D", ctypes.c_int32),
                ("H", ctypes.c_int32), ("F", ctypes.c_int32), ("n_blocks", ctypes.c_int32),
                ("dtype", ctypes.c_int32), ("kind", ctypes.c_int32), ("ln_eps", ctypes.c_float),
                ("idx_shared", ctypes.c_int32)]


class SrBlockParams(ctypes.Structure):
    _fields_ = [(n, ctypes.c_void_p) for n in PARAM_FIELDS]


class SrBlockGrads(ctypes.Structure):
    _fields_ = [(n, ctypes.c_void_p) for n in PARAM_FIELDS]


EDM_PARAM_FIELDS = ("w_film", "b_film", "w_qkv", "b_qkv", "w_o", "b_o",
                    "lnc_w", "lnc_b", "w_q", "b_q", "w_kv", "b_kv", "w_oc", "b_oc", "w_g", "b_g",
                    "ln2_w", "ln2_b", "w_fc1", "b_fc1", "w_fc2", "b_fc2")


class SrEdmBlockParams(ctypes.Structure):
    _fields_ = [(n, ctypes.c_void_p) for n in EDM_PARAM_FIELDS]


class SrEdmBlockGrads(ctypes.Structure):
    _fields_ = [(n, ctypes.c_void_p) for n in EDM_PARAM_FIELDS]


PARAM8_FIELDS = ("ln1_w", "ln1_b", "b_qkv", "b_o", "ln2_w", "ln2_b", "b_fc1", "b_fc2", "w_ada", "b_ada",
                 "w_qkv", "w_o", "w_fc1", "w_fc2", "s_qkv", "s_o", "s_fc1", "s_fc2")


class SrBlockParams8(ctypes.Structure):
    _fields_ = [(n, ctypes.c_void_p) for n in PARAM8_FIELDS]


class SrRotary(ctypes.Structure):
    """sr_rotary_cfg from sequences: one entry per axis, slowest first (freqs: one per pair, or None)."""
    _fields_ = [("axes", ctypes.c_int32), ("grid", ctypes.c_int32 * 3), ("pairs", ctypes.c_int32 * 3),
                ("layout", ctypes.c_int32), ("base", ctypes.c_double), ("origin", ctypes.c_double * 3),
                ("step", ctypes.c_double * 3), ("freqs", ctypes.POINTER(ctypes.c_double))]

    def __init__(self, grid, pairs, layout=SR_ROT_HALVES, base=10000.0, origin=None, step=None, freqs=None):
        n, grid, pairs = len(grid), list(grid), list(pairs)
        origin = [0.0] * n if origin is None else list(origin)
        step = [1.0] * n if step is None else list(step)
        if not 1 <= n <= 3 or any(len(v) != n for v in (pairs, origin, step)):
            raise ValueError("one to three axes, with an entry of pairs, origin and step for each")
        if freqs is not None and len(freqs) != sum(pairs):
            raise ValueError(f"{len(freqs)} frequencies for {sum(pairs)} pairs")
        super().__init__(axes=n, layout=layout, base=base)
        self.grid[:n], self.pairs[:n], self.origin[:n], self.step[:n] = grid, pairs, origin, step
        if freqs is not None:
            self._freqs = (ctypes.c_double * max(len(freqs), 1))(*freqs)
            self.freqs = ctypes.cast(self._freqs, ctypes.POINTER(ctypes.c_double))


class SrDrop(ctypes.Structure):
    _fields_ = [("p", ctypes.c_float), ("group", ctypes.c_int32), ("seed", ctypes.c_uint64), ("step", ctypes.c_uint64),
                ("first_row", ctypes.c_uint64), ("step_dev", ctypes.c_void_p)]


class SrResidualNorm(ctypes.Structure):
    _fields_ = [("B", ctypes.c_int32), ("S", ctypes.c_int32), ("D", ctypes.c_int32), ("dtype", ctypes.c_int32),
                ("stream_dtype", ctypes.c_int32), ("norm", ctypes.c_int32), ("post", ctypes.c_int32),
                ("eps", ctypes.c_float), ("mod_stride", ctypes.c_int64), ("drop", SrDrop)]


RESIDUAL_NORM_FIELDS = ("post_w", "post_b", "res_scale", "pre_w", "pre_b", "gate", "shift", "scale")


class SrResidualNormParams(ctypes.Structure):
    _fields_ = [(n, ctypes.c_void_p) for n in RESIDUAL_NORM_FIELDS]


class SrResidualNormGrads(ctypes.Structure):
    _fields_ = [(n, ctypes.c_void_p) for n in RESIDUAL_NORM_FIELDS]


_lib = None


def lib(path: str = LIB_PATH):
    global _lib
    if _lib is not None:
        return _lib
    if not os.path.exists(path):
        raise SrLibraryMissing(f"{path} is not built; run `python -m paper_2607_02829_amd.build`")
    try:   # torch brings a HIP runtime of its own, which has to be the process's only one: libsr then binds to it
        import torch  # noqa: F401
    except ImportError:
        pass
    L = ctypes.CDLL(path)
    P = ctypes.c_void_p
    I32, I64, U64, SZ = ctypes.c_int32, ctypes.c_int64, ctypes.c_uint64, ctypes.c_size_t
    CP = ctypes.POINTER(SrConfig)
    sig = {
        "sr_last_error": ([], ctypes.c_char_p),
        "sr_version": ([], ctypes.c_char_p),
        "sr_workspace_bytes": ([CP, I32, ctypes.POINTER(SZ), ctypes.POINTER(SZ)], I32),
        "sr_select_scratch_bytes": ([CP, I32, ctypes.POINTER(SZ)], I32),
        "sr_select_indices": ([CP, I32, I32, U64, U64, P, P, P, P, SZ, P], I32),
        "sr_select_indices_noalloc": ([CP, I32, I32, U64, U64, P, P, P, P], I32),
        "sr_gather": ([CP, I32, P, P, P, P], I32),
        "sr_scatter_delta": ([CP, I32, P, P, P, P, P], I32),
        "sr_sparse_blocks_fwd": ([CP, I32, P, P, P, P, P, SZ, P, SZ, P], I32),
        "sr_sparse_blocks_bwd": ([CP, I32, P, P, P, SZ, P, P, P, P, P, SZ, P], I32),
        "sr_dense_blocks_fwd": ([CP, P, P, P, P, P, SZ, P, SZ, P], I32),
        "sr_dense_blocks_bwd": ([CP, P, P, P, SZ, P, P, P, P, P, SZ, P], I32),
        "sr_validate_indices": ([CP, I32, P, P, P], I32),
        "sr_attention_colsums": ([CP, I32, P, SZ, I32, P, P], I32),
        "sr_routed_blocks_fwd": ([CP, I32, P, P, P, P, P, SZ, P], I32),
        "sr_cross_attention_fwd": ([CP, I32, I32, P, P, P, P, P], I32),
        "sr_cross_attention_bwd": ([CP, I32, I32, P, P, P, P, P, P, P, P, P], I32),
        "sr_routed_blocks_bwd": ([CP, I32, P, P, P, P, SZ, P, P, P, P, SZ, P], I32),
        "sr_select_topk_scores": ([CP, I32, P, I32, P, P], I32),
        "sr_edm_workspace_bytes": ([CP, I32, ctypes.POINTER(SZ), ctypes.POINTER(SZ)], I32),
        "sr_edm_blocks_fwd": ([CP, I32, P, P, P, P, P, P, SZ, P], I32),
        "sr_edm_blocks_bwd": ([CP, I32, P, P, P, P, SZ, P, P, P, P, P, P, SZ, P], I32),
        "sr_quantize8": ([I32, I32, I32, I32, P, P, P, P], I32),
        "sr_dequantize8": ([I32, I32, I32, I32, P, P, P, P], I32),
        "sr_linear8": ([I32, I32, I32, I32, I32, P, P, P, P, P, P, P], I32),
        "sr_weight_grad8_scratch_bytes": ([I32, I32, I32, I32, ctypes.POINTER(SZ)], I32),
        "sr_weight_grad8": ([I32, I32, I32, I32, P, P, P, P, P, P, SZ, P], I32),
        "sr_blocks8_scratch_bytes": ([CP, I32, ctypes.POINTER(SZ)], I32),
        "sr_blocks8_fwd": ([CP, I32, P, P, P, P, P, SZ, P], I32),
        "sr_rotary": ([P, I32, I32, I32, I32, I32, I32, P, I64, P, I32, P, I64, P], I32),
        "sr_dropout": ([P, I32, I32, I32, P, P, P, P], I32),
        "sr_residual_norm_fwd": ([P, P, P, P, P, P, P, P, P, P], I32),
        "sr_residual_norm_scratch_bytes": ([P, ctypes.POINTER(SZ)], I32),
        "sr_residual_norm_bwd": ([P, P, P, P, P, P, P, P, P, P, P, SZ, P], I32),
        "sr_quantize_f8": ([I32, I32, I32, I32, P, I64, P, P, P, P, P], I32),
        "sr_linear_f8_scratch_bytes": ([I32, I32, I32, ctypes.POINTER(SZ)], I32),
        "sr_linear_f8": ([I32, I32, I32, I32, I32, P, P, P, P, P, P, P, SZ, P], I32),
        "sr_profile_start": ([ctypes.c_char_p], I32),
        "sr_profile_stop": ([ctypes.c_char_p, SZ, ctypes.POINTER(SZ)], I32),
        "sr_probe_mfma_rate": ([P, ctypes.POINTER(ctypes.c_double), P], I32),
    }
    for name, (args, res) in sig.items():
        f = getattr(L, name)
        f.argtypes = args
        f.restype = res
    _lib = L
    return L


def _p(t):
    """torch tensor -> data_ptr; (address, nbytes) -> address; int -> int; None -> NULL."""
    if t is None:
        return None
    if isinstance(t, int):
        return t
    if isinstance(t, tuple):
        return t[0]
    return t.data_ptr()


def _nbytes(t):
    """Size in bytes of a buffer argument (0 for NULL or a bare address)."""
    if t is None or isinstance(t, int):
        return 0
    if isinstance(t, tuple):
        return t[1]
    return t.numel() * t.element_size()


_raw_stream = None   # address of the current device's current torch stream


def _stream(stream):
    if stream is not None:
        return stream if isinstance(stream, int) else stream.cuda_stream
    global _raw_stream
    if _raw_stream is None:
        import torch
        torch.cuda.current_device()   # initialises the device on first use
        get_device, get_stream = torch._C._cuda_getDevice, torch._C._cuda_getCurrentRawStream
        # the address alone: building the Stream object of torch.cuda.current_stream() costs 2.6 us a call
        _raw_stream = lambda: get_stream(get_device())  # noqa: E731
    return _raw_stream()


def _check(status: int):
    if status != SR_OK:
        raise SrError(status, lib().sr_last_error().decode())


def sr_version() -> str:
    return lib().sr_version().decode()


def sr_last_error() -> str:
    return lib().sr_last_error().decode()


def sr_workspace_bytes(cfg: SrConfig, S: int) -> tuple[int, int]:
    a, b = ctypes.c_size_t(), ctypes.c_size_t()
    _check(lib().sr_workspace_bytes(ctypes.byref(cfg), S, ctypes.byref(a), ctypes.byref(b)))
    return a.value, b.value


def sr_select_scratch_bytes(cfg: SrConfig, select_kind: int) -> int:
    a = ctypes.c_size_t()
    _check(lib().sr_select_scratch_bytes(ctypes.byref(cfg), select_kind, ctypes.byref(a)))
    return a.value


def sr_select_indices(cfg, K, select_kind, seed, step, x_t, x_prev, idx, scratch=None, stream=None):
    _check(lib().sr_select_indices(ctypes.byref(cfg), K, select_kind, seed, step, _p(x_t), _p(x_prev),
                                   _p(idx), _p(scratch), _nbytes(scratch), _stream(stream)))


def sr_select_indices_noalloc(cfg, K, select_kind, seed, step, x_t, x_prev, idx, stream=None):
    _check(lib().sr_select_indices_noalloc(ctypes.byref(cfg), K, select_kind, seed, step, _p(x_t), _p(x_prev),
                                           _p(idx), _stream(stream)))


SR_SELECT_NOALLOC_MAX_TOKENS = 1 << 20


def sr_gather(cfg, K, x, idx, h0, stream=None):
    _check(lib().sr_gather(ctypes.byref(cfg), K, _p(x), _p(idx), _p(h0), _stream(stream)))


def sr_scatter_delta(cfg, K, x, h, h0, idx, stream=None):
    _check(lib().sr_scatter_delta(ctypes.byref(cfg), K, _p(x), _p(h), _p(h0), _p(idx), _stream(stream)))


def sr_sparse_blocks_fwd(cfg, S, params, cond, h_in, h_out, saved, scratch=None, stream=None):
    _check(lib().sr_sparse_blocks_fwd(ctypes.byref(cfg), S, params, _p(cond), _p(h_in), _p(h_out),
                                      _p(saved), _nbytes(saved), _p(scratch), _nbytes(scratch),
                                      _stream(stream)))


def sr_sparse_blocks_bwd(cfg, S, params, cond, saved, dh_out, dh_in, grads, dcond, scratch, stream=None):
    _check(lib().sr_sparse_blocks_bwd(ctypes.byref(cfg), S, params, _p(cond), _p(saved), _nbytes(saved),
                                      _p(dh_out), _p(dh_in), grads, _p(dcond), _p(scratch),
                                      _nbytes(scratch), _stream(stream)))


def sr_dense_blocks_fwd(cfg, params, cond, x_in, x_out, saved, scratch=None, stream=None):
    _check(lib().sr_dense_blocks_fwd(ctypes.byref(cfg), params, _p(cond), _p(x_in), _p(x_out), _p(saved),
                                     _nbytes(saved), _p(scratch), _nbytes(scratch), _stream(stream)))


def sr_dense_blocks_bwd(cfg, params, cond, saved, dx_out, dx_in, grads, dcond, scratch, stream=None):
    _check(lib().sr_dense_blocks_bwd(ctypes.byref(cfg), params, _p(cond), _p(saved), _nbytes(saved),
                                     _p(dx_out), _p(dx_in), grads, _p(dcond), _p(scratch), _nbytes(scratch),
                                     _stream(stream)))


def sr_validate_indices(cfg, K, idx, ok_dev, stream=None):
    _check(lib().sr_validate_indices(ctypes.byref(cfg), K, _p(idx), _p(ok_dev), _stream(stream)))


def sr_routed_blocks_fwd(cfg, K, idx, params, cond, x, saved, stream=None):
    _check(lib().sr_routed_blocks_fwd(ctypes.byref(cfg), K, _p(idx), params, _p(cond), _p(x), _p(saved),
                                      _nbytes(saved), _stream(stream)))


def sr_routed_blocks_bwd(cfg, K, idx, params, cond, saved, g, grads, dcond, scratch, stream=None):
    _check(lib().sr_routed_blocks_bwd(ctypes.byref(cfg), K, _p(idx), params, _p(cond), _p(saved), _nbytes(saved),
                                      _p(g), grads, _p(dcond), _p(scratch), _nbytes(scratch), _stream(stream)))


def sr_cross_attention_fwd(cfg, Sq, Skv, q, kv, O, lse, stream=None):
    _check(lib().sr_cross_attention_fwd(ctypes.byref(cfg), Sq, Skv, _p(q), _p(kv), _p(O), _p(lse), _stream(stream)))


def sr_cross_attention_bwd(cfg, Sq, Skv, q, kv, O, dO, lse, dq, dkv, delta, stream=None):
    _check(lib().sr_cross_attention_bwd(ctypes.byref(cfg), Sq, Skv, _p(q), _p(kv), _p(O), _p(dO), _p(lse), _p(dq),
                                        _p(dkv), _p(delta), _stream(stream)))


def sr_edm_workspace_bytes(cfg: SrConfig, S: int) -> tuple[int, int]:
    a, b = ctypes.c_size_t(), ctypes.c_size_t()
    _check(lib().sr_edm_workspace_bytes(ctypes.byref(cfg), S, ctypes.byref(a), ctypes.byref(b)))
    return a.value, b.value


def sr_edm_blocks_fwd(cfg, S, params, e, zc, h_in, h_out, saved, stream=None):
    _check(lib().sr_edm_blocks_fwd(ctypes.byref(cfg), S, params, _p(e), _p(zc), _p(h_in), _p(h_out), _p(saved),
                                   _nbytes(saved), _stream(stream)))


def sr_edm_blocks_bwd(cfg, S, params, e, zc, saved, dh_out, dh_in, grads, dzc, de, scratch, stream=None):
    _check(lib().sr_edm_blocks_bwd(ctypes.byref(cfg), S, params, _p(e), _p(zc), _p(saved), _nbytes(saved),
                                   _p(dh_out), _p(dh_in), grads, _p(dzc), _p(de), _p(scratch), _nbytes(scratch),
                                   _stream(stream)))


def sr_attention_colsums(cfg, S, saved, block, colsum, stream=None):
    _check(lib().sr_attention_colsums(ctypes.byref(cfg), S, _p(saved), _nbytes(saved), block, _p(colsum),
                                      _stream(stream)))


def sr_select_topk_scores(cfg, K, planes, parts, idx, stream=None):
    _check(lib().sr_select_topk_scores(ctypes.byref(cfg), K, _p(planes), parts, _p(idx), _stream(stream)))


def sr_quantize8(q8_kind, dtype, M, N, x, q, scale, stream=None):
    _check(lib().sr_quantize8(q8_kind, dtype, M, N, _p(x), _p(q), _p(scale), _stream(stream)))


def sr_dequantize8(q8_kind, dtype, M, N, q, scale, x, stream=None):
    _check(lib().sr_dequantize8(q8_kind, dtype, M, N, _p(q), _p(scale), _p(x), _stream(stream)))


def sr_linear8(dtype, act, M, N, K, xq, xs, wq, ws, bias, y, stream=None):
    _check(lib().sr_linear8(dtype, act, M, N, K, _p(xq), _p(xs), _p(wq), _p(ws), _p(bias), _p(y), _stream(stream)))


def sr_weight_grad8_scratch_bytes(dtype: int, M: int, N: int, K: int) -> int:
    a = ctypes.c_size_t()
    _check(lib().sr_weight_grad8_scratch_bytes(dtype, M, N, K, ctypes.byref(a)))
    return a.value


def sr_weight_grad8(dtype, M, N, K, dy, xq, xe, dw, db, scratch, stream=None):
    _check(lib().sr_weight_grad8(dtype, M, N, K, _p(dy), _p(xq), _p(xe), _p(dw), _p(db), _p(scratch),
                                 _nbytes(scratch), _stream(stream)))


def sr_blocks8_scratch_bytes(cfg: SrConfig, S: int) -> int:
    a = ctypes.c_size_t()
    _check(lib().sr_blocks8_scratch_bytes(ctypes.byref(cfg), S, ctypes.byref(a)))
    return a.value


def sr_blocks8_fwd(cfg, S, params, cond, h_in, h_out, scratch, stream=None):
    _check(lib().sr_blocks8_fwd(ctypes.byref(cfg), S, params, _p(cond), _p(h_in), _p(h_out), _p(scratch),
                                _nbytes(scratch), _stream(stream)))


def sr_rotary(rot, inverse, dtype, B, S, heads, head_dim, x, ldx, idx, idx_shared, y, ldy, stream=None):
    _check(lib().sr_rotary(ctypes.byref(rot), inverse, dtype, B, S, heads, head_dim, _p(x), ldx, _p(idx), idx_shared,
                           _p(y), ldy, _stream(stream)))


def sr_dropout(drop, dtype, M, N, x, resid, y, stream=None):
    _check(lib().sr_dropout(ctypes.byref(drop), dtype, M, N, _p(x), _p(resid), _p(y), _stream(stream)))


def _residual_norm_struct(cls, tensors):
    s = cls(**{k: _p(t) for k, t in tensors.items()})
    s._tensors = tensors   # alive as long as the struct that points at them
    return s


def residual_norm_params(**tensors):
    """sr_residual_norm_params of tensors (post_w, post_b, res_scale, pre_w, pre_b, gate, shift, scale; what is left
    out stays out of the formula)."""
    return _residual_norm_struct(SrResidualNormParams, tensors)


def residual_norm_grads(**tensors):
    """sr_residual_norm_grads of fp32 tensors under the parameters' names."""
    return _residual_norm_struct(SrResidualNormGrads, tensors)


def sr_residual_norm_fwd(cfg, params, x, y, x1, u, uq=None, ue=None, stats=None, stream=None):
    _check(lib().sr_residual_norm_fwd(ctypes.byref(cfg), ctypes.byref(params), _p(x), _p(y), _p(x1), _p(u), _p(uq),
                                      _p(ue), _p(stats), _stream(stream)))


def sr_residual_norm_scratch_bytes(cfg) -> int:
    a = ctypes.c_size_t()
    _check(lib().sr_residual_norm_scratch_bytes(ctypes.byref(cfg), ctypes.byref(a)))
    return a.value


def sr_residual_norm_bwd(cfg, params, x1, y, stats, dx1, du, dx, dy, grads, scratch, stream=None):
    _check(lib().sr_residual_norm_bwd(ctypes.byref(cfg), ctypes.byref(params), _p(x1), _p(y), _p(stats), _p(dx1),
                                      _p(du), _p(dx), _p(dy), ctypes.byref(grads), _p(scratch), _nbytes(scratch),
                                      _stream(stream)))


def f8_shapes(rows: int, cols: int):
    """Shapes of the codes and exponents of `rows` rows of `cols` values (sr_quantize_f8)."""
    blocks = (cols + 127) // 128
    return (rows, 128 * blocks), (blocks, (rows + 15) // 16 * 16)


def f8_buffers(M, N, rows=True, transposed=False, device="cuda"):
    """(q, e, qt, et) of sr_quantize_f8 for an M x N matrix, as uint8 tensors; None for what is not asked for."""
    import torch
    shapes = (*(f8_shapes(M, N) if rows else (None, None)), *(f8_shapes(N, M) if transposed else (None, None)))
    return tuple(None if s is None else torch.empty(s, dtype=torch.uint8, device=device) for s in shapes)


def sr_quantize_f8(f8_kind, dtype, M, N, x, ldx, q, e, qt=None, et=None, stream=None):
    _check(lib().sr_quantize_f8(f8_kind, dtype, M, N, _p(x), ldx, _p(q), _p(e), _p(qt), _p(et), _stream(stream)))


def sr_linear_f8_scratch_bytes(M: int, N: int, K: int) -> int:
    a = ctypes.c_size_t()
    _check(lib().sr_linear_f8_scratch_bytes(M, N, K, ctypes.byref(a)))
    return a.value


def sr_linear_f8(dtype, act, M, N, K, xq, xe, wq, we, bias, y, scratch=None, stream=None):
    _check(lib().sr_linear_f8(dtype, act, M, N, K, _p(xq), _p(xe), _p(wq), _p(we), _p(bias), _p(y), _p(scratch),
                              _nbytes(scratch), _stream(stream)))


def sr_profile_start(name_filter: str = "") -> None:
    _check(lib().sr_profile_start(name_filter.encode()))


def sr_profile_stop() -> dict[str, dict[str, float]]:
    """Stop recording; returns {name: {launches, ms, flops, bytes}} (totals)."""
    buf = ctypes.create_string_buffer(1 << 20)
    need = ctypes.c_size_t()
    _check(lib().sr_profile_stop(buf, len(buf), ctypes.byref(need)))
    return _parse_profile(buf.value.decode())


def sr_probe_mfma_rate(sink, stream=None) -> float:
    """Sustained dense bf16 MFMA TFLOP/s of the current device (sink: >= 4 bytes of device memory)."""
    out = ctypes.c_double()
    _check(lib().sr_probe_mfma_rate(_p(sink), ctypes.byref(out), _stream(stream)))
    return out.value


def _parse_profile(text: str) -> dict[str, dict[str, float]]:
    out = {}
    for line in text.strip().splitlines():
        name, n, ms, fl, by = line.split()
        out[name] = {"launches": float(n), "ms": float(ms), "flops": float(fl), "bytes": float(by)}
    return out
