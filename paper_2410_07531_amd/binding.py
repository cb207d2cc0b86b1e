"""Thin ctypes binding over librov.so: argument marshalling only.

Every function takes torch tensors (device memory) and streams as plumbing and
forwards raw pointers to the C ABI declared in include/rov.h.  There is no CPU
fallback: if the library is missing or a call fails, an exception is raised.
"""
import ctypes
import os
import struct

HERE = os.path.dirname(os.path.abspath(__file__))
LIB_PATH = os.path.join(HERE, "librov.so")

OK, ERR_INVALID, ERR_UNSUPPORTED, ERR_HIP, ERR_WORKSPACE = 0, -1, -2, -3, -4
F32, BF16, FP8_E4M3 = 0, 1, 2
SCHED_SEQUENTIAL, SCHED_FUSED, SCHED_OVERLAP, SCHED_HYBRID, SCHED_OVERLAP_DEFERRED = 0, 1, 2, 3, 4
MASK_NOT_READY, MASK_READY, MASK_IN_FLIGHT = 0, 1, 2
ROPE_INTERLEAVED, ROPE_HALVES = 0, 1
ROPE_SCALE_NONE, ROPE_SCALE_LINEAR, ROPE_SCALE_PARTS = 0, 1, 2

_ERR_NAMES = {ERR_INVALID: "ROV_ERR_INVALID", ERR_UNSUPPORTED: "ROV_ERR_UNSUPPORTED",
              ERR_HIP: "ROV_ERR_HIP", ERR_WORKSPACE: "ROV_ERR_WORKSPACE"}


class RovError(RuntimeError):
    def __init__(self, code, what):
        self.code = code
        super().__init__("%s failed: %s (%d)" % (what, _ERR_NAMES.get(code, "?"), code))


class GemmDesc(ctypes.Structure):
    _fields_ = [("A", ctypes.c_void_p), ("Bm", ctypes.c_void_p), ("C", ctypes.c_void_p),
                ("M", ctypes.c_int), ("N", ctypes.c_int), ("K", ctypes.c_int),
                ("dtype", ctypes.c_int), ("transB", ctypes.c_int),
                ("scaleA", ctypes.c_float), ("scaleB", ctypes.c_float)]


class AttnDesc(ctypes.Structure):
    _fields_ = [("Q", ctypes.c_void_p), ("K", ctypes.c_void_p), ("V", ctypes.c_void_p),
                ("O", ctypes.c_void_p),
                ("B", ctypes.c_int), ("H", ctypes.c_int), ("Hkv", ctypes.c_int),
                ("S", ctypes.c_int), ("d", ctypes.c_int),
                ("strides", ctypes.c_int64 * 12),
                ("dtype", ctypes.c_int), ("causal", ctypes.c_int), ("p", ctypes.c_float)]


class BlockCfg(ctypes.Structure):
    _fields_ = [("H", ctypes.c_int), ("Hkv", ctypes.c_int), ("d", ctypes.c_int),
                ("hidden", ctypes.c_int), ("ffn", ctypes.c_int), ("dtype", ctypes.c_int),
                ("causal", ctypes.c_int), ("p", ctypes.c_float), ("eps", ctypes.c_float),
                ("rope_theta", ctypes.c_float), ("act_scale", ctypes.c_float * 4)]


class BlockWeights(ctypes.Structure):
    _fields_ = [(n, ctypes.c_void_p) for n in ("norm1", "norm2", "wqkv", "wo", "wg", "wu", "wd")] + \
               [("w_scale", ctypes.c_float * 5)]


class RopeCfg(ctypes.Structure):
    _fields_ = [("layout", ctypes.c_int), ("rot", ctypes.c_int), ("scaling", ctypes.c_int), ("trained_len", ctypes.c_int),
                ("theta", ctypes.c_float), ("factor", ctypes.c_float), ("turns_low", ctypes.c_float),
                ("turns_high", ctypes.c_float), ("magnitude", ctypes.c_float)]


class BlockOpts(ctypes.Structure):
    _fields_ = [("rope", ctypes.POINTER(RopeCfg)), ("positions", ctypes.c_void_p), ("positions_stride", ctypes.c_int64),
                ("post1", ctypes.c_void_p), ("gate1", ctypes.c_void_p), ("post2", ctypes.c_void_p), ("gate2", ctypes.c_void_p),
                ("rows_per_gate", ctypes.c_int64), ("x_scale", ctypes.c_float), ("h_scale", ctypes.c_float)]


# name -> (restype, argtypes); also the list of symbols the header declares
_u64, _i, _f, _p = ctypes.c_uint64, ctypes.c_int, ctypes.c_float, ctypes.c_void_p
_i64 = ctypes.c_int64
SIGNATURES = {
    "rov_last_hip_error": (_i, []),
    "rov_version": (ctypes.c_char_p, []),
    "rov_mask_words": (_u64, [_i, _i, _i]),
    "rov_mask_philox_calls": (_u64, [_i, _i, _i]),
    "rov_philox_raw": (_i, [_u64, _u64, _u64, _i, _p, _p]),
    "rov_dropout_mask_generate": (_i, [_u64, _u64, _i, _i, _i, _f, _p, _p]),
    "rov_dropout_mask_generate_rounds": (_i, [_u64, _u64, _i, _i, _i, _f, _i, _p, _p]),
    "rov_dropout_mask_generate_causal": (_i, [_u64, _u64, _i, _i, _i, _f, _p, _p]),
    "rov_dropout_mask_generate_bits": (_i, [_u64, _u64, _i, _i, _i, _f, _i, _p, _p]),
    "rov_mask_philox_calls_bits": (_u64, [_i, _i, _i, _i]),
    "rov_mask_words_rows": (_u64, [_i, _i, _i, _i, _i]),
    "rov_dropout_mask_generate_rows": (_i, [_u64, _u64, _i, _i, _i, _f, _i, _i, _p, _p]),
    "rov_attention_fwd_dropout_rows": (_i, [_p, _p, _p, _p, _i, _i, _i, _i, _i,
                                            ctypes.POINTER(ctypes.c_int64), _i, _i, _f, _p, _u64, _u64,
                                            _i, _i, _p]),
    "rov_layer_step_chunked": (_i, [ctypes.POINTER(GemmDesc), _i, ctypes.POINTER(AttnDesc), _u64, _u64, _i,
                                    _p, _p, _p]),
    "rov_set_rng_max_workgroups": (_i, [_i]),
    "rov_set_gemm_tile_cols": (_i, [_i]),
    "rov_gemm_tile_cols": (_i, [_i, _i]),
    "rov_gemm_tile": (_i, [_i, _i, _i, _i, _i, ctypes.POINTER(ctypes.c_int)]),
    "rov_gemm_swiglu_tile_cols": (_i, [_i, _i, _i, _i]),
    "rov_attention_key_parts": (_i, [_i, _i, _i, _i, _i, _i]),
    "rov_attention_tile_rows": (_i, [_i, _i, _i, _i, _i, _i]),
    "rov_overlap_mask_chunks": (ctypes.c_int64, [ctypes.c_double, _i, _i, _i, _i, _i, _i]),
    "rov_set_rng_overlap_workgroups_per_cu": (_i, [_i]),
    "rov_trace_enable": (_i, [_i]),
    "rov_trace_read": (_i, [ctypes.POINTER(ctypes.c_int), ctypes.POINTER(ctypes.c_float), _i,
                            ctypes.POINTER(ctypes.c_int)]),
    "rov_valu_probe": (_i, [_i, _i, _i, _p, _p]),
    "rov_gemm": (_i, [_p, _p, _p, _i, _i, _i, _i, _i, _f, _f, _p]),
    "rov_gemm_swiglu": (_i, [_p, _p, _p, _p, _i, _i, _i, _p]),
    "rov_gemm_swiglu_fp8": (_i, [_p, _p, _p, _p, _i, _i, _i, _f, _f, _f, _f, _p]),
    "rov_gemm_rng_fused": (_i, [_p, _p, _p, _i, _i, _i, _u64, _u64, _i, _i, _i, _f, _p, _p]),
    "rov_attention_fwd_dropout": (_i, [_p, _p, _p, _p, _i, _i, _i, _i, _i,
                                       ctypes.POINTER(ctypes.c_int64), _i, _i, _f, _p, _u64, _u64, _p]),
    "rov_layer_step": (_i, [_i, ctypes.POINTER(GemmDesc), _i, ctypes.POINTER(AttnDesc), _u64, _u64,
                            _p, _p, _p]),
    "rov_layer_step_rounds": (_i, [_i, ctypes.POINTER(GemmDesc), _i, ctypes.POINTER(AttnDesc), _u64, _u64,
                                   _i, _p, _p, _p]),
    "rov_layer_step_bits": (_i, [_i, ctypes.POINTER(GemmDesc), _i, ctypes.POINTER(AttnDesc), _u64, _u64,
                                 _i, _p, _p, _p]),
    "rov_attention_fwd_dropout_bits": (_i, [_p, _p, _p, _p, _i, _i, _i, _i, _i,
                                            ctypes.POINTER(ctypes.c_int64), _i, _i, _f, _p, _u64, _u64, _i, _p]),
    "rov_attention_fwd_dropout_rounds": (_i, [_p, _p, _p, _p, _i, _i, _i, _i, _i,
                                              ctypes.POINTER(ctypes.c_int64), _i, _i, _f, _p, _u64, _u64, _i,
                                              _p]),
    "rov_block_workspace_bytes": (ctypes.c_size_t, [ctypes.POINTER(BlockCfg), _i, _i, _i]),
    "rov_block_hybrid_mask_rows": (_i, [ctypes.POINTER(BlockCfg), _i, _i]),
    "rov_set_block_hybrid_mask_rows": (_i, [_i]),
    "rov_block_forward": (_i, [ctypes.POINTER(BlockWeights), _p, _p, _i, _i, ctypes.POINTER(BlockCfg),
                               _i, _u64, _u64, _i, _p, _p, _p, ctypes.c_size_t, _p, _p]),
    "rov_block_forward_opts": (_i, [ctypes.POINTER(BlockWeights), ctypes.POINTER(BlockOpts), _p, _p, _i, _i, ctypes.POINTER(BlockCfg),
                                    _i, _u64, _u64, _i, _p, _p, _p, ctypes.c_size_t, _p, _p]),
    "rov_mask_finish": (_i, [_p, _p]),
    "rov_block_static_scratch_bytes": (ctypes.c_size_t, []),
    "rov_block_forward_static": (_i, [ctypes.POINTER(BlockWeights), _p, _p, _i, _i, ctypes.POINTER(BlockCfg),
                                      _i, _u64, _u64, _i, _p, _p, _p, _p]),
    "rov_rope": (_i, [ctypes.POINTER(RopeCfg), _p, _p, _p, _p, _i, _i, _i, _i, _i, _p, _i, _p, _i64, _i, _p]),
    "rov_norm_residual": (_i, [_p] * 7 + [_i64, _i, _p, _i64, _i, _f, _f, _f, _f, _p]),
    "rov_norm_residual_bwd_workspace_bytes": (ctypes.c_size_t, [_i64, _i, _i64, _i]),
    "rov_norm_residual_bwd": (_i, [_p] * 12 + [_i64, _i, _p, _i64, _i, _f, _f, _f, _p, ctypes.c_size_t, _p]),
    "rov_linear_xent_workspace_bytes": (ctypes.c_size_t, [_i] * 6),
    "rov_linear_xent_walks": (_i, [_i] * 5),
    "rov_linear_xent": (_i, [_p, _p, _p, _i, _i, _i, _i64, _i64, _i, _f, _i64, _p, _p, _i, _p, ctypes.c_size_t, _p]),
    "rov_linear_xent_bwd": (_i, [_p] * 6 + [_i, _i, _i, _i64, _i64, _i, _f, _i64, _p, _p, _i64, _i64, _i, _p, ctypes.c_size_t, _p]),
}

_lib = None


def load():
    """Load librov.so (after torch, so that both share one HIP runtime)."""
    global _lib
    if _lib is not None:
        return _lib
    if not os.path.exists(LIB_PATH):
        raise RuntimeError("librov.so is not built: run `python -c 'import __graft_entry__ as g; g.build()'`")
    try:
        import torch  # noqa: F401  (loads libamdhip64 first)
    except ImportError:
        pass
    L = ctypes.CDLL(LIB_PATH)
    for name, (res, args) in SIGNATURES.items():
        fn = getattr(L, name)
        fn.restype = res
        fn.argtypes = args
    _lib = L
    return L


def _check(code, what):
    if code != OK:
        raise RovError(code, what)


# Small calls are bound by this file: pointers and handles go to ctypes as plain integers (its argtypes turn them into
# void*), and the current stream is asked for its handle without building a Stream object (a mask call 7.6 -> 4.5 us, attention 11.1 -> 6.3).
_raw_stream = None


def _stream_ptr(stream):
    global _raw_stream
    if stream is not None:
        return stream.cuda_stream
    if _raw_stream is None:
        import torch
        torch.cuda.current_stream()     # initialises the device
        handle, device = getattr(torch._C, "_cuda_getCurrentRawStream", None), getattr(torch._C, "_cuda_getDevice", None)
        if handle is not None and device is not None:
            _raw_stream = lambda: handle(device())
        else:
            _raw_stream = lambda: torch.cuda.current_stream().cuda_stream
    return _raw_stream()


_dtype_codes = {}


def _dtype_code(t):
    code = _dtype_codes.get(t.dtype)
    if code is not None:
        return code
    import torch
    _dtype_codes.update({torch.float32: F32, torch.bfloat16: BF16, torch.float8_e4m3fn: FP8_E4M3, torch.uint8: FP8_E4M3})
    if t.dtype not in _dtype_codes:
        raise TypeError("unsupported dtype %s" % t.dtype)
    return _dtype_codes[t.dtype]


def mask_words(B, H, S):
    return int(load().rov_mask_words(B, H, S))


def mask_philox_calls(B, H, S):
    return int(load().rov_mask_philox_calls(B, H, S))


def mask_philox_calls_bits(B, H, S, bits):
    return int(load().rov_mask_philox_calls_bits(B, H, S, int(bits)))


def set_rng_max_workgroups(n):
    return int(load().rov_set_rng_max_workgroups(int(n)))


def set_gemm_tile_cols(cols):
    r = int(load().rov_set_gemm_tile_cols(int(cols)))
    if r < 0:
        raise RovError(r, "rov_set_gemm_tile_cols")
    return r


def gemm_tile_cols(M, N):
    return int(load().rov_gemm_tile_cols(int(M), int(N)))


GEMM_256_ROWS, GEMM_SMALL_TILES, GEMM_ANY_SHAPE = 0, 1, 2


def gemm_tile(M, N, K, dtype, transB=True):
    """(kernel, rows, columns, parts of k, bytes that rows start on) of the product rov_gemm would run."""
    t = (ctypes.c_int * 4)()
    kernel = load().rov_gemm_tile(M, N, K, dtype, int(bool(transB)), t)
    if kernel < 0:
        raise RovError(kernel, "rov_gemm_tile")
    return (kernel,) + tuple(t)


def gemm_swiglu_tile_cols(M, N, K, dtype):
    r = load().rov_gemm_swiglu_tile_cols(M, N, K, dtype)
    if r < 0:
        raise RovError(r, "rov_gemm_swiglu_tile_cols")
    return r


def attention_key_parts(B, H, S, d, dtype, causal):
    r = load().rov_attention_key_parts(B, H, S, d, dtype, int(bool(causal)))
    if r < 0:
        raise RovError(r, "rov_attention_key_parts")
    return r


def attention_tile_rows(B, H, S, d, dtype, causal):
    r = load().rov_attention_tile_rows(B, H, S, d, dtype, int(bool(causal)))
    if r < 0:
        raise RovError(r, "rov_attention_tile_rows")
    return r


def overlap_mask_chunks(gemm_flop, dtype, B, H, S, causal=False, rounds=10):
    """Chunks of the mask that the grid beside the GEMMs makes; -1: a work queue."""
    r = load().rov_overlap_mask_chunks(float(gemm_flop), dtype, B, H, S, int(bool(causal)), rounds)
    if r < -1:
        raise RovError(ERR_INVALID, "rov_overlap_mask_chunks")
    return r


def set_rng_overlap_workgroups_per_cu(n):
    return int(load().rov_set_rng_overlap_workgroups_per_cu(int(n)))


def philox_raw(seed, first_counter, ncalls, rounds=10, out=None, stream=None):
    """int32-viewed uint32 [ncalls, 4] tensor of raw Philox words (test hook)."""
    if out is None:
        import torch
        out = torch.empty((int(ncalls), 4), dtype=torch.int32, device="cuda")
    _check(load().rov_philox_raw(seed & (2**64 - 1), first_counter & (2**64 - 1), int(ncalls), int(rounds),
                                 out.data_ptr(), _stream_ptr(stream)), "rov_philox_raw")
    return out


def mask_shape(B, H, S):
    """Shape of the keep-mask word array: [B, H, T, T, 16] with T = ceil(S/32)."""
    T = (S + 31) // 32
    return (B, H, T, T, 16)


def dropout_mask_generate_causal(seed, offset, B, H, S, p, out, stream=None):
    """Writes only the tiles causal attention reads (plus their chunk neighbours) into `out`."""
    _check(load().rov_dropout_mask_generate_causal(seed & (2**64 - 1), offset & (2**64 - 1), B, H, S, p,
                                                   out.data_ptr(), _stream_ptr(stream)),
           "rov_dropout_mask_generate_causal")
    return out


def dropout_mask_generate(seed, offset, B, H, S, p, out=None, rounds=None, stream=None):
    """Keep-mask words as an int64 tensor of shape mask_shape(B, H, S) (bit patterns of uint64)."""
    if out is None:
        import torch
        out = torch.empty(mask_shape(B, H, S), dtype=torch.int64, device="cuda")
    L = load()
    if rounds is None:
        rc = L.rov_dropout_mask_generate(seed & (2**64 - 1), offset & (2**64 - 1), B, H, S, p,
                                         out.data_ptr(), _stream_ptr(stream))
    else:
        rc = L.rov_dropout_mask_generate_rounds(seed & (2**64 - 1), offset & (2**64 - 1), B, H, S, p, int(rounds),
                                                out.data_ptr(), _stream_ptr(stream))
    _check(rc, "rov_dropout_mask_generate")
    return out


def dropout_mask_generate_bits(seed, offset, B, H, S, p, bits, out=None, stream=None):
    """Keep-mask drawn with `bits` (8, 16 or 32) random bits per element; same shape and layout."""
    if out is None:
        import torch
        out = torch.empty(mask_shape(B, H, S), dtype=torch.int64, device="cuda")
    _check(load().rov_dropout_mask_generate_bits(seed & (2**64 - 1), offset & (2**64 - 1), B, H, S, p, int(bits),
                                                 out.data_ptr(), _stream_ptr(stream)),
           "rov_dropout_mask_generate_bits")
    return out


def gemm(A, Bm, C=None, transB=True, scaleA=1.0, scaleB=1.0, stream=None):
    """C = scaleA*scaleB * A @ (Bm^T if transB else Bm)."""
    M, K = A.shape
    N = Bm.shape[0] if transB else Bm.shape[1]
    code = _dtype_code(A)
    if C is None:
        import torch
        C = torch.empty((M, N), dtype=torch.float32 if code == F32 else torch.bfloat16, device=A.device)
    _check(load().rov_gemm(A.data_ptr(), Bm.data_ptr(),
                           C.data_ptr(), M, N, K, code, int(bool(transB)),
                           float(scaleA), float(scaleB), _stream_ptr(stream)), "rov_gemm")
    return C


def gemm_swiglu(A, Wg, Wu, C=None, stream=None):
    """C = silu(A @ Wg^T) * (A @ Wu^T), bf16."""
    M, K = A.shape
    N = Wg.shape[0]
    if C is None:
        import torch
        C = torch.empty((M, N), dtype=torch.bfloat16, device=A.device)
    _check(load().rov_gemm_swiglu(A.data_ptr(), Wg.data_ptr(),
                                  Wu.data_ptr(), C.data_ptr(), M, N, K,
                                  _stream_ptr(stream)), "rov_gemm_swiglu")
    return C


def gemm_swiglu_fp8(A, Wg, Wu, scaleA, scaleWg, scaleWu, scaleC, C=None, stream=None):
    """C (e4m3 bytes) = e4m3(silu(sA sWg A Wg^T) * (sA sWu A Wu^T) / scaleC); A, Wg, Wu e4m3 bytes."""
    M, K = A.shape
    N = Wg.shape[0]
    if C is None:
        import torch
        C = torch.empty((M, N), dtype=torch.uint8, device=A.device)
    _check(load().rov_gemm_swiglu_fp8(A.data_ptr(), Wg.data_ptr(),
                                      Wu.data_ptr(), C.data_ptr(), M, N, K,
                                      float(scaleA), float(scaleWg), float(scaleWu), float(scaleC),
                                      _stream_ptr(stream)), "rov_gemm_swiglu_fp8")
    return C


def gemm_rng_fused(A, Bm, seed, offset, B, H, S, p, C=None, mask=None, stream=None):
    """C = A @ Bm^T (bf16) and the keep-mask of (seed, offset, B, H, S, p) from one wave-specialised kernel."""
    import torch
    M, K = A.shape
    N = Bm.shape[0]
    if C is None:
        C = torch.empty((M, N), dtype=torch.bfloat16, device=A.device)
    if mask is None:
        mask = torch.empty(mask_shape(B, H, S), dtype=torch.int64, device=A.device)
    _check(load().rov_gemm_rng_fused(A.data_ptr(), Bm.data_ptr(),
                                     C.data_ptr(), M, N, K, ctypes.c_uint64(seed),
                                     ctypes.c_uint64(offset), B, H, S, float(p), mask.data_ptr(),
                                     _stream_ptr(stream)), "rov_gemm_rng_fused")
    return C, mask


_I64x12 = ctypes.c_int64 * 12


def _strides12(Q, K, V, O):
    q, k, v, o = Q.stride(), K.stride(), V.stride(), O.stride()
    assert q[3] == 1 and k[3] == 1 and v[3] == 1 and o[3] == 1, "head dimension must be contiguous"
    return _I64x12(q[0], q[1], q[2], k[0], k[1], k[2], v[0], v[1], v[2], o[0], o[1], o[2])


def attention_fwd_dropout(Q, K, V, p, mask=None, seed=0, offset=0, causal=False, O=None, stream=None,
                          rounds=None, bits=None):
    """Q [B,S,H,d], K/V [B,S,Hkv,d] -> O [B,S,H,d]; mask=None with p>0 selects the fused variant
    (rounds: its Philox round count, 3/5/7/10, or bits: its random bits per element, 8/16/32;
    None = the 10-round, 32-bit entry point)."""
    B, S, H, d = Q.shape
    Hkv = K.shape[2]
    if O is None:
        import torch
        O = torch.empty_like(Q)
    strides = _strides12(Q, K, V, O)
    mptr = mask.data_ptr() if mask is not None else None
    if bits is not None:
        _check(load().rov_attention_fwd_dropout_bits(
            Q.data_ptr(), K.data_ptr(), V.data_ptr(),
            O.data_ptr(), B, H, Hkv, S, d, strides, _dtype_code(Q), int(bool(causal)),
            float(p), mptr, seed & (2**64 - 1), offset & (2**64 - 1), int(bits), _stream_ptr(stream)),
            "rov_attention_fwd_dropout_bits")
        return O
    if rounds is not None:
        _check(load().rov_attention_fwd_dropout_rounds(
            Q.data_ptr(), K.data_ptr(), V.data_ptr(),
            O.data_ptr(), B, H, Hkv, S, d, strides, _dtype_code(Q), int(bool(causal)),
            float(p), mptr, seed & (2**64 - 1), offset & (2**64 - 1), int(rounds), _stream_ptr(stream)),
            "rov_attention_fwd_dropout_rounds")
        return O
    _check(load().rov_attention_fwd_dropout(
        Q.data_ptr(), K.data_ptr(), V.data_ptr(),
        O.data_ptr(), B, H, Hkv, S, d, strides, _dtype_code(Q), int(bool(causal)), float(p),
        mptr, seed & (2**64 - 1), offset & (2**64 - 1), _stream_ptr(stream)), "rov_attention_fwd_dropout")
    return O


def mask_words_rows(B, H, S, q_begin, q_rows):
    return int(load().rov_mask_words_rows(B, H, S, int(q_begin), int(q_rows)))


def dropout_mask_generate_rows(seed, offset, B, H, S, p, q_begin, q_rows, out=None, stream=None):
    """Tile rows of query rows [q_begin, q_begin + q_rows): int64 tensor [B, H, nqt, T, 16]."""
    if out is None:
        import torch
        T = (S + 31) // 32
        nqt = (min(q_begin + q_rows, S) - q_begin + 31) // 32
        out = torch.empty((B, H, nqt, T, 16), dtype=torch.int64, device="cuda")
    _check(load().rov_dropout_mask_generate_rows(seed & (2**64 - 1), offset & (2**64 - 1), B, H, S, p,
                                                 int(q_begin), int(q_rows), out.data_ptr(),
                                                 _stream_ptr(stream)), "rov_dropout_mask_generate_rows")
    return out


def attention_fwd_dropout_rows(Q, K, V, p, q_begin, q_rows, O, mask_rows=None, seed=0, offset=0, causal=False,
                               stream=None):
    """Computes query rows [q_begin, q_begin + q_rows) of O in place; mask_rows holds those tile rows."""
    B, S, H, d = Q.shape
    Hkv = K.shape[2]
    strides = _strides12(Q, K, V, O)
    mptr = mask_rows.data_ptr() if mask_rows is not None else None
    _check(load().rov_attention_fwd_dropout_rows(
        Q.data_ptr(), K.data_ptr(), V.data_ptr(),
        O.data_ptr(), B, H, Hkv, S, d, strides, _dtype_code(Q), int(bool(causal)), float(p),
        mptr, seed & (2**64 - 1), offset & (2**64 - 1), int(q_begin), int(q_rows), _stream_ptr(stream)),
        "rov_attention_fwd_dropout_rows")
    return O


def layer_step_chunked(gemm_descs, attn_desc, seed, offset, q_chunk_rows, mask_ring, main_stream, side_stream):
    arr = (GemmDesc * len(gemm_descs))(*gemm_descs)
    _check(load().rov_layer_step_chunked(arr, len(gemm_descs), ctypes.byref(attn_desc), seed & (2**64 - 1),
                                         offset & (2**64 - 1), int(q_chunk_rows),
                                         mask_ring.data_ptr(), _stream_ptr(main_stream),
                                         _stream_ptr(side_stream)), "rov_layer_step_chunked")


def make_gemm_desc(A, Bm, C, transB=True, scaleA=1.0, scaleB=1.0):
    M, K = A.shape
    N = Bm.shape[0] if transB else Bm.shape[1]
    return GemmDesc(A.data_ptr(), Bm.data_ptr(), C.data_ptr(), M, N, K, _dtype_code(A), int(bool(transB)),
                    float(scaleA), float(scaleB))


def gemm_desc(desc, stream=None):
    """Runs the GEMM a GemmDesc describes."""
    _check(load().rov_gemm(desc.A, desc.Bm, desc.C, desc.M, desc.N, desc.K, desc.dtype, desc.transB,
                           desc.scaleA, desc.scaleB, _stream_ptr(stream)), "rov_gemm")


def make_attn_desc(Q, K, V, O, p, causal=False):
    B, S, H, d = Q.shape
    desc = AttnDesc(Q.data_ptr(), K.data_ptr(), V.data_ptr(), O.data_ptr(), B, H, K.shape[2], S, d,
                    _strides12(Q, K, V, O), _dtype_code(Q), int(bool(causal)), float(p))
    return desc


def layer_step(schedule, gemm_descs, attn_desc, seed, offset, mask, main_stream, side_stream, rounds=None,
               bits=None):
    arr = (GemmDesc * len(gemm_descs))(*gemm_descs)
    mptr = mask.data_ptr() if mask is not None else None
    if bits is not None:
        _check(load().rov_layer_step_bits(int(schedule), arr, len(gemm_descs), ctypes.byref(attn_desc),
                                          seed & (2**64 - 1), offset & (2**64 - 1), int(bits), mptr,
                                          _stream_ptr(main_stream), _stream_ptr(side_stream)),
               "rov_layer_step_bits")
        return
    if rounds is not None:
        _check(load().rov_layer_step_rounds(int(schedule), arr, len(gemm_descs), ctypes.byref(attn_desc),
                                            seed & (2**64 - 1), offset & (2**64 - 1), int(rounds), mptr,
                                            _stream_ptr(main_stream), _stream_ptr(side_stream)),
               "rov_layer_step_rounds")
        return
    _check(load().rov_layer_step(int(schedule), arr, len(gemm_descs), ctypes.byref(attn_desc),
                                 seed & (2**64 - 1), offset & (2**64 - 1), mptr,
                                 _stream_ptr(main_stream), _stream_ptr(side_stream)), "rov_layer_step")


def block_workspace_bytes(cfg, B, S, schedule):
    return int(load().rov_block_workspace_bytes(ctypes.byref(cfg), B, S, int(schedule)))


def block_hybrid_mask_rows(cfg, B, S):
    return int(load().rov_block_hybrid_mask_rows(ctypes.byref(cfg), B, S))


def set_block_hybrid_mask_rows(rows):
    return int(load().rov_set_block_hybrid_mask_rows(int(rows)))


def make_block_cfg(H, Hkv, d, hidden, ffn, p, causal=False, eps=1e-5, rope_theta=500000.0, dtype=BF16,
                   act_scale=None):
    """act_scale (fp8 only): dequantisation scales of the four quantised activations h1, a, h2, u."""
    sc = (ctypes.c_float * 4)(*([float(v) for v in act_scale] if act_scale is not None else [0.0] * 4))
    return BlockCfg(H, Hkv, d, hidden, ffn, dtype, int(bool(causal)), float(p), float(eps), float(rope_theta), sc)


def make_block_weights(w, w_scale=None):
    """w: dict of device tensors norm1, norm2, wqkv, wo, wg, wu, wd; w_scale (fp8 only): dict of the five
    weight matrices' dequantisation scales."""
    names = ("wqkv", "wo", "wg", "wu", "wd")
    sc = (ctypes.c_float * 5)(*([float(w_scale[n]) for n in names] if w_scale is not None else [0.0] * 5))
    return BlockWeights(*[w[n].data_ptr() for n in ("norm1", "norm2") + names], sc)


def make_block_opts(rope=None, positions=None, post1=None, gate1=None, post2=None, gate2=None, rows_per_gate=0, x_scale=1.0, h_scale=1.0):
    """Rotary form (make_rope_cfg; positions int64 [B, S] or [S]), post norms, gates and residual scales of a block (rov_block_opts).
    The opts keep the tensors and the rotary form."""
    names, tensors = ("post1", "gate1", "post2", "gate2"), (post1, gate1, post2, gate2)
    stride = 0
    if any(t is not None for t in tensors + (positions,)):
        _on_gpu("make_block_opts", None, names + ("positions",), tensors + (positions,))
        for name, t in zip(names, tensors):
            if t is not None and (t.dtype != _torch.bfloat16 or not t.is_contiguous()):
                raise TypeError("make_block_opts: %s must be torch.bfloat16, contiguous" % name)
    if positions is not None:
        if positions.dtype != _torch.int64:
            raise TypeError("make_block_opts: positions must be torch.int64, not %s" % positions.dtype)
        if positions.dim() not in (1, 2) or (positions.shape[-1] > 1 and positions.stride(-1) != 1):
            raise ValueError("make_block_opts: positions must be [B, S], [1, S] or [S], contiguous along S")
        stride = positions.stride(0) if positions.dim() == 2 and positions.shape[0] > 1 else 0
    opts = BlockOpts(ctypes.pointer(rope) if rope is not None else None, _ptr(positions), stride, _ptr(post1), _ptr(gate1), _ptr(post2), _ptr(gate2),
                     int(rows_per_gate), float(x_scale), float(h_scale))
    opts.tensors = (positions,) + tensors
    return opts


def _check_block_opts(opts, B, S, hidden):
    """Does what the opts point at have the elements that the block reads?"""
    positions, post1, gate1, post2, gate2 = getattr(opts, "tensors", (None,) * 5)   # (a BlockOpts of the caller's own has none)
    if positions is not None and positions.shape not in ((B, S), (1, S), (S,)):
        raise ValueError("block_forward: positions must be [B, S], [1, S] or [S]")
    gates = B * S // opts.rows_per_gate if opts.rows_per_gate > 0 else 1
    for name, have, want in (("post1", post1, hidden), ("gate1", gate1, gates * hidden), ("post2", post2, hidden), ("gate2", gate2, gates * hidden)):
        if have is not None and have.numel() != want:
            raise ValueError("block_forward: %s must have %d elements, not %d" % (name, want, have.numel()))


def block_forward(weights, x, y, cfg, schedule, seed, offset, mask, workspace, main_stream, side_stream,
                  mask_ready=False, next_mask=None, opts=None):
    """opts: make_block_opts, for blocks with other rotary forms, post norms, gates or residual scales."""
    B, S, _ = x.shape
    mptr = mask.data_ptr() if mask is not None else None
    nptr = next_mask.data_ptr() if next_mask is not None else None
    rest = (x.data_ptr(), y.data_ptr(), B, S, ctypes.byref(cfg), int(schedule), seed & (2**64 - 1), offset & (2**64 - 1), int(mask_ready),
            mptr, nptr, workspace.data_ptr(), workspace.numel() * workspace.element_size(), _stream_ptr(main_stream), _stream_ptr(side_stream))
    if opts is not None:
        _check_block_opts(opts, B, S, cfg.hidden)
        _check(load().rov_block_forward_opts(ctypes.byref(weights), ctypes.byref(opts), *rest), "rov_block_forward_opts")
    else:
        _check(load().rov_block_forward(ctypes.byref(weights), *rest), "rov_block_forward")
    return y


def mask_finish(mask, main_stream):
    """Completes and joins a mask that an OVERLAP_DEFERRED block_forward left in flight."""
    _check(load().rov_mask_finish(mask.data_ptr(), _stream_ptr(main_stream)), "rov_mask_finish")


def block_static_scratch_bytes():
    return int(load().rov_block_static_scratch_bytes())


def block_forward_static(weights, x, y, cfg, schedule, seed, offset, mask, main_stream, side_stream,
                         mask_ready=False, next_mask=None):
    """block_forward on the library's own static scratch (no workspace, nothing allocated)."""
    B, S, _ = x.shape
    mptr = mask.data_ptr() if mask is not None else None
    nptr = next_mask.data_ptr() if next_mask is not None else None
    _check(load().rov_block_forward_static(ctypes.byref(weights), x.data_ptr(),
                                           y.data_ptr(), B, S, ctypes.byref(cfg), int(schedule),
                                           seed & (2**64 - 1), offset & (2**64 - 1), int(mask_ready), mptr,
                                           nptr, _stream_ptr(main_stream), _stream_ptr(side_stream)),
           "rov_block_forward_static")
    return y


# ---- operators around the block.  Results and workspaces that the caller does not bring come from torch's allocator, on
# the stream that the call runs on (a block of another stream's pool could still be in use there).
# Their small calls, too, are bound by this file (norms of 16 tokens: 16.3 us at first, 10.5 now; the kernel takes 4): what a call asks
# of its tensors is asked once, in one pass, and names and messages are made only where something is refused.
# strides go to ctypes packed (bytes are taken as a pointer to them): a quarter of the time of a ctypes array
_pack4, _pack6, _pack12 = (struct.Struct("%dq" % n).pack for n in (4, 6, 12))
_torch = _current_device = None
# sizes go to the library as C ints, and ctypes would keep only their low bits
_INT_MAX = 0x7FFFFFFF


def _refuse_sizes(what):
    raise RovError(ERR_UNSUPPORTED, what + " (a size beyond 2^31 - 1)")


def _start():
    global _torch, _current_device
    import torch
    torch.cuda.current_device()     # initialises the device
    _torch, _current_device = torch, getattr(torch._C, "_cuda_getDevice", None) or torch.cuda.current_device


def _new(shape, like, stream, dtype):
    if stream is None:
        return like.new_empty(shape, dtype=dtype)
    with _torch.cuda.stream(stream):
        return like.new_empty(shape, dtype=dtype)


def _new_like(like, stream):
    if stream is None:
        return _torch.empty_like(like)
    with _torch.cuda.stream(stream):
        return _torch.empty_like(like)


def _on_gpu(what, dtype, names, tensors):
    """Refuses tensors off the current GPU or of another dtype (None: any); absent ones are None."""
    if _torch is None:
        _start()
    device = _current_device()
    for t in tensors:
        if t is not None and (t.get_device() != device or (dtype is not None and t.dtype != dtype)):
            name = names[[u is t for u in tensors].index(True)]
            if t.get_device() != device:
                raise ValueError("%s: %s must be on the current GPU" % (what, name))
            raise TypeError("%s: %s must be %s, not %s" % (what, name, dtype, t.dtype))


def make_rope_cfg(rot, theta, layout=ROPE_INTERLEAVED, scaling=ROPE_SCALE_NONE, factor=1.0, turns_low=1.0, turns_high=4.0,
                  trained_len=0, magnitude=1.0):
    """Rotary positions of a head's first `rot` elements (rov_rope_cfg)."""
    if not (-_INT_MAX <= rot <= _INT_MAX and -_INT_MAX <= trained_len <= _INT_MAX):
        _refuse_sizes("make_rope_cfg")
    return RopeCfg(layout, rot, scaling, trained_len, theta, factor, turns_low, turns_high, magnitude)


def rope(cfg, Q, K=None, positions=None, Qo=None, Ko=None, backward=False, stream=None):
    """Q [B,S,H,d] and K [B,S,Hkv,d] turned by their positions (int64 [B,S], [1,S] or [S]; None: 0..S-1) into
    Qo and Ko (new if None; Q and K themselves for in place).  backward: gradients of Q and K from those of the results."""
    B, S, H, d = shape = Q.shape
    if (B | S | H | d) > _INT_MAX:
        _refuse_sizes("rov_rope")
    _on_gpu("rope", Q.dtype, ("Q", "K", "Qo", "Ko"), (Q, K, Qo, Ko))
    if Qo is None:
        Qo = _new_like(Q, stream)
    elif Qo.shape != shape:
        raise ValueError("rope: Qo must have the shape of Q")
    q0, q1, q2, qd = Q.stride()
    o0, o1, o2, od = Qo.stride()
    inner = qd == 1 == od
    if K is not None:
        kshape = K.shape
        if len(kshape) != 4 or kshape[0] != B or kshape[1] != S or kshape[3] != d:
            raise ValueError("rope: K must be [B, S, Hkv, d] beside Q [B, S, H, d]")
        Hkv = kshape[2]
        if Hkv > _INT_MAX:
            _refuse_sizes("rov_rope")
        if Ko is None:
            Ko = _new_like(K, stream)
        elif Ko.shape != kshape:
            raise ValueError("rope: Ko must have the shape of K")
        k0, k1, k2, kd = K.stride()
        l0, l1, l2, ld = Ko.stride()
        inner = inner and kd == 1 == ld
        kp, kop = K.data_ptr(), Ko.data_ptr()
    elif Ko is not None:
        raise ValueError("rope: Ko without K")
    else:
        Hkv = k0 = k1 = k2 = l0 = l1 = l2 = 0
        kp = kop = None
    if not inner and d > 1:
        raise ValueError("rope: the head dimension must be contiguous")
    pos, pstride = None, 0
    if positions is not None:
        _on_gpu("rope", _torch.int64, ("positions",), (positions,))
        shape, ps = positions.shape, positions.stride()
        if (shape != (B, S) and shape != (1, S) and shape != (S,)) or (S > 1 and ps[-1] != 1):
            raise ValueError("rope: positions must be [B, S], [1, S] or [S], contiguous along S")
        pos = positions.data_ptr()
        if len(shape) == 2 and shape[0] > 1:
            pstride = ps[0]
    _check(load().rov_rope(cfg, Q.data_ptr(), Qo.data_ptr(), kp, kop, B, S, H, Hkv, d,
                           _pack12(q0, q1, q2, o0, o1, o2, k0, k1, k2, l0, l1, l2),
                           _dtype_code(Q), pos, pstride, 1 if backward else 0, _stream_ptr(stream)), "rov_rope")
    return (Qo, Ko) if K is not None else Qo


def _row_strides(what, names, tensors, shape, n):
    """Row strides of tensors of one shape [..., n] (n for absent ones)."""
    for t in tensors:
        if t is not None and not (t.is_contiguous() and t.shape == shape):
            break
    else:
        return (n,) * len(tensors)
    out = []
    for t in tensors:
        if t is None or t.is_contiguous():
            if t is not None and t.shape != shape:
                raise ValueError("%s: %s must be %s" % (what, names[[u is t for u in tensors].index(True)], list(shape)))
            out.append(n)
            continue
        if t.shape != shape or len(shape) != 2 or (n > 1 and t.stride(1) != 1):
            raise ValueError("%s: %s must be %s with contiguous rows" % (what, names[[u is t for u in tensors].index(True)], list(shape)))
        out.append(t.stride(0) if shape[0] > 1 else n)
    return out


def _rows_per_gate(what, rows, n, w_pre, w_post, gate):
    for t in (w_pre, w_post):
        if t is not None and (t.numel() != n or t.dim() != 1 or not t.is_contiguous()):
            raise ValueError("%s: weights must be [%d], contiguous" % (what, n))
    if gate is None:
        return rows
    gates = gate.numel() // n
    if gate.shape == (n,) and gate.is_contiguous():
        return rows
    if gate.shape[-1] != n or gate.dim() > 2 or not gate.is_contiguous() or gates == 0 or rows % gates:
        raise ValueError("%s: gate must be [%d] or [gates, %d], contiguous, its gates shared evenly by the %d rows" % (what, n, n, rows))
    return rows // gates


def _ptr(t):
    return t.data_ptr() if t is not None else None


def norm_residual(x, h, w_pre=None, w_post=None, gate=None, x_scale=1.0, h_scale=1.0, eps=1e-5, y=None, yn=None, yn_fp8_scale=None,
                  stream=None):
    """(y, yn): y = x_scale * x + h_scale * gate * (RMS(h) * w_post), yn = RMS(y) * w_pre (None without w_pre); x, h [..., n],
    gate [n] or [gates, n] (consecutive rows share a gate).  yn_fp8_scale (above 0): yn in e4m3 bytes with that scale."""
    shape = x.shape
    if x.numel() == 0 or x.dim() == 0:
        raise ValueError("norm_residual: x must be [..., n], not empty")
    # (a scale of 0, also one that fp32 rounds to 0, is the library's sign for a result of x's type: twice the bytes that yn has here)
    if yn_fp8_scale is not None and not ctypes.c_float(yn_fp8_scale).value > 0.0:
        raise ValueError("norm_residual: yn_fp8_scale must be above 0 in fp32")
    n = shape[-1]
    if n > _INT_MAX:
        _refuse_sizes("rov_norm_residual")
    _on_gpu("norm_residual", x.dtype, ("x", "h", "w_pre", "w_post", "gate", "y"), (x, h, w_pre, w_post, gate, y))
    if y is None:
        y = _new_like(x, stream)
    if yn is not None:
        _on_gpu("norm_residual", x.dtype if yn_fp8_scale is None else _torch.uint8, ("yn",), (yn,))
    elif w_pre is not None:
        yn = _new_like(x, stream) if yn_fp8_scale is None else _new(shape, x, stream, _torch.uint8)
    ld = _row_strides("norm_residual", ("x", "h", "y", "yn"), (x, h, y, yn), shape, n)
    rows = x.numel() // n
    per = _rows_per_gate("norm_residual", rows, n, w_pre, w_post, gate)
    _check(load().rov_norm_residual(x.data_ptr(), h.data_ptr(), _ptr(w_post), _ptr(gate), _ptr(w_pre), y.data_ptr(), _ptr(yn), rows, n,
                                    _pack4(*ld), per, _dtype_code(x), x_scale, h_scale, eps, yn_fp8_scale or 0.0, _stream_ptr(stream)),
           "rov_norm_residual")
    return y, yn


def norm_residual_bwd_workspace_bytes(rows, n, rows_per_gate, dtype):
    if n > _INT_MAX:
        return 0
    return int(load().rov_norm_residual_bwd_workspace_bytes(int(rows), int(n), int(rows_per_gate), int(dtype)))


def norm_residual_bwd(y, h, dy, dn=None, w_pre=None, w_post=None, gate=None, x_scale=1.0, h_scale=1.0, eps=1e-5, dx=None, dh=None,
                      workspace=None, stream=None):
    """(dx, dh, dw_pre, dw_post, dgate) of norm_residual from its y and h and the gradients of y (dy, may be None) and yn (dn);
    the last three in fp32, None without their input."""
    like = dy if dy is not None else dn
    if like is None:
        raise ValueError("norm_residual_bwd: dy or dn is needed")
    shape, dt = like.shape, like.dtype
    if like.numel() == 0 or like.dim() == 0:
        raise ValueError("norm_residual_bwd: the gradients must be [..., n], not empty")
    n = shape[-1]
    if n > _INT_MAX:
        _refuse_sizes("rov_norm_residual_bwd")
    names, tensors = ("y", "h", "dy", "dn", "dx", "dh"), (y, h, dy, dn, dx, dh)
    _on_gpu("norm_residual_bwd", dt, names + ("w_pre", "w_post", "gate"), tensors + (w_pre, w_post, gate))
    if dx is None:
        dx = _new_like(like, stream)
    if dh is None:
        dh = _new_like(like, stream)
    ld = _row_strides("norm_residual_bwd", names, (y, h, dy, dn, dx, dh), shape, n)
    rows = like.numel() // n
    per = _rows_per_gate("norm_residual_bwd", rows, n, w_pre, w_post, gate)
    f32 = _torch.float32
    dw_pre = _new((n,), like, stream, f32) if w_pre is not None else None
    dw_post = _new((n,), like, stream, f32) if w_post is not None else None
    dgate = _new(gate.shape, like, stream, f32) if gate is not None else None
    code, L = _dtype_code(like), load()
    if workspace is None:
        size = L.rov_norm_residual_bwd_workspace_bytes(rows, n, per, code) if dw_pre is not None or dw_post is not None or dgate is not None else 0
        workspace = _new((size,), like, stream, _torch.uint8) if size else None
    else:
        _on_gpu("norm_residual_bwd", None, ("workspace",), (workspace,))
        size = workspace.numel() * workspace.element_size()
    _check(L.rov_norm_residual_bwd(_ptr(y), _ptr(h), _ptr(w_post), _ptr(gate), _ptr(w_pre), _ptr(dy), _ptr(dn), dx.data_ptr(), dh.data_ptr(),
                                   _ptr(dw_post), _ptr(dgate), _ptr(dw_pre), rows, n, _pack6(*ld), per, code, x_scale, h_scale, eps,
                                   _ptr(workspace), size, _stream_ptr(stream)), "rov_norm_residual_bwd")
    return dx, dh, dw_pre, dw_post, dgate


def linear_xent_workspace_bytes(M, V, K, dtype, backward=False, vocab_piece=0):
    if max(M, V, K, vocab_piece) > _INT_MAX:
        return 0
    return int(load().rov_linear_xent_workspace_bytes(int(M), int(V), int(K), int(dtype), int(bool(backward)), int(vocab_piece)))


def linear_xent_walks(M, V, K, backward=False, vocab_piece=0):
    """The products of a bf16 call whose workgroups take several tiles: 1 logits of the loss, 2 logits of the gradients, 4 dX, 8 dW."""
    r = load().rov_linear_xent_walks(M, V, K, int(bool(backward)), vocab_piece)
    if r < 0:
        raise RovError(r, "rov_linear_xent_walks")
    return r


def _xent_operands(what, X, W, targets, f32, outs, vocab_piece):
    """Checks what both calls take; (M, V, K, row strides of X, W and the results)."""
    if X.dim() != 2 or W.dim() != 2 or X.shape[1] != W.shape[1]:
        raise ValueError("%s: X must be [M, K] and W [V, K]" % what)
    (M, K), V = X.shape, W.shape[0]
    if (M | V | K) > _INT_MAX or vocab_piece > _INT_MAX:
        _refuse_sizes("rov_" + what)
    _on_gpu(what, X.dtype, ("X", "W", "dX", "dW"), (X, W) + outs)
    _on_gpu(what, _torch.int64, ("targets",), (targets,))
    _on_gpu(what, _torch.float32, tuple(f32), tuple(f32.values()))
    for name, t in (("targets", targets),) + tuple(f32.items()):
        if t is not None and (t.shape != (M,) or not t.is_contiguous()):
            raise ValueError("%s: %s must be [M], contiguous" % (what, name))
    ldx, lddx = _row_strides(what, ("X", "dX"), (X, outs[0] if outs else None), X.shape, K)
    ldw, lddw = _row_strides(what, ("W", "dW"), (W, outs[1] if outs else None), W.shape, K)
    return M, V, K, ldx, ldw, lddx, lddw


def _xent_workspace(what, workspace, X, stream, *sizes):
    if workspace is None:
        return _new((load().rov_linear_xent_workspace_bytes(*sizes),), X, stream, _torch.uint8)
    _on_gpu(what, None, ("workspace",), (workspace,))
    return workspace


def linear_xent(X, W, targets, scale=1.0, ignore_index=-100, loss=None, lse=None, vocab_piece=0, workspace=None, stream=None):
    """(loss, lse), fp32 [M], of the logits scale * X @ W^T (X [M, K], W [V, K]) against targets (int64 [M]).  vocab_piece: fp32 only (the bf16
    loss keeps no piece of the logits)."""
    M, V, K, ldx, ldw, _, _ = _xent_operands("linear_xent", X, W, targets, dict(loss=loss, lse=lse), (), vocab_piece)
    if loss is None:
        loss = _new((M,), X, stream, _torch.float32)
    if lse is None:
        lse = _new((M,), X, stream, _torch.float32)
    code = _dtype_code(X)
    workspace = _xent_workspace("linear_xent", workspace, X, stream, M, V, K, code, 0, vocab_piece)
    _check(load().rov_linear_xent(X.data_ptr(), W.data_ptr(), targets.data_ptr(), M, V, K, ldx, ldw, code, scale, ignore_index,
                                  loss.data_ptr(), lse.data_ptr(), vocab_piece, workspace.data_ptr(),
                                  workspace.numel() * workspace.element_size(), _stream_ptr(stream)), "rov_linear_xent")
    return loss, lse


def linear_xent_bwd(X, W, targets, lse, dloss, dlse=None, scale=1.0, ignore_index=-100, dX=None, dW=None, need_dX=True, need_dW=True,
                    vocab_piece=0, workspace=None, stream=None):
    """(dX, dW) from linear_xent's lse and the gradients of loss and lse (fp32 [M]); None for one that is not needed."""
    M, V, K, ldx, ldw, lddx, lddw = _xent_operands("linear_xent_bwd", X, W, targets, dict(lse=lse, dloss=dloss, dlse=dlse), (dX, dW), vocab_piece)
    if dX is None and need_dX:
        dX = _new((M, K), X, stream, X.dtype)
    if dW is None and need_dW:
        dW = _new((V, K), W, stream, W.dtype)
    code = _dtype_code(X)
    workspace = _xent_workspace("linear_xent_bwd", workspace, X, stream, M, V, K, code, 1, vocab_piece)
    _check(load().rov_linear_xent_bwd(X.data_ptr(), W.data_ptr(), targets.data_ptr(), lse.data_ptr(), dloss.data_ptr(), _ptr(dlse), M, V, K,
                                      ldx, ldw, code, scale, ignore_index, _ptr(dX), _ptr(dW), lddx, lddw, vocab_piece,
                                      workspace.data_ptr(), workspace.numel() * workspace.element_size(), _stream_ptr(stream)),
           "rov_linear_xent_bwd")
    return dX, dW


TRACE_GEMM, TRACE_RNG, TRACE_ATTENTION, TRACE_GLUE, TRACE_RNG_HELPER = 0, 1, 2, 3, 4


def trace_enable(on, kinds=None):
    """on=False: off.  on=True: every kind, or only the kinds listed (e.g. [TRACE_GEMM])."""
    if not on:
        sel = 0
    elif kinds is None:
        sel = -1
    else:
        sel = 0
        for k in kinds:
            sel |= 1 << int(k)
    return int(load().rov_trace_enable(sel))


def trace_read(max_records=16384):
    """List of (kind, milliseconds) in launch order; waits for the traced kernels to finish."""
    kinds = (ctypes.c_int * max_records)()
    ms = (ctypes.c_float * max_records)()
    n = ctypes.c_int(0)
    _check(load().rov_trace_read(kinds, ms, max_records, ctypes.byref(n)), "rov_trace_read")
    return [(int(kinds[i]), float(ms[i])) for i in range(n.value)]
