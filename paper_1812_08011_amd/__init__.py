"""Python binding of libfp8train (include/fp8train.h, fp8train_lm.h, fp8train_tokens.h).

Argument marshalling only: every step runs in the HIP library.  Arrays are
torch tensors on the GPU (uint8 for FP8 codes, uint16 for FP16 codes, float32
for IEEE inputs); work goes onto torch's current HIP stream unless a stream is
given.  A call that the library rejects raises Fp8tError.  There is no CPU
fallback: if the library is not built, every call raises.
"""
import ctypes
import os

PKG = os.path.dirname(os.path.abspath(__file__))
LIB_PATH = os.path.join(PKG, "libfp8train.so")

OK, EINVAL, EWORKSPACE, EHIP = 0, -1, -2, -3
SRC_F32, SRC_FP16 = 0, 1
EXACT, FAST = 0, 1
FMT_F32, FMT_FP16, FMT_FP8, FMT_HALF = 0, 1, 2, 3
ATTN_MAX_D = 128
MAX_TOP, MAX_VOCAB, MAX_NORM_W = 128, 1 << 24, 1 << 20

_lib = None


class Fp8tError(RuntimeError):
    def __init__(self, fn, status):
        super().__init__(f"{fn}: {status_string(status)} (status {status})")
        self.status = status


def lib():
    """The loaded library.  Raises if it has not been built."""
    global _lib
    if _lib is None:
        if not os.path.exists(LIB_PATH):
            raise RuntimeError(
                f"{LIB_PATH} is not built; run `python -m paper_1812_08011_amd.build` "
                "or __graft_entry__.build()")
        L = ctypes.CDLL(LIB_PATH)
        i32, i64, u64, f32, vp, sz = (ctypes.c_int, ctypes.c_int64, ctypes.c_uint64,
                                      ctypes.c_float, ctypes.c_void_p, ctypes.c_size_t)
        L.fp8_quantize.restype = i32
        L.fp8_quantize.argtypes = [vp, i32, f32, vp, i64, vp]
        L.fp16_quantize.restype = i32
        L.fp16_quantize.argtypes = [vp, vp, i64, vp]
        L.chunk_gemm.restype = i32
        L.chunk_gemm.argtypes = [i32, i32, i64, i64, i64, i64, vp, i64, vp, i64, vp, i64,
                                 i32, vp, sz, vp]
        L.chunk_gemm_noalloc.restype = i32
        L.chunk_gemm_noalloc.argtypes = [i32, i32, i64, i64, i64, i64, vp, i64, vp, i64, vp, i64,
                                         i32, vp]
        L.chunk_gemm_workspace_size.restype = sz
        L.chunk_gemm_workspace_size.argtypes = [i32, i32, i64, i64, i64, i64, i32]
        L.chunk_gemm_fp8.restype = i32
        L.chunk_gemm_fp8.argtypes = [i32, i32, i64, i64, i64, i64, vp, i64, vp, i64, vp, i64,
                                     vp, i64, f32, i32, vp, sz, vp]
        L.chunk_gemm_fp8_workspace_size.restype = sz
        L.chunk_gemm_fp8_workspace_size.argtypes = [i32, i32, i64, i64, i64, i64, i32]
        L.chunk_gemm_sr.restype = i32
        L.chunk_gemm_sr.argtypes = [i32, i32, i64, i64, i64, i64, vp, i64, vp, i64, vp, i64,
                                    u64, u64, vp, sz, vp]
        L.chunk_gemm_sr_workspace_size.restype = sz
        L.chunk_gemm_sr_workspace_size.argtypes = [i32, i32, i64, i64, i64, i64]
        L.chunk_gemm_p16.restype = i32
        L.chunk_gemm_p16.argtypes = [i32, i32, i64, i64, i64, i64, vp, i64, vp, i64, vp, i64,
                                     vp, sz, vp]
        L.chunk_gemm_p16_workspace_size.restype = sz
        L.chunk_gemm_p16_workspace_size.argtypes = [i32, i32, i64, i64, i64, i64]
        L.relu_codes.restype = i32
        L.relu_codes.argtypes = [vp, i32, vp, i64, vp]
        L.relu_backward_fp8.restype = i32
        L.relu_backward_fp8.argtypes = [vp, vp, vp, i64, f32, vp]
        L.mse_grad_fp16.restype = i32
        L.mse_grad_fp16.argtypes = [vp, vp, vp, i64, f32, vp]
        L.conv2d_fwd_fp8.restype = i32
        L.conv2d_fwd_fp8.argtypes = [vp, i64, i64, i64, i64, i64, i64, i64, i64, vp, i64, i64,
                                     vp, i64, vp, sz, vp]
        L.conv2d_wgrad_fp8.restype = i32
        L.conv2d_wgrad_fp8.argtypes = list(L.conv2d_fwd_fp8.argtypes)
        L.conv2d_workspace_size.restype = sz
        L.conv2d_workspace_size.argtypes = [i32, i64, i64, i64, i64, i64, i64, i64, i64, i64,
                                            i64]
        L.col2im_fp16.restype = i32
        L.col2im_fp16.argtypes = [vp, i64, i64, i64, i64, i64, i64, i64, i64, vp, vp]
        L.adam_update.restype = i32
        L.adam_update.argtypes = [vp, vp, vp, vp, vp, i64, f32, f32, f32, f32, f32, u64, u64,
                                  u64, vp]
        L.sr_weight_update.restype = i32
        L.sr_weight_update.argtypes = [vp, vp, vp, vp, i64, f32, f32, f32, u64, u64, vp]
        L.fp16_dequantize.restype = i32
        L.fp16_dequantize.argtypes = [vp, f32, vp, i32, i64, vp]
        L.rotary_embed.restype = i32
        L.rotary_embed.argtypes = [vp, i32, i64, i64, vp, vp, i64, i64, i64, i64, i32, i32, f32,
                                   f32, vp, i32, i64, i64, vp]
        rows, sizes = [vp, i64, i64], [i64] * 8 + [i32]
        L.attn_fwd_fp8.restype = i32
        L.attn_fwd_fp8.argtypes = (rows * 3 + [vp, vp] + sizes + [f32] + rows * 2 +
                                   [f32, vp, vp, sz, vp])
        L.attn_bwd_fp8.restype = i32
        L.attn_bwd_fp8.argtypes = (rows * 3 + [vp, vp] + sizes + [f32] + rows * 2 + [vp] +
                                   rows * 3 + [i32, f32, vp, sz, vp])
        for f in (L.attn_fwd_fp8_workspace_size, L.attn_bwd_fp8_workspace_size):
            f.restype = sz
            f.argtypes = sizes
        L.distill_loss.restype = i32
        L.distill_loss.argtypes = [vp, i32, i64, vp, vp, i32, i64, vp, i64, i64, f32, f32, vp, vp,
                                   i32, i64, vp]
        L.embed_fwd.restype = i32
        L.embed_fwd.argtypes = [vp, i64, vp, i32, i64, i64, i64, f32, vp, i32, i64, vp]
        L.embed_bwd.restype = i32
        L.embed_bwd.argtypes = [vp, i64, vp, i32, i64, i64, i64, f32, vp, i32, i64, vp, sz, vp]
        L.embed_bwd_workspace_size.restype = sz
        L.embed_bwd_workspace_size.argtypes = [i64, i64, i64]
        L.rms_norm_fwd.restype = i32
        L.rms_norm_fwd.argtypes = [vp, i32, i64, vp, vp, i64, vp, i32, i64, i64, f32, vp, i32, i64,
                                   vp, i32, i64, f32, vp, vp, vp]
        L.rms_norm_bwd.restype = i32
        L.rms_norm_bwd.argtypes = [vp, i32, i64, vp, i32, vp, vp, i32, i64, vp, i64, i64, i64, vp,
                                   i32, i64, vp, i64, f32, vp, i32, vp, sz, vp]
        L.rms_norm_bwd_workspace_size.restype = sz
        L.rms_norm_bwd_workspace_size.argtypes = [i64, i64]
        L.token_logprobs.restype = i32
        L.token_logprobs.argtypes = [vp, i32, i64, vp, i64, i64, i64, f32, vp, vp, vp, i64, vp, vp,
                                     vp, sz, vp]
        L.token_logprobs_workspace_size.restype = sz
        L.token_logprobs_workspace_size.argtypes = [i64, i64, i64]
        L.token_logprobs_bwd.restype = i32
        L.token_logprobs_bwd.argtypes = [vp, i32, i64, vp, i64, vp, vp, vp, vp, i64, i64, f32, f32,
                                         vp, i32, i64, vp]
        L.fp8t_status_string.restype = ctypes.c_char_p
        L.fp8t_status_string.argtypes = [i32]
        _lib = L
    return _lib


def status_string(status):
    return lib().fp8t_status_string(int(status)).decode()


def _ptr(t):
    if t is None:
        return None
    if isinstance(t, int):
        return t
    return t.data_ptr()


def _stream(stream):
    if stream is None:
        import torch
        # the address alone, where this torch gives it: 0.3 us, a stream object 2.7
        raw = getattr(torch._C, "_cuda_getCurrentRawStream", None)
        if raw is None:
            return torch.cuda.current_stream().cuda_stream
        return raw(torch.cuda.current_device())
    if isinstance(stream, int):
        return stream
    return stream.cuda_stream


def _check(fn, status):
    if status != OK:
        raise Fp8tError(fn, status)


def fp8_quantize(src, dst, scale=1.0, stream=None):
    """dst (uint8, FP8 codes) = Q8(src * scale); src float32 or uint16 FP16 codes."""
    import torch
    if src.dtype == torch.float32:
        fmt = SRC_F32
    elif src.dtype == torch.uint16:
        fmt = SRC_FP16
    else:
        raise TypeError("fp8_quantize: src must be float32 or uint16 (FP16 codes)")
    if dst.dtype != torch.uint8 or dst.numel() != src.numel():
        raise TypeError("fp8_quantize: dst must be uint8 with as many elements as src")
    if not (src.is_contiguous() and dst.is_contiguous()):
        raise ValueError("fp8_quantize: tensors must be contiguous")
    _check("fp8_quantize", lib().fp8_quantize(_ptr(src), fmt, float(scale), _ptr(dst),
                                               src.numel(), _stream(stream)))
    return dst


def fp16_quantize(src, dst, stream=None):
    """dst (uint16, FP16 codes) = round-to-nearest-even of float32 src."""
    import torch
    if src.dtype != torch.float32 or dst.dtype != torch.uint16 or dst.numel() != src.numel():
        raise TypeError("fp16_quantize: float32 src, uint16 dst of the same size")
    if not (src.is_contiguous() and dst.is_contiguous()):
        raise ValueError("fp16_quantize: tensors must be contiguous")
    _check("fp16_quantize", lib().fp16_quantize(_ptr(src), _ptr(dst), src.numel(),
                                                 _stream(stream)))
    return dst


def chunk_gemm_workspace_size(trans_a, trans_b, M, N, K, CL, mode):
    return int(lib().chunk_gemm_workspace_size(int(trans_a), int(trans_b), int(M), int(N),
                                               int(K), int(CL), int(mode)))


def chunk_gemm(trans_a, trans_b, M, N, K, CL, A, lda, B, ldb, C, ldc, mode=EXACT,
               workspace=None, workspace_bytes=0, stream=None):
    """The C-ABI call with the same argument order; A, B, C, workspace are
    tensors (or raw device addresses)."""
    _check("chunk_gemm", lib().chunk_gemm(int(trans_a), int(trans_b), int(M), int(N), int(K),
                                          int(CL), _ptr(A), int(lda), _ptr(B), int(ldb),
                                          _ptr(C), int(ldc), int(mode), _ptr(workspace),
                                          int(workspace_bytes), _stream(stream)))
    return C


def chunk_gemm_noalloc(trans_a, trans_b, M, N, K, CL, A, lda, B, ldb, C, ldc, mode=EXACT,
                       stream=None):
    """The C-ABI call with the same argument order (no workspace: the
    library's static scratch holds shared tiles' chunk sums)."""
    _check("chunk_gemm_noalloc",
           lib().chunk_gemm_noalloc(int(trans_a), int(trans_b), int(M), int(N), int(K), int(CL),
                                    _ptr(A), int(lda), _ptr(B), int(ldb), _ptr(C), int(ldc),
                                    int(mode), _stream(stream)))
    return C


def chunk_gemm_fp8_workspace_size(trans_a, trans_b, M, N, K, CL, mode):
    return int(lib().chunk_gemm_fp8_workspace_size(int(trans_a), int(trans_b), int(M), int(N),
                                                   int(K), int(CL), int(mode)))


def chunk_gemm_fp8(trans_a, trans_b, M, N, K, CL, A, lda, B, ldb, C, ldc, C8, ldc8, scale=1.0,
                   mode=EXACT, workspace=None, workspace_bytes=0, stream=None):
    """The C-ABI call with the same argument order; C may be None (FP8 result
    only)."""
    _check("chunk_gemm_fp8",
           lib().chunk_gemm_fp8(int(trans_a), int(trans_b), int(M), int(N), int(K), int(CL),
                                _ptr(A), int(lda), _ptr(B), int(ldb), _ptr(C), int(ldc), _ptr(C8),
                                int(ldc8), float(scale), int(mode), _ptr(workspace),
                                int(workspace_bytes), _stream(stream)))
    return C8


def chunk_gemm_sr_workspace_size(trans_a, trans_b, M, N, K, CL):
    return int(lib().chunk_gemm_sr_workspace_size(int(trans_a), int(trans_b), int(M), int(N),
                                                  int(K), int(CL)))


def chunk_gemm_sr(trans_a, trans_b, M, N, K, CL, A, lda, B, ldb, C, ldc, seed, offset=0,
                  workspace=None, workspace_bytes=0, stream=None):
    """The C-ABI call with the same argument order (stochastic rounding after
    every FP16 addition)."""
    _check("chunk_gemm_sr",
           lib().chunk_gemm_sr(int(trans_a), int(trans_b), int(M), int(N), int(K), int(CL),
                               _ptr(A), int(lda), _ptr(B), int(ldb), _ptr(C), int(ldc),
                               int(seed), int(offset), _ptr(workspace), int(workspace_bytes),
                               _stream(stream)))
    return C


def sr_weight_update(w, g, v, w8, n, lr, momentum, weight_decay, seed, offset, stream=None):
    """The C-ABI call with the same argument order; w, g, v, w8 are tensors
    (v, w8 may be None)."""
    _check("sr_weight_update",
           lib().sr_weight_update(_ptr(w), _ptr(g), _ptr(v), _ptr(w8), int(n), float(lr),
                                  float(momentum), float(weight_decay), int(seed), int(offset),
                                  _stream(stream)))
    return w


def adam_update(w, g, m, v, w8, n, lr, beta1, beta2, eps, weight_decay, t, seed, offset,
                stream=None):
    """The C-ABI call with the same argument order; w8 may be None."""
    _check("adam_update",
           lib().adam_update(_ptr(w), _ptr(g), _ptr(m), _ptr(v), _ptr(w8), int(n), float(lr),
                             float(beta1), float(beta2), float(eps), float(weight_decay), int(t),
                             int(seed), int(offset), _stream(stream)))
    return w


def chunk_gemm_p16_workspace_size(trans_a, trans_b, M, N, K, CL):
    return int(lib().chunk_gemm_p16_workspace_size(int(trans_a), int(trans_b), int(M), int(N),
                                                   int(K), int(CL)))


def chunk_gemm_p16(trans_a, trans_b, M, N, K, CL, A, lda, B, ldb, C, ldc, workspace=None,
                   workspace_bytes=0, stream=None):
    """The C-ABI call with the same argument order (FP16-code operands)."""
    _check("chunk_gemm_p16",
           lib().chunk_gemm_p16(int(trans_a), int(trans_b), int(M), int(N), int(K), int(CL),
                                _ptr(A), int(lda), _ptr(B), int(ldb), _ptr(C), int(ldc),
                                _ptr(workspace), int(workspace_bytes), _stream(stream)))
    return C


def relu_codes(x, fmt, y, n, stream=None):
    """ReLU on FP8 (fmt 8) or FP16 (fmt 16) codes; y may be x."""
    _check("relu_codes", lib().relu_codes(_ptr(x), int(fmt), _ptr(y), int(n), _stream(stream)))
    return y


def relu_backward_fp8(d, z, e, n, scale=1.0, stream=None):
    _check("relu_backward_fp8", lib().relu_backward_fp8(_ptr(d), _ptr(z), _ptr(e), int(n),
                                                        float(scale), _stream(stream)))
    return e


def mse_grad_fp16(y, t, e, n, scale, stream=None):
    _check("mse_grad_fp16", lib().mse_grad_fp16(_ptr(y), _ptr(t), _ptr(e), int(n), float(scale),
                                                _stream(stream)))
    return e


def conv2d_workspace_size(wgrad, N, H, W, C, KH, KW, pad, stride, Cout, CL):
    return int(lib().conv2d_workspace_size(int(wgrad), int(N), int(H), int(W), int(C), int(KH),
                                           int(KW), int(pad), int(stride), int(Cout), int(CL)))


def conv2d_fwd_fp8(X, N, H, W, C, KH, KW, pad, stride, Wt, Cout, CL, Y, ldy, workspace=None,
                   workspace_bytes=0, stream=None):
    _check("conv2d_fwd_fp8",
           lib().conv2d_fwd_fp8(_ptr(X), int(N), int(H), int(W), int(C), int(KH), int(KW),
                                int(pad), int(stride), _ptr(Wt), int(Cout), int(CL), _ptr(Y),
                                int(ldy), _ptr(workspace), int(workspace_bytes), _stream(stream)))
    return Y


def conv2d_wgrad_fp8(X, N, H, W, C, KH, KW, pad, stride, dY, Cout, CL, dW, lddw, workspace=None,
                     workspace_bytes=0, stream=None):
    _check("conv2d_wgrad_fp8",
           lib().conv2d_wgrad_fp8(_ptr(X), int(N), int(H), int(W), int(C), int(KH), int(KW),
                                  int(pad), int(stride), _ptr(dY), int(Cout), int(CL), _ptr(dW),
                                  int(lddw), _ptr(workspace), int(workspace_bytes),
                                  _stream(stream)))
    return dW


def col2im_fp16(cols, N, H, W, C, KH, KW, pad, stride, dX, stream=None):
    _check("col2im_fp16",
           lib().col2im_fp16(_ptr(cols), int(N), int(H), int(W), int(C), int(KH), int(KW),
                             int(pad), int(stride), _ptr(dX), _stream(stream)))
    return dX


# ---- language-model operators (include/fp8train_lm.h) ------------------------------
#
# Tensors carry their sizes and strides here: T x H x D arrays may be any views
# whose last dimension is contiguous.

_formats = None


def _format(fn, t, allowed):
    global _formats
    if _formats is None:
        import torch
        _formats = {torch.float32: FMT_F32, torch.uint16: FMT_FP16, torch.uint8: FMT_FP8,
                    torch.float16: FMT_HALF}
    fmt = _formats.get(t.dtype)
    if fmt not in allowed:
        raise TypeError(f"{fn}: a tensor of type {t.dtype} is not taken here")
    return fmt


def _rows(fn, t, like, dtype):
    """(address, token stride, head stride) of a T x H x D tensor of the shape
    `like`."""
    if t.shape != like:
        raise ValueError(f"{fn}: shape {tuple(t.shape)} where {tuple(like)} is needed")
    if t.dtype != dtype:
        raise TypeError(f"{fn}: {t.dtype} where {dtype} is needed")
    ts, hs, ds = t.stride()
    if ds != 1 and like[2] > 1 and t.numel():      # an empty tensor may have any strides
        raise ValueError(f"{fn}: the last dimension must be contiguous")
    return t.data_ptr(), ts, hs


def _dense(fn, t, shape, dtype):
    if t.shape != shape or t.dtype != dtype or not t.is_contiguous():
        raise ValueError(f"{fn}: a contiguous {dtype} tensor of shape {tuple(shape)} is needed")
    return t.data_ptr()


def fp16_dequantize(src, dst, scale=1.0, stream=None):
    """dst (float32 or float16) = value of the FP16 codes src, times scale."""
    import torch
    fmt = _format("fp16_dequantize", dst, (FMT_F32, FMT_HALF))
    if src.dtype != torch.uint16 or dst.numel() != src.numel():
        raise TypeError("fp16_dequantize: uint16 src, dst of the same size")
    if not (src.is_contiguous() and dst.is_contiguous()):
        raise ValueError("fp16_dequantize: tensors must be contiguous")
    _check("fp16_dequantize", lib().fp16_dequantize(_ptr(src), float(scale), _ptr(dst), fmt,
                                                    src.numel(), _stream(stream)))
    return dst


def rotary_embed(x, positions, freqs, y, interleaved=False, inverse=False, mscale=1.0, scale=1.0,
                 stream=None):
    """y = x with the first 2 * len(freqs) entries of every head turned by
    positions * freqs; x, y: T x H x D (float32, FP16 or FP8 codes), positions:
    T int64, freqs: R/2 float64.  y may be x."""
    import torch
    fn, any_fmt, shape = "rotary_embed", (FMT_F32, FMT_FP16, FMT_FP8), x.shape
    T, H, D = shape
    xp, x_ts, x_hs = _rows(fn, x, shape, x.dtype)
    yp, y_ts, y_hs = _rows(fn, y, shape, y.dtype)
    pairs = freqs.numel()
    _check(fn, lib().rotary_embed(
        xp, _format(fn, x, any_fmt), x_ts, x_hs, _dense(fn, positions, (T,), torch.int64),
        _dense(fn, freqs, (pairs,), torch.float64), T, H, D, 2 * pairs, int(interleaved),
        int(inverse), float(mscale), float(scale), yp, _format(fn, y, any_fmt), y_ts, y_hs,
        _stream(stream)))
    return y


def _attn_operands(fn, q, k, v, cu_q, cu_k, max_q, max_k, causal, sm_scale):
    import torch
    u8, i64 = torch.uint8, torch.int64
    Tq, Hq, D = q.shape
    Tk, Hkv, Dk = k.shape
    if D != Dk:
        raise ValueError(f"{fn}: q and k have different head dimensions")
    offsets = cu_q.shape
    return (*_rows(fn, q, q.shape, u8), *_rows(fn, k, k.shape, u8), *_rows(fn, v, k.shape, u8),
            _dense(fn, cu_q, offsets, i64), _dense(fn, cu_k, offsets, i64), offsets[0] - 1, Tq, Tk,
            int(max_q), int(max_k), Hq, Hkv, D, int(causal), float(sm_scale))


def attn_fwd_fp8_workspace_size(q, k, v, cu_q, cu_k, max_q, max_k, causal, sm_scale):
    return int(lib().attn_fwd_fp8_workspace_size(
        cu_q.numel() - 1, q.shape[0], k.shape[0], int(max_q), int(max_k), q.shape[1], k.shape[1],
        q.shape[2], int(causal)))


def attn_bwd_fp8_workspace_size(q, k, v, cu_q, cu_k, max_q, max_k, causal, sm_scale):
    return int(lib().attn_bwd_fp8_workspace_size(
        cu_q.numel() - 1, q.shape[0], k.shape[0], int(max_q), int(max_k), q.shape[1], k.shape[1],
        q.shape[2], int(causal)))


def attn_fwd_fp8(q, k, v, cu_q, cu_k, max_q, max_k, causal, sm_scale, o, o8, o8_scale=1.0,
                 lse=None, workspace=None, workspace_bytes=0, stream=None):
    """Attention of FP8 codes q (Tq x Hq x D) over k, v (Tk x Hkv x D), packed
    by the int64 offsets cu_q, cu_k; o (FP16 codes), o8 (FP8 codes) and lse
    (float32, Hq x Tq) are each optional."""
    import torch
    fn = "attn_fwd_fp8"
    none = (None, 0, 0)
    _check(fn, lib().attn_fwd_fp8(
        *_attn_operands(fn, q, k, v, cu_q, cu_k, max_q, max_k, causal, sm_scale),
        *(none if o is None else _rows(fn, o, q.shape, torch.uint16)),
        *(none if o8 is None else _rows(fn, o8, q.shape, torch.uint8)), float(o8_scale),
        None if lse is None else _dense(fn, lse, (q.shape[1], q.shape[0]), torch.float32),
        _ptr(workspace), int(workspace_bytes), _stream(stream)))
    return o8 if o is None else o


def attn_bwd_fp8(q, k, v, cu_q, cu_k, max_q, max_k, causal, sm_scale, o, d_o, lse, dq, dk, dv,
                 grad_scale=1.0, workspace=None, workspace_bytes=0, stream=None):
    """Gradients dq, dk, dv (all FP16 or all FP8 codes) from attn_fwd_fp8's o
    (FP16 codes) and lse and the error d_o of o (FP8 codes)."""
    import torch
    fn = "attn_bwd_fp8"
    fmt = _format(fn, dq, (FMT_FP16, FMT_FP8))
    _check(fn, lib().attn_bwd_fp8(
        *_attn_operands(fn, q, k, v, cu_q, cu_k, max_q, max_k, causal, sm_scale),
        *_rows(fn, o, q.shape, torch.uint16), *_rows(fn, d_o, q.shape, torch.uint8),
        _dense(fn, lse, (q.shape[1], q.shape[0]), torch.float32),
        *_rows(fn, dq, q.shape, dq.dtype), *_rows(fn, dk, k.shape, dq.dtype),
        *_rows(fn, dv, k.shape, dq.dtype), fmt, float(grad_scale), _ptr(workspace),
        int(workspace_bytes), _stream(stream)))
    return dq, dk, dv


def distill_loss(z, idx, t, w, tau, grad_scale, loss, g, stream=None):
    """Distillation loss of logits z (N x V, float32 or FP16 codes) against a
    teacher's entries idx, t (N x k): loss (float32, N) and the gradient g
    (N x V: float32, FP16 or FP8 codes; may be z); either may be None, and w
    (float32 row weights) too."""
    import torch
    fn = "distill_loss"
    N, V = z.shape
    k = idx.shape[1]

    def matrix(m, allowed):
        if m.shape != z.shape or (N > 0 and V > 1 and m.stride(1) != 1):
            raise ValueError(f"{fn}: an N x V tensor with contiguous rows is needed")
        return m.data_ptr(), _format(fn, m, allowed), max(m.stride(0), V if N <= 1 else 0)
    _check(fn, lib().distill_loss(
        *matrix(z, (FMT_F32, FMT_FP16)), _dense(fn, idx, (N, k), torch.int64),
        _dense(fn, t, (N, k), t.dtype), _format(fn, t, (FMT_F32, FMT_FP16)), k,
        None if w is None else _dense(fn, w, (N,), torch.float32), N, V, float(tau),
        float(grad_scale), None if loss is None else _dense(fn, loss, (N,), torch.float32),
        *((None, FMT_F32, 0) if g is None else matrix(g, (FMT_F32, FMT_FP16, FMT_FP8))),
        _stream(stream)))
    return g


# ---- operators on tokens and rows (include/fp8train_tokens.h) ------------------------
#
# Matrices may be any views whose rows are contiguous.  Tensors have to be on the
# current device: an address that the GPU cannot reach would end the process.

_ANY, _FLOATS = (FMT_F32, FMT_FP16, FMT_FP8), (FMT_F32, FMT_FP16)
_NONE = (None, FMT_F32, 0)


def _matrix(fn, t, shape, allowed):
    """(address, format, row stride) of a matrix; (None, FMT_F32, 0) of None."""
    if t is None:
        return _NONE
    fmt = _format(fn, t, allowed)
    if t.shape != shape:
        raise ValueError(f"{fn}: shape {tuple(t.shape)} where {tuple(shape)} is needed")
    if t.is_contiguous():
        return t.data_ptr(), fmt, shape[1]
    ld, inner = t.stride()
    if inner != 1 and shape[1] > 1 and shape[0] > 0:
        raise ValueError(f"{fn}: rows must be contiguous")
    return t.data_ptr(), fmt, ld if shape[0] > 1 else max(ld, shape[1])


def _vector(fn, t, n, allowed):
    """(address, format) of n contiguous elements; (None, FMT_F32) of None."""
    if t is None:
        return None, FMT_F32
    fmt = _format(fn, t, allowed)
    if t.shape != (n,) or not t.is_contiguous():
        raise ValueError(f"{fn}: {n} contiguous elements are needed")
    return t.data_ptr(), fmt


def _array(fn, t, shape, dtype):
    """The address of a contiguous array of a dtype named like torch's, or None."""
    return None if t is None else _dense(fn, t, shape, getattr(_torch(), dtype))


def _torch():
    import torch
    return torch


def _same_type(fn, a, b):
    """The format that two optional matrices of one type share."""
    if a[0] is not None and b[0] is not None and a[1] != b[1]:
        raise TypeError(f"{fn}: two tensors of one type are needed")
    return b[1] if a[0] is None else a[1]


def _space(fn, workspace, workspace_bytes):
    if workspace is None or isinstance(workspace, int):
        return workspace, int(workspace_bytes)
    if workspace_bytes > workspace.numel() * workspace.element_size():
        raise ValueError(f"{fn}: the workspace holds fewer than {workspace_bytes} bytes")
    return workspace.data_ptr(), int(workspace_bytes)


def _place(fn, stream, workspace, *tensors):
    """The stream to work on, once all tensors are known to be on one GPU, the
    current one."""
    dev = tensors[0].get_device()
    if not isinstance(workspace, int):
        tensors += (workspace,)
    for t in tensors:
        if t is not None and (t.get_device() != dev or dev < 0):
            raise ValueError(f"{fn}: all tensors have to be on one GPU (one is on {t.device})")
    torch = _torch()
    if dev != torch.cuda.current_device():
        raise ValueError(f"{fn}: the tensors are on GPU {dev}, which is not the current one")
    return _stream(stream)


def embed_fwd(tokens, table, y, scale=1.0, stream=None):
    """y (T x W) = rows of the table (V x W) by tokens (T int64), times scale;
    each float32, FP16 or FP8 codes.  Tokens outside [0, V) give rows of 0."""
    fn, T, shape = "embed_fwd", tokens.numel(), table.shape
    V, W = shape
    tp, tf, t_ld = _matrix(fn, table, shape, _ANY)
    args = (_array(fn, tokens, (T,), "int64"), T, tp, tf, t_ld, V, W, scale,
            *_matrix(fn, y, (T, W), _ANY), _place(fn, stream, None, y, table, tokens))
    _check(fn, lib().embed_fwd(*args))
    return y


def embed_bwd_workspace_size(tokens, e, g):
    return int(lib().embed_bwd_workspace_size(tokens.numel(), *g.shape))


def embed_bwd(tokens, e, g, scale=1.0, workspace=None, workspace_bytes=0, stream=None):
    """g (V x W): the sum of scale * e[t] over the t with tokens[t] = v, for
    every v; e: T x W."""
    fn, T, shape = "embed_bwd", tokens.numel(), g.shape
    V, W = shape
    args = (_array(fn, tokens, (T,), "int64"), T, *_matrix(fn, e, (T, W), _ANY), V, W, scale,
            *_matrix(fn, g, shape, _ANY), *_space(fn, workspace, workspace_bytes),
            _place(fn, stream, workspace, g, e, tokens))
    _check(fn, lib().embed_bwd(*args))
    return g


def rms_norm_fwd(x, r, w, eps, h, y, y_scale=1.0, y_row_scale=None, rstd=None, x_row_scale=None,
                 stream=None):
    """h = x + r (T x W, float32 or FP16 codes; r and h of one type) and y =
    h / rms(h) w times y_scale, or times a scale of each row's own that brings
    its largest result to y_scale and is written to y_row_scale.  r, w, h, y and
    the float32 vectors may be None; h may be r or x itself."""
    fn, shape = "rms_norm_fwd", x.shape
    T, W = shape
    rm, hm = _matrix(fn, r, shape, _FLOATS), _matrix(fn, h, shape, _FLOATS)
    args = (*_matrix(fn, x, shape, _FLOATS), _array(fn, x_row_scale, (T,), "float32"), rm[0], rm[2],
            *_vector(fn, w, W, _FLOATS), T, W, eps, hm[0], _same_type(fn, rm, hm), hm[2],
            *_matrix(fn, y, shape, _ANY), y_scale, _array(fn, y_row_scale, (T,), "float32"),
            _array(fn, rstd, (T,), "float32"),
            _place(fn, stream, None, x, r, w, h, y, x_row_scale, y_row_scale, rstd))
    _check(fn, lib().rms_norm_fwd(*args))
    return h if y is None else y


def rms_norm_bwd_workspace_size(h):
    return int(lib().rms_norm_bwd_workspace_size(*h.shape))


def rms_norm_bwd(h, w, rstd, dy, dr, dx, dx8=None, dx8_scale=1.0, dw=None, workspace=None,
                 workspace_bytes=0, stream=None):
    """Gradients of rms_norm_fwd from its h and rstd and the error dy of the
    normed rows: dx (of h, with dr, the error that reaches h past the norm, of
    the same type; may be dr), dx8 (the same in FP8 times dx8_scale) and dw."""
    fn, shape = "rms_norm_bwd", h.shape
    T, W = shape
    rm, xm = _matrix(fn, dr, shape, _FLOATS), _matrix(fn, dx, shape, _FLOATS)
    x8 = _matrix(fn, dx8, shape, (FMT_FP8,))
    args = (*_matrix(fn, h, shape, _FLOATS), *_vector(fn, w, W, _FLOATS),
            _array(fn, rstd, (T,), "float32"), *_matrix(fn, dy, shape, _ANY), rm[0], rm[2], T, W, xm[0],
            _same_type(fn, rm, xm), xm[2], x8[0], x8[2], dx8_scale, *_vector(fn, dw, W, _FLOATS),
            *_space(fn, workspace, workspace_bytes),
            _place(fn, stream, workspace, h, w, rstd, dy, dr, dx, dx8, dw))
    _check(fn, lib().rms_norm_bwd(*args))
    return dx


def token_logprobs_workspace_size(z, k):
    return int(lib().token_logprobs_workspace_size(*z.shape, int(k)))


def token_logprobs(z, idx, tau=1.0, logp=None, entropy=None, stats=None, top_idx=None,
                   top_logp=None, workspace=None, workspace_bytes=0, stream=None):
    """Log probabilities logp (N x m) of the tokens idx (N x m int64) under
    softmax(z / tau), z: N x V float32 or FP16 codes; entropy (N), stats (N x 2:
    what token_logprobs_bwd takes) and the likeliest tokens top_idx (N x k
    int64) with their top_logp (N x k).  Results that are None are not formed."""
    fn, shape = "token_logprobs", z.shape
    N, V = shape
    m = 0 if idx is None else idx.shape[1]
    top = top_logp if top_idx is None else top_idx
    k = 0 if top is None else top.shape[1]
    args = (*_matrix(fn, z, shape, _FLOATS), _array(fn, idx, (N, m), "int64"), m, N, V, tau,
            _array(fn, logp, (N, m), "float32"), _array(fn, entropy, (N,), "float32"),
            _array(fn, stats, (N, 2), "float32"), k, _array(fn, top_idx, (N, k), "int64"),
            _array(fn, top_logp, (N, k), "float32"), *_space(fn, workspace, workspace_bytes),
            _place(fn, stream, workspace, z, idx, logp, entropy, stats, top_idx, top_logp))
    _check(fn, lib().token_logprobs(*args))
    return logp


def token_logprobs_bwd(z, idx, tau, stats, entropy, d_logp, d_entropy, grad_scale, g, stream=None):
    """g (N x V: float32, FP16 or FP8 codes; may be z): the logits' gradient
    times grad_scale from those of token_logprobs' logp (N x m) and entropy (N),
    either None, and its stats and entropy."""
    fn, shape = "token_logprobs_bwd", z.shape
    N, V = shape
    m = 0 if idx is None else idx.shape[1]
    args = (*_matrix(fn, z, shape, _FLOATS), _array(fn, idx, (N, m), "int64"), m,
            _array(fn, stats, (N, 2), "float32"), _array(fn, entropy, (N,), "float32"),
            _array(fn, d_logp, (N, m), "float32"), _array(fn, d_entropy, (N,), "float32"), N, V, tau,
            grad_scale, *_matrix(fn, g, shape, _ANY),
            _place(fn, stream, None, z, idx, stats, entropy, d_logp, d_entropy, g))
    _check(fn, lib().token_logprobs_bwd(*args))
    return g
