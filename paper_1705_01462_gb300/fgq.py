"""Python binding of libfgq (the FGQ CUDA library): argument marshalling only.

Every function here checks tensor dtypes/devices, passes raw device pointers, sizes and
the current CUDA stream to the C ABI of ``include/fgq.h`` (and ``include/fgq_decoder.h``) and raises on
a non-OK status.
All computation happens in the library's CUDA kernels; there is no CPU fallback, and
loading fails loudly if the library is missing or CUDA is unavailable.
"""
from __future__ import annotations

import ctypes
import os
from typing import Optional, Tuple

import torch

_HERE = os.path.dirname(os.path.abspath(__file__))
LIB_PATH = os.path.join(_HERE, "libfgq.so")

FGQ_OK, FGQ_ERR_ARG, FGQ_ERR_ALIGN, FGQ_ERR_UNSUPPORTED, FGQ_ERR_NONFINITE, FGQ_ERR_TIMEOUT, FGQ_ERR_CUDA = range(7)
U8, S8, U4, S4 = 0, 1, 2, 3
PATH_AUTO, PATH_SIMT, PATH_TC, PATH_GEMV, PATH_DENSE = 0, 1, 2, 3, 4
ACT_TYPES = {"u8": U8, "s8": S8, "u4": U4, "s4": S4}

F32, BF16, F16 = 0, 1, 2
FLOAT_TYPES = {torch.float32: F32, torch.bfloat16: BF16, torch.float16: F16}

_lib: Optional[ctypes.CDLL] = None

# (name, restype, argtypes) of every exported symbol of include/fgq.h, fgq_decoder.h and fgq_debug.h
_vp, _i, _i64, _u32, _u64, _f, _sz = (ctypes.c_void_p, ctypes.c_int, ctypes.c_int64, ctypes.c_uint32,
                                      ctypes.c_uint64, ctypes.c_float, ctypes.c_size_t)
SIGNATURES = [
    ("fgq_version", _i, []),
    ("fgq_status_string", ctypes.c_char_p, [_i]),
    ("fgq_codes_words_per_row", _i64, [_i, _i]),
    ("fgq_num_groups", _i64, [_i, _i]),
    ("fgq_ternarize", _i, [_vp, _i, _i, _i, _vp, _vp, _vp]),
    ("fgq_ternarize_batch", _i, [_i, _vp, _vp, _vp, _i, _vp, _vp, _vp]),
    ("fgq_ternarize_threshold_workspace_bytes", _sz, []),
    ("fgq_ternarize_threshold", _i, [_vp, _i, _i, _i, _i, _i, _vp, _vp, _vp, _sz, _vp, _vp]),
    ("fgq_ternary_error", _i, [_vp, _i, _i, _i, _vp, _vp, _vp, _vp]),
    ("fgq_quantize_act_workspace_bytes", _sz, [_sz]),
    ("fgq_quantize_act", _i, [_vp, _sz, _i, _f, _vp, _vp, _vp, _sz, _vp]),
    ("fgq_quantize_act_noalloc", _i, [_vp, _sz, _i, _f, _vp, _vp, _vp]),
    ("fgq_quantize_act_batch_workspace_bytes", _sz, [_i]),
    ("fgq_quantize_act_batch", _i, [_i, _vp, _vp, _vp, _vp, _vp, _vp, _sz, _vp]),
    ("fgq_quantize_weights_w8", _i, [_vp, _i, _i, _vp, _vp, _vp]),
    ("fgq_gemm", _i, [_vp, _i, _vp, _i, _i, _vp, _vp, _i, _i, _vp, _vp]),
    ("fgq_conv2d", _i, [_vp, _i, _vp] + [_i] * 9 + [_vp, _vp, _i, _i, _vp, _vp]),
    ("fgq_conv2d_w8", _i, [_vp, _i, _vp] + [_i] * 9 + [_vp, _vp, _i, _vp, _vp]),
    ("fgq_quantize_alpha", _i, [_vp, _i, _i, _i, _vp, _vp, _vp]),
    ("fgq_conv2d_w8_rq", _i, [_vp, _i, _vp] + [_i] * 9 + [_vp, _vp, _i, _i, _vp, _vp, _vp]),
    ("fgq_maxpool_u8", _i, [_vp] + [_i] * 7 + [_vp, _vp]),
    ("fgq_add_codes", _i, [_vp, _i, _vp, _vp, _i, _vp, _sz, _vp, _i, _vp, _vp, _vp]),
    ("fgq_gemm_rq", _i, [_vp, _i, _vp, _i, _i, _vp, _vp, _i, _i, _i, _vp, _vp, _vp]),
    ("fgq_conv2d_rq", _i, [_vp, _i, _vp] + [_i] * 9 + [_vp, _vp, _i, _i, _i, _vp, _vp, _vp]),
    ("fgq_gemm_qa", _i, [_vp, _i, _vp, _i, _i, _vp, _vp, _i, _vp, _i, _i, _vp, _vp]),
    ("fgq_conv2d_qa", _i, [_vp, _i, _vp] + [_i] * 9 + [_vp, _vp, _i, _vp, _i, _i, _vp, _vp]),
    ("fgq_group_sums", _i, [_vp, _i, _i, _i, _vp, _i, _i, _vp, _vp]),
    ("fgq_conv2d_group_sums", _i, [_vp, _i] + [_i] * 9 + [_vp, _i, _i, _vp, _vp]),
    ("fgq_conv2d_host_workspace_bytes", _sz, [_i] * 12),
    ("fgq_conv2d_host", _i, [_vp, _vp, _i] + [_i] * 11 + [_vp, _vp, _sz, _vp]),
    ("fgq_kv_append", _i, [_vp, _vp, _vp, _i, _i, _i, _i64, _i64, _i64, _i64, _vp, _i, _vp, _vp, _vp]),
    ("fgq_kv_read", _i, [_vp, _vp, _vp, _i, _i, _i, _vp, _i, _vp, _vp, _vp]),
    ("fgq_kv_attention", _i, [_vp, _vp, _i, _i, _i, _i, _i64, _i64, _vp, _i, _vp, _vp, _i, _i, _i, _f, _vp, _vp]),
    ("fgq_quantize_tokens", _i, [_vp, _i, _i, _i, _i64, _vp, _vp, _vp]),
    ("fgq_gemm_w8a8", _i, [_vp, _vp, _i, _i, _vp, _vp, _i, _vp, _vp, _i, _vp]),
    ("fgq_linear_w8a8", _i, [_vp, _i, _i, _i, _i64, _vp, _vp, _i, _vp, _vp, _vp]),
    ("fgq_stream_status", _i, [_vp]),
    ("fgq_set_path", _i, [_i]),
    ("fgq_last_path", _i, []),
    ("fgq_launch_count", _u64, []),
    ("fgq_selftest_wait_timeout", _i, [_u32, _vp]),
    ("fgq_debug_set_wait_limit_us", _i64, [_i64]),
    ("fgq_debug_set_scratch_limit", _i64, [_i64]),
    ("fgq_debug_set_resident_blocks", _i64, [_i64]),
    ("fgq_debug_set_attention_kernel", _i, [_i]),
    ("fgq_debug_allow_split_fold", _i, [_i]),
    ("fgq_debug_selftest_warp_wait", _i, [_u32, _vp]),
    ("fgq_debug_last_cuda_error", _i, [_vp, _sz]),
    ("fgq_debug_cta_pairs", _i, [_i]),
    ("fgq_debug_max_ksplit", _i, [_i]),
    ("fgq_debug_last_ksplit", _i, []),
]


class FGQError(RuntimeError):
    def __init__(self, code: int, what: str):
        name = lib().fgq_status_string(code).decode() if _lib is not None else str(code)
        super().__init__(f"{what}: {name}")
        self.code = code


def load(path: str = LIB_PATH) -> ctypes.CDLL:
    """Load libfgq.so (built by paper_1705_01462_gb300.build) and declare its signatures."""
    if not os.path.exists(path):
        raise RuntimeError(f"libfgq.so not found at {path}: build it with "
                           "`python -c 'import __graft_entry__ as g; g.build()'` (no CPU fallback exists)")
    L = ctypes.CDLL(path)
    for name, res, args in SIGNATURES:
        fn = getattr(L, name)
        fn.restype = res
        fn.argtypes = args
    return L


def lib() -> ctypes.CDLL:
    global _lib
    if _lib is None:
        _lib = load()
    return _lib


_have_cuda = False


def _require_cuda():
    global _have_cuda
    if _have_cuda:
        return
    if not torch.cuda.is_available():
        raise RuntimeError("libfgq needs a CUDA GPU; there is no CPU fallback")
    _have_cuda = True


def _check(code: int, what: str):
    if code != FGQ_OK:
        raise FGQError(code, what)


# The raw handle of the current stream (0.1 us; torch.cuda.current_stream builds a Stream object
# each time, 2.9 us a call).
_raw_stream = getattr(torch._C, "_cuda_getCurrentRawStream", None)
_get_device = getattr(torch._C, "_cuda_getDevice", None)


def _stream(stream=None) -> int:
    if stream is not None:
        return stream.cuda_stream
    if _raw_stream is None or _get_device is None:
        return torch.cuda.current_stream().cuda_stream
    return _raw_stream(_get_device())


def _dev(t: torch.Tensor, dtype, name: str) -> int:
    if isinstance(t, torch.Tensor) and t.is_cuda and t.dtype == dtype and t.is_contiguous():
        return t.data_ptr()
    if not isinstance(t, torch.Tensor) or not t.is_cuda:
        raise TypeError(f"{name} must be a CUDA tensor")
    if t.dtype != dtype:
        raise TypeError(f"{name} must be {dtype}, got {t.dtype}")
    raise ValueError(f"{name} must be contiguous")


def _act_type(t) -> int:
    return ACT_TYPES[t] if isinstance(t, str) else int(t)


# --------------------------------------------------------------------------- sizes

def codes_words_per_row(Kred: int, G: int) -> int:
    return int(lib().fgq_codes_words_per_row(Kred, G))


def num_groups(Kred: int, G: int) -> int:
    return int(lib().fgq_num_groups(Kred, G))


_GROUP_SIZES = frozenset((1, 2, 4, 8, 16, 32, 64, 128))


def _row_sizes(Kred: int, G: int) -> Tuple[int, int]:
    """(code words, groups) per filter row; the library's own answer (0) for a bad G."""
    if G in _GROUP_SIZES:
        ng = (Kred + G - 1) // G
        return (ng * G + 15) // 16, ng
    return codes_words_per_row(Kred, G), num_groups(Kred, G)


def quantize_act_workspace_bytes(n: int) -> int:
    return int(lib().fgq_quantize_act_workspace_bytes(n))


def act_bytes(n: int, act_type) -> int:
    return n if _act_type(act_type) in (U8, S8) else (n + 1) // 2


# --------------------------------------------------------------------------- calls

def fgq_ternarize(w: torch.Tensor, G: int, codes: Optional[torch.Tensor] = None,
                  alpha: Optional[torch.Tensor] = None, stream=None) -> Tuple[torch.Tensor, torch.Tensor]:
    """w fp32 [M][Kred] -> (codes int32-view of uint32 [M][words], alpha fp32 [M][ng])."""
    _require_cuda()
    M, Kred = w.shape
    words, ng = _row_sizes(Kred, G)
    if codes is None:
        codes = torch.empty((M, words), dtype=torch.int32, device=w.device)
    if alpha is None:
        alpha = torch.empty((M, ng), dtype=torch.float32, device=w.device)
    _check(lib().fgq_ternarize(_dev(w, torch.float32, "w"), M, Kred, G, _dev(codes, torch.int32, "codes"),
                               _dev(alpha, torch.float32, "alpha"), _stream(stream)), "fgq_ternarize")
    return codes, alpha


RULE_EXP, RULE_GAUSS = 0, 1


def fgq_ternarize_batch(ws, G: int, stream=None):
    """fgq_ternarize of every fp32 [M][Kred] tensor in ws (one group size, one launch) ->
    list of (codes, alpha)."""
    _require_cuda()
    n = len(ws)
    VP, I = ctypes.c_void_p * max(n, 1), ctypes.c_int * max(n, 1)
    tw, tm, tk, tc, ta = VP(), I(), I(), VP(), VP()
    outs = []
    for i, w in enumerate(ws):
        M, Kred = w.shape
        words, ng = _row_sizes(Kred, G)
        tw[i], tm[i], tk[i] = _dev(w, torch.float32, "w"), M, Kred
        codes = torch.empty((M, words), dtype=torch.int32, device=w.device)
        alpha = torch.empty((M, ng), dtype=torch.float32, device=w.device)
        tc[i], ta[i] = codes.data_ptr(), alpha.data_ptr()
        outs.append((codes, alpha))
    _check(lib().fgq_ternarize_batch(n, tw, tm, tk, G, tc, ta, _stream(stream)), "fgq_ternarize_batch")
    return outs


def fgq_ternarize_threshold(w: torch.Tensor, G: int, rule: int, per_layer: bool = False, stream=None):
    """Analytical-threshold ternarization: w fp32 [M][Kred] -> (codes, alpha, delta); delta is a
    device fp64 [1] tensor for per_layer, else None."""
    _require_cuda()
    M, Kred = w.shape
    codes = torch.empty((M, codes_words_per_row(Kred, G)), dtype=torch.int32, device=w.device)
    alpha = torch.empty((M, num_groups(Kred, G)), dtype=torch.float32, device=w.device)
    ws, wsb, delta = None, 0, None
    if per_layer:
        wsb = lib().fgq_ternarize_threshold_workspace_bytes()
        ws = torch.empty(wsb, dtype=torch.uint8, device=w.device)
        delta = torch.empty(1, dtype=torch.float64, device=w.device)
    _check(lib().fgq_ternarize_threshold(_dev(w, torch.float32, "w"), M, Kred, G, rule, int(per_layer),
                                         _dev(codes, torch.int32, "codes"), _dev(alpha, torch.float32, "alpha"),
                                         ws.data_ptr() if ws is not None else None, wsb,
                                         delta.data_ptr() if delta is not None else None, _stream(stream)),
           "fgq_ternarize_threshold")
    return codes, alpha, delta


def fgq_ternary_error(w: torch.Tensor, codes: torch.Tensor, alpha: torch.Tensor, G: int, stream=None) -> torch.Tensor:
    """Per-group ||w - alpha t||^2, device fp64 [M][ng]."""
    _require_cuda()
    M, Kred = w.shape
    err = torch.empty((M, num_groups(Kred, G)), dtype=torch.float64, device=w.device)
    _check(lib().fgq_ternary_error(_dev(w, torch.float32, "w"), M, Kred, G, _dev(codes, torch.int32, "codes"),
                                   _dev(alpha, torch.float32, "alpha"), err.data_ptr(), _stream(stream)),
           "fgq_ternary_error")
    return err


def fgq_quantize_act(x: torch.Tensor, act_type="u8", scale_in: float = 0.0, q: Optional[torch.Tensor] = None,
                     scale_out: Optional[torch.Tensor] = None, workspace: Optional[torch.Tensor] = None,
                     stream=None) -> Tuple[torch.Tensor, torch.Tensor]:
    """fp32 tensor -> (codes uint8 [n or ceil(n/2)], scale fp32 [1] = 2^E)."""
    _require_cuda()
    ty = _act_type(act_type)
    n = x.numel()
    if q is None:
        q = torch.empty(act_bytes(n, ty), dtype=torch.uint8, device=x.device)
    if scale_out is None:
        scale_out = torch.empty(1, dtype=torch.float32, device=x.device)
        if scale_in > 0:
            scale_out.fill_(scale_in)
    wsb = quantize_act_workspace_bytes(n)
    if workspace is None and scale_in <= 0:
        workspace = torch.empty(max(wsb, 4), dtype=torch.uint8, device=x.device)
    ws_ptr = workspace.data_ptr() if workspace is not None else None
    ws_len = workspace.numel() * workspace.element_size() if workspace is not None else 0
    _check(lib().fgq_quantize_act(_dev(x, torch.float32, "x"), n, ty, float(scale_in), _dev(q, torch.uint8, "q"),
                                  _dev(scale_out, torch.float32, "scale_out") if scale_in <= 0 else None,
                                  ws_ptr, ws_len, _stream(stream)), "fgq_quantize_act")
    return q, scale_out


def fgq_quantize_act_batch(xs, act_types, stream=None):
    """fgq_quantize_act_batch over a list of fp32 device tensors with derived scales: returns
    [(q, scale)] in the same order (q packed as fgq_quantize_act's)."""
    _require_cuda()
    n = len(xs)
    types = [_act_type(t) for t in act_types]
    qs = [torch.empty(act_bytes(x.numel(), t), dtype=torch.uint8, device=x.device) for x, t in zip(xs, types)]
    scs = [torch.empty(1, dtype=torch.float32, device=x.device) for x in xs]
    ws = torch.empty(max(4, int(lib().fgq_quantize_act_batch_workspace_bytes(n))), dtype=torch.uint8,
                     device=xs[0].device if n else "cuda")
    arr = lambda ptrs: (ctypes.c_void_p * n)(*ptrs)
    px = arr([_dev(x, torch.float32, "x") for x in xs])
    _check(lib().fgq_quantize_act_batch(n, px, (ctypes.c_size_t * n)(*[x.numel() for x in xs]),
                                        (ctypes.c_int * n)(*types), arr([q.data_ptr() for q in qs]),
                                        arr([sc.data_ptr() for sc in scs]), ws.data_ptr(), ws.numel(),
                                        _stream(stream)), "fgq_quantize_act_batch")
    return list(zip(qs, scs))


def fgq_quantize_weights_w8(w: torch.Tensor, stream=None) -> Tuple[torch.Tensor, torch.Tensor]:
    _require_cuda()
    M, Kred = w.shape
    wq = torch.empty((M, Kred), dtype=torch.int8, device=w.device)
    ws = torch.empty(M, dtype=torch.float32, device=w.device)
    _check(lib().fgq_quantize_weights_w8(_dev(w, torch.float32, "w"), M, Kred, wq.data_ptr(), ws.data_ptr(),
                                         _stream(stream)), "fgq_quantize_weights_w8")
    return wq, ws


def fgq_gemm(q: torch.Tensor, act_type, act_scale: torch.Tensor, P: int, Kred: int, codes: torch.Tensor,
             alpha: torch.Tensor, M: int, G: int, y: Optional[torch.Tensor] = None, stream=None) -> torch.Tensor:
    _require_cuda()
    if y is None:
        y = torch.empty((P, M), dtype=torch.float32, device=q.device)
    _check(lib().fgq_gemm(_dev(q, torch.uint8, "q"), _act_type(act_type), _dev(act_scale, torch.float32, "act_scale"),
                          P, Kred, _dev(codes, torch.int32, "codes"), _dev(alpha, torch.float32, "alpha"), M, G,
                          _dev(y, torch.float32, "y"), _stream(stream)), "fgq_gemm")
    return y


def fgq_gemm_rq(q: torch.Tensor, act_type, act_scale: torch.Tensor, P: int, Kred: int, codes: torch.Tensor,
                alpha: torch.Tensor, M: int, G: int, out_type, out_scale: torch.Tensor,
                out_q: Optional[torch.Tensor] = None, stream=None) -> torch.Tensor:
    """fgq_gemm with the output requantized in the kernel: uint8 [P][M] codes at out_scale."""
    _require_cuda()
    if out_q is None:
        out_q = torch.empty((P, M), dtype=torch.uint8, device=q.device)
    _check(lib().fgq_gemm_rq(_dev(q, torch.uint8, "q"), _act_type(act_type), _dev(act_scale, torch.float32, "act_scale"),
                             P, Kred, _dev(codes, torch.int32, "codes"), _dev(alpha, torch.float32, "alpha"), M, G,
                             _act_type(out_type), _dev(out_scale, torch.float32, "out_scale"),
                             _dev(out_q, torch.uint8, "out_q"), _stream(stream)), "fgq_gemm_rq")
    return out_q


def fgq_conv2d_rq(act: torch.Tensor, act_type, act_scale: torch.Tensor, B: int, H: int, W: int, C: int, R: int,
                  S: int, stride: int, pad: int, groups: int, codes: torch.Tensor, alpha: torch.Tensor, M: int, G: int,
                  out_type, out_scale: torch.Tensor, out_q: Optional[torch.Tensor] = None, stream=None) -> torch.Tensor:
    """fgq_conv2d with the output requantized in the kernel: uint8 NHWC [B][Ho][Wo][M] codes."""
    _require_cuda()
    Ho, Wo = conv_out_hw(H, W, R, S, stride, pad)
    if out_q is None:
        out_q = torch.empty((B, Ho, Wo, M), dtype=torch.uint8, device=act.device)
    _check(lib().fgq_conv2d_rq(_dev(act, torch.uint8, "act"), _act_type(act_type),
                               _dev(act_scale, torch.float32, "act_scale"), B, H, W, C, R, S, stride, pad, groups,
                               _dev(codes, torch.int32, "codes"), _dev(alpha, torch.float32, "alpha"), M, G,
                               _act_type(out_type), _dev(out_scale, torch.float32, "out_scale"),
                               _dev(out_q, torch.uint8, "out_q"), _stream(stream)), "fgq_conv2d_rq")
    return out_q


def fgq_quantize_alpha(alpha: torch.Tensor, bits: int, stream=None) -> Tuple[torch.Tensor, torch.Tensor]:
    """Fixed-point alphas: fp32 [M][ng] -> (aq uint8 [M][ng] or [M][ceil(ng/2)], ascale fp32 [M])."""
    _require_cuda()
    M, ng = alpha.shape
    aq = torch.empty((M, ng if bits == 8 else (ng + 1) // 2), dtype=torch.uint8, device=alpha.device)
    ascale = torch.empty(M, dtype=torch.float32, device=alpha.device)
    _check(lib().fgq_quantize_alpha(_dev(alpha, torch.float32, "alpha"), M, ng, bits, _dev(aq, torch.uint8, "aq"),
                                    _dev(ascale, torch.float32, "ascale"), _stream(stream)), "fgq_quantize_alpha")
    return aq, ascale


def fgq_gemm_qa(q: torch.Tensor, act_type, act_scale: torch.Tensor, P: int, Kred: int, codes: torch.Tensor,
                aq: torch.Tensor, abits: int, ascale: torch.Tensor, M: int, G: int, y: Optional[torch.Tensor] = None,
                stream=None) -> torch.Tensor:
    _require_cuda()
    if y is None:
        y = torch.empty((P, M), dtype=torch.float32, device=q.device)
    _check(lib().fgq_gemm_qa(_dev(q, torch.uint8, "q"), _act_type(act_type), _dev(act_scale, torch.float32, "act_scale"),
                             P, Kred, _dev(codes, torch.int32, "codes"), _dev(aq, torch.uint8, "aq"), abits,
                             _dev(ascale, torch.float32, "ascale"), M, G, _dev(y, torch.float32, "y"), _stream(stream)),
           "fgq_gemm_qa")
    return y


def fgq_conv2d_qa(act: torch.Tensor, act_type, act_scale: torch.Tensor, B: int, H: int, W: int, C: int, R: int,
                  S: int, stride: int, pad: int, groups: int, codes: torch.Tensor, aq: torch.Tensor, abits: int,
                  ascale: torch.Tensor, M: int, G: int, out: Optional[torch.Tensor] = None, stream=None) -> torch.Tensor:
    _require_cuda()
    Ho, Wo = conv_out_hw(H, W, R, S, stride, pad)
    if out is None:
        out = torch.empty((B, Ho, Wo, M), dtype=torch.float32, device=act.device)
    _check(lib().fgq_conv2d_qa(_dev(act, torch.uint8, "act"), _act_type(act_type),
                               _dev(act_scale, torch.float32, "act_scale"), B, H, W, C, R, S, stride, pad, groups,
                               _dev(codes, torch.int32, "codes"), _dev(aq, torch.uint8, "aq"), abits,
                               _dev(ascale, torch.float32, "ascale"), M, G, _dev(out, torch.float32, "out"),
                               _stream(stream)), "fgq_conv2d_qa")
    return out


def conv_out_hw(H, W, R, S, stride, pad):
    return (H + 2 * pad - R) // stride + 1, (W + 2 * pad - S) // stride + 1


def fgq_conv2d(act: torch.Tensor, act_type, act_scale: torch.Tensor, B: int, H: int, W: int, C: int, R: int, S: int,
               stride: int, pad: int, groups: int, codes: torch.Tensor, alpha: torch.Tensor, M: int, G: int,
               out: Optional[torch.Tensor] = None, stream=None) -> torch.Tensor:
    _require_cuda()
    Ho, Wo = conv_out_hw(H, W, R, S, stride, pad)
    if out is None:
        out = torch.empty((B, Ho, Wo, M), dtype=torch.float32, device=act.device)
    _check(lib().fgq_conv2d(_dev(act, torch.uint8, "act"), _act_type(act_type),
                            _dev(act_scale, torch.float32, "act_scale"), B, H, W, C, R, S, stride, pad, groups,
                            _dev(codes, torch.int32, "codes"), _dev(alpha, torch.float32, "alpha"), M, G,
                            _dev(out, torch.float32, "out"), _stream(stream)), "fgq_conv2d")
    return out


def fgq_conv2d_w8(act: torch.Tensor, act_type, act_scale: torch.Tensor, B: int, H: int, W: int, C: int, R: int,
                  S: int, stride: int, pad: int, groups: int, wq: torch.Tensor, wscale: torch.Tensor, M: int,
                  out: Optional[torch.Tensor] = None, stream=None) -> torch.Tensor:
    _require_cuda()
    Ho, Wo = conv_out_hw(H, W, R, S, stride, pad)
    if out is None:
        out = torch.empty((B, Ho, Wo, M), dtype=torch.float32, device=act.device)
    _check(lib().fgq_conv2d_w8(_dev(act, torch.uint8, "act"), _act_type(act_type),
                               _dev(act_scale, torch.float32, "act_scale"), B, H, W, C, R, S, stride, pad, groups,
                               _dev(wq, torch.int8, "wq"), _dev(wscale, torch.float32, "wscale"), M,
                               _dev(out, torch.float32, "out"), _stream(stream)), "fgq_conv2d_w8")
    return out


def fgq_conv2d_w8_rq(act: torch.Tensor, act_type, act_scale: torch.Tensor, B: int, H: int, W: int, C: int, R: int,
                     S: int, stride: int, pad: int, groups: int, wq: torch.Tensor, wscale: torch.Tensor, M: int,
                     out_type, out_scale: torch.Tensor, out_q: Optional[torch.Tensor] = None,
                     stream=None) -> torch.Tensor:
    """fgq_conv2d_w8 with the output requantized in the kernel: uint8 NHWC [B][Ho][Wo][M] codes."""
    _require_cuda()
    Ho, Wo = conv_out_hw(H, W, R, S, stride, pad)
    if out_q is None:
        out_q = torch.empty((B, Ho, Wo, M), dtype=torch.uint8, device=act.device)
    _check(lib().fgq_conv2d_w8_rq(_dev(act, torch.uint8, "act"), _act_type(act_type),
                                  _dev(act_scale, torch.float32, "act_scale"), B, H, W, C, R, S, stride, pad, groups,
                                  _dev(wq, torch.int8, "wq"), _dev(wscale, torch.float32, "wscale"), M,
                                  _act_type(out_type), _dev(out_scale, torch.float32, "out_scale"),
                                  _dev(out_q, torch.uint8, "out_q"), _stream(stream)), "fgq_conv2d_w8_rq")
    return out_q


def fgq_maxpool_u8(x: torch.Tensor, B: int, H: int, W: int, C: int, R: int, stride: int, pad: int,
                   out: Optional[torch.Tensor] = None, stream=None) -> torch.Tensor:
    """R x R max pooling of unsigned codes, NHWC -> uint8 [B][Ho][Wo][C]."""
    _require_cuda()
    Ho, Wo = conv_out_hw(H, W, R, R, stride, pad)
    if out is None:
        out = torch.empty((B, Ho, Wo, C), dtype=torch.uint8, device=x.device)
    _check(lib().fgq_maxpool_u8(_dev(x, torch.uint8, "x"), B, H, W, C, R, stride, pad, _dev(out, torch.uint8, "out"),
                                _stream(stream)), "fgq_maxpool_u8")
    return out


def fgq_add_codes(a: torch.Tensor, a_type, a_scale: torch.Tensor, b: torch.Tensor, b_type, b_scale: torch.Tensor,
                  out_type=None, out_scale: Optional[torch.Tensor] = None, out: Optional[torch.Tensor] = None,
                  stream=None) -> torch.Tensor:
    """a * a_scale + b * b_scale: fp32 (out_type None) or codes requantized at out_scale."""
    _require_cuda()
    n = a.numel()
    if b.numel() != n:
        raise ValueError("fgq_add_codes: a and b differ in size")
    if out_type is None:
        if out is None:
            out = torch.empty(a.shape, dtype=torch.float32, device=a.device)
        st = lib().fgq_add_codes(_dev(a, torch.uint8, "a"), _act_type(a_type), _dev(a_scale, torch.float32, "a_scale"),
                                 _dev(b, torch.uint8, "b"), _act_type(b_type), _dev(b_scale, torch.float32, "b_scale"),
                                 n, _dev(out, torch.float32, "out"), 0, None, None, _stream(stream))
    else:
        if out is None:
            out = torch.empty(a.shape, dtype=torch.uint8, device=a.device)
        st = lib().fgq_add_codes(_dev(a, torch.uint8, "a"), _act_type(a_type), _dev(a_scale, torch.float32, "a_scale"),
                                 _dev(b, torch.uint8, "b"), _act_type(b_type), _dev(b_scale, torch.float32, "b_scale"),
                                 n, None, _act_type(out_type), _dev(out_scale, torch.float32, "out_scale"),
                                 _dev(out, torch.uint8, "out"), _stream(stream))
    _check(st, "fgq_add_codes")
    return out


def fgq_group_sums(q: torch.Tensor, act_type, P: int, Kred: int, codes: torch.Tensor, M: int, G: int,
                   stream=None) -> torch.Tensor:
    _require_cuda()
    s = torch.empty((M, num_groups(Kred, G), P), dtype=torch.int32, device=q.device)
    _check(lib().fgq_group_sums(_dev(q, torch.uint8, "q"), _act_type(act_type), P, Kred,
                                _dev(codes, torch.int32, "codes"), M, G, s.data_ptr(), _stream(stream)),
           "fgq_group_sums")
    return s


def fgq_conv2d_group_sums(act: torch.Tensor, act_type, B: int, H: int, W: int, C: int, R: int, S: int, stride: int,
                          pad: int, groups: int, codes: torch.Tensor, M: int, G: int, stream=None) -> torch.Tensor:
    _require_cuda()
    Ho, Wo = conv_out_hw(H, W, R, S, stride, pad)
    s = torch.empty((M, num_groups(R * S * (C // groups), G), B * Ho * Wo), dtype=torch.int32, device=act.device)
    _check(lib().fgq_conv2d_group_sums(_dev(act, torch.uint8, "act"), _act_type(act_type), B, H, W, C, R, S, stride,
                                       pad, groups, _dev(codes, torch.int32, "codes"), M, G, s.data_ptr(),
                                       _stream(stream)), "fgq_conv2d_group_sums")
    return s


def conv2d_host_workspace_bytes(act_type, B: int, H: int, W: int, C: int, R: int, S: int, stride: int, pad: int,
                                groups: int, M: int, G: int) -> int:
    return int(lib().fgq_conv2d_host_workspace_bytes(_act_type(act_type), B, H, W, C, R, S, stride, pad, groups, M, G))


def fgq_conv2d_host(h_w: torch.Tensor, h_x: torch.Tensor, act_type, B: int, H: int, W: int, C: int, R: int, S: int,
                    stride: int, pad: int, groups: int, M: int, G: int, h_out: torch.Tensor, workspace: torch.Tensor,
                    stream=None) -> None:
    """One layer end to end from host fp32 tensors (h_w [M][Kred], h_x NHWC) into host fp32
    h_out, through the C ABI; asynchronous on the stream (synchronize before reading h_out)."""
    _require_cuda()
    for t, name in ((h_w, "h_w"), (h_x, "h_x"), (h_out, "h_out")):
        if t.device.type != "cpu" or t.dtype != torch.float32 or not t.is_contiguous():
            raise ValueError(f"{name} must be a contiguous float32 host tensor")
    if not workspace.is_cuda or not workspace.is_contiguous():
        raise ValueError("workspace must be a contiguous device tensor")
    _check(lib().fgq_conv2d_host(h_w.data_ptr(), h_x.data_ptr(), _act_type(act_type), B, H, W, C, R, S, stride, pad,
                                 groups, M, G, h_out.data_ptr(), workspace.data_ptr(),
                                 workspace.numel() * workspace.element_size(), _stream(stream)), "fgq_conv2d_host")


# --------------------------------------------------------------------------- decoders (fgq_decoder.h)

class _KVCacheStruct(ctypes.Structure):
    _fields_ = [("k_codes", _vp), ("k_params", _vp), ("v_codes", _vp), ("v_params", _vp), ("pages", _i),
                ("page_size", _i), ("kv_heads", _i), ("head_dim", _i), ("group", _i)]


class KVCache:
    """A paged cache of keys and values held in 4 bits: codes uint8 [pages][kv heads][page size][head_dim / 2],
    parameters int32 [pages][kv heads][page size][head_dim / group] (layouts in include/fgq_decoder.h)."""

    __slots__ = ("k_codes", "k_params", "v_codes", "v_params", "pages", "page_size", "kv_heads", "head_dim", "group",
                 "_c", "_ref")

    def __init__(self, k_codes: torch.Tensor, k_params: torch.Tensor, v_codes: torch.Tensor, v_params: torch.Tensor):
        codes = _dev(k_codes, torch.uint8, "k_codes"), _dev(v_codes, torch.uint8, "v_codes")
        params = _dev(k_params, torch.int32, "k_params"), _dev(v_params, torch.int32, "v_params")
        c, p = k_codes.shape, k_params.shape
        if len(c) != 4 or len(p) != 4 or p[3] == 0:
            raise ValueError("KVCache: codes and parameters are [pages][kv heads][page size][...]")
        if v_codes.shape != c or v_params.shape != p or c[:3] != p[:3]:
            raise ValueError("KVCache: the four tensors differ in pages, kv heads, page size or row length")
        self.k_codes, self.k_params, self.v_codes, self.v_params = k_codes, k_params, v_codes, v_params
        self.pages, self.kv_heads, self.page_size, half = c
        self.head_dim = 2 * half
        self.group = self.head_dim // p[3]
        self._c = _KVCacheStruct(codes[0], params[0], codes[1], params[1], c[0], c[2], c[1], 2 * half, self.group)
        self._ref = ctypes.addressof(self._c)


def kv_cache(pages: int, page_size: int, kv_heads: int, head_dim: int, group: int = 64, device="cuda") -> KVCache:
    """An empty cache (every value 0)."""
    _require_cuda()
    if group <= 0 or head_dim % group:
        raise ValueError("kv_cache: group must divide head_dim")
    codes = [torch.zeros((pages, kv_heads, page_size, head_dim // 2), dtype=torch.uint8, device=device) for _ in "kv"]
    params = [torch.zeros((pages, kv_heads, page_size, head_dim // group), dtype=torch.int32, device=device)
              for _ in "kv"]
    return KVCache(codes[0], params[0], codes[1], params[1])


def _float_type(t: torch.Tensor, name: str) -> int:
    if not isinstance(t, torch.Tensor) or not t.is_cuda:
        raise TypeError(f"{name} must be a CUDA tensor")
    ty = FLOAT_TYPES.get(t.dtype)
    if ty is None:
        raise TypeError(f"{name} must be float32, bfloat16 or float16, got {t.dtype}")
    return ty


def _heads(t: torch.Tensor, heads: Optional[int], D: int, name: str) -> Tuple[int, int, int]:
    """(type, batch stride, token stride) of a [B][T][heads][D] tensor whose last two axes are contiguous."""
    ty = FLOAT_TYPES.get(t.dtype) if isinstance(t, torch.Tensor) and t.is_cuda else None
    if ty is None:
        ty = _float_type(t, name)
    shape = t.shape
    if len(shape) != 4 or shape[3] != D or (heads is not None and shape[2] != heads):
        raise ValueError(f"{name} must be [B][T][{heads or 'heads'}][{D}], got {tuple(shape)}")
    sb, st, sh, sd = t.stride()
    if (sd != 1 and D > 1) or (sh != D and shape[2] > 1):
        raise ValueError(f"{name}: heads and head_dim must be contiguous")
    # an axis of one element may have any stride
    return ty, sb if shape[0] > 1 else 0, st if shape[1] > 1 else 0


def _table(table: torch.Tensor, B: int) -> Tuple[int, int]:
    p = _dev(table, torch.int32, "page_table")
    shape = table.shape
    if len(shape) != 2 or shape[0] != B:
        raise ValueError(f"page_table must be [{B}][max pages], got {tuple(shape)}")
    return p, shape[1]


def _per_sequence(t: Optional[torch.Tensor], B: int, name: str) -> Optional[int]:
    if t is None:
        return None
    p = _dev(t, torch.int32, name)
    if t.numel() != B:
        raise ValueError(f"{name} must have {B} entries, got {t.numel()}")
    return p


def fgq_kv_append(cache: KVCache, k: torch.Tensor, v: torch.Tensor, page_table: torch.Tensor, starts: torch.Tensor,
                  lens: Optional[torch.Tensor] = None, stream=None) -> None:
    """Quantizes k, v [B][T][kv heads][head_dim] into positions starts[b] + i (i < lens[b], or T) of each sequence."""
    _require_cuda()
    ty, kb, kt = _heads(k, cache.kv_heads, cache.head_dim, "k")
    tv, vb, vt = _heads(v, cache.kv_heads, cache.head_dim, "v")
    if ty != tv or k.shape != v.shape:
        raise ValueError("fgq_kv_append: k and v differ in shape or type")
    B, T = k.shape[:2]
    tp, mp = _table(page_table, B)
    _check(lib().fgq_kv_append(cache._ref, k.data_ptr(), v.data_ptr(), ty, B, T, kb, kt, vb, vt, tp, mp,
                               _per_sequence(starts, B, "starts"), _per_sequence(lens, B, "lens"), _stream(stream)),
           "fgq_kv_append")


def fgq_kv_read(cache: KVCache, page_table: torch.Tensor, starts: torch.Tensor, T: int,
                lens: Optional[torch.Tensor] = None, dtype=torch.bfloat16, stream=None):
    """(k, v) [B][T][kv heads][head_dim] of positions starts[b] + i as the values their codes stand for."""
    _require_cuda()
    B = page_table.shape[0]
    tp, mp = _table(page_table, B)
    if dtype not in FLOAT_TYPES:
        raise TypeError(f"dtype must be float32, bfloat16 or float16, got {dtype}")
    k = torch.empty((B, T, cache.kv_heads, cache.head_dim), dtype=dtype, device=page_table.device)
    v = torch.empty_like(k)
    _check(lib().fgq_kv_read(cache._ref, k.data_ptr(), v.data_ptr(), FLOAT_TYPES[dtype], B, T, tp, mp,
                             _per_sequence(starts, B, "starts"), _per_sequence(lens, B, "lens"), _stream(stream)),
           "fgq_kv_read")
    return k, v


def fgq_kv_attention(q: torch.Tensor, cache: KVCache, page_table: torch.Tensor, seq_lens: torch.Tensor,
                     q_lens: Optional[torch.Tensor] = None, causal: bool = True, window: int = 0,
                     scale: Optional[float] = None, max_len: int = 0, out: Optional[torch.Tensor] = None,
                     stream=None) -> torch.Tensor:
    """Attention of q [B][T][heads][head_dim] over the cache (scale: head_dim ** -0.5) -> out of q's shape and type."""
    _require_cuda()
    ty, qb, qt = _heads(q, None, cache.head_dim, "q")
    B, T, heads, D = q.shape
    tp, mp = _table(page_table, B)
    if out is None:
        out = torch.empty_like(q, memory_format=torch.contiguous_format)
    elif out.shape != q.shape:
        raise ValueError(f"out must be {tuple(q.shape)}, got {tuple(out.shape)}")
    _check(lib().fgq_kv_attention(cache._ref, q.data_ptr(), ty, B, T, heads, qb, qt, tp, mp,
                                  _per_sequence(seq_lens, B, "seq_lens"), _per_sequence(q_lens, B, "q_lens"), max_len,
                                  int(causal), window, D ** -0.5 if scale is None else scale,
                                  _dev(out, q.dtype, "out"), _stream(stream)), "fgq_kv_attention")
    return out


def _rows(x: torch.Tensor, name: str) -> Tuple[int, int]:
    """(type, row stride) of a [P][K] tensor with contiguous rows."""
    ty = _float_type(x, name)
    if x.dim() != 2 or (x.shape[1] > 1 and x.stride(1) != 1):
        raise ValueError(f"{name} must be [tokens][features] with contiguous rows")
    return ty, x.stride(0) if x.shape[0] > 1 else x.shape[1]


def fgq_quantize_tokens(x: torch.Tensor, stream=None) -> Tuple[torch.Tensor, torch.Tensor]:
    """Per-token symmetric 8-bit quantization: x [P][K] -> (codes int8 [P][K], scale fp32 [P])."""
    _require_cuda()
    ty, ldx = _rows(x, "x")
    P, K = x.shape
    q = torch.empty((P, K), dtype=torch.int8, device=x.device)
    scale = torch.empty(P, dtype=torch.float32, device=x.device)
    _check(lib().fgq_quantize_tokens(x.data_ptr(), ty, P, K, ldx, q.data_ptr(), scale.data_ptr(), _stream(stream)),
           "fgq_quantize_tokens")
    return q, scale


def _weights8(wq: torch.Tensor, wscale: torch.Tensor, bias: Optional[torch.Tensor], K: int):
    if wq.dim() != 2 or wq.shape[1] != K or wscale.numel() != wq.shape[0] or \
            (bias is not None and bias.numel() != wq.shape[0]):
        raise ValueError(f"weights must be int8 [M][{K}] with fp32 scales (and bias) [M]")
    return (_dev(wq, torch.int8, "wq"), _dev(wscale, torch.float32, "wscale"),
            None if bias is None else _dev(bias, torch.float32, "bias"))


def fgq_gemm_w8a8(q: torch.Tensor, scale: torch.Tensor, wq: torch.Tensor, wscale: torch.Tensor,
                  bias: Optional[torch.Tensor] = None, dtype=torch.float32, y: Optional[torch.Tensor] = None,
                  stream=None) -> torch.Tensor:
    """y[p][m] = scale[p] wscale[m] sum_k q[p][k] wq[m][k] + bias[m], of type dtype."""
    _require_cuda()
    P, K = q.shape
    pw, ps, pb = _weights8(wq, wscale, bias, K)
    if dtype not in FLOAT_TYPES:
        raise TypeError(f"dtype must be float32, bfloat16 or float16, got {dtype}")
    if scale.numel() != P:
        raise ValueError(f"scale must have {P} entries, got {scale.numel()}")
    if y is None:
        y = torch.empty((P, wq.shape[0]), dtype=dtype, device=q.device)
    elif tuple(y.shape) != (P, wq.shape[0]):
        raise ValueError(f"y must be {(P, wq.shape[0])}, got {tuple(y.shape)}")
    _check(lib().fgq_gemm_w8a8(_dev(q, torch.int8, "q"), _dev(scale, torch.float32, "scale"), P, K, pw, ps,
                               wq.shape[0], pb, _dev(y, dtype, "y"), FLOAT_TYPES[dtype], _stream(stream)),
           "fgq_gemm_w8a8")
    return y


def fgq_linear_w8a8(x: torch.Tensor, wq: torch.Tensor, wscale: torch.Tensor, bias: Optional[torch.Tensor] = None,
                    y: Optional[torch.Tensor] = None, stream=None) -> torch.Tensor:
    """A linear layer on 8-bit integers: x [P][K] quantized per token, times wq [M][K]^T, of x's type."""
    _require_cuda()
    ty, ldx = _rows(x, "x")
    P, K = x.shape
    pw, ps, pb = _weights8(wq, wscale, bias, K)
    if y is None:
        y = torch.empty((P, wq.shape[0]), dtype=x.dtype, device=x.device)
    elif tuple(y.shape) != (P, wq.shape[0]):
        raise ValueError(f"y must be {(P, wq.shape[0])}, got {tuple(y.shape)}")
    _check(lib().fgq_linear_w8a8(x.data_ptr(), ty, P, K, ldx, pw, ps, wq.shape[0], pb, _dev(y, x.dtype, "y"),
                                 _stream(stream)), "fgq_linear_w8a8")
    return y


def fgq_stream_status(stream=None) -> int:
    return int(lib().fgq_stream_status(_stream(stream)))


def fgq_set_path(path: int) -> int:
    """Kernel family of this thread's contraction calls (test and benchmark control)."""
    return int(lib().fgq_set_path(path))


def fgq_debug_set_wait_limit_us(us: int) -> int:
    """Wait limit of this thread's tensor-core kernel launches (test control; -1 restores)."""
    return int(lib().fgq_debug_set_wait_limit_us(us))


def fgq_debug_set_scratch_limit(nbytes: int) -> int:
    """Per-call temporaries above `nbytes` fail on this thread (negative: none); the previous limit."""
    return int(lib().fgq_debug_set_scratch_limit(nbytes))


def fgq_debug_set_resident_blocks(blocks: int) -> int:
    """Cooperative launches of more blocks fail on this thread (negative: none); the previous limit."""
    return int(lib().fgq_debug_set_resident_blocks(blocks))


def fgq_debug_set_attention_kernel(which: int) -> int:
    """Kernel of this thread's fgq_kv_attention calls: 1 few rows, 2 many rows, 0 the faster; the previous one."""
    return int(lib().fgq_debug_set_attention_kernel(int(which)))


def fgq_debug_allow_split_fold(allow: bool) -> int:
    """Lets FGQ_PATH_DENSE run fp32 alphas as the split-fp16 ablation on this thread."""
    return int(lib().fgq_debug_allow_split_fold(1 if allow else 0))


def fgq_debug_cta_pairs(on: bool) -> int:
    """Remembered only: every contraction kernel runs on single CTAs."""
    return int(lib().fgq_debug_cta_pairs(1 if on else 0))


def fgq_debug_max_ksplit(k: int) -> int:
    """At most k group ranges per G >= 64 tensor-core tile on this thread (1: whole tiles)."""
    return int(lib().fgq_debug_max_ksplit(int(k)))


def fgq_debug_last_ksplit() -> int:
    """Group ranges per tile of this thread's last G >= 64 tensor-core call."""
    return int(lib().fgq_debug_last_ksplit())


def fgq_debug_last_cuda_error() -> tuple:
    """(cudaError_t value, name) behind this thread's last FGQ_ERR_CUDA from a launch; clears it."""
    buf = ctypes.create_string_buffer(64)
    code = int(lib().fgq_debug_last_cuda_error(buf, 64))
    return code, buf.value.decode()


def fgq_last_path() -> int:
    return int(lib().fgq_last_path())


def fgq_launch_count() -> int:
    return int(lib().fgq_launch_count())


def fgq_selftest_wait_timeout(max_iterations: int, stream=None) -> int:
    _check(lib().fgq_selftest_wait_timeout(max_iterations, _stream(stream)), "fgq_selftest_wait_timeout")
    return fgq_stream_status(stream)


def fgq_debug_selftest_warp_wait(limit_us: int, stream=None) -> int:
    _check(lib().fgq_debug_selftest_warp_wait(limit_us, _stream(stream)), "fgq_debug_selftest_warp_wait")
    return fgq_stream_status(stream)
