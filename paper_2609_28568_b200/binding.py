"""Binding of the nb_linear C ABI: argument marshalling only. The calls of the hot path go through the
extension module built from csrc/native.cpp, the others through ctypes.

Functions named like the C entry points take torch CUDA tensors (or raw device
pointers as ints) and pass pointers and sizes straight through; every step of
the computation runs in the CUDA library. There is no CPU path: if the library
has not been built, loading raises.
"""
from __future__ import annotations

import ctypes
import importlib.machinery
import importlib.util
import os

import torch

from .build import LIB_PATH, NATIVE_PATH

NB_OK, NB_ERR_INVALID_ARG, NB_ERR_UNSUPPORTED, NB_ERR_CUDA, NB_ERR_TIMEOUT = 0, 1, 2, 3, 4
ACT_NONE, ACT_GELU, ACT_SWIGLU = 0, 1, 2
DTYPE_F32, DTYPE_BF16 = 0, 1
ROTARY_HALF, ROTARY_NEIGHBOURS = 0, 1

EXPORTS = (
    "nb_version", "nb_last_error", "nb_set_stream", "nb_get_stream", "nb_linear_out_elems",
    "nb_linear_forward", "nb_linear_forward_ex", "nb_linear_backward", "nb_linear_backward_ex",
    "nb_reduce_dbias", "nb_workspace_reserve", "nb_release", "nb_check_status",
    "nb_debug_wait_timeout", "nb_kernel_launches", "nb_gelu_dbias_noalloc",
    "nb_debug_split_plan", "nb_cast_f32_to_bf16", "nb_lm_head_ce_forward", "nb_ce_backward",
    "nb_lora_linear_forward", "nb_lora_linear_backward", "nb_debug_layer_bwd_plan", "nb_debug_gemm_timeout",
    "nb_lora_down_stacked", "nb_lora_linear_forward_stacked", "nb_lora_linear_backward_stacked",
    "nb_lora_da_stacked", "nb_debug_route", "nb_layernorm_forward", "nb_layernorm_workspace", "nb_layernorm_backward",
    "nb_muon_workspace", "nb_muon_update", "nb_muon_apply", "nb_debug_layernorm_timeout",
    "nb_debug_muon_timeout", "nb_rotary_frequencies", "nb_rotary", "nb_attention_forward", "nb_attention_workspace", "nb_attention_backward",
    "nb_debug_attention_timeout",
)

CALL_FORWARD, CALL_BACKWARD, CALL_LORA_FORWARD, CALL_LORA_BACKWARD = range(4)
ROUTES = {1: "rows", 2: "tile", 3: "tile_pair", 4: "gemm", 5: "gemm", 6: "layer_bwd", 7: "lora_udb"}

_lib = None
_vp, _i64, _int = ctypes.c_void_p, ctypes.c_int64, ctypes.c_int


class NbError(RuntimeError):
    def __init__(self, code: int, msg: str):
        super().__init__(f"nb_linear error {code}: {msg}")
        self.code = code


def lib() -> ctypes.CDLL:
    """The loaded CUDA library. Raises if it was never built: there is no fallback."""
    global _lib
    if _lib is None:
        if not os.path.exists(LIB_PATH):
            raise RuntimeError(
                f"{LIB_PATH} is missing: build it with `python -m paper_2609_28568_b200.build` "
                "(the CUDA library is the only implementation)")
        L = ctypes.CDLL(LIB_PATH)
        L.nb_version.restype = _int
        L.nb_last_error.restype = ctypes.c_char_p
        L.nb_set_stream.argtypes = [_vp]
        L.nb_get_stream.restype = _vp
        L.nb_linear_out_elems.argtypes = [_i64, _i64, _int]
        L.nb_linear_out_elems.restype = _i64
        L.nb_linear_forward.argtypes = [_vp, _vp, _vp, _vp, _i64, _i64, _i64, _int]
        L.nb_linear_forward_ex.argtypes = [_vp, _vp, _vp, _vp, _vp, _i64, _i64, _i64, _int, _vp]
        L.nb_linear_backward.argtypes = [_vp] * 7 + [_i64, _i64, _i64, _int]
        L.nb_linear_backward_ex.argtypes = [_vp] * 8 + [_i64, _i64, _i64, _int, _int, _int, _vp]
        L.nb_reduce_dbias.argtypes = [_vp, _vp, _i64, _i64, _int]
        L.nb_workspace_reserve.argtypes = [_i64]
        L.nb_debug_wait_timeout.argtypes = [_i64]
        L.nb_kernel_launches.restype = _i64
        L.nb_gelu_dbias_noalloc.argtypes = [_vp, _vp, _vp, _i64, _i64, _int, _vp]
        L.nb_cast_f32_to_bf16.argtypes = [_vp, _vp, _i64, _vp]
        L.nb_lora_linear_forward.argtypes = [_vp] * 7 + [ctypes.c_float] + [_i64] * 4 + [_vp]
        L.nb_lora_linear_backward.argtypes = [_vp] * 10 + [ctypes.c_float] + [_i64] * 4 + [_int, _vp]
        L.nb_lora_down_stacked.argtypes = [_vp, _vp, _vp, ctypes.c_float, _i64, _i64, _i64, _vp]
        L.nb_lora_linear_forward_stacked.argtypes = [_vp] * 6 + [_i64] * 6 + [_vp]
        L.nb_lora_linear_backward_stacked.argtypes = [_vp] * 8 + [ctypes.c_float] + [_i64] * 6 + [_int, _vp]
        L.nb_lora_da_stacked.argtypes = [_vp, _vp, _vp, _i64, _i64, _i64, _int, _vp]
        L.nb_lm_head_ce_forward.argtypes = [_vp] * 6 + [_i64] * 4 + [_vp]
        L.nb_ce_backward.argtypes = [_vp] * 4 + [ctypes.c_float] + [_i64] * 3 + [_vp]
        L.nb_layernorm_forward.argtypes = [_vp] * 8 + [_i64] * 2 + [ctypes.c_float, _int, _vp]
        L.nb_layernorm_workspace.argtypes = [_i64] * 2
        L.nb_layernorm_workspace.restype = _i64
        L.nb_layernorm_backward.argtypes = [_vp] * 10 + [_i64] * 2 + [_int] * 2 + [_vp, _i64, _vp]
        L.nb_muon_workspace.argtypes = [_i64] * 3
        L.nb_muon_workspace.restype = _i64
        L.nb_muon_update.argtypes = ([ctypes.POINTER(_vp)] * 3 + [_i64] * 3 + [ctypes.c_float, _int, _int] + [ctypes.c_float] * 4 +
                                     [_int, _vp, _i64, _vp])
        L.nb_muon_apply.argtypes = [ctypes.POINTER(_vp)] * 3 + [_i64] * 2 + [ctypes.c_float] * 2 + [_vp]
        L.nb_rotary_frequencies.argtypes = [ctypes.POINTER(ctypes.c_double), _i64] + [ctypes.c_double] * 4 + [_i64]
        L.nb_rotary.argtypes = [_vp] * 7 + [_i64] * 10 + [ctypes.c_float, _int, _int, _vp]
        L.nb_attention_forward.argtypes = [_vp] * 6 + [_i64] * 9 + [ctypes.c_float, _int, _vp]
        L.nb_attention_workspace.argtypes = [_i64] * 2
        L.nb_attention_workspace.restype = _i64
        L.nb_attention_backward.argtypes = [_vp] * 10 + [_i64] * 13 + [ctypes.c_float, _int, _vp, _i64, _vp]
        L.nb_debug_split_plan.argtypes = [_i64, _i64, _i64, _int, _int, ctypes.POINTER(_int)]
        L.nb_debug_gemm_timeout.argtypes = [_vp, _vp, _vp, _i64]
        L.nb_debug_layernorm_timeout.argtypes = [_vp, _vp, _vp, _vp, _int, _i64]
        L.nb_debug_muon_timeout.argtypes = [_vp, _vp, _vp, _i64, _i64]
        L.nb_debug_attention_timeout.argtypes = [ctypes.POINTER(_vp), _int, _i64]
        L.nb_debug_layer_bwd_plan.argtypes = [_i64, _i64, _i64, _int, _int, ctypes.POINTER(_int), _i64]
        L.nb_debug_route.argtypes = [_int] + [_i64] * 4 + [_int] * 3 + [ctypes.POINTER(_int)]
        _lib = L
    return _lib


_native = None


def _load_native():
    """The extension module. Raises if it was never built: there is no fallback."""
    global _native
    lib()
    if not os.path.exists(NATIVE_PATH):
        raise RuntimeError(f"{NATIVE_PATH} is missing: build it with `python -m paper_2609_28568_b200.build`")
    name = __package__ + "._native"
    loader = importlib.machinery.ExtensionFileLoader(name, NATIVE_PATH)
    module = importlib.util.module_from_spec(importlib.util.spec_from_loader(name, loader))
    loader.exec_module(module)
    module.set_python(NbError, _ptr, _stream_address)
    _native = module
    return module


def _ptr(t):
    if t is None:
        return None
    if isinstance(t, int):
        return t
    assert t.is_cuda and t.is_contiguous(), "device tensors must be contiguous CUDA tensors"
    return t.data_ptr()


def _stream_address(s):
    """The address in a stream object: a c_void_p, or what carries one as _as_parameter_ (torch.cuda.Stream)."""
    while not (s is None or isinstance(s, (int, ctypes.c_void_p))):
        if not hasattr(s, "_as_parameter_"):
            raise TypeError(f"a stream or its address is wanted, not {type(s).__name__}")
        s = s._as_parameter_
    return s.value if isinstance(s, ctypes.c_void_p) else s


def _size(nbytes: int, what: str) -> int:
    if nbytes < 0:
        raise NbError(NB_ERR_UNSUPPORTED, f"{what}: no such size")
    return nbytes


def _check(rc: int) -> None:
    if rc != NB_OK:
        raise NbError(rc, lib().nb_last_error().decode())


def _stream():
    return torch._C._cuda_getCurrentRawStream(torch.cuda.current_device())


def nb_version() -> int:
    return lib().nb_version()


def nb_last_error() -> str:
    return lib().nb_last_error().decode()


def nb_linear_out_elems(BT: int, OC: int, act: int) -> int:
    return lib().nb_linear_out_elems(BT, OC, act)


def nb_set_stream(stream) -> None:
    _check(lib().nb_set_stream(stream))


def nb_linear_forward(out, inp, weight, bias, BT, C, OC, act) -> None:
    """Short form: `out` holds the activated plane followed by the pre-activation plane."""
    lib().nb_set_stream(_stream())
    _check(lib().nb_linear_forward(_ptr(out), _ptr(inp), _ptr(weight), _ptr(bias), BT, C, OC, act))


def nb_linear_forward_ex(out, pre_act, inp, weight, bias, BT, C, OC, act, stream=None) -> None:
    (_native or _load_native()).nb_linear_forward_ex(out, pre_act, inp, weight, bias, BT, C, OC, act, stream)


def nb_linear_backward(dinp, dweight, dbias, dout, inp, weight, pre_act, BT, C, OC, accumulate) -> None:
    lib().nb_set_stream(_stream())
    _check(lib().nb_linear_backward(_ptr(dinp), _ptr(dweight), _ptr(dbias), _ptr(dout), _ptr(inp),
                                    _ptr(weight), _ptr(pre_act), BT, C, OC, int(accumulate)))


def nb_linear_backward_ex(dinp, dweight, dbias, dout, inp, weight, pre_act, inp_pre_act, BT, C, OC,
                          act, accumulate, dweight_dtype=DTYPE_F32, stream=None) -> None:
    (_native or _load_native()).nb_linear_backward_ex(dinp, dweight, dbias, dout, inp, weight, pre_act, inp_pre_act,
                                                      BT, C, OC, act, int(accumulate), dweight_dtype, stream)


def nb_reduce_dbias(dbias, dout, BT, OC, accumulate) -> None:
    lib().nb_set_stream(_stream())
    _check(lib().nb_reduce_dbias(_ptr(dbias), _ptr(dout), BT, OC, int(accumulate)))


def nb_workspace_reserve(nbytes: int) -> None:
    _check(lib().nb_workspace_reserve(nbytes))


def nb_release() -> None:
    _check(lib().nb_release())


def nb_check_status() -> None:
    """Synchronise and raise NbError(NB_ERR_TIMEOUT / NB_ERR_CUDA) if a kernel reported a failure."""
    _check(lib().nb_check_status())


NOALLOC_MAX_ELEMS = 4194304


def nb_gelu_dbias_noalloc(dbias, dout, pre_act, BT, OC, accumulate, stream=None) -> None:
    """dbias (+)= column sums of dout * gelu'(pre_act), using only the scratch array built into
    the library: for callers that may not allocate device memory. BT*OC <= NOALLOC_MAX_ELEMS."""
    (_native or _load_native()).nb_gelu_dbias_noalloc(dbias, dout, pre_act, BT, OC, int(accumulate), stream)


def nb_lora_linear_forward(out, t, inp, weight, bias, lora_a, lora_b, scale, BT, C, OC, r, stream=None) -> None:
    """out = inp @ W.T (+ bias) + t @ B.T with t = bf16(scale * inp @ A.T), the adapter term fused in."""
    (_native or _load_native()).nb_lora_linear_forward(out, t, inp, weight, bias, lora_a, lora_b, scale, BT, C, OC, r,
                                                       stream)


def nb_lora_linear_backward(dinp, dlora_a, dlora_b, u, dout, inp, weight, lora_a, lora_b, t, scale, BT, C,
                            OC, r, accumulate, stream=None) -> None:
    """Gradients of the adapter layer with the base weight frozen (dinp, dA, dB)."""
    (_native or _load_native()).nb_lora_linear_backward(dinp, dlora_a, dlora_b, u, dout, inp, weight, lora_a, lora_b, t,
                                                        scale, BT, C, OC, r, int(accumulate), stream)


def nb_lora_down_stacked(t_stack, inp, a_stack, scale, BT, C, R, stream=None) -> None:
    """t_stack = bf16(scale * inp @ a_stack.T): the down-projections of all adapters of a group at once."""
    (_native or _load_native()).nb_lora_down_stacked(t_stack, inp, a_stack, scale, BT, C, R, stream)


def nb_lora_linear_forward_stacked(out, inp, weight, bias, t_stack, lora_b, BT, C, OC, r, R, off,
                                   stream=None) -> None:
    """out = inp @ W.T (+ bias) + t_stack[:, off:off+r] @ B.T, the adapter term fused in."""
    (_native or _load_native()).nb_lora_linear_forward_stacked(out, inp, weight, bias, t_stack, lora_b, BT, C, OC, r, R,
                                                               off, stream)


def nb_lora_linear_backward_stacked(dinp, dlora_b, u_stack, dout, weight, lora_a, lora_b, t_stack, scale, BT, C,
                                    OC, r, R, off, accumulate, stream=None) -> None:
    """u slice, dinp and dB of one adapted projection of a stacked group (dA comes from nb_lora_da_stacked)."""
    (_native or _load_native()).nb_lora_linear_backward_stacked(dinp, dlora_b, u_stack, dout, weight, lora_a, lora_b,
                                                                t_stack, scale, BT, C, OC, r, R, off,
                                                                int(accumulate), stream)


def nb_lora_da_stacked(da_stack, u_stack, inp, BT, C, R, accumulate, stream=None) -> None:
    """da_stack (+)= u_stack.T @ inp: the A gradients of all adapters of a group at once."""
    (_native or _load_native()).nb_lora_da_stacked(da_stack, u_stack, inp, BT, C, R, int(accumulate), stream)


def nb_lm_head_ce_forward(logits, loss, lse, inp, weight, targets, BT, C, Vp, V, stream=None) -> None:
    """Head GEMM with the softmax statistics of the first V columns fused in: logits, loss, lse."""
    (_native or _load_native()).nb_lm_head_ce_forward(logits, loss, lse, inp, weight, targets, BT, C, Vp, V, stream)


def nb_ce_backward(dlogits, logits, lse, targets, gscale, BT, Vp, V, stream=None) -> None:
    """dlogits = gscale * (softmax - onehot) on the first V columns, 0 on the padding."""
    (_native or _load_native()).nb_ce_backward(dlogits, logits, lse, targets, gscale, BT, Vp, V, stream)


def nb_cast_f32_to_bf16(dst, src, n, stream=None) -> None:
    """Master-weight cast: dst (bf16) = src (fp32), round to nearest even."""
    (_native or _load_native()).nb_cast_f32_to_bf16(dst, src, n, stream)


def nb_layernorm_forward(out, sum, mean, rstd, inp, branch, weight, bias, BT, C, eps, stream_dtype, stream=None) -> None:
    """s = inp + branch (stored in sum, in the stream's type; branch None: s = inp); out = layer norm of s; mean and rstd for the backward
    pass, or None."""
    (_native or _load_native()).nb_layernorm_forward(out, sum, mean, rstd, inp, branch, weight, bias, BT, C, eps, stream_dtype,
                                                     stream)


def nb_layernorm_workspace(BT: int, C: int) -> int:
    """Bytes of workspace that nb_layernorm_backward needs for dweight and dbias."""
    return _size(lib().nb_layernorm_workspace(BT, C), f"layer norm of [{BT}, {C}]")


def nb_layernorm_backward(dinp, dbranch, dweight, dbias, dout, dres, inp, mean, rstd, weight, BT, C, accumulate, stream_dtype,
                          workspace, workspace_bytes, stream=None) -> None:
    """dinp = dres + the norm's input gradient (dbranch: the same in bf16); dweight, dbias (+)= column sums."""
    (_native or _load_native()).nb_layernorm_backward(dinp, dbranch, dweight, dbias, dout, dres, inp, mean, rstd, weight, BT, C,
                                                      accumulate, stream_dtype, workspace, workspace_bytes, stream)


def nb_muon_workspace(n: int, R: int, C: int) -> int:
    """Bytes of workspace that nb_muon_update needs for n matrices [R, C]."""
    return _size(lib().nb_muon_workspace(n, R, C), f"{n} matrices [{R}, {C}]")


def nb_muon_update(update, momentum, grad, n, R, C, mu, nesterov, steps, a, b, c, eps, grad_dtype, workspace, workspace_bytes,
                   stream=None) -> None:
    """m <- mu m + g, v = g + mu m or m, update = bf16 of v orthogonalised in `steps` steps, for n matrices [R, C] given as sequences."""
    (_native or _load_native()).nb_muon_update(update, momentum, grad, n, R, C, mu, nesterov, steps, a, b, c, eps, grad_dtype,
                                               workspace, workspace_bytes, stream)


def nb_muon_apply(master, weight, update, n, count, decay, step, stream=None) -> None:
    """master <- decay * master - step * update, weight <- bf16(master), for n tensors of count elements given as sequences."""
    (_native or _load_native()).nb_muon_apply(master, weight, update, n, count, decay, step, stream)


def nb_rotary_frequencies(R: int, base: float = 10000.0, factor: float = 1.0, low: float = 1.0, high: float = 32.0, original: int = 0):
    """Radians per position of R / 2 pairs, a list. factor: of a longer context; by parts where original is its positions before (see the header)."""
    freq = (ctypes.c_double * max(R // 2, 1))()
    _check(lib().nb_rotary_frequencies(freq, R, base, factor, low, high, original))
    return list(freq[:R // 2])


def nb_rotary(out_q, out_k, q, k, freq, positions, cu_seqlens, T, n, heads, kv_heads, D, R, ld_out_q, ld_out_k, ld_q, ld_k, scale, layout,
              inverse, stream=None) -> None:
    """Queries and keys turned by their positions (inverse: back). The tensors of heads may be columns of wider ones, with rows ld elements
    apart; an output may be its input."""
    (_native or _load_native()).nb_rotary(out_q, out_k, q, k, freq, positions, cu_seqlens, T, n, heads, kv_heads, D, R, ld_out_q, ld_out_k,
                                          ld_q, ld_k, scale, layout, int(inverse), stream)


def nb_attention_forward(out, lse, q, k, v, cu_seqlens, T, n, heads, kv_heads, D, ld_out, ld_q, ld_k, ld_v, scale, causal,
                         stream=None) -> None:
    """out = attention of q over k and v, per sequence and head; lse for the backward pass, or None. The tensors of heads may be columns
    of wider ones, with rows ld elements apart."""
    (_native or _load_native()).nb_attention_forward(out, lse, q, k, v, cu_seqlens, T, n, heads, kv_heads, D, ld_out, ld_q, ld_k, ld_v,
                                                     scale, int(causal), stream)


def nb_attention_workspace(T: int, heads: int) -> int:
    """Bytes of workspace that nb_attention_backward needs."""
    return _size(lib().nb_attention_workspace(T, heads), f"attention of {heads} heads over {T} rows")


def nb_attention_backward(dq, dk, dv, dout, out, lse, q, k, v, cu_seqlens, T, n, heads, kv_heads, D, ld_dq, ld_dk, ld_dv, ld_dout, ld_out, ld_q,
                          ld_k, ld_v, scale, causal, workspace, workspace_bytes, stream=None) -> None:
    """Gradients of attention with out and lse of the forward pass."""
    (_native or _load_native()).nb_attention_backward(dq, dk, dv, dout, out, lse, q, k, v, cu_seqlens, T, n, heads, kv_heads, D, ld_dq, ld_dk,
                                                      ld_dv, ld_dout, ld_out, ld_q, ld_k, ld_v, scale, int(causal), workspace, workspace_bytes,
                                                      stream)


def nb_debug_split_plan(M: int, N: int, K: int, slots: int, tile_m: int):
    """(row tiles, column tiles, split-K factor, k-blocks per split, k-blocks) of a wgrad."""
    out = (_int * 5)()
    _check(lib().nb_debug_split_plan(M, N, K, slots, tile_m, out))
    return tuple(out)


def nb_debug_layer_bwd_plan(BT: int, C: int, OC: int, pairs: int, gelu_grad: bool, launched: bool = False, fresh: bool = False,
                            sums: bool = False):
    """(header of eight ints, list of (pair, is_dweight, row tile, column tile, kb0, kb1)) of the
    one-launch layer backward; raises NbError for shapes its schedule does not cover. launched: with
    dinp tiles as wide as the launch has them, else in whole ones; fresh: for gradients that start from nothing; sums: the k-blocks that one accumulator
    sums are a record, not a unit's."""
    cap = 8 + 6 * (4 * pairs + 64 + 2 * (-(-BT // 256)) * (-(-C // 256))
                   + 2 * (-(-OC // 256)) * (-(-C // 256)) * max(1, BT // 1024)) * (8 if sums else 1)
    out = (_int * cap)()
    n = lib().nb_debug_layer_bwd_plan(BT, C, OC, pairs, int(bool(gelu_grad)) + 2 * int(bool(launched)) + 4 * int(bool(fresh))
                                      + 8 * int(bool(sums)), out, cap)
    if n < 0:
        raise NbError(-n, lib().nb_last_error().decode())
    recs = [tuple(out[8 + 6 * i: 14 + 6 * i]) for i in range(n)]
    return tuple(out[:8]), recs


def nb_debug_route(call: int, BT: int, C: int, OC: int, *, r: int = 0, act: int = ACT_NONE, dinp: bool = True,
                   dweight: bool = True, dbias: bool = True, gelu_grad: bool = False, accumulate: bool = False,
                   sms: int = 148):
    """The launches of a call as (kernel, tile width, CTAs sharing K, CTAs per SM), by name; adapters: dweight
    stands for dlora_a and dbias for dlora_b."""
    out = (_int * 12)()
    flags = sum(bool(f) << i for i, f in enumerate((dinp, dweight, dbias, gelu_grad, accumulate)))
    n = lib().nb_debug_route(call, BT, C, OC, r, act, flags, sms, out)
    if n < 0:
        raise NbError(-n, lib().nb_last_error().decode())
    return [(ROUTES[out[4 * i]], *out[4 * i + 1:4 * i + 4]) for i in range(n)]


def nb_kernel_launches() -> int:
    return int(lib().nb_kernel_launches())


def nb_debug_gemm_timeout(out, inp, weight, limit_us: int) -> None:
    """One-tile forward GEMM whose producer stops half way: exercises the kernel's time-out exit."""
    lib().nb_set_stream(_stream())
    _check(lib().nb_debug_gemm_timeout(_ptr(out), _ptr(inp), _ptr(weight), limit_us))


def nb_debug_layernorm_timeout(out, inp, weight, stats, backward: bool, limit_us: int) -> None:
    """A layer norm of [5000, 64] whose rows never come whole: exercises the kernels' time-out exit."""
    lib().nb_set_stream(_stream())
    _check(lib().nb_debug_layernorm_timeout(_ptr(out), _ptr(inp), _ptr(weight), _ptr(stats), int(backward), limit_us))


def nb_debug_muon_timeout(update, grad, workspace, workspace_bytes: int, limit_us: int) -> None:
    """An update of one matrix [128, 128] whose tiles never come whole: exercises the time-out exit of blocks that wait for one another."""
    lib().nb_set_stream(_stream())
    _check(lib().nb_debug_muon_timeout(_ptr(update), _ptr(grad), _ptr(workspace), workspace_bytes, limit_us))


def nb_debug_attention_timeout(tensors, which: int, limit_us: int) -> None:
    """A pass of attention over 256 rows (512 of passes 8 to 10) whose streamed tiles never come whole: exercises the kernels' time-out exit."""
    lib().nb_set_stream(_stream())
    _check(lib().nb_debug_attention_timeout((_vp * len(tensors))(*(_ptr(t) for t in tensors)), which, limit_us))


def nb_debug_wait_timeout(limit_us: int) -> None:
    lib().nb_set_stream(_stream())
    _check(lib().nb_debug_wait_timeout(limit_us))


# ------------------------------------------------------------------ conveniences (allocation only)

def linear_forward(inp, weight, bias=None, act=ACT_NONE):
    """Allocate the outputs and call nb_linear_forward_ex. Returns (out, pre_act or None)."""
    return (_native or _load_native()).linear_forward(inp, weight, bias, act)


def linear_backward(dout, inp, weight, pre_act=None, inp_pre_act=None, act=ACT_NONE, dweight=None,
                    dbias=None, accumulate=False, need_dinp=True, need_dweight=True,
                    need_dbias=True):
    """Allocate missing outputs and call nb_linear_backward_ex. Returns (dinp, dweight, dbias)."""
    return (_native or _load_native()).linear_backward(dout, inp, weight, pre_act, inp_pre_act, act, dweight, dbias,
                                                       accumulate, need_dinp, need_dweight, need_dbias)


def _stream_dtype(t) -> int:
    if t.dtype not in (torch.bfloat16, torch.float32):
        raise TypeError(f"a tensor of bf16 or fp32 is wanted, not {t.dtype}")
    return DTYPE_F32 if t.dtype == torch.float32 else DTYPE_BF16


def _want(t, dtype, shape, name: str) -> None:
    if t is not None and (t.dtype != dtype or tuple(t.shape) != tuple(shape)):
        raise ValueError(f"{name}: {dtype} {tuple(shape)} is wanted, not {t.dtype} {tuple(t.shape)}")


def layernorm_forward(inp, weight, bias=None, branch=None, eps=1e-5, train=True):
    """Allocate the outputs and call nb_layernorm_forward. inp [BT, C] is the residual stream (bf16 or fp32), branch what it takes
    up (bf16). Returns (out, sum, mean, rstd): sum is inp where there is no branch; mean and rstd are None unless train."""
    BT, C = inp.shape
    dtype = _stream_dtype(inp)
    _want(branch, torch.bfloat16, (BT, C), "branch")
    _want(weight, torch.bfloat16, (C,), "weight")
    _want(bias, torch.bfloat16, (C,), "bias")
    out = torch.empty((BT, C), dtype=torch.bfloat16, device=inp.device)
    total = None if branch is None else torch.empty_like(inp)
    mean, rstd = (torch.empty(BT, dtype=torch.float32, device=inp.device) for _ in range(2)) if train else (None, None)
    nb_layernorm_forward(out, total, mean, rstd, inp, branch, weight, bias, BT, C, eps, dtype)
    return out, inp if branch is None else total, mean, rstd


def layernorm_backward(dout, inp, mean, rstd, weight, dres=None, dweight=None, dbias=None, accumulate=False, need_dweight=True,
                       need_dbias=True):
    """Allocate missing outputs and call nb_layernorm_backward. inp is the sum that the forward pass normed. Returns (dinp, dbranch,
    dweight, dbias): dinp in the stream's type, dbranch the same in bf16 (dinp itself where the stream is bf16)."""
    BT, C = inp.shape
    dtype = _stream_dtype(inp)
    _want(dout, torch.bfloat16, (BT, C), "dout")
    _want(dres, inp.dtype, (BT, C), "dres")
    _want(weight, torch.bfloat16, (C,), "weight")
    for t, name in ((mean, "mean"), (rstd, "rstd")):
        _want(t, torch.float32, (BT,), name)
    for t, name in ((dweight, "dweight"), (dbias, "dbias")):
        _want(t, torch.float32, (C,), name)
    dinp = torch.empty_like(inp)
    dbranch = dinp if dtype == DTYPE_BF16 else torch.empty((BT, C), dtype=torch.bfloat16, device=inp.device)
    if need_dweight and dweight is None:
        dweight = torch.zeros(C, dtype=torch.float32, device=inp.device) if accumulate else torch.empty(C, dtype=torch.float32, device=inp.device)
    if need_dbias and dbias is None:
        dbias = torch.zeros(C, dtype=torch.float32, device=inp.device) if accumulate else torch.empty(C, dtype=torch.float32, device=inp.device)
    ws = torch.empty(nb_layernorm_workspace(BT, C) if need_dweight or need_dbias else 0, dtype=torch.uint8, device=inp.device)
    nb_layernorm_backward(dinp, None if dbranch is dinp else dbranch, dweight if need_dweight else None,
                          dbias if need_dbias else None, dout, dres, inp, mean, rstd, weight, BT, C, int(accumulate), dtype,
                          ws, ws.numel())
    return dinp, dbranch, dweight, dbias


MUON_COEFFICIENTS = (3.4445, -4.7750, 2.0315)


def muon_update(grad, momentum=None, mu=0.95, nesterov=True, steps=5, coefficients=MUON_COEFFICIENTS, eps=1e-7):
    """Allocate the updates and the workspace and call nb_muon_update. grad is a list of matrices of one shape and type (fp32 or bf16),
    momentum their fp32 momenta (changed in place) or None. Returns the list of updates (bf16)."""
    if not grad:
        return []
    R, C = grad[0].shape
    if any(g.shape != (R, C) or g.dtype != grad[0].dtype for g in grad):
        raise ValueError("the matrices of a call have one shape and one type")
    if momentum is not None and any(m.shape != (R, C) or m.dtype != torch.float32 for m in momentum):
        raise ValueError("momenta are fp32, of the gradients' shape")
    update = [torch.empty((R, C), dtype=torch.bfloat16, device=g.device) for g in grad]
    ws = torch.empty(nb_muon_workspace(len(grad), R, C), dtype=torch.uint8, device=grad[0].device)
    nb_muon_update(update, momentum, grad, len(grad), R, C, mu, int(nesterov), steps, *coefficients, eps, _stream_dtype(grad[0]), ws,
                   ws.numel())
    return update


def rotary_frequencies(R, base=10000.0, factor=1.0, low=1.0, high=32.0, original=0, device="cuda"):
    """The frequencies of nb_rotary_frequencies on the device, as nb_rotary takes them."""
    return torch.tensor(nb_rotary_frequencies(R, base, factor, low, high, original), dtype=torch.float64, device=device)


def _heads(t, name: str):
    """(heads, D, ld) of a tensor [T, heads, D], whose rows may lie inside wider ones."""
    if t.dtype != torch.bfloat16 or t.dim() != 3:
        raise ValueError(f"{name}: {torch.bfloat16} [T, heads, D] is wanted, not {t.dtype} {tuple(t.shape)}")
    T, heads, D = t.shape
    # of one row no stride is told: any will do
    return heads, D, t.stride(0) if T > 1 else heads * D


def _sequences(cu_seqlens, n: int, T: int, **others) -> int:
    for name, t in others.items():
        if t is not None and t.shape[0] != T:
            raise ValueError(f"{name}: {t.shape[0]} rows, not {T}")
    if cu_seqlens is None:
        return n
    if cu_seqlens.dtype != torch.int32 or cu_seqlens.dim() != 1 or len(cu_seqlens) < 1:
        raise ValueError(f"cu_seqlens: {torch.int32} [n + 1] is wanted, not {cu_seqlens.dtype} {tuple(cu_seqlens.shape)}")
    return len(cu_seqlens) - 1


def _like(t, cu_seqlens, n, shape=None, dtype=torch.bfloat16):
    """A dense tensor of t's shape; of zeros where there may be rows in no sequence, which a call does not write."""
    make = torch.empty if cu_seqlens is None and n > 0 else torch.zeros
    return make(t.shape if shape is None else shape, dtype=dtype, device=t.device)


def rotary(q, k, freq, positions=None, cu_seqlens=None, n=1, scale=1.0, layout=ROTARY_HALF, inverse=False, in_place=False):
    """nb_rotary of q [T, heads, D] and k [T, kv_heads, D] (or None); freq has R / 2 frequencies. Returns (q, k), new ones unless in_place."""
    T = q.shape[0]
    heads, D, ld_q = _heads(q, "q")
    kv_heads, Dk, ld_k = _heads(k, "k") if k is not None else (1, D, D)
    if Dk != D:
        raise ValueError(f"k: heads of {Dk} columns, not {D}")
    _want(freq, torch.float64, (freq.numel(),), "freq")
    _want(positions, torch.int32, (T,), "positions")
    n = _sequences(cu_seqlens, n, T, k=k)
    out_q = q if in_place else _like(q, cu_seqlens, n)
    out_k = k if in_place or k is None else _like(k, cu_seqlens, n)
    nb_rotary(out_q, out_k, q, k, freq, positions, cu_seqlens, T, n, heads, kv_heads, D, 2 * freq.numel(), ld_q if in_place else heads * D,
              ld_k if in_place else kv_heads * D, ld_q, ld_k, scale, layout, int(inverse))
    return out_q, out_k


def _attention_sizes(q, k, v):
    (heads, D, ld_q), (kv_heads, Dk, ld_k), (kv2, Dv, ld_v) = _heads(q, "q"), _heads(k, "k"), _heads(v, "v")
    if Dk != D or Dv != D or kv2 != kv_heads:
        raise ValueError(f"k and v: heads of {D} columns are wanted, as many of both, not {tuple(k.shape)} and {tuple(v.shape)}")
    return heads, kv_heads, D, ld_q, ld_k, ld_v


def attention_forward(q, k, v, cu_seqlens=None, n=1, scale=None, causal=True, train=True):
    """Allocate the outputs and call nb_attention_forward. q [T, heads, D], k and v [T, kv_heads, D]: dense, or columns of wider tensors.
    Sequences by cu_seqlens (int32), or n of one length. scale: 1 / sqrt(D) where it is None. Returns (out, lse or None); rows in no sequence are zeros."""
    T = q.shape[0]
    heads, kv_heads, D, ld_q, ld_k, ld_v = _attention_sizes(q, k, v)
    n = _sequences(cu_seqlens, n, T, k=k, v=v)
    out = _like(q, cu_seqlens, n)
    lse = _like(q, cu_seqlens, n, (heads, T), torch.float32) if train else None
    nb_attention_forward(out, lse, q, k, v, cu_seqlens, T, n, heads, kv_heads, D, heads * D, ld_q, ld_k, ld_v, D ** -0.5 if scale is None else scale,
                         int(causal))
    return out, lse


def attention_backward(dout, out, lse, q, k, v, cu_seqlens=None, n=1, scale=None, causal=True, grads=None):
    """Allocate the workspace and missing gradients and call nb_attention_backward. grads: (dq, dk, dv) to be written, columns of one
    buffer for example; rows in no sequence are left as they are (zeros where they are allocated here). Returns (dq, dk, dv)."""
    T = q.shape[0]
    heads, kv_heads, D, ld_q, ld_k, ld_v = _attention_sizes(q, k, v)
    n = _sequences(cu_seqlens, n, T, k=k, v=v)
    for t, name in ((dout, "dout"), (out, "out")):
        _want(t, torch.bfloat16, q.shape, name)
    _want(lse, torch.float32, (heads, T), "lse")
    dq, dk, dv = grads if grads is not None else (_like(t, cu_seqlens, n) for t in (q, k, v))
    for t, like, name in ((dq, q, "dq"), (dk, k, "dk"), (dv, v, "dv")):
        _want(t, torch.bfloat16, like.shape, name)
    ws = torch.empty(nb_attention_workspace(T, heads), dtype=torch.uint8, device=q.device)
    nb_attention_backward(dq, dk, dv, dout, out, lse, q, k, v, cu_seqlens, T, n, heads, kv_heads, D, *(_heads(t, "")[2] for t in (dq, dk, dv, dout, out)),
                          ld_q, ld_k, ld_v, D ** -0.5 if scale is None else scale, int(causal), ws, ws.numel())
    return dq, dk, dv
