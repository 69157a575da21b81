"""ctypes binding of libslim (``include/slim.h``): argument marshalling only.

Every computation runs in the HIP kernels of ``libslim.so``; this module only turns torch
tensors into device pointers, sizes and the current HIP stream. There is no fallback: if the
library is missing, loading it raises.

Low-level functions carry the C names (``slim_pack``, ``slim_pack_bwd``, ``slim_linear``,
``slim_linear_bwd_dx``, ...) and take raw integers. The tensor-level helpers ``pack``,
``pack_bwd``, ``linear`` and ``bwd_dx`` allocate outputs and a cached workspace with torch.
"""
from __future__ import annotations

import ctypes
import os
import re
import threading

HERE = os.path.dirname(os.path.abspath(__file__))
LIB_PATH = os.path.join(HERE, "libslim.so")
HEADER = os.path.join(os.path.dirname(HERE), "include", "slim.h")

# slim_status and slim_dtype of include/slim.h (a CPU test checks them against the header)
(SLIM_OK, SLIM_EINVAL, SLIM_ESHAPE, SLIM_EDTYPE, SLIM_EALIGN, SLIM_ENONFINITE, SLIM_EWORKSPACE, SLIM_EDEVICE,
 SLIM_EUNSUPPORTED, SLIM_ERANGE) = range(10)
SLIM_F16, SLIM_BF16, SLIM_F32 = 0, 1, 2
SLIM_Q8_E4M3 = 3

_c_i64 = ctypes.c_int64
_c_p = ctypes.c_void_p
_SIGS = {
    "slim_status_string": (ctypes.c_char_p, [ctypes.c_int]),
    "slim_abi_version": (ctypes.c_int, []),
    "slim_pack": (ctypes.c_int, [_c_p, _c_i64, _c_i64, _c_p, _c_p, _c_p, _c_p, _c_p]),
    "slim_pack_bwd": (ctypes.c_int, [_c_p, _c_p, _c_p, _c_i64, _c_i64, _c_p, _c_p, _c_p, _c_p, _c_p]),
    "slim_pack_adapter": (ctypes.c_int, [_c_p, _c_p, _c_i64, _c_i64, _c_i64, _c_p, _c_p, _c_p]),
    "slim_linear_workspace": (ctypes.c_int, [_c_i64, _c_i64, _c_i64, _c_i64, ctypes.POINTER(ctypes.c_size_t)]),
    "slim_bwd_dx_workspace": (ctypes.c_int, [_c_i64, _c_i64, _c_i64, _c_i64, ctypes.POINTER(ctypes.c_size_t)]),
    "slim_workspace_init": (ctypes.c_int, [_c_p, ctypes.c_size_t, _c_p]),
    "slim_linear": (ctypes.c_int, [_c_p, ctypes.c_int, _c_i64, _c_i64, _c_i64, _c_p, _c_p, _c_p, _c_p, _c_p, _c_i64,
                                   _c_p, _c_p, ctypes.c_size_t, _c_p]),
    "slim_linear_bwd_dx": (ctypes.c_int, [_c_p, ctypes.c_int, _c_i64, _c_i64, _c_i64, _c_p, _c_p, _c_p, _c_p, _c_p,
                                          _c_i64, _c_p, _c_p, ctypes.c_size_t, _c_p]),
    "slim_pack_adapter_q": (ctypes.c_int, [_c_p, _c_p, _c_i64, _c_i64, _c_i64, _c_p, _c_p, _c_p, _c_p, _c_p]),
    "slim_linear_qa_workspace": (ctypes.c_int, [_c_i64, _c_i64, _c_i64, _c_i64, ctypes.POINTER(ctypes.c_size_t)]),
    "slim_linear_qa": (ctypes.c_int, [_c_p, ctypes.c_int, _c_i64, _c_i64, _c_i64, _c_p, _c_p, _c_p, _c_p, _c_p, _c_p,
                                      _c_p, _c_i64, _c_p, _c_p, ctypes.c_size_t, _c_p]),
    "slim_linear_noalloc": (ctypes.c_int, [_c_p, ctypes.c_int, _c_i64, _c_i64, _c_i64, _c_p, _c_p, _c_p, _c_p, _c_p,
                                           _c_i64, _c_p, _c_p]),
    "slim_pack16": (ctypes.c_int, [_c_p, _c_i64, _c_i64, _c_p, _c_p, _c_p, _c_p]),
    "slim_pack16_t": (ctypes.c_int, [_c_p, _c_p, _c_i64, _c_i64, _c_p, _c_p, _c_p]),
    "slim_grad_w": (ctypes.c_int, [_c_p, _c_p, ctypes.c_int, _c_i64, _c_i64, _c_i64, _c_p, _c_p, _c_p]),
    "slim_sparse_add": (ctypes.c_int, [_c_p, _c_p, ctypes.c_float, ctypes.c_float, _c_p, _c_i64, _c_p]),
    "slim_update_pack16": (ctypes.c_int, [_c_p, _c_i64, _c_p, _c_p]),
    "slim_quant_bins": (ctypes.c_int, [_c_i64, _c_i64]),
    "slim_quant_search": (ctypes.c_int, [_c_p, _c_i64, ctypes.c_int, _c_i64, _c_p, _c_p, _c_p]),
    "slim_pack_alpha": (ctypes.c_int, [_c_p, _c_i64, _c_i64, _c_p, _c_p, _c_p, _c_p, _c_p, _c_p]),
    "slim_hybrid_layout": (ctypes.c_int, [_c_p, _c_i64, _c_i64, _c_p, ctypes.POINTER(ctypes.c_size_t)]),
    "slim_pack_hybrid": (ctypes.c_int, [_c_p, _c_i64, _c_i64, _c_p, _c_p, _c_p, ctypes.c_size_t, _c_p]),
    "slim_linear_hybrid_workspace": (ctypes.c_int, [_c_i64, _c_i64, _c_i64, ctypes.POINTER(ctypes.c_size_t)]),
    "slim_linear_hybrid": (ctypes.c_int, [_c_p, _c_i64, _c_i64, _c_i64, _c_p, _c_p, ctypes.c_size_t, _c_p, _c_p,
                                          ctypes.c_size_t, _c_p]),
    "slim_lora_workspace": (ctypes.c_int, [_c_i64, _c_i64, _c_i64, _c_i64, ctypes.POINTER(ctypes.c_size_t)]),
    "slim_lora": (ctypes.c_int, [_c_p, _c_i64, _c_i64, _c_p, _c_p, _c_p, _c_p, ctypes.c_int, _c_i64, _c_i64, _c_p,
                                 _c_p, _c_p, ctypes.POINTER(ctypes.c_int), _c_p, ctypes.c_size_t, _c_p]),
    "slim_quant8": (ctypes.c_int, [_c_p, ctypes.c_int, _c_i64, _c_i64, _c_i64, _c_p, _c_p, _c_p]),
    "slim_dequant8": (ctypes.c_int, [_c_p, _c_p, _c_i64, _c_i64, _c_p, ctypes.c_int, _c_i64, _c_p]),
    "slim_pack8": (ctypes.c_int, [_c_p, ctypes.c_int, _c_i64, _c_i64, _c_i64, _c_p, _c_p, _c_p, _c_p, _c_p]),
    "slim_linear8_workspace": (ctypes.c_int, [ctypes.c_int, _c_i64, _c_i64, _c_i64, ctypes.POINTER(ctypes.c_size_t)]),
    "slim_linear8": (ctypes.c_int, [_c_p, ctypes.c_int, _c_p, _c_i64, _c_i64, _c_i64, _c_i64, _c_p, _c_p, _c_p,
                                    ctypes.c_int, _c_i64, _c_p, ctypes.c_size_t, _c_p]),
    "slim_grad_w8_workspace": (ctypes.c_int, [_c_i64, _c_i64, _c_i64, ctypes.c_int, ctypes.c_int,
                                              ctypes.POINTER(ctypes.c_size_t)]),
    "slim_grad_w8": (ctypes.c_int, [_c_p, ctypes.c_int, _c_i64, _c_p, _c_p, _c_i64, _c_i64, _c_i64, _c_p, _c_p, _c_p,
                                    ctypes.c_size_t, _c_p]),
    "slim_norm": (ctypes.c_int, [_c_p, ctypes.c_int, _c_i64, _c_i64, _c_i64, _c_p, _c_p, ctypes.c_int, ctypes.c_int,
                                 ctypes.c_float, _c_p, ctypes.c_int, _c_i64, _c_p, _c_p, _c_p, _c_p]),
    "slim_norm_bwd_workspace": (ctypes.c_int, [_c_i64, _c_i64, ctypes.POINTER(ctypes.c_size_t)]),
    "slim_norm_bwd": (ctypes.c_int, [_c_p, ctypes.c_int, _c_i64, _c_p, ctypes.c_int, _c_p, _c_i64, _c_i64, _c_i64,
                                     _c_p, ctypes.c_int, _c_p, _c_p, _c_p, _c_i64, _c_p, _c_p, _c_p, ctypes.c_size_t,
                                     _c_p]),
    "slim_timing_enable": (ctypes.c_int, [ctypes.c_int]),
    "slim_timing_reset": (ctypes.c_int, []),
    "slim_timing_read": (ctypes.c_int, [ctypes.c_char_p, ctypes.c_size_t]),
}

_lib = None


class SlimError(RuntimeError):
    def __init__(self, status: int, where: str):
        self.status = status
        super().__init__(f"{where}: {status_string(status)}")


def lib():
    """The loaded libslim.so (raises if it has not been built)."""
    global _lib
    if _lib is None:
        if not os.path.exists(LIB_PATH):
            raise RuntimeError(f"{LIB_PATH} is missing; build it with `python -m paper_2608_24070_amd.build`")
        L = ctypes.CDLL(LIB_PATH)
        for name, (res, args) in _SIGS.items():
            fn = getattr(L, name)
            fn.restype = res
            fn.argtypes = args
        _lib = L
    return _lib


def header_symbols() -> list[str]:
    """Entry points declared in include/slim.h."""
    text = open(HEADER).read()
    return sorted(set(re.findall(r"^\s*(?:int|const char\*)\s+(slim_\w+)\s*\(", text, flags=re.M)))


def status_string(status: int) -> str:
    return lib().slim_status_string(status).decode()


def _check(status: int, where: str):
    if status != SLIM_OK:
        raise SlimError(status, where)


# ------------------------------------------------------------------ raw C entry points

def slim_abi_version() -> int:
    return lib().slim_abi_version()


def slim_status_string(status: int) -> str:
    return status_string(status)


def slim_pack(W, N, K, codes, meta, scales, mask, stream) -> int:
    return lib().slim_pack(W, N, K, codes, meta, scales, mask, stream)


def slim_quant_bins(N, K) -> int:
    return lib().slim_quant_bins(N, K)


def slim_quant_search(W, count, bits, bins, hist, out, stream) -> int:
    return lib().slim_quant_search(W, count, bits, bins, hist, out, stream)


def slim_pack_alpha(W, N, K, alpha, codes, meta, scales, mask, stream) -> int:
    return lib().slim_pack_alpha(W, N, K, alpha, codes, meta, scales, mask, stream)


def slim_hybrid_layout(kinds, N, K, tile_info, payload_bytes) -> int:
    return lib().slim_hybrid_layout(kinds, N, K, tile_info, payload_bytes)


def slim_pack_hybrid(W, N, K, kinds, tile_info, payload, payload_bytes, stream) -> int:
    return lib().slim_pack_hybrid(W, N, K, kinds, tile_info, payload, payload_bytes, stream)


def slim_linear_hybrid_workspace(M, N, K) -> int:
    out = ctypes.c_size_t(0)
    _check(lib().slim_linear_hybrid_workspace(M, N, K, ctypes.byref(out)), "slim_linear_hybrid_workspace")
    return out.value


def slim_linear_hybrid(X, M, N, K, tile_info, payload, payload_bytes, Y, ws, ws_bytes, stream) -> int:
    return lib().slim_linear_hybrid(X, M, N, K, tile_info, payload, payload_bytes, Y, ws, ws_bytes, stream)


def slim_lora_workspace(N, K, B, r) -> int:
    out = ctypes.c_size_t(0)
    _check(lib().slim_lora_workspace(N, K, B, r, ctypes.byref(out)), "slim_lora_workspace")
    return out.value


def slim_lora(W, N, K, codes, meta, scales, X, xdtype, B, r, L, R, sigma, sweeps, ws, ws_bytes, stream) -> int:
    return lib().slim_lora(W, N, K, codes, meta, scales, X, xdtype, B, r, L, R, sigma, sweeps, ws, ws_bytes, stream)


def slim_pack_bwd(codes, meta, scales, N, K, codesT, metaT, scalesT, mask_rc, stream) -> int:
    return lib().slim_pack_bwd(codes, meta, scales, N, K, codesT, metaT, scalesT, mask_rc, stream)


def slim_pack_adapter(L, R, K, N, r, Lt, Rt, stream) -> int:
    return lib().slim_pack_adapter(L, R, K, N, r, Lt, Rt, stream)


def slim_linear_workspace(M, N, K, r) -> int:
    out = ctypes.c_size_t(0)
    _check(lib().slim_linear_workspace(M, N, K, r, ctypes.byref(out)), "slim_linear_workspace")
    return out.value


def slim_bwd_dx_workspace(M, N, K, r) -> int:
    out = ctypes.c_size_t(0)
    _check(lib().slim_bwd_dx_workspace(M, N, K, r, ctypes.byref(out)), "slim_bwd_dx_workspace")
    return out.value


def slim_workspace_init(ws, nbytes, stream) -> int:
    return lib().slim_workspace_init(ws, nbytes, stream)


def slim_linear(X, xdtype, M, N, K, codes, meta, scales, Lt, Rt, r, Y, ws, ws_bytes, stream) -> int:
    return lib().slim_linear(X, xdtype, M, N, K, codes, meta, scales, Lt, Rt, r, Y, ws, ws_bytes, stream)


def slim_pack_adapter_q(L, R, K, N, r, Lq, Ls, Rq, Rs, stream) -> int:
    return lib().slim_pack_adapter_q(L, R, K, N, r, Lq, Ls, Rq, Rs, stream)


def slim_linear_qa_workspace(M, N, K, r) -> int:
    out = ctypes.c_size_t(0)
    _check(lib().slim_linear_qa_workspace(M, N, K, r, ctypes.byref(out)), "slim_linear_qa_workspace")
    return out.value


def slim_linear_qa(X, xdtype, M, N, K, codes, meta, scales, Lq, Ls, Rq, Rs, r, Y, ws, ws_bytes, stream) -> int:
    return lib().slim_linear_qa(X, xdtype, M, N, K, codes, meta, scales, Lq, Ls, Rq, Rs, r, Y, ws, ws_bytes, stream)


def slim_linear_noalloc(X, xdtype, M, N, K, codes, meta, scales, Lt, Rt, r, Y, stream) -> int:
    return lib().slim_linear_noalloc(X, xdtype, M, N, K, codes, meta, scales, Lt, Rt, r, Y, stream)


SLIM_NOALLOC_SCRATCH_BYTES = 64 << 20


def slim_linear_bwd_dx(dY, dydtype, M, N, K, codesT, metaT, scalesT, L, R, r, dX, ws, ws_bytes, stream) -> int:
    return lib().slim_linear_bwd_dx(dY, dydtype, M, N, K, codesT, metaT, scalesT, L, R, r, dX, ws, ws_bytes, stream)


def slim_pack16(W, N, K, vals, meta, mask, stream) -> int:
    return lib().slim_pack16(W, N, K, vals, meta, mask, stream)


def slim_pack16_t(vals, meta, N, K, valsT, metaT, stream) -> int:
    return lib().slim_pack16_t(vals, meta, N, K, valsT, metaT, stream)


def slim_grad_w(dY, X, dtype, M, N, K, meta, gW, stream) -> int:
    return lib().slim_grad_w(dY, X, dtype, M, N, K, meta, gW, stream)


def slim_sparse_add(A, B, beta, gamma, out, count, stream) -> int:
    return lib().slim_sparse_add(A, B, beta, gamma, out, count, stream)


def slim_update_pack16(Wnew, count, vals, stream) -> int:
    return lib().slim_update_pack16(Wnew, count, vals, stream)


def slim_quant8(X, dtype, M, K, ldx, codes, exps, stream) -> int:
    return lib().slim_quant8(X, dtype, M, K, ldx, codes, exps, stream)


def slim_dequant8(codes, exps, M, K, Y, dtype, ldy, stream) -> int:
    return lib().slim_dequant8(codes, exps, M, K, Y, dtype, ldy, stream)


def slim_pack8(W, dtype, N, K, ldw, codes, exps, codesT, expsT, stream) -> int:
    return lib().slim_pack8(W, dtype, N, K, ldw, codes, exps, codesT, expsT, stream)


def slim_linear8_workspace(xdtype, M, N, K) -> int:
    out = ctypes.c_size_t(0)
    _check(lib().slim_linear8_workspace(xdtype, M, N, K, ctypes.byref(out)), "slim_linear8_workspace")
    return out.value


def slim_linear8(X, xdtype, xexps, M, N, K, ldx, codes, exps, Y, ydtype, ldy, ws, ws_bytes, stream) -> int:
    return lib().slim_linear8(X, xdtype, xexps, M, N, K, ldx, codes, exps, Y, ydtype, ldy, ws, ws_bytes, stream)


def slim_grad_w8_workspace(M, N, K, masked, aligned) -> int:
    out = ctypes.c_size_t(0)
    _check(lib().slim_grad_w8_workspace(M, N, K, masked, aligned, ctypes.byref(out)), "slim_grad_w8_workspace")
    return out.value


def slim_grad_w8(dY, dtype, lddy, xcodes, xexps, M, N, K, meta, gW, ws, ws_bytes, stream) -> int:
    return lib().slim_grad_w8(dY, dtype, lddy, xcodes, xexps, M, N, K, meta, gW, ws, ws_bytes, stream)


def slim_norm(X, dtype, M, K, ldx, gamma, beta, pdtype, rms, eps, Y, ydtype, ldy, yexps, mean, rstd, stream) -> int:
    return lib().slim_norm(X, dtype, M, K, ldx, gamma, beta, pdtype, rms, eps, Y, ydtype, ldy, yexps, mean, rstd, stream)


def slim_norm_bwd_workspace(M, K) -> int:
    out = ctypes.c_size_t(0)
    _check(lib().slim_norm_bwd_workspace(M, K, ctypes.byref(out)), "slim_norm_bwd_workspace")
    return out.value


def slim_norm_bwd(dY, dtype, lddy, X, xdtype, xexps, ldx, M, K, gamma, pdtype, mean, rstd, dX, lddx, dgamma, dbeta, ws,
                  ws_bytes, stream) -> int:
    return lib().slim_norm_bwd(dY, dtype, lddy, X, xdtype, xexps, ldx, M, K, gamma, pdtype, mean, rstd, dX, lddx, dgamma,
                               dbeta, ws, ws_bytes, stream)


def slim_timing_enable(on: bool) -> int:
    return lib().slim_timing_enable(1 if on else 0)


def slim_timing_reset() -> int:
    return lib().slim_timing_reset()


def slim_timing_read() -> dict:
    """{kernel name: (launches, total_ms, median_ms)} since the last reset (waits for recorded events)."""
    need = lib().slim_timing_read(None, 0)
    buf = ctypes.create_string_buffer(max(need, 1) + 256)
    lib().slim_timing_read(buf, len(buf))
    out = {}
    for line in buf.value.decode().splitlines():
        name, n, ms, med = line.split()
        out[name] = (int(n), float(ms), float(med))
    return out


# ------------------------------------------------------------------ tensor helpers

# The helpers below run on every layer call, whose kernels take about 10 us on the smallest layers, so they
# are kept short: a 4096 x 4096 call at one row took 16.1 us through ``linear`` with a torch stream object and
# a device object made twice per call (2.6 and 0.6 us each), against 9.2 us for its C call alone; it takes 11.1
# us with the raw stream handle.
_torch_mod = None


def _torch():
    global _torch_mod
    if _torch_mod is None:
        import torch
        _torch_mod = torch
    return _torch_mod


def _ptr(t):
    return None if t is None else t.data_ptr()


def _stream(stream=None):
    """The hipStream_t of `stream`, or of the current device's current stream."""
    if stream is not None:
        return stream.cuda_stream
    torch = _torch()
    raw = getattr(torch._C, "_cuda_getCurrentRawStream", None)
    if raw is None:
        return torch.cuda.current_stream().cuda_stream
    return raw(torch.cuda.current_device())


def _dtype_code(t) -> int:
    torch = _torch()
    dt = t.dtype
    if dt is torch.bfloat16:
        return SLIM_BF16
    if dt is torch.float16:
        return SLIM_F16
    raise TypeError(f"activations must be bf16 or fp16, got {dt}")


def _on_gpu(*ts):
    for t in ts:
        if t is not None and (not t.is_cuda or not t.is_contiguous()):
            raise ValueError("tensors must be contiguous and on the GPU")


_capture_calls = None


def _capturing(dev: int | None) -> bool:
    """Whether the current stream of device `dev` (None: the current one) is being captured into a graph."""
    global _capture_calls
    if _capture_calls is None:      # the calls under torch.cuda's: 0.27 us together, against 0.48
        cuda, c = _torch().cuda, _torch()._C
        _capture_calls = (getattr(c, "_cuda_getDevice", cuda.current_device),
                          getattr(c, "_cuda_isCurrentStreamCapturing", cuda.is_current_stream_capturing))
    device, captured = _capture_calls
    if dev is None or device() == dev:
        return captured()
    with _torch().cuda.device(dev):
        return captured()


_ws_cache: dict = {}
CONTROL_BYTES = 4096 * 4      # a workspace's leading control words, which start at zero


def workspace(nbytes: int, device=None, stream=None):
    """A zero-initialised workspace of at least nbytes, cached per (device, stream), whose stream clears it. Under capture into
    a graph a workspace of that call alone, from the graph's memory: a cached one is replaced when a larger call needs more.
    The graph clears its leading control words on each replay (4096 x 4096, 16 rows: 11.2 us, 9.7 without); a call that is
    given a workspace does not."""
    torch = _torch()
    if stream is not None:
        with torch.cuda.stream(stream):
            return workspace(nbytes, device)
    dev = device if isinstance(device, torch.device) else torch.device(device if device is not None else "cuda")
    if _capturing(None):
        ws = torch.empty(max(nbytes, CONTROL_BYTES), dtype=torch.uint8, device=dev)
        ws[:CONTROL_BYTES].zero_()
        return ws
    key = (dev, _stream())
    ws = _ws_cache.get(key)
    if ws is None or ws.numel() < nbytes:
        ws = torch.zeros(max(nbytes, 1 << 16), dtype=torch.uint8, device=dev)
        _ws_cache[key] = ws
    return ws


def pack(W, with_mask: bool = False, stream=None) -> dict:
    """slim_pack of an fp32 [N, K] weight. Returns codes, meta, scales (and mask)."""
    torch = _torch()
    _on_gpu(W)
    if W.dtype != torch.float32:
        raise TypeError("W must be fp32")
    N, K = W.shape
    dev = W.device
    if N % 16 or K % 128:
        raise ValueError("slim_pack needs N % 16 == 0 and K % 128 == 0")
    # rows in blocks of 16, the reduction in chunks of 128: [N/16, K/128, 16 rows, bytes per row]
    out = {
        "codes": torch.empty((N // 16, K // 128, 16, 32), dtype=torch.uint8, device=dev),
        "meta": torch.empty((N // 16, K // 128, 16, 16), dtype=torch.uint8, device=dev),
        "scales": torch.empty((N // 16, K // 128, 16), dtype=torch.int16, device=dev),
        "N": N, "K": K,
    }
    mask = torch.empty((N, K), dtype=torch.uint8, device=dev) if with_mask else None
    st = slim_pack(_ptr(W), N, K, _ptr(out["codes"]), _ptr(out["meta"]), _ptr(out["scales"]), _ptr(mask),
                   _stream(stream))
    _check(st, "slim_pack")
    if with_mask:
        out["mask"] = mask
    return out


QUANT_OUT_LEN = 4 + 2 * 30     # alpha*, E(alpha*), max|w|, candidate count, then (alpha_i, E_i) pairs


def quant_search(W, bits: int = 4, bins: int | None = None, stream=None) -> dict:
    """slim_quant_search of an fp32 tensor (SLiM-Quant). Returns {"alpha", "error", "amax", "table"
    [(alpha_i, E_i)], "hist" int32 [bins] (uint32 counts), "out" float64 device [64]}; alpha* stays
    on the device in out[0] for slim_pack_alpha."""
    torch = _torch()
    _on_gpu(W)
    if W.dtype != torch.float32 or not W.is_contiguous():
        raise TypeError("W must be a contiguous fp32 tensor")
    if bins is None:
        n, k = W.shape
        bins = slim_quant_bins(n, k)
    hist = torch.empty(bins, dtype=torch.int32, device=W.device)
    out = torch.zeros(QUANT_OUT_LEN, dtype=torch.float64, device=W.device)
    _check(slim_quant_search(_ptr(W), W.numel(), bits, bins, _ptr(hist), _ptr(out), _stream(stream)),
           "slim_quant_search")
    o = out.cpu().tolist()
    c = int(o[3])
    return {"alpha": o[0], "error": o[1], "amax": o[2], "bins": bins, "hist": hist, "out": out,
            "table": [(o[4 + 2 * i], o[5 + 2 * i]) for i in range(c)]}


def pack_alpha(W, alpha, with_mask: bool = False, stream=None) -> dict:
    """slim_pack_alpha: slim_pack with SLiM-Quant's per-tensor alpha (a device float64 tensor whose
    first element is alpha, e.g. quant_search(...)["out"]) in place of each group's absmax."""
    torch = _torch()
    _on_gpu(W)
    if W.dtype != torch.float32:
        raise TypeError("W must be fp32")
    if alpha.dtype != torch.float64 or alpha.device != W.device:
        raise TypeError("alpha must be a float64 tensor on W's device")
    N, K = W.shape
    dev = W.device
    out = {
        "codes": torch.empty((N // 16, K // 128, 16, 32), dtype=torch.uint8, device=dev),
        "meta": torch.empty((N // 16, K // 128, 16, 16), dtype=torch.uint8, device=dev),
        "scales": torch.empty((N // 16, K // 128, 16), dtype=torch.int16, device=dev),
        "N": N, "K": K,
    }
    mask = torch.empty((N, K), dtype=torch.uint8, device=dev) if with_mask else None
    _check(slim_pack_alpha(_ptr(W), N, K, _ptr(alpha), _ptr(out["codes"]), _ptr(out["meta"]), _ptr(out["scales"]),
                           _ptr(mask), _stream(stream)), "slim_pack_alpha")
    if with_mask:
        out["mask"] = mask
    return out


def pack_hybrid(W, kinds, stream=None) -> dict:
    """slim_pack_hybrid: fp32 W [N, K] (device) with a tile map (numpy uint8 [N/128, K/128], 1 = 2:4
    sparse) -> {"tile_info" int64 [N/128, K/128] (uint64 words), "payload" uint8, "N", "K"}."""
    import numpy as np
    torch = _torch()
    _on_gpu(W)
    if W.dtype != torch.float32:
        raise TypeError("W must be fp32")
    N, K = W.shape
    kinds = np.ascontiguousarray(np.asarray(kinds, dtype=np.uint8))
    if kinds.shape != (N // 128, K // 128):
        raise ValueError("the tile map must be [N/128, K/128]")
    nbytes = ctypes.c_size_t(0)
    kp = kinds.ctypes.data_as(ctypes.c_void_p)
    _check(slim_hybrid_layout(kp, N, K, None, ctypes.byref(nbytes)), "slim_hybrid_layout")
    info = torch.empty((N // 128, K // 128), dtype=torch.int64, device=W.device)
    payload = torch.empty(max(nbytes.value, 16), dtype=torch.uint8, device=W.device)
    _check(slim_pack_hybrid(_ptr(W), N, K, kp, _ptr(info), _ptr(payload), nbytes.value, _stream(stream)),
           "slim_pack_hybrid")
    return {"tile_info": info, "payload": payload, "N": N, "K": K}


_hybrid_ws: dict = {}


def _hybrid_workspace(nbytes: int, dev, stream=None):
    """slim_linear_hybrid's workspace of at least nbytes, cached per (device, stream); a captured call's own, as in
    ``workspace``. A cache of its own: the split partials must not land in slim_linear's workspace, whose control words have
    to stay zero between calls."""
    torch = _torch()
    if stream is not None:
        with torch.cuda.stream(stream):
            return _hybrid_workspace(nbytes, dev)
    if _capturing(None):
        return torch.empty(nbytes, dtype=torch.uint8, device=dev)
    key = (dev, _stream())
    ws = _hybrid_ws.get(key)
    if ws is None or ws.numel() < nbytes:
        ws = _hybrid_ws[key] = torch.empty(nbytes, dtype=torch.uint8, device=dev)
    return ws


def linear_hybrid(X, p: dict, out=None, stream=None):
    """slim_linear_hybrid: Y fp32 [M, N] = X Wp^T for fp16 X [M, K] and a hybrid pack."""
    torch = _torch()
    _on_gpu(X)
    if X.dtype != torch.float16:
        raise TypeError("X must be fp16")
    M, K = X.shape
    N = p["N"]
    if K != p["K"]:
        raise ValueError("X width does not match the pack")
    Y = out if out is not None else torch.empty((M, N), dtype=torch.float32, device=X.device)
    nb = slim_linear_hybrid_workspace(M, N, K)
    ws = _hybrid_workspace(nb, X.device, stream) if nb else None
    _check(slim_linear_hybrid(_ptr(X), M, N, K, _ptr(p["tile_info"]), _ptr(p["payload"]), p["payload"].numel(),
                              _ptr(Y), _ptr(ws), nb, _stream(stream)), "slim_linear_hybrid")
    return Y


def lora(W, packed: dict, X, r: int, stream=None) -> dict:
    """slim_lora (SLiM-LoRA): adapters L fp32 [K, r], R fp32 [r, N] with W ~ W^C + (L R)^T from the
    uncompressed weight W fp32 [N, K], its forward pack and calibration activations X [B, K]
    (bf16/fp16). Returns {"L", "R", "sigma" float64 [r], "sweeps"}."""
    torch = _torch()
    _on_gpu(W)
    _on_gpu(X)
    if W.dtype != torch.float32:
        raise TypeError("W must be fp32")
    N, K = W.shape
    B = X.shape[0]
    if X.shape[1] != K:
        raise ValueError("X must be [B, K]")
    nbytes = slim_lora_workspace(N, K, B, r)
    dev = W.device
    ws = torch.empty(max(nbytes, 256), dtype=torch.uint8, device=dev)
    L = torch.empty((K, r), dtype=torch.float32, device=dev)
    R = torch.empty((r, N), dtype=torch.float32, device=dev)
    sigma = torch.empty(max(r, 1), dtype=torch.float64, device=dev)
    sweeps = ctypes.c_int(0)
    _check(slim_lora(_ptr(W), N, K, _ptr(packed["codes"]), _ptr(packed["meta"]), _ptr(packed["scales"]), _ptr(X),
                     _dtype_code(X), B, r, _ptr(L), _ptr(R), _ptr(sigma), ctypes.byref(sweeps), _ptr(ws), nbytes,
                     _stream(stream)), "slim_lora")
    return {"L": L, "R": R, "sigma": sigma[:r], "sweeps": sweeps.value}


def pack_bwd(packed: dict, with_mask: bool = False, stream=None) -> dict:
    """slim_pack_bwd of a forward pack. Returns codesT, metaT, scalesT (and mask_rc)."""
    torch = _torch()
    N, K = packed["N"], packed["K"]
    dev = packed["codes"].device
    if N % 128:
        raise ValueError("slim_pack_bwd needs N % 128 == 0")
    # rows (k) in blocks of 16, the reduction (n) in chunks of 128; scalesT stays [K/128, N]
    out = {
        "codesT": torch.empty((K // 16, N // 128, 16, 32), dtype=torch.uint8, device=dev),
        "metaT": torch.empty((K // 16, N // 128, 16, 16), dtype=torch.uint8, device=dev),
        "scalesT": torch.empty((K // 128, N), dtype=torch.int16, device=dev),
        "N": N, "K": K,
    }
    mask = torch.empty((N, K), dtype=torch.uint8, device=dev) if with_mask else None
    st = slim_pack_bwd(_ptr(packed["codes"]), _ptr(packed["meta"]), _ptr(packed["scales"]), N, K,
                       _ptr(out["codesT"]), _ptr(out["metaT"]), _ptr(out["scalesT"]), _ptr(mask), _stream(stream))
    _check(st, "slim_pack_bwd")
    if with_mask:
        out["mask_rc"] = mask
    return out


def pack_adapter(L, R, stream=None) -> dict:
    """slim_pack_adapter of fp16 L [K, r] and R [r, N]: returns {"Lt", "Rt", "L", "R"} (the forward
    takes Lt, Rt; the backward takes L, R). Lt is L^T [r, K]; Rt is R^T in 32 x 16 tiles,
    [ceil(N/32), r/16, 32, 16]."""
    torch = _torch()
    _on_gpu(L, R)
    K, r = L.shape
    N = R.shape[1]
    out = {"Lt": torch.empty((r, K), dtype=torch.float16, device=L.device),
           "Rt": torch.empty(((N + 31) // 32, r // 16, 32, 16), dtype=torch.float16, device=L.device),
           "L": L, "R": R}
    _check(slim_pack_adapter(_ptr(L), _ptr(R), K, N, r, _ptr(out["Lt"]), _ptr(out["Rt"]), _stream(stream)),
           "slim_pack_adapter")
    return out


def linear(X, packed: dict, adapter: dict | None = None, out=None, ws=None, stream=None):
    """Y = X Wc^T + (X L) R through slim_linear. X bf16/fp16 [M, K]; adapter from pack_adapter (or None);
    Y fp32 [M, N]."""
    torch = _torch()
    Lt = None if adapter is None else adapter["Lt"]
    Rt = None if adapter is None else adapter["Rt"]
    _on_gpu(X, Lt, Rt, out, ws)
    M, K = X.shape
    N = packed["N"]
    r = 0 if Lt is None else Lt.shape[0]
    if out is None:
        out = torch.empty((M, N), dtype=torch.float32, device=X.device)
    need = slim_linear_workspace(M, N, K, r)
    if ws is None:
        ws = workspace(need, X.device, stream)
    st = slim_linear(_ptr(X), _dtype_code(X), M, N, K, _ptr(packed["codes"]), _ptr(packed["meta"]),
                     _ptr(packed["scales"]), _ptr(Lt), _ptr(Rt), r, _ptr(out), _ptr(ws), ws.numel(), _stream(stream))
    _check(st, "slim_linear")
    return out


def bwd_dx(dY, packed_bwd: dict, L=None, R=None, out=None, ws=None, stream=None):
    """dX = dY W^{R,C} + (dY R^T) L^T through slim_linear_bwd_dx. dX fp32 [M, K]."""
    torch = _torch()
    _on_gpu(dY, L, R, out, ws)
    M, N = dY.shape
    K = packed_bwd["K"]
    r = 0 if L is None else L.shape[1]
    if out is None:
        out = torch.empty((M, K), dtype=torch.float32, device=dY.device)
    need = slim_bwd_dx_workspace(M, N, K, r)
    if ws is None:
        ws = workspace(need, dY.device, stream)
    st = slim_linear_bwd_dx(_ptr(dY), _dtype_code(dY), M, N, K, _ptr(packed_bwd["codesT"]),
                            _ptr(packed_bwd["metaT"]), _ptr(packed_bwd["scalesT"]), _ptr(L), _ptr(R), r,
                            _ptr(out), _ptr(ws), ws.numel(), _stream(stream))
    _check(st, "slim_linear_bwd_dx")
    return out


def linear_noalloc(X, packed: dict, adapter: dict | None = None, out=None, stream=None):
    """Y = X Wc^T + (X L) R through slim_linear_noalloc (the library's own per-device scratch; no
    workspace). Only `out` is allocated here when not given."""
    torch = _torch()
    Lt = None if adapter is None else adapter["Lt"]
    Rt = None if adapter is None else adapter["Rt"]
    _on_gpu(X, Lt, Rt, out)
    M, K = X.shape
    N = packed["N"]
    r = 0 if Lt is None else Lt.shape[0]
    if out is None:
        out = torch.empty((M, N), dtype=torch.float32, device=X.device)
    st = slim_linear_noalloc(_ptr(X), _dtype_code(X), M, N, K, _ptr(packed["codes"]), _ptr(packed["meta"]),
                             _ptr(packed["scales"]), _ptr(Lt), _ptr(Rt), r, _ptr(out), _stream(stream))
    _check(st, "slim_linear_noalloc")
    return out


def pack_adapter_q(L, R, stream=None) -> dict:
    """slim_pack_adapter_q of fp16 L [K, r] and R [r, N]: {"Lq", "Ls", "Rq", "Rs", "K", "N", "r"}."""
    torch = _torch()
    _on_gpu(L, R)
    K, r = L.shape
    N = R.shape[1]
    dev = L.device
    out = {"Lq": torch.empty((r, K // 2), dtype=torch.uint8, device=dev),
           "Ls": torch.empty((r, (K + 127) // 128), dtype=torch.int16, device=dev),
           "Rq": torch.empty((N, r // 2), dtype=torch.uint8, device=dev),
           "Rs": torch.empty((N, (r + 127) // 128), dtype=torch.int16, device=dev),
           "K": K, "N": N, "r": r}
    _check(slim_pack_adapter_q(_ptr(L), _ptr(R), K, N, r, _ptr(out["Lq"]), _ptr(out["Ls"]), _ptr(out["Rq"]),
                               _ptr(out["Rs"]), _stream(stream)), "slim_pack_adapter_q")
    return out


def linear_qa(X, packed: dict, qadapter: dict, out=None, ws=None, stream=None):
    """Y = X Wc^T + (X L^Q) R^Q through slim_linear_qa (qadapter from pack_adapter_q). Y fp32 [M, N]."""
    torch = _torch()
    _on_gpu(X, out, ws)
    M, K = X.shape
    N, r = packed["N"], qadapter["r"]
    if out is None:
        out = torch.empty((M, N), dtype=torch.float32, device=X.device)
    need = slim_linear_qa_workspace(M, N, K, r)
    if ws is None:
        ws = workspace(need, X.device, stream)
    st = slim_linear_qa(_ptr(X), _dtype_code(X), M, N, K, _ptr(packed["codes"]), _ptr(packed["meta"]),
                        _ptr(packed["scales"]), _ptr(qadapter["Lq"]), _ptr(qadapter["Ls"]), _ptr(qadapter["Rq"]),
                        _ptr(qadapter["Rs"]), r, _ptr(out), _ptr(ws), ws.numel(), _stream(stream))
    _check(st, "slim_linear_qa")
    return out


# ------------------------------------------------- training step (value packs, SLoPe)

def pack16(W, with_mask: bool = False, stream=None) -> dict:
    """slim_pack16 of fp32 W [N, K]: {"vals" int16 [N, K/2] (fp16 bits), "meta" uint8 [N, K/8], "N", "K"}
    (+ "mask" uint8 [N, K])."""
    torch = _torch()
    _on_gpu(W)
    N, K = W.shape
    dev = W.device
    out = {"vals": torch.empty((N, K // 2), dtype=torch.int16, device=dev),
           "meta": torch.empty((N, K // 8), dtype=torch.uint8, device=dev), "N": N, "K": K}
    mask = torch.empty((N, K), dtype=torch.uint8, device=dev) if with_mask else None
    _check(slim_pack16(_ptr(W), N, K, _ptr(out["vals"]), _ptr(out["meta"]), _ptr(mask), _stream(stream)),
           "slim_pack16")
    if with_mask:
        out["mask"] = mask
    return out


def pack16_t(p: dict, out: dict | None = None, stream=None) -> dict:
    """slim_pack16_t of a value pack: {"valsT" int16 [K, N/2], "metaT" uint8 [K, N/8]} (into `out` if given)."""
    torch = _torch()
    N, K = p["N"], p["K"]
    dev = p["vals"].device
    if out is None:
        out = {"valsT": torch.empty((K, N // 2), dtype=torch.int16, device=dev),
               "metaT": torch.empty((K, N // 8), dtype=torch.uint8, device=dev)}
    _check(slim_pack16_t(_ptr(p["vals"]), _ptr(p["meta"]), N, K, _ptr(out["valsT"]), _ptr(out["metaT"]),
                         _stream(stream)), "slim_pack16_t")
    return out


def grad_w(dY, X, p: dict, out=None, stream=None):
    """slim_grad_w: fp32 [N, K/2] = (dY^T X) at the kept positions of the value pack `p` (dY [M, N], X [M, K])."""
    torch = _torch()
    _on_gpu(dY, X, out)
    M, N = dY.shape
    K = X.shape[1]
    if dY.dtype != X.dtype:
        raise ValueError("dY and X must have one dtype")
    if out is None:
        out = torch.empty((N, K // 2), dtype=torch.float32, device=dY.device)
    _check(slim_grad_w(_ptr(dY), _ptr(X), _dtype_code(dY), M, N, K, _ptr(p["meta"]), _ptr(out), _stream(stream)),
           "slim_grad_w")
    return out


def sparse_add(A, B, beta: float, gamma: float, out=None, stream=None):
    """slim_sparse_add: beta A + gamma B (A fp32, B fp16 bits as int16 or float16), same shape."""
    torch = _torch()
    _on_gpu(A, B, out)
    if out is None:
        out = torch.empty_like(A)
    _check(slim_sparse_add(_ptr(A), _ptr(B), float(beta), float(gamma), _ptr(out), A.numel(), _stream(stream)),
           "slim_sparse_add")
    return out


def update_pack16(Wnew, p: dict, stream=None) -> dict:
    """slim_update_pack16: new fp32 values [N, K/2] into p["vals"] (in place); returns p."""
    _on_gpu(Wnew)
    _check(slim_update_pack16(_ptr(Wnew), Wnew.numel(), _ptr(p["vals"]), _stream(stream)), "slim_update_pack16")
    return p


# ------------------------------------------------- the 8-bit path

# These helpers run before kernels of a few microseconds too: a check is made once, by the cheapest of torch's properties
# (a tensor's get_device() for its device), and what a helper has just made is not checked again.

_FLOAT_CODES: dict = {}
_raw_stream = None


def _float_code(dt) -> int:
    """slim_dtype of a torch floating type (fp16, bf16, fp32)."""
    code = _FLOAT_CODES.get(dt)
    if code is None:
        if not _FLOAT_CODES:
            torch = _torch()
            _FLOAT_CODES.update({torch.float16: SLIM_F16, torch.bfloat16: SLIM_BF16, torch.float32: SLIM_F32})
            return _float_code(dt)
        raise TypeError(f"expected fp16, bf16 or fp32, got {dt}")
    return code


def _stream_on(dev: int):
    """The hipStream_t of device `dev`'s current stream."""
    global _raw_stream
    if _raw_stream is None:
        torch = _torch()
        _raw_stream = getattr(torch._C, "_cuda_getCurrentRawStream", None) or (
            lambda d: torch.cuda.current_stream(d).cuda_stream)
    return _raw_stream(dev)


def _on_its_stream(stream, call, X, *args):
    """call(X, *args) with `stream` as the current one, so that what the call allocates belongs to the stream that uses it."""
    t = X["codes"] if type(X) is dict else X
    if stream.device.index != t.get_device():
        raise ValueError("the stream must be of the tensors' device")
    with _torch().cuda.stream(stream):
        return call(X, *args)


def _matrix(t, what: str):
    """(rows, columns, row stride, device) of a 2-D tensor on the GPU whose rows are contiguous."""
    if t.dim() != 2 or not t.is_cuda:
        raise ValueError(f"{what} must be a 2-D tensor on the GPU")
    m, n = t.shape
    ld, step = t.stride()
    if step != 1 and n > 1:
        raise ValueError(f"{what} must have contiguous rows")
    if ld < n:               # one row, or rows that overlap (expanded)
        if m > 1:
            raise ValueError(f"{what} must not have overlapping rows")
        ld = n
    return m, n, ld, t.get_device()


def _matrix_out(out, m: int, n: int, dtype, dev: int, what: str = "out") -> int:
    """Row stride of a given output, checked."""
    rows, cols, ld, d = _matrix(out, what)
    if (rows, cols) != (m, n) or out.dtype != dtype:
        raise ValueError(f"{what} must be ({m}, {n}) of {dtype}, got {tuple(out.shape)} of {out.dtype}")
    if d != dev:
        raise ValueError(f"{what} must be on device {dev}, got {d}")
    return ld


def _vector(t, n: int, dev: int, what: str):
    if t.shape != (n,) or not t.is_contiguous():
        raise ValueError(f"{what} must be a contiguous vector of {n}")
    if t.get_device() != dev:
        raise ValueError(f"{what} must be on device {dev}")


def _bytes_on_gpu(*ts):
    """Codes, exponents and index words: uint8, whose bytes are what they mean. (Values of another type would be read as such.)"""
    u8 = _torch().uint8
    for t in ts:
        if t.dtype is not u8:
            raise TypeError(f"codes, exponents and index words must be uint8, got {t.dtype}")
    _on_gpu(*ts)


def _rows8(q: dict, dev: int | None = None):
    """Checked parts of 8-bit rows: codes, exps, M, K, device (`dev` if given)."""
    codes, exps, M, K = q["codes"], q["exps"], q["M"], q["K"]
    if codes.shape != (M, (K + 127) // 128 * 128) or exps.shape != (M, (K + 511) // 512 * 4):
        raise ValueError("codes and exponents do not have the shape of the 8-bit rows")
    _bytes_on_gpu(codes, exps)
    d = codes.get_device()
    if d != exps.get_device() or (dev is not None and d != dev):
        raise ValueError("8-bit rows must be on one device with the other tensors")
    return codes, exps, M, K, d


def _empty_rows8(M: int, K: int, like) -> dict:
    u8 = _torch().uint8
    return {"codes": like.new_empty((M, (K + 127) // 128 * 128), dtype=u8),
            "exps": like.new_empty((M, (K + 511) // 512 * 4), dtype=u8), "M": M, "K": K}


def quant8(X, out: dict | None = None, stream=None) -> dict:
    """slim_quant8 of X [M, K] (fp16, bf16 or fp32; rows of any stride): {"codes" uint8 [M, K up to 128],
    "exps" uint8, "M", "K"}."""
    if stream is not None:
        return _on_its_stream(stream, quant8, X, out)
    M, K, ldx, dev = _matrix(X, "X")
    if out is None:
        out = _empty_rows8(M, K, X)
    else:
        _rows8(out, dev)
        if (out["M"], out["K"]) != (M, K):
            raise ValueError("out is of another shape")
    st = lib().slim_quant8(X.data_ptr(), _float_code(X.dtype), M, K, ldx, out["codes"].data_ptr(), out["exps"].data_ptr(),
                           _stream_on(dev))
    if st:
        raise SlimError(st, "slim_quant8")
    return out


def dequant8(q: dict, dtype=None, out=None, stream=None):
    """slim_dequant8: the values of 8-bit rows as [M, K] of `dtype` (bf16 if neither it nor `out` is given)."""
    if stream is not None:
        return _on_its_stream(stream, dequant8, q, dtype, out)
    codes, exps, M, K, dev = _rows8(q)
    if dtype is None:
        dtype = out.dtype if out is not None else _torch().bfloat16
    code = _float_code(dtype)
    if out is None:
        out, ldy = codes.new_empty((M, K), dtype=dtype), K
    else:
        ldy = _matrix_out(out, M, K, dtype, dev)
    st = lib().slim_dequant8(codes.data_ptr(), exps.data_ptr(), M, K, out.data_ptr(), code, ldy, _stream_on(dev))
    if st:
        raise SlimError(st, "slim_dequant8")
    return out


def pack8(W, bwd: bool = False, stream=None) -> dict:
    """slim_pack8 of W [N, K] (fp16, bf16 or fp32): {"codes", "exps", "N", "K"}, with `bwd` also the input gradient's
    {"codesT", "expsT"}."""
    if stream is not None:
        return _on_its_stream(stream, pack8, W, bwd)
    torch = _torch()
    N, K, ldw, dev = _matrix(W, "W")
    up = lambda a, b: -(-a // b)

    def empty(n, k):
        return (torch.empty((up(n, 16), up(k, 128), 2, 4, 16, 16), dtype=torch.uint8, device=W.device),
                torch.empty((up(n, 128), up(k, 512) * 4), dtype=torch.uint8, device=W.device))

    out = {"N": N, "K": K}
    out["codes"], out["exps"] = empty(N, K)
    if bwd:
        out["codesT"], out["expsT"] = empty(K, N)
    _check(slim_pack8(W.data_ptr(), _float_code(W.dtype), N, K, ldw, _ptr(out["codes"]), _ptr(out["exps"]),
                      _ptr(out.get("codesT")), _ptr(out.get("expsT")), _stream_on(dev)), "slim_pack8")
    return out


_ws8 = threading.local()


def _workspace8(nbytes: int, like, stream: int):
    """The 8-bit calls' workspace, kept per thread, device and stream: a call's launches follow each other on the stream, but
    another thread's may come between. Its contents are of no interest between calls, so it is not slim_linear's, whose
    counters have to stay zero. A captured call has one of its own, from its graph's memory: a kept one is replaced when a
    larger call needs more and goes with its thread, and the graph would then write to memory that others were given."""
    dev = like.get_device()
    if _capturing(dev):
        return like.new_empty(nbytes, dtype=_torch().uint8)
    cache = _ws8.__dict__
    key = (dev, stream)
    ws = cache.get(key)
    if ws is None or ws.numel() < nbytes:
        ws = cache[key] = like.new_empty(max(nbytes, 1 << 16), dtype=_torch().uint8)
    return ws


def _given8(nbytes: int, ws, like, stream: int):
    """(pointer, size) of the workspace of a call that needs nbytes."""
    if ws is None:
        if not nbytes:
            return None, 0
        ws = _workspace8(nbytes, like, stream)
        return ws.data_ptr(), ws.numel()
    _on_gpu(ws)
    if ws.get_device() != like.get_device():
        raise ValueError("the workspace must be on the tensors' device")
    return ws.data_ptr(), ws.numel() * ws.element_size()


def _product8(X, codes, exps, N: int, K: int, dtype, out, ws, where: str):
    if codes.shape != ((N + 15) // 16, (K + 127) // 128, 2, 4, 16, 16) or exps.shape != ((N + 127) // 128, (K + 511) // 512 * 4):
        raise ValueError("codes and exponents do not have the shape of the 8-bit weight")
    _bytes_on_gpu(codes, exps)
    if type(X) is dict:
        x, xe, M, k, dev = _rows8(X)
        xe, xdt, ldx = xe.data_ptr(), SLIM_Q8_E4M3, 0
    else:
        x, xe, xdt = X, None, _float_code(X.dtype)
        M, k, ldx, dev = _matrix(X, "X")
    if k != K:
        raise ValueError("the rows' width does not match the pack")
    if codes.get_device() != dev or exps.get_device() != dev:
        raise ValueError("X and the pack must be on one device")
    if dtype is None:
        torch = _torch()
        dtype = out.dtype if out is not None else torch.float16 if xdt == SLIM_F16 else torch.bfloat16
    ydt = _float_code(dtype)
    if out is None:
        out, ldy = x.new_empty((M, N), dtype=dtype), N
    else:
        ldy = _matrix_out(out, M, N, dtype, dev)
    L, st = lib(), _stream_on(dev)
    need = ctypes.c_size_t()
    rc = L.slim_linear8_workspace(xdt, M, N, K, need)
    if not rc:
        wp, wn = _given8(need.value, ws, x, st)
        rc = L.slim_linear8(x.data_ptr(), xdt, xe, M, N, K, ldx, codes.data_ptr(), exps.data_ptr(), out.data_ptr(), ydt, ldy, wp,
                            wn, st)
    if rc:
        raise SlimError(rc, where)
    return out


def linear8(X, p: dict, dtype=None, out=None, ws=None, stream=None):
    """slim_linear8: Y [M, N] = X W^T with an 8-bit weight (pack8). X [M, K]: 8-bit rows (quant8, norm) or an fp16, bf16
    or fp32 tensor, which the call turns into 8 bits. Y in `dtype`, fp16 or bf16 (default: fp16 for fp16 X, else bf16)."""
    if stream is not None:
        return _on_its_stream(stream, linear8, X, p, dtype, out, ws)
    return _product8(X, p["codes"], p["exps"], p["N"], p["K"], dtype, out, ws, "slim_linear8")


def bwd_dx8(dY, p: dict, dtype=None, out=None, ws=None, stream=None):
    """slim_linear8 on the transposed pack: dX [M, K] = dY W for dY [M, N] (pack8 with bwd=True); types as linear8."""
    if stream is not None:
        return _on_its_stream(stream, bwd_dx8, dY, p, dtype, out, ws)
    return _product8(dY, p["codesT"], p["expsT"], p["K"], p["N"], dtype, out, ws, "slim_linear8")


def grad_w8(dY, q: dict, p: dict | None = None, out=None, ws=None, stream=None):
    """slim_grad_w8: dY^T X for dY [M, N] (fp16, bf16) and X [M, K] in 8 bits: fp32 [N, K], or with a value pack `p`
    (pack16) fp32 [N, K/2] at the positions it keeps."""
    if stream is not None:
        return _on_its_stream(stream, grad_w8, dY, q, p, out, ws)
    m, N, ldy, dev = _matrix(dY, "dY")
    xc, xe, M, K, _ = _rows8(q, dev)
    if m != M:
        raise ValueError("dY and the checkpoint must have one number of rows")
    dt, meta, cols = _dtype_code(dY), None, K
    if p is not None:
        meta, cols = p["meta"], K // 2
        if meta.shape != (N, K // 8):
            raise ValueError("the value pack does not match dY and the checkpoint")
        _bytes_on_gpu(meta)
        if meta.get_device() != dev:
            raise ValueError("dY and the value pack must be on one device")
        meta = meta.data_ptr()
    if out is None:
        out = dY.new_empty((N, cols), dtype=_torch().float32)
    else:
        _on_gpu(out)
        _matrix_out(out, N, cols, _torch().float32, dev)
    y, L, st = dY.data_ptr(), lib(), _stream_on(dev)
    aligned = 1 if y % 16 == 0 and ldy % 8 == 0 and ldy < 1 << 22 else 0
    need = ctypes.c_size_t()
    rc = L.slim_grad_w8_workspace(M, N, K, 0 if p is None else 1, aligned, need)
    if not rc:
        wp, wn = _given8(need.value, ws, dY, st)
        rc = L.slim_grad_w8(y, dt, ldy, xc.data_ptr(), xe.data_ptr(), M, N, K, meta, out.data_ptr(), wp, wn, st)
    if rc:
        raise SlimError(rc, "slim_grad_w8")
    return out


def norm(X, gamma=None, beta=None, eps: float = 1e-5, rms: bool = False, q8: bool = False, out=None, stream=None):
    """slim_norm over the rows of X [M, K] (fp16, bf16 or fp32): layer norm, or with `rms` the RMS norm. Returns (Y, mean,
    rstd): Y of X's type, or with `q8` 8-bit rows (as quant8); mean and rstd fp32 [M] for norm_bwd, mean None with `rms`."""
    if stream is not None:
        return _on_its_stream(stream, norm, X, gamma, beta, eps, rms, q8, out)
    M, K, ldx, dev = _matrix(X, "X")
    dt = _float_code(X.dtype)
    pdt, gp, bp = SLIM_F32, None, None
    if gamma is not None:
        _vector(gamma, K, dev, "gamma")
        pdt, gp = _float_code(gamma.dtype), gamma.data_ptr()
    if beta is not None:
        _vector(beta, K, dev, "beta")
        if gamma is not None and beta.dtype != gamma.dtype:
            raise TypeError("gamma and beta must have one dtype")
        pdt, bp = _float_code(beta.dtype), beta.data_ptr()
    f32 = _torch().float32
    rstd = X.new_empty((M,), dtype=f32)
    mean = None if rms else X.new_empty((M,), dtype=f32)
    if q8:
        if out is None:
            out = _empty_rows8(M, K, X)
        else:
            _rows8(out, dev)
            if (out["M"], out["K"]) != (M, K):
                raise ValueError("out is of another shape")
        yp, ye, ydt, ldy = out["codes"].data_ptr(), out["exps"].data_ptr(), SLIM_Q8_E4M3, 0
    else:
        if out is None:
            out, ldy = X.new_empty((M, K)), K
        else:
            ldy = _matrix_out(out, M, K, X.dtype, dev)
        yp, ye, ydt = out.data_ptr(), None, dt
    rc = lib().slim_norm(X.data_ptr(), dt, M, K, ldx, gp, bp, pdt, 1 if rms else 0, eps, yp, ydt, ldy, ye,
                         None if rms else mean.data_ptr(), rstd.data_ptr(), _stream_on(dev))
    if rc:
        raise SlimError(rc, "slim_norm")
    return out, mean, rstd


def norm_bwd(dY, X, gamma, mean, rstd, out=None, ws=None, stream=None):
    """slim_norm_bwd: (dX, dgamma, dbeta) from dY [M, K], the forward's input X (dY's type, or its 8-bit checkpoint from
    quant8), gamma (or None) and the forward's mean and rstd; mean None: RMS norm, dbeta None. dX of dY's type, dgamma
    and dbeta fp32."""
    if stream is not None:
        return _on_its_stream(stream, norm_bwd, dY, X, gamma, mean, rstd, out, ws)
    M, K, lddy, dev = _matrix(dY, "dY")
    dt, pdt, gp, mp = _float_code(dY.dtype), SLIM_F32, None, None
    if type(X) is dict:
        x, xe, m, k, _ = _rows8(X, dev)
        xp, xe, xdt, ldx = x.data_ptr(), xe.data_ptr(), SLIM_Q8_E4M3, 0
    else:
        xp, xe, xdt = X.data_ptr(), None, _float_code(X.dtype)
        m, k, ldx, d = _matrix(X, "X")
        if d != dev:
            raise ValueError("dY and X must be on one device")
    if (m, k) != (M, K):
        raise ValueError("dY and X must have one shape")
    if gamma is not None:
        _vector(gamma, K, dev, "gamma")
        pdt, gp = _float_code(gamma.dtype), gamma.data_ptr()
    f32 = _torch().float32
    _vector(rstd, M, dev, "rstd")
    if mean is not None:
        _vector(mean, M, dev, "mean")
        mp = mean.data_ptr()
    if rstd.dtype != f32 or (mean is not None and mean.dtype != f32):
        raise TypeError("mean and rstd must be fp32")
    if out is None:
        out, lddx = dY.new_empty((M, K)), K
    else:
        lddx = _matrix_out(out, M, K, dY.dtype, dev)
    dgamma = dY.new_empty((K,), dtype=f32)
    dbeta = None if mean is None else dY.new_empty((K,), dtype=f32)
    L, st = lib(), _stream_on(dev)
    need = ctypes.c_size_t()
    rc = L.slim_norm_bwd_workspace(M, K, need)
    if not rc:
        wp, wn = _given8(need.value, ws, dY, st)
        rc = L.slim_norm_bwd(dY.data_ptr(), dt, lddy, xp, xdt, xe, ldx, M, K, gp, pdt, mp, rstd.data_ptr(), out.data_ptr(), lddx,
                             dgamma.data_ptr(), None if dbeta is None else dbeta.data_ptr(), wp, wn, st)
    if rc:
        raise SlimError(rc, "slim_norm_bwd")
    return out, dgamma, dbeta
