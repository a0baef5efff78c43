"""ctypes marshalling for libmixdq.so.  Tensors are torch tensors on the GPU; torch supplies device memory
and the current stream, nothing else.  Function names and argument meaning follow include/mixdq.h."""
from __future__ import annotations

import ctypes as C
import os
from dataclasses import dataclass
from typing import Optional, Union

import torch

_HERE = os.path.dirname(os.path.abspath(__file__))
_LIB_PATH = os.path.join(_HERE, "libmixdq.so")

F16, BF16 = 0, 1
F32 = 2  # parameters of the layer norm
LAYOUT_CANONICAL, LAYOUT_KERNEL = 0, 1

_ERRORS = {
    -1: "MQ_ERR_BAD_ARG", -2: "MQ_ERR_BAD_SHAPE", -3: "MQ_ERR_UNSUPPORTED_BITS", -4: "MQ_ERR_WORKSPACE_TOO_SMALL",
    -5: "MQ_ERR_HIP", -6: "MQ_ERR_UNSUPPORTED_LAYOUT", -7: "MQ_ERR_OVERFLOW_RISK", -8: "MQ_ERR_INFEASIBLE",
    -9: "MQ_ERR_TOO_LARGE",
}

EXPORTS = ("mq_version", "mq_last_hip_error", "mq_tune_force_tile", "mq_tune_force_splits", "mq_tune_force_band", "mq_prof_enable", "mq_prof_num_slots", "mq_prof_read",
           "mq_prof_reset", "mq_prof_phase_buffer", "mq_prof_filter", "mq_prof_bracket_overhead_us", "mq_prof_copy", "mq_prof_microbench", "mq_quantize_weights", "mq_packed_bytes", "mq_pack_weights",
           "mq_unpack_weights", "mq_split_workspace_bytes", "mq_qlinear_w_only", "mq_qlinear_a8_workspace_bytes", "mq_qlinear_w8a8",
           "mq_qlinear_w4a8", "mq_qlinear_w2a8", "mq_builtin_workspace_bytes", "mq_qlinear_a8_builtin_ws", "mq_a8_row_bytes", "mq_qlinear_a8_geglu", "mq_qlinear_a8_geglu_dynamic_workspace_bytes", "mq_qlinear_a8_geglu_dynamic", "mq_qlinear_w_only_geglu", "mq_qlinear_w_only_geglu_a8", "mq_qlinear_a8_codes", "mq_conv3x3_w_only",
           "mq_conv_tap_sums", "mq_conv3x3_a8_workspace_bytes", "mq_conv3x3_a8",
           "mq_bos_aware_kv_proj_workspace_bytes", "mq_bos_aware_kv_proj", "mq_alloc_solve", "mq_alloc_split_budget",
           "mq_alloc_search", "mq_mx_bytes", "mq_mx_quantize", "mq_mx_dequantize", "mq_mx_pack", "mq_mx_unpack", "mq_mx_column_top",
           "mq_mx_linear_workspace_bytes", "mq_mx_linear", "mq_mx_linear_codes", "mq_mx_linear_grad_workspace_bytes", "mq_mx_linear_grad", "mq_layer_norm", "mq_layer_norm_mx",
           "mq_layer_norm_grad_workspace_bytes", "mq_layer_norm_grad",
           "mq_rotary_table", "mq_qk_norm_rope", "mq_qk_norm_rope_grad_workspace_bytes", "mq_qk_norm_rope_grad", "mq_mx_linear_act", "mq_mx_linear_act_codes", "mq_act_grad_workspace_bytes",
           "mq_act_grad", "mq_mx_experts_column_top", "mq_mx_linear_grouped_workspace_bytes", "mq_mx_linear_grouped", "mq_mx_linear_grouped_grad")


class MixdqError(RuntimeError):
    def __init__(self, code: int, what: str):
        self.code = code
        super().__init__(f"{what}: {_ERRORS.get(code, code)}")


_lib = None
_native = None  # csrc/host.cpp: the eager calls of small layers, see there


def _done(r, what: str):
    """The result of a native call; it returns an error code in its place."""
    if r.__class__ is int:
        raise MixdqError(r, what)
    return r


def lib_path() -> str:
    return _LIB_PATH


def load():
    """Loads the HIP library; raises if it has not been built (there is no fallback path)."""
    global _lib
    if _lib is None:
        if not os.path.exists(_LIB_PATH):
            raise RuntimeError(f"{_LIB_PATH} is missing: run `python -c 'import __graft_entry__ as g; g.build()'`")
        lib = C.CDLL(_LIB_PATH)
        for name in ("mq_a8_row_bytes", "mq_split_workspace_bytes", "mq_builtin_workspace_bytes", "mq_conv3x3_a8_workspace_bytes", "mq_packed_bytes", "mq_qlinear_a8_workspace_bytes", "mq_qlinear_a8_geglu_dynamic_workspace_bytes", "mq_bos_aware_kv_proj_workspace_bytes",
                     "mq_mx_bytes", "mq_mx_linear_workspace_bytes", "mq_mx_linear_grad_workspace_bytes", "mq_layer_norm_grad_workspace_bytes", "mq_qk_norm_rope_grad_workspace_bytes", "mq_act_grad_workspace_bytes",
                     "mq_mx_linear_grouped_workspace_bytes"):
            getattr(lib, name).restype = C.c_size_t
        lib.mq_prof_bracket_overhead_us.restype = C.c_double
        _lib = lib
    return _lib


def _load_native():
    """The native marshalling, bound to the library's entry points; raises if it has not been built, or not for this torch and
    Python.  Only the calls that go through it need it."""
    global _native
    if _native is None:
        from .build import _host_made_for
        try:
            from . import _mqhost
        except ImportError as e:
            raise RuntimeError("_mqhost.so is missing or stale: run `python -c 'import __graft_entry__ as g; g.build()'`") from e
        if _mqhost.made_for != _host_made_for():
            raise RuntimeError(f"_mqhost.so was built for {_mqhost.made_for}, this is {_host_made_for()}: build again")
        lib = load()
        _mqhost.bind(*(C.cast(getattr(lib, name), C.c_void_p).value for name in (
            "mq_qlinear_w_only", "mq_qlinear_w8a8", "mq_qlinear_w4a8", "mq_qlinear_w2a8", "mq_quantize_weights", "mq_pack_weights",
            "mq_split_workspace_bytes", "mq_qlinear_a8_workspace_bytes", "mq_packed_bytes", "mq_mx_bytes", "mq_mx_quantize", "mq_mx_dequantize",
            "mq_mx_linear_workspace_bytes", "mq_mx_linear", "mq_mx_linear_codes", "mq_mx_linear_grad_workspace_bytes", "mq_mx_linear_grad",
            "mq_layer_norm", "mq_layer_norm_mx", "mq_layer_norm_grad_workspace_bytes", "mq_layer_norm_grad",
            "mq_qk_norm_rope", "mq_qk_norm_rope_grad_workspace_bytes", "mq_qk_norm_rope_grad", "mq_mx_linear_act", "mq_mx_linear_act_codes", "mq_act_grad_workspace_bytes", "mq_act_grad",
            "mq_mx_linear_grouped_workspace_bytes", "mq_mx_linear_grouped", "mq_mx_linear_grouped_grad")))
        _native = _mqhost
    return _native


def version() -> int:
    return load().mq_version()


def tune_force_tile(tile: int) -> None:
    load().mq_tune_force_tile(int(tile))


def tune_force_splits(parts: int) -> None:
    load().mq_tune_force_splits(int(parts))


def tune_force_band(rows: int) -> None:
    load().mq_tune_force_band(int(rows))


def prof_phase_buffer(buf: Optional[torch.Tensor]) -> None:
    """buf: int64 device tensor with 4 entries per workgroup, or None to switch phase timing off."""
    load().mq_prof_phase_buffer(_ptr(buf), C.c_long(0 if buf is None else buf.numel() // 4))


def prof_enable(on: bool) -> None:
    _check(load().mq_prof_enable(int(on)), "mq_prof_enable")


def prof_filter(slot: int = -1, stride: int = 1) -> None:
    _check(load().mq_prof_filter(int(slot), int(stride)), "mq_prof_filter")


def prof_bracket_overhead_us() -> float:
    return float(load().mq_prof_bracket_overhead_us(_stream()))


def prof_copy(dst: torch.Tensor, src: torch.Tensor) -> None:
    nbytes = src.numel() * src.element_size()
    assert dst.numel() * dst.element_size() == nbytes
    _check(load().mq_prof_copy(_ptr(dst), _ptr(src), C.c_size_t(nbytes), _stream()), "mq_prof_copy")


def prof_microbench(kind: int, buf: torch.Tensor) -> float:
    """Elapsed milliseconds (best of five) of microbenchmark `kind` (see include/mixdq.h); buf: device scratch."""
    ms = C.c_double(0.0)
    _check(load().mq_prof_microbench(int(kind), _ptr(buf), C.c_size_t(buf.numel() * buf.element_size()), C.byref(ms),
                                     _stream()), "mq_prof_microbench")
    return ms.value


def machine_peaks(buf: Optional[torch.Tensor] = None) -> dict:
    """Measured rates of this machine: int8 and fp16 MFMA (T(FL)OP/s), read-only stream (GB/s), LDS reads and L2 -> LDS
    copies (bytes per second over the chip), and the overlap of matrix and vector instructions on a SIMD: with 8 vector
    instructions per MFMA (as many cycles as the MFMA itself) the elapsed time of both kinds of work together divided
    by the sum of their separate times (0.5 = perfect overlap of equal halves, 1.0 = none), in one wave and in two
    waves of one SIMD; and with 4 vector instructions per MFMA the elapsed time divided by that of the MFMAs alone
    (1.0: the vector instructions are hidden completely)."""
    if buf is None:
        buf = torch.empty(2 << 30, dtype=torch.uint8, device="cuda")
    small = buf[:4 << 20]
    t = {k: prof_microbench(k, small if k != 5 else buf) for k in range(9)}
    n_mfma = 512 * 4 * 4096 * 4
    return {
        "int8_TOPs": n_mfma * 65536.0 / (t[0] * 1e-3) / 1e12,
        "f16_TFLOPs": n_mfma * 32768.0 / (t[1] * 1e-3) / 1e12,
        "read_GBps": (buf.numel() - 4096) / (t[5] * 1e-3) / 1e9,
        "lds_read_TBps": 1024 * 4 * 4000 * 8192.0 / (t[6] * 1e-3) / 1e12,
        "l2_to_lds_TBps": 768 * 4 * 2048 * 8192.0 / (t[7] * 1e-3) / 1e12,
        "mfma_ms": t[0], "valu_ms": t[2], "same_wave_ms": t[3], "two_waves_ms": t[4],
        "serial_share_same_wave": t[3] / (t[0] + t[2]), "serial_share_two_waves": t[4] / (t[0] + t[2]),
        "four_valu_per_mfma_ms": t[8], "four_valu_per_mfma_over_mfma_only": t[8] / t[0],
    }


def prof_reset() -> None:
    _check(load().mq_prof_reset(), "mq_prof_reset")


def prof_read():
    """Per-kernel totals since the last reset: list of dicts (only kernels that ran)."""
    L = load()
    out = []
    for slot in range(L.mq_prof_num_slots()):
        name = C.create_string_buffer(128)
        n = C.c_longlong()
        ms, ops, byts = C.c_double(), C.c_double(), C.c_double()
        _check(L.mq_prof_read(slot, name, 128, C.byref(n), C.byref(ms), C.byref(ops), C.byref(byts)), "mq_prof_read")
        if n.value:
            out.append({"slot": slot, "kernel": name.value.decode(), "launches": n.value, "ms": ms.value, "ops": ops.value,
                        "bytes": byts.value})
    return out


def _ptr(t: Optional[torch.Tensor]):
    return C.c_void_p(0 if t is None else t.data_ptr())


def _stream():
    return C.c_void_p(torch.cuda.current_stream().cuda_stream)


def _check(rc: int, what: str):
    if rc != 0:
        raise MixdqError(rc, what)


def _dtype_code(t: torch.Tensor) -> int:
    if t.dtype == torch.float16:
        return F16
    if t.dtype == torch.bfloat16:
        return BF16
    raise TypeError(f"expected a 16-bit float tensor, got {t.dtype}")


@dataclass
class PackedWeight:
    """A quantised, packed weight matrix resident on the GPU (what the offline step hands to the hot path)."""
    packed: torch.Tensor      # uint8 bytes
    scale: Optional[torch.Tensor]   # float32 [N] (None for unquantised 16-bit weights)
    zp: Optional[torch.Tensor]      # int32 [N]
    colsum: Optional[torch.Tensor]  # int32 [N]
    N: int
    K: int
    bits: int
    layout: int
    signed: bool


def keep_weights_16bit(w: torch.Tensor) -> PackedWeight:
    """An unquantised fp16/bf16 weight matrix in the layout the GEMM reads (a layer kept at 16 bits)."""
    packed, _ = pack_weights(w, 16, LAYOUT_KERNEL)
    return PackedWeight(packed, None, None, None, w.shape[0], w.shape[1], 16, LAYOUT_KERNEL, False)


def stack_weights(parts) -> PackedWeight:
    """Layers that share their input (a block's q, k, v projections; the K and V projections of the text context) as
    one layer: in the kernel layout the packed form of the row-stacked matrix is the concatenation of the parts'
    packed buffers (tiles are 32 output channels tall, so every part's N must be a multiple of 32), and the
    per-channel parameters concatenate likewise.  One call on the stacked weight writes [M, N1 + N2 + ...]."""
    first = parts[0]
    for p in parts:
        assert p.N % 32 == 0 and (p.K, p.bits, p.layout, p.signed) == (first.K, first.bits, LAYOUT_KERNEL, first.signed)
    cat = lambda ts: None if ts[0] is None else torch.cat(ts)
    return PackedWeight(torch.cat([p.packed for p in parts]), cat([p.scale for p in parts]), cat([p.zp for p in parts]),
                        cat([p.colsum for p in parts]), sum(p.N for p in parts), first.K, first.bits, LAYOUT_KERNEL,
                        first.signed)


def quantize_weights(w: torch.Tensor, bits: int, symmetric: bool = False):
    """W [N,K] fp16/bf16 -> (codes uint8 [N,K], scale float32 [N], zp int32 [N])."""
    lib = load()
    r = (_native or _load_native()).quantize_weights(w, bits, int(symmetric))
    if r is not None:
        return _done(r, "mq_quantize_weights")
    assert w.is_cuda and w.dim() == 2 and w.is_contiguous()
    N, K = w.shape
    codes = torch.empty((N, K), dtype=torch.uint8, device=w.device)
    scale = torch.empty(N, dtype=torch.float32, device=w.device)
    zp = torch.empty(N, dtype=torch.int32, device=w.device)
    _check(lib.mq_quantize_weights(_ptr(w), N, K, bits, int(symmetric), _dtype_code(w), _ptr(codes), _ptr(scale),
                                  _ptr(zp), _stream()), "mq_quantize_weights")
    return codes, scale, zp


def packed_bytes(N: int, K: int, bits: int, layout: int) -> int:
    return int(load().mq_packed_bytes(N, K, bits, layout))


def pack_weights(codes: torch.Tensor, bits: int, layout: int = LAYOUT_KERNEL, codes_signed: bool = False,
                 want_colsum: bool = True):
    """codes uint8 [N,K] -> (packed uint8 [bytes], colsum int32 [N] or None).  bits = 16: `codes` is the fp16/bf16
    weight matrix itself and there is no colsum."""
    lib = load()
    r = (_native or _load_native()).pack_weights(codes, bits, layout, int(codes_signed), int(want_colsum))
    if r is not None:
        return _done(r, "mq_pack_weights")
    assert codes.is_cuda and codes.dim() == 2 and codes.is_contiguous()
    assert codes.dtype == torch.uint8 if bits != 16 else codes.dtype in (torch.float16, torch.bfloat16)
    N, K = codes.shape
    nbytes = packed_bytes(N, K, bits, layout)
    packed = torch.empty(max(nbytes, 1), dtype=torch.uint8, device=codes.device)
    colsum = torch.empty(N, dtype=torch.int32, device=codes.device) if (want_colsum and bits != 16) else None
    _check(lib.mq_pack_weights(_ptr(codes), N, K, bits, layout, int(codes_signed), _ptr(packed), _ptr(colsum), _stream()),
           "mq_pack_weights")
    return packed, colsum


def unpack_weights(packed: torch.Tensor, N: int, K: int, bits: int, layout: int, dtype=torch.float16) -> torch.Tensor:
    """Codes uint8 [N,K]; for bits = 16 the weight matrix in `dtype`."""
    codes = torch.empty((N, K), dtype=torch.uint8 if bits != 16 else dtype, device=packed.device)
    _check(load().mq_unpack_weights(_ptr(packed), N, K, bits, layout, _ptr(codes), _stream()), "mq_unpack_weights")
    return codes


def _res(residual, M, N, dtype):
    """(pointer, row stride) of an optional [M,N] residual operand."""
    if residual is None:
        return C.c_void_p(0), 0
    assert residual.is_cuda and residual.dim() == 2 and residual.shape == (M, N) and residual.stride(1) == 1
    assert residual.dtype == dtype
    return _ptr(residual), residual.stride(0)


def split_workspace_bytes(M: int, N: int, K: int) -> int:
    return int(load().mq_split_workspace_bytes(M, N, K))


def _ws_args(ws: Optional[torch.Tensor]):
    return (C.c_void_p(0), C.c_size_t(0)) if ws is None else (_ptr(ws), C.c_size_t(ws.numel() * ws.element_size()))


def qlinear_w_only(x: torch.Tensor, w: PackedWeight, bias: Optional[torch.Tensor] = None,
                   out: Optional[torch.Tensor] = None, residual: Optional[torch.Tensor] = None,
                   ws: Optional[torch.Tensor] = None) -> torch.Tensor:
    """Y = X . dequant(W)^T + bias (+ residual) with 16-bit floating-point compute (weight-only quantisation).
    ws: optional uint8 workspace of split_workspace_bytes(M, N, K) bytes; allocated here when the shape can use one."""
    lib = load()
    r = (_native or _load_native()).qlinear_w_only(x, w.packed, w.N, w.K, w.bits, w.layout, w.scale, w.zp, bias, out, residual, ws)
    if r is not None:
        return _done(r, "mq_qlinear_w_only")
    assert x.is_cuda and x.dim() == 2 and x.stride(1) == 1
    M, K = x.shape
    assert K == w.K
    y = out if out is not None else torch.empty((M, w.N), dtype=x.dtype, device=x.device)
    rp, ldr = _res(residual, M, w.N, x.dtype)
    if ws is None:
        need = split_workspace_bytes(M, w.N, K)
        ws = torch.empty(need, dtype=torch.uint8, device=x.device) if need else None
    _check(lib.mq_qlinear_w_only(_ptr(x), M, K, x.stride(0), _ptr(w.packed), w.N, w.bits, w.layout, _ptr(w.scale), _ptr(w.zp),
                                 _ptr(bias), _ptr(y), y.stride(0), _dtype_code(x), rp, ldr, *_ws_args(ws), _stream()),
           "mq_qlinear_w_only")
    return y


def qlinear_a8_workspace_bytes(M: int, K: int) -> int:
    return int(load().mq_qlinear_a8_workspace_bytes(M, K))


def _workspace(nbytes: int, device, ws: Optional[torch.Tensor]):
    if ws is None:
        ws = torch.empty(nbytes, dtype=torch.uint8, device=device)
    return ws


def _qlinear_a8(fn_name, x, w: PackedWeight, act, bias, out, ws, want_acc, want_act, residual=None):
    L = load()
    if not (want_acc or want_act):
        a_s, a_z = (None, None) if act is None else act
        r = (_native or _load_native()).qlinear_a8(x, w.packed, w.N, w.K, w.bits, w.layout, int(w.signed), w.scale, w.zp, w.colsum, a_s, a_z, bias,
                               out, residual, ws)
        if r is not None:
            return _done(r, fn_name), None, (None, None)
    assert x.is_cuda and x.dim() == 2 and x.stride(1) == 1 and x.dtype == torch.float16
    M, K = x.shape
    assert K == w.K
    dev = x.device
    y = out if out is not None else torch.empty((M, w.N), dtype=torch.float16, device=dev)
    ws = _workspace(qlinear_a8_workspace_bytes(M, K) + split_workspace_bytes(M, w.N, K), dev, ws)
    acc = torch.empty((M, w.N), dtype=torch.int32, device=dev) if want_acc else None
    s_out = torch.empty(1, dtype=torch.float32, device=dev) if want_act else None
    z_out = torch.empty(1, dtype=torch.int32, device=dev) if want_act else None
    a_s, a_z = (None, None) if act is None else act
    rp, ldr = _res(residual, M, w.N, torch.float16)
    if fn_name == "mq_qlinear_w8a8":
        rc = L.mq_qlinear_w8a8(_ptr(x), M, K, x.stride(0), _ptr(w.packed), w.N, w.layout, int(w.signed), _ptr(w.scale),
                               _ptr(w.zp), _ptr(w.colsum), _ptr(a_s), _ptr(a_z), _ptr(bias), _ptr(y), y.stride(0),
                               _ptr(acc), rp, ldr, _ptr(s_out), _ptr(z_out), _ptr(ws), C.c_size_t(ws.numel()),
                               _stream())
    else:
        fn = L.mq_qlinear_w4a8 if fn_name == "mq_qlinear_w4a8" else L.mq_qlinear_w2a8
        rc = fn(_ptr(x), M, K, x.stride(0), _ptr(w.packed), w.N, w.layout, _ptr(w.scale), _ptr(w.zp),
                               _ptr(w.colsum), _ptr(a_s), _ptr(a_z), _ptr(bias), _ptr(y), y.stride(0), _ptr(acc),
                               rp, ldr, _ptr(s_out), _ptr(z_out), _ptr(ws), C.c_size_t(ws.numel()), _stream())
    _check(rc, fn_name)
    return y, acc, (s_out, z_out)


def qlinear_w8a8(x, w: PackedWeight, act=None, bias=None, out=None, ws=None, want_acc=False, want_act=False,
                 residual=None):
    """act=None: dynamic per-tensor min-max on the device; else (scale tensor[1] f32, zp tensor[1] i32).
    Returns (y, acc or None, (act_scale, act_zp) device scalars or (None, None))."""
    assert w.bits == 8
    return _qlinear_a8("mq_qlinear_w8a8", x, w, act, bias, out, ws, want_acc, want_act, residual)


def qlinear_w4a8(x, w: PackedWeight, act=None, bias=None, out=None, ws=None, want_acc=False, want_act=False,
                 residual=None):
    assert w.bits == 4 and not w.signed
    return _qlinear_a8("mq_qlinear_w4a8", x, w, act, bias, out, ws, want_acc, want_act, residual)


def qlinear_w2a8(x, w: PackedWeight, act=None, bias=None, out=None, ws=None, want_acc=False, want_act=False,
                 residual=None):
    assert w.bits == 2 and not w.signed
    return _qlinear_a8("mq_qlinear_w2a8", x, w, act, bias, out, ws, want_acc, want_act, residual)


def builtin_workspace_bytes() -> int:
    return int(load().mq_builtin_workspace_bytes())


def qlinear_a8_builtin_ws(x, w: PackedWeight, act=None, bias=None, out=None, want_acc=False, want_act=False,
                          residual=None, y=None):
    """W8A8 / W4A8 / W2A8 (by the weight's bit-width) with the workspace inside the library: the C call allocates
    nothing.  Pass out= (and want_acc / want_act False) for a call that allocates nothing on the Python side either.
    Returns (y, acc or None, (act_scale, act_zp) or (None, None))."""
    assert x.is_cuda and x.dim() == 2 and x.stride(1) == 1 and x.dtype == torch.float16
    M, K = x.shape
    assert K == w.K
    dev = x.device
    y = out if out is not None else torch.empty((M, w.N), dtype=torch.float16, device=dev)
    acc = torch.empty((M, w.N), dtype=torch.int32, device=dev) if want_acc else None
    s_out = torch.empty(1, dtype=torch.float32, device=dev) if want_act else None
    z_out = torch.empty(1, dtype=torch.int32, device=dev) if want_act else None
    a_s, a_z = (None, None) if act is None else act
    rp, ldr = _res(residual, M, w.N, torch.float16)
    _check(load().mq_qlinear_a8_builtin_ws(_ptr(x), M, K, x.stride(0), _ptr(w.packed), w.N, w.bits, w.layout,
                                           int(w.signed), _ptr(w.scale), _ptr(w.zp), _ptr(w.colsum), _ptr(a_s), _ptr(a_z),
                                           _ptr(bias), _ptr(y), y.stride(0), _ptr(acc), rp, ldr, _ptr(s_out), _ptr(z_out),
                                           _stream()), "mq_qlinear_a8_builtin_ws")
    return y, acc, (s_out, z_out)


def a8_row_bytes(K: int) -> int:
    return int(load().mq_a8_row_bytes(K))


def qlinear_a8_geglu(x, w: PackedWeight, out_act, act=None, bias=None, ws=None, want_h16=False, want_act=False):
    """Gated projection with 8-bit output.  w has 2H rows; out_act = (scale, zp) one-element device tensors.
    Returns (a8 int8 [M, a8_row_bytes(H)], h16 fp16 [M,H] or None, (act_scale, act_zp) or None)."""
    assert x.is_cuda and x.dim() == 2 and x.stride(1) == 1 and x.dtype == torch.float16
    M, K = x.shape
    H = w.N // 2
    a8 = torch.empty((M, a8_row_bytes(H)), dtype=torch.int8, device=x.device)
    h16 = torch.empty((M, H), dtype=torch.float16, device=x.device) if want_h16 else None
    ws = _workspace(qlinear_a8_workspace_bytes(M, K), x.device, ws)
    a_s, a_z = (None, None) if act is None else act
    so = torch.empty(1, dtype=torch.float32, device=x.device) if want_act else None
    zo = torch.empty(1, dtype=torch.int32, device=x.device) if want_act else None
    _check(load().mq_qlinear_a8_geglu(_ptr(x), M, K, x.stride(0), _ptr(w.packed), H, w.bits, w.layout, int(w.signed),
                                      _ptr(w.scale), _ptr(w.zp), _ptr(w.colsum), _ptr(a_s), _ptr(a_z), _ptr(bias),
                                      _ptr(out_act[0]), _ptr(out_act[1]), _ptr(a8), _ptr(h16), H, _ptr(so), _ptr(zo),
                                      _ptr(ws), C.c_size_t(ws.numel()), _stream()), "mq_qlinear_a8_geglu")
    return a8, h16, ((so, zo) if want_act else None)


def qlinear_a8_geglu_dynamic_workspace_bytes(M: int, K: int, H: int) -> int:
    return int(load().mq_qlinear_a8_geglu_dynamic_workspace_bytes(int(M), int(K), int(H)))


def qlinear_a8_geglu_dynamic(x, w: PackedWeight, act=None, bias=None, ws=None, want_act=False):
    """Gated projection with 8-bit output whose parameters are taken from the range of the gated product itself.
    w has 2H rows.  Returns (a8 int8 [M, a8_row_bytes(H)], h16 fp16 [M,H], (out_scale, out_zp) one-element device
    tensors, (act_scale, act_zp) of the input or None)."""
    assert x.is_cuda and x.dim() == 2 and x.stride(1) == 1 and x.dtype == torch.float16
    M, K = x.shape
    H = w.N // 2
    a8 = torch.empty((M, a8_row_bytes(H)), dtype=torch.int8, device=x.device)
    h16 = torch.empty((M, H), dtype=torch.float16, device=x.device)
    ws = _workspace(qlinear_a8_geglu_dynamic_workspace_bytes(M, K, H), x.device, ws)
    a_s, a_z = (None, None) if act is None else act
    o_s = torch.empty(1, dtype=torch.float32, device=x.device)
    o_z = torch.empty(1, dtype=torch.int32, device=x.device)
    so = torch.empty(1, dtype=torch.float32, device=x.device) if want_act else None
    zo = torch.empty(1, dtype=torch.int32, device=x.device) if want_act else None
    _check(load().mq_qlinear_a8_geglu_dynamic(_ptr(x), M, K, x.stride(0), _ptr(w.packed), H, w.bits, w.layout,
                                              int(w.signed), _ptr(w.scale), _ptr(w.zp), _ptr(w.colsum), _ptr(a_s),
                                              _ptr(a_z), _ptr(bias), _ptr(h16), H, _ptr(a8), _ptr(o_s), _ptr(o_z),
                                              _ptr(so), _ptr(zo), _ptr(ws), C.c_size_t(ws.numel()), _stream()),
           "mq_qlinear_a8_geglu_dynamic")
    return a8, h16, (o_s, o_z), ((so, zo) if want_act else None)


def qlinear_w_only_geglu(x, w: PackedWeight, bias=None, out=None):
    """Weight-only gated projection: w has 2H rows; returns value * gelu(gate) as fp16 [M,H]."""
    assert x.is_cuda and x.dim() == 2 and x.stride(1) == 1 and x.dtype == torch.float16
    M, K = x.shape
    H = w.N // 2
    h = out if out is not None else torch.empty((M, H), dtype=torch.float16, device=x.device)
    _check(load().mq_qlinear_w_only_geglu(_ptr(x), M, K, x.stride(0), _ptr(w.packed), H, w.bits, w.layout, _ptr(w.scale),
                                          _ptr(w.zp), _ptr(bias), _ptr(h), h.stride(0), _stream()),
           "mq_qlinear_w_only_geglu")
    return h


def qlinear_w_only_geglu_a8(x, w: PackedWeight, out_act, bias=None, want_h16=False):
    """Weight-only gated projection with 8-bit output; out_act = (scale, zp) one-element device tensors.
    Returns (a8 int8 [M, a8_row_bytes(H)], h16 fp16 [M,H] or None)."""
    assert x.is_cuda and x.dim() == 2 and x.stride(1) == 1 and x.dtype == torch.float16
    M, K = x.shape
    H = w.N // 2
    a8 = torch.empty((M, a8_row_bytes(H)), dtype=torch.int8, device=x.device)
    h16 = torch.empty((M, H), dtype=torch.float16, device=x.device) if want_h16 else None
    _check(load().mq_qlinear_w_only_geglu_a8(_ptr(x), M, K, x.stride(0), _ptr(w.packed), H, w.bits, w.layout,
                                             _ptr(w.scale), _ptr(w.zp), _ptr(bias), _ptr(out_act[0]), _ptr(out_act[1]),
                                             _ptr(a8), _ptr(h16), H, _stream()), "mq_qlinear_w_only_geglu_a8")
    return a8, h16


def qlinear_a8_codes(a8, K: int, act, w: PackedWeight, bias=None, out=None, want_acc=False, residual=None):
    """A8 linear on activations in the A8 layout (a8 int8 [M, stride]); act = (scale, zp) one-element device tensors."""
    assert a8.is_cuda and a8.dim() == 2 and a8.stride(1) == 1 and a8.dtype == torch.int8 and K == w.K
    M = a8.shape[0]
    y = out if out is not None else torch.empty((M, w.N), dtype=torch.float16, device=a8.device)
    acc = torch.empty((M, w.N), dtype=torch.int32, device=a8.device) if want_acc else None
    rp, ldr = _res(residual, M, w.N, torch.float16)
    _check(load().mq_qlinear_a8_codes(_ptr(a8), M, K, a8.stride(0), _ptr(act[0]), _ptr(act[1]), _ptr(w.packed), w.N,
                                      w.bits, w.layout, int(w.signed), _ptr(w.scale), _ptr(w.zp), _ptr(w.colsum),
                                      _ptr(bias), _ptr(y), y.stride(0), _ptr(acc), rp, ldr, _stream()),
           "mq_qlinear_a8_codes")
    return y, acc


def plan_qlinear_a8_geglu(x, w: PackedWeight, out_act, bias, a8_out, ws, act=None):
    M, K = x.shape
    H = w.N // 2
    a_s, a_z = (None, None) if act is None else act
    null = C.c_void_p(0)
    args = (_ptr(x), M, K, x.stride(0), _ptr(w.packed), H, w.bits, w.layout, int(w.signed), _ptr(w.scale), _ptr(w.zp),
            _ptr(w.colsum), _ptr(a_s), _ptr(a_z), _ptr(bias), _ptr(out_act[0]), _ptr(out_act[1]), _ptr(a8_out), null, H,
            null, null, _ptr(ws), C.c_size_t(ws.numel()), _stream())
    return _planned(load().mq_qlinear_a8_geglu, "mq_qlinear_a8_geglu", args, (x, w, out_act, bias, a8_out, ws, act))


def plan_qlinear_a8_geglu_dynamic(x, w: PackedWeight, bias, h16, a8_out, out_act, ws, act=None):
    """out_act = (scale, zp) one-element device tensors that RECEIVE the parameters of the gated product."""
    M, K = x.shape
    H = w.N // 2
    a_s, a_z = (None, None) if act is None else act
    null = C.c_void_p(0)
    args = (_ptr(x), M, K, x.stride(0), _ptr(w.packed), H, w.bits, w.layout, int(w.signed), _ptr(w.scale), _ptr(w.zp),
            _ptr(w.colsum), _ptr(a_s), _ptr(a_z), _ptr(bias), _ptr(h16), h16.stride(0), _ptr(a8_out), _ptr(out_act[0]),
            _ptr(out_act[1]), null, null, _ptr(ws), C.c_size_t(ws.numel()), _stream())
    return _planned(load().mq_qlinear_a8_geglu_dynamic, "mq_qlinear_a8_geglu_dynamic", args,
                    (x, w, bias, h16, a8_out, out_act, ws, act))


def plan_qlinear_a8_codes(a8, K, act, w: PackedWeight, bias, out, residual=None):
    M = a8.shape[0]
    null = C.c_void_p(0)
    rp, ldr = _res(residual, M, w.N, torch.float16)
    args = (_ptr(a8), M, K, a8.stride(0), _ptr(act[0]), _ptr(act[1]), _ptr(w.packed), w.N, w.bits, w.layout,
            int(w.signed), _ptr(w.scale), _ptr(w.zp), _ptr(w.colsum), _ptr(bias), _ptr(out), out.stride(0), null,
            rp, ldr, _stream())
    return _planned(load().mq_qlinear_a8_codes, "mq_qlinear_a8_codes", args, (a8, act, w, bias, out, residual))


def conv_tap_sums(codes: torch.Tensor, Cin: int, bits: int, codes_signed: bool = False) -> torch.Tensor:
    """codes uint8 [N, 9*Cin] -> int32 [9, N]."""
    N = codes.shape[0]
    assert codes.is_cuda and codes.dtype == torch.uint8 and codes.is_contiguous() and codes.shape[1] == 9 * Cin
    out = torch.empty((9, N), dtype=torch.int32, device=codes.device)
    _check(load().mq_conv_tap_sums(_ptr(codes), N, Cin, bits, int(codes_signed), _ptr(out), _stream()), "mq_conv_tap_sums")
    return out


def _res4(residual, shape):
    if residual is None:
        return C.c_void_p(0)
    assert residual.is_cuda and tuple(residual.shape) == tuple(shape) and residual.is_contiguous()
    assert residual.dtype == torch.float16
    return _ptr(residual)


def _conv_out_hw(H: int, W: int, stride: int):
    assert stride in (1, 2)
    return (H - 1) // stride + 1, (W - 1) // stride + 1


def conv3x3_w_only(x: torch.Tensor, w: PackedWeight, bias=None, out=None, residual=None, stride: int = 1) -> torch.Tensor:
    """x [B,H,W,Cin] fp16 channels-last contiguous; w packed from the [N, 9*Cin] matrix.  Returns y [B,Ho,Wo,N]
    (+ residual of that shape, added before the rounding); stride 1 or 2."""
    assert x.is_cuda and x.dim() == 4 and x.is_contiguous() and x.dtype == torch.float16
    B, H, W, Cin = x.shape
    assert w.K == 9 * Cin
    Ho, Wo = _conv_out_hw(H, W, stride)
    y = out if out is not None else torch.empty((B, Ho, Wo, w.N), dtype=torch.float16, device=x.device)
    assert tuple(y.shape) == (B, Ho, Wo, w.N) and y.is_contiguous()
    _check(load().mq_conv3x3_w_only(_ptr(x), B, H, W, Cin, stride, _ptr(w.packed), w.N, w.bits, w.layout, _ptr(w.scale),
                                    _ptr(w.zp), _ptr(bias), _ptr(y), _res4(residual, y.shape), _stream()),
           "mq_conv3x3_w_only")
    return y


def conv3x3_a8_workspace_bytes(B: int, H: int, W: int, Cin: int) -> int:
    return int(load().mq_conv3x3_a8_workspace_bytes(B, H, W, Cin))


def conv3x3_a8(x, w: PackedWeight, tapsum, act=None, bias=None, out=None, ws=None, want_acc=False, want_act=False,
               residual=None, stride: int = 1):
    """Returns (y [B,Ho,Wo,N], acc int32 [B*Ho*Wo,N] or None, (act_scale, act_zp) or None)."""
    assert x.is_cuda and x.dim() == 4 and x.is_contiguous() and x.dtype == torch.float16
    B, H, W, Cin = x.shape
    assert w.K == 9 * Cin
    Ho, Wo = _conv_out_hw(H, W, stride)
    y = out if out is not None else torch.empty((B, Ho, Wo, w.N), dtype=torch.float16, device=x.device)
    assert tuple(y.shape) == (B, Ho, Wo, w.N) and y.is_contiguous()
    acc = torch.empty((B * Ho * Wo, w.N), dtype=torch.int32, device=x.device) if want_acc else None
    ws = _workspace(conv3x3_a8_workspace_bytes(B, H, W, Cin), x.device, ws)
    a_s, a_z = (None, None) if act is None else act
    so = torch.empty(1, dtype=torch.float32, device=x.device) if want_act else None
    zo = torch.empty(1, dtype=torch.int32, device=x.device) if want_act else None
    _check(load().mq_conv3x3_a8(_ptr(x), B, H, W, Cin, stride, _ptr(w.packed), w.N, w.bits, w.layout, int(w.signed),
                                _ptr(w.scale), _ptr(w.zp), _ptr(w.colsum), _ptr(tapsum), _ptr(a_s), _ptr(a_z), _ptr(bias),
                                _ptr(y), _ptr(acc), _res4(residual, y.shape), _ptr(so), _ptr(zo), _ptr(ws),
                                C.c_size_t(ws.numel()), _stream()), "mq_conv3x3_a8")
    return y, acc, ((so, zo) if want_act else None)


def bos_aware_kv_proj_workspace_bytes(B: int, T: int, K: int) -> int:
    return int(load().mq_bos_aware_kv_proj_workspace_bytes(B, T, K))


def bos_aware_kv_proj(ctx: torch.Tensor, w: PackedWeight, w_f16: Optional[torch.Tensor] = None,
                      bos_out: Optional[torch.Tensor] = None, act=None, bias=None, naive_all_rows: bool = False,
                      out=None, ws=None, want_act=False):
    """ctx [B,T,K] fp16 -> y [B,T,N] fp16; token 0 of each prompt bypasses activation quantisation."""
    assert ctx.is_cuda and ctx.dim() == 3 and ctx.is_contiguous() and ctx.dtype == torch.float16
    B, T, K = ctx.shape
    assert K == w.K
    dev = ctx.device
    y = out if out is not None else torch.empty((B, T, w.N), dtype=torch.float16, device=dev)
    ws = _workspace(bos_aware_kv_proj_workspace_bytes(B, T, K) + split_workspace_bytes(B * T, w.N, K), dev, ws)
    s_out = torch.empty(1, dtype=torch.float32, device=dev) if want_act else None
    z_out = torch.empty(1, dtype=torch.int32, device=dev) if want_act else None
    a_s, a_z = (None, None) if act is None else act
    rc = load().mq_bos_aware_kv_proj(_ptr(ctx), B, T, K, _ptr(w.packed), w.N, w.bits, w.layout, int(w.signed),
                                     _ptr(w.scale), _ptr(w.zp), _ptr(w.colsum), _ptr(w_f16), _ptr(bos_out), _ptr(a_s),
                                     _ptr(a_z), _ptr(bias), _ptr(y), int(naive_all_rows), _ptr(s_out), _ptr(z_out),
                                     _ptr(ws), C.c_size_t(ws.numel()), _stream())
    _check(rc, "mq_bos_aware_kv_proj")
    return y, (s_out, z_out)


# ---------------------------------------------------------------------------------------------------------------
# Pre-marshalled calls.  A serving loop runs the same layer on the same buffers over and over; marshalling two
# dozen arguments in Python each time costs more than some of the kernels.  plan_*() does the marshalling once and
# returns a zero-argument callable that only performs the C call (on the stream that was current at plan time).
# ---------------------------------------------------------------------------------------------------------------

def _planned(fn, what, args, keep):
    def call():
        rc = fn(*args)
        if rc != 0:
            raise MixdqError(rc, what)
    call.keepalive = keep  # the tensors must outlive the plan
    return call


def plan_qlinear_w_only(x, w: PackedWeight, bias, out, residual=None, ws=None):
    """ws: optional workspace (see qlinear_w_only); without one the call never splits its reduction."""
    assert x.is_cuda and x.dim() == 2 and x.stride(1) == 1 and out.shape == (x.shape[0], w.N)
    M, K = x.shape
    rp, ldr = _res(residual, M, w.N, x.dtype)
    args = (_ptr(x), M, K, x.stride(0), _ptr(w.packed), w.N, w.bits, w.layout, _ptr(w.scale), _ptr(w.zp), _ptr(bias),
            _ptr(out), out.stride(0), _dtype_code(x), rp, ldr, *_ws_args(ws), _stream())
    return _planned(load().mq_qlinear_w_only, "mq_qlinear_w_only", args, (x, w, bias, out, residual, ws))


def plan_qlinear_a8(x, w: PackedWeight, bias, out, ws, act=None, residual=None):
    """W8A8 or W4A8 by the weight's bit-width; dynamic activation parameters unless act=(scale, zp) tensors."""
    assert x.is_cuda and x.dim() == 2 and x.stride(1) == 1 and x.dtype == torch.float16
    M, K = x.shape
    a_s, a_z = (None, None) if act is None else act
    null = C.c_void_p(0)
    rp, ldr = _res(residual, M, w.N, torch.float16)
    if w.bits == 8:
        fn, what = load().mq_qlinear_w8a8, "mq_qlinear_w8a8"
        args = (_ptr(x), M, K, x.stride(0), _ptr(w.packed), w.N, w.layout, int(w.signed), _ptr(w.scale), _ptr(w.zp),
                _ptr(w.colsum), _ptr(a_s), _ptr(a_z), _ptr(bias), _ptr(out), out.stride(0), null, rp, ldr, null, null,
                _ptr(ws), C.c_size_t(ws.numel()), _stream())
    else:
        fn, what = (load().mq_qlinear_w4a8, "mq_qlinear_w4a8") if w.bits == 4 else (load().mq_qlinear_w2a8, "mq_qlinear_w2a8")
        args = (_ptr(x), M, K, x.stride(0), _ptr(w.packed), w.N, w.layout, _ptr(w.scale), _ptr(w.zp), _ptr(w.colsum),
                _ptr(a_s), _ptr(a_z), _ptr(bias), _ptr(out), out.stride(0), null, rp, ldr, null, null, _ptr(ws),
                C.c_size_t(ws.numel()), _stream())
    return _planned(fn, what, args, (x, w, bias, out, ws, act, residual))


def plan_bos_aware_kv_proj(ctx, w: PackedWeight, out, ws, w_f16=None, bos_out=None, bias=None, act=None):
    assert ctx.is_cuda and ctx.dim() == 3 and ctx.is_contiguous() and ctx.dtype == torch.float16
    B, T, K = ctx.shape
    a_s, a_z = (None, None) if act is None else act
    null = C.c_void_p(0)
    args = (_ptr(ctx), B, T, K, _ptr(w.packed), w.N, w.bits, w.layout, int(w.signed), _ptr(w.scale), _ptr(w.zp),
            _ptr(w.colsum), _ptr(w_f16), _ptr(bos_out), _ptr(a_s), _ptr(a_z), _ptr(bias), _ptr(out), 0, null, null,
            _ptr(ws), C.c_size_t(ws.numel()), _stream())
    return _planned(load().mq_bos_aware_kv_proj, "mq_bos_aware_kv_proj", args, (ctx, w, out, ws, w_f16, bos_out, bias, act))


# ---------------------------------------------------------------------------------------------------------------
# Bit-width allocation (host arrays, no GPU)
# ---------------------------------------------------------------------------------------------------------------

def _np_ptr(a):
    return a.ctypes.data_as(C.c_void_p)


def alloc_solve(sens, cost, budget: int):
    """Eq. 2 solved exactly.  sens float64 [n_layers, n_choices], cost int64 [n_layers, n_choices].
    Returns (choice int32 [n_layers], objective, cost used); raises MixdqError (code -8) when nothing fits."""
    import numpy as np
    sens = np.ascontiguousarray(sens, np.float64)
    cost = np.ascontiguousarray(cost, np.int64)
    assert sens.ndim == 2 and sens.shape == cost.shape
    n, m = sens.shape
    choice = np.empty(n, np.int32)
    obj = C.c_double(0.0)
    used = C.c_int64(0)
    _check(load().mq_alloc_solve(n, m, _np_ptr(sens), _np_ptr(cost), C.c_int64(int(budget)), _np_ptr(choice),
                                 C.byref(obj), C.byref(used)), "mq_alloc_solve")
    return choice, obj.value, used.value


def alloc_split_budget(budget_all: int, params_content: int, params_quality: int, k: float):
    bc, bq = C.c_int64(0), C.c_int64(0)
    _check(load().mq_alloc_split_budget(C.c_int64(int(budget_all)), C.c_int64(int(params_content)),
                                        C.c_int64(int(params_quality)), C.c_double(k), C.byref(bc), C.byref(bq)),
           "mq_alloc_split_budget")
    return bc.value, bq.value


def alloc_search(sens_content, params_content, sens_quality, params_quality, bits, avg_bits_target: float,
                 delta_avg_bits: float, n_budgets: int, k_lo: float, k_hi: float, n_ratios: int):
    """The budget x ratio scan around Eq. 2.  Returns a dict of arrays over the n_budgets * n_ratios candidates:
    budgets int64 [E,3] (all, content, quality), k [E], feasible [E], objectives [E,2], choice_content [E,n_c],
    choice_quality [E,n_q]."""
    import numpy as np
    sc = np.ascontiguousarray(sens_content, np.float64)
    sq = np.ascontiguousarray(sens_quality, np.float64)
    pc = np.ascontiguousarray(params_content, np.int64)
    pq = np.ascontiguousarray(params_quality, np.int64)
    bits = np.ascontiguousarray(bits, np.int32)
    nc, nq, m = sc.shape[0], sq.shape[0], bits.shape[0]
    assert sc.shape == (nc, m) and sq.shape == (nq, m) and pc.shape == (nc,) and pq.shape == (nq,)
    E = n_budgets * n_ratios
    out = dict(budgets=np.empty((E, 3), np.int64), k=np.empty(E, np.float64), feasible=np.empty(E, np.int32),
               objectives=np.empty((E, 2), np.float64), choice_content=np.empty((E, nc), np.int32),
               choice_quality=np.empty((E, nq), np.int32))
    _check(load().mq_alloc_search(nc, _np_ptr(sc), _np_ptr(pc), nq, _np_ptr(sq), _np_ptr(pq), m, _np_ptr(bits),
                                  C.c_double(avg_bits_target), C.c_double(delta_avg_bits), n_budgets, C.c_double(k_lo),
                                  C.c_double(k_hi), n_ratios, _np_ptr(out["budgets"]), _np_ptr(out["k"]),
                                  _np_ptr(out["feasible"]), _np_ptr(out["objectives"]), _np_ptr(out["choice_content"]),
                                  _np_ptr(out["choice_quality"])), "mq_alloc_search")
    return out


# ------------------------------------------- microscaled 4-bit floats, layer norm, and their gradients
#
# Matrices are [rows, columns] with contiguous rows, which may lie apart but not over one another (so a broadcast one is made contiguous() first).
# Results are no part of autograd's graph; gradients are calls of their own.


_HALF = (None, torch.float16)  # mx_linear's default


@dataclass
class MxTensor:
    """A [rows, K] matrix in microscaled 4-bit floats, in the product's form.  top: for weights whose layer is differentiated.  experts: of as many
    experts' weights, one's rows behind another's."""
    data: torch.Tensor                  # uint8, mx_bytes(rows, K)
    rows: int
    K: int
    top: Optional[torch.Tensor] = None  # uint8 [K / 32], the largest scale of every column of blocks (of each expert)
    experts: int = 1

    @property
    def shape(self):
        return (self.rows, self.K)


def _sizes(*n: int) -> None:
    """The entry points take 32-bit sizes; larger ones would reach them cut off."""
    if max(n) > 0x7FFFFFFF:
        raise ValueError(f"sizes are below 2^31, got {n}")


def _matrix(t: torch.Tensor, rows=None, cols=None, dtype=None, device=None) -> torch.Tensor:
    _sizes(*t.shape, 0)
    if t.dim() == 2 and t.shape[0] > 1 and t.stride(0) < t.shape[1]:
        raise ValueError(f"rows overlap: {tuple(t.shape)} with strides {t.stride()}; contiguous() makes a matrix of it")
    if not t.is_cuda or t.dim() != 2 or (t.shape[1] > 1 and t.stride(1) != 1):
        raise ValueError(f"expected a matrix on the GPU with contiguous rows, got {tuple(t.shape)} with strides {t.stride()} on {t.device}")
    if (rows is not None and t.shape[0] != rows) or (cols is not None and t.shape[1] != cols):
        raise ValueError(f"expected [{rows}, {cols}], got {tuple(t.shape)}")
    if device is not None and t.device != device:
        raise ValueError(f"expected a matrix on {device}, got one on {t.device}")
    if dtype is not None and t.dtype != dtype:
        raise TypeError(f"expected {dtype}, got {t.dtype}")
    return t


def _no_graph(what: str, *ts) -> None:
    """Results carry no graph: what autograd would have to go through is refused rather than cut off from it."""
    if torch.is_grad_enabled() and any(t is not None and t.requires_grad for t in ts):
        raise RuntimeError(f"{what} is no part of autograd's graph: call it under torch.no_grad(), or in the forward of a torch.autograd.Function, and "
                           "the calls named ..._grad for the gradients")


def _out(t: Optional[torch.Tensor], rows: int, cols: int, dtype, device) -> torch.Tensor:
    return torch.empty((rows, cols), dtype=dtype, device=device) if t is None else _matrix(t, rows, cols, dtype, device)


def _ld(t: Optional[torch.Tensor]):
    """Row stride; a single row's stride says nothing."""
    return C.c_long(0 if t is None else t.stride(0) if t.shape[0] > 1 else t.shape[1])


def _vector(t: Optional[torch.Tensor], n: int, dtype, device) -> Optional[torch.Tensor]:
    if t is None:
        return None
    if t.device != device or t.dim() != 1 or t.shape[0] != n or not t.is_contiguous():
        raise ValueError(f"expected a contiguous vector of {n} on {device}, got {tuple(t.shape)} on {t.device}")
    if dtype is not None and t.dtype != dtype:
        raise TypeError(f"expected {dtype}, got {t.dtype}")
    return t


def _mx_data(t: MxTensor, device=None):
    """Address of a microscaled matrix, which may have been made or moved by hand."""
    _sizes(t.rows, t.K)
    d, need = t.data, mx_bytes(t.rows, t.K)
    if d.dtype != torch.uint8 or not d.is_contiguous() or d.numel() < need:
        raise ValueError(f"a microscaled matrix of {t.rows} x {t.K} has {need} contiguous bytes, got {d.numel()} of {d.dtype} with strides {d.stride()}")
    if not d.is_cuda or (device is not None and d.device != device):
        raise ValueError(f"expected a microscaled matrix on {device or 'the GPU'}, got one on {d.device}")
    return _ptr(d)


def _mx_workspace(nbytes: int, device, ws: Optional[torch.Tensor]) -> torch.Tensor:
    if ws is not None and (ws.device != device or not ws.is_contiguous()):
        raise ValueError(f"expected a contiguous workspace on {device}, got one on {ws.device} with strides {ws.stride()}")
    return _workspace(nbytes, device, ws)


def _bytes_of(ws: torch.Tensor):
    return C.c_size_t(ws.numel() * ws.element_size())


def mx_bytes(rows: int, K: int) -> int:
    return int(load().mq_mx_bytes(rows, K))


def _new_mx(rows: int, K: int, device) -> MxTensor:
    _sizes(rows, K)
    n = mx_bytes(rows, K)
    if K <= 0 or K % 32:
        raise ValueError(f"microscaled matrices have a multiple of 32 columns, got {K}")
    return MxTensor(torch.empty(n, dtype=torch.uint8, device=device), rows, K)


def mx_quantize(x: torch.Tensor) -> MxTensor:
    """[M, K] fp16/bf16 -> MXFP4: blocks of 32 values of a row, e2m1 codes (nearest, ties to even) times a power of two."""
    r = (_native or _load_native()).mx_quantize(x)
    if r is not None:
        return MxTensor(_done(r, "mq_mx_quantize"), x.shape[0], x.shape[1])
    M, K = _matrix(x).shape
    dt = _dtype_code(x)
    t = _new_mx(M, K, x.device)
    _check(load().mq_mx_quantize(_ptr(x), M, K, _ld(x), dt, _ptr(t.data), _stream()), "mq_mx_quantize")
    return t


def mx_quantize_weights(w: torch.Tensor) -> MxTensor:
    """mx_quantize of a weight matrix [N, K], with what mx_linear_grad needs beside it."""
    return _with_top(mx_quantize(w))


def _with_top(t: MxTensor) -> MxTensor:
    data = _mx_data(t)
    t.top = torch.empty(t.K // 32, dtype=torch.uint8, device=t.data.device)
    _check(load().mq_mx_column_top(data, t.rows, t.K, _ptr(t.top), _stream()), "mq_mx_column_top")
    return t


def mx_dequantize(t: MxTensor, dtype=torch.bfloat16, out: Optional[torch.Tensor] = None) -> torch.Tensor:
    """The values that `t` stands for, rounded to dtype (bfloat16 holds every one)."""
    if out is None:
        r = (_native or _load_native()).mx_dequantize(t.data, t.rows, t.K, 0 if dtype == torch.float16 else 1 if dtype == torch.bfloat16 else -1)
        if r is not None:
            return _done(r, "mq_mx_dequantize")
    _sizes(t.rows, t.K)
    y = _out(out, t.rows, t.K, dtype, t.data.device)
    _check(load().mq_mx_dequantize(_mx_data(t), t.rows, t.K, _dtype_code(y), _ptr(y), _ld(y), _stream()), "mq_mx_dequantize")
    return y


def mx_pack(codes: torch.Tensor, scales: torch.Tensor) -> MxTensor:
    """Interchange form (codes uint8 [M, K/2], value 2i in the low half of byte i; scales uint8 [M, K/32]) -> MxTensor, ready for a weight."""
    if codes.dtype != torch.uint8 or scales.dtype != torch.uint8:
        raise TypeError("codes and scales are uint8")
    M, K = codes.shape[0], codes.shape[1] * 2
    t = _new_mx(M, K, codes.device)
    if not codes.is_cuda or not codes.is_contiguous() or not scales.is_contiguous() or scales.device != codes.device or tuple(scales.shape) != (M, K // 32):
        raise ValueError(f"expected contiguous codes [M, K/2] and scales [M, K/32] on the GPU, got {tuple(codes.shape)} and {tuple(scales.shape)}")
    _check(load().mq_mx_pack(_ptr(codes), _ptr(scales), M, K, _ptr(t.data), _stream()), "mq_mx_pack")
    return _with_top(t)


def mx_unpack(t: MxTensor):
    """(codes uint8 [M, K/2], scales uint8 [M, K/32])."""
    data = _mx_data(t)
    codes = torch.empty((t.rows, t.K // 2), dtype=torch.uint8, device=t.data.device)
    scales = torch.empty((t.rows, t.K // 32), dtype=torch.uint8, device=t.data.device)
    _check(load().mq_mx_unpack(data, t.rows, t.K, _ptr(codes), _ptr(scales), _stream()), "mq_mx_unpack")
    return codes, scales


def mx_linear_workspace_bytes(M: int, N: int, K: int) -> int:
    return int(load().mq_mx_linear_workspace_bytes(M, N, K))


def mx_linear(x: Union[torch.Tensor, MxTensor], w: MxTensor, bias: Optional[torch.Tensor] = None, out: Optional[torch.Tensor] = None,
              residual: Optional[torch.Tensor] = None, ws: Optional[torch.Tensor] = None, dtype=None, act: Optional[str] = None, gated: bool = False,
              want_pre: bool = False):
    """Y = mx(X) . W^T + bias (+ residual).  X: [M, K] fp16/bf16, quantised in the call, or an MxTensor; then dtype (fp16 unless out or
    dtype says otherwise) is the output's.  residual may be out itself.  ws: optional uint8 workspace of mx_linear_workspace_bytes(M, N, K).
    act: "gelu", "gelu_tanh" or "silu", Y = act(mx(X) . W^T + bias) (+ residual).  gated: Y [M, N / 2] = v act(g), v and g the first and the second half of the
    columns, N % 64 == 0, no residual.  want_pre: (Y, mx(X) . W^T + bias [M, N]), the latter for act_grad."""
    if act is not None or gated or want_pre:
        return _mx_linear_act(x, w, bias, out, residual, ws, dtype, act, gated, want_pre)
    packed = isinstance(x, MxTensor)
    if out is None and ws is None:
        native = _native or _load_native()
        if packed:
            if x.K == w.K:
                r = native.mx_linear_codes(x.data, x.rows, x.K, w.data, w.rows, bias, residual, 1 if dtype == torch.bfloat16 else 0 if dtype in _HALF else -1)
                if r is not None:
                    return _done(r, "mq_mx_linear_codes")
        elif dtype is None and w is not None:
            r = native.mx_linear(x, w.data, w.rows, w.K, bias, residual)
            if r is not None:
                return _done(r, "mq_mx_linear")
    lib = load()
    _no_graph("mx_linear", None if packed else x, bias, residual)
    if packed:
        M, K, device = x.rows, x.K, x.data.device
        dtype = dtype or (out.dtype if out is not None else torch.float16)
    else:
        (M, K), device = _matrix(x).shape, x.device
        if dtype is not None and dtype != x.dtype:
            raise TypeError(f"the output has the type of the activations, {x.dtype}")
        dtype = x.dtype
    if K != w.K:
        raise ValueError(f"activations have {K} columns, weights {w.K}")
    y = _out(out, M, w.rows, dtype, device)
    dt = _dtype_code(y)
    if residual is not None:
        _matrix(residual, M, w.rows, dtype, device)
    args = (_mx_data(w, device), w.rows, _ptr(_vector(bias, w.rows, dtype, device)), _ptr(y), _ld(y), dt, _ptr(residual), _ld(residual))
    if packed:
        _check(lib.mq_mx_linear_codes(_mx_data(x, device), M, K, *args, _stream()), "mq_mx_linear_codes")
    else:
        # (a few rows do without, unless the output lies over them)
        ws = _mx_workspace(mx_linear_workspace_bytes(M, w.rows, K) or (0 if out is None else mx_bytes(M, K)), device, ws)
        _check(lib.mq_mx_linear(_ptr(x), M, K, _ld(x), *args, _ptr(ws), _bytes_of(ws), _stream()), "mq_mx_linear")
    return y


def mx_linear_grad_workspace_bytes(M: int, N: int, K: int) -> int:
    return int(load().mq_mx_linear_grad_workspace_bytes(M, N, K))


def mx_linear_grad(dy: torch.Tensor, w: MxTensor, out: Optional[torch.Tensor] = None, ws: Optional[torch.Tensor] = None) -> torch.Tensor:
    """dX = dY . W, the gradient of mx_linear with respect to its input (the quantisation of X passed straight through).  ws: optional uint8
    workspace of mx_linear_grad_workspace_bytes(M, N, K).  out shares nothing with dy."""
    if w.top is None:
        raise ValueError("weights without `top`: make them with mx_quantize_weights or mx_pack")
    if out is None and ws is None:
        r = (_native or _load_native()).mx_linear_grad(dy, w.data, w.rows, w.K, w.top)
        if r is not None:
            return _done(r, "mq_mx_linear_grad")
    _no_graph("mx_linear_grad", dy)
    M, N = _matrix(dy, cols=w.rows).shape
    dx = _out(out, M, w.K, dy.dtype, dy.device)
    ws = _mx_workspace(mx_linear_grad_workspace_bytes(M, N, w.K), dy.device, ws)
    top = _vector(w.top, w.K // 32, torch.uint8, dy.device)
    _check(load().mq_mx_linear_grad(_ptr(dy), M, N, _ld(dy), _mx_data(w, dy.device), _ptr(top), w.K, _ptr(dx), _ld(dx), _dtype_code(dy), *_ws_args(ws),
                                    _stream()), "mq_mx_linear_grad")
    return dx


def _params(x: torch.Tensor, weight: Optional[torch.Tensor], bias: Optional[torch.Tensor]):
    p = weight if weight is not None else bias
    if p is None:
        return None, None, F32
    for t in (weight, bias):
        _vector(t, x.shape[1], p.dtype, x.device)
    return weight, bias, F32 if p.dtype == torch.float32 else _dtype_code(p)


def _stats(x: torch.Tensor, want: bool):
    if not want:
        return None, None
    return torch.empty(x.shape[0], dtype=torch.float32, device=x.device), torch.empty(x.shape[0], dtype=torch.float32, device=x.device)


def layer_norm(x: torch.Tensor, weight: Optional[torch.Tensor] = None, bias: Optional[torch.Tensor] = None, eps: float = 1e-5,
               out: Optional[torch.Tensor] = None, want_stats: bool = False):
    """Layer norm over the columns of x [M, C] fp16/bf16; weight, bias [C] in 16 bits or float32.  want_stats: (y, mean, rstd), the latter
    two float32 [M], for layer_norm_grad.  out may be x."""
    if out is None:
        r = (_native or _load_native()).layer_norm(x, weight, bias, eps, want_stats, False)
        if r is not None:
            return _done(r, "mq_layer_norm")
    _no_graph("layer_norm", x, weight, bias)
    M, N = _matrix(x).shape
    w, b, pt = _params(x, weight, bias)
    mean, rstd = _stats(x, want_stats)
    y = _out(out, M, N, x.dtype, x.device)
    _check(load().mq_layer_norm(_ptr(x), M, N, _ld(x), _ptr(w), _ptr(b), pt, C.c_float(eps), _ptr(y), _ld(y), _dtype_code(x), _ptr(mean), _ptr(rstd),
                                _stream()), "mq_layer_norm")
    return (y, mean, rstd) if want_stats else y


def layer_norm_mx(x: torch.Tensor, weight: Optional[torch.Tensor] = None, bias: Optional[torch.Tensor] = None, eps: float = 1e-5,
                  want_stats: bool = False):
    """Layer norm whose output is quantised to MXFP4 from its float32 values: the input of the mx_linear behind it.  C % 32 == 0."""
    r = (_native or _load_native()).layer_norm(x, weight, bias, eps, want_stats, True)
    if r is not None:
        r = _done(r, "mq_layer_norm_mx")
        return (MxTensor(r[0], *x.shape), r[1], r[2]) if want_stats else MxTensor(r, *x.shape)
    _no_graph("layer_norm_mx", x, weight, bias)
    M, N = _matrix(x).shape
    w, b, pt = _params(x, weight, bias)
    mean, rstd = _stats(x, want_stats)
    t = _new_mx(M, N, x.device)
    _check(load().mq_layer_norm_mx(_ptr(x), M, N, _ld(x), _ptr(w), _ptr(b), pt, C.c_float(eps), _ptr(t.data), _dtype_code(x), _ptr(mean), _ptr(rstd),
                                   _stream()), "mq_layer_norm_mx")
    return (t, mean, rstd) if want_stats else t


def layer_norm_grad_workspace_bytes(M: int, N: int) -> int:
    return int(load().mq_layer_norm_grad_workspace_bytes(M, N))


def layer_norm_grad(dy: torch.Tensor, x: torch.Tensor, weight: Optional[torch.Tensor], mean: torch.Tensor, rstd: torch.Tensor,
                    residual: Optional[torch.Tensor] = None, out: Optional[torch.Tensor] = None, ws: Optional[torch.Tensor] = None):
    """(dx, dweight, dbias) of layer_norm and layer_norm_mx; dweight and dbias float32 [C].  residual [M, C]: a gradient that reaches x past the norm,
    added to dx.  out may be dy or residual."""
    if out is None and ws is None:
        r = (_native or _load_native()).layer_norm_grad(dy, x, weight, mean, rstd, residual)
        if r is not None:
            return _done(r, "mq_layer_norm_grad")
    _no_graph("layer_norm_grad", dy)
    M, N = _matrix(x).shape
    _matrix(dy, M, N, x.dtype, x.device)
    if residual is not None:
        _matrix(residual, M, N, x.dtype, x.device)
    w, _, pt = _params(x, weight, None)
    _vector(mean, M, torch.float32, x.device)
    _vector(rstd, M, torch.float32, x.device)
    dx = _out(out, M, N, x.dtype, x.device)
    sums = torch.empty((2, N), dtype=torch.float32, device=x.device)
    ws = _mx_workspace(layer_norm_grad_workspace_bytes(M, N), x.device, ws)
    _check(load().mq_layer_norm_grad(_ptr(dy), _ld(dy), _ptr(x), _ld(x), M, N, _ptr(w), pt, _ptr(mean), _ptr(rstd), _ptr(residual), _ld(residual),
                                     _ptr(dx), _ld(dx), _dtype_code(x), _ptr(sums[0]), _ptr(sums[1]), _ptr(ws), _bytes_of(ws), _stream()),
           "mq_layer_norm_grad")
    return dx, sums[0], sums[1]


# ------------------------------------------------------------- around the microscaled linears of a transformer block


def _on_current(device) -> None:
    """Kernels are launched on the current device's stream."""
    if device.type != "cuda":
        raise ValueError(f"expected operands on the GPU, got them on {device}")
    if device.index != torch.cuda.current_device():
        raise ValueError(f"operands are on {device}, the current device is cuda:{torch.cuda.current_device()}")


@dataclass
class Rotary:
    """Rotation of the first 2 `pairs` values of a head: of pair p by positions[:, axis p] times its frequency.  Made by rotary()."""
    table: torch.Tensor   # int32 [pairs, 4] on the GPU: a 64-bit fraction of a turn, the axis, 0
    pairs: int
    axes: int
    interleaved: bool     # pairs (2 p, 2 p + 1); otherwise (p, p + pairs)


def rotary(sections, theta: float = 10000.0, interleaved: bool = False, device=None, freqs=None, restart: bool = True) -> Rotary:
    """sections: pairs of each of one to four axes of positions (the pairs of the first axis come first; a multiple of four in all).  Frequencies are
    theta^(-i / n) over the n pairs of an axis, restart=False: over all pairs; freqs: given ones (radians for one position), as many as pairs."""
    import numpy as np

    sections = [int(n) for n in sections]
    pairs = sum(sections)
    if not 1 <= len(sections) <= 4 or min(sections) < 0 or pairs == 0 or pairs % 4:
        raise ValueError(f"a rotation has one to four axes, and a multiple of four pairs in all, got {sections}")
    if freqs is None:
        freqs = [theta ** (-i / n) for n in sections for i in range(n)] if restart else [theta ** (-i / pairs) for i in range(pairs)]
    freq = np.ascontiguousarray([float(f) for f in freqs], np.float64)
    if freq.shape != (pairs,):
        raise ValueError(f"{pairs} pairs, {freq.shape[0]} frequencies")
    axis = np.repeat(np.arange(len(sections), dtype=np.int32), sections)
    table = np.zeros((pairs, 4), np.int32)
    _check(load().mq_rotary_table(_np_ptr(freq), _np_ptr(axis), pairs, _np_ptr(table)), "mq_rotary_table")
    device = torch.device("cuda" if device is None else device)
    return Rotary(torch.from_numpy(table).to(device), pairs, len(sections), bool(interleaved))


def _rotary_parts(r: Optional[Rotary]):
    return (None, 0, 0, False) if r is None else (r.table, r.pairs, r.axes, r.interleaved)


def _head_args(x: torch.Tensor, q_heads: int, k_heads: int, q_weight, k_weight, rot: Optional[Rotary], positions, eps, norm: bool):
    """Arguments from the sizes to the positions, checked; what they point to has to live until the call."""
    M, cols = x.shape
    heads = int(q_heads) + int(k_heads)
    if q_heads < 0 or k_heads < 0 or heads == 0 or cols % heads:
        raise ValueError(f"{cols} columns are no {q_heads} query and {k_heads} key heads")
    D = cols // heads
    if not norm and (q_weight is not None or k_weight is not None):
        raise ValueError("weights without the norm")
    p = q_weight if q_weight is not None else k_weight
    for t in (q_weight, k_weight):
        _vector(t, D, None if p is None else p.dtype, x.device)
    pt = F32 if p is None or p.dtype == torch.float32 else _dtype_code(p)
    if (rot is None) != (positions is None):
        raise ValueError("a rotation goes with positions")
    if rot is None:
        turn = (None, 0, 0, None, 4, 0, C.c_long(0))
    else:
        pos = positions if positions.dim() == 2 else positions.unsqueeze(-1)
        if pos.dim() != 2 or tuple(pos.shape) != (M, rot.axes) or pos.device != x.device:
            raise ValueError(f"expected positions [{M}, {rot.axes}] on {x.device}, got {tuple(positions.shape)} on {positions.device}")
        if pos.dtype not in (torch.int32, torch.int64):
            raise TypeError(f"positions are int32 or int64, got {pos.dtype}")
        if (rot.axes > 1 and pos.stride(1) != 1) or (M > 1 and pos.stride(0) < rot.axes):
            pos = pos.contiguous()
        if rot.table.device != x.device or rot.table.dtype != torch.int32 or tuple(rot.table.shape) != (rot.pairs, 4) or not rot.table.is_contiguous():
            raise ValueError(f"expected a rotation's table on {x.device}, got {tuple(rot.table.shape)} of {rot.table.dtype} on {rot.table.device}")
        turn = (_ptr(rot.table), rot.pairs, int(rot.interleaved), _ptr(pos), pos.element_size(), rot.axes, C.c_long(pos.stride(0) if M > 1 else rot.axes))
        positions = pos
    return (M, int(q_heads), int(k_heads), D, _ld(x), _ptr(q_weight), _ptr(k_weight), pt, C.c_float(eps), int(norm), *turn), positions


def qk_norm_rope(x: torch.Tensor, q_heads: int, k_heads: int, q_weight: Optional[torch.Tensor] = None, k_weight: Optional[torch.Tensor] = None,
                 rotary: Optional[Rotary] = None, positions: Optional[torch.Tensor] = None, eps: float = 1e-6, norm: bool = True,
                 out: Optional[torch.Tensor] = None) -> torch.Tensor:
    """Norm of every query and key head, x w / sqrt(mean x^2 + eps), and its rotation by position.  x [M, (q_heads + k_heads) D] fp16/bf16: a row's
    query heads, then its key heads (of a stacked q, k, v the columns in front of the values: qkv[:, :n], with out the same to work in place).  q_weight, k_weight [D]
    in 16 bits or float32.  rotary: from rotary(); positions: int32 or int64 [M, axes], [M] for one axis.  norm=False: the rotation alone.  out may be x."""
    if out is None:
        r = (_native or _load_native()).qk_norm_rope(x, q_heads, k_heads, q_weight, k_weight, *_rotary_parts(rotary), positions, eps, norm)
        if r is not None:
            return _done(r, "mq_qk_norm_rope")
    _no_graph("qk_norm_rope", x, q_weight, k_weight)
    _matrix(x)
    _on_current(x.device)
    dt = _dtype_code(x)
    args, positions = _head_args(x, q_heads, k_heads, q_weight, k_weight, rotary, positions, eps, norm)
    y = _out(out, *x.shape, x.dtype, x.device)
    _check(load().mq_qk_norm_rope(_ptr(x), *args, _ptr(y), _ld(y), dt, _stream()), "mq_qk_norm_rope")
    return y


def qk_norm_rope_grad_workspace_bytes(M: int, q_heads: int, k_heads: int, D: int) -> int:
    return int(load().mq_qk_norm_rope_grad_workspace_bytes(M, q_heads, k_heads, D))


def qk_norm_rope_grad(dy: torch.Tensor, x: Optional[torch.Tensor], q_heads: int, k_heads: int, q_weight: Optional[torch.Tensor] = None,
                      k_weight: Optional[torch.Tensor] = None, rotary: Optional[Rotary] = None, positions: Optional[torch.Tensor] = None, eps: float = 1e-6,
                      norm: bool = True, out: Optional[torch.Tensor] = None, ws: Optional[torch.Tensor] = None):
    """(dx, dq_weight, dk_weight) of qk_norm_rope, x its input; the latter two float32 [D], sums over rows and heads, None without a norm (which needs no x
    either).  out may be dy or x."""
    if out is None and ws is None and norm:
        r = (_native or _load_native()).qk_norm_rope_grad(dy, x, q_heads, k_heads, q_weight, k_weight, *_rotary_parts(rotary), positions, eps, norm)
        if r is not None:
            return _done(r, "mq_qk_norm_rope_grad")
    _no_graph("qk_norm_rope_grad", dy)
    _matrix(dy)
    _on_current(dy.device)
    dt = _dtype_code(dy)
    if norm:
        if x is None:
            raise ValueError("the gradient of the norm takes its input")
        _matrix(x, *dy.shape, dy.dtype, dy.device)
    else:
        x = None
    args, positions = _head_args(dy if x is None else x, q_heads, k_heads, q_weight, k_weight, rotary, positions, eps, norm)
    M, D = args[0], args[3]
    dx = _out(out, *dy.shape, dy.dtype, dy.device)
    sums = torch.empty((2, D), dtype=torch.float32, device=dy.device) if norm else None
    ws = _mx_workspace(qk_norm_rope_grad_workspace_bytes(M, q_heads, k_heads, D), dy.device, ws) if norm else None
    dq, dk = (None, None) if sums is None else (sums[0], sums[1])
    _check(load().mq_qk_norm_rope_grad(_ptr(dy), _ld(dy), _ptr(x), *args, _ptr(dx), _ld(dx), dt, _ptr(dq), _ptr(dk), *_ws_args(ws), _stream()),
           "mq_qk_norm_rope_grad")
    return dx, dq, dk


_ACTS = {None: 0, "gelu": 1, "gelu_tanh": 2, "silu": 3}


def _act_code(act: Optional[str], gated: bool) -> int:
    if act not in _ACTS:
        raise ValueError(f"activations are gelu, gelu_tanh and silu, got {act!r}")
    if gated and act is None:
        raise ValueError("a gate has an activation")
    return _ACTS[act]


def _pre_out(want: bool, rows: int, cols: int, dtype, device):
    return torch.empty((rows, cols), dtype=dtype, device=device) if want else None


def _mx_linear_act(x, w: MxTensor, bias, out, residual, ws, dtype, act, gated: bool, want_pre: bool):
    packed = isinstance(x, MxTensor)
    if act is None:
        raise ValueError("gated and want_pre go with an activation")
    code = _act_code(act, gated)
    if out is None and ws is None:
        native = _native or _load_native()
        if packed:
            if x.K == w.K:
                r = native.mx_linear_act_codes(x.data, x.rows, x.K, w.data, w.rows, bias, residual, code, gated, want_pre,
                                               1 if dtype == torch.bfloat16 else 0 if dtype in _HALF else -1)
                if r is not None:
                    return _done(r, "mq_mx_linear_act_codes")
        elif dtype is None:
            r = native.mx_linear_act(x, w.data, w.rows, w.K, bias, residual, code, gated, want_pre)
            if r is not None:
                return _done(r, "mq_mx_linear_act")
    _no_graph("mx_linear", None if packed else x, bias, residual)
    if packed:
        M, K, device = x.rows, x.K, x.data.device
        dtype = dtype or (out.dtype if out is not None else torch.float16)
    else:
        (M, K), device = _matrix(x).shape, x.device
        if dtype is not None and dtype != x.dtype:
            raise TypeError(f"the output has the type of the activations, {x.dtype}")
        dtype = x.dtype
    _on_current(device)
    if K != w.K:
        raise ValueError(f"activations have {K} columns, weights {w.K}")
    if gated and (w.rows % 64 or residual is not None):
        raise ValueError(f"a gate takes a multiple of 64 rows of weights and no residual, got {w.rows}")
    N = w.rows
    outs = N // 2 if gated else N
    y = _out(out, M, outs, dtype, device)
    dt = _dtype_code(y)
    pre = _pre_out(want_pre, M, N, dtype, device)
    if residual is not None:
        _matrix(residual, M, outs, dtype, device)
    args = (_mx_data(w, device), N, _ptr(_vector(bias, N, dtype, device)), code, int(gated), _ptr(y), _ld(y), dt, _ptr(residual), _ld(residual), _ptr(pre), _ld(pre))
    if packed:
        _check(load().mq_mx_linear_act_codes(_mx_data(x, device), M, K, *args, _stream()), "mq_mx_linear_act_codes")
    else:
        ws = _mx_workspace(mx_linear_workspace_bytes(M, N, K) or (0 if out is None else mx_bytes(M, K)), device, ws)
        _check(load().mq_mx_linear_act(_ptr(x), M, K, _ld(x), *args, _ptr(ws), _bytes_of(ws), _stream()), "mq_mx_linear_act")
    return (y, pre) if want_pre else y


def act_grad_workspace_bytes(M: int, N: int, gated: bool = False) -> int:
    return int(load().mq_act_grad_workspace_bytes(M, N, int(gated)))


def act_grad(dy: torch.Tensor, pre: torch.Tensor, act: str, gated: bool = False, want_dbias: bool = True, out: Optional[torch.Tensor] = None,
             ws: Optional[torch.Tensor] = None):
    """(da, dbias): the gradient of mx_linear's sums behind its activation, which mx_linear_grad takes, and the bias' (float32 [N], None without want_dbias).
    pre [M, N]: from want_pre.  dy [M, N], gated [M, N / 2].  out may be pre, and dy if not gated."""
    code = _act_code(act, gated)
    if not code:
        raise ValueError("act_grad is behind an activation")
    if out is None and ws is None and want_dbias:
        r = (_native or _load_native()).act_grad(dy, pre, code, gated)
        if r is not None:
            return _done(r, "mq_act_grad")
    _no_graph("act_grad", dy, pre)
    M, N = _matrix(pre).shape
    _on_current(pre.device)
    if gated and N % 2:
        raise ValueError(f"a gate has two halves, got {N} columns")
    _matrix(dy, M, N // 2 if gated else N, pre.dtype, pre.device)
    da = _out(out, M, N, pre.dtype, pre.device)
    dbias = torch.empty(N, dtype=torch.float32, device=pre.device) if want_dbias else None
    ws = _mx_workspace(act_grad_workspace_bytes(M, N, gated), pre.device, ws) if want_dbias else None
    _check(load().mq_act_grad(_ptr(dy), M, N, _ld(dy), _ptr(pre), _ld(pre), code, int(gated), _ptr(da), _ld(da), _dtype_code(pre), _ptr(dbias), *_ws_args(ws),
                              _stream()), "mq_act_grad")
    return da, dbias


def mx_experts(t: MxTensor, experts: int) -> MxTensor:
    """A microscaled matrix as the weights of `experts` experts, one's rows behind another's, a multiple of 32 rows each; with what the gradient needs."""
    if experts <= 0 or t.rows % (32 * experts):
        raise ValueError(f"{t.rows} rows are no {experts} experts of a multiple of 32 rows")
    _on_current(t.data.device)
    data = _mx_data(t)
    top = torch.empty((experts, t.K // 32), dtype=torch.uint8, device=t.data.device)
    _check(load().mq_mx_experts_column_top(data, experts, t.rows // experts, t.K, _ptr(top), _stream()), "mq_mx_experts_column_top")
    return MxTensor(t.data, t.rows, t.K, top, experts)


def mx_quantize_experts(w: torch.Tensor) -> MxTensor:
    """Weights [experts, N, K] fp16/bf16, N % 32 == 0, for mx_linear_grouped and its gradient."""
    if w.dim() != 3:
        raise ValueError(f"expected weights [experts, N, K], got {tuple(w.shape)}")
    _on_current(w.device)
    return mx_experts(mx_quantize(w.reshape(w.shape[0] * w.shape[1], w.shape[2])), w.shape[0])


def _expert_args(M: int, w: MxTensor, offsets: torch.Tensor, device):
    if w.experts <= 0 or w.rows % (32 * w.experts):
        raise ValueError(f"{w.rows} rows are no {w.experts} experts of a multiple of 32 rows")
    _vector(offsets, w.experts + 1, torch.int32, device)
    return w.rows // w.experts


def mx_linear_grouped_workspace_bytes(M: int, N: int, K: int, experts: int) -> int:
    return int(load().mq_mx_linear_grouped_workspace_bytes(M, N, K, experts))


def mx_linear_grouped(x: torch.Tensor, w: MxTensor, offsets: torch.Tensor, bias: Optional[torch.Tensor] = None, out: Optional[torch.Tensor] = None,
                      ws: Optional[torch.Tensor] = None, act: Optional[str] = None, gated: bool = False, want_pre: bool = False):
    """Rows sorted by expert, each expert's times its own weights: Y[r] = mx(X[r]) . W_e^T + bias[e] for offsets[e] <= r < offsets[e + 1]; act, gated and
    want_pre as in mx_linear.  w: from mx_quantize_experts or mx_experts; offsets: int32 [experts + 1] on the GPU, never read on the host; bias [experts, N].  Rows that
    no expert has are left as they are in out (and hold nothing in particular otherwise).  out shares nothing with x."""
    code = _act_code(act, gated)
    if want_pre and act is None:
        raise ValueError("want_pre goes with an activation")
    if out is None and ws is None and w.experts > 0 and w.rows % w.experts == 0:
        r = (_native or _load_native()).mx_linear_grouped(x, w.data, w.rows // w.experts, w.K, w.experts, offsets, bias, code, gated, want_pre)
        if r is not None:
            return _done(r, "mq_mx_linear_grouped")
    _no_graph("mx_linear_grouped", x, bias)
    M, K = _matrix(x).shape
    device = x.device
    _on_current(device)
    if K != w.K:
        raise ValueError(f"activations have {K} columns, weights {w.K}")
    N = _expert_args(M, w, offsets, device)
    if gated and N % 64:
        raise ValueError(f"a gate takes a multiple of 64 rows of weights, got {N}")
    if bias is not None and (tuple(bias.shape) != (w.experts, N) or not bias.is_contiguous() or bias.dtype != x.dtype or bias.device != device):
        raise ValueError(f"expected a contiguous bias [{w.experts}, {N}] of {x.dtype} on {device}, got {tuple(bias.shape)} of {bias.dtype} on {bias.device}")
    y = _out(out, M, N // 2 if gated else N, x.dtype, device)
    pre = _pre_out(want_pre, M, N, x.dtype, device)
    ws = _mx_workspace(mx_linear_grouped_workspace_bytes(M, N, K, w.experts), device, ws)
    _check(load().mq_mx_linear_grouped(_ptr(x), M, K, _ld(x), _mx_data(w, device), N, w.experts, _ptr(offsets), _ptr(bias), code, int(gated), _ptr(y), _ld(y),
                                       _dtype_code(x), _ptr(pre), _ld(pre), *_ws_args(ws), _stream()), "mq_mx_linear_grouped")
    return (y, pre) if want_pre else y


def mx_linear_grouped_grad(dy: torch.Tensor, w: MxTensor, offsets: torch.Tensor, out: Optional[torch.Tensor] = None) -> torch.Tensor:
    """dX[r] = dY[r] . W_e, the gradient of mx_linear_grouped with respect to its rows (the quantisation passed straight through).  out shares nothing with dy."""
    if out is None and w.top is not None and w.experts > 0 and w.rows % w.experts == 0:
        r = (_native or _load_native()).mx_linear_grouped_grad(dy, w.data, w.rows // w.experts, w.K, w.experts, w.top, offsets)
        if r is not None:
            return _done(r, "mq_mx_linear_grouped_grad")
    _no_graph("mx_linear_grouped_grad", dy)
    M, N = _matrix(dy).shape
    _on_current(dy.device)
    if _expert_args(M, w, offsets, dy.device) != N:
        raise ValueError(f"gradients have {N} columns, an expert's weights {w.rows // w.experts} rows")
    if w.top is None or w.top.numel() != w.experts * (w.K // 32) or w.top.dtype != torch.uint8 or not w.top.is_contiguous() or w.top.device != dy.device:
        raise ValueError("weights without the experts' `top`: make them with mx_quantize_experts or mx_experts")
    dx = _out(out, M, w.K, dy.dtype, dy.device)
    _check(load().mq_mx_linear_grouped_grad(_ptr(dy), M, N, _ld(dy), _mx_data(w, dy.device), _ptr(w.top), w.K, w.experts, _ptr(offsets), _ptr(dx), _ld(dx),
                                            _dtype_code(dy), _stream()), "mq_mx_linear_grouped_grad")
    return dx
