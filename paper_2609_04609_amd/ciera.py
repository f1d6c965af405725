"""ctypes binding of libciera (the C ABI in include/ciera.h).

Argument marshalling only: every function forwards to the library call of the
same name, and every step of the codec runs in the library's HIP kernels. The
``*_t`` helpers accept torch tensors and pass their device pointers and the
current HIP stream. Opening the library fails loudly when it is not built;
there is no fallback.
"""
from __future__ import annotations

import ctypes
import os

import torch

_HERE = os.path.dirname(os.path.abspath(__file__))
LIB_PATH = os.path.join(_HERE, "libciera.so")

OK, EINVAL, ENOSPC, EUNSUPPORTED, EFORMAT, EHIP = 0, -1, -2, -3, -4, -5
DEVERR_FORMAT, DEVERR_ALIGN, DEVERR_BOUNDS, DEVERR_NOSPACE = 1, 2, 4, 8
ENC_RAW = 0x1
FP16 = 0x2
ENC_UPDATE_CACHE = 0x4
WS_ANS = 0x1
SELECT_STOP_AT_MISFIT = 0x1
HEADER_BYTES = 64
ROUTE_SIGMOID, ROUTE_NORMALIZE, ROUTE_GROUP_TOP_TWO = 0x1, 0x2, 0x4
STATUS_NAMES = {OK: "OK", EINVAL: "EINVAL", ENOSPC: "ENOSPC",
                EUNSUPPORTED: "EUNSUPPORTED", EFORMAT: "EFORMAT",
                EHIP: "EHIP"}


class CieraError(RuntimeError):
    def __init__(self, fn, code):
        super().__init__(f"{fn} returned {STATUS_NAMES.get(code, code)}")
        self.code = code


class ShardStats(ctypes.Structure):
    _fields_ = [("n_elems", ctypes.c_uint64), ("block_elems", ctypes.c_uint32),
                ("flags", ctypes.c_uint32), ("q", ctypes.c_double)]


class CostModel(ctypes.Structure):
    _fields_ = [("world_size", ctypes.c_uint32), ("alpha_s", ctypes.c_double),
                ("bus_bw_Bps", ctypes.c_double), ("t_hash_s", ctypes.c_double),
                ("t_cmp_s", ctypes.c_double), ("t_decmp_s", ctypes.c_double),
                ("header_bytes", ctypes.c_double), ("overlapped", ctypes.c_int)]


_vp, _u64, _u32, _i32 = ctypes.c_void_p, ctypes.c_uint64, ctypes.c_uint32, ctypes.c_int
_f32 = ctypes.c_float
_SIGS = {
    "ciera_encoded_bound": (_u64, [_u64, _u32, _u32]),
    "ciera_workspace_bytes": (_u64, [_u64, _u32, _u32, _u32]),
    "ciera_workspace_init": (_i32, [_vp, _u64, _vp]),
    "ciera_workspace_error": (_i32, [_vp, ctypes.POINTER(_u32), _i32, _vp]),
    "ciera_encode": (_i32, [_vp, _vp, _u64, _u32, _u32, _vp, _u64, _vp, _vp,
                            _u64, _vp]),
    "ciera_decode_gathered": (_i32, [_vp, _u64, _vp, _u32, _u64, _u32, _u32,
                                     _vp, _vp, _vp, _u64, _vp]),
    "ciera_update_cache": (_i32, [_vp, _vp, _u64, _u64, _u32, _u32, _vp, _u64,
                                  _vp]),
    "ciera_decode_gathered_noalloc": (_i32, [_vp, _u64, _vp, _u32, _u64,
                                             _u32, _u32, _vp, _vp, _vp,
                                             _vp]),
    "ciera_ans_code": (_i32, [_vp, _u64, _u32, _vp, _vp, _u64, _vp]),
    "ciera_hash_blocks": (_i32, [_vp, _u64, _u32, _vp, _vp]),
    "ciera_encode_hashed": (_i32, [_vp, _vp, _vp, _u64, _u32, _vp, _u64, _vp,
                                   _vp, _u64, _vp]),
    "ciera_should_compress": (_i32, [ctypes.POINTER(ShardStats),
                                     ctypes.POINTER(CostModel),
                                     ctypes.POINTER(ctypes.c_double)]),
    "ciera_select": (_i32, [ctypes.POINTER(ctypes.c_double),
                            ctypes.POINTER(ctypes.c_double), _u64,
                            ctypes.c_double, _u32,
                            ctypes.POINTER(ctypes.c_uint8)]),
    "ciera_route": (_i32, [_vp, _u32, _u64, _u32, _u64, _vp, _u32, _u32, _u32,
                           _u32, _f32, _vp, _vp, _vp]),
    "ciera_route_backward": (_i32, [_vp, _u32, _u64, _u32, _u64, _u32, _u32,
                                    _f32, _vp, _vp, _vp, _u64, _vp]),
    "ciera_plan_workspace_bytes": (_u64, [_u64, _u32, _u32]),
    "ciera_route_plan": (_i32, [_vp, _u64, _u32, _u32, _u32, _vp, _vp, _vp,
                                _vp, _u64, _vp]),
    "ciera_quantize_rows": (_i32, [_vp, _u32, _u64, _u64, _u64, _vp, _u32,
                                   _u64, _vp, _u64, _vp, _u64, _vp]),
    "ciera_quantize_blocks": (_i32, [_vp, _u32, _u64, _u64, _u64, _vp, _u64,
                                     _vp, _u64, _vp, _u64, _vp, _u64, _vp]),
    "ciera_columns_length": (_u64, [_u64, _u32]),
    "ciera_quantize_columns": (_i32, [_vp, _u32, _u64, _u64, _u64, _u64, _vp,
                                      _u32, _vp, _u32, _vp, _u64, _vp, _u64,
                                      _vp]),
    "ciera_expert_matmul": (_i32, [_vp, _u64, _vp, _u64, _u64, _vp, _u64, _vp,
                                   _u64, _u32, _u64, _u64, _vp, _vp, _u32,
                                   _u64, _vp]),
    "ciera_expert_weight_grad": (_i32, [_vp, _vp, _u64, _vp, _vp, _u64, _u64,
                                        _u32, _u64, _u64, _vp, _vp, _u32,
                                        _vp]),
    "ciera_combine": (_i32, [_vp, _u32, _u64, _u64, _u64, _vp, _vp, _u64, _u32,
                             _vp, _u64, _vp]),
    "ciera_combine_backward": (_i32, [_vp, _u64, _vp, _u32, _u64, _u64, _u64,
                                      _vp, _vp, _u64, _u32, _vp, _u64, _vp,
                                      _vp]),
}
EXPORTED = tuple(_SIGS)

_lib = None


def lib():
    """Open libciera.so (once). Raises if it has not been built."""
    global _lib
    if _lib is None:
        if not os.path.exists(LIB_PATH):
            raise RuntimeError(
                f"{LIB_PATH} is missing: build it with "
                "`python -m paper_2609_04609_amd.build`")
        handle = ctypes.CDLL(LIB_PATH)
        for name, (res, args) in _SIGS.items():
            f = getattr(handle, name)
            f.restype, f.argtypes = res, args
        _lib = handle
    return _lib


def _check(fn, rc):
    if rc < 0:
        raise CieraError(fn, rc)
    return rc


# ---- the C ABI, name for name (pointers and the stream as integers) ----

def ciera_encoded_bound(n_elems, block_elems, flags=0):
    return lib().ciera_encoded_bound(n_elems, block_elems, flags)


def ciera_workspace_bytes(n_elems, nshards, block_elems, flags=0):
    return lib().ciera_workspace_bytes(n_elems, nshards, block_elems, flags)


def ciera_workspace_init(workspace, workspace_bytes, stream):
    return lib().ciera_workspace_init(workspace, workspace_bytes, stream)


def ciera_workspace_error(workspace, clear, stream):
    err = _u32(0)
    rc = lib().ciera_workspace_error(workspace, ctypes.byref(err), clear, stream)
    _check("ciera_workspace_error", rc)
    return err.value


def ciera_encode(w_new, exp_cache, n_elems, block_elems, flags, out,
                 out_capacity, out_bytes, workspace, workspace_bytes, stream):
    return lib().ciera_encode(w_new, exp_cache, n_elems, block_elems, flags,
                              out, out_capacity, out_bytes, workspace,
                              workspace_bytes, stream)


def ciera_decode_gathered(gathered, gathered_bytes, shard_offsets, nshards,
                          shard_elems, block_elems, out, exp_cache, workspace,
                          workspace_bytes, stream, flags=0):
    """The C call of the same name; `flags` (0 or FP16) comes last here."""
    return lib().ciera_decode_gathered(gathered, gathered_bytes,
                                       shard_offsets, nshards, shard_elems,
                                       block_elems, flags, out, exp_cache,
                                       workspace, workspace_bytes, stream)


def ciera_decode_gathered_noalloc(gathered, gathered_bytes, shard_offsets,
                                  nshards, shard_elems, block_elems, out,
                                  exp_cache, err, stream, flags=0):
    """The C call of the same name; `flags` (0 or FP16) comes last here."""
    return lib().ciera_decode_gathered_noalloc(
        gathered, gathered_bytes, shard_offsets, nshards, shard_elems,
        block_elems, flags, out, exp_cache, err, stream)


def ciera_update_cache(exp_cache, encoded, encoded_bytes, n_elems,
                       block_elems, workspace, workspace_bytes, stream,
                       flags=0):
    """The C call of the same name; `flags` (0 or FP16) comes last here."""
    return lib().ciera_update_cache(exp_cache, encoded, encoded_bytes,
                                    n_elems, block_elems, flags, workspace,
                                    workspace_bytes, stream)


def ciera_ans_code(encoded, n_elems, block_elems, out_bytes, workspace,
                   workspace_bytes, stream):
    return lib().ciera_ans_code(encoded, n_elems, block_elems, out_bytes,
                                workspace, workspace_bytes, stream)


def ciera_hash_blocks(w, n_elems, block_elems, hash_cache, stream):
    return lib().ciera_hash_blocks(w, n_elems, block_elems, hash_cache, stream)


def ciera_encode_hashed(w_new, hash_in, hash_out, n_elems, block_elems, out,
                        out_capacity, out_bytes, workspace, workspace_bytes,
                        stream):
    return lib().ciera_encode_hashed(w_new, hash_in, hash_out, n_elems,
                                     block_elems, out, out_capacity, out_bytes,
                                     workspace, workspace_bytes, stream)


def ciera_should_compress(n_elems, block_elems, q, world_size, alpha_s,
                          bus_bw_Bps, t_hash_s=0.0, t_cmp_s=0.0, t_decmp_s=0.0,
                          header_bytes=float(HEADER_BYTES), overlapped=True,
                          fp16=False):
    """Returns (decision 0/1, gain in seconds)."""
    st = ShardStats(n_elems, block_elems, FP16 if fp16 else 0, q)
    cm = CostModel(world_size, alpha_s, bus_bw_Bps, t_hash_s, t_cmp_s,
                   t_decmp_s, header_bytes, int(overlapped))
    g = ctypes.c_double(0.0)
    rc = lib().ciera_should_compress(ctypes.byref(st), ctypes.byref(cm),
                                     ctypes.byref(g))
    _check("ciera_should_compress", rc)
    return rc, g.value


def ciera_select(gains, mems, budget_bytes, flags=0):
    n = len(gains)
    G = (ctypes.c_double * n)(*gains)
    M = (ctypes.c_double * n)(*mems)
    S = (ctypes.c_uint8 * n)()
    rc = lib().ciera_select(G, M, n, budget_bytes, flags, S)
    _check("ciera_select", rc)
    return [bool(x) for x in S]


def ciera_route(logits, dtype, n_tokens, n_experts, row_stride, bias,
                n_groups, top_groups, top_k, flags, scale, expert_ids,
                weights, stream):
    return lib().ciera_route(logits, dtype, n_tokens, n_experts, row_stride,
                             bias, n_groups, top_groups, top_k, flags, scale,
                             expert_ids, weights, stream)


def ciera_route_backward(logits, dtype, n_tokens, n_experts, row_stride,
                         top_k, flags, scale, expert_ids, d_weights, d_logits,
                         d_row_stride, stream):
    return lib().ciera_route_backward(
        logits, dtype, n_tokens, n_experts, row_stride, top_k, flags, scale,
        expert_ids, d_weights, d_logits, d_row_stride, stream)


def ciera_plan_workspace_bytes(n_tokens, top_k, n_experts):
    return lib().ciera_plan_workspace_bytes(n_tokens, top_k, n_experts)


def ciera_route_plan(expert_ids, n_tokens, top_k, first_expert, n_experts,
                     offsets, source, position, workspace, workspace_bytes,
                     stream):
    return lib().ciera_route_plan(expert_ids, n_tokens, top_k, first_expert,
                                  n_experts, offsets, source, position,
                                  workspace, workspace_bytes, stream)


def ciera_quantize_rows(x, dtype, n_rows, n_cols, row_stride, position, top_k,
                        q_rows, q, q_stride, scales, scale_stride, stream):
    return lib().ciera_quantize_rows(x, dtype, n_rows, n_cols, row_stride,
                                     position, top_k, q_rows, q, q_stride,
                                     scales, scale_stride, stream)


def ciera_quantize_blocks(w, dtype, batch, n_rows, n_cols, q, q_stride, scales,
                          scale_stride, q_t, qt_stride, scales_t,
                          scale_t_stride, stream):
    return lib().ciera_quantize_blocks(w, dtype, batch, n_rows, n_cols, q,
                                       q_stride, scales, scale_stride, q_t,
                                       qt_stride, scales_t, scale_t_stride,
                                       stream)


def ciera_columns_length(n_rows, n_experts):
    return lib().ciera_columns_length(n_rows, n_experts)


def ciera_quantize_columns(x, dtype, n_x, n_rows, n_cols, row_stride, source,
                           top_k, offsets, n_experts, q_t, length, scales,
                           scale_stride, stream):
    return lib().ciera_quantize_columns(x, dtype, n_x, n_rows, n_cols,
                                        row_stride, source, top_k, offsets,
                                        n_experts, q_t, length, scales,
                                        scale_stride, stream)


def ciera_expert_matmul(a, a_stride, a_scales, a_scale_stride, n_rows, b,
                        b_stride, b_scales, b_scale_stride, n_experts, n_out,
                        depth, offsets, out, out_dtype, out_stride, stream):
    return lib().ciera_expert_matmul(a, a_stride, a_scales, a_scale_stride,
                                     n_rows, b, b_stride, b_scales,
                                     b_scale_stride, n_experts, n_out, depth,
                                     offsets, out, out_dtype, out_stride,
                                     stream)


def ciera_expert_weight_grad(dy_t, dy_scales, dy_scale_stride, x_t, x_scales,
                             x_scale_stride, length, n_experts, n_out, n_cols,
                             offsets, d_w, out_dtype, stream):
    return lib().ciera_expert_weight_grad(
        dy_t, dy_scales, dy_scale_stride, x_t, x_scales, x_scale_stride,
        length, n_experts, n_out, n_cols, offsets, d_w, out_dtype, stream)


def ciera_combine(rows, dtype, n_rows, n_cols, row_stride, weights, position,
                  n_tokens, top_k, out, out_stride, stream):
    return lib().ciera_combine(rows, dtype, n_rows, n_cols, row_stride,
                               weights, position, n_tokens, top_k, out,
                               out_stride, stream)


def ciera_combine_backward(d_out, d_out_stride, rows, dtype, n_rows, n_cols,
                           row_stride, weights, position, n_tokens, top_k,
                           d_rows, d_row_stride, d_weights, stream):
    return lib().ciera_combine_backward(
        d_out, d_out_stride, rows, dtype, n_rows, n_cols, row_stride, weights,
        position, n_tokens, top_k, d_rows, d_row_stride, d_weights, stream)


# ---- tensor-level marshalling ----

# not part of torch's public interface, so a build may lack it
_raw_stream = getattr(torch._C, "_cuda_getCurrentRawStream", None)


def _stream(device=None):
    """The current stream's handle; ``device`` is the current device's index
    where it is known. Asked for directly where torch has the call for it: the
    Stream object that torch.cuda.current_stream() builds around it costs 2.8
    us a call, as much as a kernel launch; this takes 0.3."""
    if _raw_stream is None:
        return torch.cuda.current_stream().cuda_stream
    return _raw_stream(torch.cuda.current_device() if device is None
                       else device)


def _ptr(t):
    return 0 if t is None else t.data_ptr()


class Workspace:
    """Device workspace sized for a shard size, shard count and B; with
    ans=True also for rANS coding and decoding (CIERA_WS_ANS)."""

    def __init__(self, n_elems, nshards, block_elems, device="cuda",
                 ans=False):
        self.nbytes = int(ciera_workspace_bytes(n_elems, nshards, block_elems,
                                                WS_ANS if ans else 0))
        if self.nbytes == 0:
            raise CieraError("ciera_workspace_bytes", EUNSUPPORTED)
        self.buf = torch.empty(self.nbytes, dtype=torch.uint8, device=device)
        _check("ciera_workspace_init",
               ciera_workspace_init(self.buf.data_ptr(), self.nbytes,
                                    _stream()))

    @property
    def ptr(self):
        return self.buf.data_ptr()

    def error(self, clear=True):
        return ciera_workspace_error(self.ptr, int(clear), _stream())


def encode_t(w_bits, cache, block_elems, ws, out, raw=False, out_bytes=None,
             fp16=False, update_cache=False):
    """Encode a 1-D int16 bit tensor into ``out`` (uint8, bound-sized); with
    update_cache the cache is brought forward in place."""
    n = w_bits.numel()
    flags = ((ENC_RAW if raw else 0) | (FP16 if fp16 else 0) |
             (ENC_UPDATE_CACHE if update_cache else 0))
    rc = ciera_encode(_ptr(w_bits), _ptr(cache), n, block_elems, flags,
                      _ptr(out), out.numel(), _ptr(out_bytes), ws.ptr,
                      ws.nbytes, _stream())
    return _check("ciera_encode", rc)


def hash_blocks_t(w_bits, block_elems, hash_cache):
    """HashCache (int64 tensor of 2 * ceil(n/B) words) of a 1-D bit tensor."""
    rc = ciera_hash_blocks(_ptr(w_bits), w_bits.numel(), block_elems,
                           _ptr(hash_cache), _stream())
    return _check("ciera_hash_blocks", rc)


def encode_hashed_t(w_bits, hash_in, hash_out, block_elems, ws, out,
                    out_bytes=None):
    rc = ciera_encode_hashed(_ptr(w_bits), _ptr(hash_in), _ptr(hash_out),
                             w_bits.numel(), block_elems, _ptr(out),
                             out.numel(), _ptr(out_bytes), ws.ptr, ws.nbytes,
                             _stream())
    return _check("ciera_encode_hashed", rc)


def ans_code_t(encoded, n_elems, block_elems, ws, out_bytes=None):
    """rANS-code the exception section of an encoded shard in place."""
    rc = ciera_ans_code(_ptr(encoded), n_elems, block_elems, _ptr(out_bytes),
                        ws.ptr, ws.nbytes, _stream())
    return _check("ciera_ans_code", rc)


def _nbytes(t, nbytes):
    return t.numel() * t.element_size() if nbytes is None else nbytes


def decode_gathered_t(gathered, offsets, shard_elems, block_elems, out, cache,
                      ws, fp16=False, nbytes=None):
    """Decode the shards of a gathered uint8 tensor; its length bounds every
    shard unless ``nbytes`` gives another."""
    rc = ciera_decode_gathered(_ptr(gathered), _nbytes(gathered, nbytes),
                               _ptr(offsets), offsets.numel(), shard_elems,
                               block_elems, _ptr(out), _ptr(cache), ws.ptr,
                               ws.nbytes, _stream(), FP16 if fp16 else 0)
    return _check("ciera_decode_gathered", rc)


def decode_gathered_noalloc_t(gathered, offsets, shard_elems, block_elems,
                              out, cache, err, fp16=False, nbytes=None):
    """decode_gathered_t without a workspace; ``err`` is a one-element int32
    device tensor that receives the call's device error bits."""
    rc = ciera_decode_gathered_noalloc(
        _ptr(gathered), _nbytes(gathered, nbytes), _ptr(offsets),
        offsets.numel(), shard_elems, block_elems, _ptr(out), _ptr(cache),
        _ptr(err), _stream(), FP16 if fp16 else 0)
    return _check("ciera_decode_gathered_noalloc", rc)


def update_cache_t(cache, encoded, n_elems, block_elems, ws, fp16=False,
                   nbytes=None):
    rc = ciera_update_cache(_ptr(cache), _ptr(encoded),
                            _nbytes(encoded, nbytes), n_elems, block_elems,
                            ws.ptr, ws.nbytes, _stream(), FP16 if fp16 else 0)
    return _check("ciera_update_cache", rc)


# ---- the experts' products ----
#
# Outputs are the caller's, as above. Shapes, types and devices are checked here,
# since the library sees pointers alone: a mistake raises ValueError before
# anything is enqueued. A call asks everything of its arguments in one expression
# (`_packed`, `_strided`), some 0.3 us a tensor, and only where that fails goes
# through them one by one for the words (`_refuse`).

_WIDE = {torch.bfloat16: 0, torch.float16: 1, torch.float32: 2}
_E4M3, _INT, _FLOAT, _BYTE = ((torch.float8_e4m3fn,), (torch.int32,),
                              (torch.float32,), (torch.uint8,))

# the current device's index, asked for directly as the stream is
_current_device = getattr(torch._C, "_cuda_getDevice",
                          torch.cuda.current_device)


def _packed(t, dev, dtypes, shape):
    """Whether ``t`` is contiguous, of ``shape`` and one of ``dtypes`` and on
    device ``dev`` (an index; the CPU's is -1)."""
    return (t.get_device() == dev and t.dtype in dtypes and t.shape == shape and
            t.is_contiguous())


def _strided(t, dev, dtypes, shape):
    """The same for a matrix whose rows may be apart, by ``stride(0)``."""
    return (t.get_device() == dev and t.dtype in dtypes and t.shape == shape and
            (t.is_contiguous() or
             (len(shape) == 2 and (shape[1] <= 1 or t.stride(1) == 1) and
              (shape[0] <= 1 or t.stride(0) >= shape[1]))))


def _refuse(dev, *args):
    """Say which of (tensor, name, types, shape, check) does not fit."""
    for t, name, dtypes, shape, check in args:
        if t is None or check(t, dev, dtypes, shape):
            continue
        if t.get_device() != dev:
            raise ValueError(f"{name} is on {t.device}, not on the current "
                             "device")
        if t.dtype not in dtypes:
            raise ValueError(f"{name} has type {t.dtype}")
        if t.shape != shape:
            raise ValueError(f"{name} has shape {tuple(t.shape)}, not "
                             f"{tuple(shape)}")
        raise ValueError(f"{name} is not contiguous")
    raise ValueError("arguments do not fit each other")


def _device(t, name):
    """The current device's index, for a call whose first tensor is ``t``."""
    if not t.is_cuda:
        raise ValueError(f"{name} is on {t.device}, not on the current device")
    return _current_device()


def _dims(t, name, n):
    """The shape of a tensor of ``n`` dimensions."""
    if t.dim() != n:
        raise ValueError(f"{name} has {t.dim()} dimensions, not {n}")
    return t.shape


def _refuse_dims(*args):
    """Say which (tensor, name, dimensions) has others, after its shape did not
    unpack; asked first, it would cost 0.2 us a tensor."""
    for t, name, n in args:
        _dims(t, name, n)
    raise ValueError("arguments do not fit each other")


def _row_stride(t, cols):
    """Elements from a row of a checked matrix of ``cols`` columns to the next.
    Asking a tensor for one stride costs four times what is_contiguous does."""
    return (cols or 1) if t.is_contiguous() else t.stride(0)


def _scales_fit(s, filled):
    return s.shape[-1] * 128 >= filled


def quantized_shapes(rows, cols):
    """Shapes of an 8-bit matrix of ``rows`` x ``cols`` values and of its
    scales, one a block of 128 values of a row: rows are filled up to whole
    blocks, scale rows to whole dwords."""
    blocks = -(-cols // 128)
    return (rows, 128 * blocks), (rows, -(-blocks // 4) * 4)


def route_t(logits, expert_ids, weights, bias=None, groups=1, top_groups=1,
            group_top_two=False, sigmoid=False, normalize=False, scale=1.0):
    """Choose experts: ``logits`` [T, E] -> ``expert_ids`` int32 and
    ``weights`` fp32, both [T, k]; ``bias`` fp32 [E]."""
    try:
        (T, E), (_, k) = logits.shape, expert_ids.shape
    except ValueError:
        _refuse_dims((logits, "logits", 2), (expert_ids, "expert_ids", 2))
    dev = _device(logits, "logits")
    if not (_strided(logits, dev, _WIDE, (T, E)) and
            _packed(expert_ids, dev, _INT, (T, k)) and
            _packed(weights, dev, _FLOAT, (T, k)) and
            (bias is None or _packed(bias, dev, _FLOAT, (E,)))):
        _refuse(dev, (logits, "logits", _WIDE, (T, E), _strided),
                (expert_ids, "expert_ids", _INT, (T, k), _packed),
                (weights, "weights", _FLOAT, (T, k), _packed),
                (bias, "bias", _FLOAT, (E,), _packed))
    flags = ((ROUTE_SIGMOID if sigmoid else 0) |
             (ROUTE_NORMALIZE if normalize else 0) |
             (ROUTE_GROUP_TOP_TWO if group_top_two else 0))
    rc = lib().ciera_route(
        logits.data_ptr(), _WIDE[logits.dtype], T, E, _row_stride(logits, E),
        _ptr(bias), groups, top_groups, k, flags, scale,
        expert_ids.data_ptr(), weights.data_ptr(), _stream(dev))
    return _check("ciera_route", rc)


def route_backward_t(logits, expert_ids, d_weights, d_logits, sigmoid=False,
                     normalize=False, scale=1.0):
    """Gradient of route_t's weights -> gradient of its logits."""
    try:
        (T, E), (_, k) = logits.shape, expert_ids.shape
    except ValueError:
        _refuse_dims((logits, "logits", 2), (expert_ids, "expert_ids", 2))
    dev = _device(logits, "logits")
    same = (logits.dtype,)
    if not (_strided(logits, dev, _WIDE, (T, E)) and
            _packed(expert_ids, dev, _INT, (T, k)) and
            _packed(d_weights, dev, _FLOAT, (T, k)) and
            _strided(d_logits, dev, same, (T, E))):
        _refuse(dev, (logits, "logits", _WIDE, (T, E), _strided),
                (expert_ids, "expert_ids", _INT, (T, k), _packed),
                (d_weights, "d_weights", _FLOAT, (T, k), _packed),
                (d_logits, "d_logits", same, (T, E), _strided))
    flags = ((ROUTE_SIGMOID if sigmoid else 0) |
             (ROUTE_NORMALIZE if normalize else 0))
    rc = lib().ciera_route_backward(
        logits.data_ptr(), _WIDE[logits.dtype], T, E, _row_stride(logits, E),
        k, flags, scale, expert_ids.data_ptr(), d_weights.data_ptr(),
        d_logits.data_ptr(), _row_stride(d_logits, E), _stream(dev))
    return _check("ciera_route_backward", rc)


class PlanWorkspace:
    """Device workspace of route_plan_t for up to ``n_tokens`` tokens."""

    def __init__(self, n_tokens, top_k, n_experts, device="cuda"):
        self.nbytes = int(ciera_plan_workspace_bytes(n_tokens, top_k,
                                                     n_experts))
        if self.nbytes == 0:
            raise CieraError("ciera_plan_workspace_bytes", EINVAL)
        self.buf = torch.empty(self.nbytes, dtype=torch.uint8, device=device)


def route_plan_t(expert_ids, n_experts, offsets, source, position, ws,
                 first_expert=0):
    """Sort the (token, slot) pairs of ``expert_ids`` [T, k] by expert:
    ``offsets`` [n_experts + 1], ``source`` [T k], ``position`` [T, k]."""
    try:
        T, k = expert_ids.shape
    except ValueError:
        _refuse_dims((expert_ids, "expert_ids", 2))
    dev = _device(expert_ids, "expert_ids")
    if not (_packed(expert_ids, dev, _INT, (T, k)) and
            _packed(offsets, dev, _INT, (n_experts + 1,)) and
            _packed(source, dev, _INT, (T * k,)) and
            _packed(position, dev, _INT, (T, k)) and
            ws.buf.get_device() == dev):
        _refuse(dev, (expert_ids, "expert_ids", _INT, (T, k), _packed),
                (offsets, "offsets", _INT, (n_experts + 1,), _packed),
                (source, "source", _INT, (T * k,), _packed),
                (position, "position", _INT, (T, k), _packed),
                (ws.buf, "the workspace", _BYTE, (ws.nbytes,), _packed))
    rc = lib().ciera_route_plan(
        expert_ids.data_ptr(), T, k, first_expert, n_experts,
        offsets.data_ptr(), source.data_ptr(), position.data_ptr(),
        ws.buf.data_ptr(), ws.nbytes, _stream(dev))
    return _check("ciera_route_plan", rc)


def quantize_rows_t(x, q, scales, position=None):
    """``x`` [R, C] -> 8-bit rows with a scale per 1 x 128 block: row r to row
    r, or with ``position`` [R, k] to the k rows that it names. ``q`` and
    ``scales`` have the shapes of quantized_shapes()."""
    k = 1
    try:
        (R, C), (Q, _), (_, S) = x.shape, q.shape, scales.shape
        if position is not None:
            _, k = position.shape
    except ValueError:
        _refuse_dims((x, "x", 2), (q, "q", 2), (scales, "scales of q", 2),
                     (position, "position", 2))
    filled = -(-C // 128) * 128
    dev = _device(x, "x")
    if not (_strided(x, dev, _WIDE, (R, C)) and
            _packed(q, dev, _E4M3, (Q, filled)) and
            _packed(scales, dev, _BYTE, (Q, S)) and
            _scales_fit(scales, filled) and
            (position is None or _packed(position, dev, _INT, (R, k)))):
        _refuse(dev, (x, "x", _WIDE, (R, C), _strided),
                (q, "q", _E4M3, (Q, filled), _packed),
                (scales, "scales of q", _BYTE, (Q, S), _packed),
                (position, "position", _INT, (R, k), _packed))
    rc = lib().ciera_quantize_rows(
        x.data_ptr(), _WIDE[x.dtype], R, C, _row_stride(x, C), _ptr(position),
        k, Q, q.data_ptr(), filled, scales.data_ptr(), S, _stream(dev))
    return _check("ciera_quantize_rows", rc)


def quantize_blocks_t(w, q, scales, q_t=None, scales_t=None):
    """``w`` [E, N, C] -> 8-bit with a scale per 128 x 128 block, and with
    ``q_t`` and ``scales_t`` the transpose [E, C, N] too. Shapes: those of
    quantized_shapes() of a matrix, with one scale row per 128 rows."""
    E, N, C = _dims(w, "w", 3)
    nb, cb = -(-N // 128), -(-C // 128)
    if (q_t is None) != (scales_t is None):
        raise ValueError("q_t and scales_t go together")
    S = _dims(scales, "scales of q", 3)[2]
    St = 0 if q_t is None else _dims(scales_t, "scales of q_t", 3)[2]
    dev = _device(w, "w")
    if not (_packed(w, dev, _WIDE, (E, N, C)) and
            _packed(q, dev, _E4M3, (E, N, 128 * cb)) and
            _packed(scales, dev, _BYTE, (E, nb, S)) and
            _scales_fit(scales, 128 * cb) and
            (q_t is None or
             (_packed(q_t, dev, _E4M3, (E, C, 128 * nb)) and
              _packed(scales_t, dev, _BYTE, (E, cb, St)) and
              _scales_fit(scales_t, 128 * nb)))):
        _refuse(dev, (w, "w", _WIDE, (E, N, C), _packed),
                (q, "q", _E4M3, (E, N, 128 * cb), _packed),
                (scales, "scales of q", _BYTE, (E, nb, S), _packed),
                (q_t, "q_t", _E4M3, (E, C, 128 * nb), _packed),
                (scales_t, "scales of q_t", _BYTE, (E, cb, St), _packed))
    rc = lib().ciera_quantize_blocks(
        w.data_ptr(), _WIDE[w.dtype], E, N, C, q.data_ptr(), 128 * cb,
        scales.data_ptr(), S, _ptr(q_t), 128 * nb, _ptr(scales_t), St,
        _stream(dev))
    return _check("ciera_quantize_blocks", rc)


def quantize_columns_t(x, offsets, q_t, scales_t, source=None, top_k=1):
    """Rows of experts -> 8-bit columns with a scale per 128 rows, every
    expert's rows filled up to a multiple of 128: ``q_t`` [C, L], L at least
    ciera_columns_length(). Sorted row p is row p of ``x``, or with ``source``
    row source[p] // top_k."""
    R, C = _dims(x, "x", 2)
    E = _dims(offsets, "offsets", 1)[0] - 1
    L = _dims(q_t, "q_t", 2)[1]
    S = _dims(scales_t, "scales of q_t", 2)[1]
    P = R if source is None else _dims(source, "source", 1)[0]
    dev = _device(x, "x")
    if not (_strided(x, dev, _WIDE, (R, C)) and E >= 1 and
            _packed(offsets, dev, _INT, (E + 1,)) and
            _packed(q_t, dev, _E4M3, (C, L)) and
            _packed(scales_t, dev, _BYTE, (C, S)) and
            _scales_fit(scales_t, L) and
            (source is None or _packed(source, dev, _INT, (P,)))):
        _refuse(dev, (x, "x", _WIDE, (R, C), _strided),
                (offsets, "offsets", _INT, (max(E, 1) + 1,), _packed),
                (q_t, "q_t", _E4M3, (C, L), _packed),
                (scales_t, "scales of q_t", _BYTE, (C, S), _packed),
                (source, "source", _INT, (P,), _packed))
    rc = lib().ciera_quantize_columns(
        x.data_ptr(), _WIDE[x.dtype], R, P, C, _row_stride(x, C),
        _ptr(source), top_k, offsets.data_ptr(), E, q_t.data_ptr(), L,
        scales_t.data_ptr(), S, _stream(dev))
    return _check("ciera_quantize_columns", rc)


def expert_matmul_t(a, a_scales, b, b_scales, offsets, out):
    """8-bit rows ``a`` [P, D] times the 8-bit weights ``b`` [E, N, D] of their
    experts -> ``out`` [P, N]; ``offsets`` int32 [E + 1], or None for one
    expert."""
    try:
        (P, D), (E, N, _), (_, Sa), (_, _, Sb) = (a.shape, b.shape,
                                                  a_scales.shape,
                                                  b_scales.shape)
    except ValueError:
        _refuse_dims((a, "a", 2), (b, "b", 3), (a_scales, "scales of a", 2),
                     (b_scales, "scales of b", 3))
    nb = -(-N // 128)
    dev = _device(a, "a")
    if not (_strided(a, dev, _E4M3, (P, D)) and
            _strided(a_scales, dev, _BYTE, (P, Sa)) and
            _packed(b, dev, _E4M3, (E, N, D)) and
            _packed(b_scales, dev, _BYTE, (E, nb, Sb)) and
            _scales_fit(a_scales, D) and _scales_fit(b_scales, D) and
            _strided(out, dev, _WIDE, (P, N)) and
            (offsets is None or _packed(offsets, dev, _INT, (E + 1,)))):
        _refuse(dev, (a, "a", _E4M3, (P, D), _strided),
                (a_scales, "scales of a", _BYTE, (P, Sa), _strided),
                (b, "b", _E4M3, (E, N, D), _packed),
                (b_scales, "scales of b", _BYTE, (E, nb, Sb), _packed),
                (out, "out", _WIDE, (P, N), _strided),
                (offsets, "offsets", _INT, (E + 1,), _packed))
    rc = lib().ciera_expert_matmul(
        a.data_ptr(), _row_stride(a, D), a_scales.data_ptr(),
        _row_stride(a_scales, Sa), P, b.data_ptr(), D, b_scales.data_ptr(),
        Sb, E, N, D, _ptr(offsets), out.data_ptr(), _WIDE[out.dtype],
        _row_stride(out, N), _stream(dev))
    return _check("ciera_expert_matmul", rc)


def expert_weight_grad_t(dy_t, dy_scales, x_t, x_scales, offsets, d_w):
    """The experts' weight gradients ``d_w`` [E, N, C] from the 8-bit columns
    ``dy_t`` [N, L] and ``x_t`` [C, L] of quantize_columns_t."""
    E, N, C = _dims(d_w, "d_w", 3)
    L = _dims(dy_t, "dy_t", 2)[1]
    Sy = _dims(dy_scales, "scales of dy_t", 2)[1]
    Sx = _dims(x_scales, "scales of x_t", 2)[1]
    dev = _device(dy_t, "dy_t")
    if not (_packed(dy_t, dev, _E4M3, (N, L)) and
            _packed(dy_scales, dev, _BYTE, (N, Sy)) and
            _packed(x_t, dev, _E4M3, (C, L)) and
            _packed(x_scales, dev, _BYTE, (C, Sx)) and
            _scales_fit(dy_scales, L) and _scales_fit(x_scales, L) and
            _packed(offsets, dev, _INT, (E + 1,)) and
            _packed(d_w, dev, _WIDE, (E, N, C))):
        _refuse(dev, (dy_t, "dy_t", _E4M3, (N, L), _packed),
                (dy_scales, "scales of dy_t", _BYTE, (N, Sy), _packed),
                (x_t, "x_t", _E4M3, (C, L), _packed),
                (x_scales, "scales of x_t", _BYTE, (C, Sx), _packed),
                (offsets, "offsets", _INT, (E + 1,), _packed),
                (d_w, "d_w", _WIDE, (E, N, C), _packed))
    rc = lib().ciera_expert_weight_grad(
        dy_t.data_ptr(), dy_scales.data_ptr(), Sy, x_t.data_ptr(),
        x_scales.data_ptr(), Sx, L, E, N, C, offsets.data_ptr(),
        d_w.data_ptr(), _WIDE[d_w.dtype], _stream(dev))
    return _check("ciera_expert_weight_grad", rc)


def combine_t(rows, position, out, weights=None):
    """``out`` [T, C]: for every token the sum of the rows [P, C] that
    ``position`` [T, k] names, times ``weights`` [T, k] if given."""
    try:
        (P, C), (T, k) = rows.shape, position.shape
    except ValueError:
        _refuse_dims((rows, "rows", 2), (position, "position", 2))
    dev = _device(rows, "rows")
    same = (rows.dtype,)
    if not (_strided(rows, dev, _WIDE, (P, C)) and
            _packed(position, dev, _INT, (T, k)) and
            _strided(out, dev, same, (T, C)) and
            (weights is None or _packed(weights, dev, _FLOAT, (T, k)))):
        _refuse(dev, (rows, "rows", _WIDE, (P, C), _strided),
                (position, "position", _INT, (T, k), _packed),
                (out, "out", same, (T, C), _strided),
                (weights, "weights", _FLOAT, (T, k), _packed))
    rc = lib().ciera_combine(
        rows.data_ptr(), _WIDE[rows.dtype], P, C, _row_stride(rows, C),
        _ptr(weights), position.data_ptr(), T, k, out.data_ptr(),
        _row_stride(out, C), _stream(dev))
    return _check("ciera_combine", rc)


def combine_backward_t(d_out, rows, weights, position, d_rows, d_weights):
    """Gradients of combine_t: ``d_rows`` [P, C] and ``d_weights`` [T, k]."""
    P, C = _dims(rows, "rows", 2)
    T, k = _dims(position, "position", 2)
    dev = _device(rows, "rows")
    same = (rows.dtype,)
    if not (_strided(rows, dev, _WIDE, (P, C)) and
            _packed(position, dev, _INT, (T, k)) and
            _strided(d_out, dev, same, (T, C)) and
            _packed(weights, dev, _FLOAT, (T, k)) and
            _strided(d_rows, dev, same, (P, C)) and
            _packed(d_weights, dev, _FLOAT, (T, k))):
        _refuse(dev, (rows, "rows", _WIDE, (P, C), _strided),
                (position, "position", _INT, (T, k), _packed),
                (d_out, "d_out", same, (T, C), _strided),
                (weights, "weights", _FLOAT, (T, k), _packed),
                (d_rows, "d_rows", same, (P, C), _strided),
                (d_weights, "d_weights", _FLOAT, (T, k), _packed))
    rc = lib().ciera_combine_backward(
        d_out.data_ptr(), _row_stride(d_out, C), rows.data_ptr(),
        _WIDE[rows.dtype], P, C, _row_stride(rows, C), weights.data_ptr(),
        position.data_ptr(), T, k, d_rows.data_ptr(), _row_stride(d_rows, C),
        d_weights.data_ptr(), _stream(dev))
    return _check("ciera_combine_backward", rc)
