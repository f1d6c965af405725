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


def _stream():
    """The current stream's handle. Asked for directly where torch has the call
    for it: the Stream object that torch.cuda.current_stream() builds around it
    costs 2.8 us a call, as much as a kernel launch; this takes 0.3."""
    if _raw_stream is None:
        return torch.cuda.current_stream().cuda_stream
    return _raw_stream(torch.cuda.current_device())


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
# anything is enqueued.

_WIDE = {torch.bfloat16: 0, torch.float16: 1, torch.float32: 2}
_E4M3 = (torch.float8_e4m3fn,)


def _need(ok, what):
    if not ok:
        raise ValueError(what)


# the current device's index, asked for directly as the stream is
_current_device = getattr(torch._C, "_cuda_getDevice",
                          torch.cuda.current_device)


def _arg(t, name, dtypes, shape, packed=True):
    """``t`` as an argument: on the current device, of one of ``dtypes``, of
    ``shape`` (None: any size), its last dimension contiguous (``packed``: all
    of it). Only a mistake costs the words for it."""
    m = t.shape
    if (t.is_cuda and t.get_device() == _current_device() and
            t.dtype in dtypes and len(m) == len(shape) and
            (t.is_contiguous() if packed else
             m[-1] <= 1 or t.stride(-1) == 1 or t.numel() == 0)):
        for n, have in zip(shape, m):
            if n is not None and n != have:
                break
        else:
            return
    _refuse(t, name, dtypes, shape)


def _refuse(t, name, dtypes, shape):
    _need(t.is_cuda and t.get_device() == _current_device(),
          f"{name} is on {t.device}, not on the current device")
    _need(t.dtype in dtypes, f"{name} has type {t.dtype}")
    _need(t.dim() == len(shape) and
          all(n is None or n == m for n, m in zip(shape, t.shape)),
          f"{name} has shape {tuple(t.shape)}, not "
          f"{tuple('any' if n is None else n for n in shape)}")
    raise ValueError(f"{name} is not contiguous")


def _row_stride(t, name):
    """Elements from a row of a matrix to the next."""
    rows, cols = t.shape
    if rows <= 1 or cols == 0:
        return cols or 1
    stride = t.stride(0)
    if stride < cols:
        raise ValueError(f"the rows of {name} overlap")
    return stride


_INT, _FLOAT, _BYTE = (torch.int32,), (torch.float32,), (torch.uint8,)


def _ints(t, name, *shape):
    _arg(t, name, _INT, shape)


def _floats(t, name, *shape):
    _arg(t, name, _FLOAT, shape)


def quantized_shapes(rows, cols):
    """Shapes of an 8-bit matrix of ``rows`` x ``cols`` values and of its
    scales, one a block of 128 values of a row: rows are filled up to whole
    blocks, scale rows to whole dwords."""
    blocks = -(-cols // 128)
    return (rows, 128 * blocks), (rows, -(-blocks // 4) * 4)


def _narrow(q, s, name, rows, filled, packed=True):
    """An 8-bit matrix of ``rows`` rows and its scales."""
    _arg(q, name, _E4M3, (rows, filled), packed)
    _arg(s, "scales of " + name, _BYTE, (rows, None), packed)
    if q.shape[1] % 128 or s.shape[1] < q.shape[1] // 128:
        raise ValueError(f"{name} has rows of {q.shape[1]} bytes and "
                         f"{s.shape[1]} scales")


def route_t(logits, expert_ids, weights, bias=None, groups=1, top_groups=1,
            group_top_two=False, sigmoid=False, normalize=False, scale=1.0):
    """Choose experts: ``logits`` [T, E] -> ``expert_ids`` int32 and
    ``weights`` fp32, both [T, k]; ``bias`` fp32 [E]."""
    _arg(logits, "logits", _WIDE, (None, None), packed=False)
    T, E = logits.shape
    _ints(expert_ids, "expert_ids", T, None)
    _floats(weights, "weights", T, expert_ids.shape[1])
    if bias is not None:
        _floats(bias, "bias", E)
    flags = ((ROUTE_SIGMOID if sigmoid else 0) |
             (ROUTE_NORMALIZE if normalize else 0) |
             (ROUTE_GROUP_TOP_TWO if group_top_two else 0))
    rc = ciera_route(_ptr(logits), _WIDE[logits.dtype], T, E,
                     _row_stride(logits, "logits"), _ptr(bias), groups,
                     top_groups, expert_ids.shape[1], flags, scale,
                     _ptr(expert_ids), _ptr(weights), _stream())
    return _check("ciera_route", rc)


def route_backward_t(logits, expert_ids, d_weights, d_logits, sigmoid=False,
                     normalize=False, scale=1.0):
    """Gradient of route_t's weights -> gradient of its logits."""
    _arg(logits, "logits", _WIDE, (None, None), packed=False)
    T, E = logits.shape
    _ints(expert_ids, "expert_ids", T, None)
    k = expert_ids.shape[1]
    _floats(d_weights, "d_weights", T, k)
    _arg(d_logits, "d_logits", (logits.dtype,), (T, E), packed=False)
    flags = ((ROUTE_SIGMOID if sigmoid else 0) |
             (ROUTE_NORMALIZE if normalize else 0))
    rc = ciera_route_backward(_ptr(logits), _WIDE[logits.dtype], T, E,
                              _row_stride(logits, "logits"), k, flags, scale,
                              _ptr(expert_ids), _ptr(d_weights),
                              _ptr(d_logits),
                              _row_stride(d_logits, "d_logits"), _stream())
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
    _ints(expert_ids, "expert_ids", None, None)
    T, k = expert_ids.shape
    _ints(offsets, "offsets", n_experts + 1)
    _ints(source, "source", T * k)
    _ints(position, "position", T, k)
    _arg(ws.buf, "the workspace", _BYTE, (None,))
    rc = ciera_route_plan(_ptr(expert_ids), T, k, first_expert, n_experts,
                          _ptr(offsets), _ptr(source), _ptr(position),
                          _ptr(ws.buf), ws.nbytes, _stream())
    return _check("ciera_route_plan", rc)


def quantize_rows_t(x, q, scales, position=None):
    """``x`` [R, C] -> 8-bit rows with a scale per 1 x 128 block: row r to row
    r, or with ``position`` [R, k] to the k rows that it names. ``q`` and
    ``scales`` have the shapes of quantized_shapes()."""
    _arg(x, "x", _WIDE, (None, None), packed=False)
    R, C = x.shape
    _narrow(q, scales, "q", None, -(-C // 128) * 128)
    _need(scales.shape[0] == q.shape[0], "q and its scales differ in rows")
    k = 1
    if position is not None:
        _ints(position, "position", R, None)
        k = position.shape[1]
    rc = ciera_quantize_rows(_ptr(x), _WIDE[x.dtype], R, C,
                             _row_stride(x, "x"), _ptr(position), k,
                             q.shape[0], _ptr(q), q.shape[1], _ptr(scales),
                             scales.shape[1], _stream())
    return _check("ciera_quantize_rows", rc)


def quantize_blocks_t(w, q, scales, q_t=None, scales_t=None):
    """``w`` [E, N, C] -> 8-bit with a scale per 128 x 128 block, and with
    ``q_t`` and ``scales_t`` the transpose [E, C, N] too. Shapes: those of
    quantized_shapes() of a matrix, with one scale row per 128 rows."""
    _arg(w, "w", _WIDE, (None, None, None))
    E, N, C = w.shape
    nb, cb = -(-N // 128), -(-C // 128)

    def pair(q, s, name, rows, blocks, filled):
        _arg(q, name, _E4M3, (E, rows, filled))
        _arg(s, "scales of " + name, _BYTE, (E, blocks, None))

    pair(q, scales, "q", N, nb, 128 * cb)
    _need((q_t is None) == (scales_t is None),
          "q_t and scales_t go together")
    qt_stride = st_stride = 0
    if q_t is not None:
        pair(q_t, scales_t, "q_t", C, cb, 128 * nb)
        qt_stride, st_stride = q_t.shape[2], scales_t.shape[2]
    rc = ciera_quantize_blocks(_ptr(w), _WIDE[w.dtype], E, N, C, _ptr(q),
                               q.shape[2], _ptr(scales), scales.shape[2],
                               _ptr(q_t), qt_stride, _ptr(scales_t),
                               st_stride, _stream())
    return _check("ciera_quantize_blocks", rc)


def quantize_columns_t(x, offsets, q_t, scales_t, source=None, top_k=1):
    """Rows of experts -> 8-bit columns with a scale per 128 rows, every
    expert's rows filled up to a multiple of 128: ``q_t`` [C, L], L at least
    ciera_columns_length(). Sorted row p is row p of ``x``, or with ``source``
    row source[p] // top_k."""
    _arg(x, "x", _WIDE, (None, None), packed=False)
    R, C = x.shape
    _ints(offsets, "offsets", None)
    _need(offsets.shape[0] >= 2, "offsets holds no expert")
    P = R
    if source is not None:
        _ints(source, "source", None)
        P = source.shape[0]
    _narrow(q_t, scales_t, "q_t", C, None)
    rc = ciera_quantize_columns(_ptr(x), _WIDE[x.dtype], R, P, C,
                                _row_stride(x, "x"), _ptr(source), top_k,
                                _ptr(offsets), offsets.shape[0] - 1,
                                _ptr(q_t), q_t.shape[1], _ptr(scales_t),
                                scales_t.shape[1], _stream())
    return _check("ciera_quantize_columns", rc)


def expert_matmul_t(a, a_scales, b, b_scales, offsets, out):
    """8-bit rows ``a`` [P, D] times the 8-bit weights ``b`` [E, N, D] of their
    experts -> ``out`` [P, N]; ``offsets`` int32 [E + 1], or None for one
    expert."""
    _narrow(a, a_scales, "a", None, None, packed=False)
    P, D = a.shape
    _need(a_scales.shape[0] == P, "a and its scales differ in rows")
    _arg(b, "b", _E4M3, (None, None, D))
    E, N, _ = b.shape
    _arg(b_scales, "scales of b", _BYTE, (E, -(-N // 128), None))
    _arg(out, "out", _WIDE, (P, N), packed=False)
    if offsets is not None:
        _ints(offsets, "offsets", E + 1)
    rc = ciera_expert_matmul(_ptr(a), _row_stride(a, "a"), _ptr(a_scales),
                             _row_stride(a_scales, "scales of a"), P, _ptr(b),
                             D, _ptr(b_scales), b_scales.shape[2], E, N, D,
                             _ptr(offsets), _ptr(out), _WIDE[out.dtype],
                             _row_stride(out, "out"), _stream())
    return _check("ciera_expert_matmul", rc)


def expert_weight_grad_t(dy_t, dy_scales, x_t, x_scales, offsets, d_w):
    """The experts' weight gradients ``d_w`` [E, N, C] from the 8-bit columns
    ``dy_t`` [N, L] and ``x_t`` [C, L] of quantize_columns_t."""
    _arg(d_w, "d_w", _WIDE, (None, None, None))
    E, N, C = d_w.shape
    _narrow(dy_t, dy_scales, "dy_t", N, None)
    L = dy_t.shape[1]
    _narrow(x_t, x_scales, "x_t", C, L)
    _ints(offsets, "offsets", E + 1)
    rc = ciera_expert_weight_grad(_ptr(dy_t), _ptr(dy_scales),
                                  dy_scales.shape[1], _ptr(x_t),
                                  _ptr(x_scales), x_scales.shape[1], L, E, N,
                                  C, _ptr(offsets), _ptr(d_w),
                                  _WIDE[d_w.dtype], _stream())
    return _check("ciera_expert_weight_grad", rc)


def combine_t(rows, position, out, weights=None):
    """``out`` [T, C]: for every token the sum of the rows [P, C] that
    ``position`` [T, k] names, times ``weights`` [T, k] if given."""
    _arg(rows, "rows", _WIDE, (None, None), packed=False)
    P, C = rows.shape
    _ints(position, "position", None, None)
    T, k = position.shape
    _arg(out, "out", (rows.dtype,), (T, C), packed=False)
    if weights is not None:
        _floats(weights, "weights", T, k)
    rc = ciera_combine(_ptr(rows), _WIDE[rows.dtype], P, C,
                       _row_stride(rows, "rows"), _ptr(weights),
                       _ptr(position), T, k, _ptr(out),
                       _row_stride(out, "out"), _stream())
    return _check("ciera_combine", rc)


def combine_backward_t(d_out, rows, weights, position, d_rows, d_weights):
    """Gradients of combine_t: ``d_rows`` [P, C] and ``d_weights`` [T, k]."""
    _arg(rows, "rows", _WIDE, (None, None), packed=False)
    P, C = rows.shape
    _ints(position, "position", None, None)
    T, k = position.shape
    _arg(d_out, "d_out", (rows.dtype,), (T, C), packed=False)
    _floats(weights, "weights", T, k)
    _arg(d_rows, "d_rows", (rows.dtype,), (P, C), packed=False)
    _floats(d_weights, "d_weights", T, k)
    rc = ciera_combine_backward(
        _ptr(d_out), _row_stride(d_out, "d_out"), _ptr(rows),
        _WIDE[rows.dtype], P, C, _row_stride(rows, "rows"), _ptr(weights),
        _ptr(position), T, k, _ptr(d_rows), _row_stride(d_rows, "d_rows"),
        _ptr(d_weights), _stream())
    return _check("ciera_combine_backward", rc)
