"""ctypes binding of ``include/pallas.h``.

Argument marshalling only: torch tensors become device pointers, Python
lists become host arrays, the current torch stream becomes the hipStream_t.
Every step of the computation runs in the HIP library.
"""
from __future__ import annotations

import ctypes as C
import enum
import os
from typing import List, Optional, Sequence

PKG = os.path.dirname(os.path.abspath(__file__))


def library_path() -> str:
    return os.path.join(PKG, "libpallas.so")


class Status(enum.IntEnum):
    OK = 0
    INVALID_ARG = 1
    OUT_OF_RANGE = 2
    COVERAGE = 3
    STALE_EPOCH = 4
    WRONG_REQUEST = 5
    UNSUPPORTED = 6
    HIP = 7
    WORKSPACE = 8


class PallasError(RuntimeError):
    def __init__(self, status: int, msg: str):
        self.status = Status(status)
        super().__init__(f"{self.status.name}: {msg}")


# ------------------------------------------------------------------ structs
class ModelConfigC(C.Structure):
    _fields_ = [("n_layers", C.c_int32), ("hidden", C.c_int32), ("n_q_heads", C.c_int32),
                ("n_kv_heads", C.c_int32), ("head_dim", C.c_int32), ("ffn", C.c_int32),
                ("vocab", C.c_int32), ("rms_eps", C.c_float), ("rope_theta", C.c_float),
                ("qk_norm", C.c_int32), ("page_size", C.c_int32)]


class LayerWeightsC(C.Structure):
    _fields_ = [(n, C.c_void_p) for n in ("attn_norm", "w_qkv", "q_norm", "k_norm", "w_o",
                                          "mlp_norm", "w_gate_up", "w_down")]


class WeightsC(C.Structure):
    _fields_ = [("embed", C.c_void_p), ("final_norm", C.c_void_p), ("lm_head", C.c_void_p),
                ("layers", C.POINTER(LayerWeightsC))]


class KVPoolC(C.Structure):
    _fields_ = [("base", C.c_void_p), ("num_pages", C.c_int32), ("page_size", C.c_int32),
                ("n_layers", C.c_int32), ("n_kv_heads", C.c_int32), ("head_dim", C.c_int32)]


class ChunkDesc(C.Structure):
    _fields_ = [("start_pos", C.c_int32), ("num_tokens", C.c_int32), ("arena_offset", C.c_uint64)]


class ChunkHeader(C.Structure):
    _fields_ = [("request_id", C.c_uint64), ("epoch", C.c_uint64), ("start_pos", C.c_int32),
                ("num_tokens", C.c_int32), ("arena_offset", C.c_uint64), ("n_layers", C.c_int32),
                ("n_kv_heads", C.c_int32), ("head_dim", C.c_int32), ("elem_bytes", C.c_int32)]


class WindowParams(C.Structure):
    _fields_ = [(n, C.c_double) for n in ("r_p", "r_d", "goodput", "s_kv", "t_load", "t_0", "alpha",
                                          "t_max", "dt")]


class WindowDecision(C.Structure):
    _fields_ = [(n, C.c_double) for n in ("t_w", "cost", "t_sit", "t_early", "t_hist", "t_res",
                                          "l_hist")] + [("n_candidates", C.c_int32), ("trigger", C.c_int32)]


class Ewma(C.Structure):
    _fields_ = [("value", C.c_double), ("primed", C.c_int32)]


ROPE_LAYOUTS = ("half", "interleaved")
ROPE_SCALINGS = ("none", "linear", "ntk", "yarn", "bands")
ROPE_MAX_DIM = 256


class RopeConfigC(C.Structure):
    _fields_ = [("rotary_dim", C.c_int32), ("layout", C.c_int32), ("scaling", C.c_int32), ("trained_len", C.c_int32),
                ("theta", C.c_double), ("factor", C.c_double), ("fast", C.c_double), ("slow", C.c_double),
                ("magnitude", C.c_double)]


class RopePlan(C.Structure):
    _fields_ = [("rotary_dim", C.c_int32), ("layout", C.c_int32), ("magnitude", C.c_float), ("reserved", C.c_int32),
                ("turns", C.c_uint64 * (ROPE_MAX_DIM // 2))]


class QuantPoolC(C.Structure):
    _fields_ = [("codes", C.c_void_p), ("scales", C.c_void_p), ("num_pages", C.c_int32), ("page_size", C.c_int32),
                ("n_layers", C.c_int32), ("n_kv_heads", C.c_int32), ("head_dim", C.c_int32), ("format", C.c_int32)]


class BoundsPoolC(C.Structure):
    _fields_ = [("codes", C.c_void_p), ("scales", C.c_void_p), ("num_pages", C.c_int32), ("n_layers", C.c_int32),
                ("n_kv_heads", C.c_int32), ("head_dim", C.c_int32)]


_vp, _i32, _u64, _sz = C.c_void_p, C.c_int32, C.c_uint64, C.c_size_t
_i64 = C.c_int64
_pi32 = C.POINTER(C.c_int32)

# name -> (restype, argtypes); mirrors include/pallas.h
EXPORTS = {
    "pallas_abi_version": (_i32, []),
    "pallas_last_error": (C.c_char_p, []),
    "pallas_model_create": (C.c_int, [C.POINTER(ModelConfigC), C.POINTER(WeightsC), C.POINTER(_vp)]),
    "pallas_model_destroy": (None, [_vp]),
    "pallas_workspace_size": (_sz, [_vp, _i32, _i32]),
    "pallas_prefill_prefix": (C.c_int, [_vp, _i32, _vp, _pi32, _vp, _i32, C.POINTER(KVPoolC),
                                        _vp, _sz, _vp, _vp]),
    "pallas_prefill_chunk": (C.c_int, [_vp, _i32, _vp, _pi32, _pi32, _vp, _i32, C.POINTER(KVPoolC),
                                       _vp, _sz, _vp, _vp]),
    "pallas_pack_suffix_blocks": (C.c_int, [C.POINTER(KVPoolC), _vp, _i32, C.POINTER(ChunkDesc),
                                            _i32, _vp, _sz, _vp, _vp]),
    "pallas_assemble_kv": (C.c_int, [C.POINTER(KVPoolC), _vp, _i32, C.POINTER(ChunkHeader), _vp,
                                     _sz, _i32, _u64, _u64, _vp, _vp]),
    "pallas_decode_step": (C.c_int, [_vp, _i32, _vp, _pi32, _vp, _i32, C.POINTER(KVPoolC), _vp,
                                     _vp, _sz, _vp, _vp]),
    "pallas_decode_step_static": (C.c_int, [_vp, _i32, _vp, _pi32, _vp, _i32, C.POINTER(KVPoolC), _vp,
                                            _vp, _vp]),
    "pallas_rope_init": (C.c_int, [C.POINTER(RopeConfigC), C.POINTER(RopePlan)]),
    "pallas_rope_apply": (C.c_int, [C.POINTER(RopePlan), _i32, _i32, _i32, _i32, _vp, _vp, _i64, _i64, _vp, _i64,
                                    _i64, _vp]),
    "pallas_quant_store": (C.c_int, [C.POINTER(QuantPoolC), _i32, _i32, _vp, _vp, _vp, _i64, _vp, _i64, _i32, _vp,
                                     _i32, _vp, _vp]),
    "pallas_quant_load": (C.c_int, [C.POINTER(QuantPoolC), _i32, _i32, _vp, _vp, _vp, _i64, _vp, _i64, _i32, _vp,
                                    _i32, _vp, _vp]),
    "pallas_append_kv": (C.c_int, [C.POINTER(RopePlan), C.POINTER(KVPoolC), _i32, _i32, _vp, _vp, _i32, _vp, _i64, _vp, _i64,
                                   _vp, _i64, _vp, _i64, _i32, _vp, _i32, _vp, _vp]),
    "pallas_append_quant": (C.c_int, [C.POINTER(RopePlan), C.POINTER(QuantPoolC), _i32, _i32, _vp, _vp, _i32, _vp, _i64, _vp,
                                      _i64, _vp, _i64, _vp, _i64, _i32, _vp, _i32, _vp, _vp]),
    "pallas_attend_kv": (C.c_int, [C.POINTER(KVPoolC), _i32, _i32, _i32, _vp, _i64, _vp, _i32, _vp, _i32, C.c_float,
                                   _vp, _i64, _vp, _vp, _sz, _vp, _vp]),
    "pallas_attend_quant": (C.c_int, [C.POINTER(QuantPoolC), _i32, _i32, _i32, _vp, _i64, _vp, _i32, _vp, _i32,
                                      C.c_float, _vp, _i64, _vp, _vp, _sz, _vp, _vp]),
    "pallas_attend_workspace_size": (_sz, [_i32, _i32, _i32, _i32, _i32]),
    "pallas_bounds_kv": (C.c_int, [C.POINTER(KVPoolC), C.POINTER(BoundsPoolC), _i32, _i32, _vp, _vp, _i32, _vp, _i32, _vp,
                                   _vp]),
    "pallas_bounds_quant": (C.c_int, [C.POINTER(QuantPoolC), C.POINTER(BoundsPoolC), _i32, _i32, _vp, _vp, _i32, _vp, _i32,
                                      _vp, _vp]),
    "pallas_select_blocks": (C.c_int, [C.POINTER(BoundsPoolC), _i32, _i32, _i32, _vp, _i64, _vp, _i32, _vp, _i32, _i32, _i32,
                                       _i32, _vp, _vp, _sz, _vp, _vp]),
    "pallas_select_workspace_size": (_sz, [_i32, _i32, _i32]),
    "pallas_attend_blocks_kv": (C.c_int, [C.POINTER(KVPoolC), _i32, _i32, _i32, _vp, _i64, _vp, _i32, _vp, _i32, _vp, _i32,
                                          C.c_float, _vp, _i64, _vp, _vp, _sz, _vp, _vp]),
    "pallas_attend_blocks_quant": (C.c_int, [C.POINTER(QuantPoolC), _i32, _i32, _i32, _vp, _i64, _vp, _i32, _vp, _i32, _vp,
                                             _i32, C.c_float, _vp, _i64, _vp, _vp, _sz, _vp, _vp]),
    "pallas_check_coverage": (C.c_int, [_i32, _pi32, _pi32, _i32, _i32]),
    "pallas_window_evaluate": (C.c_int, [C.POINTER(WindowParams), C.c_double, C.c_double, C.c_double,
                                         C.POINTER(WindowDecision)]),
    "pallas_window_select": (C.c_int, [C.POINTER(WindowParams), C.c_double, C.c_double,
                                       C.POINTER(WindowDecision)]),
    "pallas_ewma_update": (C.c_double, [C.POINTER(Ewma), C.c_double, C.c_double]),
    "pallas_admit": (_i32, [_i32, C.c_double, C.c_double, C.c_double, C.c_double, C.c_double]),
    "pallas_waste_bound": (C.c_double, [C.c_double, C.c_double, C.c_double]),
    "pallas_profile_enable": (None, [C.c_uint32]),
    "pallas_profile_read": (C.c_int, [C.POINTER(C.c_double), C.POINTER(C.c_int64)]),
    "pallas_profile_reset": (None, []),
    "pallas_profile_clock": (C.c_int, [_i32, C.POINTER(C.c_double), C.POINTER(C.c_int64)]),
}

KERNEL_CLASSES = ("embed", "rmsnorm", "rope_table", "gemm_qkv", "qkv_epilogue", "attention",
                  "gemm_o", "gemm_gate_up", "gemm_down", "pack", "assemble", "decode_proj",
                  "decode_attention")

_LIB = None


def lib():
    """The loaded library; raises if it has not been built."""
    global _LIB
    if _LIB is None:
        path = library_path()
        if not os.path.exists(path):
            raise RuntimeError(f"{path} is missing: build it with `python -m "
                               "paper_2608_16477_amd.build` (there is no fallback path)")
        h = C.CDLL(path)
        for name, (res, args) in EXPORTS.items():
            f = getattr(h, name)
            f.restype = res
            f.argtypes = args
        _LIB = h
    return _LIB


def _ptr(t) -> Optional[int]:
    return None if t is None else t.data_ptr()


def _stream(stream) -> Optional[int]:
    if stream is None:
        import torch
        return torch.cuda.current_stream().cuda_stream
    if isinstance(stream, int):
        return stream
    return stream.cuda_stream


def _i32_array(vals: Sequence[int]):
    arr = (C.c_int32 * max(1, len(vals)))(*[int(v) for v in vals])
    return arr


def _check(rc: int):
    if rc != 0:
        raise PallasError(rc, pallas_last_error())


def pallas_abi_version() -> int:
    return lib().pallas_abi_version()


def pallas_last_error() -> str:
    return lib().pallas_last_error().decode()


def pallas_check_coverage(prefix_len: int, starts: Sequence[int], lens: Sequence[int], n: int) -> Status:
    """Returns the status (OK or COVERAGE / INVALID_ARG); does not raise."""
    return Status(lib().pallas_check_coverage(prefix_len, _i32_array(starts), _i32_array(lens),
                                              len(starts), n))


def kv_pool_struct(pool) -> KVPoolC:
    """``pool``: bf16 tensor [L, 2, P, page, Hkv, d]."""
    L, two, P, page, hkv, d = pool.shape
    assert two == 2
    return KVPoolC(pool.data_ptr(), P, page, L, hkv, d)


def pallas_pack_suffix_blocks(pool, src_block_table, descs: Sequence[ChunkDesc], arena,
                              err=None, stream=None):
    arr = (ChunkDesc * max(1, len(descs)))(*descs)
    ps = kv_pool_struct(pool)
    _check(lib().pallas_pack_suffix_blocks(C.byref(ps), _ptr(src_block_table),
                                           src_block_table.shape[-1], arr, len(descs),
                                           _ptr(arena), arena.numel() * arena.element_size(),
                                           _ptr(err), _stream(stream)))


def pallas_assemble_kv(pool, dst_block_table, hdrs: Sequence[ChunkHeader], arena,
                       expected_request_id: int, expected_epoch: int, err=None, stream=None):
    arr = (ChunkHeader * max(1, len(hdrs)))(*hdrs)
    ps = kv_pool_struct(pool)
    nbytes = 0 if arena is None else arena.numel() * arena.element_size()
    _check(lib().pallas_assemble_kv(C.byref(ps), _ptr(dst_block_table), dst_block_table.shape[-1],
                                    arr, _ptr(arena), nbytes, len(hdrs), expected_request_id,
                                    expected_epoch, _ptr(err), _stream(stream)))


def pallas_model_create(cfg, glob, layers):
    """Returns ``(handle, keepalive)``; ``glob``/``layers`` are dicts of bf16
    device tensors named as in ``pallas_layer_weights`` / ``pallas_weights``."""
    c = ModelConfigC(cfg.n_layers, cfg.hidden, cfg.n_q_heads, cfg.n_kv_heads, cfg.head_dim,
                     cfg.ffn, cfg.vocab, cfg.rms_eps, cfg.rope_theta, int(bool(cfg.qk_norm)),
                     cfg.page_size)
    la = (LayerWeightsC * cfg.n_layers)()
    for i, l in enumerate(layers):
        for name, _ in LayerWeightsC._fields_:
            setattr(la[i], name, l[name].data_ptr())
    w = WeightsC(glob["embed"].data_ptr(), glob["final_norm"].data_ptr(),
                 glob["lm_head"].data_ptr(), la)
    h = C.c_void_p()
    _check(lib().pallas_model_create(C.byref(c), C.byref(w), C.byref(h)))
    return h


def pallas_model_destroy(h):
    lib().pallas_model_destroy(h)


def pallas_workspace_size(h, max_tokens: int, max_seqs: int) -> int:
    return int(lib().pallas_workspace_size(h, max_tokens, max_seqs))


def pallas_prefill_prefix(h, token_ids, cu_seqlens: Sequence[int], block_tables, pool,
                          workspace, err=None, stream=None):
    ps = kv_pool_struct(pool)
    _check(lib().pallas_prefill_prefix(h, len(cu_seqlens) - 1, _ptr(token_ids),
                                       _i32_array(cu_seqlens), _ptr(block_tables),
                                       block_tables.shape[-1], C.byref(ps), _ptr(workspace),
                                       workspace.numel() * workspace.element_size(), _ptr(err),
                                       _stream(stream)))


def pallas_prefill_chunk(h, token_ids, cu_seqlens: Sequence[int], start_pos: Sequence[int],
                         block_tables, pool, workspace, err=None, stream=None):
    assert len(start_pos) == len(cu_seqlens) - 1
    ps = kv_pool_struct(pool)
    _check(lib().pallas_prefill_chunk(h, len(cu_seqlens) - 1, _ptr(token_ids),
                                      _i32_array(cu_seqlens), _i32_array(start_pos),
                                      _ptr(block_tables), block_tables.shape[-1], C.byref(ps),
                                      _ptr(workspace), workspace.numel() * workspace.element_size(),
                                      _ptr(err), _stream(stream)))


def pallas_decode_step(h, tokens, positions: Sequence[int], block_tables, pool, logits,
                       workspace, err=None, stream=None):
    ps = kv_pool_struct(pool)
    _check(lib().pallas_decode_step(h, len(positions), _ptr(tokens), _i32_array(positions),
                                    _ptr(block_tables), block_tables.shape[-1], C.byref(ps),
                                    _ptr(logits), _ptr(workspace),
                                    workspace.numel() * workspace.element_size(), _ptr(err),
                                    _stream(stream)))


def pallas_decode_step_static(h, tokens, positions: Sequence[int], block_tables, pool, logits,
                              err=None, stream=None):
    """pallas_decode_step with the library's static scratch (no workspace)."""
    ps = kv_pool_struct(pool)
    _check(lib().pallas_decode_step_static(h, len(positions), _ptr(tokens), _i32_array(positions),
                                           _ptr(block_tables), block_tables.shape[-1], C.byref(ps),
                                           _ptr(logits), _ptr(err), _stream(stream)))


# ------------------------------------------------------------ cache operators
# These check what they are given (type, rank, strides, device), as the library sees
# addresses alone.  A call's checks cost as much as its launch where tensors are asked
# more than needed, so each is asked once: shape and stride as tuples, the device as an
# index (-1: host).
_torch = None
_formats = None


def _load_torch():
    global _torch
    import torch
    _torch = torch
    return torch


def _bad(msg: str):
    raise PallasError(Status.INVALID_ARG, msg)


def _refuse(t, what: str, dtype, ndim: int, dev: int):
    _bad(f"{what}: {t.dtype} {tuple(t.shape)}, strides {t.stride()}, on {t.device}; wanted {dtype} of rank {ndim} on "
         f"{'GPU ' + str(dev) if dev >= 0 else 'a GPU'}, contiguous (in its last dimension at least)")


def _whole(t, what: str, dtype, ndim: int, dev: int):
    """The shape of a contiguous tensor of this type and rank on GPU ``dev``."""
    shape = t.shape
    if t.dtype is not dtype or len(shape) != ndim or t.get_device() != dev or dev < 0 or not t.is_contiguous():
        _refuse(t, what, dtype, ndim, dev)
    return shape


def _rows(t, what: str, dev: int):
    """Shape and strides of bf16 rows [tokens, heads, d] whose d elements are contiguous."""
    shape, stride = t.shape, t.stride()
    if t.dtype is not (_torch or _load_torch()).bfloat16 or len(shape) != 3 or t.get_device() != dev or dev < 0 or (
            stride[2] != 1 and shape[2] > 1):
        _refuse(t, what, "bfloat16", 3, dev)
    return shape, stride


def _packed_rows(t, what: str, dev: int, shape):
    """The row stride of rows of this shape with their heads one behind the other."""
    if t.is_contiguous() and t.shape == shape and len(shape) == 3 and t.get_device() == dev >= 0 and (
            t.dtype is (_torch or _load_torch()).bfloat16):
        return shape[1] * shape[2]
    got, stride = _rows(t, what, dev)
    if got != shape or (stride[1] != shape[2] and shape[1] > 1):
        _bad(f"{what}: {tuple(got)}, strides {stride}; wanted {tuple(shape)}, its heads contiguous")
    return stride[0] if shape[0] > 1 else shape[1] * shape[2]     # (the stride of a single row says nothing)


def _launch(dev: int, stream, call, *args):
    """``call(*args, stream)`` with the tensors' GPU current, on its current stream unless one is given."""
    # (The raw handle: a torch.cuda.Stream object costs 1 us of a call's 9.)
    handle = _torch._C._cuda_getCurrentRawStream(dev) if stream is None else _stream(stream)
    if _torch._C._cuda_getDevice() == dev:
        rc = call(*args, handle)
    else:
        with _torch.cuda.device(dev):
            rc = call(*args, handle)
    if rc:
        _check(rc)


def pallas_rope_init(rotary_dim: int, theta: float, layout: str = "half", scaling: str = "none", factor: float = 1.0,
                     trained_len: int = 0, fast: float = 0.0, slow: float = 0.0, magnitude: float = 0.0) -> RopePlan:
    """The plan of a rotary embedding: ``layout`` of ROPE_LAYOUTS, ``scaling`` of ROPE_SCALINGS."""
    if layout not in ROPE_LAYOUTS or scaling not in ROPE_SCALINGS:
        _bad(f"rope: layout {layout!r}, scaling {scaling!r}")
    cfg = RopeConfigC(rotary_dim, ROPE_LAYOUTS.index(layout), ROPE_SCALINGS.index(scaling), trained_len, theta, factor,
                      fast, slow, magnitude)
    plan = RopePlan()
    _check(lib().pallas_rope_init(C.byref(cfg), C.byref(plan)))
    return plan


def pallas_rope_apply(plan: RopePlan, x, positions, out=None, inverse: bool = False, stream=None):
    """``x``, ``out``: bf16 [tokens, heads, head_dim] of any token and head strides; in place without ``out``."""
    torch = _torch or _load_torch()
    dev = x.get_device()
    shape, xs = _rows(x, "rope: x", dev)
    if out is None:
        out, ys = x, xs
    else:
        to, ys = _rows(out, "rope: out", dev)
        if to != shape:
            _bad(f"rope: {tuple(shape)} to {tuple(to)}")
    T, H, d = shape
    if _whole(positions, "rope: positions", torch.int32, 1, dev)[0] != T:
        _bad(f"rope: {positions.shape[0]} positions of {T} tokens")
    if T and H:
        _launch(dev, stream, lib().pallas_rope_apply, C.byref(plan), 1 if inverse else 0, T, H, d, positions.data_ptr(),
                x.data_ptr(), xs[0], xs[1], out.data_ptr(), ys[0], ys[1])
    return out


def _quant_formats():
    torch = _torch or _load_torch()
    # dtype of the codes -> format, codes to a value of the tensor, the scales' dtype and rank
    formats = {torch.float8_e4m3fn: (1, 1, torch.float32, 5), torch.int8: (2, 1, torch.float32, 5)}
    packed, units = getattr(torch, "float4_e2m1fn_x2", None), getattr(torch, "float8_e8m0fnu", None)
    if packed is not None and units is not None:      # (a torch without them has the 8-bit pools)
        formats[packed] = 4, 2, units, 6
    return formats


def quant_pool_struct(codes, scales) -> QuantPoolC:
    """``codes``: float8_e4m3fn or int8 [L, 2, P, page, Hkv, d] with ``scales`` float32 [L, 2, P, page, Hkv], or
    float4_e2m1fn_x2 [L, 2, P, page, Hkv, d / 2] with float8_e8m0fnu [L, 2, P, page, Hkv, 4]."""
    global _formats
    if _formats is None:
        _formats = _quant_formats()
    dtype, dev = codes.dtype, codes.get_device()
    kind = _formats.get(dtype)
    if kind is None:
        _bad(f"quant pool: codes of {dtype}, wanted float8_e4m3fn, int8 or float4_e2m1fn_x2")
    fmt, per, of, rank = kind
    L, two, P, page, hkv, d = shape = _whole(codes, "quant pool: codes", dtype, 6, dev)
    of_rows = (L, 2, P, page, hkv) if rank == 5 else (L, 2, P, page, hkv, 4)
    if two != 2 or _whole(scales, "quant pool: scales", of, rank, dev) != of_rows:
        _bad(f"quant pool: codes {tuple(shape)}, scales {tuple(scales.shape)}")
    return QuantPoolC(codes.data_ptr(), scales.data_ptr(), P, page, L, hkv, d * per, fmt)


def _quant_call(what, call, codes, scales, layer, k, v, positions, block_tables, seq_ids, err, stream):
    ps = quant_pool_struct(codes, scales)
    i32, dev = _torch.int32, codes.get_device()
    T, = n = _whole(positions, what + ": positions", i32, 1, dev)
    shape = (T, ps.n_kv_heads, ps.head_dim)
    ks, vs = _packed_rows(k, what + ": k", dev, shape), _packed_rows(v, what + ": v", dev, shape)
    seqs, pages = _whole(block_tables, what + ": block tables", i32, 2, dev)
    if seq_ids is not None and _whole(seq_ids, what + ": sequence ids", i32, 1, dev) != n:
        _bad(f"{what}: {seq_ids.shape[0]} sequence ids of {T} tokens")
    if err is not None and not _whole(err, what + ": err", i32, 1, dev)[0]:
        _bad(f"{what}: an empty err")
    if T:
        _launch(dev, stream, call, C.byref(ps), layer, T, _ptr(seq_ids), positions.data_ptr(), k.data_ptr(), ks,
                v.data_ptr(), vs, seqs, block_tables.data_ptr(), pages, _ptr(err))


def pallas_quant_store(codes, scales, layer: int, k, v, positions, block_tables, seq_ids=None, err=None, stream=None):
    """Quantises ``k``, ``v`` (bf16 [tokens, Hkv, d], any token stride) into a layer of the pool (quant_pool_struct)."""
    _quant_call("quant store", lib().pallas_quant_store, codes, scales, layer, k, v, positions, block_tables, seq_ids,
                err, stream)


def pallas_quant_load(codes, scales, layer: int, k, v, positions, block_tables, seq_ids=None, err=None, stream=None):
    """Reads rows of a layer back into ``k``, ``v`` (bf16 [tokens, Hkv, d], any token stride)."""
    _quant_call("quant load", lib().pallas_quant_load, codes, scales, layer, k, v, positions, block_tables, seq_ids, err,
                stream)


def _append_call(call, plan, ps, dev, layer, k, v, positions, block_tables, q, q_out, seq_ids, err, stream):
    i32 = _torch.int32
    T, = n = _whole(positions, "append: positions", i32, 1, dev)
    shape = (T, ps.n_kv_heads, ps.head_dim)
    ks, vs = _packed_rows(k, "append: k", dev, shape), _packed_rows(v, "append: v", dev, shape)
    heads, qp, qs, op, os_ = 0, None, 0, None, 0
    if q is not None:
        q_shape = q.shape
        qs = _packed_rows(q, "append: q", dev, q_shape)
        out = q if q_out is None else q_out
        os_ = qs if q_out is None else _packed_rows(out, "append: q_out", dev, q_shape)
        if q_shape[0] != T or q_shape[2] != ps.head_dim:
            _bad(f"append: {tuple(q_shape)} queries of {T} tokens, a pool of head_dim {ps.head_dim}")
        heads, qp, op = q_shape[1], q.data_ptr(), out.data_ptr()
    elif q_out is not None:
        _bad("append: q_out without q")
    seqs, pages = _whole(block_tables, "append: block tables", i32, 2, dev)
    if seq_ids is not None and _whole(seq_ids, "append: sequence ids", i32, 1, dev) != n:
        _bad(f"append: {seq_ids.shape[0]} sequence ids of {T} tokens")
    if err is not None and not _whole(err, "append: err", i32, 1, dev)[0]:
        _bad("append: an empty err")
    if T:
        _launch(dev, stream, call, C.byref(plan), C.byref(ps), layer, T, _ptr(seq_ids), positions.data_ptr(), heads, qp, qs,
                op, os_, k.data_ptr(), ks, v.data_ptr(), vs, seqs, block_tables.data_ptr(), pages, _ptr(err))


def pallas_append_kv(plan: RopePlan, pool, layer: int, k, v, positions, block_tables, q=None, q_out=None, seq_ids=None,
                     err=None, stream=None):
    """Rotates ``k`` and ``q`` and stores ``k``, ``v`` (bf16 [tokens, Hkv, d], any token stride) into a layer of a bf16
    pool; ``q`` (bf16 [tokens, Hq, d]) goes to ``q_out``, or in place without it."""
    dev = pool.get_device()
    _whole(pool, "append: pool", (_torch or _load_torch()).bfloat16, 6, dev)
    _append_call(lib().pallas_append_kv, plan, kv_pool_struct(pool), dev, layer, k, v, positions, block_tables, q, q_out,
                 seq_ids, err, stream)


def pallas_append_quant(plan: RopePlan, codes, scales, layer: int, k, v, positions, block_tables, q=None, q_out=None,
                        seq_ids=None, err=None, stream=None):
    """The same into an 8- or 4-bit pool (quant_pool_struct)."""
    _append_call(lib().pallas_append_quant, plan, quant_pool_struct(codes, scales), codes.get_device(), layer, k, v,
                 positions, block_tables, q, q_out, seq_ids, err, stream)


def pallas_attend_workspace_size(num_seqs: int, n_q_heads: int, n_kv_heads: int, head_dim: int, max_length: int) -> int:
    return int(lib().pallas_attend_workspace_size(num_seqs, n_q_heads, n_kv_heads, head_dim, max_length))


def _attend_call(call, ps, dev, layer, q, lengths, max_length, block_tables, scale, out, workspace, lse, err, stream,
                 blocks=None):
    i32, shape = _torch.int32, q.shape
    qs, os_ = _packed_rows(q, "attend: q", dev, shape), _packed_rows(out, "attend: out", dev, shape)
    S, H, d = shape
    seqs, pages = _whole(block_tables, "attend: block tables", i32, 2, dev)
    if d != ps.head_dim or seqs != S or _whole(lengths, "attend: lengths", i32, 1, dev)[0] != S:
        _bad(f"attend: {tuple(shape)} queries, {lengths.shape[0]} lengths, {seqs} tables, a pool of head_dim {ps.head_dim}")
    if lse is not None and _whole(lse, "attend: lse", _torch.float32, 2, dev) != (S, H):
        _bad(f"attend: lse {tuple(lse.shape)}")
    if err is not None and not _whole(err, "attend: err", i32, 1, dev)[0]:
        _bad("attend: an empty err")
    if workspace.get_device() != dev or not workspace.is_contiguous():
        _bad("attend: workspace on another device, or not contiguous")
    lists = ()
    if blocks is not None:
        got = _whole(blocks, "attend: blocks", i32, 3, dev)
        if got != (S, ps.n_kv_heads, got[2]):
            _bad(f"attend: blocks {tuple(got)} of {S} sequences and {ps.n_kv_heads} KV heads")
        lists = (blocks.data_ptr(), got[2])
    if S:
        _launch(dev, stream, call, C.byref(ps), layer, S, H, q.data_ptr(), qs, lengths.data_ptr(), max_length,
                block_tables.data_ptr(), pages, *lists, scale, out.data_ptr(), os_, _ptr(lse), workspace.data_ptr(),
                workspace.nbytes, _ptr(err))


def pallas_attend_kv(pool, layer: int, q, lengths, max_length: int, block_tables, scale: float, out, workspace, lse=None,
                     err=None, stream=None):
    """One new token per sequence: ``q``, ``out`` bf16 [num_seqs, Hq, d] (any row stride) over a bf16 pool.  As with
    the other operators nothing is enqueued for an empty batch."""
    dev = pool.get_device()
    _whole(pool, "attend: pool", (_torch or _load_torch()).bfloat16, 6, dev)
    _attend_call(lib().pallas_attend_kv, kv_pool_struct(pool), dev, layer, q, lengths, max_length, block_tables, scale, out,
                 workspace, lse, err, stream)


def pallas_attend_quant(codes, scales, layer: int, q, lengths, max_length: int, block_tables, scale: float, out,
                        workspace, lse=None, err=None, stream=None):
    """The same over an 8- or 4-bit pool (quant_pool_struct)."""
    _attend_call(lib().pallas_attend_quant, quant_pool_struct(codes, scales), codes.get_device(), layer, q, lengths,
                 max_length, block_tables, scale, out, workspace, lse, err, stream)


def pallas_attend_blocks_kv(pool, layer: int, q, lengths, max_length: int, block_tables, blocks, scale: float, out,
                            workspace, lse=None, err=None, stream=None):
    """pallas_attend_kv over the blocks that ``blocks`` (int32 [num_seqs, Hkv, max_blocks]) lists for each KV head."""
    dev = pool.get_device()
    _whole(pool, "attend: pool", (_torch or _load_torch()).bfloat16, 6, dev)
    if blocks is None:
        _bad("attend: no blocks")
    _attend_call(lib().pallas_attend_blocks_kv, kv_pool_struct(pool), dev, layer, q, lengths, max_length, block_tables,
                 scale, out, workspace, lse, err, stream, blocks)


def pallas_attend_blocks_quant(codes, scales, layer: int, q, lengths, max_length: int, block_tables, blocks, scale: float,
                               out, workspace, lse=None, err=None, stream=None):
    """The same over an 8- or 4-bit pool (quant_pool_struct)."""
    if blocks is None:
        _bad("attend: no blocks")
    _attend_call(lib().pallas_attend_blocks_quant, quant_pool_struct(codes, scales), codes.get_device(), layer, q, lengths,
                 max_length, block_tables, scale, out, workspace, lse, err, stream, blocks)


def bounds_pool_struct(bounds, bound_scales) -> BoundsPoolC:
    """``bounds``: int8 [L, P, Hkv, 2 (largest, smallest), d]; ``bound_scales``: float32 [L, P, Hkv]."""
    torch = _torch or _load_torch()
    dev = bounds.get_device()
    L, P, hkv, two, d = shape = _whole(bounds, "bounds", torch.int8, 5, dev)
    if two != 2 or _whole(bound_scales, "bounds: scales", torch.float32, 3, dev) != (L, P, hkv):
        _bad(f"bounds: {tuple(shape)}, scales {tuple(bound_scales.shape)}")
    return BoundsPoolC(bounds.data_ptr(), bound_scales.data_ptr(), P, L, hkv, d)


def _bounds_call(call, ps, dev, layer, bounds, bound_scales, start, lengths, max_new, block_tables, err, stream):
    i32 = _torch.int32
    bs = bounds_pool_struct(bounds, bound_scales)
    if bounds.get_device() != dev:
        _bad("bounds: on another device than the cache")
    seqs, pages = _whole(block_tables, "bounds: block tables", i32, 2, dev)
    if _whole(start, "bounds: start", i32, 1, dev)[0] != seqs or _whole(lengths, "bounds: lengths", i32, 1, dev)[0] != seqs:
        _bad(f"bounds: {start.shape[0]} starts, {lengths.shape[0]} lengths, {seqs} tables")
    if err is not None and not _whole(err, "bounds: err", i32, 1, dev)[0]:
        _bad("bounds: an empty err")
    if seqs:
        _launch(dev, stream, call, C.byref(ps), C.byref(bs), layer, seqs, start.data_ptr(), lengths.data_ptr(), max_new,
                block_tables.data_ptr(), pages, _ptr(err))


def pallas_bounds_kv(pool, layer: int, bounds, bound_scales, start, lengths, max_new: int, block_tables, err=None,
                     stream=None):
    """Bounds (bounds_pool_struct) of the blocks that hold positions [start, lengths) of a bf16 pool's sequences."""
    dev = pool.get_device()
    _whole(pool, "bounds: pool", (_torch or _load_torch()).bfloat16, 6, dev)
    _bounds_call(lib().pallas_bounds_kv, kv_pool_struct(pool), dev, layer, bounds, bound_scales, start, lengths, max_new,
                 block_tables, err, stream)


def pallas_bounds_quant(codes, scales, layer: int, bounds, bound_scales, start, lengths, max_new: int, block_tables, err=None,
                        stream=None):
    """The same of an 8- or 4-bit pool (quant_pool_struct)."""
    _bounds_call(lib().pallas_bounds_quant, quant_pool_struct(codes, scales), codes.get_device(), layer, bounds, bound_scales,
                 start, lengths, max_new, block_tables, err, stream)


def pallas_select_workspace_size(num_seqs: int, n_kv_heads: int, max_length: int) -> int:
    return int(lib().pallas_select_workspace_size(num_seqs, n_kv_heads, max_length))


def pallas_select_blocks(bounds, bound_scales, layer: int, q, lengths, max_length: int, block_tables, blocks, workspace,
                         first: int = 1, last: int = 2, err=None, stream=None):
    """Lists, in ``blocks`` (int32 [num_seqs, Hkv, max_blocks]), the blocks of each sequence that ``q`` (bf16 [num_seqs,
    Hq, d], any row stride) scores highest, its ``first`` first and ``last`` last ones among them."""
    bs, dev = bounds_pool_struct(bounds, bound_scales), bounds.get_device()
    i32, shape = _torch.int32, q.shape
    qs = _packed_rows(q, "select: q", dev, shape)
    S, H, d = shape
    seqs, pages = _whole(block_tables, "select: block tables", i32, 2, dev)
    got = _whole(blocks, "select: blocks", i32, 3, dev)
    if d != bs.head_dim or seqs != S or _whole(lengths, "select: lengths", i32, 1, dev)[0] != S or got != (
            S, bs.n_kv_heads, got[2]):
        _bad(f"select: {tuple(shape)} queries, {lengths.shape[0]} lengths, {seqs} tables, blocks {tuple(got)}, bounds of "
             f"{bs.n_kv_heads} heads of {bs.head_dim}")
    if err is not None and not _whole(err, "select: err", i32, 1, dev)[0]:
        _bad("select: an empty err")
    if workspace.get_device() != dev or not workspace.is_contiguous():
        _bad("select: workspace on another device, or not contiguous")
    if S:
        _launch(dev, stream, lib().pallas_select_blocks, C.byref(bs), layer, S, H, q.data_ptr(), qs, lengths.data_ptr(),
                max_length, block_tables.data_ptr(), pages, got[2], first, last, blocks.data_ptr(), workspace.data_ptr(),
                workspace.nbytes, _ptr(err))


def _window_params(r_p, r_d, goodput, s_kv, t_load=0.0, t_0=0.0, alpha=0.8, t_max=5.0, dt=0.01):
    return WindowParams(r_p, r_d, goodput, s_kv, t_load, t_0, alpha, t_max, dt)


def pallas_window_select(k_curr: float, t_remain: float, **params) -> WindowDecision:
    """Algorithm 1's window decision; ``params`` are the fields of
    pallas_window_params (r_p, r_d, goodput, s_kv, t_load, t_0, alpha,
    t_max, dt)."""
    p = _window_params(**params)
    d = WindowDecision()
    _check(lib().pallas_window_select(C.byref(p), k_curr, t_remain, C.byref(d)))
    return d


def pallas_window_evaluate(k_curr: float, t_remain: float, t_w: float, **params) -> WindowDecision:
    p = _window_params(**params)
    d = WindowDecision()
    _check(lib().pallas_window_evaluate(C.byref(p), k_curr, t_remain, t_w, C.byref(d)))
    return d


def pallas_ewma_update(state: Ewma, sample: float, weight: float) -> float:
    return lib().pallas_ewma_update(C.byref(state), sample, weight)


def pallas_admit(model_compatible: bool, vram_free_bytes: float, s_kv: float, k_curr: float,
                 r_d: float, t_remain: float) -> bool:
    return bool(lib().pallas_admit(int(bool(model_compatible)), vram_free_bytes, s_kv, k_curr, r_d,
                                   t_remain))


def pallas_waste_bound(t_max: float, e_early: float, t_avail: float) -> float:
    return lib().pallas_waste_bound(t_max, e_early, t_avail)


def pallas_profile_enable(classes=KERNEL_CLASSES):
    """Time every launch of the named kernel classes (empty: disable)."""
    mask = 0
    for c in classes:
        mask |= 1 << KERNEL_CLASSES.index(c)
    lib().pallas_profile_enable(mask)


def pallas_profile_reset():
    lib().pallas_profile_reset()


def pallas_profile_clock(kernel_class: str):
    """(mean shader clock in GHz, workgroups sampled) inside the timed
    launches of one kernel class since the last reset."""
    ghz = C.c_double()
    wgs = C.c_int64()
    _check(lib().pallas_profile_clock(KERNEL_CLASSES.index(kernel_class), C.byref(ghz), C.byref(wgs)))
    return ghz.value, wgs.value


def pallas_profile_read():
    """{class: (total_ms, launches)} since the last reset."""
    n = len(KERNEL_CLASSES)
    ms = (C.c_double * n)()
    cnt = (C.c_int64 * n)()
    _check(lib().pallas_profile_read(ms, cnt))
    return {k: (ms[i], cnt[i]) for i, k in enumerate(KERNEL_CLASSES)}


class Model:
    """A model handle over caller-owned bf16 device weights."""

    def __init__(self, cfg, glob, layers):
        self.cfg = cfg
        self._keep = (glob, layers)
        self.handle = pallas_model_create(cfg, glob, layers)

    def close(self):
        if self.handle:
            pallas_model_destroy(self.handle)
            self.handle = None

    def __del__(self):
        try:
            self.close()
        except Exception:
            pass

    def workspace_size(self, max_tokens: int, max_seqs: int = 1) -> int:
        return pallas_workspace_size(self.handle, max_tokens, max_seqs)

    def workspace(self, max_tokens: int, max_seqs: int = 1, device="cuda"):
        import torch
        return torch.empty(self.workspace_size(max_tokens, max_seqs), dtype=torch.uint8, device=device)

    def prefill_prefix(self, token_ids, cu_seqlens, block_tables, pool, workspace, err=None,
                       stream=None):
        pallas_prefill_prefix(self.handle, token_ids, cu_seqlens, block_tables, pool, workspace,
                              err, stream)

    def prefill_chunk(self, token_ids, cu_seqlens, start_pos, block_tables, pool, workspace,
                      err=None, stream=None):
        pallas_prefill_chunk(self.handle, token_ids, cu_seqlens, start_pos, block_tables, pool,
                             workspace, err, stream)

    def decode_step(self, tokens, positions, block_tables, pool, logits, workspace, err=None,
                    stream=None):
        pallas_decode_step(self.handle, tokens, positions, block_tables, pool, logits, workspace,
                           err, stream)

    def decode_step_static(self, tokens, positions, block_tables, pool, logits, err=None, stream=None):
        pallas_decode_step_static(self.handle, tokens, positions, block_tables, pool, logits, err, stream)
