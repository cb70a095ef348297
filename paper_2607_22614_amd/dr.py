"""ctypes binding of libdr.so: the C ABI of include/dr.h with the same names.

Argument marshalling only: every step of staging runs in the HIP library.
Device buffers are passed as torch tensors (or raw integer addresses), streams
as torch streams (default: the current stream).  Importing this module loads
the library and raises ImportError when it has not been built, so nothing can
silently fall back to another implementation.

The C ABI carries pointers without sizes.  For tensor and array arguments the
binding checks, before calling the library, what the library would otherwise
trust: the number of shard pointers equals the plan's, every buffer is dense,
device arguments are device tensors and the host store is host memory, and each
buffer holds the bytes the plan will touch (ValueError otherwise).  Raw integer
addresses are passed through unchecked.
"""
from __future__ import annotations

import ctypes
import importlib.util
import os
from typing import Sequence

_LIB_PATH = os.path.join(os.path.dirname(os.path.abspath(__file__)), "libdr.so")
if not os.path.exists(_LIB_PATH):
    raise ImportError(f"{_LIB_PATH} is missing: build it with `python -m paper_2607_22614_amd.build` "
                      "(or __graft_entry__.build())")


def _share_runtime() -> None:
    """Loads the HIP runtime that torch brings, where it brings one, so that libdr.so takes it too whichever of the two is imported
    first: of two runtimes in a process the second finds no device."""
    spec = importlib.util.find_spec("torch")
    path = os.path.join(os.path.dirname(spec.origin), "lib", "libamdhip64.so") if spec and spec.origin else ""
    if os.path.exists(path):
        ctypes.CDLL(path)


_share_runtime()
_lib = ctypes.CDLL(_LIB_PATH)

DR_OK, DR_EINVAL, DR_ERANGE, DR_ENOMEM, DR_EHIP = 0, -1, -2, -3, -4
DR_MAX_SHARDS = 64
DR_SEG_VEC4 = 1
DR_OP_CAST_BF16, DR_OP_COPY_F32, DR_OP_ZERO_F32 = 0, 1, 2
DR_PLAN_ROLLOUT, DR_PLAN_RESHARD = 0, 1
DR_TILE_DEPTH_AUTO = 0
_CODES = {DR_EINVAL: "DR_EINVAL", DR_ERANGE: "DR_ERANGE", DR_ENOMEM: "DR_ENOMEM", DR_EHIP: "DR_EHIP"}


class dr_model(ctypes.Structure):
    _fields_ = [(n, ctypes.c_int32) for n in
                ("n_layers", "hidden", "n_q_heads", "n_kv_heads", "head_dim", "ffn", "vocab")]


class dr_layout(ctypes.Structure):
    _fields_ = [("train_shards", ctypes.c_int32), ("tp", ctypes.c_int32),
                ("chunk_bytes", ctypes.c_uint64), ("moment_chunk_bytes", ctypes.c_uint64),
                ("tile_depth", ctypes.c_int32), ("reserved", ctypes.c_int32)]


class dr_checksum(ctypes.Structure):
    _fields_ = [("s1", ctypes.c_uint64), ("s2", ctypes.c_uint64)]


class dr_plan_info(ctypes.Structure):
    _fields_ = [(n, ctypes.c_uint64) for n in
                ("n_elems", "padded_elems", "shard_elems", "norm_elems", "rank_elems", "rollout_bytes",
                 "num_chunks", "last_chunk_bytes", "moment_bytes", "num_moment_chunks", "num_segments",
                 "num_tiles", "device_table_bytes", "pinned_bytes")] + \
              [("device", ctypes.c_int32), ("kind", ctypes.c_int32), ("dst_shard_elems", ctypes.c_uint64),
               ("tile_elems", ctypes.c_uint64), ("train_shards", ctypes.c_int32), ("tp", ctypes.c_int32),
               ("dst_shards", ctypes.c_int32), ("reserved", ctypes.c_int32), ("chunk_bytes", ctypes.c_uint64),
               ("moment_chunk_bytes", ctypes.c_uint64), ("deep_tile_elems", ctypes.c_uint64),
               ("deep_num_tiles", ctypes.c_uint64), ("last_tile_depth", ctypes.c_int32),
               ("reserved2", ctypes.c_int32)]


class dr_tensor_desc(ctypes.Structure):
    _fields_ = [("name", ctypes.c_char * 32), ("rank", ctypes.c_int32), ("ndim", ctypes.c_int32),
                ("byte_offset", ctypes.c_uint64), ("rows", ctypes.c_int64), ("cols", ctypes.c_int64)]


class dr_segment(ctypes.Structure):
    _fields_ = [("dst_elem", ctypes.c_uint64), ("src_elem", ctypes.c_uint64),
                ("shard", ctypes.c_uint32), ("chunk", ctypes.c_uint32),
                ("rows", ctypes.c_uint32), ("cols", ctypes.c_uint32),
                ("src_row_stride", ctypes.c_uint32), ("flags", ctypes.c_uint32),
                ("dst_shard", ctypes.c_uint32), ("op", ctypes.c_uint32)]


class dr_hyst_params(ctypes.Structure):
    _fields_ = [("num_configs", ctypes.c_int32), ("initial", ctypes.c_int32),
                ("train_gpus", ctypes.POINTER(ctypes.c_int32)), ("rollout_gpus", ctypes.POINTER(ctypes.c_int32)),
                ("enter", ctypes.c_double), ("exit", ctypes.c_double), ("consecutive", ctypes.c_int32),
                ("dwell", ctypes.c_int32), ("cooldown", ctypes.c_int32), ("horizon_steps", ctypes.c_int32),
                ("switch_cost_s", ctypes.c_double)]


class dr_hyst_decision(ctypes.Structure):
    _fields_ = [("config", ctypes.c_int32), ("action", ctypes.c_int32), ("reason", ctypes.c_int32),
                ("run", ctypes.c_int32), ("imbalance", ctypes.c_double), ("predicted_gain_s", ctypes.c_double)]


class dr_qmatrix(ctypes.Structure):
    _fields_ = [("data", ctypes.c_void_p), ("scales", ctypes.c_void_p), ("rows", ctypes.c_int64),
                ("cols", ctypes.c_int64), ("stride", ctypes.c_int64), ("block_rows", ctypes.c_int32),
                ("reserved", ctypes.c_int32)]


class dr_grad(ctypes.Structure):
    _fields_ = [("grad", ctypes.c_void_p), ("out", ctypes.c_void_p), ("numel", ctypes.c_int64),
                ("grad_type", ctypes.c_int32), ("out_type", ctypes.c_int32)]


DR_TYPE_F32, DR_TYPE_BF16 = 0, 1
DR_QUANT_BLOCK = 128
DR_ACCUMULATE, DR_FAST_SUMS = 1, 2
DR_ACT_SILU, DR_ACT_GELU_TANH = 0, 1
DR_HYST_BALANCED, DR_HYST_PERSISTENCE, DR_HYST_COOLDOWN, DR_HYST_DWELL, DR_HYST_EDGE, DR_HYST_AMORTIZE, \
    DR_HYST_RESIZE = range(7)

_P = ctypes.c_void_p
_PP = ctypes.POINTER(ctypes.c_void_p)
_I64, _PU64, _PQ = ctypes.c_int64, ctypes.POINTER(ctypes.c_uint64), ctypes.POINTER(dr_qmatrix)
_SIGS = {
    "dr_plan_create": ([ctypes.POINTER(dr_model), ctypes.POINTER(dr_layout), ctypes.POINTER(_P)], ctypes.c_int),
    "dr_plan_create_host": ([ctypes.POINTER(dr_model), ctypes.POINTER(dr_layout), ctypes.POINTER(_P)], ctypes.c_int),
    "dr_reshard_plan_create": ([ctypes.POINTER(dr_model), ctypes.c_int32, ctypes.c_int32, ctypes.c_uint64,
                                ctypes.POINTER(_P)], ctypes.c_int),
    "dr_reshard_plan_create_host": ([ctypes.POINTER(dr_model), ctypes.c_int32, ctypes.c_int32, ctypes.c_uint64,
                                     ctypes.POINTER(_P)], ctypes.c_int),
    "dr_plan_destroy": ([_P], None),
    "dr_plan_get_info": ([_P, ctypes.POINTER(dr_plan_info)], ctypes.c_int),
    "dr_plan_tensor": ([_P, ctypes.c_int32, ctypes.c_int32, ctypes.POINTER(dr_tensor_desc)], ctypes.c_int),
    "dr_plan_segment": ([_P, ctypes.c_uint64, ctypes.POINTER(dr_segment)], ctypes.c_int),
    "dr_stage_chunk": ([_P, ctypes.c_uint64, _PP, _P, _P, _P], ctypes.c_int),
    "dr_stage_chunk_noalloc": ([_P, ctypes.c_uint64, _PP, _P, _P, _P], ctypes.c_int),
    "dr_stage_all": ([_P, _PP, _P, _P, _P], ctypes.c_int),
    "dr_stage_through_host": ([_P, _PP, _P, _P, _P], ctypes.c_int),
    "dr_reshard": ([_P, _PP, _PP, _P, _P], ctypes.c_int),
    "dr_offload_moments": ([_P, _PP, _PP, _P, _P], ctypes.c_int),
    "dr_restore_moments": ([_P, _P, _PP, _PP, _P], ctypes.c_int),
    "dr_reshard_through_host": ([_P, _PP, _PP, _P, _P], ctypes.c_int),
    "dr_offload_moments_range": ([_P, _PP, _PP, _P, ctypes.c_uint64, ctypes.c_uint64, _P], ctypes.c_int),
    "dr_restore_moments_range": ([_P, _P, _PP, _PP, ctypes.c_uint64, ctypes.c_uint64, _P], ctypes.c_int),
    "dr_restore_moments_begin": ([_P, _P, _PP, _PP, _P], ctypes.c_int),
    "dr_restore_moments_end": ([_P], ctypes.c_int),
    "dr_moment_checksums": ([_P, _PP, _PP, _P, _P], ctypes.c_int),
    "dr_hyst_create": ([ctypes.POINTER(dr_hyst_params), ctypes.POINTER(_P)], ctypes.c_int),
    "dr_hyst_step": ([_P, ctypes.c_double, ctypes.c_double, ctypes.POINTER(dr_hyst_decision)], ctypes.c_int),
    "dr_hyst_destroy": ([_P], None),
    "dr_break_even_steps": ([ctypes.c_double, ctypes.c_double, ctypes.c_double], ctypes.c_double),
    "dr_qmatrix_sizes": ([_I64, _I64, ctypes.c_int32, ctypes.POINTER(_I64), _PU64, _PU64], ctypes.c_int),
    "dr_quantize": ([_P, ctypes.c_int32, _I64, _I64, _I64, _PQ, _PQ, _P], ctypes.c_int),
    "dr_qmatmul": ([_PQ, _PQ, _P, ctypes.c_int32, _I64, ctypes.c_int32, _P, ctypes.c_uint64, _P], ctypes.c_int),
    "dr_qmatmul_workspace": ([_I64, _I64, _I64, _PU64], ctypes.c_int),
    "dr_qlinear": ([_P, ctypes.c_int32, _I64, _I64, _PQ, _P, ctypes.c_int32, _I64, ctypes.c_int32, _P,
                    ctypes.c_uint64, _P], ctypes.c_int),
    "dr_qlinear_workspace": ([_I64, _I64, _I64, _PU64], ctypes.c_int),
    "dr_qgated": ([_P, ctypes.c_int32, _I64, _I64, _PQ, ctypes.c_int32, _P, ctypes.c_int32, _I64, ctypes.c_int32, _P,
                   ctypes.c_uint64, _P], ctypes.c_int),
    "dr_qgated_workspace": ([_I64, _I64, _I64, _PU64], ctypes.c_int),
    "dr_qgated_save": ([_PQ, _PQ, ctypes.c_int32, _PQ, _PQ, _PQ, ctypes.c_int32, _P, ctypes.c_uint64, _P],
                       ctypes.c_int),
    "dr_qgated_save_workspace": ([_I64, _I64, _I64, _PU64], ctypes.c_int),
    "dr_gated_backward": ([_P, ctypes.c_int32, _I64, _PQ, _PQ, ctypes.c_int32, _PQ, _PQ, _PQ, _P], ctypes.c_int),
    "dr_qtranspose": ([_PQ, _PQ, _P], ctypes.c_int),
    "dr_grad_workspace": ([_PU64], ctypes.c_int),
    "dr_grad_norm": ([ctypes.POINTER(dr_grad), _I64, _P, _P, _P, _P], ctypes.c_int),
    "dr_grad_scale": ([ctypes.POINTER(dr_grad), _I64, _P, ctypes.c_double, _P, _P], ctypes.c_int),
    "dr_grad_clip": ([ctypes.POINTER(dr_grad), _I64, ctypes.c_double, _P, _P, _P], ctypes.c_int),
    "dr_last_error": ([], ctypes.c_char_p),
}
for _name, (_args, _res) in _SIGS.items():
    _f = getattr(_lib, _name)
    _f.argtypes = _args
    _f.restype = _res

EXPORTED = tuple(_SIGS)


class DrError(RuntimeError):
    def __init__(self, code: int, where: str):
        self.code = code
        msg = _lib.dr_last_error().decode(errors="replace")
        super().__init__(f"{where}: {_CODES.get(code, code)}: {msg}")


def _check(rc: int, where: str) -> None:
    if rc != DR_OK:
        raise DrError(rc, where)


def _addr(x) -> int:
    """Device/host address of a tensor, numpy array or integer."""
    if x is None:
        return 0
    if isinstance(x, int):
        return x
    if hasattr(x, "data_ptr"):
        return x.data_ptr()
    if hasattr(x, "ctypes"):
        return x.ctypes.data
    raise TypeError(f"cannot take the address of {type(x)!r}")


def _fits(x, nbytes: int) -> bool:
    """Whether x is a dense device tensor of at least nbytes (the common case, in three attribute reads);
    anything else is left to _buf's checks."""
    if type(x) is int:
        return False
    try:
        return x.is_cuda and x.is_contiguous() and x.nbytes >= nbytes
    except AttributeError:
        return False


def _buf(x, nbytes: int, where: str, device: bool) -> int:
    """Address of a buffer the library will access as `nbytes` dense bytes.

    The C ABI carries no sizes, so a tensor or array argument is checked here: dense
    (contiguous), on the right side (device tensor for device arguments, host memory for the
    host store) and at least nbytes long.  A plain integer address is passed through unchecked.
    """
    if x is None or isinstance(x, int):
        return _addr(x)
    if device and _fits(x, nbytes):
        return x.data_ptr()
    if hasattr(x, "data_ptr"):  # torch tensor
        if not x.is_contiguous():
            raise ValueError(f"{where}: tensor is not contiguous")
        if bool(x.is_cuda) != device:
            raise ValueError(f"{where}: expected a {'device' if device else 'host'} tensor, got one on {x.device}")
        have = x.numel() * x.element_size()
    elif hasattr(x, "ctypes"):  # numpy array: host memory
        if device:
            raise ValueError(f"{where}: a numpy array is host memory; a device buffer is needed")
        if not x.flags["C_CONTIGUOUS"]:
            raise ValueError(f"{where}: array is not contiguous")
        have = x.nbytes
    else:
        raise TypeError(f"{where}: cannot take the address of {type(x)!r}")
    if have < nbytes:
        raise ValueError(f"{where}: {have} bytes, the plan needs {nbytes}")
    return _addr(x)


def _ptr_array(xs: Sequence) -> ctypes.Array:
    return (ctypes.c_void_p * len(xs))(*[_addr(x) for x in xs])


def _shards(xs: Sequence, count: int, nbytes: int, where: str) -> ctypes.Array:
    """Host array of `count` device pointers; the library reads exactly `count` of them.
    count None: a call on the wrong kind of plan, passed through for the library to reject."""
    if count is None:
        return _ptr_array(xs)
    if len(xs) != count:
        raise ValueError(f"{where}: {len(xs)} shard buffers given, the plan has {count}")
    # the text that names a shard is made only for one that needs the full checks
    return (ctypes.c_void_p * count)(*[x.data_ptr() if _fits(x, nbytes) else _buf(x, nbytes, f"{where}[{i}]", True)
                                       for i, x in enumerate(xs)])


_current = None  # () -> the current stream's handle, without a Stream object around it where torch has a call for that


def _find_current():
    import torch
    raw, device = getattr(torch._C, "_cuda_getCurrentRawStream", None), getattr(torch._C, "_cuda_getDevice", None)
    torch.cuda.current_device()  # initialises torch's side of the GPU
    if raw and device:
        return lambda: raw(device())
    return lambda: torch.cuda.current_stream().cuda_stream


def _forget_current():
    global _current
    _current = None


# the first look initialises torch's side of the GPU, which torch refuses in a fork of a process that has used it
os.register_at_fork(after_in_child=_forget_current)


def _stream(stream) -> int:
    global _current
    if stream is None:
        if _current is None:
            _current = _find_current()
        return _current()
    if isinstance(stream, int):
        return stream
    return stream.cuda_stream


class Plan:
    """Owns a dr_plan*; destroyed with the object (after the caller has synchronized)."""

    def __init__(self, handle: int):
        self._h = handle
        # buffers a deferred restore reads and writes from a library thread: held until it ends
        self._restore_refs = None
        info = dr_plan_info()
        _check(_lib.dr_plan_get_info(handle, ctypes.byref(info)), "dr_plan_get_info")
        self.info = {n: getattr(info, n) for n, _ in dr_plan_info._fields_}

    @property
    def handle(self) -> int:
        return self._h

    def close(self) -> None:
        if self._h:
            _lib.dr_plan_destroy(self._h)  # joins a deferred restore still in flight
            self._h = None
        self._restore_refs = None

    def __del__(self):
        try:
            self.close()
        except Exception:
            pass

    def __enter__(self):
        return self

    def __exit__(self, *exc):
        self.close()


def _model(model) -> dr_model:
    if isinstance(model, dr_model):
        return model
    return dr_model(*[int(v) for v in model])


def _layout(train_shards, tp, chunk_bytes, moment_chunk_bytes=0, tile_depth=DR_TILE_DEPTH_AUTO) -> dr_layout:
    return dr_layout(int(train_shards), int(tp), int(chunk_bytes), int(moment_chunk_bytes), int(tile_depth), 0)


def dr_plan_create(model, train_shards: int, tp: int, chunk_bytes: int, moment_chunk_bytes: int = 0,
                   tile_depth: int = DR_TILE_DEPTH_AUTO) -> Plan:
    """model: (n_layers, hidden, n_q_heads, n_kv_heads, head_dim, ffn, vocab) or dr_model."""
    h = ctypes.c_void_p()
    _check(_lib.dr_plan_create(ctypes.byref(_model(model)),
                               ctypes.byref(_layout(train_shards, tp, chunk_bytes, moment_chunk_bytes, tile_depth)),
                               ctypes.byref(h)), "dr_plan_create")
    return Plan(h.value)


def dr_plan_create_host(model, train_shards: int, tp: int, chunk_bytes: int, moment_chunk_bytes: int = 0,
                        tile_depth: int = DR_TILE_DEPTH_AUTO) -> Plan:
    h = ctypes.c_void_p()
    _check(_lib.dr_plan_create_host(ctypes.byref(_model(model)),
                                    ctypes.byref(_layout(train_shards, tp, chunk_bytes, moment_chunk_bytes,
                                                         tile_depth)),
                                    ctypes.byref(h)), "dr_plan_create_host")
    return Plan(h.value)


def dr_reshard_plan_create(model, from_shards: int, to_shards: int, chunk_bytes: int) -> Plan:
    h = ctypes.c_void_p()
    _check(_lib.dr_reshard_plan_create(ctypes.byref(_model(model)), int(from_shards), int(to_shards),
                                       int(chunk_bytes), ctypes.byref(h)), "dr_reshard_plan_create")
    return Plan(h.value)


def dr_reshard_plan_create_host(model, from_shards: int, to_shards: int, chunk_bytes: int) -> Plan:
    h = ctypes.c_void_p()
    _check(_lib.dr_reshard_plan_create_host(ctypes.byref(_model(model)), int(from_shards), int(to_shards),
                                            int(chunk_bytes), ctypes.byref(h)), "dr_reshard_plan_create_host")
    return Plan(h.value)


def dr_plan_get_info(plan: Plan) -> dict:
    info = dr_plan_info()
    _check(_lib.dr_plan_get_info(plan.handle, ctypes.byref(info)), "dr_plan_get_info")
    return {n: getattr(info, n) for n, _ in dr_plan_info._fields_}


def dr_plan_tensor(plan: Plan, rank: int, index: int) -> dict:
    d = dr_tensor_desc()
    _check(_lib.dr_plan_tensor(plan.handle, rank, index, ctypes.byref(d)), "dr_plan_tensor")
    return {"name": d.name.decode(), "rank": d.rank, "ndim": d.ndim, "byte_offset": d.byte_offset,
            "rows": d.rows, "cols": d.cols}


def dr_plan_segment(plan: Plan, index: int) -> dict:
    s = dr_segment()
    _check(_lib.dr_plan_segment(plan.handle, index, ctypes.byref(s)), "dr_plan_segment")
    return {n: getattr(s, n) for n, _ in dr_segment._fields_}


def _rollout(plan: Plan) -> bool:
    return plan.info["kind"] == DR_PLAN_ROLLOUT


def _chunk_len(i: dict, chunk: int) -> int:
    if 0 <= chunk < i["num_chunks"] - 1:
        return i["chunk_bytes"]
    return i["last_chunk_bytes"] if chunk == i["num_chunks"] - 1 else 0


def dr_stage_chunk(plan: Plan, chunk: int, shards: Sequence, dst_chunk, d_ck, stream=None) -> None:
    """shards: W device tensors/addresses; dst_chunk: device buffer; d_ck: device dr_checksum slot."""
    i = plan.info
    arr = _shards(shards, i["train_shards"] if _rollout(plan) else None, 4 * i["shard_elems"], "dr_stage_chunk shards")
    _check(_lib.dr_stage_chunk(plan.handle, int(chunk), arr,
                               _buf(dst_chunk, _chunk_len(i, int(chunk)), "dr_stage_chunk dst_chunk", True),
                               _buf(d_ck, 16, "dr_stage_chunk d_ck", True), _stream(stream)), "dr_stage_chunk")


def dr_stage_chunk_noalloc(plan: Plan, chunk: int, shards: Sequence, dst_chunk, d_ck, stream=None) -> None:
    """dr_stage_chunk without any device allocation: the checksum accumulators are the library's
    static per-GPU array.  Calls on one GPU must not overlap."""
    i = plan.info
    arr = _shards(shards, i["train_shards"] if _rollout(plan) else None, 4 * i["shard_elems"],
                  "dr_stage_chunk_noalloc shards")
    _check(_lib.dr_stage_chunk_noalloc(plan.handle, int(chunk), arr,
                                       _buf(dst_chunk, _chunk_len(i, int(chunk)), "dr_stage_chunk_noalloc dst_chunk",
                                            True),
                                       _buf(d_ck, 16, "dr_stage_chunk_noalloc d_ck", True), _stream(stream)),
           "dr_stage_chunk_noalloc")


def dr_stage_all(plan: Plan, shards: Sequence, dst, d_cks, stream=None) -> None:
    i = plan.info
    arr = _shards(shards, i["train_shards"] if _rollout(plan) else None, 4 * i["shard_elems"], "dr_stage_all shards")
    _check(_lib.dr_stage_all(plan.handle, arr, _buf(dst, i["rollout_bytes"], "dr_stage_all dst", True),
                             _buf(d_cks, 16 * i["num_chunks"], "dr_stage_all d_cks", True), _stream(stream)),
           "dr_stage_all")


def dr_stage_through_host(plan: Plan, shards: Sequence, dst, d_cks, stream=None) -> None:
    i = plan.info
    arr = _shards(shards, i["train_shards"] if _rollout(plan) else None, 4 * i["shard_elems"], "dr_stage_through_host shards")
    _check(_lib.dr_stage_through_host(plan.handle, arr,
                                      _buf(dst, i["rollout_bytes"], "dr_stage_through_host dst", True),
                                      _buf(d_cks, 16 * i["num_chunks"], "dr_stage_through_host d_cks", True),
                                      _stream(stream)), "dr_stage_through_host")


def dr_reshard(plan: Plan, src_shards: Sequence, dst_shards: Sequence, d_cks, stream=None) -> None:
    i = plan.info
    ok = i["kind"] == DR_PLAN_RESHARD
    a = _shards(src_shards, i["train_shards"] if ok else None, 4 * i["shard_elems"], "dr_reshard src_shards")
    b = _shards(dst_shards, i["dst_shards"] if ok else None, 4 * i["dst_shard_elems"], "dr_reshard dst_shards")
    _check(_lib.dr_reshard(plan.handle, a, b,
                           _buf(d_cks, 16 * i["num_chunks"], "dr_reshard d_cks", True), _stream(stream)), "dr_reshard")


def dr_reshard_through_host(plan: Plan, src_shards: Sequence, dst_shards: Sequence, d_cks, stream=None) -> None:
    i = plan.info
    ok = i["kind"] == DR_PLAN_RESHARD
    a = _shards(src_shards, i["train_shards"] if ok else None, 4 * i["shard_elems"], "dr_reshard_through_host src_shards")
    b = _shards(dst_shards, i["dst_shards"] if ok else None, 4 * i["dst_shard_elems"],
                "dr_reshard_through_host dst_shards")
    _check(_lib.dr_reshard_through_host(plan.handle, a, b,
                                        _buf(d_cks, 16 * i["num_chunks"], "dr_reshard_through_host d_cks", True),
                                        _stream(stream)), "dr_reshard_through_host")


def _moment_args(plan: Plan, m_shards: Sequence, v_shards: Sequence, host_store, where: str):
    i = plan.info
    m = _shards(m_shards, i["train_shards"], 4 * i["shard_elems"], f"{where} m_shards")
    v = _shards(v_shards, i["train_shards"], 4 * i["shard_elems"], f"{where} v_shards")
    return m, v, _buf(host_store, i["moment_bytes"], f"{where} host_store", False)


def dr_offload_moments(plan: Plan, m_shards: Sequence, v_shards: Sequence, host_store, side_stream) -> None:
    m, v, store = _moment_args(plan, m_shards, v_shards, host_store, "dr_offload_moments")
    _check(_lib.dr_offload_moments(plan.handle, m, v, store,
                                   _stream(side_stream)), "dr_offload_moments")


def dr_restore_moments(plan: Plan, host_store, m_shards: Sequence, v_shards: Sequence, side_stream) -> None:
    m, v, store = _moment_args(plan, m_shards, v_shards, host_store, "dr_restore_moments")
    _check(_lib.dr_restore_moments(plan.handle, store, m, v,
                                   _stream(side_stream)), "dr_restore_moments")


def dr_offload_moments_range(plan: Plan, m_shards: Sequence, v_shards: Sequence, host_store, first_chunk: int,
                             num_chunks: int, side_stream) -> None:
    m, v, store = _moment_args(plan, m_shards, v_shards, host_store, "dr_offload_moments_range")
    _check(_lib.dr_offload_moments_range(plan.handle, m, v, store,
                                         int(first_chunk), int(num_chunks), _stream(side_stream)),
           "dr_offload_moments_range")


def dr_restore_moments_range(plan: Plan, host_store, m_shards: Sequence, v_shards: Sequence, first_chunk: int,
                             num_chunks: int, side_stream) -> None:
    m, v, store = _moment_args(plan, m_shards, v_shards, host_store, "dr_restore_moments_range")
    _check(_lib.dr_restore_moments_range(plan.handle, store, m, v,
                                         int(first_chunk), int(num_chunks), _stream(side_stream)),
           "dr_restore_moments_range")


def dr_restore_moments_begin(plan: Plan, host_store, m_shards: Sequence, v_shards: Sequence, side_stream) -> None:
    """Starts the deferred restore on a library thread.  The plan keeps references to the host
    store, the shard tensors and the side stream until dr_restore_moments_end (or close), so
    none of them is freed while the thread still copies."""
    m, v, store = _moment_args(plan, m_shards, v_shards, host_store, "dr_restore_moments_begin")
    refs = (host_store, tuple(m_shards), tuple(v_shards), side_stream)
    _check(_lib.dr_restore_moments_begin(plan.handle, store, m, v,
                                         _stream(side_stream)), "dr_restore_moments_begin")
    plan._restore_refs = refs


def dr_restore_moments_end(plan: Plan) -> None:
    try:
        _check(_lib.dr_restore_moments_end(plan.handle), "dr_restore_moments_end")
    finally:
        plan._restore_refs = None  # the thread has been joined, whatever it returned


def dr_moment_checksums(plan: Plan, m_shards: Sequence, v_shards: Sequence, d_cks, stream=None) -> None:
    """Checksum of every moment chunk (num_moment_chunks dr_checksum slots in d_cks)."""
    i = plan.info
    m = _shards(m_shards, i["train_shards"], 4 * i["shard_elems"], "dr_moment_checksums m_shards")
    v = _shards(v_shards, i["train_shards"], 4 * i["shard_elems"], "dr_moment_checksums v_shards")
    _check(_lib.dr_moment_checksums(plan.handle, m, v,
                                    _buf(d_cks, 16 * i["num_moment_chunks"], "dr_moment_checksums d_cks", True),
                                    _stream(stream)), "dr_moment_checksums")


class Hysteresis:
    """Owns a dr_hyst*."""

    def __init__(self, handle: int):
        self._h = handle

    @property
    def handle(self) -> int:
        return self._h

    def close(self) -> None:
        if self._h:
            _lib.dr_hyst_destroy(self._h)
            self._h = None

    def __del__(self):
        try:
            self.close()
        except Exception:
            pass


def dr_hyst_create(train_gpus: Sequence[int], rollout_gpus: Sequence[int], initial: int, enter: float, exit: float,
                   consecutive: int, dwell: int, cooldown: int, switch_cost_s: float = 0.0,
                   horizon_steps: int = 0) -> Hysteresis:
    """train_gpus/rollout_gpus: the pre-specified splits, most training GPUs first."""
    n = len(train_gpus)
    tg = (ctypes.c_int32 * max(n, 1))(*[int(x) for x in train_gpus])
    rg = (ctypes.c_int32 * max(len(rollout_gpus), 1))(*[int(x) for x in rollout_gpus])
    p = dr_hyst_params(int(n) if len(rollout_gpus) == n else -1, int(initial), tg, rg, float(enter), float(exit),
                       int(consecutive), int(dwell), int(cooldown), int(horizon_steps), float(switch_cost_s))
    h = ctypes.c_void_p()
    _check(_lib.dr_hyst_create(ctypes.byref(p), ctypes.byref(h)), "dr_hyst_create")
    return Hysteresis(h.value)


def dr_hyst_step(h: Hysteresis, t_rollout: float, t_train: float) -> dict:
    d = dr_hyst_decision()
    _check(_lib.dr_hyst_step(h.handle, float(t_rollout), float(t_train), ctypes.byref(d)), "dr_hyst_step")
    return {"config": d.config, "action": d.action, "reason": d.reason, "run": d.run, "imbalance": d.imbalance,
            "predicted_gain_s": d.predicted_gain_s}


def dr_break_even_steps(switch_cost_s: float, step_before_s: float, step_after_s: float) -> float:
    return _lib.dr_break_even_steps(float(switch_cost_s), float(step_before_s), float(step_after_s))


# ------------------------------------------------------------------ 8-bit matrices
def _find_device() -> None:
    global _device, _raw_stream
    import torch
    torch.cuda.current_device()  # initialises torch's side of the GPU
    _device = getattr(torch._C, "_cuda_getDevice", None) or torch.cuda.current_device
    _raw_stream = getattr(torch._C, "_cuda_getCurrentRawStream", None)
    if _raw_stream is None:
        _raw_stream = lambda d: torch.cuda.current_stream(d).cuda_stream  # noqa: E731


def _first_device() -> int:
    _find_device()
    return _device()


def _first_raw_stream(device: int) -> int:
    _find_device()
    return _raw_stream(device)


def _forget_device():
    global _device, _raw_stream
    _device, _raw_stream = _first_device, _first_raw_stream


_forget_device()  # _device(): the current device's index; _raw_stream(device): the handle of its current stream
os.register_at_fork(after_in_child=_forget_device)


def _elsewhere(where: str, *devices: int) -> None:
    raise ValueError(f"{where}: arguments on devices {list(devices)}, the current device is {_device()}")


def _stream_on(device: int, stream, where: str) -> int:
    """The stream's handle, for a call with arguments on `device`: the calls run on the current one, on a stream of its own."""
    current = _device()
    if device != current:
        _elsewhere(where, device)
    if stream is None:
        return _raw_stream(current)
    if isinstance(stream, int):
        return stream
    if stream.device_index != current:
        raise ValueError(f"{where}: a stream of device {stream.device_index}, the current device is {current}")
    return stream.cuda_stream


_TYPES: dict = {}  # torch dtype -> DR_TYPE_*, filled at the first tensor


def _type(t, where: str) -> int:
    """DR_TYPE_* of a tensor."""
    kind = _TYPES.get(t.dtype)
    if kind is None:
        import torch
        _TYPES.update({torch.float32: DR_TYPE_F32, torch.bfloat16: DR_TYPE_BF16})
        kind = _TYPES.get(t.dtype)
        if kind is None:
            raise ValueError(f"{where}: {t.dtype} is neither float32 nor bfloat16")
    return kind


def _dense_rows(t, where: str):
    """(address, type, rows, cols, row stride) of a 2-d device tensor whose rows are dense."""
    shape = t.shape
    if len(shape) != 2 or not t.is_cuda:
        raise ValueError(f"{where}: expected a 2-d device tensor, got {t.dim()}-d on {t.device}")
    rows, cols = shape
    step = cols
    if not t.is_contiguous():
        step, inner = t.stride()
        if inner != 1 and cols > 1:
            raise ValueError(f"{where}: the elements of a row are not adjacent")
        if rows == 1:
            step = max(step, cols)
        elif step < cols:
            raise ValueError(f"{where}: rows overlap")
    return t.data_ptr(), _TYPES.get(t.dtype) or _type(t, where), rows, cols, step


def dr_qmatrix_sizes(rows: int, cols: int, block_rows: int = 1) -> dict:
    """{"stride", "data_bytes", "scale_bytes"} of a rows x cols 8-bit matrix."""
    stride, data, scales = ctypes.c_int64(), ctypes.c_uint64(), ctypes.c_uint64()
    _check(_lib.dr_qmatrix_sizes(int(rows), int(cols), int(block_rows), ctypes.byref(stride), ctypes.byref(data),
                                 ctypes.byref(scales)), "dr_qmatrix_sizes")
    return {"stride": stride.value, "data_bytes": data.value, "scale_bytes": scales.value}


class QMatrix:
    """An 8-bit matrix over two device tensors of one-byte elements, which it keeps: data [rows, at least
    cols rounded up to 128] with dense rows, and scales (dense, [ceil(ceil(cols/128)/4), block rows, 4])."""

    __slots__ = ("data", "scales", "rows", "cols", "block_rows", "c", "ref", "device")

    def __init__(self, data, scales, rows: int, cols: int, block_rows: int = 1):
        need = dr_qmatrix_sizes(rows, cols, block_rows)
        if data.element_size() != 1 or scales.element_size() != 1 or not data.is_cuda or not scales.is_cuda:
            raise ValueError("QMatrix: data and scales are device tensors of one-byte elements")
        if data.dim() != 2 or data.shape[0] != rows or data.shape[1] < need["stride"] or data.stride(1) != 1:
            raise ValueError(f"QMatrix: data is not [{rows}, at least {need['stride']}] with dense rows")
        if not scales.is_contiguous() or scales.numel() < need["scale_bytes"]:
            raise ValueError(f"QMatrix: scales are not {need['scale_bytes']} dense bytes")
        self.device = data.get_device()
        if scales.get_device() != self.device:
            raise ValueError(f"QMatrix: data on device {self.device}, scales on {scales.get_device()}")
        stride = data.stride(0) if rows > 1 and cols else need["stride"]
        if stride < need["stride"]:
            raise ValueError("QMatrix: rows overlap")
        self.data, self.scales, self.rows, self.cols, self.block_rows = data, scales, int(rows), int(cols), int(block_rows)
        self.c = dr_qmatrix(data.data_ptr(), scales.data_ptr(), self.rows, self.cols, stride, self.block_rows, 0)
        self.ref = ctypes.byref(self.c)

    @classmethod
    def empty(cls, rows: int, cols: int, block_rows: int = 1, device="cuda") -> "QMatrix":
        import torch
        stride = dr_qmatrix_sizes(rows, cols, block_rows)["stride"]
        words, block = -(-stride // (4 * DR_QUANT_BLOCK)), -(-rows // block_rows)
        return cls(torch.empty((rows, stride), dtype=torch.uint8, device=device),
                   torch.empty((words, block, 4), dtype=torch.uint8, device=device), rows, cols, block_rows)


def dr_quantize(src, q: QMatrix | None = None, qt: QMatrix | None = None, stream=None) -> None:
    """src (2-d float32 or bfloat16) to 8 bits: as it is into q, transposed into qt."""
    addr, kind, rows, cols, step = _dense_rows(src, "dr_quantize src")
    device = src.get_device()
    if q and q.device != device or qt and qt.device != device:
        _elsewhere("dr_quantize", device, *[m.device for m in (q, qt) if m])
    _check(_lib.dr_quantize(addr, kind, rows, cols, step, q.ref if q else None, qt.ref if qt else None,
                            _stream_on(device, stream, "dr_quantize")), "dr_quantize")


def _workspace(ws, device: int, where: str):
    """(address, bytes) of a workspace tensor on `device`, or of None."""
    if ws is None:
        return 0, 0
    if not ws.is_cuda or not ws.is_contiguous():
        raise ValueError(f"{where}: expected a dense device tensor")
    if ws.get_device() != device:
        _elsewhere(where, ws.get_device())
    return ws.data_ptr(), ws.nbytes


def dr_qmatmul(a: QMatrix, b: QMatrix, out, accumulate: bool = False, fast: bool = False, workspace=None,
               stream=None) -> None:
    """out = a b^T (+= with accumulate), out 2-d float32 or bfloat16; fast: DR_FAST_SUMS."""
    addr, kind, rows, cols, step = _dense_rows(out, "dr_qmatmul out")
    if rows != a.rows or cols != b.rows:
        raise ValueError(f"dr_qmatmul out: {rows} x {cols}, the product is {a.rows} x {b.rows}")
    device = a.device
    if not device == b.device == out.get_device():
        _elsewhere("dr_qmatmul", device, b.device, out.get_device())
    _check(_lib.dr_qmatmul(a.ref, b.ref, addr, kind, step,
                           (DR_ACCUMULATE if accumulate else 0) | (DR_FAST_SUMS if fast else 0),
                           *_workspace(workspace, device, "dr_qmatmul workspace"),
                           _stream_on(device, stream, "dr_qmatmul")), "dr_qmatmul")


def _bytes(call, where: str, *args) -> int:
    n = ctypes.c_uint64()
    _check(call(*args, ctypes.byref(n)), where)
    return n.value


def dr_qmatmul_workspace(m: int, n: int, k: int) -> int:
    """Bytes of workspace that an m x n product over k columns needs."""
    return _bytes(_lib.dr_qmatmul_workspace, "dr_qmatmul_workspace", int(m), int(n), int(k))


def dr_qlinear(x, w: QMatrix, out, fast: bool = False, workspace=None, stream=None) -> None:
    """out = x w^T with x (2-d float32 or bfloat16) quantized in blocks of 1 x 128; fast: DR_FAST_SUMS."""
    addr, kind, rows, cols, step = _dense_rows(x, "dr_qlinear x")
    oaddr, okind, orows, ocols, ostep = _dense_rows(out, "dr_qlinear out")
    if cols != w.cols or orows != rows or ocols != w.rows:
        raise ValueError(f"dr_qlinear: x {rows} x {cols}, w {w.rows} x {w.cols}, out {orows} x {ocols}")
    device = w.device
    if not device == x.get_device() == out.get_device():
        _elsewhere("dr_qlinear", x.get_device(), device, out.get_device())
    _check(_lib.dr_qlinear(addr, kind, rows, step, w.ref, oaddr, okind, ostep, DR_FAST_SUMS if fast else 0,
                           *_workspace(workspace, device, "dr_qlinear workspace"),
                           _stream_on(device, stream, "dr_qlinear")), "dr_qlinear")


def dr_qlinear_workspace(m: int, w: QMatrix) -> int:
    """Bytes of workspace that dr_qlinear needs for m rows and these weights."""
    return _bytes(_lib.dr_qlinear_workspace, "dr_qlinear_workspace", int(m), w.rows, w.cols)


# ------------------------------------------------------------------ the gated feed-forward block
def dr_qgated(x, w: QMatrix, out, act: int = DR_ACT_SILU, fast: bool = False, workspace=None, stream=None) -> None:
    """out = act(x w_gate^T) * (x w_up^T) with w = [w_gate; w_up] and x (2-d float32 or bfloat16) quantized in blocks of
    1 x 128; fast: DR_FAST_SUMS."""
    addr, kind, rows, cols, step = _dense_rows(x, "dr_qgated x")
    oaddr, okind, orows, ocols, ostep = _dense_rows(out, "dr_qgated out")
    if cols != w.cols or orows != rows or 2 * ocols != w.rows:
        raise ValueError(f"dr_qgated: x {rows} x {cols}, w {w.rows} x {w.cols}, out {orows} x {ocols}")
    device = w.device
    if not device == x.get_device() == out.get_device():
        _elsewhere("dr_qgated", x.get_device(), device, out.get_device())
    _check(_lib.dr_qgated(addr, kind, rows, step, w.ref, act, oaddr, okind, ostep, DR_FAST_SUMS if fast else 0,
                          *_workspace(workspace, device, "dr_qgated workspace"),
                          _stream_on(device, stream, "dr_qgated")), "dr_qgated")


def dr_qgated_workspace(m: int, w: QMatrix) -> int:
    """Bytes of workspace that dr_qgated needs for m rows and these weights."""
    return _bytes(_lib.dr_qgated_workspace, "dr_qgated_workspace", int(m), w.rows // 2, w.cols)


def dr_qgated_save(x: QMatrix, w: QMatrix, h: QMatrix, gate: QMatrix | None = None, up: QMatrix | None = None,
                   act: int = DR_ACT_SILU, fast: bool = False, workspace=None, stream=None) -> None:
    """h = act(x w_gate^T) * (x w_up^T) in 8 bits, and the halves of x w^T as the checkpoint for dr_gated_backward;
    fast: DR_FAST_SUMS."""
    device = x.device
    if not device == w.device == h.device == (gate or x).device == (up or x).device:
        _elsewhere("dr_qgated_save", *[q.device for q in (x, w, h, gate, up) if q])
    _check(_lib.dr_qgated_save(x.ref, w.ref, act, h.ref, gate and gate.ref, up and up.ref, DR_FAST_SUMS if fast else 0,
                               *_workspace(workspace, device, "dr_qgated_save workspace"),
                               _stream_on(device, stream, "dr_qgated_save")), "dr_qgated_save")


def dr_qgated_save_workspace(m: int, w: QMatrix) -> int:
    """Bytes of workspace that dr_qgated_save needs for m rows and these weights."""
    return _bytes(_lib.dr_qgated_save_workspace, "dr_qgated_save_workspace", int(m), w.rows // 2, w.cols)


def dr_gated_backward(dh, gate: QMatrix, up: QMatrix, d: QMatrix | None = None, dt: QMatrix | None = None,
                      ht: QMatrix | None = None, act: int = DR_ACT_SILU, stream=None) -> None:
    """From dh (2-d float32 or bfloat16) and the checkpoint: d = [dgate dup], its transpose dt, and ht, the transpose of
    act(gate) * up."""
    addr, kind, rows, cols, step = _dense_rows(dh, "dr_gated_backward dh")
    if rows != gate.rows or cols != gate.cols:
        raise ValueError(f"dr_gated_backward: dh {rows} x {cols}, gate {gate.rows} x {gate.cols}")
    device = gate.device
    if not device == up.device == dh.get_device() == (d or gate).device == (dt or gate).device == (ht or gate).device:
        _elsewhere("dr_gated_backward", dh.get_device(), *[q.device for q in (gate, up, d, dt, ht) if q])
    _check(_lib.dr_gated_backward(addr, kind, step, gate.ref, up.ref, act, d and d.ref, dt and dt.ref, ht and ht.ref,
                                  _stream_on(device, stream, "dr_gated_backward")), "dr_gated_backward")


def dr_qtranspose(src: QMatrix, qt: QMatrix, stream=None) -> None:
    """qt = the transpose of src, quantized anew in blocks of 1 x 128."""
    if src.device != qt.device:
        _elsewhere("dr_qtranspose", src.device, qt.device)
    _check(_lib.dr_qtranspose(src.ref, qt.ref, _stream_on(src.device, stream, "dr_qtranspose")), "dr_qtranspose")


# ------------------------------------------------------------------ gradients
class GradList:
    """The gradients of a model and where their scaled values go (outs None: in place), any shapes: the list that
    the dr_grad_* calls take.  Keeps the tensors."""

    __slots__ = ("grads", "outs", "c", "count")

    def __init__(self, grads: Sequence, outs: Sequence | None = None):
        self.grads, self.outs = tuple(grads), tuple(grads if outs is None else outs)
        if len(self.outs) != len(self.grads):
            raise ValueError(f"GradList: {len(self.grads)} gradients, {len(self.outs)} outputs")
        self.count = len(self.grads)
        self.c = (dr_grad * max(self.count, 1))()
        for i, (g, o) in enumerate(zip(self.grads, self.outs)):
            for t in (g, o):
                if not t.is_cuda or not t.is_contiguous():
                    raise ValueError(f"GradList[{i}]: expected a dense device tensor")
            if g.numel() != o.numel():
                raise ValueError(f"GradList[{i}]: {g.numel()} elements to {o.numel()}")
            self.c[i] = dr_grad(g.data_ptr(), o.data_ptr(), g.numel(), _type(g, f"GradList[{i}]"),
                                _type(o, f"GradList[{i}]"))


def dr_grad_workspace() -> int:
    """Bytes of workspace that dr_grad_norm and dr_grad_clip need."""
    return _bytes(_lib.dr_grad_workspace, "dr_grad_workspace")


_GRAD_WORKSPACE = dr_grad_workspace()


def _grad_space(ws, where: str) -> int:
    return _buf(ws, _GRAD_WORKSPACE, where, True)


def dr_grad_norm(grads: GradList, workspace, sum_squares=None, norm=None, stream=None) -> None:
    """sum_squares (one float64) and norm (one float32) of all gradients, on the device."""
    _check(_lib.dr_grad_norm(grads.c, grads.count, _grad_space(workspace, "dr_grad_norm workspace"),
                             _buf(sum_squares, 8, "dr_grad_norm sum_squares", True),
                             _buf(norm, 4, "dr_grad_norm norm", True), _stream(stream)), "dr_grad_norm")


def dr_grad_scale(grads: GradList, sum_squares, max_norm: float, norm_out=None, stream=None) -> None:
    """Every gradient times min(1, max_norm / (norm + 1e-6)), with the norm of sum_squares (one float64)."""
    _check(_lib.dr_grad_scale(grads.c, grads.count, _buf(sum_squares, 8, "dr_grad_scale sum_squares", True),
                              float(max_norm), _buf(norm_out, 4, "dr_grad_scale norm_out", True), _stream(stream)),
           "dr_grad_scale")


def dr_grad_clip(grads: GradList, max_norm: float, norm_out, workspace, stream=None) -> None:
    """dr_grad_norm and dr_grad_scale in one call; norm_out may be None."""
    _check(_lib.dr_grad_clip(grads.c, grads.count, float(max_norm), _grad_space(workspace, "dr_grad_clip workspace"),
                             _buf(norm_out, 4, "dr_grad_clip norm_out", True), _stream(stream)), "dr_grad_clip")


def dr_last_error() -> str:
    return _lib.dr_last_error().decode(errors="replace")


def library_path() -> str:
    return _LIB_PATH
