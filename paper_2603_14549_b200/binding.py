"""ctypes binding of libasap.so: same names as the C entry points, argument marshalling only.

Every step of the prune path runs in the CUDA library.  PyTorch is used here for device
memory (the tensors whose data pointers are handed to the library) and for the current
stream.  There is no CPU fallback: if the library is missing or was not built, loading
raises.
"""
from __future__ import annotations

import ctypes as C
import dataclasses
import math
import os
from typing import Optional

import torch

_HERE = os.path.dirname(os.path.abspath(__file__))
LIB_PATH = os.path.join(_HERE, "libasap.so")

ASAP_OK = 0
STATUS_NAMES = {0: "ASAP_OK", -1: "ASAP_ERR_INVALID", -2: "ASAP_ERR_ALIGN", -3: "ASAP_ERR_WORKSPACE",
                -4: "ASAP_ERR_CUDA", -5: "ASAP_ERR_UNSUPPORTED", -6: "ASAP_ERR_DEVICE"}

EXPORTS = ("asap_init", "asap_score", "asap_select", "asap_merge", "asap_prune_step", "asap_check",
           "asap_last_error", "asap_launch_count", "asap_free", "asap_profile", "asap_profile_read", "asap_debug_wait_limit", "asap_select_static", "asap_compact_kv",
           "asap_consolidate", "asap_consolidate_scratch_bytes", "asap_attention", "asap_attention_scratch_bytes",
           "asap_rope_make", "asap_rope", "asap_cache_attention", "asap_cache_attention_scratch_bytes", "asap_cache_evict",
           "asap_cache_slot")
DTYPES = {torch.bfloat16: 0, torch.float16: 1}
ROPE_SCALINGS = {"none": 0, "linear": 1, "ntk": 2, "yarn": 3, "bands": 4}


class AsapError(RuntimeError):
    def __init__(self, status: int, text: str):
        super().__init__(f"{STATUS_NAMES.get(status, status)}: {text}")
        self.status = status


class CInputs(C.Structure):
    _fields_ = [("B", C.c_int32), ("H", C.c_int32), ("head_dim", C.c_int32), ("D", C.c_int32),
                ("total_tokens", C.c_int32), ("min_vis", C.c_int32), ("max_vis", C.c_int32),
                ("max_seq", C.c_int32), ("max_rank", C.c_int32),
                ("cu_seqlens", C.c_void_p), ("vis_start", C.c_void_p), ("vis_len", C.c_void_p),
                ("text_start", C.c_void_p), ("text_len", C.c_void_p), ("rank_start", C.c_void_p),
                ("rank_len", C.c_void_p), ("q", C.c_void_p), ("k", C.c_void_p), ("hidden", C.c_void_p),
                ("pos_ids", C.c_void_p)]


class CParams(C.Structure):
    _fields_ = [("keep_k", C.c_int32), ("lambda_max", C.c_float), ("eps", C.c_float),
                ("sim_threshold", C.c_float), ("mask_enable", C.c_int32), ("merge_enable", C.c_int32),
                ("per_head_mask", C.c_int32)]


class CKernelTime(C.Structure):
    _fields_ = [("name", C.c_char * 32), ("launches", C.c_uint64), ("total_ms", C.c_double)]


class COutputs(C.Structure):
    _fields_ = [("mass", C.c_void_p), ("salience", C.c_void_p), ("mask_log", C.c_void_p),
                ("rank_score", C.c_void_p), ("keep_idx", C.c_void_p), ("drop_idx", C.c_void_p),
                ("assign", C.c_void_p), ("best_sim", C.c_void_p), ("out_hidden", C.c_void_p),
                ("out_pos", C.c_void_p), ("src_row", C.c_void_p), ("out_cu_seqlens", C.c_void_p),
                ("out_rows_capacity", C.c_int32), ("mask_log_heads", C.c_void_p)]


class CRopePlan(C.Structure):
    _fields_ = [("n_pairs", C.c_int32), ("interleaved", C.c_int32), ("magnitude", C.c_float), ("reserved", C.c_int32),
                ("turns", C.c_uint64 * 128)]


class CRopeTensor(C.Structure):
    _fields_ = [("src", C.c_void_p), ("dst", C.c_void_p), ("heads", C.c_int32), ("rotate", C.c_int32), ("mapped", C.c_int32),
                ("reserved", C.c_int32), ("src_row", C.c_int64), ("src_head", C.c_int64), ("dst_row", C.c_int64),
                ("dst_head", C.c_int64)]


class CRopeArgs(C.Structure):
    _fields_ = [("n_rows", C.c_int32), ("head_dim", C.c_int32), ("dtype", C.c_int32), ("inverse", C.c_int32),
                ("n_tensors", C.c_int32), ("dst_rows", C.c_int32), ("pos", C.c_void_p), ("dst_map", C.c_void_p),
                ("tensors", C.POINTER(CRopeTensor))]


class CCacheAttentionArgs(C.Structure):
    _fields_ = [("B", C.c_int32), ("H", C.c_int32), ("kv_heads", C.c_int32), ("head_dim", C.c_int32), ("dtype", C.c_int32),
                ("n_q", C.c_int32), ("max_q", C.c_int32), ("max_len", C.c_int32), ("max_prefix", C.c_int32),
                ("n_groups", C.c_int32), ("cache_rows", C.c_int32), ("scale", C.c_float), ("q_row", C.c_int64),
                ("q_head", C.c_int64), ("out_row", C.c_int64), ("out_head", C.c_int64), ("kv_row", C.c_int64),
                ("kv_head", C.c_int64), ("q_cu", C.c_void_p), ("start", C.c_void_p), ("len", C.c_void_p),
                ("group_cu", C.c_void_p), ("prefix_start", C.c_void_p), ("prefix_len", C.c_void_p), ("q", C.c_void_p),
                ("k", C.c_void_p), ("v", C.c_void_p), ("out", C.c_void_p), ("lse", C.c_void_p), ("weights", C.c_void_p)]


class CCacheEvictArgs(C.Structure):
    _fields_ = [("B", C.c_int32), ("max_len", C.c_int32), ("keep", C.c_int32), ("sink", C.c_int32), ("recent", C.c_int32),
                ("rows", C.c_int32), ("dst_rows", C.c_int32), ("n_tensors", C.c_int32), ("row_bytes", C.c_size_t),
                ("start", C.c_void_p), ("len", C.c_void_p), ("dst_start", C.c_void_p), ("weights", C.c_void_p),
                ("pos", C.c_void_p), ("keep_idx", C.c_void_p), ("new_len", C.c_void_p), ("dst_weights", C.c_void_p),
                ("dst_pos", C.c_void_p), ("src", C.POINTER(C.c_void_p)), ("dst", C.POINTER(C.c_void_p))]


class CCacheSlotArgs(C.Structure):
    _fields_ = [("B", C.c_int32), ("capacity", C.c_int32), ("sink", C.c_int32), ("recent", C.c_int32), ("rows", C.c_int32),
                ("start", C.c_void_p), ("len", C.c_void_p), ("weights", C.c_void_p), ("pos", C.c_void_p),
                ("new_pos", C.c_void_p), ("row", C.c_void_p)]


_lib = None


def load_library() -> C.CDLL:
    """Loads libasap.so; raises if it has not been built (python -m paper_2603_14549_b200.build)."""
    global _lib
    if _lib is not None:
        return _lib
    if not os.path.exists(LIB_PATH):
        raise FileNotFoundError(
            f"{LIB_PATH} is missing: build it with `python paper_2603_14549_b200/build.py` "
            "(there is no fallback path)")
    lib = C.CDLL(LIB_PATH)
    lib.asap_init.restype = C.c_int
    lib.asap_init.argtypes = [C.POINTER(C.c_void_p), C.c_int, C.c_size_t, C.c_int, C.c_int, C.c_int, C.c_size_t]
    for name in ("asap_score", "asap_prune_step"):
        fn = getattr(lib, name)
        fn.restype = C.c_int
        fn.argtypes = [C.c_void_p, C.POINTER(CInputs), C.POINTER(CParams), C.POINTER(COutputs), C.c_void_p]
    lib.asap_select.restype = C.c_int
    lib.asap_select.argtypes = [C.c_void_p, C.POINTER(CInputs), C.POINTER(CParams), C.c_void_p,
                                C.POINTER(COutputs), C.c_void_p]
    lib.asap_merge.restype = C.c_int
    lib.asap_merge.argtypes = [C.c_void_p, C.POINTER(CInputs), C.POINTER(CParams), C.c_void_p, C.c_void_p,
                               C.c_void_p, C.POINTER(COutputs), C.c_void_p]
    lib.asap_select_static.restype = C.c_int
    lib.asap_select_static.argtypes = [C.POINTER(CInputs), C.POINTER(CParams), C.c_void_p, C.c_void_p,
                                       C.c_void_p, C.c_void_p, C.c_void_p]
    lib.asap_compact_kv.restype = C.c_int
    lib.asap_compact_kv.argtypes = [C.c_void_p, C.c_void_p, C.c_void_p, C.c_int32, C.c_int32, C.c_size_t, C.c_int32,
                                    C.POINTER(C.c_void_p), C.POINTER(C.c_void_p), C.c_void_p]
    lib.asap_consolidate_scratch_bytes.restype = C.c_size_t
    lib.asap_consolidate_scratch_bytes.argtypes = [C.c_int32, C.c_int32]
    lib.asap_consolidate.restype = C.c_int
    lib.asap_consolidate.argtypes = [C.c_void_p, C.POINTER(CInputs), C.POINTER(CParams), C.c_void_p, C.c_void_p,
                                     C.c_void_p, C.c_void_p, C.c_void_p, C.c_size_t, C.POINTER(COutputs),
                                     C.c_void_p, C.c_void_p]
    lib.asap_attention_scratch_bytes.restype = C.c_size_t
    lib.asap_attention_scratch_bytes.argtypes = [C.c_int32, C.c_int32]
    lib.asap_attention.restype = C.c_int
    lib.asap_attention.argtypes = [C.c_void_p, C.POINTER(CInputs), C.POINTER(CParams), C.c_void_p, C.c_void_p,
                                   C.c_void_p, C.c_size_t, C.c_void_p, C.c_void_p]
    lib.asap_rope_make.restype = C.c_int
    lib.asap_rope_make.argtypes = [C.POINTER(CRopePlan), C.c_int32, C.c_int32, C.c_int32, C.c_double, C.c_double, C.c_double,
                                   C.c_double, C.c_double]
    lib.asap_rope.restype = C.c_int
    lib.asap_rope.argtypes = [C.c_void_p, C.c_void_p, C.c_void_p, C.c_void_p]
    lib.asap_cache_attention_scratch_bytes.restype = C.c_size_t
    lib.asap_cache_attention_scratch_bytes.argtypes = [C.c_void_p, C.c_void_p]
    lib.asap_cache_attention.restype = C.c_int
    lib.asap_cache_attention.argtypes = [C.c_void_p, C.c_void_p, C.c_void_p, C.c_size_t, C.c_void_p]
    for name in ("asap_cache_evict", "asap_cache_slot"):
        fn = getattr(lib, name)
        fn.restype = C.c_int
        fn.argtypes = [C.c_void_p, C.c_void_p, C.c_void_p]
    lib.asap_check.restype = C.c_int
    lib.asap_check.argtypes = [C.c_void_p, C.c_void_p]
    lib.asap_last_error.restype = C.c_char_p
    lib.asap_last_error.argtypes = [C.c_void_p]
    lib.asap_launch_count.restype = C.c_uint64
    lib.asap_launch_count.argtypes = [C.c_void_p]
    lib.asap_profile.restype = C.c_int
    lib.asap_profile.argtypes = [C.c_void_p, C.c_int]
    lib.asap_debug_wait_limit.restype = C.c_int
    lib.asap_debug_wait_limit.argtypes = [C.c_void_p, C.c_longlong]
    lib.asap_profile_read.restype = C.c_int
    lib.asap_profile_read.argtypes = [C.c_void_p, C.POINTER(CKernelTime), C.c_int]
    lib.asap_free.restype = None
    lib.asap_free.argtypes = [C.c_void_p]
    _lib = lib
    return lib


def _ptr(t: Optional[torch.Tensor]) -> Optional[int]:
    return None if t is None else t.data_ptr()


@dataclasses.dataclass
class Inputs:
    """Device tensors plus the host-known sizes of one packed batch."""
    B: int
    H: int
    head_dim: int
    D: int
    total_tokens: int
    min_vis: int
    max_vis: int
    max_seq: int
    max_rank: int
    cu_seqlens: torch.Tensor
    vis_start: torch.Tensor
    vis_len: torch.Tensor
    text_start: torch.Tensor
    text_len: torch.Tensor
    q: Optional[torch.Tensor]
    k: Optional[torch.Tensor]
    hidden: Optional[torch.Tensor]
    pos_ids: Optional[torch.Tensor]
    rank_start: Optional[torch.Tensor] = None
    rank_len: Optional[torch.Tensor] = None

    def c_struct(self) -> CInputs:
        return CInputs(self.B, self.H, self.head_dim, self.D, self.total_tokens, self.min_vis, self.max_vis,
                       self.max_seq, self.max_rank, _ptr(self.cu_seqlens), _ptr(self.vis_start),
                       _ptr(self.vis_len), _ptr(self.text_start), _ptr(self.text_len), _ptr(self.rank_start),
                       _ptr(self.rank_len), _ptr(self.q), _ptr(self.k), _ptr(self.hidden), _ptr(self.pos_ids))


def make_inputs(batch, device, rank_start=None, rank_len=None) -> Inputs:
    """Moves a workloads.Batch to `device` and derives the host-known bounds."""
    dev = lambda t: t.to(device, non_blocking=False).contiguous()
    seq = (batch.cu_seqlens[1:] - batch.cu_seqlens[:-1])
    rl = batch.text_len if rank_len is None else torch.as_tensor(rank_len, dtype=torch.int32)
    rs = None if rank_start is None else torch.as_tensor(rank_start, dtype=torch.int32)
    return Inputs(B=batch.B, H=batch.H, head_dim=batch.head_dim, D=batch.D, total_tokens=batch.total,
                  min_vis=int(batch.vis_len.min()), max_vis=int(batch.vis_len.max()), max_seq=int(seq.max()),
                  max_rank=int(rl.max()), cu_seqlens=dev(batch.cu_seqlens), vis_start=dev(batch.vis_start),
                  vis_len=dev(batch.vis_len), text_start=dev(batch.text_start), text_len=dev(batch.text_len),
                  q=dev(batch.q), k=dev(batch.k), hidden=dev(batch.hidden), pos_ids=dev(batch.pos_ids),
                  rank_start=None if rs is None else dev(rs),
                  rank_len=None if rank_len is None else dev(rl))


@dataclasses.dataclass
class Params:
    keep_k: int
    lambda_max: float = 1.0
    eps: float = 1e-6
    sim_threshold: float = -math.inf
    mask_enable: bool = True
    merge_enable: bool = True
    per_head_mask: bool = False

    def c_struct(self) -> CParams:
        return CParams(self.keep_k, self.lambda_max, self.eps, self.sim_threshold, int(self.mask_enable),
                       int(self.merge_enable), int(self.per_head_mask))


@dataclasses.dataclass
class Outputs:
    mass: torch.Tensor
    salience: torch.Tensor
    mask_log: torch.Tensor
    rank_score: torch.Tensor
    keep_idx: torch.Tensor
    drop_idx: torch.Tensor
    assign: torch.Tensor
    best_sim: Optional[torch.Tensor]
    out_hidden: torch.Tensor
    out_pos: torch.Tensor
    src_row: torch.Tensor
    out_cu_seqlens: torch.Tensor
    mask_log_heads: Optional[torch.Tensor] = None

    def c_struct(self) -> COutputs:
        return COutputs(_ptr(self.mass), _ptr(self.salience), _ptr(self.mask_log), _ptr(self.rank_score),
                        _ptr(self.keep_idx), _ptr(self.drop_idx), _ptr(self.assign), _ptr(self.best_sim),
                        _ptr(self.out_hidden), _ptr(self.out_pos), _ptr(self.src_row),
                        _ptr(self.out_cu_seqlens), int(self.out_hidden.shape[0]), _ptr(self.mask_log_heads))


def alloc_outputs(inp: Inputs, keep_k: int, best_sim: bool = True, fill: bool = False,
                  per_head: bool = False) -> Outputs:
    """Caller-owned output tensors with the capacities the header states."""
    dev = inp.cu_seqlens.device
    B, mv = inp.B, inp.max_vis
    nd = max(mv - keep_k, 0)
    rows = inp.total_tokens - B * (inp.min_vis - keep_k)
    f32 = lambda *s: (torch.full(s, float("nan"), dtype=torch.float32, device=dev) if fill
                      else torch.empty(s, dtype=torch.float32, device=dev))
    i32 = lambda *s: (torch.full(s, -7, dtype=torch.int32, device=dev) if fill
                      else torch.empty(s, dtype=torch.int32, device=dev))
    return Outputs(mass=f32(B, mv), salience=f32(B, mv), mask_log=f32(B, mv), rank_score=f32(B, mv),
                   keep_idx=i32(B, keep_k), drop_idx=i32(B, nd), assign=i32(B, nd),
                   best_sim=f32(B, nd) if best_sim else None,
                   out_hidden=torch.zeros(rows, inp.D, dtype=torch.bfloat16, device=dev) if fill
                   else torch.empty(rows, inp.D, dtype=torch.bfloat16, device=dev),
                   out_pos=i32(rows), src_row=i32(rows), out_cu_seqlens=i32(B + 1),
                   mask_log_heads=f32(B, inp.H, mv) if per_head else None)


def _stream(stream) -> int:
    if stream is None:
        return torch.cuda.current_stream().cuda_stream
    return stream.cuda_stream if hasattr(stream, "cuda_stream") else int(stream)


_raw_stream = getattr(torch._C, "_cuda_getCurrentRawStream", None)     # (the stream's handle without an object around it: 1 us less a call)


def _stream_of(device, stream) -> int:
    """The given stream, or the current one of the device that holds the tensors."""
    if stream is None:
        return _raw_stream(device.index) if _raw_stream is not None else torch.cuda.current_stream(device).cuda_stream
    return stream.cuda_stream if hasattr(stream, "cuda_stream") else int(stream)


def _raise(ctx, status: int):
    if status != ASAP_OK:
        text = load_library().asap_last_error(ctx)
        raise AsapError(status, text.decode() if text else "")


# ------------------------------------------------------------------------------------ entry points
def asap_init(device: int, max_total_tokens: int, max_B: int, max_H: int, max_D: int,
              max_keep_rows: int = 0) -> C.c_void_p:
    lib = load_library()
    ctx = C.c_void_p()
    st = lib.asap_init(C.byref(ctx), int(device), int(max_total_tokens), int(max_B), int(max_H), int(max_D),
                       int(max_keep_rows))
    _raise(None, st)
    return ctx


def asap_score(ctx, inp: Inputs, params: Params, out: Outputs, stream=None) -> None:
    ci, cp, co = inp.c_struct(), params.c_struct(), out.c_struct()
    _raise(ctx, load_library().asap_score(ctx, C.byref(ci), C.byref(cp), C.byref(co), _stream(stream)))


def asap_select(ctx, inp: Inputs, params: Params, rank_score: torch.Tensor, out: Outputs, stream=None) -> None:
    ci, cp, co = inp.c_struct(), params.c_struct(), out.c_struct()
    _raise(ctx, load_library().asap_select(ctx, C.byref(ci), C.byref(cp), _ptr(rank_score), C.byref(co),
                                           _stream(stream)))


def asap_select_static(inp: Inputs, params: Params, rank_score: torch.Tensor, keep_idx: torch.Tensor,
                       drop_idx: Optional[torch.Tensor], device_status: Optional[torch.Tensor] = None,
                       stream=None) -> None:
    """Top-k selection without a context: the library's fixed device array is the scratch, so
    nothing is allocated.  Works on the current CUDA device; B <= 64, B * max_vis <= 262144."""
    ci, cp = inp.c_struct(), params.c_struct()
    _raise(None, load_library().asap_select_static(C.byref(ci), C.byref(cp), _ptr(rank_score), _ptr(keep_idx),
                                                   _ptr(drop_idx), _ptr(device_status), _stream(stream)))


def asap_merge(ctx, inp: Inputs, params: Params, salience: torch.Tensor, keep_idx: torch.Tensor,
               drop_idx: torch.Tensor, out: Outputs, stream=None) -> None:
    ci, cp, co = inp.c_struct(), params.c_struct(), out.c_struct()
    _raise(ctx, load_library().asap_merge(ctx, C.byref(ci), C.byref(cp), _ptr(salience), _ptr(keep_idx),
                                          _ptr(drop_idx), C.byref(co), _stream(stream)))


def asap_attention_scratch_bytes(total_tokens: int, D: int) -> int:
    return int(load_library().asap_attention_scratch_bytes(int(total_tokens), int(D)))


def asap_attention(ctx, inp: Inputs, params: Params, mask_log: Optional[torch.Tensor], v: torch.Tensor,
                   scratch: torch.Tensor, out: torch.Tensor, stream=None) -> None:
    """out[i, h, :] = sum_j Softmax_j(q_i.k_j / sqrt(d) + M_ij) v_j; `v`, `out`: bf16 [total_tokens, H, head_dim]."""
    ci, cp = inp.c_struct(), params.c_struct()
    _raise(ctx, load_library().asap_attention(ctx, C.byref(ci), C.byref(cp), _ptr(mask_log), _ptr(v), _ptr(scratch),
                                              int(scratch.numel() * scratch.element_size()), _ptr(out), _stream(stream)))


def asap_consolidate_scratch_bytes(B: int, keep_k: int) -> int:
    return int(load_library().asap_consolidate_scratch_bytes(int(B), int(keep_k)))


def asap_consolidate(ctx, inp: Inputs, params: Params, mass: torch.Tensor, salience: torch.Tensor,
                     keep_idx: torch.Tensor, drop_idx: torch.Tensor, scratch: torch.Tensor, out: Outputs,
                     n_absorbed: Optional[torch.Tensor] = None, stream=None) -> None:
    """`scratch`: a contiguous device tensor of at least asap_consolidate_scratch_bytes(B, keep_k) bytes."""
    ci, cp, co = inp.c_struct(), params.c_struct(), out.c_struct()
    _raise(ctx, load_library().asap_consolidate(
        ctx, C.byref(ci), C.byref(cp), _ptr(mass), _ptr(salience), _ptr(keep_idx), _ptr(drop_idx), _ptr(scratch),
        int(scratch.numel() * scratch.element_size()), C.byref(co), _ptr(n_absorbed), _stream(stream)))


def asap_prune_step(ctx, inp: Inputs, params: Params, out: Outputs, stream=None) -> None:
    ci, cp, co = inp.c_struct(), params.c_struct(), out.c_struct()
    _raise(ctx, load_library().asap_prune_step(ctx, C.byref(ci), C.byref(cp), C.byref(co), _stream(stream)))


def asap_compact_kv(ctx, src_row: torch.Tensor, n_rows: torch.Tensor, src, dst, stream=None) -> None:
    """dst[t][r] = src[t][src_row[r]] for r < n_rows[0]: `src` / `dst` are equally long lists of 2-D device
    tensors (rows x anything, contiguous); `n_rows` is a one-element int32 device tensor (or a view
    such as out_cu_seqlens[B:])."""
    assert len(src) == len(dst) and len(src) > 0
    row_bytes = src[0][0].numel() * src[0].element_size()
    ps = (C.c_void_p * len(src))(*[t.data_ptr() for t in src])
    pd = (C.c_void_p * len(dst))(*[t.data_ptr() for t in dst])
    _raise(ctx, load_library().asap_compact_kv(ctx, _ptr(src_row), _ptr(n_rows), int(min(dst[0].shape[0], src_row.numel())),
                                               int(src[0].shape[0]), int(row_bytes), len(src), ps, pd, _stream(stream)))


# ------------------------------------------------------------------------------------ around the key / value cache
# The arguments of these calls are objects that a program makes once for a set of buffers and passes with every step: they hold
# the tensors and the C struct of their addresses.
def _tensors_ok(device, *tensors) -> None:
    for t in tensors:
        if t is not None and (t.device != device or not t.is_cuda):
            raise ValueError(f"all tensors must be on one CUDA device: {t.device} beside {device}")


def _dense(dtype, **tensors) -> None:
    for name, t in tensors.items():
        if t is not None and (t.dtype != dtype or not t.is_contiguous()):
            raise ValueError(f"{name} must be a contiguous {dtype} tensor")


def _rows_heads(name: str, t: torch.Tensor, dtype) -> None:
    if t.dim() != 3 or t.dtype != dtype or (t.stride(2) != 1 and t.shape[2] > 1):
        raise ValueError(f"{name} must be [rows, heads, head_dim] of {dtype} with contiguous heads")


def asap_rope_make(rot_dim: int, layout: str = "half", theta: float = 10000.0, scaling: str = "none", factor: float = 1.0,
                   original_positions: float = 4096, fast: Optional[float] = None, slow: float = 1.0) -> CRopePlan:
    """Plan of a rotation: `layout` "half" or "interleaved", `scaling` "none", "linear", "ntk", "yarn" or "bands"."""
    if layout not in ("half", "interleaved") or scaling not in ROPE_SCALINGS:
        raise ValueError(f"unknown layout {layout!r} or scaling {scaling!r}")
    plan = CRopePlan()
    fast = (4.0 if scaling == "bands" else 32.0) if fast is None else fast
    _raise(None, load_library().asap_rope_make(C.byref(plan), int(rot_dim), int(layout == "interleaved"), ROPE_SCALINGS[scaling],
                                               float(theta), float(factor), float(original_positions), float(fast), float(slow)))
    return plan


@dataclasses.dataclass
class RopeTensor:
    """One tensor of a rotation: `src`, `dst` [rows, heads, head_dim] with any row and head strides."""
    src: torch.Tensor
    dst: torch.Tensor
    mapped: bool = False
    rotate: bool = True


class RopeArgs:
    def __init__(self, pos: torch.Tensor, tensors, dst_row: Optional[torch.Tensor] = None, inverse: bool = False):
        n, dim = pos.numel(), tensors[0].src.shape[2]
        dtype, self.device = tensors[0].src.dtype, pos.device
        if dtype not in DTYPES:
            raise ValueError(f"unsupported dtype {dtype}")
        _dense(torch.int32, pos=pos, dst_row=dst_row)
        if dst_row is not None and dst_row.numel() != n:
            raise ValueError("dst_row must have one entry per row")
        c = (CRopeTensor * len(tensors))()
        dst_rows = [t.dst.shape[0] for t in tensors if t.mapped]
        for i, t in enumerate(tensors):
            _rows_heads("src", t.src, dtype)
            _rows_heads("dst", t.dst, dtype)
            _tensors_ok(self.device, t.src, t.dst, dst_row)
            if t.src.shape[0] != n or t.src.shape[1:] != t.dst.shape[1:] or t.src.shape[2] != dim or (not t.mapped and t.dst.shape[0] < n):
                raise ValueError(f"tensor {i}: shapes {tuple(t.src.shape)} -> {tuple(t.dst.shape)} for {n} rows of {dim}")
            c[i] = CRopeTensor(_ptr(t.src), _ptr(t.dst), t.src.shape[1], int(t.rotate), int(t.mapped), 0, t.src.stride(0),
                               t.src.stride(1), t.dst.stride(0), t.dst.stride(1))
        self.keep = (pos, dst_row, list(tensors), c)
        self.c = CRopeArgs(n, dim, DTYPES[dtype], int(inverse), len(tensors), min(dst_rows, default=0), _ptr(pos), _ptr(dst_row), c)
        self.ref = C.addressof(self.c)


def asap_rope(ctx, plan: CRopePlan, args: RopeArgs, stream=None) -> None:
    status = (_lib or load_library()).asap_rope(ctx, C.addressof(plan), args.ref, _stream_of(args.device, stream))
    if status:
        _raise(ctx, status)


class CacheAttention:
    """Arguments of asap_cache_attention.  q, out: [n_q, H, 128]; k, v: [cache_rows, kv_heads, 128] of the same strides; start, len,
    q_cu, group_cu, prefix_start, prefix_len: int32; lse: fp32 [n_q, H]; weights: fp32 [cache_rows]."""

    def __init__(self, q, k, v, out, start, len, max_len, q_cu=None, max_q=1, group_cu=None, prefix_start=None, prefix_len=None,
                 max_prefix=0, lse=None, weights=None, scale=0.0):
        if q.dtype not in DTYPES:
            raise ValueError(f"unsupported dtype {q.dtype}")
        for name, t in (("q", q), ("k", k), ("v", v), ("out", out)):
            _rows_heads(name, t, q.dtype)
        _tensors_ok(q.device, q, k, v, out, start, len, q_cu, group_cu, prefix_start, prefix_len, lse, weights)
        _dense(torch.int32, start=start, len=len, q_cu=q_cu, group_cu=group_cu, prefix_start=prefix_start, prefix_len=prefix_len)
        _dense(torch.float32, lse=lse, weights=weights)
        B, groups = start.numel(), 0 if group_cu is None else group_cu.numel() - 1
        if k.shape != v.shape or (k.stride() != v.stride() and k.numel() > 0) or q.shape != out.shape or k.shape[2] != q.shape[2]:
            raise ValueError("k and v must have the same shape and strides, q and out the same shape")
        if len.numel() != B or (q_cu is not None and q_cu.numel() != B + 1) or groups < 0 or any(
                t is None or t.numel() != groups for t in (prefix_start, prefix_len) if groups):
            raise ValueError("start, len: [B]; q_cu: [B + 1]; group_cu: [G + 1]; prefix_start, prefix_len: [G]")
        if (lse is not None and lse.numel() != q.shape[0] * q.shape[1]) or (weights is not None and weights.numel() != k.shape[0]):
            raise ValueError("lse: [n_q, H]; weights: [cache_rows]")
        self.device = q.device
        self.keep = (q, k, v, out, start, len, q_cu, group_cu, prefix_start, prefix_len, lse, weights)
        self.c = CCacheAttentionArgs(B, q.shape[1], k.shape[1], q.shape[2], DTYPES[q.dtype], q.shape[0], max_q, max_len, max_prefix,
                                     groups, k.shape[0], scale, q.stride(0), q.stride(1), out.stride(0), out.stride(1), k.stride(0),
                                     k.stride(1), _ptr(q_cu), _ptr(start), _ptr(len), _ptr(group_cu), _ptr(prefix_start),
                                     _ptr(prefix_len), _ptr(q), _ptr(k), _ptr(v), _ptr(out), _ptr(lse), _ptr(weights))
        self.ref = C.addressof(self.c)


def asap_cache_attention_scratch_bytes(ctx, args: CacheAttention) -> int:
    return int(load_library().asap_cache_attention_scratch_bytes(ctx, args.ref))


def asap_cache_attention(ctx, args: CacheAttention, scratch: torch.Tensor, stream=None) -> None:
    """`scratch`: a contiguous tensor of at least asap_cache_attention_scratch_bytes(ctx, args) bytes on the device of the others."""
    if scratch.device != args.device or not scratch.is_contiguous():
        raise ValueError(f"scratch must be a contiguous tensor on {args.device}")
    status = (_lib or load_library()).asap_cache_attention(ctx, args.ref, scratch.data_ptr(), scratch.nbytes, _stream_of(args.device, stream))
    if status:
        _raise(ctx, status)


class CacheEvict:
    """Arguments of asap_cache_evict.  src, dst: lists of contiguous tensors [rows, ...] and [dst_rows, ...] (the same tensors: in
    place); weights, pos: [rows]; dst_weights, dst_pos: [dst_rows]; keep_idx: int32 [B, keep]; new_len: int32 [B] (may be len)."""

    def __init__(self, start, len, max_len, keep, weights, pos, keep_idx, new_len, src=(), dst=(), dst_start=None, dst_weights=None,
                 dst_pos=None, sink=0, recent=0):
        src, dst = list(src), list(dst)          # (iterables that can be walked once would look empty the second time)
        B, n, rows = start.numel(), 0, weights.numel()
        _tensors_ok(weights.device, start, len, weights, pos, keep_idx, new_len, dst_start, dst_weights, dst_pos, *src, *dst)
        _dense(torch.int32, start=start, len=len, pos=pos, keep_idx=keep_idx, new_len=new_len, dst_start=dst_start, dst_pos=dst_pos)
        _dense(torch.float32, weights=weights, dst_weights=dst_weights)
        dst_rows = [t.shape[0] for t in dst] + [t.numel() for t in (dst_weights, dst_pos) if t is not None] or [rows]
        row_bytes, src_n, dst_n = 0, sum(1 for _ in src), sum(1 for _ in dst)
        for s, d in zip(src, dst):
            if not s.is_contiguous() or not d.is_contiguous() or s.shape[0] != rows or s.shape[1:] != d.shape[1:] or s.dtype != d.dtype:
                raise ValueError("src / dst must be contiguous, src with one row per weight, with rows alike")
            n += 1
            rb = s.stride(0) * s.element_size()
            if n > 1 and rb != row_bytes:
                raise ValueError("all tensors must have rows of the same size")
            row_bytes = rb
        if tuple(keep_idx.shape) != (B, keep) or any(t.numel() != B for t in (len, new_len, dst_start) if t is not None) or any(
                x != dst_rows[0] for x in dst_rows) or (pos is not None and pos.numel() != rows) or n != src_n or n != dst_n:
            raise ValueError("keep_idx: [B, keep]; len, new_len, dst_start: [B]; pos: [rows]; destinations with the same rows; as many src as dst")
        ps = (C.c_void_p * max(n, 1))(*[t.data_ptr() for t in src])
        pd = (C.c_void_p * max(n, 1))(*[t.data_ptr() for t in dst])
        self.device = weights.device
        self.keep = (start, len, weights, pos, keep_idx, new_len, src, dst, dst_start, dst_weights, dst_pos, ps, pd)
        self.c = CCacheEvictArgs(B, max_len, keep, sink, recent, rows, dst_rows[0], n, row_bytes, _ptr(start), _ptr(len), _ptr(dst_start),
                                 _ptr(weights), _ptr(pos), _ptr(keep_idx), _ptr(new_len), _ptr(dst_weights), _ptr(dst_pos), ps, pd)
        self.ref = C.addressof(self.c)


def asap_cache_evict(ctx, args: CacheEvict, stream=None) -> None:
    status = (_lib or load_library()).asap_cache_evict(ctx, args.ref, _stream_of(args.device, stream))
    if status:
        _raise(ctx, status)


class CacheSlot:
    """Arguments of asap_cache_slot: start, len, new_pos, row: int32 [B]; weights: fp32, pos: int32 [rows]."""

    def __init__(self, start, len, capacity, weights, pos, new_pos, row, sink=0, recent=0):
        B = start.numel()
        _tensors_ok(weights.device, start, len, weights, pos, new_pos, row)
        _dense(torch.int32, start=start, len=len, pos=pos, new_pos=new_pos, row=row)
        _dense(torch.float32, weights=weights)
        if any(t.numel() != B for t in (len, new_pos, row)) or pos.numel() != weights.numel():
            raise ValueError("start, len, new_pos, row: [B]; weights, pos: [rows]")
        self.device = weights.device
        self.keep = (start, len, weights, pos, new_pos, row)
        self.c = CCacheSlotArgs(B, capacity, sink, recent, weights.numel(), _ptr(start), _ptr(len), _ptr(weights), _ptr(pos),
                                _ptr(new_pos), _ptr(row))
        self.ref = C.addressof(self.c)


def asap_cache_slot(ctx, args: CacheSlot, stream=None) -> None:
    status = (_lib or load_library()).asap_cache_slot(ctx, args.ref, _stream_of(args.device, stream))
    if status:
        _raise(ctx, status)


def asap_check(ctx, stream=None) -> None:
    _raise(ctx, load_library().asap_check(ctx, _stream(stream)))


def asap_launch_count(ctx) -> int:
    return int(load_library().asap_launch_count(ctx))


def asap_last_error(ctx) -> str:
    text = load_library().asap_last_error(ctx)
    return text.decode() if text else ""


def asap_debug_wait_limit(ctx, cycles: int) -> None:
    _raise(ctx, load_library().asap_debug_wait_limit(ctx, int(cycles)))


def asap_profile(ctx, enable: bool) -> None:
    _raise(ctx, load_library().asap_profile(ctx, int(bool(enable))))


def asap_profile_read(ctx) -> dict:
    """{kernel name: (launches, total_ms)} accumulated since profiling was enabled."""
    buf = (CKernelTime * 32)()
    n = load_library().asap_profile_read(ctx, buf, 32)
    return {buf[i].name.decode(): (int(buf[i].launches), float(buf[i].total_ms)) for i in range(min(n, 32))}


def asap_free(ctx) -> None:
    load_library().asap_free(ctx)
