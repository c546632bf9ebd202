"""ctypes binding of libmla_online.so (argument marshalling only).

Every step runs in the HIP library; PyTorch supplies device memory and the
stream.  Importing this module loads the library and raises if it is missing
or cannot be loaded: there is no fallback implementation.
"""
from __future__ import annotations

import ctypes
import os

import numpy as np
import torch  # loads the HIP runtime the library binds to

HERE = os.path.dirname(os.path.abspath(__file__))
LIB_PATH = os.path.join(HERE, "libmla_online.so")

MLA_OK = 0
MLA_BF16, MLA_F32 = 0, 1
STATUS = {0: "MLA_OK", 1: "MLA_ERR_NULL", 2: "MLA_ERR_SHAPE", 3: "MLA_ERR_UNSUPPORTED",
          4: "MLA_ERR_SEGMENTS", 5: "MLA_ERR_ROWS", 6: "MLA_ERR_WORKSPACE", 7: "MLA_ERR_HIP"}
EXPORTS = ("mla_online_attend_query", "mla_online_attend", "mla_segment_merge", "mla_sliced_oproj_add",
           "mla_online_plan_query", "mla_online_plan", "mla_online_attend_planned",
           "mla_online_attend_planned_noalloc", "mla_sliced_oproj_add_planned",
           "mla_offline_produce_query", "mla_offline_produce", "mla_protected_rows_query", "mla_protected_rows",
           "mla_protected_rows_planned_query", "mla_protected_rows_planned",
           "mla_moe_fanout", "mla_shared_wb", "mla_mx4_quantize", "mla_mx4_dequantize", "mla_shared_wb_mx4",
           "mla_cache_append", "mla_cache_gather", "mla_cache_attend_query", "mla_cache_attend",
           "mla_moe_route", "mla_i8_quantize", "mla_i8_dequantize", "mla_shared_wb_i8", "mla_moe_experts_i8_query",
           "mla_moe_experts_i8", "mla_probe_mfma_bf16", "mla_status_str", "mla_last_error_detail",
           "mla_version")


class MlaError(RuntimeError):
    def __init__(self, status: int, detail: str):
        super().__init__(f"{STATUS.get(status, status)}: {detail}")
        self.status = status
        self.detail = detail


class Geom(ctypes.Structure):
    _fields_ = [("n_heads", ctypes.c_int32), ("n_groups", ctypes.c_int32), ("d_latent", ctypes.c_int32),
                ("d_rope", ctypes.c_int32), ("d_model", ctypes.c_int32), ("n_proj_groups", ctypes.c_int32),
                ("softmax_scale", ctypes.c_float), ("rope_base", ctypes.c_double), ("value_rope", ctypes.c_int32)]


class Segment(ctypes.Structure):
    _fields_ = [("kv_start", ctypes.c_int64), ("length", ctypes.c_int64), ("req_offset", ctypes.c_int64)]


class PlanInfo(ctypes.Structure):
    """mla_plan_info: host description of a plan built by mla_online_plan."""
    _fields_ = [("geom", Geom), ("n_rows", ctypes.c_int64), ("split_keys", ctypes.c_int64),
                ("max_slots", ctypes.c_int64), ("max_parts", ctypes.c_int64), ("n_segs", ctypes.c_int32),
                ("prot_cap", ctypes.c_int32), ("max_items", ctypes.c_int32), ("one_chunk", ctypes.c_int32),
                ("plan_bytes", ctypes.c_size_t), ("ws_bytes", ctypes.c_size_t), ("layout", ctypes.c_int64 * 24),
                ("check", ctypes.c_uint64)]


class ProtectCfg(ctypes.Structure):
    _fields_ = [("query_seg", ctypes.c_int32), ("edge_rows", ctypes.c_int32), ("tail_rows", ctypes.c_int64),
                ("budget", ctypes.c_double)]


class RouteCfg(ctypes.Structure):
    _fields_ = [("scoring", ctypes.c_int32), ("n_groups", ctypes.c_int32), ("top_groups", ctypes.c_int32),
                ("group_best", ctypes.c_int32), ("top_k", ctypes.c_int32), ("min_k", ctypes.c_int32),
                ("renormalize", ctypes.c_int32), ("scale", ctypes.c_float), ("tau", ctypes.c_float)]


class MoeLayer(ctypes.Structure):
    _fields_ = [("d_model", ctypes.c_int32), ("d_ffn", ctypes.c_int32), ("n_experts", ctypes.c_int32),
                ("first_expert", ctypes.c_int32), ("top_k", ctypes.c_int32)]


def _load(path: str = LIB_PATH):
    if not os.path.exists(path):
        raise ImportError(f"{path} is not built; run `python -m paper_2609_07008_amd.build`")
    lib = ctypes.CDLL(path)
    P, I32, I64, SZ = ctypes.c_void_p, ctypes.c_int32, ctypes.c_int64, ctypes.c_size_t
    GP, SP = ctypes.POINTER(Geom), ctypes.POINTER(Segment)
    lib.mla_online_attend_query.argtypes = [GP, SP, I32, P, I32, I64, ctypes.POINTER(I64), ctypes.POINTER(I64),
                                            ctypes.POINTER(SZ)]
    lib.mla_online_attend.argtypes = [GP, SP, I32, P, I32, I64, P, P, P, P, P, P, P, P, P, SZ, P]
    lib.mla_segment_merge.argtypes = [I64, I32, P, P, P, I32, P, P, P]
    lib.mla_sliced_oproj_add.argtypes = [GP, I64, P, P, P, P, I32, P, P, P, P]
    IP = ctypes.POINTER(PlanInfo)
    lib.mla_online_plan_query.argtypes = [GP, SP, I32, I64, I32, IP]
    lib.mla_online_plan.argtypes = [GP, SP, I32, I64, I32, IP, P, SZ, P]
    lib.mla_online_attend_planned.argtypes = [GP, IP, P, P, P, P, P, P, I32, P, P, P, P, P, P, P, SZ, P]
    lib.mla_online_attend_planned_noalloc.argtypes = [GP, IP, P, P, P, P, P, P, I32, P, P, P, P, P, P, P]
    lib.mla_sliced_oproj_add_planned.argtypes = [GP, IP, P, P, P, P, P, P, P, I32, P, P]
    lib.mla_offline_produce_query.argtypes = [GP, SP, I32, ctypes.POINTER(SZ)]
    lib.mla_offline_produce.argtypes = [GP, SP, I32, P, P, P, P, I32, P, P, SZ, P]
    lib.mla_protected_rows_query.argtypes = [SP, I32, ctypes.POINTER(SZ)]
    lib.mla_protected_rows.argtypes = [SP, I32, ctypes.POINTER(ProtectCfg), P, P, P, P, P, SZ, P]
    lib.mla_protected_rows_planned_query.argtypes = [IP, ctypes.POINTER(SZ)]
    lib.mla_protected_rows_planned.argtypes = [IP, P, ctypes.POINTER(ProtectCfg), P, P, P, P, P, SZ, P]
    lib.mla_moe_fanout.argtypes = [I64, I32, P, I32, I32, ctypes.c_float, P, P, P, P, P]
    lib.mla_shared_wb.argtypes = [I64, I32, I32, P, P, I32, P, P]
    lib.mla_mx4_quantize.argtypes = [I64, I32, P, I64, P, P, P]
    lib.mla_mx4_dequantize.argtypes = [I64, I32, P, P, P, I64, P]
    lib.mla_shared_wb_mx4.argtypes = [I64, I32, I32, P, P, P, I32, P, P]
    lib.mla_cache_append.argtypes = [GP, I64, P, I64, P, P, I64, I32, P, P]
    lib.mla_cache_gather.argtypes = [GP, I64, P, I64, I32, P, P, I64, P]
    lib.mla_cache_attend_query.argtypes = [GP, I32, I32, I32, I32, ctypes.POINTER(SZ)]
    lib.mla_cache_attend.argtypes = [GP, I32, I32, P, P, P, P, I32, I64, I32, P, P, P, P, SZ, P]
    lib.mla_moe_route.argtypes = [I64, I32, P, I32, I64, P, ctypes.POINTER(RouteCfg), P, P, P, P, P]
    lib.mla_i8_quantize.argtypes = [I64, I32, P, I64, P, P, P]
    lib.mla_i8_dequantize.argtypes = [I64, I32, P, P, P, I64, P]
    lib.mla_shared_wb_i8.argtypes = [I64, I32, I32, P, P, P, P, I32, P, P]
    LP = ctypes.POINTER(MoeLayer)
    lib.mla_moe_experts_i8_query.argtypes = [LP, I64, I32, ctypes.POINTER(SZ)]
    lib.mla_moe_experts_i8.argtypes = [LP, I64, P, I64, P, P, P, P, P, P, P, I32, P, P, SZ, P]
    lib.mla_probe_mfma_bf16.argtypes = [I32, ctypes.POINTER(ctypes.c_double), P, P]
    for f in ("mla_online_attend_query", "mla_online_attend", "mla_segment_merge", "mla_sliced_oproj_add",
              "mla_online_plan_query", "mla_online_plan", "mla_online_attend_planned",
              "mla_online_attend_planned_noalloc", "mla_sliced_oproj_add_planned", "mla_offline_produce_query",
              "mla_offline_produce", "mla_protected_rows_query", "mla_protected_rows",
              "mla_protected_rows_planned_query", "mla_protected_rows_planned", "mla_moe_fanout", "mla_shared_wb",
              "mla_mx4_quantize", "mla_mx4_dequantize", "mla_shared_wb_mx4", "mla_cache_append", "mla_cache_gather",
              "mla_cache_attend_query", "mla_cache_attend", "mla_moe_route", "mla_i8_quantize", "mla_i8_dequantize",
              "mla_shared_wb_i8", "mla_moe_experts_i8_query", "mla_moe_experts_i8", "mla_probe_mfma_bf16"):
        getattr(lib, f).restype = ctypes.c_int
    lib.mla_status_str.argtypes = [ctypes.c_int]
    lib.mla_status_str.restype = ctypes.c_char_p
    lib.mla_last_error_detail.argtypes = []
    lib.mla_last_error_detail.restype = ctypes.c_char_p
    lib.mla_version.restype = ctypes.c_char_p
    return lib


LIB = _load()


def _check(status: int):
    if status != MLA_OK:
        raise MlaError(status, LIB.mla_last_error_detail().decode())


def _refuse(what: str, status: int = 2):
    raise MlaError(status, what)


def _int32(*values):
    """Refuses numbers that the C ABI's int32 arguments cannot hold (ctypes would pass their lower
    32 bits).  Calls that are made often ask it only of what has a bit past the 31st."""
    for v in values:
        if not -0x80000000 <= v <= 0x7FFFFFFF:
            _refuse(f"{v} does not fit 32 bits", 3)


def make_geom(g) -> Geom:
    """Geometry from any object with the fields of mla_geom."""
    return Geom(int(g.n_heads), int(g.n_groups), int(g.d_latent), int(g.d_rope), int(g.d_model),
                int(g.n_proj_groups), float(g.softmax_scale), float(g.rope_base),
                int(bool(getattr(g, "value_rope", False))))


def head_width(g) -> int:
    """d_v: width of one head output (d_c, or d_c + d_r with a rotary value)."""
    return int(g.d_latent) + (int(g.d_rope) if getattr(g, "value_rope", False) else 0)


def make_segments(segs) -> ctypes.Array:
    segs = np.asarray(segs, dtype=np.int64).reshape(-1, 3)
    arr = (Segment * max(1, segs.shape[0]))()
    for i, (ks, ln, ro) in enumerate(segs):
        arr[i] = Segment(int(ks), int(ln), int(ro))
    return arr, int(segs.shape[0])


def _ptr(t):
    if t is None:
        return None
    if isinstance(t, torch.Tensor):
        return ctypes.c_void_p(t.data_ptr())
    if isinstance(t, np.ndarray):
        return t.ctypes.data_as(ctypes.c_void_p)
    return ctypes.c_void_p(int(t))


def _stream(stream):
    if stream is None:
        stream = torch.cuda.current_stream()
    return ctypes.c_void_p(stream.cuda_stream)


def attend_query(geom, segs, prot_rows, split_keys: int):
    """Host-only size query: (n_slots, n_parts, workspace bytes)."""
    g = make_geom(geom)
    sarr, ns = make_segments(segs)
    prot = np.ascontiguousarray(prot_rows, dtype=np.int32)
    n_slots, n_parts, ws = ctypes.c_int64(), ctypes.c_int64(), ctypes.c_size_t()
    _check(LIB.mla_online_attend_query(ctypes.byref(g), sarr, ns, _ptr(prot), int(prot.shape[0]),
                                       int(split_keys), ctypes.byref(n_slots), ctypes.byref(n_parts),
                                       ctypes.byref(ws)))
    return n_slots.value, n_parts.value, ws.value


def online_attend(geom, segs, prot_rows, split_keys, kv, q_glob, q_loc, part_o, part_lse, part_ptr,
                  part_seg, row_src, workspace, stream=None):
    """Relocation + segment-wise attention (mla_online_attend).  Device tensors in,
    device tensors out; prot_rows is a host int32 array."""
    g = make_geom(geom)
    sarr, ns = make_segments(segs)
    prot = np.ascontiguousarray(prot_rows, dtype=np.int32)
    _check(LIB.mla_online_attend(ctypes.byref(g), sarr, ns, _ptr(prot), int(prot.shape[0]), int(split_keys),
                                 _ptr(kv), _ptr(q_glob), _ptr(q_loc), _ptr(part_o), _ptr(part_lse),
                                 _ptr(part_ptr), _ptr(part_seg), _ptr(row_src), _ptr(workspace),
                                 workspace.numel() * workspace.element_size(), _stream(stream)))


def segment_merge(n_slots, d_latent, part_o, part_lse, part_ptr, out_dtype, out_o, out_lse, stream=None):
    _check(LIB.mla_segment_merge(int(n_slots), int(d_latent), _ptr(part_o), _ptr(part_lse), _ptr(part_ptr),
                                 int(out_dtype), _ptr(out_o), _ptr(out_lse), _stream(stream)))


def sliced_oproj_add(geom, n_rows, o_glob, o_loc, glob_head, prot_rows_d, n_prot, w_o, z_off, z, stream=None):
    g = make_geom(geom)
    gh = np.ascontiguousarray(glob_head, dtype=np.int32)
    _check(LIB.mla_sliced_oproj_add(ctypes.byref(g), int(n_rows), _ptr(o_glob), _ptr(o_loc), _ptr(gh),
                                    _ptr(prot_rows_d), int(n_prot), _ptr(w_o), _ptr(z_off), _ptr(z),
                                    _stream(stream)))


def plan_query(geom, segs, split_keys: int, prot_cap: int) -> PlanInfo:
    """Host-only: the PlanInfo (sizes and bounds) of a plan."""
    g = make_geom(geom)
    sarr, ns = make_segments(segs)
    info = PlanInfo()
    _check(LIB.mla_online_plan_query(ctypes.byref(g), sarr, ns, int(split_keys), int(prot_cap), ctypes.byref(info)))
    return info


def online_plan(geom, segs, split_keys: int, prot_cap: int, plan, stream=None) -> PlanInfo:
    """mla_online_plan: writes the plan image into the device tensor `plan` and
    returns its PlanInfo."""
    g = make_geom(geom)
    sarr, ns = make_segments(segs)
    info = PlanInfo()
    _check(LIB.mla_online_plan(ctypes.byref(g), sarr, ns, int(split_keys), int(prot_cap), ctypes.byref(info),
                               _ptr(plan), plan.numel() * plan.element_size(), _stream(stream)))
    return info


def online_attend_planned(geom, info, plan, prot_rows, n_prot, kv, q_glob, q_loc, out_o, out_lse=None,
                          part_ptr=None, part_seg=None, row_src=None, status=None, workspace=None, stream=None):
    """mla_online_attend_planned: every argument a device tensor (prot_rows int32,
    n_prot int32 [1]); out_o bfloat16 or float32 [info.max_slots, d_v]."""
    g = make_geom(geom)
    out = MLA_BF16 if out_o.dtype == torch.bfloat16 else MLA_F32
    _check(LIB.mla_online_attend_planned(ctypes.byref(g), ctypes.byref(info), _ptr(plan), _ptr(prot_rows),
                                         _ptr(n_prot), _ptr(kv), _ptr(q_glob), _ptr(q_loc), out, _ptr(out_o),
                                         _ptr(out_lse), _ptr(part_ptr), _ptr(part_seg), _ptr(row_src), _ptr(status),
                                         _ptr(workspace), workspace.numel() * workspace.element_size(),
                                         _stream(stream)))


NOALLOC_SCRATCH_BYTES = 16 << 20   # MLA_NOALLOC_SCRATCH_BYTES


def online_attend_planned_noalloc(geom, info, plan, prot_rows, n_prot, kv, q_glob, q_loc, out_o, out_lse=None,
                                  part_ptr=None, part_seg=None, row_src=None, status=None, stream=None):
    """mla_online_attend_planned_noalloc: as online_attend_planned, with the
    library's per-GPU scratch array in place of a workspace (nothing allocated)."""
    g = make_geom(geom)
    out = MLA_BF16 if out_o.dtype == torch.bfloat16 else MLA_F32
    _check(LIB.mla_online_attend_planned_noalloc(ctypes.byref(g), ctypes.byref(info), _ptr(plan), _ptr(prot_rows),
                                                 _ptr(n_prot), _ptr(kv), _ptr(q_glob), _ptr(q_loc), out, _ptr(out_o),
                                                 _ptr(out_lse), _ptr(part_ptr), _ptr(part_seg), _ptr(row_src),
                                                 _ptr(status), _stream(stream)))


def sliced_oproj_add_planned(geom, info, o_glob, o_loc, glob_head, prot_rows, n_prot, w_o, z_off, z, stream=None):
    """mla_sliced_oproj_add_planned: |A| from the device tensor n_prot; z float32
    or bfloat16."""
    g = make_geom(geom)
    gh = np.ascontiguousarray(glob_head, dtype=np.int32)
    zt = MLA_BF16 if z.dtype == torch.bfloat16 else MLA_F32
    _check(LIB.mla_sliced_oproj_add_planned(ctypes.byref(g), ctypes.byref(info), _ptr(o_glob), _ptr(o_loc), _ptr(gh),
                                            _ptr(prot_rows), _ptr(n_prot), _ptr(w_o), _ptr(z_off), zt, _ptr(z),
                                            _stream(stream)))


def offline_produce_query(geom, segs) -> int:
    """Host-only: workspace bytes of mla_offline_produce."""
    g = make_geom(geom)
    sarr, ns = make_segments(segs)
    ws = ctypes.c_size_t()
    _check(LIB.mla_offline_produce_query(ctypes.byref(g), sarr, ns, ctypes.byref(ws)))
    return ws.value


def offline_produce(geom, segs, kv, q_loc, glob_head, w_o, out_dtype, z_off, workspace, stream=None):
    """MLA-Off producer (mla_offline_produce): the Local-head artifact z_off of
    every row.  Device tensors in and out; segs and glob_head are host arrays."""
    g = make_geom(geom)
    sarr, ns = make_segments(segs)
    gh = np.ascontiguousarray(glob_head, dtype=np.int32)
    _check(LIB.mla_offline_produce(ctypes.byref(g), sarr, ns, _ptr(kv), _ptr(q_loc), _ptr(gh), _ptr(w_o),
                                   int(out_dtype), _ptr(z_off), _ptr(workspace),
                                   workspace.numel() * workspace.element_size(), _stream(stream)))


def protected_rows_query(segs) -> int:
    """Host-only: workspace bytes of mla_protected_rows."""
    sarr, ns = make_segments(segs)
    ws = ctypes.c_size_t()
    _check(LIB.mla_protected_rows_query(sarr, ns, ctypes.byref(ws)))
    return ws.value


def protected_rows(segs, query_seg, edge_rows, tail_rows, budget, row_flags, scores, prot_rows, n_prot,
                   workspace, stream=None):
    """The protected token-row set (mla_protected_rows) into the device tensors
    prot_rows [N] int32 and n_prot [1] int32; row_flags and scores are device
    tensors or None."""
    sarr, ns = make_segments(segs)
    cfg = ProtectCfg(int(query_seg), int(edge_rows), int(tail_rows), float(budget))
    _check(LIB.mla_protected_rows(sarr, ns, ctypes.byref(cfg), _ptr(row_flags), _ptr(scores), _ptr(prot_rows),
                                  _ptr(n_prot), _ptr(workspace), workspace.numel() * workspace.element_size(),
                                  _stream(stream)))


def protected_rows_planned_query(info) -> int:
    """Host-only: workspace bytes of mla_protected_rows_planned."""
    ws = ctypes.c_size_t()
    _check(LIB.mla_protected_rows_planned_query(ctypes.byref(info), ctypes.byref(ws)))
    return ws.value


def protected_rows_planned(info, plan, query_seg, edge_rows, tail_rows, budget, row_flags, scores, prot_rows, n_prot,
                           workspace, stream=None):
    """mla_protected_rows_planned: the protected set with the segment table taken
    from the plan image; kernels only."""
    cfg = ProtectCfg(int(query_seg), int(edge_rows), int(tail_rows), float(budget))
    _check(LIB.mla_protected_rows_planned(ctypes.byref(info), _ptr(plan), ctypes.byref(cfg), _ptr(row_flags),
                                          _ptr(scores), _ptr(prot_rows), _ptr(n_prot), _ptr(workspace),
                                          workspace.numel() * workspace.element_size(), _stream(stream)))


def moe_fanout(router, tau, expert_idx, expert_w, fanout, expert_count=None, top_k: int = 6, min_k: int = 3,
               stream=None):
    """Adaptive MoE fanout (mla_moe_fanout) of the device tensor router [N, E]
    float32 into expert_idx [N, top_k] int32, expert_w [N, top_k] float32,
    fanout [N] int32 and, if given, expert_count [E] int32."""
    n, e = (int(router.shape[0]), int(router.shape[1])) if router is not None else (0, 0)
    _int32(e, int(top_k), int(min_k))
    _check(LIB.mla_moe_fanout(n, e, _ptr(router), int(top_k), int(min_k), float(tau), _ptr(expert_idx),
                              _ptr(expert_w), _ptr(fanout), _ptr(expert_count), _stream(stream)))


def shared_wb(z, w_b, y, stream=None):
    """y = W_b z (mla_shared_wb): z [N, d_in] bf16 and w_b [d_out, d_in] bf16 device
    tensors, y [N, d_out] float32 or bfloat16."""
    n, d_in = int(z.shape[0]), int(z.shape[1])
    d_out = int(w_b.shape[0])
    if (d_in | d_out) >> 31:
        _int32(d_in, d_out)
    out = MLA_BF16 if y.dtype == torch.bfloat16 else MLA_F32
    _check(LIB.mla_shared_wb(n, d_in, d_out, _ptr(z), _ptr(w_b), out, _ptr(y), _stream(stream)))


# The calls below take tensors on the current device and check what the C ABI cannot see
# (types, shapes, strides, the device); a refusal raises MlaError like the library's own.
WB_MAX_D_IN, WB_MX4_MAX_ROWS, WB_MX4_MAX_D_OUT = 16384, 1024, 1 << 24   # MLA_WB_MAX_D_IN, MLA_WB_MX4_MAX_ROWS, MLA_WB_MX4_MAX_D_OUT
CACHE_ROW_BYTES = 400   # a row of the paged 4-bit cache: 256 code bytes, 16 scales, 64 bf16


def _device():
    """The current device; None before the first use of one, when no tensor lies on any."""
    return torch.cuda.current_device() if torch.cuda.is_initialized() else None


def _queue(stream, dev) -> int:
    """The handle of stream, or of the current stream of dev (an object for it would cost a
    quarter of a small call)."""
    if stream is None:
        return torch._C._cuda_getCurrentRawStream(dev)
    if stream.device_index != dev:
        _refuse(f"the stream is of device {stream.device_index}, not the current device")
    return stream.cuda_stream


def _tensor(name, t, dev, dtype, shape=None, rows=False):
    """t is a tensor on dev, of dtype and, if given, shape (a tuple); contiguous, or (rows)
    two-dimensional with contiguous rows."""
    if not isinstance(t, torch.Tensor):
        _refuse(f"{name} is not a tensor", 1)
    if t.dtype != dtype:
        _refuse(f"{name} is {t.dtype}, expected {dtype}")
    if t.get_device() != dev:
        _refuse(f"{name} is on {t.device}, not the current device")
    if shape is not None and t.shape != shape:
        _refuse(f"{name} is {tuple(t.shape)}, expected {shape}")
    if rows:
        if t.dim() != 2 or (t.stride(1) != 1 and t.numel() != 0):
            _refuse(f"{name} is {tuple(t.shape)} with strides {t.stride()}")
    elif not t.is_contiguous():
        _refuse(f"{name} is not contiguous")


def check_tensor(name, t, dtype):
    """Refuses what is not a contiguous tensor of dtype on the current device."""
    _tensor(name, t, _device(), dtype)


def _row_stride(t) -> int:
    """Elements between rows; of a single row (whose stride is arbitrary) its width rounded up."""
    return t.stride(0) if t.shape[0] > 1 else -(-t.shape[1] // 8) * 8


def _addr(t):
    return None if t is None else t.data_ptr()


def mx4_quantize(x, codes, scales, stream=None):
    """bf16 rows into the 4-bit format (mla_mx4_quantize): x [N, C] bfloat16 with
    contiguous rows, codes [N, C/2] and scales [N, C/32] uint8, written."""
    dev = _device()
    _tensor("x", x, dev, torch.bfloat16, rows=True)
    n, c = x.shape
    if c >> 31:
        _int32(c)
    _tensor("codes", codes, dev, torch.uint8, (n, c // 2))
    _tensor("scales", scales, dev, torch.uint8, (n, c // 32))
    _check(LIB.mla_mx4_quantize(n, c, _addr(x), _row_stride(x), _addr(codes), _addr(scales), _queue(stream, dev)))


def mx4_dequantize(codes, scales, x, stream=None):
    """The values of codes [N, C/2] and scales [N, C/32] into x [N, C] bfloat16 with
    contiguous rows (mla_mx4_dequantize)."""
    dev = _device()
    _tensor("x", x, dev, torch.bfloat16, rows=True)
    n, c = x.shape
    if c >> 31:
        _int32(c)
    _tensor("codes", codes, dev, torch.uint8, (n, c // 2))
    _tensor("scales", scales, dev, torch.uint8, (n, c // 32))
    _check(LIB.mla_mx4_dequantize(n, c, _addr(codes), _addr(scales), _addr(x), _row_stride(x), _queue(stream, dev)))


def shared_wb_mx4(z, w_codes, w_scales, y, stream=None):
    """y = W_b z with W_b in 4 bits (mla_shared_wb_mx4): z [N, d_in] bfloat16,
    w_codes [d_out, d_in/2] and w_scales [d_out, d_in/32] uint8, y [N, d_out] float32
    or bfloat16."""
    dev = _device()
    _tensor("z", z, dev, torch.bfloat16)
    _tensor("w_codes", w_codes, dev, torch.uint8)
    if z.dim() != 2 or w_codes.dim() != 2 or w_codes.shape[1] * 2 != z.shape[1]:
        _refuse(f"z is {tuple(z.shape)}, w_codes {tuple(w_codes.shape)}")
    n, d_in = z.shape
    d_out = w_codes.shape[0]
    if (d_in | d_out) >> 31:
        _int32(d_in, d_out)
    _tensor("w_scales", w_scales, dev, torch.uint8, (d_out, d_in // 32))
    bf16 = isinstance(y, torch.Tensor) and y.dtype == torch.bfloat16
    _tensor("y", y, dev, torch.bfloat16 if bf16 else torch.float32, (n, d_out))
    _check(LIB.mla_shared_wb_mx4(n, d_in, d_out, _addr(z), _addr(w_codes), _addr(w_scales), MLA_BF16 if bf16 else MLA_F32,
                                 _addr(y), _queue(stream, dev)))


def _cache_pages(cache, dev, page_rows: int) -> int:
    """Pages of a cache tensor [pages, page_rows * CACHE_ROW_BYTES] uint8."""
    _tensor("cache", cache, dev, torch.uint8)
    if cache.dim() != 2 or cache.shape[1] != page_rows * CACHE_ROW_BYTES:
        _refuse(f"cache is {tuple(cache.shape)}, expected [pages, {page_rows} * {CACHE_ROW_BYTES}]")
    return cache.shape[0]


def cache_append(geom, kv, slots, cache, page_rows: int, pos=None, stream=None):
    """Rows of kv [N, d_latent + d_rope] bfloat16 (contiguous rows) into the paged 4-bit
    cache [pages, page_rows * CACHE_ROW_BYTES] uint8 at slots [N] int32, the RoPE part
    turned to pos [N] int32 if given (mla_cache_append)."""
    g, dev = make_geom(geom), _device()
    pages = _cache_pages(cache, dev, page_rows)
    _tensor("kv", kv, dev, torch.bfloat16, rows=True)
    n, d = kv.shape
    if d != g.d_latent + g.d_rope:
        _refuse(f"kv is {tuple(kv.shape)}, expected [N, {g.d_latent + g.d_rope}]")
    _tensor("slots", slots, dev, torch.int32, (n,))
    if pos is not None:
        _tensor("pos", pos, dev, torch.int32, (n,))
    _check(LIB.mla_cache_append(ctypes.byref(g), n, _addr(kv), _row_stride(kv), _addr(pos), _addr(slots), pages, page_rows,
                                _addr(cache), _queue(stream, dev)))


def cache_gather(geom, slots, cache, page_rows: int, kv, stream=None):
    """Rows slots [N] int32 of the cache into kv [N, d_latent + d_rope] bfloat16 with
    contiguous rows (mla_cache_gather); rows whose slot is outside the cache are left as
    they were."""
    g, dev = make_geom(geom), _device()
    pages = _cache_pages(cache, dev, page_rows)
    _tensor("kv", kv, dev, torch.bfloat16, rows=True)
    n, d = kv.shape
    if d != g.d_latent + g.d_rope:
        _refuse(f"kv is {tuple(kv.shape)}, expected [N, {g.d_latent + g.d_rope}]")
    _tensor("slots", slots, dev, torch.int32, (n,))
    _check(LIB.mla_cache_gather(ctypes.byref(g), n, _addr(slots), pages, page_rows, _addr(cache), _addr(kv), _row_stride(kv),
                                _queue(stream, dev)))


def cache_attend_query(geom, n_seqs: int, n_q: int, max_pages: int, page_rows: int) -> int:
    """Host-only: workspace bytes of mla_cache_attend."""
    g = make_geom(geom)
    ws = ctypes.c_size_t()
    _check(LIB.mla_cache_attend_query(ctypes.byref(g), int(n_seqs), int(n_q), int(max_pages), int(page_rows), ctypes.byref(ws)))
    return ws.value


def cache_attend(geom, q, pos, pages, seq_pages, cache, page_rows: int, out_o, out_lse=None, workspace=None, stream=None):
    """Attention of new tokens over the paged 4-bit cache (mla_cache_attend): q
    [B, n_q, H, d_latent + d_rope] bfloat16, pos [B, n_q] int32, pages [B, max_pages, 4]
    int32 (page, rows, req_pos, frame), seq_pages [B] int32, out_o [B, n_q, H, d_latent]
    bfloat16, out_lse [B, n_q, H] float32 or None."""
    g, dev = make_geom(geom), _device()
    n_pages = _cache_pages(cache, dev, page_rows)
    _tensor("q", q, dev, torch.bfloat16)
    _tensor("pages", pages, dev, torch.int32)
    if q.dim() != 4 or q.shape[2] != g.n_heads or q.shape[3] != g.d_latent + g.d_rope:
        _refuse(f"q is {tuple(q.shape)}, expected [B, n_q, {g.n_heads}, {g.d_latent + g.d_rope}]")
    b, n_q, heads, _ = q.shape
    if pages.dim() != 3 or pages.shape[0] != b or pages.shape[2] != 4:
        _refuse(f"pages is {tuple(pages.shape)}, expected [{b}, max_pages, 4]")
    _tensor("pos", pos, dev, torch.int32, (b, n_q))
    _tensor("seq_pages", seq_pages, dev, torch.int32, (b,))
    _tensor("out_o", out_o, dev, torch.bfloat16, (b, n_q, heads, g.d_latent))
    if out_lse is not None:
        _tensor("out_lse", out_lse, dev, torch.float32, (b, n_q, heads))
    _tensor("workspace", workspace, dev, torch.uint8)
    _check(LIB.mla_cache_attend(ctypes.byref(g), b, n_q, _addr(q), _addr(pos), _addr(pages), _addr(seq_pages), pages.shape[1],
                                n_pages, page_rows, _addr(cache), _addr(out_o), _addr(out_lse), _addr(workspace),
                                workspace.numel(), _queue(stream, dev)))


SCORINGS = {"softmax": 0, "sigmoid": 1}   # MLA_SOFTMAX, MLA_SIGMOID


def _route_cfg(top_k, scoring="softmax", n_groups=1, top_groups=1, group_best=1, renormalize=True, scale=1.0, min_k=1, tau=2.0):
    if scoring not in SCORINGS:
        _refuse(f"scoring {scoring!r}, expected one of {sorted(SCORINGS)}")
    if (top_k | n_groups | top_groups | group_best | min_k) >> 31:
        _int32(top_k, n_groups, top_groups, group_best, min_k)
    return RouteCfg(SCORINGS[scoring], n_groups, top_groups, group_best, top_k, min_k, bool(renormalize), scale, tau)


def check_route(n_experts: int, top_k: int, **cfg):
    """Host-only: refuses what mla_moe_route would refuse for these experts and this choice
    (keyword arguments of moe_route)."""
    _int32(int(n_experts))
    _check(LIB.mla_moe_route(0, int(n_experts), None, MLA_F32, int(n_experts), None, ctypes.byref(_route_cfg(int(top_k), **cfg)), None, None, None,
                             None, None))


def moe_route(logits, expert_idx, expert_w, fanout=None, expert_count=None, bias=None, scoring: str = "softmax", n_groups: int = 1,
              top_groups: int = 1, group_best: int = 1, renormalize: bool = True, scale: float = 1.0, min_k: int = 1,
              tau: float = 2.0, stream=None):
    """The experts of token rows (mla_moe_route): logits [N, E] float32 or bfloat16 with
    contiguous rows, bias [E] float32 or None, into expert_idx [N, top_k] int32, expert_w
    [N, top_k] float32 and, if given, fanout [N] and expert_count [E] int32."""
    dev = _device()
    bf16 = isinstance(logits, torch.Tensor) and logits.dtype == torch.bfloat16
    _tensor("logits", logits, dev, torch.bfloat16 if bf16 else torch.float32, rows=True)
    n, e = logits.shape
    if e >> 31:
        _int32(e)
    _tensor("expert_idx", expert_idx, dev, torch.int32)
    if expert_idx.dim() != 2 or expert_idx.shape[0] != n:
        _refuse(f"expert_idx is {tuple(expert_idx.shape)}, expected [{n}, top_k]")
    k = expert_idx.shape[1]
    _tensor("expert_w", expert_w, dev, torch.float32, (n, k))
    if fanout is not None:
        _tensor("fanout", fanout, dev, torch.int32, (n,))
    if expert_count is not None:
        _tensor("expert_count", expert_count, dev, torch.int32, (e,))
    if bias is not None:
        _tensor("bias", bias, dev, torch.float32, (e,))
    cfg = _route_cfg(k, scoring, n_groups, top_groups, group_best, renormalize, scale, min_k, tau)
    _check(LIB.mla_moe_route(n, e, _addr(logits), MLA_BF16 if bf16 else MLA_F32, logits.stride(0) if n > 1 else e, _addr(bias),
                             ctypes.byref(cfg), _addr(expert_idx), _addr(expert_w), _addr(fanout), _addr(expert_count),
                             _queue(stream, dev)))


def i8_quantize(x, codes, scales, stream=None):
    """bf16 rows into 8-bit codes and a scale each (mla_i8_quantize): x [N, C] bfloat16
    with contiguous rows, codes [N, C] int8 and scales [N] float32, written."""
    dev = _device()
    _tensor("x", x, dev, torch.bfloat16, rows=True)
    n, c = x.shape
    if c >> 31:
        _int32(c)
    _tensor("codes", codes, dev, torch.int8, (n, c))
    _tensor("scales", scales, dev, torch.float32, (n,))
    _check(LIB.mla_i8_quantize(n, c, _addr(x), _row_stride(x), _addr(codes), _addr(scales), _queue(stream, dev)))


def i8_dequantize(codes, scales, x, stream=None):
    """The values of codes [N, C] int8 and scales [N] float32 into x [N, C] bfloat16 with
    contiguous rows (mla_i8_dequantize)."""
    dev = _device()
    _tensor("x", x, dev, torch.bfloat16, rows=True)
    n, c = x.shape
    if c >> 31:
        _int32(c)
    _tensor("codes", codes, dev, torch.int8, (n, c))
    _tensor("scales", scales, dev, torch.float32, (n,))
    _check(LIB.mla_i8_dequantize(n, c, _addr(codes), _addr(scales), _addr(x), _row_stride(x), _queue(stream, dev)))


def shared_wb_i8(z_codes, z_scales, w_codes, w_scales, y, stream=None):
    """y = W_b z in 8 bits (mla_shared_wb_i8): z_codes [N, d_in] and w_codes [d_out, d_in]
    int8, z_scales [N] and w_scales [d_out] float32, y [N, d_out] float32 or bfloat16."""
    dev = _device()
    _tensor("z_codes", z_codes, dev, torch.int8)
    _tensor("w_codes", w_codes, dev, torch.int8)
    if z_codes.dim() != 2 or w_codes.dim() != 2 or w_codes.shape[1] != z_codes.shape[1]:
        _refuse(f"z_codes is {tuple(z_codes.shape)}, w_codes {tuple(w_codes.shape)}")
    n, d_in = z_codes.shape
    d_out = w_codes.shape[0]
    if (d_in | d_out) >> 31:
        _int32(d_in, d_out)
    _tensor("z_scales", z_scales, dev, torch.float32, (n,))
    _tensor("w_scales", w_scales, dev, torch.float32, (d_out,))
    bf16 = isinstance(y, torch.Tensor) and y.dtype == torch.bfloat16
    _tensor("y", y, dev, torch.bfloat16 if bf16 else torch.float32, (n, d_out))
    _check(LIB.mla_shared_wb_i8(n, d_in, d_out, _addr(z_codes), _addr(z_scales), _addr(w_codes), _addr(w_scales),
                                MLA_BF16 if bf16 else MLA_F32, _addr(y), _queue(stream, dev)))


def _moe_layer(d_model: int, d_ffn: int, n_experts: int, first_expert: int, top_k: int) -> MoeLayer:
    if (d_model | d_ffn | n_experts | first_expert | top_k) >> 31:
        _int32(d_model, d_ffn, n_experts, first_expert, top_k)
    return MoeLayer(d_model, d_ffn, n_experts, first_expert, top_k)


def moe_experts_i8_query(n_rows: int, d_model: int, d_ffn: int, n_experts: int, top_k: int, y_dtype=torch.bfloat16) -> int:
    """Host-only: workspace bytes of mla_moe_experts_i8."""
    if y_dtype not in (torch.bfloat16, torch.float32):
        _refuse(f"y_dtype {y_dtype}, expected torch.bfloat16 or torch.float32")
    if not 0 <= n_rows < 1 << 63:
        _refuse(f"n_rows = {n_rows}")
    layer = _moe_layer(int(d_model), int(d_ffn), int(n_experts), 0, int(top_k))
    ws = ctypes.c_size_t()
    _check(LIB.mla_moe_experts_i8_query(ctypes.byref(layer), int(n_rows), MLA_BF16 if y_dtype == torch.bfloat16 else MLA_F32,
                                        ctypes.byref(ws)))
    return ws.value


def moe_experts_i8(x, expert_idx, expert_w, w_gate_up, s_gate_up, w_down, s_down, y, workspace, fanout=None, first_expert: int = 0,
                   stream=None):
    """The experts of an MoE layer in 8 bits (mla_moe_experts_i8): x [N, d_model] bfloat16
    with contiguous rows, expert_idx [N, top_k] int32, expert_w [N, top_k] float32, fanout [N]
    int32 or None; w_gate_up [E, 2 d_ffn, d_model] and w_down [E, d_model, d_ffn] int8 of the
    experts [first_expert, first_expert + E) with s_gate_up [E, 2 d_ffn] and s_down [E,
    d_model] float32; y [N, d_model] bfloat16 or float32."""
    dev = _device()
    _tensor("x", x, dev, torch.bfloat16, rows=True)
    n, d = x.shape
    _tensor("expert_idx", expert_idx, dev, torch.int32)
    if expert_idx.dim() != 2 or expert_idx.shape[0] != n:
        _refuse(f"expert_idx is {tuple(expert_idx.shape)}, expected [{n}, top_k]")
    k = expert_idx.shape[1]
    _tensor("expert_w", expert_w, dev, torch.float32, (n, k))
    if fanout is not None:
        _tensor("fanout", fanout, dev, torch.int32, (n,))
    _tensor("w_down", w_down, dev, torch.int8)
    if w_down.dim() != 3 or w_down.shape[1] != d:
        _refuse(f"w_down is {tuple(w_down.shape)}, expected [E, {d}, d_ffn]")
    e, _, f = w_down.shape
    _tensor("w_gate_up", w_gate_up, dev, torch.int8, (e, 2 * f, d))
    _tensor("s_gate_up", s_gate_up, dev, torch.float32, (e, 2 * f))
    _tensor("s_down", s_down, dev, torch.float32, (e, d))
    bf16 = isinstance(y, torch.Tensor) and y.dtype == torch.bfloat16
    _tensor("y", y, dev, torch.bfloat16 if bf16 else torch.float32, (n, d))
    _tensor("workspace", workspace, dev, torch.uint8)
    layer = _moe_layer(d, f, e, first_expert, k)
    _check(LIB.mla_moe_experts_i8(ctypes.byref(layer), n, _addr(x), _row_stride(x), _addr(expert_idx), _addr(expert_w), _addr(fanout),
                                  _addr(w_gate_up), _addr(s_gate_up), _addr(w_down), _addr(s_down), MLA_BF16 if bf16 else MLA_F32,
                                  _addr(y), _addr(workspace), workspace.numel(), _queue(stream, dev)))


def probe_mfma_bf16(iters, sink, stream=None) -> float:
    """Enqueue the matrix-core rate probe (mla_probe_mfma_bf16, a diagnostic of
    mla_probe.h) with `iters` products per chain; sink is a device tensor of at
    least 4 bytes.  Returns the launch's flop; time it with events on `stream`."""
    flop = ctypes.c_double(0.0)
    _check(LIB.mla_probe_mfma_bf16(int(iters), ctypes.byref(flop), _ptr(sink), _stream(stream)))
    return flop.value


def version() -> str:
    return LIB.mla_version().decode()
