"""One MLA-Online step on device tensors: attend -> merge -> sliced o-proj + artifact.

Holds the output and scratch buffers for a fixed geometry, segment table and
protected set, sized by the library's own size query.  Argument marshalling
and allocation only; every computation is a call into libmla_online.so.
"""
from __future__ import annotations

from types import SimpleNamespace

import numpy as np
import torch

from . import mla


class OnlineStep:
    def __init__(self, geom, segs, prot_rows, glob_head, split_keys: int, device="cuda",
                 with_part_seg: bool = True, out_dtype: int = mla.MLA_BF16):
        self.geom = geom
        self.segs = np.asarray(segs, dtype=np.int64).reshape(-1, 3)
        self.prot = np.ascontiguousarray(prot_rows, dtype=np.int32)
        self.glob_head = np.ascontiguousarray(glob_head, dtype=np.int32)
        self.split_keys = int(split_keys)
        self.n_rows = int(self.segs[:, 1].sum())
        self.n_slots, self.n_parts, ws = mla.attend_query(geom, self.segs, self.prot, self.split_keys)
        d_c = mla.head_width(geom)
        dev = torch.device(device)
        self.part_o = torch.empty((self.n_parts, d_c), dtype=torch.float32, device=dev)
        self.part_lse = torch.empty((self.n_parts,), dtype=torch.float32, device=dev)
        self.part_ptr = torch.empty((self.n_slots + 1,), dtype=torch.int64, device=dev)
        self.part_seg = (torch.empty((self.n_parts, 2), dtype=torch.int32, device=dev)
                         if with_part_seg else None)
        self.row_src = torch.empty((self.n_rows,), dtype=torch.uint8, device=dev)
        self.ws = torch.empty((max(ws, 256),), dtype=torch.uint8, device=dev)
        self.out_dtype = out_dtype
        self.out_o = torch.empty((self.n_slots, d_c),
                                 dtype=torch.bfloat16 if out_dtype == mla.MLA_BF16 else torch.float32,
                                 device=dev)
        self.out_lse = torch.empty((self.n_slots,), dtype=torch.float32, device=dev)
        self.z = torch.empty((self.n_rows, int(geom.d_model)), dtype=torch.float32, device=dev)
        self.prot_d = torch.from_numpy(self.prot.copy()).to(dev)
        G = int(geom.n_groups)
        self.n_glob_slots = self.n_rows * G

    def attend(self, kv, q_glob, q_loc, stream=None):
        mla.online_attend(self.geom, self.segs, self.prot, self.split_keys, kv, q_glob, q_loc, self.part_o,
                          self.part_lse, self.part_ptr, self.part_seg, self.row_src, self.ws, stream)

    def merge(self, stream=None):
        mla.segment_merge(self.n_slots, mla.head_width(self.geom), self.part_o, self.part_lse, self.part_ptr,
                          self.out_dtype, self.out_o, self.out_lse, stream)

    def oproj(self, w_o, z_off, stream=None):
        if self.out_dtype != mla.MLA_BF16:
            raise ValueError("the sliced o-proj consumes bf16 head outputs")
        o_glob = self.out_o[: self.n_glob_slots]
        o_loc = self.out_o[self.n_glob_slots:] if self.n_slots > self.n_glob_slots else None
        mla.sliced_oproj_add(self.geom, self.n_rows, o_glob, o_loc, self.glob_head, self.prot_d,
                             int(self.prot.shape[0]), w_o, z_off, self.z, stream)

    def run(self, kv, q_glob, q_loc, w_o, z_off, stream=None):
        self.attend(kv, q_glob, q_loc, stream)
        self.merge(stream)
        self.oproj(w_o, z_off, stream)
        return self.z


class PlannedStep:
    """The step with the protected set in device memory: the plan is built once
    for a segment table, split mode and capacity (mla_online_plan); each call then
    takes prot_rows / |A| from device tensors and only enqueues kernels
    (mla_online_attend_planned, mla_sliced_oproj_add_planned).  Buffers are sized
    for the capacity; argument marshalling and allocation only."""

    def __init__(self, geom, segs, glob_head, split_keys: int, prot_cap: int, device="cuda",
                 out_dtype: int = mla.MLA_BF16, z_dtype=torch.float32, bookkeeping: bool = True,
                 with_lse: bool = True):
        self.geom = geom
        self.segs = np.asarray(segs, dtype=np.int64).reshape(-1, 3)
        self.glob_head = np.ascontiguousarray(glob_head, dtype=np.int32)
        dev = torch.device(device)
        info = mla.plan_query(geom, self.segs, split_keys, prot_cap)
        self.plan = torch.empty((max(int(info.plan_bytes), 256),), dtype=torch.uint8, device=dev)
        self.info = mla.online_plan(geom, self.segs, split_keys, prot_cap, self.plan)
        self.ws = torch.empty((max(int(self.info.ws_bytes), 256),), dtype=torch.uint8, device=dev)
        self.n_rows = int(self.info.n_rows)
        self.n_glob_slots = self.n_rows * int(geom.n_groups)
        d_v = mla.head_width(geom)
        self.out_o = torch.empty((int(self.info.max_slots), d_v),
                                 dtype=torch.bfloat16 if out_dtype == mla.MLA_BF16 else torch.float32, device=dev)
        self.out_lse = torch.empty((int(self.info.max_slots),), dtype=torch.float32, device=dev) if with_lse else None
        self.part_ptr = (torch.empty((int(self.info.max_slots) + 1,), dtype=torch.int64, device=dev)
                         if bookkeeping else None)
        self.part_seg = (torch.empty((max(int(self.info.max_parts), 1), 2), dtype=torch.int32, device=dev)
                         if bookkeeping else None)
        self.row_src = torch.empty((self.n_rows,), dtype=torch.uint8, device=dev) if bookkeeping else None
        self.status = torch.empty((1,), dtype=torch.int32, device=dev)
        self.z = torch.empty((self.n_rows, int(geom.d_model)), dtype=z_dtype, device=dev)

    def attend(self, prot_rows, n_prot, kv, q_glob, q_loc, stream=None):
        mla.online_attend_planned(self.geom, self.info, self.plan, prot_rows, n_prot, kv, q_glob, q_loc, self.out_o,
                                  self.out_lse, self.part_ptr, self.part_seg, self.row_src, self.status, self.ws,
                                  stream)

    def oproj(self, prot_rows, n_prot, w_o, z_off, stream=None):
        if self.out_o.dtype != torch.bfloat16:
            raise ValueError("the sliced o-proj consumes bf16 head outputs")
        o_glob = self.out_o[: self.n_glob_slots]
        o_loc = self.out_o[self.n_glob_slots:] if self.out_o.shape[0] > self.n_glob_slots else None
        mla.sliced_oproj_add_planned(self.geom, self.info, o_glob, o_loc, self.glob_head, prot_rows, n_prot, w_o,
                                     z_off, self.z, stream)

    def run(self, prot_rows, n_prot, kv, q_glob, q_loc, w_o, z_off, stream=None):
        self.attend(prot_rows, n_prot, kv, q_glob, q_loc, stream)
        self.oproj(prot_rows, n_prot, w_o, z_off, stream)
        return self.z


class DecodeStep:
    """The attention part of a decode layer on the paged 4-bit cache, for a fixed batch of
    n_seqs requests of n_q new tokens each (a padded request: slots and positions -1):
      mla_cache_append  the tokens' rows into their pages,
      mla_cache_attend  every head over the request's pages,
      mla_sliced_oproj_add_planned  z = W_a O with every head Global (new tokens have no
                        artifact, so all rows are protected and z_off is never read),
      mla_shared_wb_mx4 y = W_b z.
    Every call only enqueues kernels: run() may be captured and replayed while positions,
    slots and pages change in their tensors.  Buffers and argument marshalling only."""

    def __init__(self, geom, n_seqs: int, n_q: int, max_pages: int, page_rows: int, d_out: int, device="cuda",
                 y_dtype=torch.bfloat16, with_lse: bool = False):
        self.geom = geom
        self.page_rows = int(page_rows)
        heads, self.n_rows = int(geom.n_heads), int(n_seqs) * int(n_q)
        if self.n_rows > mla.WB_MX4_MAX_ROWS:
            raise mla.MlaError(3, f"{self.n_rows} new tokens; the 4-bit W_b takes up to {mla.WB_MX4_MAX_ROWS}")
        npg, d_model = int(geom.n_proj_groups), int(geom.d_model)
        if npg < 1 or heads % npg or d_model < 1 or d_model % (32 * npg) or d_model % 64:
            raise mla.MlaError(2, f"{heads} heads, d_model {d_model}, {npg} projection groups")
        if d_model > mla.WB_MAX_D_IN:
            raise mla.MlaError(3, f"d_model {d_model}; the 4-bit W_b takes up to {mla.WB_MAX_D_IN}")
        if not 1 <= int(d_out) <= mla.WB_MX4_MAX_D_OUT:
            raise mla.MlaError(2 if d_out < 1 else 3, f"d_out {d_out}; the 4-bit W_b writes 1 to {mla.WB_MX4_MAX_D_OUT}")
        if y_dtype not in (torch.bfloat16, torch.float32):
            raise mla.MlaError(2, f"y_dtype {y_dtype}, expected torch.bfloat16 or torch.float32")
        fields = ("d_latent", "d_rope", "d_model", "n_proj_groups", "softmax_scale", "rope_base")
        self.all_global = SimpleNamespace(n_heads=heads, n_groups=heads, **{f: getattr(geom, f) for f in fields})
        self.info = mla.plan_query(self.all_global, [(0, self.n_rows, 0)], 0, self.n_rows)
        dev = torch.device(device)
        ws = mla.cache_attend_query(geom, n_seqs, n_q, max_pages, page_rows)
        self.ws = torch.empty((max(ws, 256),), dtype=torch.uint8, device=dev)
        d_c = int(geom.d_latent)
        self.out_o = torch.empty((n_seqs, n_q, heads, d_c), dtype=torch.bfloat16, device=dev)
        self.out_lse = torch.empty((n_seqs, n_q, heads), dtype=torch.float32, device=dev) if with_lse else None
        self.glob_head = np.zeros((heads,), dtype=np.int32)
        self.w_o_size = heads * d_c * (d_model // npg)   # [n_pg, H / n_pg * d_latent, d_model / n_pg]
        self.all_rows = torch.arange(self.n_rows, dtype=torch.int32, device=dev)
        self.n_prot = torch.full((1,), self.n_rows, dtype=torch.int32, device=dev)
        self.z = torch.empty((self.n_rows, int(geom.d_model)), dtype=torch.bfloat16, device=dev)
        self.y = torch.empty((self.n_rows, int(d_out)), dtype=y_dtype, device=dev)

    def append(self, kv, slots, cache, turn, stream=None):
        mla.cache_append(self.geom, kv, slots, cache, self.page_rows, pos=turn, stream=stream)

    def attend(self, q, pos, pages, seq_pages, cache, stream=None):
        mla.cache_attend(self.geom, q, pos, pages, seq_pages, cache, self.page_rows, self.out_o, self.out_lse,
                         workspace=self.ws, stream=stream)

    def oproj(self, w_o, stream=None):
        mla.check_tensor("w_o", w_o, torch.bfloat16)
        if w_o.numel() != self.w_o_size:
            raise mla.MlaError(2, f"w_o is {tuple(w_o.shape)}, expected {self.w_o_size} values")
        mla.sliced_oproj_add_planned(self.all_global, self.info, self.out_o, None, self.glob_head, self.all_rows,
                                     self.n_prot, w_o, self.z, self.z, stream)

    def project(self, wb_codes, wb_scales, stream=None):
        mla.shared_wb_mx4(self.z, wb_codes, wb_scales, self.y, stream)

    def run(self, kv, slots, q, pos, pages, seq_pages, cache, w_o, wb_codes, wb_scales, turn=None, stream=None):
        """kv [n_rows, D] bfloat16, slots [n_rows] int32, q [n_seqs, n_q, H, D], pos [n_seqs,
        n_q] int32; turn [n_rows] int32: each row's position in its page's RoPE frame (pos
        where the frame is 0).  Returns y [n_rows, d_out].  Every call checks its own
        arguments: where one refuses, those before it have run, and the append of the same
        rows may be repeated."""
        self.append(kv, slots, cache, pos.view(-1) if turn is None else turn, stream)
        self.attend(q, pos, pages, seq_pages, cache, stream)
        self.oproj(w_o, stream)
        self.project(wb_codes, wb_scales, stream)
        return self.y


class MoeStep:
    """A mixture-of-experts layer for a fixed batch of n_rows tokens:
      mla_shared_wb      logits = W_r x, the router's own weight in bf16,
      mla_moe_route      each row's experts, weights and (tau <= 1) fanout,
      mla_moe_experts_i8 y = the weighted experts in 8 bits,
    for the experts [first_expert, first_expert + n_local) of n_experts; with a share of them
    run() returns this device's part of y.  Every call only enqueues kernels: run() may be
    captured and replayed.  Buffers and argument marshalling only."""

    def __init__(self, n_rows: int, d_model: int, d_ffn: int, n_experts: int, top_k: int, device="cuda", n_local=None,
                 first_expert: int = 0, min_k=None, tau: float = 2.0, y_dtype=torch.bfloat16, with_count: bool = False, **route):
        """route: scoring, n_groups, top_groups, group_best, renormalize, scale of mla.moe_route."""
        self.n_local = int(n_experts if n_local is None else n_local)
        self.first_expert, self.n_experts, self.d_model, self.d_ffn = int(first_expert), int(n_experts), int(d_model), int(d_ffn)
        if self.n_local < 1 or self.first_expert < 0 or self.first_expert + self.n_local > self.n_experts:
            raise mla.MlaError(2, f"experts [{first_expert}, {first_expert} + {self.n_local}) of {n_experts}")
        if d_model % 64 or d_model > mla.WB_MAX_D_IN:
            raise mla.MlaError(2 if d_model % 64 else 3, f"d_model {d_model}; the router's product takes multiples of 64 up to {mla.WB_MAX_D_IN}")
        self.route_args = dict(route, min_k=int(top_k if min_k is None else min_k), tau=float(tau))
        mla.check_route(n_experts, top_k, **self.route_args)
        dev = torch.device(device)
        ws = mla.moe_experts_i8_query(n_rows, d_model, d_ffn, self.n_local, top_k, y_dtype)
        self.ws = torch.empty((ws,), dtype=torch.uint8, device=dev)
        self.logits = torch.empty((n_rows, n_experts), dtype=torch.float32, device=dev)
        self.expert_idx = torch.empty((n_rows, top_k), dtype=torch.int32, device=dev)
        self.expert_w = torch.empty((n_rows, top_k), dtype=torch.float32, device=dev)
        self.fanout = torch.empty((n_rows,), dtype=torch.int32, device=dev)
        self.count = torch.empty((n_experts,), dtype=torch.int32, device=dev) if with_count else None
        self.y = torch.empty((n_rows, d_model), dtype=y_dtype, device=dev)

    def route(self, x, w_r, bias=None, stream=None):
        mla.check_tensor("x", x, torch.bfloat16)
        mla.check_tensor("w_r", w_r, torch.bfloat16)
        if x.shape != (self.logits.shape[0], self.d_model) or w_r.shape != (self.n_experts, self.d_model):
            raise mla.MlaError(2, f"x is {tuple(x.shape)}, w_r {tuple(w_r.shape)}; made for {self.logits.shape[0]} rows, [{self.n_experts}, {self.d_model}]")
        mla.shared_wb(x, w_r, self.logits, stream)
        mla.moe_route(self.logits, self.expert_idx, self.expert_w, self.fanout, self.count, bias=bias, stream=stream, **self.route_args)

    def experts(self, x, w_gate_up, s_gate_up, w_down, s_down, stream=None):
        mla.check_tensor("w_down", w_down, torch.int8)
        if w_down.shape != (self.n_local, self.d_model, self.d_ffn):
            raise mla.MlaError(2, f"w_down is {tuple(w_down.shape)}; made for [{self.n_local}, {self.d_model}, {self.d_ffn}]")
        mla.moe_experts_i8(x, self.expert_idx, self.expert_w, w_gate_up, s_gate_up, w_down, s_down, self.y, self.ws, fanout=self.fanout,
                           first_expert=self.first_expert, stream=stream)

    def run(self, x, w_r, w_gate_up, s_gate_up, w_down, s_down, bias=None, stream=None):
        """x [n_rows, d_model] bfloat16, w_r [n_experts, d_model] bfloat16, bias [n_experts]
        float32 or None, the weights as mla.moe_experts_i8 takes them.  Returns y [n_rows,
        d_model].  Every call checks its own arguments: where one refuses, those before it have
        run, and run() may be called again."""
        self.route(x, w_r, bias, stream)
        self.experts(x, w_gate_up, s_gate_up, w_down, s_down, stream)
        return self.y
