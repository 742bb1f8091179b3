"""Per-frame driver of the hot path (Algorithm 1's per-frame loop, restricted
to what the library implements): device buffers for one workload and the three
library calls of a frame -- select (Eq. 1/2/4/5), readout (Eq. 6/7) and
commit (Eq. 8).  Buffers come from torch; all arithmetic runs in librs3.
"""
from __future__ import annotations

from typing import Optional

import torch

from . import rs3
from .synth import Workload


class Pipeline:
    def __init__(self, w: Workload, device="cuda", dense: bool = False,
                 ring_cap: Optional[int] = None, params: Optional[rs3.Params] = None,
                 stream=None):
        self.w = w
        self.device = torch.device(device)
        self.dense = dense
        rho = 1.0 if dense else w.rho
        self.params = params if params is not None else rs3.default_params(
            rho=rho, r_s=w.r_s, c=w.c, union_mode=w.union_mode)
        self.k_max = rs3.rs3_kmax(self.params.rho, w.mn)
        dev = self.device
        self.unit_group = torch.tensor(w.unit_group(), dtype=torch.int32, device=dev)
        self.track = torch.zeros((w.U, 6), dtype=torch.int32, device=dev)
        # two keep-set buffers, so the selection of frame t+1 can be issued
        # while the readout of frame t still reads its own keep-set
        self.idx_buf = [torch.zeros((w.U, max(self.k_max, 1)), dtype=torch.int32, device=dev)
                        for _ in range(2)]
        self.count_buf = [torch.zeros(w.U, dtype=torch.int32, device=dev) for _ in range(2)]
        self.idx, self.count = self.idx_buf[0], self.count_buf[0]
        self.status = torch.zeros(1, dtype=torch.int32, device=dev)
        self.ws_select = torch.empty(rs3.rs3_select_workspace_bytes(w.G, w.U, w.m, w.n),
                                     dtype=torch.uint8, device=dev)
        # two readout workspaces, paired with the keep-set buffers: the merge of
        # frame t reads its workspace while frame t+1 plans and attends in the other
        nws = rs3.rs3_readout_workspace_bytes(w.U, w.H, w.d, self.k_max, w.dtype)
        self.ws_buf = [torch.empty(nws, dtype=torch.uint8, device=dev) for _ in range(2)]
        self.ws_readout = self.ws_buf[0]
        if ring_cap is None:
            ring_cap = w.ring_cap_rows() if (dense or w.window > 0) else w.ring_cap_rows_tight()
        self.bank = rs3.Bank(w.U, w.H, w.d, w.dtype, w.mn, w.n_cond, w.window, ring_cap,
                             w.max_frames(), w.n_ptr, device=dev, stream=stream)
        self.stream = stream

    # -- library calls -------------------------------------------------------
    def use_buffer(self, i: int):
        """Selects which keep-set buffer (and readout workspace) the next
        select / readout use."""
        self.idx, self.count = self.idx_buf[i], self.count_buf[i]
        self.ws_readout = self.ws_buf[i]

    def select(self, z: torch.Tensor, prev_masks: torch.Tensor, stream=None):
        w = self.w
        rs3.rs3_select_queries(z, w.dtype, w.G, w.m, w.n, w.C, prev_masks, self.unit_group, w.U,
                               self.track, self.params, self.idx, self.count, self.ws_select,
                               self.status, stream if stream is not None else self.stream)

    def readout(self, q: torch.Tensor, residual: Optional[torch.Tensor], out: torch.Tensor,
                rope: Optional[torch.Tensor] = None, scale: float = 0.0):
        w = self.w
        rs3.rs3_memory_readout(q, w.dtype, w.G, w.mn, w.H, w.d, self.unit_group, self.idx,
                               self.count, self.k_max, self.bank, rope, residual, out, scale,
                               self.ws_readout, self.status, self.stream)

    def readout_attend(self, q: torch.Tensor, residual: Optional[torch.Tensor], out: torch.Tensor,
                       rope: Optional[torch.Tensor] = None, scale: float = 0.0, stream=None):
        """First phase of readout(): the attention over the bank."""
        w = self.w
        rs3.rs3_memory_readout_attend(q, w.dtype, w.G, w.mn, w.H, w.d, self.unit_group, self.idx,
                                      self.count, self.k_max, self.bank, rope, residual, out, scale,
                                      self.ws_readout, self.status,
                                      stream if stream is not None else self.stream)

    def readout_plan(self, q: torch.Tensor, residual: Optional[torch.Tensor], out: torch.Tensor,
                     rope: Optional[torch.Tensor] = None, scale: float = 0.0, stream=None):
        """First launch of readout_attend(): the pass-through and the work list."""
        w = self.w
        rs3.rs3_memory_readout_plan(q, w.dtype, w.G, w.mn, w.H, w.d, self.unit_group, self.idx,
                                    self.count, self.k_max, self.bank, rope, residual, out, scale,
                                    self.ws_readout, self.status,
                                    stream if stream is not None else self.stream)

    def readout_run(self, q: torch.Tensor, residual: Optional[torch.Tensor], out: torch.Tensor,
                    rope: Optional[torch.Tensor] = None, scale: float = 0.0, stream=None):
        """Second launch of readout_attend(): the attention kernel alone."""
        w = self.w
        rs3.rs3_memory_readout_run(q, w.dtype, w.G, w.mn, w.H, w.d, self.unit_group, self.idx,
                                   self.count, self.k_max, self.bank, rope, residual, out, scale,
                                   self.ws_readout, self.status,
                                   stream if stream is not None else self.stream)

    def readout_merge(self, q: torch.Tensor, residual: Optional[torch.Tensor], out: torch.Tensor,
                      rope: Optional[torch.Tensor] = None, scale: float = 0.0, stream=None):
        """Second phase of readout(): the split-KV merge; reads no bank."""
        w = self.w
        rs3.rs3_memory_readout_merge(q, w.dtype, w.G, w.mn, w.H, w.d, self.unit_group, self.idx,
                                     self.count, self.k_max, self.bank, rope, residual, out, scale,
                                     self.ws_readout, self.status,
                                     stream if stream is not None else self.stream)

    def commit(self, k_new: torch.Tensor, v_new: torch.Tensor, mask: Optional[torch.Tensor],
               is_cond: int, rope: Optional[torch.Tensor] = None):
        """Eq. 8's sparse write; with a RoPE table the keys are stored rotated
        by their own cell (Eq. 7 on the key side)."""
        m = None if self.dense else mask
        if rope is None:
            rs3.rs3_bank_commit(self.bank, k_new, v_new, m, is_cond, self.status, self.stream)
        else:
            rs3.rs3_bank_commit_rope(self.bank, k_new, v_new, m, is_cond, rope, self.status, self.stream)

    def set_pointers(self, kp: torch.Tensor, vp: torch.Tensor):
        rs3.rs3_bank_set_pointers(self.bank, kp, vp, self.status, self.stream)

    # -- long banks ------------------------------------------------------------
    def norm(self, q: Optional[torch.Tensor], q_out: Optional[torch.Tensor], k: Optional[torch.Tensor] = None,
             k_out: Optional[torch.Tensor] = None, q_weight: Optional[torch.Tensor] = None,
             k_weight: Optional[torch.Tensor] = None, eps: float = 1e-6, rope: Optional[torch.Tensor] = None,
             k_keep: Optional[torch.Tensor] = None):
        """RMS norm of the frame's query and key heads, rotated by their own cells: what
        readout() and commit() then take without a table.  k_keep: the commit's mask."""
        w = self.w
        rs3.rs3_qk_norm_rope(q, q_out, k, k_out, w.dtype, w.mn, w.H, w.H, w.d, q_weight, k_weight, eps, rope,
                             k_keep=k_keep, stream=self.stream)

    def use_blocks(self, block: int, n_top: int):
        """Buffers for reading the bank by blocks: digests, the chosen blocks and workspaces."""
        w, dev, nb = self.w, self.device, self.bank.blocks(block)
        self.block, self.n_top = block, n_top
        with torch.cuda.stream(self.stream):               # (filled in the order of the calls that use them)
            self.block_digest = torch.zeros((w.U, w.H, nb, w.d), dtype=torch.int8, device=dev)
            self.block_step = torch.zeros((w.U, w.H, nb), dtype=torch.float32, device=dev)
            self.block_sel = torch.full((w.U, w.H, max(self.k_max, 1), n_top), -1, dtype=torch.int32, device=dev)
            self.ws_blocks = torch.empty(rs3.rs3_block_select_workspace_bytes(w.U, w.H, self.k_max, nb), dtype=torch.uint8,
                                         device=dev)
            self.ws_sparse = torch.empty(rs3.rs3_sparse_readout_workspace_bytes(w.U, w.H, w.d, self.k_max, n_top, nb, w.dtype, block),
                                         dtype=torch.uint8, device=dev)

    def digest(self, refresh: int = 1):
        """Brings the digests up to date: 1 after a ring commit, -1 after anything else."""
        rs3.rs3_bank_digest(self.bank, self.block, refresh, self.block_digest, self.block_step, self.status, self.stream)

    def select_blocks(self, q: torch.Tensor, rope: Optional[torch.Tensor] = None):
        """The blocks that score highest for each kept query and head (block_sel)."""
        w = self.w
        rs3.rs3_block_select(q, w.dtype, w.G, w.mn, w.H, w.d, self.unit_group, self.idx, self.count, self.k_max, self.bank,
                             self.block, self.block_digest, self.block_step, rope, self.n_top, self.block_sel,
                             self.ws_blocks, self.status, self.stream)

    def readout_blocks(self, q: torch.Tensor, residual: Optional[torch.Tensor], out: torch.Tensor,
                       rope: Optional[torch.Tensor] = None, scale: float = 0.0):
        """readout() over the blocks of block_sel."""
        w = self.w
        rs3.rs3_sparse_readout(q, w.dtype, w.G, w.mn, w.H, w.d, self.unit_group, self.idx, self.count, self.k_max,
                               self.bank, self.block, self.block_sel, self.n_top, rope, residual, out, scale,
                               self.ws_sparse, self.status, self.stream)

    # -- a memory-attention layer around the readout ----------------------------
    def use_scores(self, cap: float = 0.0, frame_bias: Optional[torch.Tensor] = None,
                   frame_keep: Optional[torch.Tensor] = None):
        """How readout_scored() changes its scores: capped at `cap` (0: not), biased by frame_bias [H, F+2] or
        [U, H, F+2], over the frames that frame_keep uint8 [U, F+2] leaves (ages of ring frames, F =
        bank.max_frames of them, then conditioning frames, then pointers).  The tensors are read by every call."""
        self.cap, self.frame_bias, self.frame_keep = cap, frame_bias, frame_keep
        if not hasattr(self, "ws_scored"):
            with torch.cuda.stream(self.stream):           # (made in the order of the calls that use it)
                self.ws_scored = torch.empty(rs3.rs3_scored_readout_workspace_bytes(self.bank, self.k_max), dtype=torch.uint8,
                                             device=self.device)

    def readout_scored(self, q: torch.Tensor, residual: Optional[torch.Tensor], out: torch.Tensor,
                       rope: Optional[torch.Tensor] = None, scale: float = 0.0):
        """readout() with the scores of use_scores()."""
        w = self.w
        rs3.rs3_scored_readout(q, w.dtype, w.G, w.mn, w.H, w.d, self.unit_group, self.idx, self.count, self.k_max, self.bank,
                               self.cap, self.frame_bias, self.frame_keep, rope, residual, out, scale, self.ws_scored,
                               self.status, self.stream)

    def share(self, prefix: "Pipeline", prefix_unit: torch.Tensor):
        """readout_shared() reads unit prefix_unit[u] (int32 [U], -1: none) of `prefix`'s bank before each unit's own rows:
        what fork() would copy, read in place."""
        self.prefix, self.prefix_unit = prefix, prefix_unit
        with torch.cuda.stream(self.stream):
            self.ws_shared = torch.empty(rs3.rs3_shared_readout_workspace_bytes(self.bank, prefix.bank, self.k_max),
                                         dtype=torch.uint8, device=self.device)

    def readout_shared(self, q: torch.Tensor, residual: Optional[torch.Tensor], out: torch.Tensor,
                       rope: Optional[torch.Tensor] = None, scale: float = 0.0):
        """readout() over the rows of share()'s prefix and the own ones.  Where the prefix has another stream, the call
        comes after what was issued there, and what is issued there next (a commit, say) comes after it."""
        w = self.w
        here, there = self._on(), self.prefix._on()
        if there != here:
            here.wait_stream(there)
        rs3.rs3_shared_readout(q, w.dtype, w.G, w.mn, w.H, w.d, self.unit_group, self.idx, self.count, self.k_max, self.bank,
                               self.prefix.bank, self.prefix_unit, rope, residual, out, scale, self.ws_shared, self.status,
                               self.stream)
        if there != here:
            there.wait_stream(here)

    def rotate(self, q: Optional[torch.Tensor], q_out: Optional[torch.Tensor], q_pos: Optional[torch.Tensor],
               k: Optional[torch.Tensor], k_out: Optional[torch.Tensor], k_pos: Optional[torch.Tensor],
               spec: rs3.RopeSpec, k_keep: Optional[torch.Tensor] = None):
        """The frame's query and key heads turned by their positions (int32 [rows, axes]): what readout() and commit()
        then take without a table.  k_keep: the commit's mask."""
        w = self.w
        rs3.rs3_rope_rows(q, q_out, q_pos, k, k_out, k_pos, w.dtype, w.H, w.H, w.d, spec, k_keep=k_keep, stream=self.stream)

    def norm_residual(self, y: Optional[torch.Tensor], x: torch.Tensor, x_out: Optional[torch.Tensor],
                      h_out: Optional[torch.Tensor], **norms):
        """x_out = alpha x + gate post(y), h_out = pre(x_out) at the kept cells of every unit (rs3_norm_residual)."""
        # (idx has a column where nothing is ever kept; its counts are 0 then)
        rs3.rs3_norm_residual(y, x, x_out, h_out, self.w.dtype, idx=self.idx, count=self.count, status=self.status,
                              stream=self.stream, **norms)

    def _on(self):
        """The stream of this pipeline's calls."""
        return self.stream if self.stream is not None else torch.cuda.current_stream(self.device)

    def fork(self, parent: torch.Tensor, keep: Optional[torch.Tensor] = None, into: Optional["Pipeline"] = None) -> "Pipeline":
        """A pipeline (`into`, or a new one with this one's sizes; `into` may have another number of units)
        whose unit u holds the rows of this one's unit parent[u], those that keep[u] leaves, and its
        tracker.  A unit that the copy leaves as it is (`into`'s status tells why) keeps its tracker
        too.  Digests are not copied: the target's digest(-1) follows.  The copy runs on this pipeline's
        stream; where `into` has another, it comes after what was issued there, and what is issued there
        next comes after it."""
        U = self.w.U if into is None else into.w.U
        if parent.shape != (U,):
            raise ValueError(f"parent: one for each of the {U} units wanted, got {tuple(parent.shape)}")
        here, there = self._on(), into._on() if into is not None else None
        if there is not None and there != here:
            here.wait_stream(there)
        # the new buffers are filled, and the workspace comes and goes, in the order of this pipeline's stream
        with torch.cuda.stream(self.stream):
            if into is None:
                into = Pipeline(self.w, self.device, self.dense, int(self.bank.ring_cap), self.params, self.stream)
                if hasattr(self, "block"):
                    into.use_blocks(self.block, self.n_top)
            stride = 0 if keep is None else keep.shape[1]
            ws = torch.empty(rs3.rs3_bank_copy_workspace_bytes(U, stride), dtype=torch.uint8, device=self.device)
            copies = into.bank.copies.clone()
            rs3.rs3_bank_copy(into.bank, self.bank, parent, keep, ws, into.status, self.stream)
            # the trackers of the units that the copy replaced (it refuses parents that are no unit: the gather stays inside)
            chosen = self.track[parent.clamp(0, self.w.U - 1).long()]
            into.track.copy_(torch.where((into.bank.copies != copies)[:, None], chosen, into.track))
        if there is not None and there != here:
            there.wait_stream(here)
        return into

    def drop_frames(self, n_oldest: Optional[torch.Tensor], n_newest: Optional[torch.Tensor] = None):
        """Gives up ring frames at either end; digest(0) follows."""
        rs3.rs3_bank_drop_frames(self.bank, n_oldest, n_newest, self.status, self.stream)

    def reset(self):
        rs3.rs3_bank_reset(self.bank, -1, self.stream)
        self.track.zero_()
        self.status.zero_()

    def status_code(self) -> int:
        return int(self.status.item())
