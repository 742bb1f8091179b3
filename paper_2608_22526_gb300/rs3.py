"""Python binding of librs3 (include/rs3.h): argument marshalling only.

Every step of the hot path runs in the CUDA library; this module turns torch
tensors into pointers and checks return codes.  There is no fallback: if the
library is missing the import of this module fails.
"""
from __future__ import annotations

import ctypes
import os
from typing import Optional

import torch

PKG = os.path.dirname(os.path.abspath(__file__))
LIB_PATH = os.path.join(PKG, "librs3.so")

RS3_OK, RS3_EINVAL, RS3_ECAPACITY, RS3_EUNSUPPORTED, RS3_ECUDA, RS3_EINTERNAL, RS3_ETIMEOUT = range(7)
RS3_F32, RS3_BF16 = 0, 1
DTYPES = {"f32": RS3_F32, "bf16": RS3_BF16}
TORCH_DTYPES = {"f32": torch.float32, "bf16": torch.bfloat16}


class RS3Error(RuntimeError):
    def __init__(self, code: int, what: str):
        super().__init__(f"{what}: rs3 status {code} ({status_string(code)})")
        self.code = code


class Params(ctypes.Structure):
    _fields_ = [("rho", ctypes.c_double), ("r_s", ctypes.c_int32), ("c", ctypes.c_int32),
                ("D_w", ctypes.c_int32), ("union_mode", ctypes.c_int32),
                ("fall_lo", ctypes.c_double), ("fall_hi", ctypes.c_double),
                ("fall_through", ctypes.c_int32), ("bbox_mode", ctypes.c_int32)]


class BankDesc(ctypes.Structure):
    _fields_ = [("U", ctypes.c_int32), ("H", ctypes.c_int32), ("d", ctypes.c_int32),
                ("D", ctypes.c_int32), ("dtype", ctypes.c_int32), ("mn", ctypes.c_int32),
                ("n_cond", ctypes.c_int32), ("window", ctypes.c_int32),
                ("max_frames", ctypes.c_int32), ("n_ptr", ctypes.c_int32),
                ("pinned_cap", ctypes.c_int64), ("ring_cap", ctypes.c_int64),
                ("rows_per_unit", ctypes.c_int64), ("meta_stride", ctypes.c_int64),
                ("k_store", ctypes.c_void_p), ("v_store", ctypes.c_void_p),
                ("meta", ctypes.c_void_p), ("magic", ctypes.c_uint32),
                ("reserved", ctypes.c_uint32)]


# Exported symbols and their signatures (checked against include/rs3.h by the tests)
_P = ctypes.c_void_p
_I = ctypes.c_int
_I64 = ctypes.c_int64
_SZ = ctypes.c_size_t
SIGNATURES = {
    "rs3_default_params": (None, [_P]),
    "rs3_kmax": (_I64, [ctypes.c_double, _I64]),
    "rs3_status_string": (ctypes.c_char_p, [_I]),
    "rs3_version": (_I, []),
    "rs3_select_workspace_bytes": (_SZ, [_I, _I, _I, _I]),
    "rs3_select_queries": (_I, [_P, _I, _I, _I, _I, _I, _P, _P, _I, _P, _P, _P, _P, _P, _SZ, _P, _P]),
    "rs3_select_queries_noalloc": (_I, [_P, _I, _I, _I, _I, _I, _P, _P, _I, _P, _P, _P, _P, _P, _P]),
    "rs3_bank_layout": (_I, [_I, _I, _I, _I, _I, _I, _I, _I64, _I, _I, _P, _P]),
    "rs3_bank_init": (_I, [_P, _I, _I, _I, _I, _I, _I, _I, _I64, _I, _I, _P, _P, _P, _P]),
    "rs3_bank_commit": (_I, [_P, _P, _P, _P, _I, _P, _P]),
    "rs3_bank_commit_rope": (_I, [_P, _P, _P, _P, _I, _P, _P, _P]),
    "rs3_bank_set_pointers": (_I, [_P, _P, _P, _P, _P]),
    "rs3_bank_reset": (_I, [_P, _I, _P]),
    "rs3_bank_read_meta": (_I, [_P, _P, _P, _P]),
    "rs3_bank_drop_frames": (_I, [_P, _P, _P, _P, _P]),
    "rs3_bank_copy_workspace_bytes": (_SZ, [_I, _I64]),
    "rs3_bank_copy": (_I, [_P, _P, _P, _P, _I64, _P, _SZ, _P, _P]),
    "rs3_bank_blocks": (_I64, [_P, _I]),
    "rs3_bank_digest": (_I, [_P, _I, _I, _P, _P, _P, _P]),
    "rs3_block_select_workspace_bytes": (_SZ, [_I, _I, _I, _I]),
    "rs3_block_select": (_I, [_P, _I, _I, _I, _I, _I, _P, _P, _P, _I, _P, _I, _P, _P, _P, _I, _P, _P, _SZ, _P, _P]),
    "rs3_sparse_readout_workspace_bytes": (_SZ, [_I, _I, _I, _I, _I, _I, _I]),
    "rs3_sparse_readout_block_workspace_bytes": (_SZ, [_I, _I, _I, _I, _I, _I, _I, _I]),
    "rs3_sparse_readout": (_I, [_P, _I, _I, _I, _I, _I, _P, _P, _P, _I, _P, _I, _P, _I, _P, _P, _P,
                                ctypes.c_float, _P, _SZ, _P, _P]),
    "rs3_qk_norm_rope": (_I, [_P, _I64, _I64, _I, _P, _P, _P, _I64, _P, _I64, _I64, _I, _P, _P, _P, _I64,
                              _I, _I, _I, ctypes.c_float, _P, _P]),
    "rs3_readout_workspace_bytes": (_SZ, [_I, _I, _I, _I, _I]),
    "rs3_memory_readout": (_I, [_P, _I, _I, _I, _I, _I, _P, _P, _P, _I, _P, _P, _P, _P,
                                ctypes.c_float, _P, _SZ, _P, _P]),
    "rs3_memory_readout_attend": (_I, [_P, _I, _I, _I, _I, _I, _P, _P, _P, _I, _P, _P, _P, _P,
                                ctypes.c_float, _P, _SZ, _P, _P]),
    "rs3_memory_readout_merge": (_I, [_P, _I, _I, _I, _I, _I, _P, _P, _P, _I, _P, _P, _P, _P,
                                ctypes.c_float, _P, _SZ, _P, _P]),
    "rs3_memory_readout_plan": (_I, [_P, _I, _I, _I, _I, _I, _P, _P, _P, _I, _P, _P, _P, _P,
                                ctypes.c_float, _P, _SZ, _P, _P]),
    "rs3_memory_readout_run": (_I, [_P, _I, _I, _I, _I, _I, _P, _P, _P, _I, _P, _P, _P, _P,
                                ctypes.c_float, _P, _SZ, _P, _P]),
    "rs3_set_wait_limit_ns": (None, [ctypes.c_uint64]),
    "rs3_get_wait_limit_ns": (ctypes.c_uint64, []),
    "rs3_write_keepset": (_I, [_P, _P, _I, _I, _I, _P, _P, _P, _P]),
    "rs3_close_argmax": (_I, [_P, _P, _I, _I, _I, _I, _I, _I, _P, _P, _P, _P, _P]),
    "rs3_seed_from_masks": (_I, [_P, _I, _I, _I, _I, _P, _P, _P, _P]),
}


def _load():
    if not os.path.exists(LIB_PATH):
        raise ImportError(f"librs3.so is not built ({LIB_PATH}); run __graft_entry__.build()")
    lib = ctypes.CDLL(LIB_PATH)
    for name, (res, args) in SIGNATURES.items():
        fn = getattr(lib, name)
        fn.restype = res
        fn.argtypes = args
    return lib


lib = _load()


def status_string(code: int) -> str:
    return lib.rs3_status_string(int(code)).decode()


def _check(code: int, what: str):
    if code != RS3_OK:
        raise RS3Error(code, what)


def _ptr(t: Optional[torch.Tensor]):
    if t is None:
        return None
    if not t.is_contiguous():
        raise ValueError("tensors passed to librs3 must be contiguous")
    return t.data_ptr()


def _stream(stream):
    if stream is None:                 # the current stream's handle, without a Stream object around it
        return torch._C._cuda_getCurrentRawStream(torch.cuda.current_device())
    return stream.cuda_stream


def _bytes(t: Optional[torch.Tensor]) -> int:
    return 0 if t is None else t.numel() * t.element_size()


def _want(dev: int, name: str, t: Optional[torch.Tensor], dtype, numel: int):
    """A tensor of at least `numel` elements of this type on device `dev`, the current one."""
    if t is None:
        raise ValueError(f"{name} is missing")
    if t.get_device() != dev:
        raise ValueError(f"{name} is not on the current CUDA device")
    if t.dtype != dtype or t.numel() < numel:
        raise ValueError(f"{name}: at least {numel} elements of {dtype} wanted, got {tuple(t.shape)} of {t.dtype}")

def _want_bank(dev: int, bank: "Bank"):
    """A bank whose storage is on device `dev`."""
    if bank.k_store.get_device() != dev:
        raise ValueError("the bank is not on the current CUDA device")


def _want_workspace(dev: int, t: Optional[torch.Tensor]):
    """A workspace on device `dev`, or none (its size is the library's to check)."""
    if t is not None and t.get_device() != dev and t.numel():
        raise ValueError("workspace is not on the current CUDA device")


# ---------------------------------------------------------------------------
# small helpers
# ---------------------------------------------------------------------------

def default_params(**over) -> Params:
    p = Params()
    lib.rs3_default_params(ctypes.byref(p))
    for k, v in over.items():
        setattr(p, k, v)
    return p


def rs3_kmax(rho: float, mn: int) -> int:
    return int(lib.rs3_kmax(float(rho), int(mn)))


def rs3_select_workspace_bytes(G: int, U: int, m: int, n: int) -> int:
    return int(lib.rs3_select_workspace_bytes(G, U, m, n))


def rs3_readout_workspace_bytes(U: int, H: int, d: int, k_max: int, dtype: str) -> int:
    return int(lib.rs3_readout_workspace_bytes(U, H, d, k_max, DTYPES[dtype]))


# ---------------------------------------------------------------------------
# read side
# ---------------------------------------------------------------------------

def rs3_select_queries(z, dtype: str, G: int, m: int, n: int, C: int, prev_masks, unit_group,
                       U: int, track, params: Params, idx, count, workspace, status, stream=None):
    rc = lib.rs3_select_queries(_ptr(z), DTYPES[dtype], G, m, n, C, _ptr(prev_masks),
                                _ptr(unit_group), U, _ptr(track), ctypes.byref(params), _ptr(idx),
                                _ptr(count), _ptr(workspace), workspace.numel() * workspace.element_size(),
                                _ptr(status), _stream(stream))
    _check(rc, "rs3_select_queries")


def rs3_select_queries_noalloc(z, dtype: str, G: int, m: int, n: int, C: int, prev_masks,
                               unit_group, U: int, track, params: Params, idx, count, status,
                               stream=None):
    """rs3_select_queries without a workspace: always one launch."""
    rc = lib.rs3_select_queries_noalloc(_ptr(z), DTYPES[dtype], G, m, n, C, _ptr(prev_masks),
                                        _ptr(unit_group), U, _ptr(track), ctypes.byref(params),
                                        _ptr(idx), _ptr(count), _ptr(status), _stream(stream))
    _check(rc, "rs3_select_queries_noalloc")


def rs3_memory_readout(q, dtype: str, G: int, mn: int, H: int, d: int, unit_group, idx, count,
                       k_max: int, bank: "Bank", rope, residual, out, scale: float, workspace,
                       status, stream=None):
    rc = lib.rs3_memory_readout(_ptr(q), DTYPES[dtype], G, mn, H, d, _ptr(unit_group), _ptr(idx),
                                _ptr(count), k_max, ctypes.byref(bank.desc), _ptr(rope),
                                _ptr(residual), _ptr(out), float(scale), _ptr(workspace),
                                workspace.numel() * workspace.element_size(), _ptr(status),
                                _stream(stream))
    _check(rc, "rs3_memory_readout")


def _readout_phase(fn, name, q, dtype, G, mn, H, d, unit_group, idx, count, k_max, bank, rope, residual,
                   out, scale, workspace, status, stream):
    rc = fn(_ptr(q), DTYPES[dtype], G, mn, H, d, _ptr(unit_group), _ptr(idx), _ptr(count), k_max,
            ctypes.byref(bank.desc), _ptr(rope), _ptr(residual), _ptr(out), float(scale), _ptr(workspace),
            workspace.numel() * workspace.element_size(), _ptr(status), _stream(stream))
    _check(rc, name)


def rs3_memory_readout_attend(q, dtype: str, G: int, mn: int, H: int, d: int, unit_group, idx, count,
                              k_max: int, bank: "Bank", rope, residual, out, scale: float, workspace,
                              status, stream=None):
    _readout_phase(lib.rs3_memory_readout_attend, "rs3_memory_readout_attend", q, dtype, G, mn, H, d,
                   unit_group, idx, count, k_max, bank, rope, residual, out, scale, workspace, status, stream)


def rs3_memory_readout_plan(q, dtype: str, G: int, mn: int, H: int, d: int, unit_group, idx, count,
                            k_max: int, bank: "Bank", rope, residual, out, scale: float, workspace,
                            status, stream=None):
    _readout_phase(lib.rs3_memory_readout_plan, "rs3_memory_readout_plan", q, dtype, G, mn, H, d,
                   unit_group, idx, count, k_max, bank, rope, residual, out, scale, workspace, status, stream)


def rs3_memory_readout_run(q, dtype: str, G: int, mn: int, H: int, d: int, unit_group, idx, count,
                           k_max: int, bank: "Bank", rope, residual, out, scale: float, workspace,
                           status, stream=None):
    _readout_phase(lib.rs3_memory_readout_run, "rs3_memory_readout_run", q, dtype, G, mn, H, d,
                   unit_group, idx, count, k_max, bank, rope, residual, out, scale, workspace, status, stream)


def rs3_memory_readout_merge(q, dtype: str, G: int, mn: int, H: int, d: int, unit_group, idx, count,
                             k_max: int, bank: "Bank", rope, residual, out, scale: float, workspace,
                             status, stream=None):
    _readout_phase(lib.rs3_memory_readout_merge, "rs3_memory_readout_merge", q, dtype, G, mn, H, d,
                   unit_group, idx, count, k_max, bank, rope, residual, out, scale, workspace, status, stream)


def rs3_write_keepset(seed_masks, unit_group, U: int, m: int, n: int, params: Params, kw_out,
                      status, stream=None):
    rc = lib.rs3_write_keepset(_ptr(seed_masks), _ptr(unit_group), U, m, n, ctypes.byref(params),
                               _ptr(kw_out), _ptr(status), _stream(stream))
    _check(rc, "rs3_write_keepset")


# ---------------------------------------------------------------------------
# memory bank
# ---------------------------------------------------------------------------

def rs3_bank_layout(U, H, d, dtype, mn, n_cond, window, ring_cap, max_frames, n_ptr):
    rows = ctypes.c_int64()
    mb = ctypes.c_size_t()
    rc = lib.rs3_bank_layout(U, H, d, DTYPES[dtype], mn, n_cond, window, ring_cap, max_frames,
                             n_ptr, ctypes.byref(rows), ctypes.byref(mb))
    _check(rc, "rs3_bank_layout")
    return rows.value, mb.value


class Bank:
    """A set of U per-unit banks whose storage is owned by torch tensors."""

    def __init__(self, U: int, H: int, d: int, dtype: str, mn: int, n_cond: int, window: int,
                 ring_cap: int, max_frames: int, n_ptr: int, device="cuda", stream=None):
        rows, mb = rs3_bank_layout(U, H, d, dtype, mn, n_cond, window, ring_cap, max_frames, n_ptr)
        self.U, self.H, self.d, self.D, self.dtype, self.mn = U, H, d, H * d, dtype, mn
        self.rows_per_unit = rows
        tdt = TORCH_DTYPES[dtype]
        self.k_store = torch.empty((U, rows, H * d), dtype=tdt, device=device)
        self.v_store = torch.empty((U, rows, H * d), dtype=tdt, device=device)
        self.meta = torch.empty(max(mb // 8, 1), dtype=torch.int64, device=device)
        self.desc = BankDesc()
        rc = lib.rs3_bank_init(ctypes.byref(self.desc), U, H, d, DTYPES[dtype], mn, n_cond, window,
                               ring_cap, max_frames, n_ptr, _ptr(self.k_store), _ptr(self.v_store),
                               _ptr(self.meta), _stream(stream))
        _check(rc, "rs3_bank_init")
        # per unit, on the device: {head, tail, cond_len, n_frames, oldest, n_cond_frames, ptr_len},
        # int64 [U, 7], a view of the bank's own
        self.counters = self.meta.view(U, -1)[:, :7]
        # int64 [U], a view too (word BM_COPIES): rises where rs3_bank_copy replaced the unit, not where it left it as it was
        self.copies = self.meta.view(U, -1)[:, 9]

    def blocks(self, block: int) -> int:
        """Blocks of `block` storage rows of a unit (rs3_bank_blocks)."""
        return int(lib.rs3_bank_blocks(ctypes.byref(self.desc), int(block)))

    @property
    def pinned_cap(self):
        return self.desc.pinned_cap

    @property
    def ring_cap(self):
        return self.desc.ring_cap

    @property
    def max_frames(self):
        return self.desc.max_frames


def rs3_bank_commit(bank: Bank, k_new, v_new, keep_mask, is_cond: int, status, stream=None):
    rc = lib.rs3_bank_commit(ctypes.byref(bank.desc), _ptr(k_new), _ptr(v_new), _ptr(keep_mask),
                             int(is_cond), _ptr(status), _stream(stream))
    _check(rc, "rs3_bank_commit")


def rs3_bank_commit_rope(bank: Bank, k_new, v_new, keep_mask, is_cond: int, rope, status, stream=None):
    rc = lib.rs3_bank_commit_rope(ctypes.byref(bank.desc), _ptr(k_new), _ptr(v_new), _ptr(keep_mask),
                                  int(is_cond), _ptr(rope), _ptr(status), _stream(stream))
    _check(rc, "rs3_bank_commit_rope")


def rs3_bank_set_pointers(bank: Bank, k_ptr, v_ptr, status, stream=None):
    rc = lib.rs3_bank_set_pointers(ctypes.byref(bank.desc), _ptr(k_ptr), _ptr(v_ptr), _ptr(status),
                                   _stream(stream))
    _check(rc, "rs3_bank_set_pointers")


def rs3_bank_reset(bank: Bank, unit: int = -1, stream=None):
    rc = lib.rs3_bank_reset(ctypes.byref(bank.desc), int(unit), _stream(stream))
    _check(rc, "rs3_bank_reset")


def rs3_bank_drop_frames(bank: Bank, n_oldest, n_newest, status, stream=None):
    """Gives up the n_oldest[u] oldest and n_newest[u] newest ring frames of every unit."""
    dev = torch.cuda.current_device()
    _want_bank(dev, bank)
    if n_oldest is not None:
        _want(dev, "n_oldest", n_oldest, torch.int32, bank.U)
    if n_newest is not None:
        _want(dev, "n_newest", n_newest, torch.int32, bank.U)
    _want(dev, "status", status, torch.int32, 1)
    rc = lib.rs3_bank_drop_frames(ctypes.byref(bank.desc), _ptr(n_oldest), _ptr(n_newest), _ptr(status),
                                  _stream(stream))
    _check(rc, "rs3_bank_drop_frames")


def rs3_bank_copy_workspace_bytes(U: int, keep_stride: int) -> int:
    return int(lib.rs3_bank_copy_workspace_bytes(U, keep_stride))


def rs3_bank_copy(dst: Bank, src: Bank, parent, keep, workspace, status, stream=None):
    """Unit u of dst becomes the kept rows of unit parent[u] of src (-1: left as it
    is); keep: uint8 [dst.U, at least the parents' length] over logical rows, or None."""
    dev = torch.cuda.current_device()
    _want_bank(dev, dst)
    _want_bank(dev, src)
    _want(dev, "parent", parent, torch.int32, dst.U)
    _want(dev, "status", status, torch.int32, 1)
    stride = 0
    if keep is not None:
        if keep.dim() != 2 or keep.shape[0] != dst.U:
            raise ValueError("keep: one row per destination unit")
        _want(dev, "keep", keep, torch.uint8, dst.U)
        stride = keep.shape[1]
    _want_workspace(dev, workspace)
    rc = lib.rs3_bank_copy(ctypes.byref(dst.desc), ctypes.byref(src.desc), _ptr(parent), _ptr(keep), stride,
                           _ptr(workspace), _bytes(workspace), _ptr(status), _stream(stream))
    _check(rc, "rs3_bank_copy")


def rs3_bank_read_meta(bank: Bank, stream=None):
    """(counters int64 [U, 8], frames int64 [U, max_frames, 2]); synchronises."""
    import numpy as np
    out = np.zeros((bank.U, 8), dtype=np.int64)
    fr = np.zeros((bank.U, bank.max_frames, 2), dtype=np.int64)
    rc = lib.rs3_bank_read_meta(ctypes.byref(bank.desc), out.ctypes.data_as(ctypes.c_void_p),
                                fr.ctypes.data_as(ctypes.c_void_p), _stream(stream))
    _check(rc, "rs3_bank_read_meta")
    return out, fr


# ---------------------------------------------------------------------------
# read side over chosen blocks of a long bank
# ---------------------------------------------------------------------------

def _block_heads(bank: Bank, block: int) -> int:
    return bank.U * bank.H * (-(-bank.rows_per_unit // block) if block > 0 else 0)


def rs3_bank_digest(bank: Bank, block: int, refresh: int, digest, step, status, stream=None):
    """Digests (int8 [U, H, blocks, d] and their steps fp32 [U, H, blocks]) of the
    blocks of the `refresh` newest ring frames, or of all blocks (-1)."""
    dev, n = torch.cuda.current_device(), _block_heads(bank, block)
    _want_bank(dev, bank)
    _want(dev, "digest", digest, torch.int8, n * bank.d)
    _want(dev, "step", step, torch.float32, n)
    _want(dev, "status", status, torch.int32, 1)
    rc = lib.rs3_bank_digest(ctypes.byref(bank.desc), block, refresh, _ptr(digest), _ptr(step), _ptr(status),
                             _stream(stream))
    _check(rc, "rs3_bank_digest")


def _want_read(q, dtype, G, mn, H, d, unit_group, idx, count, k_max, bank, rope, status):
    dev = torch.cuda.current_device()
    _want_bank(dev, bank)
    _want(dev, "q", q, TORCH_DTYPES[dtype], G * mn * H * d)
    _want(dev, "unit_group", unit_group, torch.int32, bank.U)
    _want(dev, "idx", idx, torch.int32, bank.U * k_max)
    _want(dev, "count", count, torch.int32, bank.U)
    if rope is not None:
        _want(dev, "rope", rope, torch.float32, mn * d)
    _want(dev, "status", status, torch.int32, 1)
    return dev


def rs3_block_select_workspace_bytes(U: int, H: int, k_max: int, n_blocks: int) -> int:
    return int(lib.rs3_block_select_workspace_bytes(U, H, k_max, n_blocks))


def rs3_block_select(q, dtype: str, G: int, mn: int, H: int, d: int, unit_group, idx, count, k_max: int,
                     bank: "Bank", block: int, digest, step, rope, n_top: int, sel, workspace, status,
                     stream=None):
    """The n_top blocks whose digests score highest for each kept query and head:
    sel int32 [U, H, k_max, n_top], ascending, -1 where there are fewer."""
    dev = _want_read(q, dtype, G, mn, H, d, unit_group, idx, count, k_max, bank, rope, status)
    n = _block_heads(bank, block)
    _want(dev, "digest", digest, torch.int8, n * bank.d)
    _want(dev, "step", step, torch.float32, n)
    _want(dev, "sel", sel, torch.int32, bank.U * bank.H * k_max * n_top)
    _want_workspace(dev, workspace)
    rc = lib.rs3_block_select(_ptr(q), DTYPES[dtype], G, mn, H, d, _ptr(unit_group), _ptr(idx), _ptr(count), k_max,
                              ctypes.byref(bank.desc), block, _ptr(digest), _ptr(step), _ptr(rope), n_top, _ptr(sel),
                              _ptr(workspace), _bytes(workspace), _ptr(status), _stream(stream))
    _check(rc, "rs3_block_select")


def rs3_sparse_readout_workspace_bytes(U: int, H: int, d: int, k_max: int, n_top: int, n_blocks: int,
                                       dtype: str, block: Optional[int] = None) -> int:
    """For blocks of any size, or for `block` rows (n_blocks of them), which takes a half or a quarter."""
    if block is None:
        return int(lib.rs3_sparse_readout_workspace_bytes(U, H, d, k_max, n_top, n_blocks, DTYPES[dtype]))
    return int(lib.rs3_sparse_readout_block_workspace_bytes(U, H, d, k_max, n_top, n_blocks, DTYPES[dtype], block))


def rs3_sparse_readout(q, dtype: str, G: int, mn: int, H: int, d: int, unit_group, idx, count, k_max: int,
                       bank: "Bank", block: int, sel, n_top: int, rope, residual, out, scale: float,
                       workspace, status, stream=None):
    """rs3_memory_readout over the blocks that sel lists for each query and head."""
    dev = _want_read(q, dtype, G, mn, H, d, unit_group, idx, count, k_max, bank, rope, status)
    _want(dev, "sel", sel, torch.int32, bank.U * bank.H * k_max * n_top)
    _want_workspace(dev, workspace)
    if residual is not None:
        _want(dev, "residual", residual, TORCH_DTYPES[dtype], bank.U * mn * H * d)
    _want(dev, "out", out, TORCH_DTYPES[dtype], bank.U * mn * H * d)
    rc = lib.rs3_sparse_readout(_ptr(q), DTYPES[dtype], G, mn, H, d, _ptr(unit_group), _ptr(idx), _ptr(count),
                                k_max, ctypes.byref(bank.desc), block, _ptr(sel), n_top, _ptr(rope), _ptr(residual),
                                _ptr(out), float(scale), _ptr(workspace), _bytes(workspace), _ptr(status),
                                _stream(stream))
    _check(rc, "rs3_sparse_readout")


# ---------------------------------------------------------------------------
# query and key heads: RMS norm with the position rotation
# ---------------------------------------------------------------------------

def _rows_of(name: str, t: torch.Tensor, width: int):
    """(rows, elements between rows) of a tensor [..., width] whose rows are evenly spaced."""
    if t.dim() >= 1 and t.shape[-1] == width and t.is_contiguous():
        return t.numel() // width, width
    if t.dim() < 1 or t.shape[-1] != width or (width > 1 and t.stride(-1) != 1):
        raise ValueError(f"{name}: rows of {width} adjacent elements wanted, got {tuple(t.shape)}")
    rows, step, reach = 1, None, None
    for n, st in zip(reversed(t.shape[:-1]), reversed(t.stride()[:-1])):
        if n != 1 and rows != 0:
            if step is None:
                step, reach = st, st
            if st != reach:
                raise ValueError(f"{name}: its rows are not evenly spaced")
            reach = st * n
        rows *= n
    return rows, (width if step is None else step)


def rs3_qk_norm_rope(q, q_out, k, k_out, dtype: str, mn: int, Hq: int, Hk: int, d: int, q_weight=None,
                     k_weight=None, eps: float = 1e-6, rope=None, q_keep=None, k_keep=None, stream=None):
    """RMS norm of every head of q [..., Hq*d] and k [..., Hk*d] (either may be None),
    rotated by the row's own cell, row r being cell r mod mn.  Rows may be evenly
    spaced parts of a wider tensor; out may be the input."""
    dev, dt, sides = torch.cuda.current_device(), TORCH_DTYPES[dtype], []
    for name, x, y, H, w, keep in (("q", q, q_out, Hq, q_weight, q_keep), ("k", k, k_out, Hk, k_weight, k_keep)):
        if x is None and y is None:
            sides += [None, 0, 0, 0, None, None, None, 0]
            continue
        _want(dev, name, x, dt, 0)
        _want(dev, name + "_out", y, dt, 0)
        (rows, stride), (rows_out, out_stride) = _rows_of(name, x, H * d), _rows_of(name + "_out", y, H * d)
        if rows != rows_out:
            raise ValueError(f"{name}_out has {rows_out} rows, {name} {rows}")
        if w is not None:
            _want(dev, name + "_weight", w, torch.float32, d)
        if keep is not None:
            _want(dev, name + "_keep", keep, torch.uint8, rows)
        sides += [x.data_ptr(), rows, stride, H, _ptr(w), _ptr(keep), y.data_ptr(), out_stride]
    if rope is not None:
        _want(dev, "rope", rope, torch.float32, mn * d)
    rc = lib.rs3_qk_norm_rope(*sides, DTYPES[dtype], mn, d, float(eps), _ptr(rope), _stream(stream))
    _check(rc, "rs3_qk_norm_rope")


# ---------------------------------------------------------------------------
# decoder side and pixel-space front end
# ---------------------------------------------------------------------------

def rs3_close_argmax(logits, group_start, G: int, U: int, h: int, w: int, radius: int, s: int,
                     palette, closed, grid_masks, status, stream=None):
    rc = lib.rs3_close_argmax(_ptr(logits), _ptr(group_start), G, U, h, w, radius, s, _ptr(palette),
                              _ptr(closed), _ptr(grid_masks), _ptr(status), _stream(stream))
    _check(rc, "rs3_close_argmax")


def rs3_seed_from_masks(masks, U: int, h: int, w: int, s: int, track, grid_masks, box_masks,
                        stream=None):
    rc = lib.rs3_seed_from_masks(_ptr(masks), U, h, w, s, _ptr(track), _ptr(grid_masks),
                                 _ptr(box_masks), _stream(stream))
    _check(rc, "rs3_seed_from_masks")


def rs3_set_wait_limit_ns(ns: int):
    lib.rs3_set_wait_limit_ns(int(ns))


def rs3_get_wait_limit_ns() -> int:
    return int(lib.rs3_get_wait_limit_ns())
