"""Python binding of librs3 (include/rs3.h): argument marshalling only.

Every step of the hot path runs in the CUDA library; this module turns torch
tensors into pointers and checks return codes.  There is no fallback: if the
library is missing the import of this module fails.
"""
from __future__ import annotations

import ctypes
import os
import struct
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


class RopeSpec(ctypes.Structure):
    _fields_ = [("layout", ctypes.c_int32), ("rot", ctypes.c_int32), ("axes", ctypes.c_int32),
                ("pairs", ctypes.c_int32 * 3), ("inverse", ctypes.c_int32), ("magnitude", ctypes.c_float),
                ("base", ctypes.c_double), ("factor", ctypes.c_double), ("context", ctypes.c_double),
                ("beta_fast", ctypes.c_double), ("beta_slow", ctypes.c_double)]


class Norm(ctypes.Structure):
    _fields_ = [("kind", ctypes.c_int32), ("eps", ctypes.c_float), ("weight", ctypes.c_void_p),
                ("bias", ctypes.c_void_p), ("weight_stride", ctypes.c_int64), ("bias_stride", ctypes.c_int64)]


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
    "rs3_scored_readout_workspace_bytes": (_SZ, [_P, _I]),
    "rs3_scored_readout": (_I, [_P, _I, _I, _I, _I, _I, _P, _P, _P, _I, _P, ctypes.c_float, _P, _I64, _P, _P, _P, _P, ctypes.c_float,
                                _P, _SZ, _P, _P]),
    "rs3_shared_readout_workspace_bytes": (_SZ, [_P, _P, _I]),
    "rs3_shared_readout": (_I, [_P, _I, _I, _I, _I, _I, _P, _P, _P, _I, _P, _P, _P, _P, _P, _P, ctypes.c_float, _P, _SZ, _P, _P]),
    "rs3_default_rope_spec": (None, [_P]),
    "rs3_rope_table": (_I, [_P, _I64, _P, _P, _P]),
    "rs3_rope_rows": (_I, [_P, _I64, _I64, _I, _P, _P, _P, _I64, _P, _I64, _I64, _I, _P, _P, _P, _I64, _I, _I, _P, _P]),
    "rs3_norm_residual": (_I, [_P, _P, _I, _I, _I, _I, _P, _P, _I, _P, _P, _I64, ctypes.c_float, _P, _P, _P, _P, _P]),
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


def _arg(dev: int, name: str, t: Optional[torch.Tensor], dtype, numel: int) -> int:
    """The pointer of a contiguous tensor of at least `numel` elements of this type on device `dev`, the current one."""
    if t is None or t.dtype is not dtype or t.numel() < numel or t.get_device() != dev or not t.is_contiguous():
        _want(dev, name, t, dtype, numel)
        return _ptr(t)
    return t.data_ptr()


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


def _read_args(q, dtype: str, G: int, mn: int, H: int, d: int, unit_group, idx, count, k_max: int, bank: "Bank", rope, residual, out,
               workspace, status):
    """What the readouts of scores or of a prefix have in common, checked: (device, arguments up to the bank, those from
    rope to out, the workspace's and the status)."""
    dev, dt, U, grid = torch.cuda.current_device(), TORCH_DTYPES[dtype], bank.U, mn * H * d
    _want_bank(dev, bank)
    _want_workspace(dev, workspace)
    head = (_arg(dev, "q", q, dt, G * grid), DTYPES[dtype], G, mn, H, d, _arg(dev, "unit_group", unit_group, torch.int32, U),
            _arg(dev, "idx", idx, torch.int32, U * k_max), _arg(dev, "count", count, torch.int32, U), k_max, ctypes.byref(bank.desc))
    to = (None if rope is None else _arg(dev, "rope", rope, torch.float32, mn * d),
          None if residual is None else _arg(dev, "residual", residual, dt, U * grid), _arg(dev, "out", out, dt, U * grid))
    return dev, head, to, (_ptr(workspace), _bytes(workspace), _arg(dev, "status", status, torch.int32, 1))


def rs3_scored_readout_workspace_bytes(bank: "Bank", k_max: int) -> int:
    return int(lib.rs3_scored_readout_workspace_bytes(ctypes.byref(bank.desc), k_max))


def rs3_scored_readout(q, dtype: str, G: int, mn: int, H: int, d: int, unit_group, idx, count, k_max: int, bank: "Bank", cap: float,
                       frame_bias, frame_keep, rope, residual, out, scale: float, workspace, status, stream=None):
    """rs3_memory_readout with scores capped at `cap` (0: not), biased by frame_bias fp32 [H, F+2] or [U, H, F+2], over
    the frames that frame_keep uint8 [U, F+2] leaves; F = bank.max_frames: ages of ring frames, then conditioning
    frames, then pointers."""
    dev, head, to, tail = _read_args(q, dtype, G, mn, H, d, unit_group, idx, count, k_max, bank, rope, residual, out, workspace, status)
    F, stride, bias_ptr, keep_ptr = bank.max_frames, 0, None, None
    if frame_bias is not None:
        if tuple(frame_bias.shape) not in ((H, F + 2), (bank.U, H, F + 2)):
            raise ValueError(f"frame_bias: [{H}, {F + 2}] or [{bank.U}, {H}, {F + 2}] wanted, got {tuple(frame_bias.shape)}")
        bias_ptr = _arg(dev, "frame_bias", frame_bias, torch.float32, 0)
        stride = H * (F + 2) if frame_bias.dim() == 3 else 0
    if frame_keep is not None:
        if tuple(frame_keep.shape) != (bank.U, F + 2):
            raise ValueError(f"frame_keep: [{bank.U}, {F + 2}] wanted, got {tuple(frame_keep.shape)}")
        keep_ptr = _arg(dev, "frame_keep", frame_keep, torch.uint8, 0)
    rc = lib.rs3_scored_readout(*head, float(cap), bias_ptr, stride, keep_ptr, *to, float(scale), *tail, _stream(stream))
    _check(rc, "rs3_scored_readout")


def rs3_shared_readout_workspace_bytes(bank: "Bank", prefix: "Bank", k_max: int) -> int:
    return int(lib.rs3_shared_readout_workspace_bytes(ctypes.byref(bank.desc), ctypes.byref(prefix.desc), k_max))


def rs3_shared_readout(q, dtype: str, G: int, mn: int, H: int, d: int, unit_group, idx, count, k_max: int, bank: "Bank",
                       prefix: "Bank", prefix_unit, rope, residual, out, scale: float, workspace, status, stream=None):
    """rs3_memory_readout over the rows of unit prefix_unit[u] of `prefix` (-1: none) and the unit's own in `bank`."""
    dev, head, to, tail = _read_args(q, dtype, G, mn, H, d, unit_group, idx, count, k_max, bank, rope, residual, out, workspace, status)
    _want_bank(dev, prefix)
    rc = lib.rs3_shared_readout(*head, ctypes.byref(prefix.desc), _arg(dev, "prefix_unit", prefix_unit, torch.int32, bank.U), *to,
                                float(scale), *tail, _stream(stream))
    _check(rc, "rs3_shared_readout")


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


def _rows_arg(dev: int, name: str, t, dt, width: int):
    """(rows, elements between rows, pointer) of a tensor [..., width] of this type on device `dev`."""
    if t is None or t.dtype is not dt or t.get_device() != dev:
        _want(dev, name, t, dt, 0)
    return *_rows_of(name, t, width), t.data_ptr()


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
# rotary positions from coordinates
# ---------------------------------------------------------------------------
ROPE_LAYOUTS = {"pairs": 0, "halves": 1}


def rope_spec(rot: int, pairs=None, layout: str = "pairs", base: float = 10000.0, factor: float = 1.0, context: float = 0.0,
              beta_fast: float = 32.0, beta_slow: float = 1.0, magnitude: float = 1.0, inverse: bool = False) -> RopeSpec:
    """How a head turns: `rot` leading elements, pairs[a] pairs of them with coordinate a (default: all with one)."""
    s = RopeSpec()
    lib.rs3_default_rope_spec(ctypes.byref(s))
    pairs = [rot // 2] if pairs is None else [int(n) for n in pairs]
    if not 1 <= len(pairs) <= 3:
        raise ValueError("pairs: one to three coordinates")
    s.layout, s.rot, s.axes, s.pairs = ROPE_LAYOUTS[layout], rot, len(pairs), (ctypes.c_int32 * 3)(*pairs)
    s.base, s.factor, s.context, s.beta_fast, s.beta_slow = base, factor, context, beta_fast, beta_slow
    s.magnitude, s.inverse = magnitude, int(inverse)
    return s


def _positions(dev: int, name: str, pos, axes: int, rows: int) -> int:
    """The pointer of positions int32 [..., axes] of so many rows; with one axis its extent may be left out."""
    if (pos is None or pos.dtype is not torch.int32 or pos.numel() != rows * axes or (axes != 1 and pos.size(-1) != axes)
            or pos.get_device() != dev or not pos.is_contiguous()):
        _want(dev, name, pos, torch.int32, 0)
        _ptr(pos)
        raise ValueError(f"{name}: int32 [{rows}, {axes}] wanted, got {tuple(pos.shape)}")
    return pos.data_ptr()


def rs3_rope_table(pos, spec: RopeSpec, cos_sin, stream=None):
    """(cos, sin) of every pair at the positions pos int32 [rows, axes]: fp32 [rows, rot/2, 2]."""
    dev = torch.cuda.current_device()
    _want(dev, "pos", pos, torch.int32, 0)
    if pos.shape[-1:] != (spec.axes,) and not (spec.axes == 1 and pos.dim() == 1):
        raise ValueError(f"pos: int32 [rows, {spec.axes}] wanted, got {tuple(pos.shape)}")
    rows = pos.numel() // spec.axes
    _want(dev, "cos_sin", cos_sin, torch.float32, rows * spec.rot)
    _check(lib.rs3_rope_table(_ptr(pos), rows, ctypes.byref(spec), _ptr(cos_sin), _stream(stream)), "rs3_rope_table")


def _rope_side(dev: int, name: str, x, y, dt, H: int, d: int, pos, axes: int, keep):
    """What rs3_rope_rows takes for the queries or the keys."""
    if x is None and y is None:
        return None, 0, 0, 0, None, None, None, 0
    width = H * d
    rows, stride, x_ptr = _rows_arg(dev, name, x, dt, width)
    rows_out, out_stride, y_ptr = _rows_arg(dev, name + "_out", y, dt, width)
    if rows != rows_out:
        raise ValueError(f"{name}_out has {rows_out} rows, {name} {rows}")
    return (x_ptr, rows, stride, H, _positions(dev, name + "_pos", pos, axes, rows),
            None if keep is None else _arg(dev, name + "_keep", keep, torch.uint8, rows), y_ptr, out_stride)


def rs3_rope_rows(q, q_out, q_pos, k, k_out, k_pos, dtype: str, Hq: int, Hk: int, d: int, spec: RopeSpec, q_keep=None,
                  k_keep=None, stream=None):
    """Every head of q [..., Hq*d] and k [..., Hk*d] (either may be None) turned by its row's
    position (int32 [rows, axes]).  Rows may be evenly spaced parts of a wider tensor; out may
    be the input; rows whose keep byte is 0 are neither read nor written."""
    dev, dt, axes = torch.cuda.current_device(), TORCH_DTYPES[dtype], spec.axes
    rc = lib.rs3_rope_rows(*_rope_side(dev, "q", q, q_out, dt, Hq, d, q_pos, axes, q_keep),
                           *_rope_side(dev, "k", k, k_out, dt, Hk, d, k_pos, axes, k_keep), DTYPES[dtype], d, ctypes.byref(spec),
                           _stream(stream))
    _check(rc, "rs3_rope_rows")


# ---------------------------------------------------------------------------
# between two blocks: norms, gate and residual
# ---------------------------------------------------------------------------
NORM_KINDS = {"none": 0, "rms": 1, "layer": 2}


def _vector(dev: int, name: str, t, U: int, C: int):
    """(pointer, elements between units) of a vector fp32 [C] or [U, C]; (None, 0) without one."""
    if t is None:
        return None, 0
    n = t.numel()
    if n == C and t.dim() == 1:
        return _arg(dev, name, t, torch.float32, C), 0
    if n != U * C or tuple(t.shape) != (U, C):
        raise ValueError(f"{name}: [{C}] or [{U}, {C}] wanted, got {tuple(t.shape)}")
    return _arg(dev, name, t, torch.float32, C), C


_norm_bytes = struct.Struct("ifNNqq").pack                 # a Norm, without its object


def _norm(dev: int, name: str, kind: str, eps: float, weight, bias, U: int, C: int):
    if weight is None and bias is None:
        return None if kind == "none" else _norm_bytes(NORM_KINDS[kind], eps, 0, 0, 0, 0)
    w, w_stride = _vector(dev, name + "_weight", weight, U, C)
    b, b_stride = _vector(dev, name + "_bias", bias, U, C)
    return _norm_bytes(NORM_KINDS[kind], eps, w or 0, b or 0, w_stride, b_stride)


def rs3_norm_residual(y, x, x_out, h_out, dtype: str, idx=None, count=None, post: str = "none", post_weight=None,
                      post_bias=None, gate=None, alpha: float = 1.0, pre: str = "none", pre_weight=None, pre_bias=None,
                      eps: float = 1e-6, status=None, stream=None):
    """x_out = alpha x + gate post(y), h_out = pre(x_out) over x, y [U, mn, C], at every cell or
    at the kept ones (idx int32 [U, k_max], count int32 [U]).  Vectors are fp32 [C] or [U, C]."""
    dev, dt = torch.cuda.current_device(), TORCH_DTYPES[dtype]
    if x.dim() != 3:
        raise ValueError(f"x: [units, cells, channels] wanted, got {tuple(x.shape)}")
    U, mn, C = x.shape
    n = U * mn * C
    k_max, idx_ptr, count_ptr, status_ptr = 0, None, None, None
    if idx is not None or count is not None:
        if idx is None or idx.dim() != 2 or idx.shape[0] != U:
            raise ValueError("idx: one row per unit, with count")
        k_max = idx.shape[1]
        idx_ptr, count_ptr = _arg(dev, "idx", idx, torch.int32, 0), _arg(dev, "count", count, torch.int32, U)
        status_ptr = _arg(dev, "status", status, torch.int32, 1)
    g, g_stride = _vector(dev, "gate", gate, U, C)
    rc = lib.rs3_norm_residual(None if y is None else _arg(dev, "y", y, dt, n), _arg(dev, "x", x, dt, n), DTYPES[dtype], U, mn, C,
                               idx_ptr, count_ptr, k_max, _norm(dev, "post", post, eps, post_weight, post_bias, U, C), g, g_stride,
                               alpha, _norm(dev, "pre", pre, eps, pre_weight, pre_bias, U, C),
                               None if x_out is None else _arg(dev, "x_out", x_out, dt, n),
                               None if h_out is None else _arg(dev, "h_out", h_out, dt, n),
                               status_ptr, _stream(stream))
    _check(rc, "rs3_norm_residual")


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
