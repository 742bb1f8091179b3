"""Refusals of the calls for long banks (norms, copies, digests, block selection, sparse
readout): bad arguments are rejected on the host, before anything is launched.  CPU only."""
import ctypes

import pytest
import torch


@pytest.fixture(scope="module")
def b():
    from paper_2608_22526_gb300 import _build
    _build.build()
    from paper_2608_22526_gb300 import rs3
    return rs3


ONE = ctypes.c_void_p(16)          # non-null and aligned; never dereferenced
ODD = ctypes.c_void_p(24)


def _bank(b, U=2, H=4, d=64, dtype="bf16", mn=64, n_cond=1, window=-1, ring=1000, max_frames=20, n_ptr=4, k=1 << 20, v=1 << 30,
          meta=1 << 40):
    """A descriptor as rs3_bank_init fills it, over memory that is never touched."""
    rows, _ = b.rs3_bank_layout(U, H, d, dtype, mn, n_cond, window, ring, max_frames, n_ptr)
    x = b.BankDesc()
    x.U, x.H, x.d, x.D, x.dtype, x.mn = U, H, d, H * d, b.DTYPES[dtype], mn
    x.n_cond, x.window, x.max_frames, x.n_ptr = n_cond, window, max_frames, n_ptr
    x.pinned_cap, x.ring_cap, x.rows_per_unit = n_cond * mn, ring, rows
    x.meta_stride = (16 + 2 * max_frames) * 8
    x.k_store, x.v_store, x.meta, x.magic = k, v, meta, 0x52533342
    return x


def _norm(b, **over):
    a = dict(q=ONE, q_rows=64, q_stride=256, Hq=4, qw=None, qk=None, qo=ONE, qs=256, k=ONE, k_rows=64, k_stride=256, Hk=4, kw=None,
             kk=None, ko=ONE, ks=256, dtype=1, mn=64, d=64, eps=1e-6, rope=None)
    a.update(over)
    return b.lib.rs3_qk_norm_rope(*a.values(), None)


@pytest.mark.parametrize("over,code", [
    (dict(q=None), "EINVAL"), (dict(qo=None), "EINVAL"), (dict(q=ODD), "EINVAL"), (dict(ko=ODD), "EINVAL"),
    (dict(q_rows=-1), "EINVAL"), (dict(Hq=0), "EINVAL"), (dict(d=0), "EINVAL"), (dict(d=60), "EINVAL"), (dict(mn=0), "EINVAL"),
    (dict(q_stride=255), "EINVAL"), (dict(q_stride=260), "EINVAL"), (dict(ks=248), "EINVAL"), (dict(ks=512), "EINVAL"),
    (dict(eps=-1.0), "EINVAL"), (dict(eps=float("nan")), "EINVAL"), (dict(rope=ODD), "EINVAL"), (dict(qw=ODD), "EINVAL"),
    (dict(dtype=2), "EINVAL"), (dict(d=264, q_stride=1056, k_stride=1056, qs=1056, ks=1056), "EUNSUPPORTED"),
    (dict(mn=20000), "EUNSUPPORTED")])
def test_norm_refusals(b, over, code):
    assert _norm(b, **over) == getattr(b, "RS3_" + code)


def test_norm_of_nothing(b):
    none = dict(q=None, qo=None, q_rows=0, k=None, ko=None, k_rows=0)
    assert _norm(b, **none) == b.RS3_OK
    assert _norm(b, q_rows=0, k=None, ko=None, k_rows=0) == b.RS3_OK


def test_bank_blocks(b):
    x = _bank(b)                                           # 64 + 1000 + 4 rows
    assert [b.lib.rs3_bank_blocks(ctypes.byref(x), n) for n in (32, 64, 128)] == [34, 17, 9]
    assert b.lib.rs3_bank_blocks(ctypes.byref(x), 0) == -1
    assert b.lib.rs3_bank_blocks(ctypes.byref(b.BankDesc()), 64) == -1
    assert b.lib.rs3_bank_blocks(None, 64) == -1


def test_copy_refusals(b):
    def call(dst, src, parent=ONE, keep=None, stride=0, ws=None, n=0, status=ONE):
        return b.lib.rs3_bank_copy(ctypes.byref(dst), ctypes.byref(src), parent, keep, stride, ws, n, status, None)

    far = dict(k=1 << 41, v=1 << 42, meta=1 << 43)
    src, dst = _bank(b), _bank(b, **far)
    E = b.RS3_EINVAL
    assert call(b.BankDesc(), src) == E and call(dst, b.BankDesc()) == E
    assert call(dst, src, parent=None) == E and call(dst, src, status=None) == E
    for over in (dict(H=2), dict(d=32), dict(dtype="f32"), dict(mn=32)):
        assert call(_bank(b, **over, **far), src) == E, over
    assert call(dst, src, keep=ONE, stride=0, ws=ONE, n=1 << 20) == E
    assert call(dst, src, keep=ONE, stride=1068, ws=None, n=0) == E
    assert call(dst, src, keep=ONE, stride=1068, ws=ODD, n=1 << 20) == E
    need = b.rs3_bank_copy_workspace_bytes(2, 1068)
    assert call(dst, src, keep=ONE, stride=1068, ws=ONE, n=need - 1) == b.RS3_ECAPACITY
    # storage that overlaps without being the same bank
    assert call(_bank(b, k=(1 << 20) + 4096, v=1 << 42, meta=1 << 43), src) == E
    assert call(_bank(b, k=1 << 41, v=1 << 20, meta=1 << 43), src) == E
    assert call(_bank(b, k=1 << 41, v=1 << 42, meta=1 << 40), src) == E
    assert call(_bank(b, U=1), src) == E                   # the same storage in another shape
    assert b.rs3_bank_copy_workspace_bytes(2, 0) == 0 and b.rs3_bank_copy_workspace_bytes(0, 5) == 0
    sizes = [b.rs3_bank_copy_workspace_bytes(3, n) for n in (1, 255, 256, 257, 5000, 1 << 20)]
    assert sizes == sorted(sizes)
    assert b.lib.rs3_bank_drop_frames(ctypes.byref(src), ONE, None, None, None) == E
    assert b.lib.rs3_bank_drop_frames(ctypes.byref(b.BankDesc()), ONE, None, ONE, None) == E


def test_digest_refusals(b):
    def call(bank, block=64, refresh=-1, digest=ONE, step=ONE, status=ONE):
        return b.lib.rs3_bank_digest(ctypes.byref(bank), block, refresh, digest, step, status, None)

    x = _bank(b)
    E, U = b.RS3_EINVAL, b.RS3_EUNSUPPORTED
    assert call(b.BankDesc()) == E and call(x, digest=None) == E and call(x, step=None) == E and call(x, status=None) == E
    assert call(x, digest=ODD) == E and call(x, step=ODD) == E and call(x, refresh=-2) == E
    for block in (0, 16, 48, 256):
        assert call(x, block=block) == U
    assert call(_bank(b, d=80)) == U and call(_bank(b, d=8)) == U and call(_bank(b, d=512)) == U


def test_select_and_readout_refusals(b):
    x = _bank(b)
    nb = b.lib.rs3_bank_blocks(ctypes.byref(x), 64)
    base = dict(q=ONE, dtype=1, G=1, mn=64, H=4, d=64, ug=ONE, idx=ONE, count=ONE, k_max=20, bank=x, block=64)

    def select(digest=ONE, step=ONE, rope=None, n_top=4, sel=ONE, ws=ONE, n=1 << 30, status=ONE, **over):
        a = {**base, **over}
        a["bank"] = ctypes.byref(a["bank"])
        return b.lib.rs3_block_select(*a.values(), digest, step, rope, n_top, sel, ws, n, status, None)

    def readout(sel=ONE, n_top=4, rope=None, residual=None, out=ONE, scale=0.0, ws=ONE, n=1 << 40, status=ONE, **over):
        a = {**base, **over}
        a["bank"] = ctypes.byref(a["bank"])
        return b.lib.rs3_sparse_readout(*a.values(), sel, n_top, rope, residual, out, scale, ws, n, status, None)

    E, U = b.RS3_EINVAL, b.RS3_EUNSUPPORTED
    for call in (select, readout):
        for over in (dict(q=None), dict(ug=None), dict(idx=None), dict(count=None), dict(status=None), dict(bank=b.BankDesc()),
                     dict(G=0), dict(mn=0), dict(mn=32), dict(H=2), dict(d=128), dict(dtype=0), dict(k_max=-1), dict(k_max=65),
                     dict(q=ODD), dict(rope=ODD), dict(n_top=0), dict(sel=None), dict(ws=None), dict(ws=ODD)):
            assert call(**over) == E, over
        for over in (dict(block=16), dict(block=0), dict(n_top=1025), dict(d=80, bank=_bank(b, d=80))):
            assert call(**over) == U, over
    for over in (dict(digest=None), dict(step=None), dict(digest=ODD)):
        assert select(**over) == E, over
    assert select(n=b.rs3_block_select_workspace_bytes(2, 4, 20, nb) - 1) == b.RS3_ECAPACITY
    assert select(bank=_bank(b, ring=49153 * 64)) == U
    for over in (dict(out=None), dict(out=ODD), dict(residual=ODD), dict(scale=-1.0), dict(scale=float("nan")),
                 dict(scale=float("inf"))):
        assert readout(**over) == E, over
    assert readout(n=b.rs3_sparse_readout_workspace_bytes(2, 4, 64, 20, 4, nb, "bf16") - 1) == b.RS3_ECAPACITY


def test_workspace_sizes_never_fall(b):
    grow = [(1, 1, 1, 1, 1), (1, 1, 1, 4, 1), (1, 1, 9, 4, 1), (1, 1, 9, 4, 100), (1, 3, 9, 4, 100), (5, 3, 9, 4, 100),
            (5, 3, 1228, 4, 100), (5, 3, 1228, 32, 100), (5, 3, 1228, 32, 5000), (48, 4, 2764, 64, 9000)]
    for dtype in ("bf16", "f32"):
        for d in (16, 64, 256):
            sizes = [b.rs3_sparse_readout_workspace_bytes(U, H, d, k, n, nb, dtype) for U, H, k, n, nb in grow]
            assert sizes == sorted(sizes) and sizes[0] > 0
    sizes = [b.rs3_block_select_workspace_bytes(U, H, k, nb) for U, H, k, n, nb in grow]
    assert sizes == sorted(sizes) and sizes[0] > 0
    assert b.rs3_block_select_workspace_bytes(0, 1, 1, 1) == 0
    assert b.rs3_sparse_readout_workspace_bytes(1, 1, 64, 1, 0, 1, "bf16") == 0


def test_binding_refuses_tensors_that_are_not_what_the_call_reads(b):
    x = torch.zeros(64, 256, dtype=torch.bfloat16)
    for dev, t, dtype, n in ((0, x, torch.bfloat16, 1), (0, None, torch.bfloat16, 1), (-1, x, torch.float32, 1),
                             (-1, x, torch.bfloat16, 64 * 256 + 1)):
        with pytest.raises(ValueError):
            b._want(dev, "x", t, dtype, n)
    b._want(-1, "x", x, torch.bfloat16, 64 * 256)          # (a CPU tensor's device is -1)
    with pytest.raises(ValueError):
        b._ptr(x.T)
    assert b._rows_of("q", torch.zeros(3, 5, 7, 16)[..., :8], 8) == (105, 16)
    assert b._rows_of("q", torch.zeros(1, 5, 24)[..., 8:16], 8) == (5, 24)
    assert b._rows_of("q", torch.zeros(8), 8) == (1, 8)
    assert b._rows_of("q", torch.zeros(1, 1, 8), 8) == (1, 8)
    assert b._rows_of("q", torch.zeros(0, 5, 8), 8)[0] == 0
    for t in (torch.zeros(4, 6, 8)[:, :5], torch.zeros(6, 4, 8).transpose(0, 1), torch.zeros(4, 9), torch.zeros(8, 4).T):
        with pytest.raises(ValueError):
            b._rows_of("q", t, 8)


def test_copy_refuses_one_storage_in_two_layouts(b):
    """The same stores and counters, regions of other sizes; counters of one bank inside the rows of the other."""
    def call(dst, src):
        return b.lib.rs3_bank_copy(ctypes.byref(dst), ctypes.byref(src), ONE, None, 0, None, 0, ONE, None)

    src = _bank(b)                                         # 64 + 1000 + 4 rows
    for over in (dict(n_cond=0, ring=1064), dict(ring=1003, n_ptr=1), dict(n_cond=0, ring=1000, n_ptr=68), dict(U=1),
                 dict(max_frames=19), dict(ring=999)):
        other = _bank(b, **over)
        assert call(other, src) == b.RS3_EINVAL and call(src, other) == b.RS3_EINVAL, over
    far = dict(k=1 << 41, v=1 << 42, meta=1 << 43)
    inside = (1 << 20) + 4096
    assert call(_bank(b, k=1 << 41, v=1 << 42, meta=inside), src) == b.RS3_EINVAL
    assert call(_bank(b, **far), _bank(b, meta=(1 << 42) + 4096)) == b.RS3_EINVAL


def _at(n):
    return ctypes.c_void_p(4096 + n)


@pytest.mark.parametrize("over", [
    # 64 rows of 4 heads of 64 in bf16 are 32 KB: rows of 512 bytes, adjacent or in rows of 1536 (queries, keys, values)
    dict(qo=_at(16)),                                      # over its input, shifted by a piece
    dict(qo=_at(512)),                                     # shifted by a row
    dict(qo=_at(0), qs=512),                               # in place with rows further apart
    dict(qo=_at(1 << 16), ko=_at(1 << 16)),                # both results in one place
    dict(qo=_at(1 << 17)),                                 # queries' results over the keys
    dict(qo=_at((1 << 17) + 32256)),                       # ... over their last row
    dict(ko=_at(0)),                                       # keys' results over the queries
    dict(k=_at(0), qo=_at(0)),                             # queries in place, the keys the same tensor
    dict(q_stride=768, qo=_at(256), qs=768),               # columns that overlap
    dict(q_stride=768, qo=_at(1280), qs=768),              # ... around the end of a row
    dict(q_stride=768, k=_at(512), k_stride=768, qo=_at(0), qs=768, ko=_at(768), ks=768)])
def test_norm_refuses_results_over_other_operands(b, over):
    a = dict(q=_at(0), qo=_at(1 << 18), k=_at(1 << 17), ko=_at(1 << 19))
    a.update(over)
    assert _norm(b, **a) == b.RS3_EINVAL


def test_readout_workspace_for_one_block_size(b):
    """No more than for any block, what the call asks for, and never falling."""
    x = _bank(b, U=3, H=2, mn=1024, ring=20_000, max_frames=40)
    for dtype, code in (("bf16", 1), ("f32", 0)):
        for d in (16, 64, 128, 256):
            x = _bank(b, U=3, H=2, d=d, dtype=dtype, mn=1024, ring=20_000, max_frames=40)
            for block in (32, 64, 128):
                nb = b.lib.rs3_bank_blocks(ctypes.byref(x), block)
                for k_max, n_top in ((4, 2), (700, 16)):
                    n = b.rs3_sparse_readout_workspace_bytes(3, 2, d, k_max, n_top, nb, dtype, block)
                    most = b.rs3_sparse_readout_workspace_bytes(3, 2, d, k_max, n_top, nb, dtype)
                    if d < 64 or k_max == 4:
                        assert n == most == 16
                    else:
                        # partial results in fp32 are nearly all of it: rows of a part in bytes
                        parts = block // (32 if block == 32 or (dtype == "f32" and d > 64) else 64)
                        assert parts * 3 * 2 * k_max * n_top * d * 4 < n <= most and (n == most) == (block == 128)
                    args = [ONE, code, 1, 1024, 2, d, ONE, ONE, ONE, k_max, ctypes.byref(x), block, ONE, n_top, None, None, ONE, 0.0, ONE]
                    assert b.lib.rs3_sparse_readout(*args, n - 1, ONE, None) == b.RS3_ECAPACITY
    assert b.rs3_sparse_readout_workspace_bytes(1, 1, 64, 1, 1, 1, "bf16", 16) == 0
    grow = [(1, 1, 1, 1, 1), (1, 1, 9, 4, 100), (1, 3, 9, 4, 100), (5, 3, 1228, 4, 100), (5, 3, 1228, 32, 5000), (48, 4, 2764, 64, 9000)]
    for block in (32, 64, 128):
        sizes = [b.rs3_sparse_readout_workspace_bytes(U, H, 64, k, n, nb, "bf16", block) for U, H, k, n, nb in grow]
        assert sizes == sorted(sizes) and sizes[0] > 0
