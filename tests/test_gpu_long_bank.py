"""The calls for long banks against plain implementations in 64 bits: norms of query and
key heads, copies of banks, block digests, block selection, and the readout over chosen blocks."""
import ctypes
import math

import numpy as np
import pytest
import torch

pytestmark = pytest.mark.gpu

DT = {"f32": torch.float32, "bf16": torch.bfloat16}
HALF = {"f32": 2.0 ** -24, "bf16": 2.0 ** -8}              # a rounding to the stored type, relative


@pytest.fixture(scope="module")
def rs3():
    from paper_2608_22526_gb300 import rs3
    return rs3


def gen(seed):
    return torch.Generator(device="cuda").manual_seed(seed)


def status():
    return torch.zeros(1, dtype=torch.int32, device="cuda")


def rope_table(mn, d, seed=1):
    a = torch.rand((mn, d // 2), generator=gen(seed), device="cuda", dtype=torch.float64) * 6.3
    return torch.stack([a.cos(), a.sin()], -1).float().contiguous()


def turned(x, d, table):
    """x [..., mn, D] in 64 bits with every head's pairs turned by their cell's angles."""
    z = torch.view_as_complex(x.unflatten(-1, (-1, d // 2, 2)).contiguous())
    return torch.view_as_real(z * torch.view_as_complex(table.double().contiguous())[:, None]).flatten(-3)


# ---------------------------------------------------------------------------
# norms
# ---------------------------------------------------------------------------
def norm_ref(x, d, w, table, mn, eps):
    """(value, size of its terms) in 64 bits; x [rows, H*d]."""
    h = x.double().unflatten(-1, (-1, d))
    h = h / (h.square().mean(-1, keepdim=True) + eps).sqrt()
    h = h * (1.0 if w is None else w.double())
    y = h.flatten(-2)
    if table is None:
        return y, y.abs()
    cell = torch.arange(x.shape[0], device="cuda") % mn
    t = table.double()[cell]
    p = h.unflatten(-1, (d // 2, 2))
    c, s = t[:, None, :, 0], t[:, None, :, 1]
    out = torch.stack([p[..., 0] * c - p[..., 1] * s, p[..., 0] * s + p[..., 1] * c], -1)
    size = torch.stack([(p[..., 0] * c).abs() + (p[..., 1] * s).abs(), (p[..., 0] * s).abs() + (p[..., 1] * c).abs()], -1)
    return out.flatten(-3), size.flatten(-3)


def check_norm(got, ref, size, dtype):
    # one rounding to the stored type, and in fp32: the sum of at most 256 squares (16 adds in a
    # chain and a tree of five, 21 half-steps of 2^-24, half of it after the root), the mean, the
    # reciprocal root (2 steps = 4 half-steps), three products and a sum: under 32 half-steps of the terms
    tol = HALF[dtype] * ref.abs() + 32 * 2.0 ** -24 * size * (1 + HALF[dtype])
    err = (got.double() - ref).abs()
    assert (err <= tol + 1e-42).all(), float((err - tol).max())


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("d", [8, 16, 24, 64, 80, 128, 248, 256])
@pytest.mark.parametrize("rows,mn,Hq,Hk", [(1, 1, 1, 1), (1, 35, 3, 1), (35, 35, 2, 5), (3 * 35, 35, 1, 2), (71, 35, 4, 4)])
def test_norm_matches_64_bits(rs3, dtype, d, rows, mn, Hq, Hk):
    g = gen(d + rows)
    q = (torch.randn((rows, Hq * d), generator=g, device="cuda") * 3).to(DT[dtype])
    k = torch.randn((2 * rows, Hk * d), generator=g, device="cuda").to(DT[dtype])
    w = [1 + torch.randn(d, generator=g, device="cuda") * 0.3, None]
    table = rope_table(mn, d) if rows % 2 else None
    qo, ko = torch.zeros_like(q), torch.zeros_like(k)
    rs3.rs3_qk_norm_rope(q, qo, k, ko, dtype, mn, Hq, Hk, d, w[0], w[1], 1e-5, table)
    check_norm(qo, *norm_ref(q, d, w[0], table, mn, 1e-5), dtype)
    check_norm(ko, *norm_ref(k, d, w[1], table, mn, 1e-5), dtype)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_norm_packed_in_place_with_masks(rs3, dtype):
    """Queries, keys and values side by side; in place; rows that the mask leaves hold NaN."""
    G, mn, H, d = 3, 20, 2, 64
    x = torch.randn((G, mn, 3 * H * d), generator=gen(5), device="cuda").to(DT[dtype])
    keep = (torch.rand((G, mn), generator=gen(6), device="cuda") < 0.5).to(torch.uint8)
    keep[1] = 0                                            # a grid without any kept row
    x[keep == 0, H * d:2 * H * d] = math.nan
    before = x.clone()
    q, k = x[..., :H * d], x[..., H * d:2 * H * d]
    table = rope_table(mn, d)
    rs3.rs3_qk_norm_rope(q, q, k, k, dtype, mn, H, H, d, eps=1e-6, rope=table, k_keep=keep)
    flat = before.view(-1, 3 * H * d)
    check_norm(q.reshape(-1, H * d), *norm_ref(flat[:, :H * d], d, None, table, mn, 1e-6), dtype)
    on = keep.view(-1) != 0
    ref, size = norm_ref(flat[:, H * d:2 * H * d], d, None, table, mn, 1e-6)
    check_norm(k.reshape(-1, H * d)[on], ref[on], size[on], dtype)
    same = torch.ones_like(x, dtype=torch.bool)
    same[..., :H * d] = False
    same[..., H * d:2 * H * d] = (keep == 0)[..., None]
    bits = torch.int16 if dtype == "bf16" else torch.int32
    assert torch.equal(x.view(bits)[same], before.view(bits)[same])


def test_norm_one_side_zero_rows_and_zero_heads(rs3):
    x = torch.zeros((4, 64), device="cuda")
    x[1:] = torch.randn((3, 64), generator=gen(1), device="cuda") * 1e-3
    y = torch.full_like(x, 7.0)
    rs3.rs3_qk_norm_rope(None, None, x, y, "f32", 2, 0, 1, 64, eps=1e-6)
    assert torch.equal(y[0], torch.zeros(64, device="cuda"))     # a head of zeros
    check_norm(y, *norm_ref(x, 64, None, None, 2, 1e-6), "f32")
    e = x[:0]
    rs3.rs3_qk_norm_rope(e, e, x, y, "f32", 2, 1, 1, 64)
    with pytest.raises(ValueError):
        rs3.rs3_qk_norm_rope(x, y[:3], None, None, "f32", 2, 1, 1, 64)
    with pytest.raises(ValueError):
        rs3.rs3_qk_norm_rope(x.bfloat16(), y, None, None, "f32", 2, 1, 1, 64)


# ---------------------------------------------------------------------------
# banks with known contents
# ---------------------------------------------------------------------------
class Built:
    """A bank filled through commits, and its logical rows as read back from its counters."""

    def __init__(self, rs3, U=3, H=2, d=16, dtype="bf16", m=5, n=7, n_cond=1, window=3, ring_frames=3, commits=5, n_ptr=4, seed=0,
                 density=0.5, empty=(), ring=None, scale=1.0):
        self.rs3, self.U, self.H, self.d, self.D, self.dtype, self.mn = rs3, U, H, d, H * d, dtype, m * n
        g = gen(seed)
        ring = (window * self.mn if window > 0 else ring_frames * self.mn) if ring is None else ring
        self.bank = rs3.Bank(U, H, d, dtype, self.mn, n_cond, window, ring, window if window > 0 else ring_frames, n_ptr)
        # rows that are not live hold NaN: nothing may come of them
        self.bank.k_store.fill_(math.nan)
        self.bank.v_store.fill_(math.nan)
        self.st = status()
        for f in range(n_cond + commits):
            self.commit(g, int(f < n_cond), density, empty, scale)
        if n_ptr:
            kp, vp = (torch.randn((U, n_ptr, self.D), generator=g, device="cuda").to(DT[dtype]) for _ in range(2))
            rs3.rs3_bank_set_pointers(self.bank, kp, vp, self.st)
        assert int(self.st) == 0

    def commit(self, g, is_cond=0, density=0.5, empty=(), scale=1.0):
        shape = (self.U, self.mn, self.D)
        k, v = (torch.randn(shape, generator=g, device="cuda") * s for s in (scale, 1.0))
        mask = (torch.rand(shape[:2], generator=g, device="cuda") < density).to(torch.uint8)
        for u in empty:
            mask[u] = 0
        self.rs3.rs3_bank_commit(self.bank, k.to(DT[self.dtype]), v.to(DT[self.dtype]), mask, is_cond, self.st)

    def places(self, u, bank=None):
        """Storage rows of unit u in logical order, and its frames' lengths."""
        bank = self.bank if bank is None else bank
        meta, frames = self.rs3.rs3_bank_read_meta(bank)
        head, tail, cond, nf, _, _, ptr, length = meta[u]
        ring = [bank.pinned_cap + p % max(1, bank.ring_cap) for p in range(head, tail)]
        rows = list(range(cond)) + ring + [bank.pinned_cap + bank.ring_cap + i for i in range(ptr)]
        assert len(rows) == length
        lens = [int(x) for x in frames[u, :nf, 1]]
        assert sum(lens) == tail - head and [int(x) for x in frames[u, :nf, 0]] == list(head + np.cumsum([0] + lens[:-1]))[:nf]
        return np.array(rows, dtype=np.int64), lens, (int(cond), int(tail - head), int(ptr))


def rows_of(bank, u, rows):
    i = torch.from_numpy(rows).cuda()
    return bank.k_store[u][i], bank.v_store[u][i]


def bits(t):
    return t.contiguous().view(torch.int16 if t.dtype == torch.bfloat16 else torch.int32)


# ---------------------------------------------------------------------------
# copies
# ---------------------------------------------------------------------------
LAYOUTS = [dict(window=3, commits=5), dict(window=3, commits=2), dict(window=-1, ring_frames=9, commits=8),
           dict(window=2, commits=4, n_cond=0, n_ptr=0), dict(window=1, commits=0, n_cond=2), dict(window=-1, ring_frames=400, commits=330, m=2, n=3)]


@pytest.mark.parametrize("layout", LAYOUTS)
@pytest.mark.parametrize("keep", [None, 0.0, 0.4, 1.0])
@pytest.mark.parametrize("dtype,H,d", [("bf16", 1, 8), ("f32", 3, 20)])
def test_copy_takes_the_kept_rows(rs3, layout, keep, dtype, H, d):
    s = Built(rs3, U=4, H=H, d=d, dtype=dtype, empty=(2,), seed=3, **layout)
    t = Built(rs3, U=5, H=H, d=d, dtype=dtype, seed=4, **layout)
    parent = [3, -1, 0, 3, 2]
    before_k, before_v = t.bank.k_store.clone(), t.bank.v_store.clone()
    meta0, _ = rs3.rs3_bank_read_meta(t.bank)
    most = max(len(s.places(u)[0]) for u in range(4))
    mask = None
    if keep is not None:
        mask = (torch.rand((5, most + 3), generator=gen(9), device="cuda") < keep).to(torch.uint8) * 3
    st = status()
    ws = torch.full((rs3.rs3_bank_copy_workspace_bytes(5, most + 3),), 255, dtype=torch.uint8, device="cuda")
    for _ in range(2):                                     # the second call finds the first's workspace and counters
        rs3.rs3_bank_copy(t.bank, s.bank, torch.tensor(parent, dtype=torch.int32, device="cuda"), mask, ws, st)
    assert int(st) == 0
    meta, _ = rs3.rs3_bank_read_meta(t.bank)
    assert np.array_equal(meta[1], meta0[1])
    for u, p in enumerate(parent):
        if p < 0:
            assert torch.equal(bits(t.bank.k_store[u]), bits(before_k[u])) and torch.equal(bits(t.bank.v_store[u]), bits(before_v[u]))
            continue
        rows, lens, (cond, ring, ptr) = s.places(p)
        on = np.ones(len(rows), bool) if mask is None else mask[u, :len(rows)].cpu().numpy() != 0
        got, got_lens, got_n = t.places(u)
        want_n = (int(on[:cond].sum()), int(on[cond:cond + ring].sum()), int(on[cond + ring:].sum()))
        assert got_n == want_n
        ends = cond + np.cumsum([0] + lens)
        assert got_lens == [int(on[a:b].sum()) for a, b in zip(ends[:-1], ends[1:])]
        assert meta[u, 0] == 0 and meta[u, 5] == rs3.rs3_bank_read_meta(s.bank)[0][p, 5]
        for a, b, old in zip(rows_of(s.bank, p, rows[on]), rows_of(t.bank, u, got), (before_k, before_v)):
            assert torch.equal(bits(a), bits(b))
        other = np.setdiff1d(np.arange(t.bank.rows_per_unit), got)
        assert torch.equal(bits(t.bank.k_store[u][other]), bits(before_k[u][other]))
    # the copy takes commits and drops as any bank does
    t.commit(gen(11))
    if layout["window"] > 0:
        assert int(t.st) == 0
    [t.places(u) for u in range(5)]


def test_copy_into_a_larger_ring_and_what_does_not_fit(rs3):
    s = Built(rs3, window=-1, ring_frames=6, commits=6, density=1.0, seed=1)
    big = rs3.Bank(3, s.H, s.d, s.dtype, s.mn, 2, -1, 20 * s.mn, 30, 9)
    st = status()
    same = torch.arange(3, dtype=torch.int32, device="cuda")
    rs3.rs3_bank_copy(big, s.bank, same, None, None, st)
    assert int(st) == 0
    for u in range(3):
        a, b = rows_of(s.bank, u, s.places(u)[0]), rows_of(big, u, s.places(u, big)[0])
        assert torch.equal(bits(a[0]), bits(b[0])) and torch.equal(bits(a[1]), bits(b[1]))
    for over in (dict(n_cond=0), dict(ring=5 * s.mn), dict(max_frames=5), dict(n_ptr=3)):
        a = dict(n_cond=2, ring=20 * s.mn, max_frames=30, n_ptr=9)
        a.update(over)
        small = rs3.Bank(3, s.H, s.d, s.dtype, s.mn, a["n_cond"], -1, a["ring"], a["max_frames"], a["n_ptr"])
        for keep in (None, torch.ones((3, 7 * s.mn + 4), dtype=torch.uint8, device="cuda")):
            st = status()
            ws = torch.empty(rs3.rs3_bank_copy_workspace_bytes(3, 7 * s.mn + 4), dtype=torch.uint8, device="cuda")
            rs3.rs3_bank_copy(small, s.bank, same, keep, ws, st)
            assert int(st) == rs3.RS3_ECAPACITY, over
            assert (rs3.rs3_bank_read_meta(small)[0] == 0).all() and not small.k_store.any()
    # rows that are left fit again
    keep = torch.zeros((3, 7 * s.mn + 4), dtype=torch.uint8, device="cuda")
    keep[:, s.mn:3 * s.mn + 1] = 1
    small = rs3.Bank(3, s.H, s.d, s.dtype, s.mn, 1, -1, 2 * s.mn + 1, 6, 4)
    st = status()
    rs3.rs3_bank_copy(small, s.bank, same, keep, ws, st)
    assert int(st) == 0 and s.places(0, small)[1] == [s.mn, s.mn, 1, 0, 0, 0]


def test_copy_refuses_units_on_the_device(rs3):
    s = Built(rs3, seed=2)
    t = Built(rs3, seed=5)
    length = max(len(s.places(u)[0]) for u in range(3))

    def run(dst, parent, keep=None):
        st = status()
        stride = 1 if keep is None else keep.shape[1]
        ws = torch.empty(rs3.rs3_bank_copy_workspace_bytes(3, stride), dtype=torch.uint8, device="cuda")
        m0 = rs3.rs3_bank_read_meta(dst.bank)[0]
        rs3.rs3_bank_copy(dst.bank, s.bank, torch.tensor(parent, dtype=torch.int32, device="cuda"), keep, ws, st)
        m1 = rs3.rs3_bank_read_meta(dst.bank)[0]
        return int(st), [bool((m0[u] == m1[u]).all()) for u in range(3)]

    assert run(t, [3, -1, -1]) == (rs3.RS3_EINVAL, [True] * 3)
    assert run(t, [-2, -1, -1]) == (rs3.RS3_EINVAL, [True] * 3)
    code, same = run(t, [5, 1, 1])
    assert code == rs3.RS3_EINVAL and same[0] and not same[1] and not same[2]      # the others proceed
    short = torch.ones((3, length - 1), dtype=torch.uint8, device="cuda")
    assert run(t, [0, 1, 2], short)[0] == rs3.RS3_EINVAL
    # one bank: a source stays as it is
    assert run(s, [0, 1, 2])[0] == 0
    assert run(s, [1, 2, -1])[0] == rs3.RS3_EINVAL
    ones = torch.ones((3, length), dtype=torch.uint8, device="cuda")
    assert run(s, [0, -1, -1], ones)[0] == rs3.RS3_EINVAL
    s = Built(rs3, seed=2)
    want = [rows_of(s.bank, 0, s.places(0)[0])[i].clone() for i in range(2)]
    assert run(s, [-1, 0, 0]) == (0, [True, False, False])
    for u in range(3):
        got = rows_of(s.bank, u, s.places(u)[0])
        assert all(torch.equal(bits(a), bits(b)) for a, b in zip(got, want))


@pytest.mark.parametrize("layout", LAYOUTS[:5])
def test_drop_frames(rs3, layout):
    s = Built(rs3, seed=7, **layout)
    before = [s.places(u) for u in range(3)]
    nf = [len(x[1]) for x in before]
    old, new = [min(1, n) for n in nf], [max(0, n - 2) for n in nf]
    old[2], new[2] = nf[2], 0                              # all of them
    st = status()
    rs3.rs3_bank_drop_frames(s.bank, torch.tensor(old, dtype=torch.int32, device="cuda"),
                             torch.tensor(new, dtype=torch.int32, device="cuda"), st)
    assert int(st) == 0
    for u in range(3):
        rows, lens, (cond, ring, ptr) = before[u]
        a, b = sum(lens[:old[u]]), sum(lens[nf[u] - new[u]:])
        got, got_lens, _ = s.places(u)
        assert got_lens == lens[old[u]:nf[u] - new[u]]
        assert np.array_equal(got, np.concatenate([rows[:cond], rows[cond + a:cond + ring - b], rows[cond + ring:]]))
    s.commit(gen(8))
    assert int(s.st) == 0
    [s.places(u) for u in range(3)]
    meta = rs3.rs3_bank_read_meta(s.bank)[0]
    for bad in ([-1, 0, 0], [99, 0, 0]):
        for side in (0, 1):
            st = status()
            arg = [None, None]
            arg[side] = torch.tensor(bad, dtype=torch.int32, device="cuda")
            rs3.rs3_bank_drop_frames(s.bank, *arg, st)
            assert int(st) == rs3.RS3_EINVAL
    assert np.array_equal(meta, rs3.rs3_bank_read_meta(s.bank)[0])


# ---------------------------------------------------------------------------
# digests
# ---------------------------------------------------------------------------
def eight_bits(x):
    """[..., d] fp32 on the CPU -> whole numbers, steps (np.float32)."""
    a = np.abs(x).max(-1)
    e = np.frexp(a)[1] - 1
    some = a >= np.float32(2.0 ** -100)
    t = np.clip(np.rint(np.ldexp(x.astype(np.float64), (6 - e)[..., None])), -127, 127)
    return np.where(some[..., None], t, 0), np.where(some, np.ldexp(1.0, e - 6), 0.0)


def digest_ref(b, u, bs, nb):
    rows = b.places(u)[0]
    k = b.bank.k_store[u].float().cpu().numpy()
    x = np.zeros((nb * bs, b.D), np.float32)
    x[rows] = k[rows]
    n = np.bincount(rows // bs, minlength=nb)
    x = x.reshape(nb, bs // 8, 8, b.D)
    p = x[:, 0].copy()
    for i in range(1, bs // 8):
        p = p + x[:, i]
    s = ((p[:, 0] + p[:, 4]) + (p[:, 2] + p[:, 6])) + ((p[:, 1] + p[:, 5]) + (p[:, 3] + p[:, 7]))
    mean = (s / np.maximum(n, 1)[:, None].astype(np.float32)).reshape(nb, b.H, b.d)
    t, step = eight_bits(mean)
    return t.transpose(1, 0, 2), step.T, n


def make_digest(b, block, fill=None):
    nb = b.bank.blocks(block)
    dig = torch.full((b.U, b.H, nb, b.d), 77, dtype=torch.int8, device="cuda")
    step = torch.full((b.U, b.H, nb), 0.5, device="cuda")
    return dig, step, nb


HEADS = [("bf16", 1, 16), ("bf16", 5, 64), ("bf16", 3, 256), ("f32", 1, 32), ("f32", 3, 64), ("f32", 2, 256), ("f32", 3, 16)]


@pytest.mark.parametrize("dtype,H,d", HEADS)
@pytest.mark.parametrize("block", [32, 64, 128])
def test_digest_of_all_blocks(rs3, dtype, H, d, block):
    b = Built(rs3, H=H, d=d, dtype=dtype, m=9, n=11, window=3, commits=5, empty=(1,), seed=block)
    b.bank.k_store[0, :block] *= 1e-36 if dtype == "f32" else 1.0      # a block below 2^-100
    dig, step, nb = make_digest(b, block)
    rs3.rs3_bank_digest(b.bank, block, -1, dig, step, b.st)
    assert int(b.st) == 0
    for u in range(b.U):
        t, s, n = digest_ref(b, u, block, nb)
        assert np.array_equal(step[u].cpu().numpy(), s.astype(np.float32))
        assert np.array_equal(dig[u].cpu().numpy(), t.astype(np.int8))
        assert (s[:, n == 0] == 0).all()


@pytest.mark.parametrize("window,n_ptr", [(3, 4), (-1, 0), (2, 5)])
@pytest.mark.parametrize("block", [32, 64])
def test_digest_refresh_follows_commits_and_drops(rs3, window, n_ptr, block):
    """After every commit refresh = 1, after a drop refresh = 0: every block with a live row is up to date."""
    b = Built(rs3, m=6, n=7, window=window, ring_frames=12, commits=1, n_ptr=n_ptr, seed=13)
    dig, step, nb = make_digest(b, block)
    rs3.rs3_bank_digest(b.bank, block, -1, dig, step, b.st)
    g = gen(17)

    def same():
        for u in range(b.U):
            t, s, n = digest_ref(b, u, block, nb)
            on = n > 0
            assert np.array_equal(step[u].cpu().numpy()[:, on], s.astype(np.float32)[:, on])
            assert np.array_equal(dig[u].cpu().numpy()[:, on], t.astype(np.int8)[:, on])

    for i in range(9):
        b.commit(g, density=[0.5, 1.0, 0.1][i % 3], empty=(i % 3,))
        rs3.rs3_bank_digest(b.bank, block, 1, dig, step, b.st)
        same()
        if i % 3 == 2:
            one = torch.ones(3, dtype=torch.int32, device="cuda")
            rs3.rs3_bank_drop_frames(b.bank, one, None, b.st)
            rs3.rs3_bank_digest(b.bank, block, 0, dig, step, b.st)
            same()
            rs3.rs3_bank_drop_frames(b.bank, None, one, b.st)
            rs3.rs3_bank_digest(b.bank, block, 0, dig, step, b.st)
            same()
            b.commit(g)
            b.commit(g)
            rs3.rs3_bank_digest(b.bank, block, 2, dig, step, b.st)
            same()
    assert int(b.st) == 0


# ---------------------------------------------------------------------------
# selection
# ---------------------------------------------------------------------------
def queries(b, G, k_max, counts, seed=21, scale=1.0):
    g = gen(seed)
    q = (torch.randn((G, b.mn, b.D), generator=g, device="cuda") * scale).to(DT[b.dtype])
    idx = torch.full((b.U, max(1, k_max)), -9, dtype=torch.int32, device="cuda")
    for u, n in enumerate(counts):
        idx[u, :n] = torch.randperm(b.mn, generator=g, device="cuda")[:n].sort().values.to(torch.int32)
    group = torch.arange(b.U, dtype=torch.int32, device="cuda") % G
    return q, idx[:, :k_max].contiguous(), torch.tensor(counts, dtype=torch.int32, device="cuda"), group


def select_ref(b, q, idx, counts, group, dig, step, table, block, nb, n_top, sel):
    sel = sel.copy()
    qf = q.float().cpu().numpy()
    if table is not None:
        t = table.cpu().numpy()
        p = qf.reshape(qf.shape[0], b.mn, b.H, b.d // 2, 2)
        c, s = t[:, None, :, 0], t[:, None, :, 1]
        qf = np.stack([p[..., 0] * c - p[..., 1] * s, p[..., 0] * s + p[..., 1] * c], -1).astype(np.float32).reshape(qf.shape)
    dig, step = dig.cpu().numpy().astype(np.int64), step.cpu().numpy().astype(np.float64)
    for u, n in enumerate(counts):
        live = np.bincount(b.places(u)[0] // block, minlength=nb) > 0
        for j in range(n):
            x = qf[int(group[u]), int(idx[u, j])].reshape(b.H, b.d)
            tq, _ = eight_bits(x)
            for h in range(b.H):
                score = (dig[u, h] @ tq[h].astype(np.int64)) * step[u, h]
                order = [i for i in np.argsort(-score, kind="stable") if live[i]][:n_top]
                sel[u, h, j] = sorted(order) + [-1] * (n_top - len(order))
    return sel


@pytest.mark.parametrize("dtype,H,d", [("bf16", 1, 16), ("bf16", 3, 64), ("bf16", 2, 256), ("bf16", 1, 128), ("bf16", 4, 32), ("f32", 2, 64),
                                       ("f32", 1, 256), ("f32", 3, 16)])
@pytest.mark.parametrize("n_top,block,commits,rope", [(1, 32, 9, False), (5, 32, 40, True), (16, 64, 40, False), (200, 32, 9, True)])
def test_select_is_exact(rs3, dtype, H, d, n_top, block, commits, rope):
    b = Built(rs3, U=3, H=H, d=d, dtype=dtype, m=8, n=9, window=-1, ring_frames=commits, commits=commits, empty=(1,), n_ptr=0, n_cond=1,
              seed=n_top, ring=commits * 50)
    dig, step, nb = make_digest(b, block)
    rs3.rs3_bank_digest(b.bank, block, -1, dig, step, b.st)
    counts = [21, 5, 0]
    q, idx, count, group = queries(b, 2, 21, counts)
    table = rope_table(b.mn, d) if rope else None
    q[1] = 0                                               # scores all zero: ties everywhere
    sel = torch.full((b.U, H, 21, n_top), -5, dtype=torch.int32, device="cuda")
    want = select_ref(b, q, idx, counts, group, dig, step, table, block, nb, n_top, sel.cpu().numpy())
    ws = torch.full((rs3.rs3_block_select_workspace_bytes(b.U, H, 21, nb),), 255, dtype=torch.uint8, device="cuda")
    for _ in range(2):
        rs3.rs3_block_select(q, dtype, 2, b.mn, H, d, group, idx, count, 21, b.bank, block, dig, step, table, n_top, sel, ws, b.st)
        assert int(b.st) == 0
        assert np.array_equal(sel.cpu().numpy(), want)


@pytest.mark.parametrize("rows,n_top,block", [(70_000, 32, 64), (260_000, 7, 32), (400_000, 64, 32), (49_152 * 32 - 64, 3, 32), (300, 1024, 32),
                                              (49_152 * 32 - 64, 64, 32), (32_700, 40, 32), (32_700, 1024, 32), (33_000, 65, 32),
                                              (200_000, 65, 32), (200_000, 1024, 64)])
def test_select_over_many_blocks(rs3, rows, n_top, block):
    """Thousands of blocks, digests and steps given: few different scores, so most choices are ties."""
    d, H, mn = 16, 1, 64
    bank = rs3.Bank(1, H, d, "bf16", mn, 1, -1, rows, 4, 0)
    st = status()
    k = torch.randn((1, mn, d), generator=gen(1), device="cuda").bfloat16()
    rs3.rs3_bank_commit(bank, k, k, None, 1, st)
    bank.counters[0, 1] = rows - 100                       # as if the ring had been filled
    nb = bank.blocks(block)
    g = gen(2)
    dig = torch.randint(-3, 4, (1, H, nb, d), generator=g, device="cuda").to(torch.int8)
    step = torch.randint(1, 3, (1, H, nb), generator=g, device="cuda").float() / 64
    q = torch.randint(-2, 3, (1, mn, d), generator=g, device="cuda").bfloat16()
    q[..., 0] = 2                                          # every query has the same step: t = 32 q
    n = 20
    idx = torch.arange(n, dtype=torch.int32, device="cuda").view(1, n)
    sel = torch.full((1, H, n, n_top), -5, dtype=torch.int32, device="cuda")
    ws = torch.empty(rs3.rs3_block_select_workspace_bytes(1, H, n, nb), dtype=torch.uint8, device="cuda")
    one = torch.tensor([n], dtype=torch.int32, device="cuda")
    zero = torch.zeros(1, dtype=torch.int32, device="cuda")
    rs3.rs3_block_select(q, "bf16", 1, mn, H, d, zero, idx, one, n, bank, block, dig, step, None, n_top, sel, ws, st)
    assert int(st) == 0
    score = (q[0, :n].double() @ dig[0, 0].double().T) * step[0, 0].double()
    live = torch.arange(nb, device="cuda") * block < mn + rows - 100
    score[:, ~live] = -math.inf
    order = score.argsort(dim=1, descending=True, stable=True)[:, :n_top]
    m = min(n_top, int(live.sum()))
    want = torch.full((n, n_top), -1, device="cuda", dtype=torch.int32)
    want[:, :m] = order[:, :m].sort(1).values.to(torch.int32)
    assert torch.equal(sel[0, 0], want)


@pytest.mark.parametrize("dtype,H,d,U,k_max,n_top,rows,spread,rope", [
    ("bf16", 4, 64, 40, 21, 16, 900, 127, True), ("bf16", 1, 16, 160, 130, 5, 3_000, 2, False), ("bf16", 2, 32, 80, 40, 32, 70_000, 127, False),
    ("f32", 2, 64, 80, 33, 7, 2_000, 1, True), ("f32", 1, 32, 80, 250, 32, 9_000, 2, False), ("bf16", 1, 64, 160, 9, 20, 300_000, 0, False),
    ("bf16", 1, 64, 160, 9, 1, 40, 9, False), ("bf16", 2, 64, 40, 250, 30, 40_000, 40, False)])
def test_select_for_many_queries(rs3, dtype, H, d, U, k_max, n_top, rows, spread, rope):
    """Enough queries to fill the SMs; digests given: `spread` 127 is random, small ones are full of ties, 0 is nothing but
    them; units of every length from none to all rows; scores that grow with the blocks."""
    mn = 256
    bank = rs3.Bank(U, H, d, dtype, mn, 1, -1, rows, 4, 3)
    st = status()
    g = gen(rows)
    # counters as if the rings had been filled and turned over
    counters = bank.counters.cpu()
    for u in range(U):
        live = rows * (u % 7) // 6
        head = (u * 37) % max(1, rows)
        counters[u] = torch.tensor([head, head + live, [0, 5, mn][u % 3], int(live > 0), 0, int(u % 3 > 0), [3, 0, 1][u % 3]])
    bank.counters.copy_(counters)
    nb = bank.blocks(32)
    shape = (U, H, nb, d)
    dig = torch.randint(-max(1, spread), max(1, spread) + 1, shape, generator=g, device="cuda") * (spread > 0)
    if U == 80:
        dig[..., 0] = torch.arange(nb, device="cuda") * 127 // nb
    dig = dig.to(torch.int8)
    step = torch.randint(1, 3, shape[:3], generator=g, device="cuda").float() / 64
    q = torch.randn((2, mn, H * d), generator=g, device="cuda").to(DT[dtype])
    if U == 80:
        q.view(2, mn, H, d)[..., 0] = 3.0
    counts = [(k_max * (5 + u) // 7) % (k_max + 1) for u in range(U)]
    idx = torch.stack([torch.randperm(mn, generator=g, device="cuda")[:k_max].sort().values for _ in range(U)]).to(torch.int32)
    count = torch.tensor(counts, dtype=torch.int32, device="cuda")
    group = (torch.arange(U, device="cuda") % 2).to(torch.int32)
    table = rope_table(mn, d) if rope else None
    sel = torch.full((U, H, k_max, n_top), -5, dtype=torch.int32, device="cuda")
    ws = torch.empty(rs3.rs3_block_select_workspace_bytes(U, H, k_max, nb), dtype=torch.uint8, device="cuda")
    rs3.rs3_block_select(q, dtype, 2, mn, H, d, group, idx, count, k_max, bank, 32, dig, step, table, n_top, sel, ws, st)
    assert int(st) == 0
    x = q.float().cpu()
    if rope:
        p, t = x.view(2, mn, H, d // 2, 2), table.cpu()[:, None]
        x = torch.stack([p[..., 0] * t[..., 0] - p[..., 1] * t[..., 1], p[..., 0] * t[..., 1] + p[..., 1] * t[..., 0]], -1).view(2, mn, H * d)
    tq = torch.from_numpy(eight_bits(x.view(2, mn, H, d).numpy())[0]).cuda()
    for u in range(U):
        head, tail, cond, _, _, _, ptr = counters[u].tolist()
        at = torch.arange(tail - head, device="cuda")
        places = torch.cat([torch.arange(cond, device="cuda"), mn + (head + at) % rows, mn + rows + torch.arange(ptr, device="cuda")])
        live = torch.zeros(nb, dtype=torch.bool, device="cuda")
        live[places // 32] = True
        n = counts[u]
        assert (sel[u, :, n:] == -5).all()
        if n == 0:
            continue
        score = torch.einsum("jhd,hbd->hjb", tq[u % 2, idx[u, :n].long()], dig[u].double()) * step[u].double()[:, None]
        score.masked_fill_(~live, -math.inf)
        m = min(n_top, int(live.sum()))
        best = score.argsort(dim=-1, descending=True, stable=True)[..., :m].sort(-1).values
        assert torch.equal(sel[u, :, :n, :m].long(), best), u
        assert (sel[u, :, :n, m:] == -1).all()


def test_select_wait_limit_runs_out_and_the_context_stays_usable(rs3):
    U, H, d, mn, k_max = 160, 1, 64, 64, 5
    bank = rs3.Bank(U, H, d, "bf16", mn, 1, -1, 640, 4, 0)
    st = status()
    k = torch.randn((U, mn, d), generator=gen(1), device="cuda").bfloat16()
    rs3.rs3_bank_commit(bank, k, k, None, 1, st)
    bank.counters[:, 1] = 640                              # as if the ring had been filled
    nb = bank.blocks(32)
    dig = torch.zeros((U, H, nb, d), dtype=torch.int8, device="cuda")
    step = torch.zeros((U, H, nb), device="cuda")
    idx = torch.arange(k_max, dtype=torch.int32, device="cuda").expand(U, k_max).contiguous()
    count = torch.full((U,), k_max, dtype=torch.int32, device="cuda")
    zero = torch.zeros(U, dtype=torch.int32, device="cuda")
    ws = torch.empty(rs3.rs3_block_select_workspace_bytes(U, H, k_max, nb), dtype=torch.uint8, device="cuda")
    codes, sels, digs = [], [], []
    for limit in (10 ** 9, 0, 10 ** 9):
        st = status()
        sel = torch.zeros((U, H, k_max, 2), dtype=torch.int32, device="cuda")
        rs3.rs3_set_wait_limit_ns(limit)
        try:
            rs3.rs3_bank_digest(bank, 32, -1, dig, step, st)
            torch.cuda.synchronize()
            codes.append(int(st))
            st.zero_()
            rs3.rs3_block_select(k[:1], "bf16", 1, mn, H, d, zero, idx, count, k_max, bank, 32, dig, step, None, 2, sel, ws, st)
            torch.cuda.synchronize()
        finally:
            rs3.rs3_set_wait_limit_ns(10 ** 9)
        codes.append(int(st))
        sels.append(sel)
        digs.append(dig.clone())
    T = rs3.RS3_ETIMEOUT
    assert codes == [0, 0, T, T, 0, 0]
    assert torch.equal(sels[0], sels[2]) and torch.equal(digs[0], digs[2])


# ---------------------------------------------------------------------------
# the readout over chosen blocks
# ---------------------------------------------------------------------------
def readout_ref(b, q, idx, counts, group, sel, table, block, scale, res, out0):
    """(out, tolerance) in 64 bits: out starts as out0 outside the kept cells."""
    bf = b.dtype == "bf16"
    half = HALF[b.dtype]
    out = (out0 if res is None else res).double().clone()
    tol = torch.zeros_like(out)
    qd = q.double()
    if table is not None:
        qd = turned(qd, b.d, table)
    for u, n in enumerate(counts):
        rows = torch.from_numpy(b.places(u)[0]).cuda()
        k, v = (x[u][rows].double() for x in (b.bank.k_store, b.bank.v_store))
        blk = rows // block
        for j in range(n):
            cell = int(idx[u, j])
            for h in range(b.H):
                col = slice(h * b.d, (h + 1) * b.d)
                times = torch.zeros(b.bank.blocks(block), device="cuda", dtype=torch.float64)
                for e in sel[u, h, j].tolist():
                    if 0 <= e < times.numel():
                        times[e] += 1
                w = times[blk] if rows.numel() else times[:0]
                A = torch.zeros(b.d, device="cuda", dtype=torch.float64)
                size = A.clone()
                s_abs = 0.0
                if float(w.sum()) > 0:
                    x = k[:, col] @ qd[int(group[u]), cell, col] * scale
                    x[w == 0] = -math.inf
                    p = torch.exp(x - x.max()) * w
                    p = p / p.sum()
                    A, size = p @ v[:, col], p @ v[:, col].abs()
                    s_abs = float(((k[:, col].abs() @ qd[int(group[u]), cell, col].abs()) * scale)[w > 0].max())
                r = torch.zeros_like(A) if res is None else res[u, cell, col].double()
                out[u, cell, col] = r + A
                # fp32 sums of scores, weights and values: under 300 half-steps; bf16: the weights are rounded
                # once (2^-8 of each), a rotated query too (its scores off by 2^-8 of their terms, a weight by
                # twice that beside its neighbours), and the result
                e_s = s_abs * (2.0 ** -24 * 300 + (half if bf and table is not None else 0.0))
                tol[u, cell, col] = half * (r + A).abs() + size * (math.expm1(2 * e_s) + 300 * 2.0 ** -24 + (half if bf else 0.0)) * 1.01 + 1e-30
    return out, tol


def run_readout(rs3, b, q, idx, count, group, sel, table, block, scale, res, out, G):
    nb, k_max, n_top = b.bank.blocks(block), sel.shape[2], sel.shape[3]
    ws = torch.full((rs3.rs3_sparse_readout_workspace_bytes(b.U, b.H, b.d, k_max, n_top, nb, b.dtype),), 255, dtype=torch.uint8,
                    device="cuda")
    rs3.rs3_sparse_readout(q, b.dtype, G, b.mn, b.H, b.d, group, idx, count, k_max, b.bank, block, sel, n_top, table, res, out, scale,
                           ws, b.st)
    return ws


SHAPES = [("bf16", 1, 16), ("bf16", 2, 32), ("bf16", 3, 64), ("bf16", 2, 128), ("bf16", 1, 256), ("f32", 2, 16), ("f32", 3, 64),
          ("f32", 1, 128), ("f32", 2, 256)]


@pytest.mark.parametrize("dtype,H,d", SHAPES)
@pytest.mark.parametrize("n_top,block,residual,rope", [(1, 32, "none", False), (4, 64, "inplace", True), (7, 32, "other", False),
                                                       (3, 128, "inplace", False)])
@pytest.mark.parametrize("counts", [[1, 0, 3], [40, 17, 33]])
def test_sparse_readout_matches_64_bits(rs3, dtype, H, d, n_top, block, residual, rope, counts):
    """Lists with gaps, a unit without rows, wrapped rings, blocks across region ends, NaN in dead rows."""
    b = Built(rs3, U=3, H=H, d=d, dtype=dtype, m=8, n=9, window=4, commits=7, n_ptr=5, empty=(1,), seed=n_top, scale=1.5)
    if counts[1]:
        rs3.rs3_bank_reset(b.bank, 1)                      # unit 1: not even pointers
    nb = b.bank.blocks(block)
    q, idx, count, group = queries(b, 2, 40, counts, scale=1.2)
    g = gen(31)
    sel = torch.rand((b.U, H, 40, nb), generator=g, device="cuda").argsort(-1)[..., :n_top].to(torch.int32)
    if sel.shape[-1] < n_top:
        sel = torch.nn.functional.pad(sel, (0, n_top - sel.shape[-1]), value=-1)
    sel = torch.where(torch.rand(sel.shape, generator=g, device="cuda") < 0.2, -1, sel).contiguous()
    sel[0, :, 0] = -1                                      # a query without blocks
    table = rope_table(b.mn, d) if rope else None
    x = torch.randn((b.U, b.mn, b.D), generator=g, device="cuda").to(DT[dtype])
    res = None if residual == "none" else x.clone()
    out = res if residual == "inplace" else torch.full_like(x, math.nan)
    want, tol = readout_ref(b, q, idx, counts, group, sel, table, block, 0.11 if rope else d ** -0.5, None if res is None else x,
                            torch.zeros_like(x))
    run_readout(rs3, b, q, idx, count, group, sel, table, block, 0.11 if rope else 0.0, res, out, 2)
    assert int(b.st) == 0
    err = (out.double() - want).abs()
    assert (err <= tol).all(), (float((err - tol).max()), float(err.max()))


@pytest.mark.parametrize("dtype,H,d", [("bf16", 2, 64), ("bf16", 1, 64), ("bf16", 1, 128), ("bf16", 3, 256), ("f32", 1, 64), ("f32", 2, 64),
                                       ("f32", 2, 128), ("f32", 1, 256)])
@pytest.mark.parametrize("block,n_top", [(32, 19), (64, 11), (128, 6)])
@pytest.mark.parametrize("residual,rope", [("none", True), ("inplace", False), ("other", True)])
def test_sparse_readout_of_many_queries(rs3, dtype, H, d, block, n_top, residual, rope):
    """Enough queries that a block's go together; half of them choose among a few blocks, others have gaps; NaN in
    dead rows, a unit without rows, one without queries, a wrapped ring."""
    counts = [143, 90, 0, 131]
    b = Built(rs3, U=4, H=H, d=d, dtype=dtype, m=12, n=12, window=5, commits=8, n_ptr=5, empty=(1,), seed=n_top)
    rs3.rs3_bank_reset(b.bank, 1)
    nb = b.bank.blocks(block)
    k_max = 143
    q, idx, count, group = queries(b, 2, k_max, counts)
    g = gen(33)
    key = torch.rand((b.U, H, k_max, nb), generator=g, device="cuda")
    key[:, :, ::2, n_top + 1:] += 1.0
    sel = key.argsort(-1)[..., :n_top].to(torch.int32)
    if nb < n_top:
        sel = torch.nn.functional.pad(sel, (0, n_top - nb), value=-1)
    sel = torch.where(torch.rand(sel.shape, generator=g, device="cuda") < 0.1, -1, sel).contiguous()
    sel[0, :, 5] = -1
    table = rope_table(b.mn, d) if rope else None
    x = torch.randn((b.U, b.mn, b.D), generator=g, device="cuda").to(DT[dtype])
    res = None if residual == "none" else x.clone()
    out = res if residual == "inplace" else torch.full_like(x, math.nan)
    some = list(range(0, 143, 9)) + [1, 142]
    part = idx[:, some].contiguous()
    counts_of = [sum(i < n for i in some) for n in counts]
    order = [sorted((i >= n, i) for i in some) for n in counts]
    for u in range(b.U):                                   # the checked queries of a unit: those that are kept
        part[u] = idx[u, [i for _, i in order[u]]]
    sub = torch.stack([sel[u][:, [i for _, i in order[u]]] for u in range(b.U)])
    want, tol = readout_ref(b, q, part, counts_of, group, sub, table, block, d ** -0.5, None if res is None else x, torch.zeros_like(x))
    run_readout(rs3, b, q, idx, count, group, sel, table, block, 0.0, res, out, 2)
    assert int(b.st) == 0
    checked = torch.zeros((b.U, b.mn), dtype=torch.bool, device="cuda")
    for u, n in enumerate(counts):
        checked[u] = True
        checked[u, idx[u, :n].long()] = False              # cells that are not kept pass through
        checked[u, part[u, :counts_of[u]].long()] = True
    err = (out.double() - want).abs()
    assert (err <= tol)[checked].all(), float((err - tol)[checked].max())
    assert not out.isnan().any()


def test_sparse_readout_wait_limit_runs_out_and_the_context_stays_usable(rs3):
    b = Built(rs3, U=1, H=1, d=64, m=20, n=20, window=-1, ring_frames=8, commits=8, n_ptr=0, seed=6)
    q, idx, count, group = queries(b, 1, 400, [400])
    nb = b.bank.blocks(64)
    sel = torch.arange(nb, dtype=torch.int32, device="cuda").expand(1, 1, 400, nb).contiguous()
    outs = [torch.zeros((1, b.mn, 64), dtype=torch.bfloat16, device="cuda") for _ in range(2)]
    run_readout(rs3, b, q, idx, count, group, sel, None, 64, 0.0, None, outs[0], 1)
    torch.cuda.synchronize()
    assert int(b.st) == 0
    rs3.rs3_set_wait_limit_ns(0)
    try:
        run_readout(rs3, b, q, idx, count, group, sel, None, 64, 0.0, None, outs[1], 1)
        torch.cuda.synchronize()
    finally:
        rs3.rs3_set_wait_limit_ns(10 ** 9)
    assert int(b.st) == rs3.RS3_ETIMEOUT
    b.st.zero_()
    run_readout(rs3, b, q, idx, count, group, sel, None, 64, 0.0, None, outs[1], 1)
    assert int(b.st) == 0 and torch.equal(outs[0], outs[1])


@pytest.mark.parametrize("dtype,H,d", [("bf16", 2, 64), ("bf16", 1, 256), ("f32", 1, 64)])
@pytest.mark.parametrize("same_blocks", [False, True])
def test_sparse_readout_over_all_blocks_is_the_memory_readout(rs3, dtype, H, d, same_blocks):
    """Many queries, every block listed: what rs3_memory_readout gives, within both calls' roundings."""
    b = Built(rs3, U=2, H=H, d=d, dtype=dtype, m=20, n=20, window=-1, ring_frames=6, commits=6, n_ptr=3, seed=5)
    k_max = 400
    q, idx, count, group = queries(b, 1, k_max, [400, 131])
    nb = b.bank.blocks(64)
    if same_blocks:
        sel = torch.arange(nb, dtype=torch.int32, device="cuda").expand(2, H, k_max, nb).contiguous()
    else:
        sel = torch.rand((2, H, k_max, nb), generator=gen(1), device="cuda").argsort(-1).to(torch.int32)
    outs = [torch.zeros((2, b.mn, b.D), dtype=DT[dtype], device="cuda") for _ in range(2)]
    run_readout(rs3, b, q, idx, count, group, sel, None, 64, 0.0, None, outs[0], 1)
    ws = torch.empty(rs3.rs3_readout_workspace_bytes(2, H, d, k_max, dtype), dtype=torch.uint8, device="cuda")
    b.bank.k_store.nan_to_num_(0)
    b.bank.v_store.nan_to_num_(0)
    rs3.rs3_memory_readout(q, dtype, 1, b.mn, H, d, group, idx, count, k_max, b.bank, None, None, outs[1], 0.0, ws, b.st)
    assert int(b.st) == 0
    # |A| <= sum p |v| <= max |v|: two roundings of the weights and two of the result (bf16), fp32 sums of scores
    vmax = float(b.bank.v_store.float().abs().max())
    tol = vmax * (4 * 2.0 ** -8 if dtype == "bf16" else 2.0 ** -14)
    assert float((outs[0].float() - outs[1].float()).abs().max()) <= tol


def test_one_block_chosen_by_everybody_and_scores_far_apart(rs3):
    """Skewed lists, and scores so far apart that all but one weight vanish."""
    b = Built(rs3, U=1, H=1, d=64, dtype="bf16", m=20, n=20, window=-1, ring_frames=8, commits=8, n_ptr=0, density=0.9, seed=6, scale=6.0)
    q, idx, count, group = queries(b, 1, 300, [300], scale=6.0)
    sel = torch.full((1, 1, 300, 3), -1, dtype=torch.int32, device="cuda")
    sel[..., 0] = 2
    sel[:, :, ::7, 1] = 11
    out = torch.zeros((1, b.mn, 64), dtype=torch.bfloat16, device="cuda")
    want, tol = readout_ref(b, q, idx, [300], group, sel, None, 64, 1.0, None, torch.zeros_like(out))
    run_readout(rs3, b, q, idx, count, group, sel, None, 64, 1.0, None, out, 1)
    err = (out.double() - want).abs()
    assert int(b.st) == 0 and (err <= tol).all(), float((err - tol).max())


@pytest.mark.parametrize("block,dtype,H,d,n,n_top", [(32, "bf16", 2, 64, 300, 9), (32, "bf16", 1, 128, 1000, 40), (64, "f32", 1, 64, 20, 5), (64, "f32", 2, 64, 300, 9)])
def test_sparse_readout_over_many_blocks(rs3, block, dtype, H, d, n, n_top):
    """A bank of thousands of blocks, all of its rows live; blocks chosen by one query, by many, twice by one."""
    rows, mn = (600_000 if block == 64 else 300_000), 1024
    bank = rs3.Bank(1, H, d, dtype, mn, 0, -1, rows, 4, 0)
    g, st = gen(41), status()
    for x in (bank.k_store, bank.v_store):
        x.normal_(generator=g)
    rs3.rs3_bank_commit(bank, bank.k_store[:, :mn].clone(), bank.v_store[:, :mn].clone(), None, 0, st)
    bank.counters[0, 1] = rows                             # as if the ring had been filled
    nb = bank.blocks(block)
    assert nb > 8192
    q = torch.randn((1, mn, H * d), generator=g, device="cuda").to(DT[dtype])
    idx = torch.randperm(mn, generator=g, device="cuda")[:n].to(torch.int32).view(1, n).contiguous()
    sel = torch.randint(0, rows // block, (1, H, n, n_top), generator=g, device="cuda").to(torch.int32)
    sel[..., 0] = 8192                                     # everybody's
    sel[:, :, ::5, 2] = sel[:, :, ::5, 3]
    out = torch.zeros((1, mn, H * d), dtype=DT[dtype], device="cuda")
    ws = torch.empty(rs3.rs3_sparse_readout_workspace_bytes(1, H, d, n, n_top, nb, dtype), dtype=torch.uint8, device="cuda")
    one, zero = torch.tensor([n], dtype=torch.int32, device="cuda"), torch.zeros(1, dtype=torch.int32, device="cuda")
    rs3.rs3_sparse_readout(q, dtype, 1, mn, H, d, zero, idx, one, n, bank, block, sel, n_top, None, None, out, 0.0, ws, st)
    assert int(st) == 0
    want, tol = torch.zeros_like(out, dtype=torch.float64), torch.zeros_like(out, dtype=torch.float64)
    bf, half = dtype == "bf16", HALF[dtype]
    for h in range(H):
        col = slice(h * d, (h + 1) * d)
        for j0 in range(0, n, 50):
            cells = idx[0, j0:j0 + 50].long()
            r = (sel[0, h, j0:j0 + 50].long()[..., None] * block + torch.arange(block, device="cuda")).flatten(1)
            k, v, x = bank.k_store[0, :, col][r].double(), bank.v_store[0, :, col][r].double(), q[0, cells, col].double()
            p = torch.softmax(torch.einsum("nrd,nd->nr", k, x) * d ** -0.5, 1)
            A, size = torch.einsum("nr,nrd->nd", p, v), torch.einsum("nr,nrd->nd", p, v.abs())
            s_abs = (torch.einsum("nrd,nd->nr", k.abs(), x.abs()) * d ** -0.5).max(1).values[:, None]
            want[0, cells, col] = A                        # (the bounds of readout_ref)
            tol[0, cells, col] = half * A.abs() + size * (torch.expm1(2 * s_abs * 2.0 ** -24 * 300) + 300 * 2.0 ** -24 + (half if bf else 0.0)) * 1.01
    err = (out.double() - want).abs()
    assert (err <= tol).all(), float((err - tol).max())


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_sparse_readout_by_block_latches_what_the_device_finds(rs3, dtype):
    """As below, for a call large enough to go by block; a bad entry leaves the others' results as they are."""
    U, H, n, n_top = 3, 2, 150, 14
    b = Built(rs3, U=U, H=H, d=64, dtype=dtype, m=13, n=13, window=-1, ring_frames=4, commits=4, n_ptr=0, seed=8)
    nb = b.bank.blocks(32)
    q, idx, count, group = queries(b, 1, n, [n, n, n])
    group.zero_()
    sel0 = torch.randint(0, nb, (U, H, n, n_top), generator=gen(3), device="cuda").to(torch.int32)

    def read(idx=idx, count=count, group=group, sel=sel0):
        b.st.zero_()
        out = torch.zeros((U, b.mn, H * 64), dtype=DT[dtype], device="cuda")
        run_readout(rs3, b, q, idx, count, group, sel, None, 32, 0.0, None, out, 1)
        return int(b.st), out

    code, good = read()
    assert code == 0
    E = rs3.RS3_EINVAL
    for bad in (-1, n + 1, -(1 << 31), (1 << 31) - 1):
        c = count.clone()
        c[1] = bad
        code, out = read(count=c)
        assert code == E and not out[1].any() and torch.equal(out[0], good[0]) and torch.equal(out[2], good[2])
    for bad in (-1, 1):
        gr = group.clone()
        gr[2] = bad
        code, out = read(group=gr)
        assert code == E and not out[2].any() and torch.equal(out[:2], good[:2])
    for bad in (-1, b.mn, -(1 << 31), (1 << 31) - 1):
        i = idx.clone()
        i[0, 3] = bad
        code, out = read(idx=i)
        left = torch.ones(b.mn, dtype=torch.bool, device="cuda")
        left[int(idx[0, 3])] = False
        assert code == E and torch.equal(out[1:], good[1:]) and torch.equal(out[0, left], good[0, left])
    for bad in (nb, 1 << 30, (1 << 31) - 1):
        sel = sel0.clone()
        sel[0, 0, 4, 1] = bad
        code, out = read(sel=sel)
        assert code == E and torch.equal(out[1:], good[1:])
        sel[0, 0, 4, 1] = -1
        code, same = read(sel=sel)
        assert code == 0 and torch.equal(out, same)


def test_digest_and_drop_leave_out_units_whose_frame_counters_are_unsound(rs3):
    b = Built(rs3, U=3, H=1, d=64, m=8, n=8, window=-1, ring_frames=4, commits=4, n_ptr=0, seed=9)
    dig, step, _ = make_digest(b, 32)
    one = torch.ones(3, dtype=torch.int32, device="cuda")
    for word, value in ((3, -1), (3, 1 << 20), (4, -1), (4, b.bank.max_frames)):
        was = b.bank.counters.clone()
        b.bank.counters[1, word] = value
        bad = b.bank.counters[1].clone()
        st, d, s = status(), torch.full_like(dig, 9), torch.full_like(step, 9.0)
        rs3.rs3_bank_digest(b.bank, 32, 1, d, s, st)
        assert int(st) == rs3.RS3_EINTERNAL and (d[1] == 9).all() and (s[1] == 9.0).all() and (s[0] != 9.0).any()
        st = status()
        rs3.rs3_bank_drop_frames(b.bank, one, None, st)
        assert int(st) == rs3.RS3_EINTERNAL and torch.equal(b.bank.counters[1], bad)
        b.bank.counters.copy_(was)


@pytest.mark.parametrize("n", [150, 10])
def test_reads_leave_out_units_whose_counters_are_unsound(rs3, n):
    b = Built(rs3, U=3, H=2, d=64, m=13, n=13, window=-1, ring_frames=4, commits=4, n_ptr=0, seed=8)
    nb, n_top = b.bank.blocks(32), 6
    dig, step, _ = make_digest(b, 32)
    rs3.rs3_bank_digest(b.bank, 32, -1, dig, step, b.st)
    q, idx, count, group = queries(b, 1, n, [n, n, n])
    group.zero_()
    w1 = torch.empty(rs3.rs3_block_select_workspace_bytes(3, 2, n, nb), dtype=torch.uint8, device="cuda")

    def read():
        b.st.zero_()
        st, sel = status(), torch.full((3, 2, n, n_top), 1, dtype=torch.int32, device="cuda")
        rs3.rs3_block_select(q, "bf16", 1, b.mn, 2, 64, group, idx, count, n, b.bank, 32, dig, step, None, n_top, sel, w1, st)
        out = torch.zeros((3, b.mn, 128), dtype=torch.bfloat16, device="cuda")
        run_readout(rs3, b, q, idx, count, group, sel, None, 32, 0.0, None, out, 1)
        return int(st), int(b.st), sel, out

    good = read()
    assert good[:2] == (0, 0)
    for word, value in ((0, -1), (1, 1 << 40), (2, -5), (6, 7)):
        was = int(b.bank.counters[1, word])
        b.bank.counters[1, word] = value
        bad = read()
        b.bank.counters[1, word] = was
        assert bad[:2] == (rs3.RS3_EINTERNAL, rs3.RS3_EINTERNAL) and not bad[3][1].any()
        for i in (0, 2):
            assert torch.equal(bad[2][i], good[2][i]) and torch.equal(bad[3][i], good[3][i])


def test_sparse_calls_latch_what_the_device_finds(rs3):
    b = Built(rs3, U=3, H=1, d=64, m=8, n=8, window=-1, ring_frames=4, commits=4, n_ptr=0, seed=8)
    nb = b.bank.blocks(32)
    dig, step, _ = make_digest(b, 32)
    rs3.rs3_bank_digest(b.bank, 32, -1, dig, step, b.st)
    q, idx, count, group = queries(b, 1, 10, [10, 10, 10])
    group.zero_()
    sel0 = torch.zeros((3, 1, 10, 2), dtype=torch.int32, device="cuda")
    ws = torch.empty(rs3.rs3_block_select_workspace_bytes(3, 1, 10, nb), dtype=torch.uint8, device="cuda")

    def both(idx=idx, count=count, group=group, sel=sel0):
        codes = []
        st, s = status(), torch.full_like(sel0, -5)
        rs3.rs3_block_select(q, "bf16", 1, b.mn, 1, 64, group, idx, count, 10, b.bank, 32, dig, step, None, 2, s, ws, st)
        codes.append(int(st))
        b.st.zero_()
        out = torch.zeros((3, b.mn, 64), dtype=torch.bfloat16, device="cuda")
        run_readout(rs3, b, q, idx, count, group, sel, None, 32, 0.0, None, out, 1)
        codes.append(int(b.st))
        return codes, s, out

    codes, s, good = both()
    assert codes == [0, 0] and (s >= 0).all()
    E = rs3.RS3_EINVAL
    for bad in (-1, 11):
        c = count.clone()
        c[1] = bad
        codes, s, out = both(count=c)
        assert codes == [E, E] and (s[1] == -5).all() and not out[1].any()
        assert torch.equal(out[0], good[0]) and torch.equal(out[2], good[2])
    for bad in (-1, 1):
        gr = group.clone()
        gr[2] = bad
        codes, s, out = both(group=gr)
        assert codes == [E, E] and (s[2] == -5).all() and not out[2].any() and torch.equal(out[0], good[0])
    for bad in (-1, b.mn):
        i = idx.clone()
        i[0, 3] = bad
        codes, s, out = both(idx=i)
        assert codes == [E, E] and torch.equal(out[1], good[1])
    for bad in (nb, 1 << 30):
        sel = sel0.clone()
        sel[0, 0, 4, 1] = bad
        codes, _, out = both(sel=sel)
        assert codes == [0, E] and torch.equal(out[1], good[1])
        sel[0, 0, 4, 1] = -1
        assert torch.equal(out, both(sel=sel)[2])


def test_reading_a_long_bank_frame_by_frame(rs3):
    """Norm, commit, digest, select and readout as a frame makes them, captured in a graph on a stream of its own, then a
    branch: the fork reads as its parent did."""
    from paper_2608_22526_gb300 import synth
    from paper_2608_22526_gb300.pipeline import Pipeline
    w = synth.Workload("t", 0, 12, 12, 2, 64, "bf16", 1, 2, 6, 0.2, 0.4, 1, -1, 0)
    pipe = Pipeline(w, ring_cap=20 * w.mn)
    pipe.use_blocks(32, 3)
    g = gen(3)
    mask = torch.zeros((2, w.mn), dtype=torch.uint8, device="cuda")
    mask[:, 30:90] = 1
    z = torch.randn((1, w.mn, w.D), generator=g, device="cuda").bfloat16()
    kv = [torch.randn((2, w.mn, w.D), generator=g, device="cuda").bfloat16() for _ in range(2)]
    table = rope_table(w.mn, 64)
    qn, kn = torch.zeros_like(z), torch.zeros_like(kv[0])
    x = torch.zeros((2, w.mn, w.D), dtype=torch.bfloat16, device="cuda")
    pipe.norm(z, qn, kv[0], kn, rope=table, k_keep=mask)
    pipe.commit(kn, kv[1], mask, 1)
    pipe.digest(-1)

    def frame():
        pipe.norm(z, qn, kv[0], kn, rope=table, k_keep=mask)
        pipe.select(z, mask)
        pipe.select_blocks(qn)
        pipe.readout_blocks(qn, None, x)
        pipe.commit(kn, kv[1], mask, 0)
        pipe.digest(1)

    frame()
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        frame()
    for _ in range(3):
        graph.replay()
    torch.cuda.synchronize()
    assert pipe.status_code() == 0
    assert rs3.rs3_bank_read_meta(pipe.bank)[0][0, 3] == 4
    before = x.clone()
    # the same frame again, read from a fork of unit 0
    pipe.select_blocks(qn)
    pipe.readout_blocks(qn, None, x)
    fork = pipe.fork(torch.tensor([0, 0], dtype=torch.int32, device="cuda"))
    y = torch.zeros_like(x)
    fork.digest(-1)
    fork.idx.copy_(pipe.idx[:1].expand_as(pipe.idx))
    fork.count.copy_(pipe.count[:1].expand_as(pipe.count))
    fork.select_blocks(qn)
    fork.readout_blocks(qn, None, y)
    assert pipe.status_code() == 0 and fork.status_code() == 0
    assert torch.equal(y[0], x[0]) and torch.equal(y[1], x[0]) and before.shape == x.shape


def small_pipeline(stream=None):
    """Two units of a few frames, ready to be read by blocks; its queries."""
    from paper_2608_22526_gb300 import synth
    from paper_2608_22526_gb300.pipeline import Pipeline
    w = synth.Workload("t", 0, 12, 12, 2, 64, "bf16", 1, 2, 6, 0.2, 0.4, 1, -1, 0)
    pipe = Pipeline(w, ring_cap=20 * w.mn, stream=stream)
    g = gen(3)
    mask = torch.zeros((2, w.mn), dtype=torch.uint8, device="cuda")
    mask[:, 30:90] = 1
    z = torch.randn((1, w.mn, w.D), generator=g, device="cuda").bfloat16()
    k, v = (torch.randn((2, w.mn, w.D), generator=g, device="cuda").bfloat16() for _ in range(2))
    torch.cuda.synchronize()
    for _ in range(3):
        pipe.commit(k, v, mask, 0)
    return pipe, z, mask


def test_pipeline_buffers_belong_to_its_stream(rs3):
    """The current stream is busy while a pipeline on another makes its buffers, digests and forks."""
    want, _, _ = small_pipeline()
    want.use_blocks(32, 3)
    want.digest(-1)
    side = torch.cuda.Stream()
    pipe, _, _ = small_pipeline(side)
    parent = torch.tensor([1, 0], dtype=torch.int32, device="cuda")
    torch.cuda.synchronize()
    torch.cuda._sleep(100_000_000)                         # some 50 ms on the current stream
    pipe.use_blocks(32, 3)
    pipe.digest(-1)
    fork = pipe.fork(parent)
    fork.digest(-1)
    pipe.fork(parent, into=fork)
    torch.cuda.synchronize()
    assert pipe.status_code() == 0 and fork.status_code() == 0
    assert want.block_digest.any() and torch.equal(pipe.block_digest, want.block_digest) and torch.equal(pipe.block_step, want.block_step)
    assert torch.equal(fork.block_digest, want.block_digest.flip(0)) and torch.equal(fork.block_step, want.block_step.flip(0))
    assert (rs3.rs3_bank_read_meta(fork.bank)[0][:, 7] == rs3.rs3_bank_read_meta(want.bank)[0][:, 7]).all()


def test_two_reads_at_once_on_two_streams(rs3):
    """One bank read by two calls at a time, each with workspaces of its own, on streams other than the current one."""
    b = Built(rs3, U=3, H=2, d=64, m=12, n=12, window=-1, ring_frames=12, commits=12, n_ptr=5, seed=4)
    nb, n, n_top = b.bank.blocks(32), 140, 7
    dig, step, _ = make_digest(b, 32)
    rs3.rs3_bank_digest(b.bank, 32, -1, dig, step, b.st)
    q, idx, count, group = queries(b, 2, n, [n, 77, n])
    x = [torch.randn((3, b.mn, b.D), generator=gen(9), device="cuda").bfloat16() for _ in range(2)]
    table = rope_table(b.mn, 64)

    def buffers():
        return dict(sel=torch.zeros((3, 2, n, n_top), dtype=torch.int32, device="cuda"), st=status(),
                    out=torch.zeros((3, b.mn, b.D), dtype=torch.bfloat16, device="cuda"),
                    w1=torch.empty(rs3.rs3_block_select_workspace_bytes(3, 2, n, nb), dtype=torch.uint8, device="cuda"),
                    w2=torch.empty(rs3.rs3_sparse_readout_workspace_bytes(3, 2, 64, n, n_top, nb, "bf16"), dtype=torch.uint8, device="cuda"))

    def read(o, res, rope, stream=None):
        rs3.rs3_block_select(q, "bf16", 2, b.mn, 2, 64, group, idx, count, n, b.bank, 32, dig, step, rope, n_top, o["sel"], o["w1"],
                             o["st"], stream)
        rs3.rs3_sparse_readout(q, "bf16", 2, b.mn, 2, 64, group, idx, count, n, b.bank, 32, o["sel"], n_top, rope, res, o["out"], 0.0,
                               o["w2"], o["st"], stream)

    want = [buffers(), buffers()]
    for o, res, rope in zip(want, x, (None, table)):
        read(o, res, rope)
    got, streams = [buffers(), buffers()], [torch.cuda.Stream(), torch.cuda.Stream()]
    torch.cuda.synchronize()
    for _ in range(20):
        for o, res, rope, s in zip(got, x, (None, table), streams):
            read(o, res, rope, s)
    torch.cuda.synchronize()
    for o, p in zip(got, want):
        assert int(o["st"]) == 0 and int(p["st"]) == 0
        assert torch.equal(o["sel"], p["sel"]) and torch.equal(o["out"], p["out"])


@pytest.mark.parametrize("n", [150, 6])
def test_captured_reads_share_workspaces(rs3, n):
    """Two captured graphs with one set of workspaces, replayed in turn with other queries, counts and rows (sizes
    that go by block, and by query)."""
    b = Built(rs3, U=2, H=2, d=64, m=13, n=13, window=-1, ring_frames=12, commits=6, n_ptr=0, seed=5)
    nb, n_top = b.bank.blocks(64), 9
    dig, step, _ = make_digest(b, 64)
    q, idx, count, group = queries(b, 1, n, [n, n - 3])
    group.zero_()
    w1 = torch.empty(rs3.rs3_block_select_workspace_bytes(2, 2, n, nb), dtype=torch.uint8, device="cuda")
    w2 = torch.empty(rs3.rs3_sparse_readout_workspace_bytes(2, 2, 64, n, n_top, nb, "bf16"), dtype=torch.uint8, device="cuda")
    sel = torch.zeros((2, 2, n, n_top), dtype=torch.int32, device="cuda")
    outs = [torch.zeros((2, b.mn, b.D), dtype=torch.bfloat16, device="cuda") for _ in range(2)]

    def read(out):
        rs3.rs3_bank_digest(b.bank, 64, -1, dig, step, b.st)
        rs3.rs3_block_select(q, "bf16", 1, b.mn, 2, 64, group, idx, count, n, b.bank, 64, dig, step, None, n_top, sel, w1, b.st)
        rs3.rs3_sparse_readout(q, "bf16", 1, b.mn, 2, 64, group, idx, count, n, b.bank, 64, sel, n_top, None, None, out, 0.0, w2, b.st)

    graphs = []
    for out in outs:
        read(out)
        torch.cuda.synchronize()
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph):
            read(out)
        graphs.append(graph)
    for i in range(4):
        q.copy_(torch.randn(q.shape, generator=gen(50 + i), device="cuda"))
        count.copy_(torch.tensor([n - i, i], dtype=torch.int32))
        b.commit(gen(60 + i), 0)
        want = torch.zeros_like(outs[0])
        graphs[i % 2].replay()
        first = sel.clone()
        read(want)
        live = torch.arange(n, device="cuda")[None, :] < count[:, None]
        assert int(b.st) == 0 and torch.equal(want, outs[i % 2])
        assert torch.equal(first.transpose(1, 2)[live], sel.transpose(1, 2)[live])


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("k_max,n_top", [(8, 5), (2, 1), (0, 3)])
def test_read_of_many_units(rs3, k_max, n_top, dtype):
    """More (unit, head) pairs than a CTA keeps counts of; few queries of each, none of some, or none at all."""
    U, H, d, mn = 400, 4, 64, 16
    bank = rs3.Bank(U, H, d, dtype, mn, 1, -1, 64, 4, 0)
    st, g = status(), gen(71)
    for f in range(4):
        k, v = (torch.randn((U, mn, H * d), generator=g, device="cuda").to(DT[dtype]) for _ in range(2))
        rs3.rs3_bank_commit(bank, k, v, None, int(f == 0), st)
    nb = bank.blocks(32)                                    # 80 rows: two blocks and a half
    dig, step = torch.zeros((U, H, nb, d), dtype=torch.int8, device="cuda"), torch.zeros((U, H, nb), device="cuda")
    rs3.rs3_bank_digest(bank, 32, -1, dig, step, st)
    q = torch.randn((1, mn, H * d), generator=g, device="cuda").to(DT[dtype])
    idx = torch.stack([torch.randperm(mn, generator=g, device="cuda")[:max(k_max, 1)] for _ in range(U)]).to(torch.int32)
    count = (torch.arange(U, device="cuda") % (k_max + 1)).to(torch.int32)
    group = torch.zeros(U, dtype=torch.int32, device="cuda")
    sel = torch.full((U, H, max(k_max, 1), n_top), -5, dtype=torch.int32, device="cuda")
    x = torch.randn((U, mn, H * d), generator=g, device="cuda").to(DT[dtype])
    out = torch.zeros_like(x)
    w1 = torch.empty(rs3.rs3_block_select_workspace_bytes(U, H, k_max, nb), dtype=torch.uint8, device="cuda")
    w2 = torch.empty(rs3.rs3_sparse_readout_workspace_bytes(U, H, d, k_max, n_top, nb, dtype), dtype=torch.uint8, device="cuda")
    rs3.rs3_block_select(q, dtype, 1, mn, H, d, group, idx, count, k_max, bank, 32, dig, step, None, n_top, sel, w1, st)
    rs3.rs3_sparse_readout(q, dtype, 1, mn, H, d, group, idx, count, k_max, bank, 32, sel, n_top, None, x, out, 0.0, w2, st)
    assert int(st) == 0
    kept = torch.zeros((U, mn), dtype=torch.bool, device="cuda")
    live = torch.arange(max(k_max, 1), device="cuda")[None, :] < count[:, None]
    kept.scatter_(1, idx.long(), live)
    assert torch.equal(out[~kept], x[~kept]) and (sel.transpose(1, 2)[~live] == -5).all()
    if not k_max:
        return
    # all 64 live rows in 64 bits: blocks 0 and 1 are live, so a query of one block reads it, of more reads both
    K, V = (t[:, :80].double().view(U, 80, H, d) for t in (bank.k_store, bank.v_store))
    Q = q[0].double().view(mn, H, d)[idx.long()]            # [U, k_max, H, d]
    s = torch.einsum("ujhd,urhd->ujhr", Q, K) * d ** -0.5
    rows = torch.arange(80, device="cuda") // 32
    sel_ = sel.transpose(1, 2)                              # [U, k_max, H, n_top]
    chosen = torch.stack([(sel_ == b).any(-1) for b in range(nb)], -1)
    length = torch.tensor(rs3.rs3_bank_read_meta(bank)[0][:, 7].tolist(), device="cuda")
    assert (length == 64).all()                             # (the rows fill the storage from its start)
    assert (chosen[live].sum(-1) == min(n_top, 2)).all() and not chosen[..., 2][live].any()
    s = s.masked_fill(~chosen[..., rows.clamp(max=nb - 1)] | (torch.arange(80, device="cuda") >= 64), -math.inf)
    A = torch.einsum("ujhr,urhd->ujhd", torch.softmax(s, -1).nan_to_num(0.0), V).flatten(2)
    size = torch.einsum("ujhr,urhd->ujhd", torch.softmax(s, -1).nan_to_num(0.0), V.abs()).flatten(2)
    want = x.double().gather(1, idx.long()[..., None].expand(-1, -1, H * d)) + A
    got = out.double().gather(1, idx.long()[..., None].expand(-1, -1, H * d))
    s_abs = (torch.einsum("ujhd,urhd->ujhr", Q.abs(), K.abs()) * d ** -0.5).amax(-1)[..., None].expand(-1, -1, -1, d).flatten(2)
    half = HALF[dtype]                                      # (the bounds of readout_ref)
    tol = half * want.abs() + size * (torch.expm1(2 * s_abs * 2.0 ** -24 * 300) + 300 * 2.0 ** -24 + (half if dtype == "bf16" else 0.0)) * 1.01 + 1e-30
    assert ((got - want).abs() <= tol)[live].all(), float(((got - want).abs() - tol)[live].max())


@pytest.mark.parametrize("masked", [False, True])
def test_copy_of_more_units_than_a_cta_counts(rs3, masked):
    U, H, d, mn = 1100, 1, 16, 8
    a, b = (rs3.Bank(U, H, d, "f32", mn, 1, -1, 40, 5, 0) for _ in range(2))
    st, g = status(), gen(81)
    for f in range(4):
        k, v = (torch.randn((U, mn, d), generator=g, device="cuda") for _ in range(2))
        mask = (torch.rand((U, mn), generator=g, device="cuda") < 0.6).to(torch.uint8)
        rs3.rs3_bank_commit(a, k, v, mask, int(f == 0), st)
    meta, frames = rs3.rs3_bank_read_meta(a)
    parent = torch.randint(-1, U, (U,), generator=g, device="cuda").to(torch.int32)
    keep = (torch.rand((U, 33), generator=g, device="cuda") < 0.5).to(torch.uint8) if masked else None
    ws = torch.full((rs3.rs3_bank_copy_workspace_bytes(U, 33),), 255, dtype=torch.uint8, device="cuda") if masked else None
    rs3.rs3_bank_copy(b, a, parent, keep, ws, st)
    assert int(st) == 0
    got, got_frames = rs3.rs3_bank_read_meta(b)
    for u, p in enumerate(parent.tolist()):
        if p < 0:
            assert got[u, 7] == 0
            continue
        cond, ring = int(meta[p, 2]), int(meta[p, 1] - meta[p, 0])
        rows = list(range(cond)) + [mn + int(meta[p, 0]) + i for i in range(ring)]
        on = [True] * len(rows) if keep is None else keep[u, :len(rows)].bool().tolist()
        from_cond = [r for r, k in zip(rows[:cond], on[:cond]) if k]
        from_ring = [r for r, k in zip(rows[cond:], on[cond:]) if k]
        assert (int(got[u, 2]), int(got[u, 1])) == (len(from_cond), len(from_ring)) and got[u, 3] == meta[p, 3]
        to = list(range(len(from_cond))) + [mn + i for i in range(len(from_ring))]
        if u % 50 == 0:
            assert torch.equal(b.k_store[u][to], a.k_store[p][from_cond + from_ring])
            assert torch.equal(b.v_store[u][to], a.v_store[p][from_cond + from_ring])


def test_fork_with_a_parent_that_is_no_unit(rs3):
    """The status word tells; the unit and its tracker stay as they are, and the context lives."""
    pipe, _, _ = small_pipeline()
    other, _, _ = small_pipeline()
    pipe.track.copy_(torch.arange(12).view(2, 6))
    other.track.fill_(-7)
    before = rs3.rs3_bank_read_meta(other.bank)[0]
    for bad in (2, (1 << 31) - 1, -2):
        other.status.zero_()
        pipe.fork(torch.tensor([bad, 0], dtype=torch.int32, device="cuda"), into=other)
        assert other.status_code() == rs3.RS3_EINVAL
        assert (other.track[0] == -7).all() and torch.equal(other.track[1], pipe.track[0])
        assert (rs3.rs3_bank_read_meta(other.bank)[0][0] == before[0]).all()


@pytest.mark.parametrize("busy", ["source", "target"])
def test_fork_into_a_pipeline_on_another_stream(rs3, busy):
    """What the target's stream still has to do comes before the copy, what it does next after it."""
    want, _, _ = small_pipeline()
    want.use_blocks(32, 3)
    want.digest(-1)
    streams = [torch.cuda.Stream(), torch.cuda.Stream()]
    (pipe, _, mask), (other, _, _) = (small_pipeline(s) for s in streams)
    pipe.track.copy_(torch.arange(12).view(2, 6))
    parent = torch.tensor([1, 0], dtype=torch.int32, device="cuda")
    k = torch.randn((2, other.w.mn, other.w.D), generator=gen(8), device="cuda").bfloat16()
    other.use_blocks(32, 3)
    torch.cuda.synchronize()
    with torch.cuda.stream(streams[busy == "target"]):
        torch.cuda._sleep(100_000_000)                     # some 50 ms
    with torch.cuda.stream(streams[1]):
        other.commit(k, k, mask, 0)                        # (a frame that the copy takes away)
        other.track.fill_(-7)
        pipe.fork(parent, into=other)
        other.digest(-1)
        track = other.track.clone()
    torch.cuda.synchronize()
    assert pipe.status_code() == 0 and other.status_code() == 0
    live = want.block_step != 0
    assert live.any() and torch.equal(other.block_step.flip(0)[live], want.block_step[live])
    assert torch.equal(other.block_digest.flip(0)[live], want.block_digest[live])
    assert torch.equal(track, pipe.track.flip(0))
    assert (rs3.rs3_bank_read_meta(other.bank)[0][:, 7] == rs3.rs3_bank_read_meta(want.bank)[0][:, 7]).all()


def test_fork_leaves_the_trackers_of_refused_units(rs3):
    """No room, a mask shorter than the parent, a source that does not stay as it is: the unit's tracker stays with its bank."""
    from paper_2608_22526_gb300.pipeline import Pipeline
    pipe, _, _ = small_pipeline()
    pipe.track.copy_(torch.arange(12).view(2, 6))
    both = torch.tensor([1, 0], dtype=torch.int32, device="cuda")
    small = Pipeline(pipe.w, ring_cap=100)                 # three frames of 60 rows do not fit
    small.track.fill_(-7)
    pipe.fork(both, into=small)
    assert small.status_code() == rs3.RS3_ECAPACITY and (small.track == -7).all()
    keep = torch.ones((2, 180), dtype=torch.uint8, device="cuda")
    keep[1] = 0
    small.status.zero_()
    pipe.fork(both, keep, into=small)                      # of unit 1 nothing is left, which fits
    assert small.status_code() == rs3.RS3_ECAPACITY
    assert (small.track[0] == -7).all() and torch.equal(small.track[1], pipe.track[0])
    small.status.zero_()
    small.track.fill_(-7)
    pipe.fork(both, torch.zeros((2, 179), dtype=torch.uint8, device="cuda"), into=small)
    assert small.status_code() == rs3.RS3_EINVAL and (small.track == -7).all()
    pipe.fork(both, into=pipe)                             # each other's source
    assert pipe.status_code() == rs3.RS3_EINVAL and torch.equal(pipe.track, torch.arange(12, dtype=torch.int32, device="cuda").view(2, 6))
    pipe.status.zero_()
    pipe.fork(torch.tensor([-1, 0], dtype=torch.int32, device="cuda"), into=pipe)
    assert pipe.status_code() == 0 and torch.equal(pipe.track[1], pipe.track[0])
    # the words count what became of the units, no more
    assert pipe.bank.copies.tolist() == [0, 1] and small.bank.copies.tolist() == [0, 1]


def test_fork_into_a_pipeline_with_another_number_of_units(rs3):
    import dataclasses
    from paper_2608_22526_gb300.pipeline import Pipeline
    pipe, _, _ = small_pipeline()
    pipe.track.copy_(torch.arange(12).view(2, 6))
    for parent in ([1], [1, -1, 0, 1, 1]):
        wide = Pipeline(dataclasses.replace(pipe.w, units_per_group=len(parent)), ring_cap=20 * pipe.w.mn)
        wide.track.fill_(-7)
        keep = (torch.rand((len(parent), 180), generator=gen(2), device="cuda") < 0.5).to(torch.uint8)
        pipe.fork(torch.tensor(parent, dtype=torch.int32, device="cuda"), keep, into=wide)
        assert wide.status_code() == 0
        length = rs3.rs3_bank_read_meta(wide.bank)[0][:, 7]
        for u, p in enumerate(parent):
            on = keep[u] != 0
            assert length[u] == (0 if p < 0 else int(on.sum()))
            assert torch.equal(wide.track[u], pipe.track[p]) if p >= 0 else (wide.track[u] == -7).all()
            if p >= 0:
                n, at = int(length[u]), pipe.w.n_cond * pipe.w.mn
                assert torch.equal(bits(wide.bank.k_store[u, at:at + n]), bits(pipe.bank.k_store[p, at:at + 180][on]))


# ---------------------------------------------------------------------------
# keys and scores that are no numbers
# ---------------------------------------------------------------------------
def eight_bits_of_anything(x):
    """eight_bits() of the whole definition: a NaN counts as 0, and no step is above 2^104."""
    x = np.nan_to_num(x.astype(np.float64), nan=0.0, posinf=np.inf, neginf=-np.inf)
    a = np.abs(x).max(-1)
    e = np.minimum(np.where(np.isinf(a), 110, np.frexp(np.where(np.isinf(a), 1.0, a))[1] - 1), 110)
    some = a >= 2.0 ** -100
    t = np.clip(np.rint(np.ldexp(x, (6 - e)[..., None])), -127, 127)
    return np.where(some[..., None], t, 0), np.where(some, np.ldexp(1.0, e - 6), 0.0)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("U,k_max,rows,n_top", [(1, 5, 640, 20), (1, 5, 640, 3), (160, 9, 640, 20), (160, 9, 640, 4), (1, 5, 40_000, 60),
                                                (1, 5, 40_000, 1024)])
def test_digest_and_selection_of_keys_that_are_no_numbers(rs3, dtype, U, k_max, rows, n_top):
    """Blocks with a NaN, an infinity, means past the largest number and means above 2^111: scores stay finite, so
    every live block can be chosen, and no entry of a list is left unwritten."""
    d, mn, nb = 64, 64, rows // 32
    bank = rs3.Bank(U, 1, d, dtype, mn, 0, -1, rows, 4, 0)
    st, g = status(), gen(rows + n_top)
    k = torch.randn((U, nb, 32, d), generator=g, device="cuda").to(DT[dtype])
    b = torch.arange(nb, device="cuda") % 6
    k[:, b == 0, 3, 1] = math.nan
    k[:, b == 1, 7, 2] = -math.inf
    k[:, b == 2] = -3e38
    k[:, b == 3, :, 5] = 1e35
    k[:, b == 4, :, 9] = -1e36
    bank.k_store.copy_(k.view(U, rows, d))
    bank.counters[:, 1] = rows                             # as if the ring had been filled
    dig, step = torch.full((U, 1, nb, d), 77, dtype=torch.int8, device="cuda"), torch.full((U, 1, nb), 0.5, device="cuda")
    rs3.rs3_bank_digest(bank, 32, -1, dig, step, st)
    assert int(st) == 0
    x = k.float().view(U, nb, 4, 8, d)
    p = x[:, :, 0]
    for i in range(1, 4):
        p = p + x[:, :, i]
    s = ((p[:, :, 0] + p[:, :, 4]) + (p[:, :, 2] + p[:, :, 6])) + ((p[:, :, 1] + p[:, :, 5]) + (p[:, :, 3] + p[:, :, 7]))
    t, e = eight_bits_of_anything((s / 32).cpu().numpy())
    assert np.array_equal(dig[:, 0].cpu().numpy(), t.astype(np.int8)) and np.array_equal(step[:, 0].cpu().numpy(), e.astype(np.float32))
    q = torch.randn((1, mn, d), generator=g, device="cuda").to(DT[dtype])
    q[0, 1, 3], q[0, 2, 4], q[0, 3] = math.nan, math.inf, math.nan
    idx = torch.arange(k_max, dtype=torch.int32, device="cuda").expand(U, k_max).contiguous()
    sel = torch.full((U, 1, k_max, n_top), -5, dtype=torch.int32, device="cuda")
    ws = torch.empty(rs3.rs3_block_select_workspace_bytes(U, 1, k_max, nb), dtype=torch.uint8, device="cuda")
    count, zero = torch.full((U,), k_max, dtype=torch.int32, device="cuda"), torch.zeros(U, dtype=torch.int32, device="cuda")
    rs3.rs3_block_select(q, dtype, 1, mn, 1, d, zero, idx, count, k_max, bank, 32, dig, step, None, n_top, sel, ws, st)
    assert int(st) == 0
    tq, _ = eight_bits_of_anything(q[0, :k_max].float().cpu().numpy())
    score = (torch.from_numpy(tq).cuda() @ torch.from_numpy(t).cuda().transpose(1, 2)) * torch.from_numpy(e).cuda()[:, None]
    best = score.argsort(dim=-1, descending=True, stable=True)[..., :n_top].sort(-1).values
    assert torch.equal(sel[:, 0].long(), best)


@pytest.mark.parametrize("dtype,H,d,n", [("bf16", 2, 64, 9), ("bf16", 1, 256, 5), ("f32", 2, 64, 9), ("bf16", 2, 64, 300), ("bf16", 1, 256, 300),
                                         ("f32", 2, 64, 300), ("f32", 2, 256, 300), ("bf16", 2, 32, 300)])
@pytest.mark.parametrize("block,n_top", [(32, 21), (64, 11)])
def test_sparse_readout_of_scores_that_are_no_numbers(rs3, dtype, H, d, n, block, n_top):
    """A NaN key, query or value that counts makes its results NaN, wherever its row lies; a score of minus infinity is a
    weight of nothing, and queries whose blocks hold no such row are as without them."""
    b = Built(rs3, U=1, H=H, d=d, dtype=dtype, m=20, n=20, window=-1, ring_frames=8, commits=8, n_ptr=3, seed=n_top)
    nb = b.bank.blocks(block)
    q, idx, count, group = queries(b, 1, n, [n])
    sel = torch.rand((1, H, n, nb), generator=gen(3), device="cuda").argsort(-1)[..., :n_top].to(torch.int32).contiguous()
    sel[0, :, 1] = 0                                       # two queries of one block each
    sel[0, :, 2] = 20
    sel[0, :, 1:3, 1:] = -1
    sel[0, :, 3, 0] = 27
    rows = torch.from_numpy(b.places(0)[0]).cuda()

    def read():
        out = torch.zeros((1, b.mn, b.D), dtype=DT[dtype], device="cuda")
        run_readout(rs3, b, q, idx, count, group, sel, None, block, 0.0, None, out, 1)
        assert int(b.st) == 0
        return out[0, idx[0].long()].view(n, H, d)

    def listed(blocks):                                    # [n, H]: the query's list holds one of them
        return torch.stack([(sel[0] == x).any(-1) for x in blocks]).any(0).T

    good = read()
    assert not good.isnan().any()
    whole = rows[rows // block == 20]
    one = rows[rows // block == 24][-1:]
    keys, values = b.bank.k_store.clone(), b.bank.v_store.clone()
    # every key of a block, and one key of another
    b.bank.k_store[0, whole] = math.nan
    b.bank.k_store[0, one, d // 2] = math.nan              # (the first head's)
    got, hit = read(), listed([20])
    hit[:, 0] |= listed([24])[:, 0]
    assert hit.any() and not hit.all() and got[hit].isnan().all() and torch.equal(bits(got[~hit]), bits(good[~hit]))
    # a value
    b.bank.k_store.copy_(keys)
    b.bank.v_store[0, one, 3] = math.nan
    got, hit = read(), listed([24])[:, 0]
    assert got[hit, 0, 3].isnan().all()
    got[:, 0, 3] = good[:, 0, 3]
    assert torch.equal(bits(got), bits(good))
    # a query
    b.bank.v_store.copy_(values)
    was = q.clone()
    q[0, idx[0, 3].long(), 1] = math.nan
    got = read()
    assert got[3, 0].isnan().all()
    got[3, 0] = good[3, 0]
    assert torch.equal(bits(got), bits(good))
    # scores of minus infinity: a block of them counts for nothing, and a query that reads no other row gets A = 0
    q.copy_(was)
    q[0, :, ::d] = q[0, :, ::d].abs() + 1
    good = read()
    b.bank.k_store[0, whole] = 0
    b.bank.k_store[0, whole, ::d] = -math.inf
    got = read()
    sel[sel == 20] = -1
    want = read()
    assert not got.isnan().any() and not got[2].any() and torch.equal(bits(got), bits(want))


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_norm_into_columns_of_the_same_rows(rs3, dtype):
    """Results in other columns of the rows that hold the operands, and in the rows between."""
    rows, H, d = 37, 2, 64
    W = H * d
    x = torch.randn((rows, 4 * W), generator=gen(4), device="cuda").to(DT[dtype])
    was = x.clone()
    col = [slice(i * W, (i + 1) * W) for i in range(4)]
    rs3.rs3_qk_norm_rope(x[:, col[0]], x[:, col[3]], x[:, col[1]], x[:, col[1]], dtype, rows, H, H, d, eps=1e-6)
    check_norm(x[:, col[3]], *norm_ref(was[:, col[0]].contiguous(), d, None, None, rows, 1e-6), dtype)
    check_norm(x[:, col[1]], *norm_ref(was[:, col[1]].contiguous(), d, None, None, rows, 1e-6), dtype)
    assert torch.equal(bits(x[:, col[0]]), bits(was[:, col[0]])) and torch.equal(bits(x[:, col[2]]), bits(was[:, col[2]]))
    y = torch.randn((2 * rows, W), generator=gen(5), device="cuda").to(DT[dtype])
    was = y.clone()
    rs3.rs3_qk_norm_rope(y[::2], y[1::2], y[::2], torch.empty_like(y[::2]), dtype, rows, H, H, d, eps=1e-6)
    check_norm(y[1::2], *norm_ref(was[::2].contiguous(), d, None, None, rows, 1e-6), dtype)
    assert torch.equal(bits(y[::2]), bits(was[::2]))
    with pytest.raises(RuntimeError):
        rs3.rs3_qk_norm_rope(y[:-1], y[1:], None, None, dtype, rows, H, H, d)


# ---------------------------------------------------------------------------
# sizes that take several CTAs, turns or operand blocks
# ---------------------------------------------------------------------------
@pytest.mark.parametrize("stride", [20_064, 20_011])
@pytest.mark.parametrize("keep", [0.0, 0.5, 0.98, 1.0])
def test_copy_with_a_mask_of_thousands_of_rows(rs3, stride, keep):
    """Parents of 4096, 4097 and some 20 000 rows: their kept rows are counted by several CTAs, and frames begin and end in
    either part; aligned and unaligned mask rows."""
    U, d, mn, frames, n_ptr = 3, 8, 1500, 14, 5
    src = rs3.Bank(U, 1, d, "bf16", mn, 1, -1, 20_000, 20, n_ptr)
    g, st = gen(stride), status()
    for f in range(1 + frames):
        k, v = (torch.randn((U, mn, d), generator=g, device="cuda").bfloat16() for _ in range(2))
        n = [[101, 285], [102, 285], [100, 1400]]
        n = torch.tensor([x[min(f, 1)] for x in n], device="cuda")
        mask = torch.rand((U, mn), generator=g, device="cuda").argsort(-1).argsort(-1) < n[:, None]
        rs3.rs3_bank_commit(src, k, v, mask.to(torch.uint8), int(f == 0), st)
    rs3.rs3_bank_set_pointers(src, *(torch.randn((U, n_ptr, d), generator=g, device="cuda").bfloat16() for _ in range(2)), st)
    meta, table = rs3.rs3_bank_read_meta(src)
    assert meta[:, 7].tolist() == [4096, 4097, 19_705]
    parent = [2, 0, 2, 1]
    dst = rs3.Bank(4, 1, d, "bf16", mn, 1, -1, 19_700, 14, n_ptr)
    mask = (torch.rand((4, stride), generator=g, device="cuda") < keep).to(torch.uint8)
    ws = torch.full((rs3.rs3_bank_copy_workspace_bytes(4, stride),), 255, dtype=torch.uint8, device="cuda")
    for _ in range(2):                                     # the second call finds the first's workspace and counters
        rs3.rs3_bank_copy(dst, src, torch.tensor(parent, dtype=torch.int32, device="cuda"), mask, ws, st)
    assert int(st) == 0 and dst.copies.tolist() == [2] * 4
    got, got_table = rs3.rs3_bank_read_meta(dst)
    for u, p in enumerate(parent):
        cond, ring = int(meta[p, 2]), int(meta[p, 1])      # (heads at 0: nothing was evicted)
        on = mask[u, :cond + ring + n_ptr] != 0
        regions = [(torch.arange(cond), 0), (torch.arange(ring) + mn, mn), (torch.arange(n_ptr) + mn + 20_000, mn + 19_700)]
        at = 0
        for i, (rows, first) in enumerate(regions):
            rows = rows.cuda()[on[at:at + rows.numel()]]
            at += regions[i][0].numel()
            for a, b in ((src.k_store, dst.k_store), (src.v_store, dst.v_store)):
                assert torch.equal(bits(b[u, first:first + rows.numel()]), bits(a[p][rows]))
        upto = torch.cat([torch.zeros(1, dtype=torch.int64, device="cuda"), on.long().cumsum(0)]).cpu().numpy()
        want = upto[cond + table[p, :frames, 0]] - upto[cond], upto[cond + table[p, :frames].sum(-1)] - upto[cond + table[p, :frames, 0]]
        assert np.array_equal(got_table[u, :frames, 0], want[0]) and np.array_equal(got_table[u, :frames, 1], want[1])
        assert got[u].tolist() == [0, int(upto[cond + ring] - upto[cond]), int(upto[cond]), frames, 0, 1, int(upto[-1] - upto[cond + ring]),
                                   int(upto[-1])]


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("n_top", [1, 4])
@pytest.mark.parametrize("spread,rope", [(127, True), (1, False), (0, False)])
def test_select_for_many_queries_of_wide_heads(rs3, dtype, n_top, spread, rope):
    """Heads of 128 with few choices, which a tile of queries takes too: random digests, ties, nothing but ties."""
    U, H, d, mn, k_max, rows = 80, 1, 128, 256, 150, 5000
    bank = rs3.Bank(U, H, d, dtype, mn, 0, -1, rows, 4, 0)
    bank.counters[:, 1] = torch.arange(U, device="cuda") * (rows // U)         # as if the rings had been filled so far
    st, g, nb = status(), gen(spread + n_top), bank.blocks(32)
    dig = (torch.randint(-max(1, spread), max(1, spread) + 1, (U, H, nb, d), generator=g, device="cuda") * (spread > 0)).to(torch.int8)
    step = torch.randint(1, 3, (U, H, nb), generator=g, device="cuda").float() / 64
    q = torch.randn((1, mn, d), generator=g, device="cuda").to(DT[dtype])
    idx = torch.stack([torch.randperm(mn, generator=g, device="cuda")[:k_max] for _ in range(U)]).to(torch.int32)
    count = torch.tensor([k_max - u % 7 for u in range(U)], dtype=torch.int32, device="cuda")
    zero = torch.zeros(U, dtype=torch.int32, device="cuda")
    table = rope_table(mn, d) if rope else None
    sel = torch.full((U, H, k_max, n_top), -5, dtype=torch.int32, device="cuda")
    ws = torch.empty(rs3.rs3_block_select_workspace_bytes(U, H, k_max, nb), dtype=torch.uint8, device="cuda")
    rs3.rs3_block_select(q, dtype, 1, mn, H, d, zero, idx, count, k_max, bank, 32, dig, step, table, n_top, sel, ws, st)
    assert int(st) == 0
    x = q[0].float().cpu().numpy()
    if table is not None:
        t, p = table.cpu().numpy(), x.reshape(mn, d // 2, 2)
        c, s = t[..., 0], t[..., 1]
        x = np.stack([p[..., 0] * c - p[..., 1] * s, p[..., 0] * s + p[..., 1] * c], -1).astype(np.float32).reshape(mn, d)
    tq = torch.from_numpy(eight_bits(x)[0]).cuda()
    for u in range(U):
        n, live = int(count[u]), -(-int(bank.counters[u, 1]) // 32)
        m = min(n_top, live)
        score = (tq[idx[u, :n].long()] @ dig[u, 0, :live].double().T) * step[u, 0, :live].double()
        best = score.argsort(dim=-1, descending=True, stable=True)[:, :m].sort(-1).values
        assert torch.equal(sel[u, 0, :n, :m].long(), best), u
        assert (sel[u, 0, :n, m:] == -1).all() and (sel[u, 0, n:] == -5).all()


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_digest_of_more_blocks_than_a_warp_s_first_turn(rs3, dtype):
    """A warp looks 32 blocks ahead; units of over 384 blocks give it a second turn, and a third."""
    U, d, rows = 160, 16, 26_000
    bank = rs3.Bank(U, 1, d, dtype, 64, 0, -1, rows, 4, 0)
    st, nb = status(), bank.blocks(32)
    bank.k_store.normal_(generator=gen(5))
    bank.counters[:, 0] = 1000                             # as if the rings had been filled: 1000 dead rows, then live ones
    bank.counters[:, 1] = rows - 7
    dig, step = torch.full((U, 1, nb, d), 77, dtype=torch.int8, device="cuda"), torch.full((U, 1, nb), 0.5, device="cuda")
    rs3.rs3_bank_digest(bank, 32, -1, dig, step, st)
    assert int(st) == 0
    live = torch.zeros(nb * 32, dtype=torch.bool, device="cuda")
    live[1000:rows - 7] = True
    n = live.view(nb, 32).sum(-1).clamp(min=1).float()
    for u in (0, 77, U - 1):
        x = torch.zeros((nb * 32, d), device="cuda")
        x[live] = bank.k_store[u].float()[live[:rows]]
        x = x.view(nb, 4, 8, d)
        p = x[:, 0]
        for i in range(1, 4):
            p = p + x[:, i]
        s = ((p[:, 0] + p[:, 4]) + (p[:, 2] + p[:, 6])) + ((p[:, 1] + p[:, 5]) + (p[:, 3] + p[:, 7]))
        t, e = eight_bits((s / n[:, None]).cpu().numpy())
        assert np.array_equal(dig[u, 0].cpu().numpy(), t.astype(np.int8)) and np.array_equal(step[u, 0].cpu().numpy(), e.astype(np.float32))


def test_captured_frames_read_what_frames_one_by_one_read(rs3):
    """Frames replayed from a graph leave what the same frames leave when each call is made: results, choices, digests, rows."""
    pipes, outs = [], []
    for _ in range(2):
        pipe, z, mask = small_pipeline()
        pipe.use_blocks(32, 3)
        pipe.digest(-1)
        pipes.append(pipe)
        outs.append(torch.zeros((2, pipe.w.mn, pipe.w.D), dtype=torch.bfloat16, device="cuda"))
    k, v = (torch.randn((2, z.shape[1], z.shape[2]), generator=gen(6), device="cuda").bfloat16() for _ in range(2))

    def frame(pipe, out):
        pipe.select(z, mask)
        pipe.select_blocks(z)
        pipe.readout_blocks(z, None, out)
        pipe.commit(k, v, mask, 0)
        pipe.digest(1)

    for p, o in zip(pipes, outs):
        frame(p, o)
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        frame(pipes[0], outs[0])
    for _ in range(2):
        graph.replay()
        frame(pipes[1], outs[1])
        torch.cuda.synchronize()
        a, b = pipes
        assert a.status_code() == 0 and b.status_code() == 0 and outs[1].any()
        for x, y in ((outs[0], outs[1]), (a.bank.k_store, b.bank.k_store), (a.bank.v_store, b.bank.v_store)):
            assert torch.equal(bits(x), bits(y))
        for x, y in ((a.block_digest, b.block_digest), (a.block_step, b.block_step), (a.block_sel, b.block_sel), (a.bank.counters, b.bank.counters)):
            assert torch.equal(x, y)


@pytest.mark.parametrize("dtype,H,d", [("bf16", 4, 64), ("bf16", 1, 256), ("f32", 2, 64)])
def test_sparse_readout_repeats_itself(rs3, dtype, H, d):
    """By block: entries of a block's list come in any order, the result's bits do not depend on it."""
    b = Built(rs3, U=2, H=H, d=d, dtype=dtype, m=24, n=24, window=-1, ring_frames=8, commits=8, n_ptr=3, seed=2)
    n, nb = 500, b.bank.blocks(64)
    q, idx, count, group = queries(b, 1, n, [n, n - 100])
    sel = torch.rand((2, H, n, nb), generator=gen(3), device="cuda").argsort(-1)[..., :12].to(torch.int32).contiguous()
    table = rope_table(b.mn, d)
    first = None
    for _ in range(5):
        out = torch.zeros((2, b.mn, b.D), dtype=DT[dtype], device="cuda")
        run_readout(rs3, b, q, idx, count, group, sel, table, 64, 0.0, None, out, 1)
        assert int(b.st) == 0
        first = out if first is None else first
        assert torch.equal(bits(out), bits(first))


@pytest.mark.parametrize("dtype,H,d,U,k_max,n_top,rows,spread,rope", [
    ("bf16", 2, 64, 160, 40, 17, 20_000, 127, True), ("f32", 1, 32, 160, 250, 24, 9_000, 2, False), ("bf16", 4, 16, 160, 21, 25, 3_000, 2, True),
    ("bf16", 4, 64, 160, 33, 32, 9_000, 127, False), ("f32", 4, 64, 160, 9, 32, 900, 0, False)])
def test_select_for_more_choices_of_many_queries(rs3, dtype, H, d, U, k_max, n_top, rows, spread, rope):
    """Several tiles of queries per SM, where more than 16 choices go by tiles too."""
    test_select_for_many_queries(rs3, dtype, H, d, U, k_max, n_top, rows, spread, rope)


@pytest.mark.parametrize("dtype,H,d", [("bf16", 2, 64), ("f32", 2, 64), ("f32", 2, 256), ("bf16", 1, 256)])
@pytest.mark.parametrize("block", [32, 64, 128])
def test_sparse_readout_stays_inside_the_workspace_of_its_block(rs3, dtype, H, d, block):
    """By block with the smaller workspace: the same bits, and nothing is written behind it."""
    b = Built(rs3, U=2, H=H, d=d, dtype=dtype, m=24, n=24, window=-1, ring_frames=8, commits=8, n_ptr=3, seed=2)
    n, n_top, nb = 500, 14, b.bank.blocks(block)
    q, idx, count, group = queries(b, 1, n, [n, n - 100])
    sel = torch.rand((2, H, n, nb), generator=gen(3), device="cuda").argsort(-1)[..., :n_top].to(torch.int32).contiguous()
    table = rope_table(b.mn, d)
    want, out = (torch.zeros((2, b.mn, b.D), dtype=DT[dtype], device="cuda") for _ in range(2))
    run_readout(rs3, b, q, idx, count, group, sel, table, block, 0.0, None, want, 1)
    size = rs3.rs3_sparse_readout_workspace_bytes(2, H, d, n, n_top, nb, dtype, block)
    assert size > 1 << 20
    room = torch.full((size + 4096,), 0x5a, dtype=torch.uint8, device="cuda")
    rs3.rs3_sparse_readout(q, dtype, 1, b.mn, H, d, group, idx, count, n, b.bank, block, sel, n_top, table, None, out, 0.0, room[:size], b.st)
    assert int(b.st) == 0 and torch.equal(bits(out), bits(want)) and (room[size:] == 0x5a).all()
