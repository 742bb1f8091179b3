"""Readouts over a shared prefix, and with capped and biased scores, against plain implementations in 64 bits."""
import math
import types

import numpy as np
import pytest
import torch

from test_gpu_long_bank import DT, HALF, Built, bits, gen, rope_table, status, turned

pytestmark = pytest.mark.gpu

STEP = 2.0 ** -24


@pytest.fixture(scope="module")
def rs3():
    from paper_2608_22526_gb300 import rs3
    return rs3


def built(rs3, **kw):
    """A bank whose dead rows hold finite values (large ones: nothing may come of them)."""
    b = Built(rs3, **kw)
    for t in (b.bank.k_store, b.bank.v_store):
        t.copy_(torch.where(t.isnan(), torch.full_like(t, 1000.0), t))
    return b


def frames_of(b, u):
    """(storage rows of unit u in logical order, the frame of each: its age, F or F + 1)."""
    rows, lens, (cond, ring, ptr) = b.places(u)
    F = b.bank.max_frames
    slot = [F] * cond + [len(lens) - 1 - i for i, n in enumerate(lens) for _ in range(n)] + [F + 1] * ptr
    return torch.from_numpy(rows).cuda(), torch.tensor(slot, dtype=torch.int64, device="cuda")


def keep_sets(U, mn, k_max, counts, seed=17):
    g = gen(seed)
    idx = torch.stack([torch.randperm(mn, generator=g, device="cuda")[:k_max].sort().values for _ in range(U)]).to(torch.int32).contiguous()
    return idx, torch.tensor(counts, dtype=torch.int32, device="cuda")


def reference(dtype, H, d, q, idx, counts, group, table, scale, res, shape, rows_of, cap=0.0, bias=None):
    """(out, tolerance) in 64 bits.  rows_of(u): keys, values [N, D] and the frame of each; bias(u, h): [frames] or None."""
    bf, half = dtype == "bf16", HALF[dtype]
    out = torch.zeros(shape, dtype=torch.float64, device="cuda") if res is None else res.double().clone()
    tol = torch.zeros_like(out)
    qd = q.double()
    if table is not None:
        qd = turned(qd, d, table)
    for u, n in enumerate(counts):
        if n == 0:
            continue
        k, v, slot = rows_of(u)
        k, v = k.double(), v.double()
        cells = idx[u, :n].long()
        for h in range(H):
            col = slice(h * d, (h + 1) * d)
            r = 0.0 if res is None else res[u, cells, col].double()
            if k.shape[0] == 0:
                out[u, cells, col] = r
                tol[u, cells, col] = 0.0
                continue
            qq = qd[int(group[u]), cells, col]
            x = qq @ k[:, col].T * scale
            terms = qq.abs() @ k[:, col].abs().T * scale
            # a score: fp32 sums of at most 256 products and its scaling, under 300 half-steps of the terms; a rotated query's
            # rounding to bf16
            e = terms * (300 * STEP + (half if bf and table is not None else 0.0))
            if cap > 0:
                # |d tanh| <= 1; the change's own error: a power, a sum, a quotient and a product or two, under 32 half-steps of cap
                x = cap * torch.tanh(x / cap)
                e = e + 32 * STEP * cap
            if bias is not None:
                b = bias(u, h).double()[slot]
                x = x + b
                e = e + 8 * STEP * (x.abs() + b.abs().clamp(max=1e30)).nan_to_num(0.0, 0.0, 0.0)
            top = x.amax(1, keepdim=True)
            # (a weight is 2^(x - reference): the argument's own rounding, and the reference's, are of their sizes)
            on = x > -math.inf
            e = e + 16 * STEP * torch.where(on, x.abs(), 0.0).amax(1, keepdim=True)
            w = torch.where(on, torch.exp(x - torch.where(top > -math.inf, top, 0.0)), 0.0)
            total = w.sum(1, keepdim=True)
            p = w / torch.where(total > 0, total, 1.0)
            A, size = p @ v[:, col], p @ v[:, col].abs()
            # a weight's error beside the row's mean error is at most twice the largest one's; far keys weigh by p
            es = torch.where(on, e, 0.0)
            share = (p * torch.expm1(2 * es)) @ v[:, col].abs() + (p * torch.expm1(2 * es)).sum(1, keepdim=True) * size
            out[u, cells, col] = r + A
            # weights and values: under 300 half-steps, in bf16 a rounding of each weight; then the result's own
            tol[u, cells, col] = half * (r + A).abs() + (share + size * (300 * STEP + (half if bf else 0.0))) * 1.01 + 1e-30
    return out, tol


# ---------------------------------------------------------------------------
# a shared prefix
# ---------------------------------------------------------------------------
SHAPES = [("bf16", 1, 16), ("bf16", 2, 32), ("bf16", 3, 64), ("bf16", 2, 128), ("bf16", 1, 256), ("f32", 2, 16), ("f32", 1, 32),
          ("f32", 3, 64), ("f32", 1, 128), ("f32", 2, 256)]


def shared_rows(b, p, prefix_unit):
    def rows(u):
        at = torch.from_numpy(b.places(u)[0]).cuda()
        k, v = b.bank.k_store[u][at], b.bank.v_store[u][at]
        x = int(prefix_unit[u])
        if x >= 0:
            pt = torch.from_numpy(p.places(x)[0]).cuda()
            k, v = torch.cat([p.bank.k_store[x][pt], k]), torch.cat([p.bank.v_store[x][pt], v])
        return k, v, torch.zeros(k.shape[0], dtype=torch.int64, device="cuda")
    return rows


def run_shared(rs3, b, p, q, G, idx, count, group, prefix_unit, table, scale, res, out, ws=None, stream=None):
    k_max = idx.shape[1]
    if ws is None:
        ws = torch.full((rs3.rs3_shared_readout_workspace_bytes(b.bank, p.bank, k_max),), 255, dtype=torch.uint8, device="cuda")
    rs3.rs3_shared_readout(q, b.dtype, G, b.mn, b.H, b.d, group, idx, count, k_max, b.bank, p.bank, prefix_unit, table, res, out, scale, ws,
                           b.st, stream)
    return ws


def shared_case(rs3, b, p, counts, group, prefix, G, residual="none", rope=False, seed=5, k_max=None, scale=0.0):
    U, mn, D, dtype = b.U, b.mn, b.D, b.dtype
    g = gen(seed)
    q = (torch.randn((G, mn, D), generator=g, device="cuda") * 1.2).to(DT[dtype])
    k_max = max(1, max(counts)) if k_max is None else k_max
    idx, count = keep_sets(U, mn, k_max, counts, seed)
    group = torch.tensor(group, dtype=torch.int32, device="cuda")
    prefix_unit = torch.tensor(prefix, dtype=torch.int32, device="cuda")
    table = rope_table(mn, b.d) if rope else None
    x = torch.randn((U, mn, D), generator=g, device="cuda").to(DT[dtype])
    res = None if residual == "none" else x.clone()
    out = res if residual == "inplace" else torch.full_like(x, math.nan)
    want, tol = reference(dtype, b.H, b.d, q, idx, counts, group, table, scale or b.d ** -0.5, None if res is None else x, x.shape,
                          shared_rows(b, p, prefix_unit))
    run_shared(rs3, b, p, q, G, idx, count, group, prefix_unit, table, scale, res, out)
    assert int(b.st) == 0
    err = (out.double() - want).abs()
    assert (err <= tol).all(), (float((err - tol).max()), float(err.max()))
    return q, idx, count, group, prefix_unit, table, out


@pytest.mark.parametrize("dtype,H,d", SHAPES)
@pytest.mark.parametrize("counts", [[1, 0, 3, 2, 1], [40, 17, 33, 72, 5]])
@pytest.mark.parametrize("residual,rope", [("none", False), ("inplace", True), ("other", False)])
def test_shared_readout_matches_64_bits(rs3, dtype, H, d, counts, residual, rope):
    """Two groups, classes of several units and of one, units without a prefix, without rows of their own, an empty prefix."""
    b = built(rs3, U=5, H=H, d=d, dtype=dtype, m=8, n=9, window=4, commits=7, n_ptr=5, empty=(1,), seed=2)
    p = built(rs3, U=3, H=H, d=d, dtype=dtype, m=8, n=9, window=-1, ring_frames=9, commits=9, n_ptr=3, seed=3)
    rs3.rs3_bank_reset(b.bank, 1)
    rs3.rs3_bank_reset(p.bank, 2)
    shared_case(rs3, b, p, counts, [0, 0, 0, 1, 1], [1, 1, 0, 1, 2], 2, residual, rope)
    shared_case(rs3, b, p, counts, [0, 1, 0, 1, 1], [-1, -1, 2, 0, 0], 2, residual, rope, scale=0.11)


@pytest.mark.parametrize("dtype,H,d", [("bf16", 1, 64), ("bf16", 2, 128), ("bf16", 1, 256), ("f32", 1, 64), ("f32", 1, 256)])
def test_shared_readout_of_long_prefixes_and_many_queries(rs3, dtype, H, d):
    """Rows split over many pieces; keep-sets that overlap in part; classes of more tiles than any unit."""
    b = built(rs3, U=4, H=H, d=d, dtype=dtype, m=32, n=33, window=3, commits=4, n_ptr=0, seed=2)
    p = built(rs3, U=2, H=H, d=d, dtype=dtype, m=32, n=33, window=-1, ring_frames=24, commits=24, n_ptr=3, seed=3)
    shared_case(rs3, b, p, [300, 290, 131, 7], [0, 0, 0, 0], [1, 1, 1, 0], 1, "inplace")
    shared_case(rs3, b, p, [1056, 1056, 1, 129], [0, 0, 1, 1], [0, 0, 1, 1], 2, "none", rope=True)
    shared_case(rs3, b, p, [3, 2, 1, 1], [0, 0, 0, 0], [0, 0, 0, 0], 1, "other")


@pytest.mark.parametrize("d", [64, 128])
def test_shared_readout_by_pairs_of_query_tiles(rs3, d):
    """Enough work that the plan takes two query tiles per CTA, for the prefix at least."""
    H, frames = 512 // d, 3 if d == 64 else 10
    b = built(rs3, U=4, H=H, d=d, dtype="bf16", m=64, n=64, window=2, commits=2, n_ptr=0, seed=2, density=0.3)
    p = built(rs3, U=1, H=H, d=d, dtype="bf16", m=64, n=64, window=-1, ring_frames=frames, commits=frames, n_ptr=0, seed=3)
    shared_case(rs3, b, p, [2500, 1200, 900, 640], [0, 0, 0, 0], [0, 0, 0, 0], 1, "inplace")


def test_shared_readout_of_many_units(rs3):
    """Hundreds of units in classes that lie apart; the grid's last word of cells is a part."""
    U = 600
    b = built(rs3, U=U, H=1, d=16, dtype="f32", m=3, n=11, window=1, commits=1, n_ptr=0, n_cond=0, seed=2)
    p = built(rs3, U=7, H=1, d=16, dtype="f32", m=3, n=11, window=2, commits=2, n_ptr=0, seed=3)
    shared_case(rs3, b, p, [(5 * u) % 34 for u in range(U)], [u % 3 for u in range(U)], [(u * 7) % 8 - 1 for u in range(U)], 3, "none", k_max=33)


def test_shared_readout_of_a_bank_that_is_its_own_prefix(rs3):
    """Unit 0's rows as the prefix of the others, in one bank; twice the same cell."""
    b = built(rs3, U=3, H=2, d=64, dtype="bf16", m=8, n=9, window=4, commits=7, n_ptr=5, seed=2)
    q, idx, count, group, prefix_unit, table, out = shared_case(rs3, b, b, [9, 30, 20], [0, 0, 0], [-1, 0, 0], 1)
    idx[1, 7] = idx[1, 3]
    again = torch.full_like(out, math.nan)
    run_shared(rs3, b, b, q, 1, idx, count, group, prefix_unit, table, 0.0, None, again)
    same = torch.ones(b.mn, dtype=torch.bool, device="cuda")
    same[torch.from_numpy(np.setdiff1d(np.arange(b.mn), idx[1].cpu().numpy())).cuda()] = False
    assert torch.equal(bits(again[0]), bits(out[0])) and not again.isnan().any()


def test_shared_readout_of_copies_is_the_memory_readout_of_the_fork(rs3):
    """What a fork that copies its parent's rows reads, within the tolerance of both."""
    p = built(rs3, U=1, H=1, d=64, dtype="f32", m=8, n=9, window=-1, ring_frames=9, commits=6, n_ptr=0, seed=3)
    b = built(rs3, U=4, H=1, d=64, dtype="f32", m=8, n=9, window=-1, ring_frames=3, commits=2, n_ptr=0, n_cond=0, seed=4)
    q, idx, count, group, prefix_unit, table, out = shared_case(rs3, b, p, [20, 30, 40, 9], [0] * 4, [0] * 4, 1)
    whole = rs3.Bank(4, 1, 64, "f32", 72, 1, -1, 12 * 72, 12, 0)
    st = status()
    rs3.rs3_bank_copy(whole, p.bank, torch.zeros(4, dtype=torch.int32, device="cuda"), None, None, st)
    for f in range(2):                                     # the children's own frames, once more
        rows = [b.places(u)[0] for u in range(4)]
        lens = [b.places(u)[1] for u in range(4)]
        k, v = (torch.zeros((4, 72, 64), device="cuda") for _ in range(2))
        mask = torch.zeros((4, 72), dtype=torch.uint8, device="cuda")
        for u in range(4):
            at = torch.from_numpy(rows[u][sum(lens[u][:f]):sum(lens[u][:f + 1])]).cuda()
            k[u, :len(at)], v[u, :len(at)], mask[u, :len(at)] = b.bank.k_store[u][at], b.bank.v_store[u][at], 1
        rs3.rs3_bank_commit(whole, k, v, mask, 0, st)
    ref = torch.zeros_like(out)
    ws = torch.empty(rs3.rs3_readout_workspace_bytes(4, 1, 64, 40, "f32"), dtype=torch.uint8, device="cuda")
    rs3.rs3_memory_readout(q, "f32", 1, 72, 1, 64, group, idx, count, 40, whole, None, None, ref, 0.0, ws, st)
    assert int(st) == 0
    vmax = float(torch.cat([p.bank.v_store[0], b.bank.v_store.view(-1, 64)]).abs().clamp(max=999).max())
    assert float((out - ref).abs().max()) <= vmax * 2.0 ** -13


def test_shared_readout_latches_what_the_device_finds(rs3):
    b = built(rs3, U=6, H=1, d=64, dtype="bf16", m=8, n=9, window=4, commits=5, n_ptr=0, seed=2)
    p = built(rs3, U=3, H=1, d=64, dtype="bf16", m=8, n=9, window=4, commits=5, n_ptr=0, seed=3)
    g = gen(1)
    q = torch.randn((2, 72, 64), generator=g, device="cuda").bfloat16()
    idx, count = keep_sets(6, 72, 20, [20, 20, 20, 20, 20, 20])
    good = (torch.tensor([0, 0, 1, 0, 0, 0], dtype=torch.int32, device="cuda"), torch.tensor([0, 0, 0, 1, 2, -1], dtype=torch.int32, device="cuda"))
    clean = torch.zeros((6, 72, 64), dtype=torch.bfloat16, device="cuda")
    run_shared(rs3, b, p, q, 2, idx, count, good[0], good[1], None, 0.0, None, clean)
    assert int(b.st) == 0

    def call(group=good[0], prefix=good[1], idx=idx, count=count):
        b.st.zero_()
        res = torch.full((6, 72, 64), 5.0, dtype=torch.bfloat16, device="cuda")
        out = torch.zeros_like(res)
        run_shared(rs3, b, p, q, 2, idx, count, group, prefix, None, 0.0, res, out)
        code = int(b.st)
        b.st.zero_()
        return code, out, [bool((out[u] == 5).all()) for u in range(6)]

    def put(t, i, v):
        t = t.clone()
        t[i] = v
        return t

    for bad in (dict(group=put(good[0], 1, 2)), dict(group=put(good[0], 1, -1)), dict(prefix=put(good[1], 1, 3)), dict(prefix=put(good[1], 1, -2)),
                dict(count=put(count, 1, 21)), dict(count=put(count, 1, -1))):
        code, out, skipped = call(**bad)
        assert code == rs3.RS3_EINVAL and skipped == [False, True, False, False, False, False], bad
    code, out, skipped = call(idx=put(put(idx, (1, 3), -1), (1, 4), 72))
    assert code == rs3.RS3_EINVAL and not any(skipped)
    # unsound counters: of a unit, and of a prefix (which skips the units that read it)
    for store, unit, gone in ((b, 3, [3]), (p, 0, [0, 1, 2])):
        old = store.bank.counters[unit, 1].clone()
        store.bank.counters[unit, 1] = -5
        code, out, skipped = call()
        store.bank.counters[unit, 1] = old
        assert code == rs3.RS3_EINTERNAL and skipped == [u in gone for u in range(6)]


def test_shared_readout_stays_inside_its_workspace_and_repeats_itself(rs3):
    for dtype, H, d in (("bf16", 2, 64), ("bf16", 1, 256), ("f32", 1, 32)):
        b = built(rs3, U=3, H=H, d=d, dtype=dtype, m=16, n=20, window=4, commits=5, n_ptr=0, seed=2)
        p = built(rs3, U=2, H=H, d=d, dtype=dtype, m=16, n=20, window=4, commits=5, n_ptr=0, seed=3)
        q, idx, count, group, prefix_unit, table, out = shared_case(rs3, b, p, [320, 200, 90], [0, 0, 0], [1, 1, 0], 1)
        n = rs3.rs3_shared_readout_workspace_bytes(b.bank, p.bank, idx.shape[1])
        ws = torch.full((n + 4096,), 77, dtype=torch.uint8, device="cuda")
        for _ in range(3):
            again = torch.full_like(out, math.nan)
            run_shared(rs3, b, p, q, 1, idx, count, group, prefix_unit, table, 0.0, None, again, ws[:n])
            assert torch.equal(bits(again), bits(out))
        assert (ws[n:] == 77).all()
        with pytest.raises(rs3.RS3Error) as e:
            run_shared(rs3, b, p, q, 1, idx, count, group, prefix_unit, table, 0.0, None, out, ws[:n - 256])
        assert e.value.code == rs3.RS3_ECAPACITY


def test_shared_readout_captured_and_on_another_stream(rs3):
    b = built(rs3, U=3, H=1, d=64, dtype="bf16", m=8, n=9, window=4, commits=5, n_ptr=0, seed=2)
    p = built(rs3, U=1, H=1, d=64, dtype="bf16", m=8, n=9, window=4, commits=5, n_ptr=0, seed=3)
    q, idx, count, group, prefix_unit, table, out = shared_case(rs3, b, p, [30, 20, 9], [0, 0, 0], [0, 0, 0], 1)
    ws = run_shared(rs3, b, p, q, 1, idx, count, group, prefix_unit, table, 0.0, None, out)
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        run_shared(rs3, b, p, q, 1, idx, count, group, prefix_unit, table, 0.0, None, out, ws)
    b.commit(gen(9))
    q.mul_(0.5)
    graph.replay()
    torch.cuda.synchronize()
    got = out.clone()
    out.zero_()
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    run_shared(rs3, b, p, q, 1, idx, count, group, prefix_unit, table, 0.0, None, out, ws, side)
    side.synchronize()
    assert torch.equal(bits(got), bits(out)) and (got != 0).any()


@pytest.mark.parametrize("dtype,d", [("bf16", 64), ("bf16", 256)])
def test_shared_readout_wait_limit_runs_out_and_the_context_stays_usable(rs3, dtype, d):
    b = built(rs3, U=3, H=1, d=d, dtype=dtype, m=8, n=9, window=4, commits=5, n_ptr=0, seed=2)
    p = built(rs3, U=1, H=1, d=d, dtype=dtype, m=8, n=9, window=4, commits=5, n_ptr=0, seed=3)
    q, idx, count, group, prefix_unit, table, out = shared_case(rs3, b, p, [30, 20, 9], [0, 0, 0], [0, 0, 0], 1)
    limit = rs3.rs3_get_wait_limit_ns()
    try:
        rs3.rs3_set_wait_limit_ns(0)
        again = torch.zeros_like(out)
        run_shared(rs3, b, p, q, 1, idx, count, group, prefix_unit, table, 0.0, None, again)
        code = int(b.st)
    finally:
        rs3.rs3_set_wait_limit_ns(limit)
    assert code == rs3.RS3_ETIMEOUT
    b.st.zero_()
    run_shared(rs3, b, p, q, 1, idx, count, group, prefix_unit, table, 0.0, None, again)
    assert int(b.st) == 0 and torch.equal(bits(again), bits(out))


# ---------------------------------------------------------------------------
# capped and biased scores, frames left out
# ---------------------------------------------------------------------------
def run_scored(rs3, b, q, G, idx, count, group, cap, bias, keep, table, scale, res, out, ws=None, stream=None):
    k_max = idx.shape[1]
    if ws is None:
        ws = torch.full((rs3.rs3_scored_readout_workspace_bytes(b.bank, k_max),), 255, dtype=torch.uint8, device="cuda")
    rs3.rs3_scored_readout(q, b.dtype, G, b.mn, b.H, b.d, group, idx, count, k_max, b.bank, cap, bias, keep, table, res, out, scale, ws,
                           b.st, stream)
    return ws


def scored_rows(b, keep):
    def rows(u):
        at, slot = frames_of(b, u)
        if keep is not None:
            on = keep[u][slot] != 0
            at, slot = at[on], slot[on]
        return b.bank.k_store[u][at], b.bank.v_store[u][at], slot
    return rows


def scored_case(rs3, b, counts, group, G, cap=0.0, bias=None, keep=None, residual="none", rope=False, seed=5, k_max=None, scale=0.0, qs=1.2):
    U, mn, D, dtype = b.U, b.mn, b.D, b.dtype
    g = gen(seed)
    q = (torch.randn((G, mn, D), generator=g, device="cuda") * qs).to(DT[dtype])
    k_max = max(1, max(counts)) if k_max is None else k_max
    idx, count = keep_sets(U, mn, k_max, counts, seed)
    group = torch.tensor(group, dtype=torch.int32, device="cuda")
    table = rope_table(mn, b.d) if rope else None
    x = torch.randn((U, mn, D), generator=g, device="cuda").to(DT[dtype])
    res = None if residual == "none" else x.clone()
    out = res if residual == "inplace" else torch.full_like(x, math.nan)
    of = None if bias is None else lambda u, h: bias[u, h] if bias.dim() == 3 else bias[h]
    want, tol = reference(dtype, b.H, b.d, q, idx, counts, group, table, scale or b.d ** -0.5, None if res is None else x, x.shape,
                          scored_rows(b, keep), cap, of)
    ws = run_scored(rs3, b, q, G, idx, count, group, cap, bias, keep, table, scale, res, out)
    assert int(b.st) == 0
    err = (out.double() - want).abs()
    assert (err <= tol).all(), (float((err - tol).max()), float(err.max()))
    return q, idx, count, group, table, out, ws


def biases(b, kind, seed=3):
    F = b.bank.max_frames
    if kind == "age":
        age = torch.arange(F + 2, device="cuda").float()
        age[F:] = 0
        return (-age[None] * torch.tensor([2.0 ** (-h) for h in range(b.H)], device="cuda")[:, None]).contiguous()
    if kind == "unit":
        return torch.randn((b.U, b.H, F + 2), generator=gen(seed), device="cuda") * 2
    if kind == "holes":                                    # minus infinity for some frames, for all of one head of a unit
        t = torch.randn((b.U, b.H, F + 2), generator=gen(seed), device="cuda")
        t = torch.where(torch.rand(t.shape, generator=gen(seed + 1), device="cuda") < 0.5, -math.inf, t)
        t[0, 0] = -math.inf
        return t
    return None


def keeps(b, kind, seed=7):
    F = b.bank.max_frames
    if kind == "all":
        return None
    t = (torch.rand((b.U, F + 2), generator=gen(seed), device="cuda") < 0.5).to(torch.uint8) * 3
    if kind == "alternate":
        t[:] = (torch.arange(F + 2, device="cuda") % 2 == 0).to(torch.uint8)
    if kind == "nothing":
        t[0] = 0
    return t


def spoil(b, keep):
    """NaN in every row that is not read."""
    for u in range(b.U):
        at, slot = frames_of(b, u)
        on = torch.zeros(b.bank.rows_per_unit, dtype=torch.bool, device="cuda")
        on[at if keep is None else at[keep[u][slot] != 0]] = True
        for t in (b.bank.k_store, b.bank.v_store):
            t[u, ~on] = math.nan


LAYOUTS = [dict(window=4, commits=7, n_ptr=5), dict(window=-1, ring_frames=9, commits=9, n_ptr=3, n_cond=2),
           dict(window=1, commits=2, n_cond=0, n_ptr=0), dict(window=6, commits=3, n_ptr=0)]


@pytest.mark.parametrize("dtype,H,d", SHAPES)
@pytest.mark.parametrize("counts", [[1, 0, 3], [72, 17, 33]])
@pytest.mark.parametrize("cap,bias,keep,residual,rope", [(0.0, None, "some", "none", False), (5.0, None, "all", "inplace", True),
                                                         (0.0, "age", "alternate", "other", False), (2.5, "unit", "nothing", "inplace", False),
                                                         (30.0, "holes", "some", "none", True), (0.0, "holes", "all", "other", False)])
def test_scored_readout_matches_64_bits(rs3, dtype, H, d, counts, cap, bias, keep, residual, rope):
    """Wrapped rings, units without rows, NaN in dead rows and in those that are left out."""
    b = Built(rs3, U=3, H=H, d=d, dtype=dtype, m=8, n=9, empty=(1,), seed=2, **LAYOUTS[(d // 16 + len(residual)) % 4])
    rs3.rs3_bank_reset(b.bank, 1)
    kp = keeps(b, keep)
    spoil(b, kp)
    scored_case(rs3, b, counts, [0, 1, 0], 2, cap, biases(b, bias), kp, residual, rope, scale=0.2 if rope else 0.0)


@pytest.mark.parametrize("dtype,H,d", [("bf16", 2, 64), ("bf16", 2, 128), ("bf16", 1, 256), ("f32", 1, 64), ("f32", 1, 256), ("bf16", 2, 32)])
@pytest.mark.parametrize("keep", ["all", "some"])
def test_scored_readout_of_long_banks(rs3, dtype, H, d, keep):
    """Rows split over many pieces, hundreds of small frames, many query tiles."""
    b = Built(rs3, U=2, H=H, d=d, dtype=dtype, m=32, n=33, window=-1, ring_frames=300, commits=290, n_ptr=3, seed=3, density=0.03)
    kp = keeps(b, keep)
    spoil(b, kp)
    scored_case(rs3, b, [300, 7], [0, 0], 1, 8.0, biases(b, "unit"), kp, "inplace")
    scored_case(rs3, b, [1, 1056], [0, 0], 1, 0.0, biases(b, "age"), kp, "none")
    c = Built(rs3, U=2, H=H, d=d, dtype=dtype, m=32, n=33, window=5, commits=8, n_ptr=0, seed=3, density=0.9)
    kp = keeps(c, keep)
    spoil(c, kp)
    scored_case(rs3, c, [1056, 513], [0, 1], 2, 8.0, biases(c, "unit"), kp, "other", rope=True)


@pytest.mark.parametrize("d", [64, 128])
@pytest.mark.parametrize("cap,bias,keep", [(10.0, "unit", "some"), (0.0, "age", "alternate"), (6.0, None, "all"), (0.0, "holes", "all"), (0.0, None, "some")])
def test_scored_readout_by_pairs_of_query_tiles(rs3, d, cap, bias, keep):
    """Enough work that the plan takes two query tiles per CTA."""
    H, frames = 512 // d, 4 if d == 64 else 11
    b = Built(rs3, U=4, H=H, d=d, dtype="bf16", m=64, n=64, window=-1, ring_frames=frames, commits=frames, n_ptr=3, seed=2, density=0.6)
    kp = keeps(b, keep)
    spoil(b, kp)
    scored_case(rs3, b, [2500, 1200, 129, 640], [0, 0, 0, 0], 1, cap, biases(b, bias), kp, "inplace")


@pytest.mark.parametrize("dtype,H,d", SHAPES)
@pytest.mark.parametrize("cap,bias,keep,residual", [(0.0, None, "some", "none"), (5.0, "age", "all", "inplace"), (0.0, "unit", "alternate", "other"),
                                                    (30.0, "holes", "nothing", "none")])
def test_scored_readout_of_one_unit(rs3, dtype, H, d, cap, bias, keep, residual):
    for layout in LAYOUTS:
        b = Built(rs3, U=1, H=H, d=d, dtype=dtype, m=8, n=9, seed=2, **layout)
        kp = keeps(b, keep)
        spoil(b, kp)
        scored_case(rs3, b, [33], [1], 2, cap, biases(b, bias), kp, residual)
        scored_case(rs3, b, [0], [0], 1, cap, biases(b, bias), kp, residual, k_max=5)


@pytest.mark.parametrize("d", [64, 128])
@pytest.mark.parametrize("residual", ["inplace", "other"])
def test_scored_readout_of_one_unit_of_much_work(rs3, d, residual):
    """Two tables of key tiles, two query tiles per CTA, hundreds of frames."""
    b = Built(rs3, U=1, H=1024 // d, d=d, dtype="bf16", m=63, n=65, window=-1, ring_frames=300, commits=290, n_ptr=3, seed=2, density=0.1,
              ring=126000)
    kp = keeps(b, "some")
    spoil(b, kp)
    scored_case(rs3, b, [3000], [0], 1, 10.0, biases(b, "unit"), kp, residual)
    words, good = b.bank.meta, b.bank.meta.clone()
    q, idx, count, group, _, out, ws = scored_case(rs3, b, [300], [0], 1, 10.0, None, kp, "none", k_max=3000)
    for word, value in ((16 + 100, int(words[16 + 100]) + 1), (3, 301), (1, -5)):
        words[word] = value
        again = torch.full_like(out, 5.0)
        run_scored(rs3, b, q, 1, idx, count, group, 10.0, None, kp, None, 0.0, again, again, ws)
        words.copy_(good)
        assert int(b.st) == rs3.RS3_EINTERNAL and (again == 5).all()
        b.st.zero_()


@pytest.mark.parametrize("d", [64, 128])
@pytest.mark.parametrize("residual", ["none", "other"])
@pytest.mark.parametrize("counts", [[2500, 1200, 129, 0], [70, 3, 0, 1], [0, 0, 0, 0], [4095, 4095, 4095, 4095]])
def test_scored_readout_of_much_work_passes_the_other_cells_through(rs3, d, residual, counts):
    """Out of place: cells that are not kept are the residual's bit for bit, or zeros, whichever kernel reaches them; the
    grid's last word of cells is a part; few queries leave all of it to the merge."""
    H, frames = 512 // d, 4 if d == 64 else 11
    b = Built(rs3, U=4, H=H, d=d, dtype="bf16", m=63, n=65, window=-1, ring_frames=frames, commits=frames, n_ptr=3, seed=2, density=0.6)
    spoil(b, None)
    for _ in range(2):
        scored_case(rs3, b, counts, [0, 0, 0, 0], 1, 6.0, biases(b, "age"), None, residual, k_max=4095)


def test_scored_readout_of_much_work_passes_skipped_units_through(rs3):
    """A unit whose group, count or frames are unsound, or whose cells are partly none, is the residual there."""
    b = Built(rs3, U=4, H=8, d=64, dtype="bf16", m=63, n=65, window=-1, ring_frames=4, commits=4, n_ptr=3, seed=2, density=0.6)
    spoil(b, None)
    counts = [2500, 1200, 900, 640]
    q, idx, count, group, _, clean, ws = scored_case(rs3, b, counts, [0] * 4, 1, 6.0, None, None, "none", k_max=4095)
    res = torch.randn(clean.shape, generator=gen(3), device="cuda").bfloat16()
    words = b.bank.meta.view(4, -1)
    good = words.clone()
    for what in ("group", "count", "tail", "frame", "cell"):
        g, c, i = group.clone(), count.clone(), idx.clone()
        if what == "group":
            g[1] = 1
        elif what == "count":
            c[1] = 4096
        elif what == "tail":
            words[1, 1] = -5
        elif what == "frame":
            words[1, 16] += 1
        else:
            i[1, 3], i[1, 4] = -1, 4095
        out = torch.full_like(clean, math.nan)
        run_scored(rs3, b, q, 1, i, c, g, 6.0, None, None, None, 0.0, res, out, ws)
        code = int(b.st)
        b.st.zero_()
        words.copy_(good)
        assert code == (rs3.RS3_EINTERNAL if what in ("tail", "frame") else rs3.RS3_EINVAL), what
        assert not out.isnan().any(), what
        if what != "cell":
            assert torch.equal(bits(out[1]), bits(res[1])), what
        for u, n in enumerate(counts):
            other = torch.ones(b.mn, dtype=torch.bool, device="cuda")
            other[idx[u, :n].long()] = False
            assert torch.equal(bits(out[u, other]), bits(res[u, other])), (what, u)
        if what == "cell":
            gone = idx[1, 3:5].long()
            assert torch.equal(bits(out[1, gone]), bits(res[1, gone]))


@pytest.mark.parametrize("dtype,d", [("bf16", 64), ("bf16", 256), ("f32", 32)])
def test_scored_readout_of_scores_of_all_sizes(rs3, dtype, d):
    """Scores far beyond the cap and far below it, biases of thousands, references that move late."""
    b = Built(rs3, U=2, H=1, d=d, dtype=dtype, m=16, n=17, window=-1, ring_frames=12, commits=12, n_ptr=0, seed=3, scale=6.0)
    F = b.bank.max_frames
    spoil(b, None)
    scored_case(rs3, b, [100, 40], [0, 0], 1, 2.0 ** -10, None, None)
    scored_case(rs3, b, [100, 40], [0, 0], 1, 2.0 ** 10, None, None, qs=0.01)
    scored_case(rs3, b, [100, 40], [0, 0], 1, 20.0, None, None, qs=3.0)
    # the oldest rows are read first: the reference climbs by 100 from frame to frame, or starts at minus infinity
    climb = -100.0 * torch.arange(F + 2, device="cuda").float()[None]
    climb[:, F:] = -5000.0
    scored_case(rs3, b, [100, 40], [0, 0], 1, 10.0, climb.contiguous(), None)
    late = torch.full((1, F + 2), -math.inf, device="cuda")
    late[:, 0] = -3000.0
    scored_case(rs3, b, [100, 40], [0, 0], 1, 0.0, late, None)
    late[:, 5] = 3000.0
    scored_case(rs3, b, [100, 40], [0, 0], 1, 3.0, late, None)


@pytest.mark.parametrize("dtype,H,d,m", [("bf16", 2, 64, 16), ("bf16", 1, 128, 16), ("bf16", 1, 256, 16), ("bf16", 8, 64, 64), ("bf16", 4, 128, 80),
                                         ("f32", 1, 64, 16)])
@pytest.mark.parametrize("cap", [55.0, 55.5, 200.0])
def test_scored_readout_of_rows_at_either_end_of_the_cap(rs3, dtype, H, d, m, cap):
    """Rows whose scores are all near minus the cap, all near the cap, some of either, and within half of it, on both sides of
    the largest cap whose weights need no running maximum; biases that lift and sink frames by more than the cap."""
    b = Built(rs3, U=2, H=H, d=d, dtype=dtype, m=m, n=m, window=4 if m == 16 else 8, commits=6 if m == 16 else 8, n_ptr=3, seed=5, density=0.7)
    spoil(b, None)
    b.bank.k_store.abs_()
    U, mn, D = 2, b.mn, b.D
    counts = [mn // 2, mn - 1]
    idx, count = keep_sets(U, mn, mn, counts, 6)
    g = gen(8)
    q = torch.randn((1, mn, D), generator=g, device="cuda").abs() * 8.0
    kind = torch.arange(mn, device="cuda")[None, :, None] // 32 % 4
    mixed = torch.randn((1, mn, D), generator=g, device="cuda")
    q = torch.where(kind == 0, -q, torch.where(kind == 1, q, torch.where(kind == 2, 20.0 * mixed, mixed))).to(DT[dtype])
    group = torch.zeros(2, dtype=torch.int32, device="cuda")
    unit = biases(b, "unit") * 60.0
    for bias in (None, unit, torch.where(torch.rand(unit.shape, generator=g, device="cuda") < 0.3, -math.inf, unit)):
        out = torch.full((U, mn, D), math.nan, dtype=DT[dtype], device="cuda")
        want, tol = reference(dtype, H, d, q, idx, counts, group, None, d ** -0.5, None, out.shape, scored_rows(b, None), cap,
                              None if bias is None else lambda u, h: bias[u, h])
        run_scored(rs3, b, q, 1, idx, count, group, cap, bias, None, None, 0.0, None, out)
        assert int(b.st) == 0
        err = (out.double() - want).abs()
        assert (err <= tol).all(), (float((err - tol).max()), float(err.max()))
        assert tol.max() < 1.0


@pytest.mark.parametrize("dtype,H,d", [("f32", 4, 64), ("f32", 8, 32), ("f32", 8, 16), ("f32", 4, 256), ("bf16", 8, 16), ("bf16", 8, 32)])
def test_readouts_of_whole_query_tiles_on_the_cuda_cores(rs3, dtype, H, d):
    """Enough queries and keys that a CTA takes its largest query tile, and calls with a few of either on the same workspace."""
    U, counts = 8, [300, 1, 0, 129, 128, 300, 257, 64]
    b = Built(rs3, U=U, H=H, d=d, dtype=dtype, m=30, n=30, window=2, commits=3, n_ptr=5, seed=4)
    BM, ctas = (64, 1) if d == 256 else (128, 2)
    assert U * H * -(-300 // BM) * (b.bank.rows_per_unit // 32) >= 16 * ctas * torch.cuda.get_device_properties(0).multi_processor_count
    kp, bias = keeps(b, "some"), biases(b, "unit")
    spoil(b, kp)
    scored_case(rs3, b, counts, [0, 1] * 4, 2, 9.0, bias, kp, "inplace")
    q, idx, count, group, table, out, ws = scored_case(rs3, b, counts, [0] * U, 1, 0.0, None, kp, "none", rope=True, k_max=300)
    few, first = torch.full_like(out, math.nan), idx[:, :20].contiguous()
    run_scored(rs3, b, q, 1, first, count.clamp(max=20), group, 0.0, None, kp, table, 0.0, None, few, ws)
    assert int(b.st) == 0
    want, tol = reference(dtype, H, d, q, first, [min(n, 20) for n in counts], group, table, d ** -0.5, None, out.shape, scored_rows(b, kp))
    assert ((few.double() - want).abs() <= tol).all()
    c = built(rs3, U=U, H=H, d=d, dtype=dtype, m=30, n=30, window=2, commits=3, n_ptr=5, seed=4)
    p = built(rs3, U=2, H=H, d=d, dtype=dtype, m=30, n=30, window=3, commits=3, n_ptr=0, seed=6)
    shared_case(rs3, c, p, counts, [0] * U, [0, 0, 1, 1, 1, 0, -1, 1], 1, "other")


@pytest.mark.parametrize("dtype,d", [("bf16", 64), ("bf16", 256), ("f32", 32)])
@pytest.mark.parametrize("lowest", [-3.4028234663852886e38, -math.inf])
def test_scored_readout_masked_by_the_lowest_value(rs3, dtype, d, lowest):
    """Frames that a bias of the type's lowest value masks weigh nothing, and a query with no other reads 0."""
    b = Built(rs3, U=2, H=2, d=d, dtype=dtype, m=8, n=9, window=4, commits=5, n_ptr=3, seed=2)
    spoil(b, None)
    bias = torch.zeros((2, 2, b.bank.max_frames + 2), device="cuda")
    bias[0, 0], bias[1, 1, 1:] = lowest, lowest
    same = torch.where(bias < -1e30, -math.inf, bias)
    q = torch.randn((1, 72, 2 * d), generator=gen(1), device="cuda").to(DT[dtype])
    idx, count = keep_sets(2, 72, 40, [40, 40])
    group = torch.zeros(2, dtype=torch.int32, device="cuda")
    outs = []
    for t in (bias, same):
        out = torch.zeros((2, 72, 2 * d), dtype=DT[dtype], device="cuda")
        run_scored(rs3, b, q, 1, idx, count, group, 7.0, t, None, None, 0.0, None, out)
        outs.append(out)
    assert torch.equal(bits(outs[0]), bits(outs[1])) and not outs[0].isnan().any()
    assert (outs[0][0, :, :d] == 0).all() and (outs[0][0, idx[0].long(), d:] != 0).any() and (outs[0][1, idx[1].long(), d:] != 0).any()
    want, tol = reference(dtype, 2, d, q, idx, [40, 40], group, None, d ** -0.5, None, outs[0].shape, scored_rows(b, None), 7.0, lambda u, h: same[u, h])
    assert ((outs[0].double() - want).abs() <= tol).all()


@pytest.mark.parametrize("dtype,H,d", [("bf16", 4, 64), ("f32", 1, 128)])
def test_readouts_of_rows_past_32_bit_offsets(rs3, dtype, H, d):
    """A bank whose ring and pointers begin past 2^31 elements."""
    D = H * d
    n_cond = -(-(1 << 31) // (D * 16384)) + 3
    b = types.SimpleNamespace(rs3=rs3, U=1, H=H, d=d, D=D, dtype=dtype, mn=16384, st=status())
    b.bank = rs3.Bank(1, H, d, dtype, b.mn, n_cond, 2, 2 * b.mn, 2, 7)
    b.places = lambda u, bank=None: Built.places(b, u, bank)
    assert b.bank.pinned_cap * D > 1 << 31
    g = gen(5)
    for f in range(4):
        k, v = (torch.randn((1, b.mn, D), generator=g, device="cuda").to(DT[dtype]) for _ in range(2))
        mask = (torch.rand((1, b.mn), generator=g, device="cuda") < 0.02).to(torch.uint8)
        rs3.rs3_bank_commit(b.bank, k, v, mask, int(f == 0), b.st)
    rs3.rs3_bank_set_pointers(b.bank, *(torch.randn((1, 7, D), generator=g, device="cuda").to(DT[dtype]) for _ in range(2)), b.st)
    bias = torch.randn((H, 4), generator=g, device="cuda")
    keep = torch.tensor([[1, 1, 0, 1]], dtype=torch.uint8, device="cuda")
    scored_case(rs3, b, [150], [0], 1, 9.0, bias, keep)
    shared_case(rs3, b, b, [150], [0], [0], 1)


@pytest.mark.parametrize("dtype,H,d", [("bf16", 2, 64), ("bf16", 1, 256), ("f32", 2, 64)])
def test_scored_readout_without_a_change_is_the_memory_readout(rs3, dtype, H, d):
    b = built(rs3, U=3, H=H, d=d, dtype=dtype, m=16, n=17, window=4, commits=7, n_ptr=5, seed=2)
    q, idx, count, group, table, out, _ = scored_case(rs3, b, [250, 0, 100], [0, 0, 0], 1, rope=True)
    ref = torch.full_like(out, math.nan)
    ws = torch.empty(rs3.rs3_readout_workspace_bytes(3, H, d, 250, dtype), dtype=torch.uint8, device="cuda")
    rs3.rs3_memory_readout(q, dtype, 1, b.mn, H, d, group, idx, count, 250, b.bank, table, None, ref, 0.0, ws, b.st)
    vmax = float(b.bank.v_store.float().where(b.bank.v_store.float() < 999, 0.0).abs().max())
    assert float((out.float() - ref.float()).abs().max()) <= vmax * (2.0 ** -6 if dtype == "bf16" else 2.0 ** -13)


@pytest.mark.parametrize("dtype,H,d", [("bf16", 1, 64), ("bf16", 1, 256), ("f32", 1, 64)])
def test_scored_readout_of_scores_that_are_no_numbers(rs3, dtype, H, d):
    """A key with NaN makes its queries NaN, unless its frame is left out."""
    b = Built(rs3, U=2, H=H, d=d, dtype=dtype, m=8, n=9, window=4, commits=5, n_ptr=0, seed=2)
    spoil(b, None)
    at, slot = frames_of(b, 0)
    b.bank.k_store[0, at[slot == 1][0]] = math.nan
    q = torch.randn((1, 72, H * d), generator=gen(1), device="cuda").to(DT[dtype])
    idx, count = keep_sets(2, 72, 30, [30, 30])
    group = torch.zeros(2, dtype=torch.int32, device="cuda")
    for cap in (0.0, 4.0):
        out = torch.zeros((2, 72, H * d), dtype=DT[dtype], device="cuda")
        run_scored(rs3, b, q, 1, idx, count, group, cap, biases(b, "age"), None, None, 0.0, None, out)
        assert out[0, idx[0].long()].isnan().all() and not out[1].isnan().any()
        keep = torch.ones((2, b.bank.max_frames + 2), dtype=torch.uint8, device="cuda")
        keep[:, 1] = 0
        out.zero_()
        run_scored(rs3, b, q, 1, idx, count, group, cap, biases(b, "age"), keep, None, 0.0, None, out)
        assert not out.isnan().any() and (out[0] != 0).any()


def test_scored_readout_latches_what_the_device_finds(rs3):
    for dtype, d in (("bf16", 64), ("f32", 32)):
        b = built(rs3, U=4, H=1, d=d, dtype=dtype, m=8, n=9, window=4, commits=5, n_ptr=0, seed=2)
        q = torch.randn((2, 72, d), generator=gen(1), device="cuda").to(DT[dtype])
        idx, count = keep_sets(4, 72, 20, [20] * 4)
        group = torch.tensor([0, 0, 1, 0], dtype=torch.int32, device="cuda")

        def call(group=group, idx=idx, count=count):
            b.st.zero_()
            res = torch.full((4, 72, d), 5.0, dtype=DT[dtype], device="cuda")
            out = torch.zeros_like(res)
            run_scored(rs3, b, q, 2, idx, count, group, 9.0, biases(b, "age"), None, None, 0.0, res, out)
            code = int(b.st)
            b.st.zero_()
            return code, out, [bool((out[u] == 5).all()) for u in range(4)]

        def put(t, i, v):
            t = t.clone()
            t[i] = v
            return t

        assert call()[0] == 0
        for bad in (dict(group=put(group, 1, 2)), dict(group=put(group, 1, -1)), dict(count=put(count, 1, 21)), dict(count=put(count, 1, -1))):
            code, out, skipped = call(**bad)
            assert code == rs3.RS3_EINVAL and skipped == [False, True, False, False], bad
        clean = call()[1]
        for bad in (-1, 72):
            code, out, skipped = call(idx=put(idx, (1, 3), bad))
            gone = torch.zeros(72, dtype=torch.bool, device="cuda")
            gone[int(idx[1, 3])] = True
            assert code == rs3.RS3_EINVAL and (out[1, gone] == 5).all() and torch.equal(bits(out[1, ~gone]), bits(clean[1, ~gone]))
        old = b.bank.counters[3, 1].clone()
        b.bank.counters[3, 1] = -5
        code, out, skipped = call()
        b.bank.counters[3, 1] = old
        assert code == rs3.RS3_EINTERNAL and skipped == [False, False, False, True]


def test_scored_readout_skips_units_whose_frames_do_not_fill_the_ring(rs3):
    """Frames that overlap, leave rows between them, or are more than the table holds: the unit is skipped, nothing past its
    tables is written."""
    for dtype, H, d, bias in (("bf16", 1, 64, "age"), ("bf16", 1, 256, "unit"), ("f32", 1, 32, None)):
        b = Built(rs3, U=3, H=H, d=d, dtype=dtype, m=16, n=20, window=6, commits=8, n_ptr=0, seed=2)
        b.bank.k_store.nan_to_num_(0.0)
        b.bank.v_store.nan_to_num_(0.0)
        words = b.bank.meta.view(3, -1)
        kp, bias = keeps(b, "alternate"), biases(b, bias)
        q, idx, count, group, table, out, _ = scored_case(rs3, b, [40, 300, 200], [0, 0, 0], 1, 6.0, bias, kp)
        n, F, good = rs3.rs3_scored_readout_workspace_bytes(b.bank, idx.shape[1]), b.bank.max_frames, words.clone()
        off, length = 16, 16 + F
        head, tail, oldest = int(good[1, 0]), int(good[1, 1]), int(good[1, 4])
        wide = {off + i: head for i in range(F)} | {length + i: tail - head for i in range(F)}
        second = (oldest + 1) % F
        for change in (wide, {3: F + 1}, {3: -1}, {4: F}, {4: -1}, {3: 0}, {off + second: int(good[1, off + second]) + 1},
                       {length + second: int(good[1, length + second]) - 1}, {length + second: -1}, {off + oldest: head - 1},
                       {off + oldest: -(2 ** 62)}, {length + oldest: 2 ** 62}):
            for word, value in change.items():
                words[1, word] = value
            ws = torch.full((n + 65536,), 77, dtype=torch.uint8, device="cuda")
            again = torch.full_like(out, 5.0)
            b.st.zero_()
            run_scored(rs3, b, q, 1, idx, count, group, 6.0, bias, kp, table, 0.0, again, again, ws[:n])
            code = int(b.st)
            b.st.zero_()
            words.copy_(good)
            assert code == rs3.RS3_EINTERNAL, change
            assert (again[1] == 5).all() and not (again[0] == 5).all() and not (again[2] == 5).all(), change
            assert (ws[n:] == 77).all()


def test_scored_readout_stays_inside_its_workspace_and_repeats_itself(rs3):
    for dtype, H, d in (("bf16", 2, 64), ("bf16", 1, 256), ("f32", 1, 32)):
        b = Built(rs3, U=3, H=H, d=d, dtype=dtype, m=16, n=20, window=4, commits=5, n_ptr=7, seed=2)
        kp = keeps(b, "alternate")
        spoil(b, kp)
        bias = biases(b, "unit")
        q, idx, count, group, table, out, _ = scored_case(rs3, b, [320, 200, 90], [0, 0, 0], 1, 6.0, bias, kp)
        n = rs3.rs3_scored_readout_workspace_bytes(b.bank, idx.shape[1])
        ws = torch.full((n + 4096,), 77, dtype=torch.uint8, device="cuda")
        for _ in range(3):
            again = torch.full_like(out, math.nan)
            run_scored(rs3, b, q, 1, idx, count, group, 6.0, bias, kp, table, 0.0, None, again, ws[:n])
            assert torch.equal(bits(again), bits(out))
        assert (ws[n:] == 77).all()
        with pytest.raises(rs3.RS3Error) as e:
            run_scored(rs3, b, q, 1, idx, count, group, 6.0, bias, kp, table, 0.0, None, out, ws[:n - 256])
        assert e.value.code == rs3.RS3_ECAPACITY


def test_scored_readout_captured_and_on_another_stream(rs3):
    b = Built(rs3, U=3, H=1, d=64, dtype="bf16", m=8, n=9, window=4, commits=5, n_ptr=0, seed=2)
    b.bank.k_store.nan_to_num_(0.0)
    b.bank.v_store.nan_to_num_(0.0)
    bias, kp = biases(b, "unit"), keeps(b, "some")
    q, idx, count, group, table, out, ws = scored_case(rs3, b, [30, 20, 9], [0, 0, 0], 1, 6.0, bias, kp)
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        run_scored(rs3, b, q, 1, idx, count, group, 6.0, bias, kp, None, 0.0, None, out, ws)
    b.commit(gen(9))
    kp[:, :2] = 1
    bias.add_(0.5)
    q.mul_(0.5)
    graph.replay()
    torch.cuda.synchronize()
    got = out.clone()
    out.zero_()
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    run_scored(rs3, b, q, 1, idx, count, group, 6.0, bias, kp, None, 0.0, None, out, ws, side)
    side.synchronize()
    assert torch.equal(bits(got), bits(out)) and (got != 0).any()


@pytest.mark.parametrize("d,pairs", [(64, False), (128, False), (256, False), (64, True)])
def test_scored_readout_wait_limit_runs_out_and_the_context_stays_usable(rs3, d, pairs):
    if pairs:
        b = Built(rs3, U=2, H=16, d=d, dtype="bf16", m=64, n=64, window=-1, ring_frames=4, commits=4, n_ptr=0, seed=2)
    else:
        b = Built(rs3, U=2, H=1, d=d, dtype="bf16", m=8, n=9, window=4, commits=5, n_ptr=0, seed=2)
    spoil(b, None)
    bias = biases(b, "age")
    q, idx, count, group, table, out, ws = scored_case(rs3, b, [2000, 1100] if pairs else [30, 9], [0, 0], 1, 6.0, bias)
    limit = rs3.rs3_get_wait_limit_ns()
    again = torch.zeros_like(out)
    try:
        rs3.rs3_set_wait_limit_ns(0)
        run_scored(rs3, b, q, 1, idx, count, group, 6.0, bias, None, None, 0.0, None, again, ws)
        code = int(b.st)
    finally:
        rs3.rs3_set_wait_limit_ns(limit)
    assert code == rs3.RS3_ETIMEOUT
    b.st.zero_()
    again.zero_()
    run_scored(rs3, b, q, 1, idx, count, group, 6.0, bias, None, None, 0.0, None, again, ws)
    assert int(b.st) == 0 and (again != 0).any()
    on = torch.zeros_like(again, dtype=torch.bool)
    for u in range(2):
        on[u, idx[u, :int(count[u])].long()] = True
    assert torch.equal(bits(again)[on], bits(out)[on])
