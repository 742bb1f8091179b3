"""What the speed of a memory-attention layer's other operators is measured on, from one 32 x 32
fp32 grid to 300 000 keys and 48 objects.

Kinds of case:
  scored   per frame: the pruned readout with capped scores, a bias by the age of a key's frame, and
           frames left out (rs3_scored_readout)
  shared   per frame, while hypotheses of a track are open: the readout of units that share the rows
           of the bank that they were forked from (rs3_shared_readout)
  rope     per frame: query and key heads turned by the frame, row and column of their cells (rs3_rope_rows)
  block    between two blocks of a layer: the norm behind the first with its gate and residual scale, and
           the norm before the second (rs3_norm_residual)

Inputs are drawn on the GPU from the seed.  A group's cells carry a smooth random field, and its
queries and the keys of every frame are that field with noise, so that a query finds its like at its
own place in every frame, as a tracker's does.  An object is the given number of cells nearest to a
moving centre: how many rows a bank holds depends on the case alone.
"""
import math

import torch

own = False

DTYPE = {"f32": torch.float32, "bf16": torch.bfloat16}


# ---------------------------------------------------------------------------
# the cases
# ---------------------------------------------------------------------------
def _bank(G, per, m, n, H, d, dtype, n_cond, window, frames, n_ptr, lo, hi, rho):
    """frames: ring frames committed; window < 0: a bank that keeps all of them."""
    return dict(G=G, per=per, m=m, n=n, H=H, d=d, dtype=dtype, n_cond=n_cond, window=window, frames=frames, n_ptr=n_ptr, lo=lo, hi=hi,
                rho=rho)


def listed():
    return [
        # The fp32 configuration: one head of 64 on a 32 x 32 grid, two frames; latency.
        dict(name="scored_tiny_fp32", kind="scored", cap=30.0, bias="age", keep="all", rope=False, residual="inplace",
             **_bank(1, 1, 32, 32, 1, 64, "f32", 0, 2, 2, 0, 0.3, 0.9, 0.3)),
        # Eight objects on one grid, seven frames each: capped scores, older frames weigh less.
        dict(name="scored_8obj", kind="scored", cap=50.0, bias="age", keep="all", rope=False, residual="inplace",
             **_bank(1, 8, 64, 64, 1, 256, "bf16", 1, 6, 8, 0, 0.02, 0.40, 0.3)),
        # A long video after a cut: of 490 frames those of the present shot and the conditioning frame.
        dict(name="scored_long_cut", kind="scored", cap=0.0, bias="age", keep="cut", rope=False, residual="inplace",
             **_bank(1, 1, 64, 64, 1, 256, "bf16", 1, -1, 490, 0, 0.14, 0.16, 0.3)),
        # Serving: 16 streams of 3 objects on 96 x 96 grids, four heads of 64, learned biases, every unit its own frames.
        dict(name="scored_16x3", kind="scored", cap=20.0, bias="unit", keep="some", rope=True, residual="other",
             **_bank(16, 3, 96, 96, 4, 64, "bf16", 1, 6, 8, 16, 0.03, 0.25, 0.3)),
        # Three hypotheses of an fp32 track; latency.
        dict(name="shared_tiny_fp32", kind="shared", prefix=4, lone=False, rope=False, residual="none",
             **_bank(1, 3, 32, 32, 1, 64, "f32", 0, 3, 3, 0, 0.1, 0.3, 0.3)),
        # Eight hypotheses that branched after 490 frames and have six frames of their own.
        dict(name="shared_8hyp_long", kind="shared", prefix=490, lone=False, rope=False, residual="inplace",
             **_bank(1, 8, 64, 64, 1, 256, "bf16", 0, 6, 6, 0, 0.14, 0.16, 0.3)),
        # Four streams of four hypotheses in four heads, some tracks new; 60 frames behind the branch.
        dict(name="shared_4x4", kind="shared", prefix=60, lone=True, rope=True, residual="other",
             **_bank(4, 4, 64, 64, 4, 64, "bf16", 1, 6, 7, 16, 0.05, 0.25, 0.3)),
        # The heads of the fp32 configuration's grid; latency.
        dict(name="rope_tiny_fp32", kind="rope", G=1, per=1, m=32, n=32, Hq=1, Hk=1, d=64, dtype="f32", layout="pairs", rot=64, axes=2,
             stretch=1.0, context=0, time=3, masked=False, lo=0.1, hi=0.1),
        # Queries of 16 streams and keys of their 48 objects, far into a video, three quarters of each head turned by three axes.
        dict(name="rope_16x3", kind="rope", G=16, per=3, m=96, n=96, Hq=4, Hk=4, d=64, dtype="bf16", layout="halves", rot=48, axes=3,
             stretch=8.0, context=64, time=90000, masked=True, lo=0.2, hi=0.6),
        # One object's kept cells between two blocks; latency.
        dict(name="block_1obj", kind="block", U=1, m=64, n=64, C=256, dtype="bf16", post="rms", pre="rms", gate="shared", alpha=1.0,
             kept=0.3, inplace=True),
        # Serving: every cell of 16 streams, gates and norms given by the stream, mean and variance.
        dict(name="block_16", kind="block", U=16, m=96, n=96, C=256, dtype="bf16", post="none", pre="layer", gate="unit", alpha=1.0,
             kept=1.0, inplace=False),
        # Wide rows in fp32.
        dict(name="block_wide_fp32", kind="block", U=4, m=64, n=64, C=1024, dtype="f32", post="layer", pre="rms", gate="shared", alpha=0.5,
             kept=0.5, inplace=False),
    ]


def _log(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


HEADS = {"bf16": [(1, 256), (1, 256), (4, 64), (2, 128), (8, 64), (1, 64), (2, 32)], "f32": [(1, 64), (4, 64), (2, 32), (2, 128), (1, 256)]}


def draw(rng):
    """A case of the listed kinds, anywhere in their ranges, odd sizes among them."""
    bounds = {}
    for c in listed():
        w = work(c)
        b = bounds.setdefault(c["kind"], [0.0, 0.0])
        b[0], b[1] = max(b[0], w["bytes"]), max(b[1], w["flops"])
    while True:
        kind = rng.choice(["scored", "scored", "scored", "shared", "shared", "shared", "rope", "block"])
        G, m, n = _log(rng, 1, 16), _log(rng, 8, 112), _log(rng, 8, 112)
        per = _log(rng, 1, 8)
        dtype = "bf16" if rng.random() < 0.7 else "f32"
        H, d = rng.choice(HEADS[dtype])
        lo = rng.choice([0.02, 0.05, 0.14])
        hi = rng.choice([0.16, 0.25, 0.40])
        if kind == "rope":
            axes = rng.choice([1, 2, 3])
            d = rng.choice([d, 80, 96])
            c = dict(kind=kind, G=G, per=per, m=m, n=n, Hq=rng.choice([H, 2 * H]), Hk=H, d=d, dtype=dtype,
                     layout=rng.choice(["pairs", "halves"]), rot=2 * rng.randint(axes, d // 2), axes=axes,
                     stretch=rng.choice([1.0, 2.0, 8.0, 32.0]), context=rng.choice([0, 64, 4096]), time=_log(rng, 1, 200000),
                     masked=rng.random() < 0.5, lo=lo, hi=hi)
        elif kind == "block":
            c = dict(kind=kind, U=G * per, m=m, n=n, C=8 * _log(rng, 1, 256), dtype=dtype, post=rng.choice(["none", "rms", "layer"]),
                     pre=rng.choice(["rms", "layer"]), gate=rng.choice(["none", "shared", "unit"]), alpha=rng.choice([1.0, 0.5, 0.7071]),
                     kept=rng.choice([0.002, 0.03, 0.3, 1.0]), inplace=rng.random() < 0.5)
        else:
            window = rng.choice([3, 6, 6, -1, -1])
            c = dict(kind=kind, rope=rng.random() < 0.3, residual=rng.choice(["inplace", "inplace", "none", "other"]),
                     **_bank(min(G, 4), per, m, n, H, d, dtype, rng.choice([0, 1, 1, 2]), window,
                             rng.randint(1, 10) if window > 0 else _log(rng, 2, 200), rng.choice([0, 4, 16, 61]), lo, hi,
                             rng.choice([0.002, 0.02, 0.1, 0.3])))
            if kind == "scored":
                c.update(cap=rng.choice([0.0, 10.0, 30.0, 50.0]), bias=rng.choice(["none", "age", "age", "unit"]),
                         keep=rng.choice(["all", "cut", "some", "nothing"]))
            else:
                c.update(prefix=_log(rng, 1, 300), lone=rng.random() < 0.3)
            # banks of a state, in bytes; half as much again while it is made
            rows = c["G"] * (per * _rows(c)[3] + (_rows(_prefix_case(c))[3] if kind == "shared" else 0))
            if rows * H * d * (2 if dtype == "bf16" else 4) > 6e8:
                continue
        w, b = work(c), bounds[kind]
        # no more than the largest listed case; fp32 attention runs on the CUDA cores
        if w["bytes"] > b[0] or w["flops"] > (b[1] if dtype == "bf16" or kind in ("rope", "block") else b[1] / 16):
            continue
        return c


# ---------------------------------------------------------------------------
# sizes, which depend on the case alone
# ---------------------------------------------------------------------------
def _cells(c, u, frame):
    """Cells of unit u's object in a frame."""
    mn = c["m"] * c["n"]
    return min(mn, int(mn * (c["lo"] + (c["hi"] - c["lo"]) * (0.5 + 0.5 * math.sin(1.7 * u + 0.35 * frame + 0.9)))))


def _rows(c):
    """(pinned capacity, ring capacity, ring frames that a table holds, rows per unit)."""
    mn = c["m"] * c["n"]
    ring = c["window"] * mn if c["window"] > 0 else c["frames"] * (int(math.ceil(c["hi"] * mn)) + 1) + 5
    table = c["window"] if c["window"] > 0 else c["frames"] + 1
    return c["n_cond"] * mn, ring, table, c["n_cond"] * mn + ring + c["n_ptr"]


def _units(c):
    return c["G"] * c["per"]


def _prefix_case(c):
    """The bank that a shared case's hypotheses branched from: one unit per group."""
    return dict(c, per=1, n_cond=1, window=-1, frames=c["prefix"], n_ptr=0)


def _prefix_of(c):
    """The prefix unit of every unit; `lone`: every fifth has none."""
    return [-1 if c["lone"] and u % 5 == 4 else u // c["per"] for u in range(_units(c))]


def _kmax(c):
    return max(1, int(math.floor(c["rho"] * c["m"] * c["n"])))


def _queries(c, u):
    """Kept queries of unit u: a fifth more than its object's cells, at most rho of the grid."""
    return min(_kmax(c), int(1.2 * _cells(c, u, c["frames"])) + 3)


def _lengths(c, u):
    """(pinned frames, ring frames held, oldest first, ring rows gone before them) of unit u."""
    cond = [_cells(c, u, f) for f in range(c["n_cond"])]
    ring = [_cells(c, u, c["n_cond"] + f) for f in range(c["frames"])]
    kept = ring[-c["window"]:] if c["window"] > 0 else ring
    return cond, kept, sum(ring) - sum(kept)


def _held(c):
    """Ring frames held by every unit."""
    return min(c["frames"], c["window"]) if c["window"] > 0 else c["frames"]


def _read_frames(c, u):
    """Which ages, then the conditioning frames and the pointers, unit u of a scored case reads."""
    F, held = _rows(c)[2], _held(c)
    keep = [True] * (F + 2)
    if c["keep"] == "cut":                     # the shot began two fifths into the video
        keep = [a < held - int(0.4 * held) or a >= F for a in range(F + 2)]
    elif c["keep"] == "some":
        keep = [(7 * a + 5 * u) % 4 != 1 for a in range(F + 2)]
    elif c["keep"] == "nothing" and u % 3 == 0:
        keep = [False] * (F + 2)
    return keep


def _read_rows(c, u):
    cond, ring, _ = _lengths(c, u)
    keep, F = _read_frames(c, u), _rows(c)[2]
    return (sum(cond) if keep[F] else 0) + sum(x for a, x in enumerate(reversed(ring)) if keep[a]) + (c["n_ptr"] if keep[F + 1] else 0)


def _length(c, u):
    cond, ring, _ = _lengths(c, u)
    return sum(cond) + sum(ring) + c["n_ptr"]


def work(case):
    c = dict(case)
    es = 2 if c["dtype"] == "bf16" else 4
    mn = c["m"] * c["n"]
    if c["kind"] == "rope":
        k_rows = sum(_cells(c, u, 0) for u in range(_units(c))) if c["masked"] else _units(c) * mn
        heads, rows = c["G"] * mn * c["Hq"] + k_rows * c["Hk"], c["G"] * mn + k_rows
        return {"bytes": 2 * heads * c["d"] * es + rows * c["axes"] * 4 + (_units(c) * mn if c["masked"] else 0),
                "flops": 3 * heads * c["rot"] + 20 * rows * c["rot"]}
    if c["kind"] == "block":
        rows = c["U"] * max(1, int(c["kept"] * mn))
        return {"bytes": 4 * rows * c["C"] * es, "flops": 12 * rows * c["C"]}
    U, D = _units(c), c["H"] * c["d"]
    nq = [_queries(c, u) for u in range(U)]
    grid = (2 if c["residual"] != "none" else 1) * D * es
    by, fl = sum(q * D * es + grid * (q if c["residual"] == "inplace" else mn) for q in nq), 0
    for u in range(U):
        n = _read_rows(c, u) if c["kind"] == "scored" else _length(c, u)
        by += 2 * n * D * es
        fl += 4 * nq[u] * n * D
    if c["kind"] == "shared":
        p, of = _prefix_case(c), _prefix_of(c)
        for g in range(c["G"]):
            # the hypotheses of a group keep much the same cells: at least those of the one that keeps most
            users = [nq[u] for u in range(U) if of[u] == g]
            if users:
                by += 2 * _length(p, g) * D * es
                fl += 4 * max(users) * _length(p, g) * D
    return {"bytes": int(by), "flops": int(fl)}


# ---------------------------------------------------------------------------
# inputs
# ---------------------------------------------------------------------------
class _Gen:
    """Draws from (seed, tag): any part of a case's inputs can be drawn again on its own."""

    def __init__(self, seed):
        self.seed = int(seed)

    def __call__(self, *tag):
        x = self.seed & 0x7FFFFFFF
        for t in tag:
            x = (x * 1000003 + int(t) + 12345) % ((1 << 61) - 1)
        g = torch.Generator(device="cuda")
        g.manual_seed(x)
        return g


def _field(g, c, D):
    """[G, mn, D]: a smooth field over the cells, unit variance or so."""
    m, n = c["m"], c["n"]
    low = torch.randn((c["G"], D, m // 6 + 2, n // 6 + 2), generator=g(1), device="cuda")
    f = torch.nn.functional.interpolate(low, size=(m, n), mode="bilinear", align_corners=True)
    return f.permute(0, 2, 3, 1).reshape(c["G"], m * n, D) * 1.4


def _near(g, c, frame, counts):
    """[U, most]: each unit's cells in the order of their distance to the object's centre, the first counts[u] of them its own."""
    U, m, n = _units(c), c["m"], c["n"]
    r = torch.rand((U, 4), generator=g(2), device="cuda")
    t = 0.05 * frame
    # (the hypotheses of a track differ by a few cells)
    r = r.view(c["G"], c["per"], 4)
    r = (r[:, :1] + 0.02 * r).reshape(U, 4) if c["kind"] == "shared" else r.reshape(U, 4)
    cy, cx = (0.5 + 0.25 * torch.sin(t + 6.3 * r[:, 0])) * m, (0.5 + 0.25 * torch.cos(t + 6.3 * r[:, 1])) * n
    y = torch.arange(m, device="cuda")[None, :, None] - cy[:, None, None]
    x = torch.arange(n, device="cuda")[None, None, :] - cx[:, None, None]
    dist = (y * y + (0.5 + r[:, 2])[:, None, None] * x * x).reshape(U, -1)
    return dist.topk(max(1, max(counts)), dim=1, largest=False).indices


def _mask(g, c, frame):
    """uint8 [U, mn]: exactly _cells(c, u, frame) cells of unit u."""
    counts = [_cells(c, u, frame) for u in range(_units(c))]
    near = _near(g, c, frame, counts)
    mine = torch.arange(near.shape[1], device="cuda")[None] < torch.tensor(counts, device="cuda")[:, None]
    return torch.zeros((_units(c), c["m"] * c["n"]), dtype=torch.uint8, device="cuda").scatter_(1, near, mine.to(torch.uint8))


def _table(c):
    """[mn, d/2, 2] (cos, sin): half of the pairs turn with the column, half with the row."""
    m, n, half = c["m"], c["n"], c["d"] // 4
    cell = torch.arange(m * n, device="cuda", dtype=torch.float64)
    freq = 10000.0 ** (-torch.arange(half, device="cuda", dtype=torch.float64) / half)
    ang = torch.cat([(cell % n)[:, None] * freq, (cell // n)[:, None] * freq], 1)
    return torch.stack([ang.cos(), ang.sin()], -1).float().contiguous()


class _Store:
    """The rows of a set of banks where the framework keeps them: pinned frames, the ring, pointers."""

    def __init__(self, g, c, field, tag):
        dt, U, mn, D = DTYPE[c["dtype"]], _units(c), c["m"] * c["n"], c["H"] * c["d"]
        pinned_cap, ring_cap, self.table, rows = _rows(c)
        self.k = torch.zeros((U, rows, D), dtype=dt, device="cuda")
        self.v = torch.zeros_like(self.k)
        self.bank = None
        if own:
            from paper_2608_22526_gb300 import rs3
            status = torch.zeros(1, dtype=torch.int32, device="cuda")
            self.bank = rs3.Bank(U, c["H"], c["d"], c["dtype"], mn, c["n_cond"], c["window"], ring_cap, self.table, c["n_ptr"])
        lengths = [_lengths(c, u) for u in range(U)]
        self.cond = torch.tensor([sum(x[0]) for x in lengths], device="cuda")
        self.frames = torch.tensor([x[1] for x in lengths], device="cuda").view(U, -1)        # held, oldest first
        self.head = torch.tensor([x[2] for x in lengths], device="cuda")
        self.pinned_cap, self.ring_cap, self.n_ptr = pinned_cap, ring_cap, c["n_ptr"]
        self.most = max(_length(c, u) for u in range(U))
        at = torch.zeros((U, 2), dtype=torch.int64, device="cuda")
        unit = torch.arange(U, device="cuda")[:, None]
        for f in range(c["n_cond"] + c["frames"]):
            k = torch.randn((U, mn, D), generator=g(3, tag, f), device="cuda").mul_(0.7)
            k = k.view(c["G"], c["per"], mn, D).add_(field[:, None]).view(U, mn, D).to(dt)
            v = torch.randn((U, mn, D), generator=g(4, tag, f), device="cuda").to(dt)
            mask, cond = _mask(g, c, f), f < c["n_cond"]
            if own:
                rs3.rs3_bank_commit(self.bank, k, v, mask, int(cond), status)
            cells = [_cells(c, u, f) for u in range(U)]
            n = torch.tensor(cells, device="cuda")
            order = mask.to(torch.int16).argsort(dim=1, descending=True, stable=True)[:, :max(1, max(cells))]
            r = torch.arange(order.shape[1], device="cuda")[None]
            place = at[:, 0 if cond else 1, None] + r
            place = place if cond else pinned_cap + place % max(1, ring_cap)
            here = r < n[:, None]
            uu, pp, oo = unit.expand_as(here)[here], place.expand_as(here)[here], order[here]
            self.k[uu, pp], self.v[uu, pp] = k[uu, oo], v[uu, oo]
            at[:, 0 if cond else 1] += n
        if c["n_ptr"]:
            kv = [torch.randn((U, c["n_ptr"], D), generator=g(5, tag, i), device="cuda").to(dt) for i in range(2)]
            self.k[:, rows - c["n_ptr"]:], self.v[:, rows - c["n_ptr"]:] = kv
            if own:
                rs3.rs3_bank_set_pointers(self.bank, *kv, status)

    def rows(self):
        """Of every unit, padded to the longest: storage rows in logical order, whether there is one, and the frame
        that it is of (0: the newest ring frame, `table`: conditioning frames, `table` + 1: pointers)."""
        r = torch.arange(self.most, device="cuda")[None]
        upto = self.frames.cumsum(1)
        live = upto[:, -1:] if upto.shape[1] else torch.zeros_like(self.cond)[:, None]
        ring = r - self.cond[:, None]
        ptr = ring - live
        place = torch.where(ring < 0, r, torch.where(ptr < 0, self.pinned_cap + (self.head[:, None] + ring) % max(1, self.ring_cap),
                                                     self.pinned_cap + self.ring_cap + ptr))
        age = upto.shape[1] - 1 - torch.searchsorted(upto, ring.contiguous(), right=True)
        slot = torch.where(ring < 0, self.table, torch.where(ptr < 0, age, self.table + 1))
        there = ptr < self.n_ptr
        return torch.where(there, place, 0), there, torch.where(there, slot, 0)


def _prepare_read(c, seed):
    g = _Gen(seed)
    U, mn, k_max, D, H = _units(c), c["m"] * c["n"], _kmax(c), c["H"] * c["d"], c["H"]
    field = _field(g, c, D)
    s = _Store(g, c, field, 0)
    q = ((field + 0.7 * torch.randn(field.shape, generator=g(6), device="cuda")) * 0.35).to(DTYPE[c["dtype"]]).contiguous()
    counts = [_queries(c, u) for u in range(U)]
    near = _near(g, c, c["frames"], counts)
    count = torch.tensor(counts, dtype=torch.int32, device="cuda")
    mine = torch.arange(near.shape[1], device="cuda")[None] < count[:, None]
    cells = torch.where(mine, near, mn).sort(1).values
    idx = torch.zeros((U, k_max), dtype=torch.int32, device="cuda")
    idx[:, :cells.shape[1]] = torch.where(cells < mn, cells, 0).to(torch.int32)
    st = dict(c=c, s=s, q=q, idx=idx, count=count, rope=_table(c) if c["rope"] else None, most=max(counts),
              unit_group=torch.arange(c["G"], dtype=torch.int32, device="cuda").repeat_interleave(c["per"]),
              status=torch.zeros(1, dtype=torch.int32, device="cuda"), bias=None, keep=None, res=None, x0=None)
    if c["residual"] != "none":
        st["res"] = torch.randn((U, mn, D), generator=g(9), device="cuda").to(DTYPE[c["dtype"]])
    if c["residual"] == "inplace":
        st["x0"] = st["res"].clone()
    st["out"] = st["res"] if c["residual"] == "inplace" else torch.zeros((U, mn, D), dtype=DTYPE[c["dtype"]], device="cuda")
    if c["kind"] == "scored":
        F = s.table
        if c["bias"] == "age":                                  # a slope for each head, as ages grow
            age = torch.arange(F + 2, device="cuda").clamp(max=F).float()
            age[F:] = 0.0
            st["bias"] = -age[None] * torch.tensor([2.0 ** (-8.0 * (h + 1) / H) for h in range(H)], device="cuda")[:, None]
        elif c["bias"] == "unit":
            st["bias"] = torch.randn((U, H, F + 2), generator=g(10), device="cuda")
        if c["keep"] != "all":
            st["keep"] = torch.tensor([_read_frames(c, u) for u in range(U)], device="cuda").to(torch.uint8)
    else:
        st["prefix"] = _Store(g, _prefix_case(c), field, 1)
        st["prefix_unit"] = torch.tensor(_prefix_of(c), dtype=torch.int32, device="cuda")
    if own:
        from paper_2608_22526_gb300 import rs3
        n = rs3.rs3_scored_readout_workspace_bytes(s.bank, k_max) if c["kind"] == "scored" else \
            rs3.rs3_shared_readout_workspace_bytes(s.bank, st["prefix"].bank, k_max)
        st["ws"] = torch.empty(n, dtype=torch.uint8, device="cuda")
    return st


# ---------------------------------------------------------------------------
# readouts
# ---------------------------------------------------------------------------
def _turned(x, H, table):
    """Pairs (2p, 2p + 1) of every head of x [G, mn, D] turned by their cell's angles."""
    p = x.reshape(*x.shape[:-1], H, -1, 2)
    co, si = table[:, None, :, 0], table[:, None, :, 1]
    return torch.stack([p[..., 0] * co - p[..., 1] * si, p[..., 0] * si + p[..., 1] * co], -1).reshape(x.shape)


def _attend(st, k, v, there, slot):
    """out = residual + softmax(scores) V at the kept cells; k, v [U, rows, D], there [U, rows]."""
    c = st["c"]
    U, mn, H, d = _units(c), c["m"] * c["n"], c["H"], c["d"]
    q = st["q"].float()
    if st["rope"] is not None:
        q = _turned(q, H, st["rope"])
    cells = st["idx"][:, :st["most"]].long()
    row = q[st["unit_group"].long()[:, None], cells]                     # [U, queries, D]
    parts = []
    for h in range(H):
        cols = slice(h * d, (h + 1) * d)
        x = (row[..., cols] @ k[..., cols].float().transpose(1, 2)) / math.sqrt(d)
        if c.get("cap", 0.0) > 0:
            x = c["cap"] * torch.tanh(x / c["cap"])
        if st["bias"] is not None:
            b = st["bias"][..., h, :].expand(U, -1).gather(1, slot)
            x = x + b[:, None]
        x = torch.where(there[:, None], x, -math.inf)
        top = x.amax(2, keepdim=True)
        p = torch.exp(x - torch.where(top > -math.inf, top, 0.0))
        total = p.sum(2, keepdim=True)
        parts.append((p @ v[..., cols].float()) / torch.where(total > 0, total, 1.0))
    o = torch.cat(parts, 2)
    res = st["x0"] if st["x0"] is not None else st["res"]
    out = torch.zeros_like(st["out"]) if res is None else res.clone()
    unit = torch.arange(U, device="cuda")[:, None].expand_as(cells)
    mine = torch.arange(st["most"], device="cuda")[None] < st["count"][:, None]
    at = (unit[mine], cells[mine])
    out[at] = (o[mine] if res is None else res[at].float() + o[mine]).to(out.dtype)
    return out


def _run_scored(st):
    c, s = st["c"], st["s"]
    if own:
        from paper_2608_22526_gb300 import rs3
        if st["x0"] is not None:
            st["out"].copy_(st["x0"])                                    # a frame's new residual, which the call adds to in place
        rs3.rs3_scored_readout(st["q"], c["dtype"], c["G"], c["m"] * c["n"], c["H"], c["d"], st["unit_group"], st["idx"], st["count"],
                               st["idx"].shape[1], s.bank, c["cap"], st["bias"], st["keep"], st["rope"], st["res"], st["out"], 0.0,
                               st["ws"], st["status"])
        return st["out"]
    place, there, slot = s.rows()
    if st["keep"] is not None:
        there = there & (st["keep"].gather(1, slot) != 0)
    unit = torch.arange(_units(c), device="cuda")[:, None]
    return _attend(st, s.k[unit, place], s.v[unit, place], there, slot)


def _run_shared(st):
    c, s, p = st["c"], st["s"], st["prefix"]
    if own:
        from paper_2608_22526_gb300 import rs3
        if st["x0"] is not None:
            st["out"].copy_(st["x0"])
        rs3.rs3_shared_readout(st["q"], c["dtype"], c["G"], c["m"] * c["n"], c["H"], c["d"], st["unit_group"], st["idx"], st["count"],
                               st["idx"].shape[1], s.bank, p.bank, st["prefix_unit"], st["rope"], st["res"], st["out"], 0.0, st["ws"],
                               st["status"])
        return st["out"]
    place, there, _ = s.rows()
    unit = torch.arange(_units(c), device="cuda")[:, None]
    of = st["prefix_unit"].long()
    place_p, there_p, _ = p.rows()
    back = of.clamp(min=0)
    there_p = there_p[back] & (of >= 0)[:, None]
    k = torch.cat([p.k[back[:, None], place_p[back]], s.k[unit, place]], 1)
    v = torch.cat([p.v[back[:, None], place_p[back]], s.v[unit, place]], 1)
    return _attend(st, k, v, torch.cat([there_p, there], 1), None)


# ---------------------------------------------------------------------------
# rotary positions
# ---------------------------------------------------------------------------
BASE, FAST, SLOW = 10000.0, 32.0, 1.0


def _split(c):
    """Pairs of each axis: as even as they go, the first axes one more."""
    half, a = c["rot"] // 2, c["axes"]
    return [half // a + (i < half % a) for i in range(a)]


def _positions(c, units):
    """int32 [units, mn, axes]: one number per cell of the video, (row, column), or (frame, row, column)."""
    m, n, t = c["m"], c["n"], c["time"]
    cell = torch.arange(m * n, device="cuda")
    y, x = cell // n, cell % n
    p = {1: [t * m * n % 2 ** 30 + cell], 2: [y, x], 3: [torch.full_like(y, t), y, x]}[c["axes"]]
    return torch.stack(p, -1).to(torch.int32)[None].repeat(units, 1, 1).contiguous()


def _prepare_rope(c, seed):
    g, mn = _Gen(seed), c["m"] * c["n"]
    dt, U, G = DTYPE[c["dtype"]], _units(c), c["G"]
    q = torch.randn((G, mn, c["Hq"] * c["d"]), generator=g(1), device="cuda").mul_(1.5).to(dt)
    k = torch.randn((U, mn, c["Hk"] * c["d"]), generator=g(2), device="cuda").to(dt)
    st = dict(c=c, q=q, k=k, q_pos=_positions(c, G), k_pos=_positions(c, U), keep=_mask(g, c, 0) if c["masked"] else None,
              q_out=torch.zeros_like(q), k_out=torch.zeros_like(k))
    if own:
        from paper_2608_22526_gb300 import rs3
        st["spec"] = rs3.rope_spec(layout=c["layout"], rot=c["rot"], pairs=_split(c), base=BASE, factor=c["stretch"],
                                   context=float(c["context"]), beta_fast=FAST, beta_slow=SLOW)
    return st


def _frequencies(c):
    """Radians per position of each pair, in 64 bits: with a context, the pairs that turn seldom in it are slowed."""
    f = torch.cat([BASE ** (-torch.arange(n, device="cuda", dtype=torch.float64) / n) for n in _split(c)])
    if c["context"] == 0:
        return f / c["stretch"]
    share = ((c["context"] * f / (2 * math.pi) - SLOW) / (FAST - SLOW)).clamp(0, 1)
    return f * (share + (1 - share) / c["stretch"])


def _rotate(c, x, pos, freq, H):
    axis = torch.repeat_interleave(torch.arange(c["axes"], device="cuda"), torch.tensor(_split(c), device="cuda"))
    ang = pos.double()[..., axis] * freq
    co, si = ang.cos().float()[..., None, :], ang.sin().float()[..., None, :]
    h = x.float().unflatten(-1, (H, c["d"]))
    turn, rest = h[..., :c["rot"]], h[..., c["rot"]:]
    if c["layout"] == "pairs":
        a, b = turn[..., 0::2], turn[..., 1::2]
        turn = torch.stack([a * co - b * si, a * si + b * co], -1).flatten(-2)
    else:
        a, b = turn[..., :c["rot"] // 2], turn[..., c["rot"] // 2:]
        turn = torch.cat([a * co - b * si, a * si + b * co], -1)
    return torch.cat([turn, rest], -1).flatten(-2).to(x.dtype)


def _run_rope(st):
    c = st["c"]
    if own:
        from paper_2608_22526_gb300 import rs3
        rs3.rs3_rope_rows(st["q"], st["q_out"], st["q_pos"], st["k"], st["k_out"], st["k_pos"], c["dtype"], c["Hq"], c["Hk"], c["d"],
                          st["spec"], k_keep=st["keep"])
        return st["q_out"], st["k_out"]
    freq = _frequencies(c)
    k = _rotate(c, st["k"], st["k_pos"], freq, c["Hk"])
    if st["keep"] is not None:
        k = torch.where(st["keep"][..., None] != 0, k, st["k_out"])
    return _rotate(c, st["q"], st["q_pos"], freq, c["Hq"]), k


# ---------------------------------------------------------------------------
# norms around a block
# ---------------------------------------------------------------------------
EPS = 1e-6


def _prepare_block(c, seed):
    g, U, mn, C = _Gen(seed), c["U"], c["m"] * c["n"], c["C"]
    dt = DTYPE[c["dtype"]]
    y = torch.randn((U, mn, C), generator=g(1), device="cuda").mul_(0.8).to(dt)
    x = torch.randn((U, mn, C), generator=g(2), device="cuda").mul_(2.0).add_(0.3).to(dt)
    kept = max(1, int(c["kept"] * mn))
    idx = count = None
    if c["kept"] < 1:
        idx = torch.rand((U, mn), generator=g(3), device="cuda").topk(kept, dim=1).indices.sort(1).values.to(torch.int32)
        count = torch.full((U,), kept, dtype=torch.int32, device="cuda")

    def vector(tag, centre, per_unit):
        return centre + 0.2 * torch.randn((U, C) if per_unit else (C,), generator=g(4, tag), device="cuda")

    unit = c["gate"] == "unit"
    st = dict(c=c, y=y, x=x, idx=idx, count=count, x0=x.clone() if c["inplace"] else None,
              gate=None if c["gate"] == "none" else vector(1, 0.5, unit), post_w=None if c["post"] == "none" else vector(2, 1.0, False),
              post_b=vector(3, 0.0, False) if c["post"] == "layer" else None, pre_w=vector(4, 1.0, unit),
              pre_b=vector(5, 0.0, unit) if c["pre"] == "layer" else None, x_out=x if c["inplace"] else torch.zeros_like(x),
              h_out=torch.zeros_like(x), status=torch.zeros(1, dtype=torch.int32, device="cuda"))
    return st


def _normed(kind, v, w, b):
    if kind == "layer":
        v = v - v.mean(-1, keepdim=True)
    if kind != "none":
        v = v / torch.sqrt((v * v).mean(-1, keepdim=True) + EPS)
    w, b = (t if t is None or t.dim() == 1 else t[:, None] for t in (w, b))
    v = v if w is None else v * w
    return v if b is None else v + b


def _run_block(st):
    c = st["c"]
    if own:
        from paper_2608_22526_gb300 import rs3
        if c["inplace"]:
            st["x"].copy_(st["x0"])                                      # a frame's new rows, which the call adds to in place
        rs3.rs3_norm_residual(st["y"], st["x"], st["x_out"], st["h_out"], c["dtype"], idx=st["idx"], count=st["count"],
                              post=c["post"], post_weight=st["post_w"], post_bias=st["post_b"], gate=st["gate"], alpha=c["alpha"],
                              pre=c["pre"], pre_weight=st["pre_w"], pre_bias=st["pre_b"], eps=EPS, status=st["status"])
        return st["x_out"], st["h_out"]
    x0 = st["x0"] if c["inplace"] else st["x"]
    t = _normed(c["post"], st["y"].float(), st["post_w"], st["post_b"])
    gate = st["gate"]
    if gate is not None:
        t = t * (gate if gate.dim() == 1 else gate[:, None])
    x = c["alpha"] * x0.float() + t
    h = _normed(c["pre"], x, st["pre_w"], st["pre_b"]).to(x0.dtype)
    x = x.to(x0.dtype)
    if st["idx"] is not None:
        on = torch.zeros(x.shape[:2], dtype=torch.bool, device="cuda").scatter_(1, st["idx"].long(), True)[..., None]
        x = torch.where(on, x, x0 if c["inplace"] else 0.0)
        h = torch.where(on, h, 0.0)
    return x, h


# ---------------------------------------------------------------------------
# the module's entry points
# ---------------------------------------------------------------------------
PREPARE = {"scored": _prepare_read, "shared": _prepare_read, "rope": _prepare_rope, "block": _prepare_block}
RUN = {"scored": _run_scored, "shared": _run_shared, "rope": _run_rope, "block": _run_block}


def prepare(case, seed):
    return PREPARE[case["kind"]](dict(case), seed)


def run(state):
    return RUN[state["c"]["kind"]](state)


# ---------------------------------------------------------------------------
# in 64 bits, from the definitions
# ---------------------------------------------------------------------------
def exact(case, seed):
    c = dict(case)
    st = prepare(c, seed)
    return {"scored": _exact_read, "shared": _exact_read, "rope": _exact_rope, "block": _exact_block}[c["kind"]](st)


def _exact_rows(c, s, u):
    """Unit u's rows, frame after frame: (keys, values, the frame of each) in 64 bits."""
    cond, ring, gone = _lengths(c, u)
    at = list(range(sum(cond)))
    slot = [s.table] * len(at)
    for i, n in enumerate(ring):
        at += [s.pinned_cap + (gone + j) % s.ring_cap for j in range(n)]
        slot += [len(ring) - 1 - i] * n
        gone += n
    at += [s.pinned_cap + s.ring_cap + j for j in range(c["n_ptr"])]
    slot += [s.table + 1] * c["n_ptr"]
    at = torch.tensor(at, dtype=torch.int64, device="cuda")
    return s.k[u].index_select(0, at), s.v[u].index_select(0, at), torch.tensor(slot, dtype=torch.int64, device="cuda")


def _exact_read(st):
    """Weights exp(score - largest) one unit and head after another, some queries at a time."""
    c, s = st["c"], st["s"]
    mn, H, d = c["m"] * c["n"], c["H"], c["d"]
    res = st["x0"] if st["x0"] is not None else st["res"]
    out = torch.zeros(st["out"].shape, dtype=torch.float64, device="cuda") if res is None else res.double()
    for u, n in enumerate(_queries(c, u) for u in range(_units(c))):
        k, v, slot = _exact_rows(c, s, u)
        if c["kind"] == "scored" and st["keep"] is not None:
            on = st["keep"][u][slot].bool()
            k, v, slot = k[on], v[on], slot[on]
        if c["kind"] == "shared" and _prefix_of(c)[u] >= 0:
            kp, vp, _ = _exact_rows(_prefix_case(c), st["prefix"], _prefix_of(c)[u])
            k, v = torch.cat([k, kp]), torch.cat([v, vp])
        if k.shape[0] == 0:
            continue
        cells = st["idx"][u, :n].long()
        q = st["q"][u // c["per"], cells].double().view(n, H, d)
        if st["rope"] is not None:
            z = torch.view_as_complex(q.reshape(n, H, d // 2, 2).contiguous())
            q = torch.view_as_real(z * torch.view_as_complex(st["rope"].double())[cells][:, None]).reshape(n, H, d)
        step = max(1, int(2e8 // k.shape[0]))
        for h in range(H):
            kh, vh = k[:, h * d:(h + 1) * d].double(), v[:, h * d:(h + 1) * d].double()
            b = 0.0
            if st["bias"] is not None:
                b = (st["bias"][u, h] if st["bias"].dim() == 3 else st["bias"][h]).double()[slot]
            for a in range(0, n, step):
                x = torch.einsum("qd,kd->qk", q[a:a + step, h], kh) * d ** -0.5
                if c.get("cap", 0.0) > 0:
                    e = torch.exp(-2.0 * x.abs() / c["cap"])
                    x = torch.sign(x) * c["cap"] * (1.0 - e) / (1.0 + e)
                w = torch.softmax(x + b, 1)
                out[u, cells[a:a + step], h * d:(h + 1) * d] += w @ vh
    return out


def _exact_rope(st):
    c = st["c"]
    freq, sizes, outs = [], _split(c), []
    for size in sizes:
        for p in range(size):
            f = math.exp(-math.log(BASE) * p / size)
            turns = c["context"] * f / (2 * math.pi)
            share = 0.0 if c["context"] == 0 else min(1.0, max(0.0, (turns - SLOW) / (FAST - SLOW)))
            freq.append(share * f + (1.0 - share) * f / c["stretch"])
    for side, H in (("q", c["Hq"]), ("k", c["Hk"])):
        x, pos = st[side].double(), st[side + "_pos"]
        y = x.clone().unflatten(-1, (H, c["d"]))
        x = x.unflatten(-1, (H, c["d"]))
        p = 0
        for axis, size in enumerate(sizes):
            for _ in range(size):
                i, j = (2 * p, 2 * p + 1) if c["layout"] == "pairs" else (p, p + c["rot"] // 2)
                z = torch.complex(x[..., i], x[..., j])
                t = pos[..., axis].double() * freq[p]
                z = z * torch.polar(torch.ones_like(t), t)[..., None]
                y[..., i], y[..., j] = z.real, z.imag
                p += 1
        y = y.flatten(-2)
        if side == "k" and st["keep"] is not None:
            y[st["keep"] == 0] = 0.0
        outs.append(y)
    return tuple(outs)


def _exact_block(st):
    c = st["c"]
    x0 = (st["x0"] if c["inplace"] else st["x"]).double()
    xs, hs = torch.zeros_like(x0), torch.zeros_like(x0)
    if c["inplace"]:
        xs.copy_(x0)
    for u in range(c["U"]):
        cells = torch.arange(x0.shape[1], device="cuda") if st["idx"] is None else st["idx"][u].long()

        def of(t):
            return None if t is None else (t if t.dim() == 1 else t[u]).double()

        def norm(kind, v, w, b):
            if kind == "layer":
                var, mean = torch.var_mean(v, 1, unbiased=False, keepdim=True)
                v = (v - mean) * (var + EPS) ** -0.5
            elif kind == "rms":
                v = v * (v.square().sum(1, keepdim=True) / v.shape[1] + EPS) ** -0.5
            return v * (1.0 if w is None else w) + (0.0 if b is None else b)

        t = norm(c["post"], st["y"][u, cells].double(), of(st["post_w"]), of(st["post_b"]))
        gate = of(st["gate"])
        x = c["alpha"] * x0[u, cells] + (t if gate is None else gate * t)
        xs[u, cells] = x
        hs[u, cells] = norm(c["pre"], x, of(st["pre_w"]), of(st["pre_b"]))
    return xs, hs
