"""What the speed of the operators for long memory banks is measured on: the calls
that a program with banks of hundreds of frames makes beside selection, readout and
commit, from one 32 x 32 fp32 grid to 300 000 keys.

Kinds of case:
  norm     per frame: RMS norm of every query and key head with the position rotation
           in the same pass (rs3_qk_norm_rope)
  copy     when hypotheses branch or a bank is pruned: units of one bank copied, forked
           and compacted into another, its oldest frames freed (rs3_bank_copy,
           rs3_bank_drop_frames)
  digest   per frame: the 8-bit mean key of each block of a bank's rows, of the blocks
           that the last frames touched or of all (rs3_bank_digest)
  select   per frame: the blocks whose digests score highest for each kept query and
           head (rs3_block_select)
  attend   per frame: attention of each kept query over its own blocks, scattered back
           (rs3_sparse_readout)
  read     the last two as a frame makes them

Inputs are drawn on the GPU from the seed.  A group's cells carry a smooth random field,
and its queries and the keys of every frame are that field with noise, so that a query
finds its like at its own place in every frame, as a tracker's does.  An object is the
given number of cells nearest to a moving centre: how many rows a bank holds depends on
the case alone.
"""
import math

import torch

own = False

DTYPE = {"f32": torch.float32, "bf16": torch.bfloat16}
EPS = 1e-6
TINY = 2.0 ** -100                      # a vector whose largest element is below this is quantised to zeros


# ---------------------------------------------------------------------------
# the cases
# ---------------------------------------------------------------------------
def _bank(G, per, m, n, H, d, dtype, n_cond, window, frames, n_ptr, lo, hi, empty=False):
    """frames: ring frames committed; window < 0: a bank that keeps all of them."""
    return dict(G=G, per=per, m=m, n=n, H=H, d=d, dtype=dtype, n_cond=n_cond, window=window, frames=frames, n_ptr=n_ptr, lo=lo, hi=hi,
                empty=empty)


def listed():
    # SAM2 with banks that are never pruned by age: one object, one head of 256, 490 frames
    long = _bank(1, 1, 64, 64, 1, 256, "bf16", 1, -1, 490, 0, 0.14, 0.16)
    # eight objects on one grid, four heads of 64, 99 frames: some 60 000 keys each
    objs = _bank(1, 8, 64, 64, 4, 64, "bf16", 1, -1, 98, 16, 0.05, 0.25)
    return [
        # The fp32 configuration's frame: one head of 64 on a 32 x 32 grid; latency.
        dict(name="norm_tiny_fp32", kind="norm", G=1, per=1, m=32, n=32, Hq=1, Hk=1, d=64, dtype="f32", rope=True, weight=True,
             masked=False, packed=False, lo=0.1, hi=0.1),
        # Serving: queries of 16 streams and keys of their 48 objects on 96 x 96 grids; only
        # the cells that will be committed have their keys normed.
        dict(name="norm_16x3", kind="norm", G=16, per=3, m=96, n=96, Hq=4, Hk=4, d=64, dtype="bf16", rope=True, weight=True,
             masked=True, packed=False, lo=0.2, hi=0.6),
        # Hypotheses branch: eight units of seven frames, the window wrapped; four parents
        # have two children each, whose oldest frame is freed.
        dict(name="copy_fork_8", kind="copy", mode="fork", drop=1, keep=1.0,
             **_bank(1, 8, 64, 64, 1, 256, "bf16", 1, 6, 9, 16, 0.02, 0.40)),
        # A long bank is pruned to half of its rows.
        dict(name="copy_compact_long", kind="copy", mode="compact", drop=0, keep=0.5, **long),
        # Every frame of a long video: the blocks of the newest frame.
        dict(name="digest_newest", kind="digest", block=64, refresh=1, **long),
        # After a branch: all blocks of eight banks.
        dict(name="digest_all", kind="digest", block=64, refresh=-1, **objs),
        # The blocks of each query: one head, 757 queries over 4 700 blocks.
        dict(name="select_long", kind="select", block=64, top=32, rho=0.3, rope=False, **long),
        # 8 x 4 heads, about 940 blocks each.
        dict(name="select_8obj", kind="select", block=64, top=16, rho=0.3, rope=True, **objs),
        # Attention over 32 of 4 700 blocks.
        dict(name="attend_long", kind="attend", block=64, top=32, rho=0.3, rope=False, residual="inplace", **long),
        # Attention over 16 of 940 blocks, in every head.
        dict(name="attend_8obj", kind="attend", block=64, top=16, rho=0.3, rope=True, residual="other", **objs),
        # A small object far away: a dozen queries, both calls; latency.
        dict(name="read_few", kind="read", block=64, top=16, rho=0.003, rope=False, residual="inplace",
             **_bank(1, 1, 64, 64, 4, 64, "bf16", 1, -1, 60, 4, 0.02, 0.05)),
        # fp32 networks: 300 queries of two heads of 64.
        dict(name="read_fp32", kind="read", block=32, top=12, rho=0.3, rope=True, residual="none",
             **_bank(1, 1, 32, 32, 2, 64, "f32", 1, -1, 60, 0, 0.10, 0.30)),
    ]


def _log(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


HEADS = {"bf16": [(1, 256), (4, 64), (2, 128), (8, 64), (1, 64), (2, 32)], "f32": [(1, 64), (4, 64), (2, 32), (2, 128), (1, 256)]}


def draw(rng):
    """A case of the listed kinds, anywhere in their ranges, odd sizes among them."""
    bounds = {}
    for c in listed():
        w = work(c)
        b = bounds.setdefault(c["kind"], [0.0, 0.0])
        b[0], b[1] = max(b[0], w["bytes"]), max(b[1], w["flops"])
    bounds["read"] = [bounds["attend"][0], bounds["attend"][1] / 4]
    while True:
        kind = rng.choice(["norm", "copy", "copy", "digest", "select", "select", "attend", "attend", "attend", "read"])
        G, m, n = _log(rng, 1, 16), _log(rng, 8, 112), _log(rng, 8, 112)
        per = _log(rng, 1, 8)
        dtype = "bf16" if rng.random() < 0.7 else "f32"
        H, d = rng.choice(HEADS[dtype])
        if kind == "norm":
            lo = rng.choice([0.02, 0.1, 0.3])
            packed = rng.random() < 0.3
            c = dict(kind=kind, G=G, per=1 if packed else per, m=m, n=n, Hq=H if rng.random() < 0.7 else 2 * H, Hk=H,
                     d=rng.choice([d, d, 80, 96]), dtype=dtype, rope=rng.random() < 0.8, weight=rng.random() < 0.8,
                     masked=rng.random() < 0.4, packed=packed, lo=lo, hi=min(1.0, lo * rng.choice([1, 2, 3])))
        else:
            window = rng.choice([3, 6, -1, -1, -1])
            lo = rng.choice([0.02, 0.05, 0.14])
            c = dict(kind=kind, **_bank(min(G, 4), per, m, n, H, d, dtype, rng.choice([0, 1, 1, 2]), window,
                                        rng.randint(1, 10) if window > 0 else _log(rng, 4, 300), rng.choice([0, 4, 16, 61]),
                                        lo, rng.choice([0.16, 0.25, 0.40]), rng.random() < 0.15))
            if kind == "copy":
                c.update(mode=rng.choice(["fork", "compact", "grow"]), drop=rng.choice([0, 1, 2]), keep=rng.choice([0.1, 0.5, 0.9]))
            else:
                c.update(block=rng.choice([32, 64, 64, 128]))
                if kind == "digest":
                    c.update(refresh=rng.choice([0, 1, 1, 2, -1]))
                else:
                    c.update(top=_log(rng, 1, 48), rho=rng.choice([0.002, 0.02, 0.1, 0.3]), rope=rng.random() < 0.4)
                    if kind != "select":
                        c.update(residual=rng.choice(["inplace", "inplace", "none", "other"]))
            # two banks of a state, in bytes; half as much again while it is made
            if c["G"] * per * _rows(c)[3] * H * d * (2 if dtype == "bf16" else 4) > 6e8:
                continue
        w, b = work(c), bounds[kind]
        # no more than the largest listed case; fp32 runs on the CUDA cores
        if w["bytes"] > b[0] or w["flops"] > (b[1] if dtype == "bf16" else b[1] / 8):
            continue
        return c


# ---------------------------------------------------------------------------
# sizes, which depend on the case alone
# ---------------------------------------------------------------------------
def _cells(c, u, frame):
    """Cells of unit u's object in a frame; `empty`: the first unit never had one."""
    if c.get("empty") and u == 0:
        return 0
    mn = c["m"] * c["n"]
    return min(mn, int(mn * (c["lo"] + (c["hi"] - c["lo"]) * (0.5 + 0.5 * math.sin(1.7 * u + 0.35 * frame + 0.9)))))


def _rows(c):
    """(pinned capacity, ring capacity, ring frames that a table holds, rows per unit)."""
    mn = c["m"] * c["n"]
    ring = c["window"] * mn if c["window"] > 0 else c["frames"] * (int(math.ceil(c["hi"] * mn)) + 1) + 5
    table = c["window"] if c["window"] > 0 else c["frames"] + 1
    return c["n_cond"] * mn, ring, table, c["n_cond"] * mn + ring + c["n_ptr"]


class _Counts:
    """A unit's counters, as the bank's commits leave them."""

    def __init__(self, c, u):
        self.pinned_cap, self.ring_cap, self.table, self.rows = _rows(c)
        self.n_ptr = c["n_ptr"]
        self.cond = [_cells(c, u, f) for f in range(c["n_cond"])]
        self.lens = [_cells(c, u, c["n_cond"] + f) for f in range(c["frames"])]
        kept = self.lens[-c["window"]:] if c["window"] > 0 else self.lens
        self.tail = sum(self.lens)
        self.head = self.tail - sum(kept)
        self.frames = kept
        self.oldest = (len(self.lens) - len(kept)) % self.table
        self.live = self.tail - self.head
        self.length = sum(self.cond) + self.live + self.n_ptr

    def counters(self):
        return [self.head, self.tail, sum(self.cond), len(self.frames), self.oldest, len(self.cond), self.n_ptr]

    def places(self):
        """Storage rows in logical order: pinned, ring (oldest first), pointers."""
        r = torch.arange(self.length, device="cuda")
        ring = r - sum(self.cond)
        ptr = ring - self.live
        return torch.where(ring < 0, r, torch.where(ptr < 0, self.pinned_cap + (self.head + ring) % max(1, self.ring_cap),
                                                    self.pinned_cap + self.ring_cap + ptr))

    def alive(self):
        a = torch.zeros(self.rows, dtype=torch.bool, device="cuda")
        a[self.places()] = True
        return a


def _units(c):
    return c["G"] * c["per"]


def _queries(c, u):
    """Kept queries of unit u: a fifth more than its object's cells, at most rho of the grid."""
    mn = c["m"] * c["n"]
    return min(int(math.floor(c["rho"] * mn)), int(1.2 * _cells(c, u, c["frames"])) + 3)


def _kmax(c):
    return max(1, int(math.floor(c["rho"] * c["m"] * c["n"])))


def _blocks(c):
    return -(-_rows(c)[3] // c["block"])


def work(case):
    c = dict(case)
    es = 2 if c["dtype"] == "bf16" else 4
    mn, U = c["m"] * c["n"], _units(c)
    if c["kind"] == "norm":
        k_rows = sum(_cells(c, u, 0) for u in range(U)) if c["masked"] else U * mn
        heads = c["G"] * mn * c["Hq"] + k_rows * c["Hk"]
        return {"bytes": 2 * heads * c["d"] * es + (mn * c["d"] * 4 if c["rope"] else 0) + (U * mn if c["masked"] else 0),
                "flops": 10 * heads * c["d"]}
    n = [_Counts(c, u) for u in range(U)]
    D = c["H"] * c["d"]
    if c["kind"] == "copy":
        parents = _parents(c)
        share = c["keep"] if c["mode"] == "compact" else 1.0
        read = (sum(n[p].length for p in set(parents)) if c["mode"] == "fork" else sum(n[p].length for p in parents)) * share
        write = sum(n[p].length for p in parents) * share
        return {"bytes": (read + write) * 2 * D * es + (sum(n[p].length for p in parents) if c["mode"] == "compact" else 0), "flops": 0}
    nb, bs = _blocks(c), c["block"]
    if c["kind"] == "digest":
        rows = sum(x.length if c["refresh"] < 0 else min(x.length, sum(x.frames[len(x.frames) - c["refresh"]:]) + 4 * bs) for x in n)
        return {"bytes": rows * D * es + rows / bs * c["H"] * (c["d"] + 4), "flops": rows * D}
    nq = [_queries(c, u) for u in range(U)]
    kept = [-(-x.length // bs) for x in n]
    out = {"bytes": 0, "flops": 0}
    if c["kind"] in ("select", "read"):
        out["bytes"] += sum(q * D * es + k * c["H"] * (c["d"] + 4) + q * c["H"] * c["top"] * 4 for q, k in zip(nq, kept))
        out["flops"] += sum(2 * q * k * D for q, k in zip(nq, kept))
    if c["kind"] in ("attend", "read"):
        for q, k, x in zip(nq, kept, n):
            top = min(c["top"], k)
            # neighbouring queries choose much the same blocks: about a quarter of those that independent choices would touch
            touched = max(top, 0.25 * k * (1 - (1 - top / k) ** q)) if k else 0
            out["bytes"] += 2 * touched * min(bs, x.length / max(1, k)) * D * es + q * D * es + q * c["H"] * top * 4
            out["bytes"] += (2 if c["residual"] != "none" else 1) * (q if c["residual"] == "inplace" else mn) * D * es
            out["flops"] += 4 * q * top * min(bs, x.length / max(1, k)) * D
    return {k: int(v) for k, v in out.items()}


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


def _near(g, c, frame, counts, tag):
    """[U, most]: each unit's cells in the order of their distance to the object's centre, the first counts[u] of them its own."""
    U, m, n = _units(c), c["m"], c["n"]
    r = torch.rand((U, 4), generator=g(2), device="cuda")
    t = 0.05 * frame
    cy, cx = (0.5 + 0.25 * torch.sin(t + 6.3 * r[:, 0])) * m, (0.5 + 0.25 * torch.cos(t + 6.3 * r[:, 1])) * n
    y = torch.arange(m, device="cuda")[None, :, None] - cy[:, None, None]
    x = torch.arange(n, device="cuda")[None, None, :] - cx[:, None, None]
    dist = (y * y + (0.5 + r[:, 2])[:, None, None] * x * x).reshape(U, -1)
    return dist.topk(max(1, max(counts)), dim=1, largest=False).indices


def _mask(g, c, frame):
    """uint8 [U, mn]: exactly _cells(c, u, frame) cells of unit u."""
    counts = [_cells(c, u, frame) for u in range(_units(c))]
    near = _near(g, c, frame, counts, 0)
    own_cells = torch.arange(near.shape[1], device="cuda")[None] < torch.tensor(counts, device="cuda")[:, None]
    return torch.zeros((_units(c), c["m"] * c["n"]), dtype=torch.uint8, device="cuda").scatter_(1, near, own_cells.to(torch.uint8))


def _rope(c):
    """[mn, d/2, 2] (cos, sin): half of the pairs turn with the column, half with the row."""
    m, n, half = c["m"], c["n"], c["d"] // 4
    cell = torch.arange(m * n, device="cuda", dtype=torch.float64)
    freq = 10000.0 ** (-torch.arange(half, device="cuda", dtype=torch.float64) / half)
    ang = torch.cat([(cell % n)[:, None] * freq, (cell // n)[:, None] * freq], 1)
    return torch.stack([ang.cos(), ang.sin()], -1).float().contiguous()


def _turn(x, H, table):
    """Pairs (2p, 2p + 1) of every head of x [..., mn, D] turned by their cell's angles; each product and sum rounded."""
    p = x.reshape(*x.shape[:-1], H, -1, 2)
    co, si = table[:, None, :, 0], table[:, None, :, 1]
    return torch.stack([p[..., 0] * co - p[..., 1] * si, p[..., 0] * si + p[..., 1] * co], -1).reshape(x.shape)


def _unit_group(c):
    return torch.arange(c["G"], dtype=torch.int32, device="cuda").repeat_interleave(c["per"])


def _frame_kv(g, c, frame, field, table):
    """Keys and values [U, mn, D] of a frame, as committed."""
    shape = (_units(c), c["m"] * c["n"], c["H"] * c["d"])
    k = torch.randn(shape, generator=g(3, frame), device="cuda").mul_(0.7)
    k = k.view(c["G"], c["per"], *shape[1:]).add_(field[:, None]).view(shape)
    if table is not None:
        k = _turn(k, c["H"], table)
    return k.to(DTYPE[c["dtype"]]), torch.randn(shape, generator=g(4, frame), device="cuda").to(DTYPE[c["dtype"]])


def _pointers(g, c):
    shape = (_units(c), c["n_ptr"], c["H"] * c["d"])
    return tuple(torch.randn(shape, generator=g(5, i), device="cuda").to(DTYPE[c["dtype"]]) for i in range(2))


class _Store:
    """The rows of a set of banks where the framework keeps them: pinned frames, ring, pointers."""

    def __init__(self, c):
        self.c, self.n = c, [_Counts(c, u) for u in range(_units(c))]
        self.k = torch.zeros((_units(c), self.n[0].rows, c["H"] * c["d"]), dtype=DTYPE[c["dtype"]], device="cuda")
        self.v = torch.zeros_like(self.k)
        self.bank = None


def _fill(g, c, field, table=None):
    """The case's banks after all of their frames."""
    s = _Store(c)
    pinned_cap, ring_cap, table_len, rows = _rows(c)
    if own:
        from paper_2608_22526_gb300 import rs3
        status = torch.zeros(1, dtype=torch.int32, device="cuda")
        s.bank = rs3.Bank(_units(c), c["H"], c["d"], c["dtype"], c["m"] * c["n"], c["n_cond"], c["window"], ring_cap, table_len, c["n_ptr"])
        for f in range(c["n_cond"] + c["frames"]):
            k, v = _frame_kv(g, c, f, field, table)
            rs3.rs3_bank_commit(s.bank, k, v, _mask(g, c, f), int(f < c["n_cond"]), status)
        if c["n_ptr"]:
            rs3.rs3_bank_set_pointers(s.bank, *_pointers(g, c), status)
        s.k, s.v = s.bank.k_store, s.bank.v_store
        return s
    at = [[0, 0] for _ in s.n]
    for f in range(c["n_cond"] + c["frames"]):
        k, v = _frame_kv(g, c, f, field, table)
        order = _mask(g, c, f).to(torch.int16).argsort(dim=1, descending=True, stable=True)
        for u, x in enumerate(s.n):
            L = _cells(c, u, f)
            cond = f < c["n_cond"]
            start = at[u][0 if cond else 1]
            at[u][0 if cond else 1] += L
            place = torch.arange(start, start + L, device="cuda")
            place = place if cond else pinned_cap + place % max(1, ring_cap)
            s.k[u, place], s.v[u, place] = k[u, order[u, :L]], v[u, order[u, :L]]
    if c["n_ptr"]:
        s.k[:, pinned_cap + ring_cap:], s.v[:, pinned_cap + ring_cap:] = _pointers(g, c)
    return s


def _read_inputs(g, c, field):
    """Query grid, kept cells and their numbers."""
    U, mn, k_max = _units(c), c["m"] * c["n"], _kmax(c)
    q = ((field + 0.7 * torch.randn(field.shape, generator=g(6), device="cuda")) * 0.35).to(DTYPE[c["dtype"]])
    counts = [_queries(c, u) for u in range(U)]
    near = _near(g, c, c["frames"], counts, 1)
    mine = torch.arange(near.shape[1], device="cuda")[None] < torch.tensor(counts, device="cuda")[:, None]
    cells = torch.where(mine, near, mn).sort(1).values
    idx = torch.zeros((U, k_max), dtype=torch.int32, device="cuda")
    idx[:, :cells.shape[1]] = torch.where(cells < mn, cells, 0).to(torch.int32)[:, :k_max]
    return q.contiguous(), idx, torch.tensor(counts, dtype=torch.int32, device="cuda"), counts


# ---------------------------------------------------------------------------
# norm and rotation
# ---------------------------------------------------------------------------
def _prepare_norm(c, seed):
    g, mn, U, G = _Gen(seed), c["m"] * c["n"], _units(c), c["G"]
    dt, Dq, Dk = DTYPE[c["dtype"]], c["Hq"] * c["d"], c["Hk"] * c["d"]
    if c["packed"]:                               # one projection's output: queries, keys and values side by side
        x = torch.randn((G, mn, Dq + 2 * Dk), generator=g(1), device="cuda").to(dt)
        q, k = x[..., :Dq], x[..., Dq:Dq + Dk]
    else:
        q = torch.randn((G, mn, Dq), generator=g(1), device="cuda").mul_(1.5).to(dt)
        k = torch.randn((U, mn, Dk), generator=g(2), device="cuda").to(dt)
    w = [1.0 + 0.2 * torch.randn(c["d"], generator=g(3, i), device="cuda") if c["weight"] else None for i in range(2)]
    keep = None
    if c["masked"]:
        keep = _mask(g, c, 0)
    return dict(c=c, q=q, k=k, q_weight=w[0], k_weight=w[1], k_keep=keep, rope=_rope(c) if c["rope"] else None,
                q_out=torch.zeros((G, mn, Dq), dtype=dt, device="cuda"), k_out=torch.zeros((U, mn, Dk), dtype=dt, device="cuda"))


def _normed(x, d, weight, table):
    y = x.float()
    h = y.reshape(*y.shape[:-1], -1, d)
    h = h / torch.sqrt((h * h).mean(-1, keepdim=True) + EPS)
    if weight is not None:
        h = h * weight
    if table is not None:
        h = _turn(h.reshape(y.shape), h.shape[-2], table)
    return h.reshape(y.shape).to(x.dtype)


def _run_norm(s):
    c = s["c"]
    if own:
        from paper_2608_22526_gb300 import rs3
        rs3.rs3_qk_norm_rope(s["q"], s["q_out"], s["k"], s["k_out"], c["dtype"], c["m"] * c["n"], c["Hq"], c["Hk"], c["d"], s["q_weight"],
                             s["k_weight"], EPS, s["rope"], k_keep=s["k_keep"])
        return s["q_out"], s["k_out"]
    k = _normed(s["k"], c["d"], s["k_weight"], s["rope"])
    if s["k_keep"] is not None:
        k = torch.where(s["k_keep"][..., None] != 0, k, s["k_out"])
    return _normed(s["q"], c["d"], s["q_weight"], s["rope"]), k


# ---------------------------------------------------------------------------
# copying, forking and compacting banks
# ---------------------------------------------------------------------------
def _parents(c):
    """fork: every other unit's rows go to two units; else each unit keeps its own."""
    U = _units(c)
    return [(u // 2 * 3 + 1) % U for u in range(U)] if c["mode"] == "fork" else list(range(U))


def _target(c):
    """The destination's layout: `grow` has room for as many frames again."""
    if c["mode"] == "grow" and c["window"] < 0:
        return dict(c, frames=2 * c["frames"] + 2)
    return c


def _prepare_copy(c, seed):
    g = _Gen(seed)
    s = _fill(g, c, _field(g, c, c["H"] * c["d"]))
    t = _target(c)
    keep = None
    if c["mode"] == "compact":
        longest = max(x.length for x in s.n)
        keep = (torch.rand((_units(c), max(1, longest)), generator=g(7), device="cuda") < c["keep"]).to(torch.uint8)
    st = dict(c=c, s=s, keep=keep, parent=torch.tensor(_parents(c), dtype=torch.int32, device="cuda"), rows=_rows(t))
    # frames that the children free: no more than any of them holds
    drop = min([c["drop"]] + [len(x.frames) for x in s.n])
    st["drop"] = torch.full((_units(c),), drop, dtype=torch.int32, device="cuda")
    st["n_drop"] = drop
    if own:
        from paper_2608_22526_gb300 import rs3
        st["dst"] = rs3.Bank(_units(c), c["H"], c["d"], c["dtype"], c["m"] * c["n"], c["n_cond"], c["window"], _rows(t)[1], _rows(t)[2],
                             c["n_ptr"])
        st["ws"] = torch.empty(rs3.rs3_bank_copy_workspace_bytes(_units(c), 0 if keep is None else keep.shape[1]), dtype=torch.uint8,
                               device="cuda")
        st["status"] = torch.zeros(1, dtype=torch.int32, device="cuda")
    else:
        st["dk"] = torch.zeros((_units(c), _rows(t)[3] + 1, c["H"] * c["d"]), dtype=DTYPE[c["dtype"]], device="cuda")
        st["dv"] = torch.zeros_like(st["dk"])
    return st


def _run_copy(st):
    c, s = st["c"], st["s"]
    if own:
        from paper_2608_22526_gb300 import rs3
        rs3.rs3_bank_copy(st["dst"], s.bank, st["parent"], st["keep"], st["ws"], st["status"])
        if st["n_drop"]:
            rs3.rs3_bank_drop_frames(st["dst"], st["drop"], None, st["status"])
        return st["dst"].k_store, st["dst"].v_store, st["dst"].counters
    pinned_cap, ring_cap, table, rows = st["rows"]
    counters = []
    for u, p in enumerate(_parents(c)):
        x, src = s.n[p], s.n[p].places()
        r = torch.arange(x.length, device="cuda")
        n_cond = sum(x.cond)
        kept = torch.ones(x.length, dtype=torch.bool, device="cuda") if st["keep"] is None else st["keep"][u, :x.length] != 0
        upto = torch.cat([torch.zeros(1, dtype=torch.int64, device="cuda"), kept.long().cumsum(0)])
        c_kept, r_kept = upto[n_cond], upto[n_cond + x.live]
        place = torch.where(r < n_cond, upto[:-1], torch.where(r < n_cond + x.live, pinned_cap + upto[:-1] - c_kept,
                                                               pinned_cap + ring_cap + upto[:-1] - r_kept))
        place = torch.where(kept, place, rows)                       # rows that go: a row behind the storage
        st["dk"][u].index_copy_(0, place, s.k[p].index_select(0, src))
        st["dv"][u].index_copy_(0, place, s.v[p].index_select(0, src))
        # the first `drop` frames leave: the ring's head moves past their kept rows
        d = st["n_drop"]
        head = upto[n_cond + sum(x.frames[:d])] - c_kept
        tail, ptr = r_kept - c_kept, upto[-1] - r_kept
        whole = torch.tensor([len(x.frames) - d, d % table, len(x.cond)], device="cuda")
        counters.append(torch.cat([torch.stack([head, tail, c_kept]), whole, ptr[None]]))
    return st["dk"][:, :rows], st["dv"][:, :rows], torch.stack(counters)


# ---------------------------------------------------------------------------
# digests
# ---------------------------------------------------------------------------
def _eight_bits(x):
    """x [..., d] in 8 bits with a power of two for each vector: whole numbers of at most
    127 in size, and what one of them stands for."""
    a = x.abs().amax(-1, keepdim=True)
    e = torch.frexp(a)[1] - 1                                        # floor(log2 a)
    up = ((133 - e).to(torch.int32) << 23).view(torch.float32)       # 2^(6 - e)
    step = ((121 + e).to(torch.int32) << 23).view(torch.float32)     # 2^(e - 6)
    t = torch.where(a >= TINY, (x * up).round().clamp(-127, 127), 0.0)
    return t, torch.where(a >= TINY, step, 0.0)[..., 0]


def _digest_of(c, k, alive, n_live):
    """Digests [nb, H, d] (whole numbers) and steps [nb, H] of one unit's rows k [nb * bs, D]:
    eight partial sums of every eighth row, then (0 + 4), (1 + 5), ... of those."""
    bs, H, d = c["block"], c["H"], c["d"]
    x = torch.where(alive[:, None], k, torch.zeros((), dtype=k.dtype, device="cuda")).float().view(-1, bs // 8, 8, H, d)
    a = x[:, 0]
    for i in range(1, bs // 8):
        a = a + x[:, i]
    a = a[:, :4] + a[:, 4:]
    a = a[:, :2] + a[:, 2:]
    a = a[:, 0] + a[:, 1]
    return _eight_bits(a / n_live.clamp(min=1).float()[:, None, None])


def _padded(c, s, u):
    """Unit u's keys, which of its rows live, and how many of each block."""
    rows, total = s.n[u].rows, _blocks(c) * c["block"]
    alive = torch.zeros(total, dtype=torch.bool, device="cuda")
    alive[:rows] = s.n[u].alive()
    k = torch.cat([s.k[u], torch.zeros((total - rows, s.k.shape[-1]), dtype=s.k.dtype, device="cuda")])
    return k, alive, alive.view(-1, c["block"]).sum(1)


def _digests(c, s):
    """int8 [U, H, nb, d] and float [U, H, nb] of every block."""
    t, step = zip(*[_digest_of(c, *_padded(c, s, u)) for u in range(_units(c))])
    return torch.stack(t).permute(0, 2, 1, 3).to(torch.int8).contiguous(), torch.stack(step).permute(0, 2, 1).contiguous()


def _touched(c, x):
    """Blocks that a refresh of the newest frames visits: theirs, and those of the ring's oldest and newest rows and of its two ends."""
    if c["refresh"] < 0:
        return list(range(_blocks(c)))
    got = set()
    if x.ring_cap:
        ends = [x.pinned_cap, x.pinned_cap + x.ring_cap - 1]
        if x.live:
            ends += [x.pinned_cap + x.head % x.ring_cap, x.pinned_cap + (x.tail - 1) % x.ring_cap]
        got |= {r // c["block"] for r in ends}
        new = sum(x.frames[max(0, len(x.frames) - c["refresh"]):])
        a = (x.tail - new) % x.ring_cap
        for lo, hi in ((a, min(a + new, x.ring_cap)), (0, a + new - x.ring_cap)):
            if hi > lo:
                got |= set(range((x.pinned_cap + lo) // c["block"], (x.pinned_cap + hi - 1) // c["block"] + 1))
    return sorted(got)


def _prepare_digest(c, seed):
    g = _Gen(seed)
    s = _fill(g, c, _field(g, c, c["H"] * c["d"]))
    nb = _blocks(c)
    # what an earlier call left
    t = torch.randint(-127, 128, (_units(c), c["H"], nb, c["d"]), generator=g(8), device="cuda").to(torch.int8)
    st = dict(c=c, s=s, digest=t, step=torch.full((_units(c), c["H"], nb), 2.0 ** -7, device="cuda"))
    st["visit"] = [torch.tensor(_touched(c, x), dtype=torch.int64, device="cuda") for x in s.n]
    st["status"] = torch.zeros(1, dtype=torch.int32, device="cuda")
    return st


def _run_digest(st):
    c, s = st["c"], st["s"]
    if own:
        from paper_2608_22526_gb300 import rs3
        rs3.rs3_bank_digest(s.bank, c["block"], c["refresh"], st["digest"], st["step"], st["status"])
    else:
        for u in range(_units(c)):
            k, alive, n_live = _padded(c, s, u)
            if c["refresh"] >= 0:
                b = st["visit"][u]
                rows = (b[:, None] * c["block"] + torch.arange(c["block"], device="cuda")).view(-1)
                k, alive, n_live = k[rows], alive[rows], n_live[b]
            else:
                b = slice(None)
            t, step = _digest_of(c, k, alive, n_live)
            st["digest"][u][:, b], st["step"][u][:, b] = t.permute(1, 0, 2).to(torch.int8), step.permute(1, 0)
    # what the 8-bit values stand for
    return st["digest"].float() * st["step"][..., None], st["step"]


# ---------------------------------------------------------------------------
# block selection and the attention over the blocks
# ---------------------------------------------------------------------------
def _prepare_read(c, seed):
    g = _Gen(seed)
    field = _field(g, c, c["H"] * c["d"])
    table = _rope(c) if c["rope"] else None
    s = _fill(g, c, field, table)
    q, idx, count, counts = _read_inputs(g, c, field)
    U, mn, k_max, D = _units(c), c["m"] * c["n"], _kmax(c), c["H"] * c["d"]
    digest, step = _digests(c, s)
    st = dict(c=c, s=s, q=q, idx=idx, count=count, counts=counts, rope=table, digest=digest, step=step, unit_group=_unit_group(c),
              sel=torch.full((U, c["H"], k_max, c["top"]), -1, dtype=torch.int32, device="cuda"),
              status=torch.zeros(1, dtype=torch.int32, device="cuda"))
    if c["kind"] != "select":
        st["res"] = None
        if c["residual"] != "none":
            st["res"] = torch.randn((U, mn, D), generator=g(9), device="cuda").to(DTYPE[c["dtype"]])
        st["x0"] = st["res"].clone() if c["residual"] == "inplace" else None
        st["out"] = st["res"] if c["residual"] == "inplace" else torch.zeros((U, mn, D), dtype=DTYPE[c["dtype"]], device="cuda")
        st["cells"] = [idx[u, :n].long() for u, n in enumerate(counts)]
    if c["kind"] == "attend":
        st["sel"] = _select_plain(st)
    if own:
        from paper_2608_22526_gb300 import rs3
        nb, B = _blocks(c), s.bank
        if c["kind"] != "attend":
            st["ws_select"] = torch.empty(rs3.rs3_block_select_workspace_bytes(U, c["H"], k_max, nb), dtype=torch.uint8, device="cuda")
        if c["kind"] != "select":
            st["ws"] = torch.empty(rs3.rs3_sparse_readout_workspace_bytes(U, c["H"], c["d"], k_max, c["top"], nb, c["dtype"]),
                                   dtype=torch.uint8, device="cuda")
    return st


def _select_plain(st):
    """Scores are whole numbers times a power of two, exact in 32 bits; ties go to the lower block."""
    c, s = st["c"], st["s"]
    H, d, bs, nb = c["H"], c["d"], c["block"], _blocks(c)
    q = st["q"].float()
    if st["rope"] is not None:
        q = _turn(q, H, st["rope"])
    sel = st["sel"].clone()
    for u, n in enumerate(st["counts"]):
        if n == 0:
            continue
        _, _, n_live = _padded(c, s, u)
        k = min(c["top"], nb)
        row = q[u // c["per"]].index_select(0, st["idx"][u, :n].long()).view(n, H, d)
        t, _ = _eight_bits(row)
        for h in range(H):
            score = (t[:, h] @ st["digest"][u, h].float().T) * st["step"][u, h]
            score = torch.where(n_live > 0, score, -math.inf)
            val, b = score.sort(dim=1, descending=True, stable=True)
            b = torch.where(val[:, :k] > -math.inf, b[:, :k], nb).sort(1).values
            sel[u, h, :n, :k] = torch.where(b < nb, b, -1).to(torch.int32)
            sel[u, h, :n, k:] = -1
    return sel


def _attend_plain(st, sel):
    """out = residual + softmax(q K^T / sqrt d) V over the rows of each query's blocks."""
    c, s = st["c"], st["s"]
    H, d, bs, nb = c["H"], c["d"], c["block"], _blocks(c)
    q = st["q"].float()
    if st["rope"] is not None:
        q = _turn(q, H, st["rope"])
    res = st["x0"] if st["x0"] is not None else st["res"]
    out = torch.zeros_like(st["out"]) if res is None else res.clone()
    for u, n in enumerate(st["counts"]):
        if n == 0:
            continue
        rows, alive = s.n[u].rows, s.n[u].alive()
        cells = st["cells"][u]
        row = q[u // c["per"]].index_select(0, cells).view(n, H, d)
        o = torch.zeros((n, H, d), device="cuda")
        step = max(1, int(1e9 // (sel.shape[3] * bs * d * 8)))
        for h in range(H):
            K, V = s.k[u, :, h * d:(h + 1) * d], s.v[u, :, h * d:(h + 1) * d]
            for a in range(0, n, step):
                b = sel[u, h, a:min(n, a + step)].long()
                at = (b[..., None] * bs + torch.arange(bs, device="cuda")).view(b.shape[0], -1)
                ok = (b[..., None] >= 0).expand(-1, -1, bs).reshape(b.shape[0], -1) & (at < rows)
                at = at.clamp(0, rows - 1)
                ok &= alive[at]
                x = torch.einsum("qd,qkd->qk", row[a:a + step, h], K[at].float()) / math.sqrt(d)
                x = torch.where(ok, x, -math.inf)
                top = x.amax(1, keepdim=True)
                p = torch.where(ok, torch.exp(x - torch.where(top > -math.inf, top, 0.0)), 0.0)
                total = p.sum(1, keepdim=True)
                o[a:a + step, h] = torch.einsum("qk,qkd->qd", p / torch.where(total > 0, total, 1.0), V[at].float())
        o = o.view(n, H * d)
        out[u].index_copy_(0, cells, (o if res is None else o + res[u].index_select(0, cells).float()).to(out.dtype))
    return out


def _run_read(st):
    c, s = st["c"], st["s"]
    kind = c["kind"]
    if not own:
        sel = st["sel"] if kind == "attend" else _select_plain(st)
        if kind == "select":
            return sel
        out = _attend_plain(st, sel)
        return out if kind == "attend" else (sel, out)
    from paper_2608_22526_gb300 import rs3
    args = (st["q"], c["dtype"], c["G"], c["m"] * c["n"], c["H"], c["d"], st["unit_group"], st["idx"], st["count"], st["idx"].shape[1],
            s.bank, c["block"])
    if kind != "attend":
        rs3.rs3_block_select(*args, st["digest"], st["step"], st["rope"], c["top"], st["sel"], st["ws_select"], st["status"])
        if kind == "select":
            return st["sel"]
    if st["x0"] is not None:
        st["out"].copy_(st["x0"])                                    # a frame's new residual, which the call adds to in place
    rs3.rs3_sparse_readout(*args, st["sel"], c["top"], st["rope"], st["res"], st["out"], 0.0, st["ws"], st["status"])
    return st["out"] if kind == "attend" else (st["sel"], st["out"])


# ---------------------------------------------------------------------------
# the module's entry points
# ---------------------------------------------------------------------------
PREPARE = {"norm": _prepare_norm, "copy": _prepare_copy, "digest": _prepare_digest, "select": _prepare_read, "attend": _prepare_read,
           "read": _prepare_read}
RUN = {"norm": _run_norm, "copy": _run_copy, "digest": _run_digest, "select": _run_read, "attend": _run_read, "read": _run_read}


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
    if c["kind"] == "norm":
        return _exact_norm(st, "q"), _exact_norm(st, "k")
    if c["kind"] == "copy":
        return _exact_copy(st)
    if c["kind"] == "digest":
        return _exact_digest(st)
    if c["kind"] == "select":
        return _exact_select(st)
    if c["kind"] == "attend":
        return _exact_attend(st, st["sel"])
    sel = _exact_select(st)
    return sel, _exact_attend(st, sel)


def _exact_copy(st):
    """The rows themselves, one unit after another."""
    c, s, (pinned_cap, ring_cap, table, rows) = st["c"], st["s"], st["rows"]
    outs = [torch.zeros((_units(c), rows, c["H"] * c["d"]), dtype=torch.float64, device="cuda") for _ in range(2)]
    counters = []
    for u, p in enumerate(_parents(c)):
        x, n_cond = s.n[p], sum(s.n[p].cond)
        kept = st["keep"][u, :x.length].cpu().bool() if st["keep"] is not None else torch.ones(x.length, dtype=torch.bool)
        parts = [kept[:n_cond], kept[n_cond:n_cond + x.live], kept[n_cond + x.live:]]
        n = [int(t.sum()) for t in parts]
        for o, store in zip(outs, (s.k, s.v)):
            got = store[p][x.places()[kept.cuda()]].double()
            o[u, :n[0]] = got[:n[0]]
            o[u, pinned_cap:pinned_cap + n[1]] = got[n[0]:n[0] + n[1]]
            o[u, pinned_cap + ring_cap:pinned_cap + ring_cap + n[2]] = got[n[0] + n[1]:]
        head = int(parts[1][:sum(x.frames[:st["n_drop"]])].sum())
        counters.append([head, n[1], n[0], len(x.frames) - st["n_drop"], st["n_drop"] % table, len(x.cond), n[2]])
    return outs[0], outs[1], torch.tensor(counters)


def _exact_bits(x):
    """_eight_bits in 64 bits."""
    a = x.abs().amax(-1)
    e = torch.floor(torch.log2(a.clamp(min=TINY)))
    step = torch.where(a >= TINY, torch.exp2(e - 6), 0.0)
    return torch.where(step[..., None] > 0, x / torch.where(step > 0, step, 1.0)[..., None], 0.0).round().clamp(-127, 127), step


def _exact_digest(st):
    c, s, bs = st["c"], st["s"], st["c"]["block"]
    value, step = st["digest"].double() * st["step"].double()[..., None], st["step"].double()
    for u in range(_units(c)):
        place = s.n[u].places()
        k = s.k[u][place].double()
        total = torch.zeros((_blocks(c), k.shape[1]), dtype=torch.float64, device="cuda").index_add_(0, place // bs, k)
        n = torch.bincount(place // bs, minlength=_blocks(c)).clamp(min=1)
        t, e = _exact_bits((total / n[:, None]).view(-1, c["H"], c["d"]))
        b = st["visit"][u]
        value[u][:, b], step[u][:, b] = (t * e[..., None])[b].transpose(0, 1), e[b].transpose(0, 1)
    return value, step


def _exact_select(st):
    """The definition rounds the turned query to 32 bits product by product; from there on all is exact."""
    c, s, H, d = st["c"], st["s"], st["c"]["H"], st["c"]["d"]
    q = st["q"].double().unflatten(-1, (H, d // 2, 2))
    if st["rope"] is not None:
        co, si = st["rope"].double()[:, None, :, 0], st["rope"].double()[:, None, :, 1]
        products = [(q[..., i] * t).float().double() for i, t in ((0, co), (1, si), (0, si), (1, co))]
        q = torch.stack([(products[0] - products[1]).float().double(), (products[2] + products[3]).float().double()], -1)
    q = q.flatten(-2)
    sel = torch.where(torch.arange(st["sel"].shape[2], device="cuda")[None, None, :, None] < st["count"][:, None, None, None], -1, st["sel"])
    for u, n in enumerate(st["counts"]):
        lives = torch.unique(s.n[u].places() // c["block"])              # ascending
        k = min(c["top"], lives.numel())
        if n == 0 or k == 0:
            continue
        t, _ = _exact_bits(q[u // c["per"]][st["idx"][u, :n].long()])
        for h in range(H):
            score = (t[:, h] @ st["digest"][u, h][lives].double().T) * st["step"][u, h][lives].double()
            best = score.argsort(dim=1, descending=True, stable=True)[:, :k]
            sel[u, h, :n, :k] = lives[best.sort(dim=1).values].to(torch.int32)
    return sel


def _exact_norm(st, which):
    c, x = st["c"], st[which].double()
    d, w, table = c["d"], st[which + "_weight"], st["rope"]
    heads = x.unflatten(-1, (x.shape[-1] // d, d))
    heads = heads * (heads.square().sum(-1, keepdim=True) / d + EPS).rsqrt()
    if w is not None:
        heads = heads * w.double()
    if table is not None:
        turn = torch.view_as_complex(table.double().contiguous())[:, None]
        heads = torch.view_as_real(torch.view_as_complex(heads.unflatten(-1, (d // 2, 2)).contiguous()) * turn).flatten(-2)
    y = heads.flatten(-2)
    if which == "k" and st["k_keep"] is not None:
        y = y * (st["k_keep"] != 0).unsqueeze(-1)
    return y


def _exact_attend(st, sel):
    """One query tile after another against all of the unit's live rows, the rows outside a query's blocks masked."""
    c, s = st["c"], st["s"]
    d, H, bs = c["d"], c["H"], c["block"]
    pairs = sum(n * x.length * H for n, x in zip(st["counts"], s.n))
    if pairs * d > 6e11:
        return None
    q = st["q"].double()
    if st["rope"] is not None:
        z = torch.view_as_complex(q.unflatten(-1, (H, d // 2, 2)).contiguous())
        q = torch.view_as_real(z * torch.view_as_complex(st["rope"].double().contiguous())[:, None]).flatten(-3)
    base = st["x0"] if st["x0"] is not None else st["res"]
    out = torch.zeros(st["out"].shape, dtype=torch.float64, device="cuda") if base is None else base.double()
    for u, n in enumerate(st["counts"]):
        place = s.n[u].places()
        if n == 0 or place.numel() == 0:
            continue
        block = place // bs
        cells = st["idx"][u, :n].long()
        for h in range(H):
            col = slice(h * d, (h + 1) * d)
            k, v = s.k[u][place][:, col].double(), s.v[u][place][:, col].double()
            for a in range(0, n, 128):
                cell = cells[a:a + 128]
                chosen = torch.zeros((cell.numel(), _blocks(c) + 1), dtype=torch.bool, device="cuda")
                listed_blocks = sel[u, h, a:a + cell.numel()].long()
                chosen.scatter_(1, torch.where(listed_blocks < 0, _blocks(c), listed_blocks), True)
                x = (q[u // c["per"]][cell][:, col] @ k.T) * d ** -0.5
                x.masked_fill_(~chosen[:, block], -math.inf)
                x -= x.amax(1, keepdim=True).clamp(min=-1e300)
                p = x.exp_()
                out[u][cell, col] += (p @ v) / p.sum(1, keepdim=True).clamp(min=1e-300)
    return out
