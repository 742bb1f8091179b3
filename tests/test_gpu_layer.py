"""Rotary positions and the norms around a block against plain implementations in 64 bits."""
import math

import pytest
import torch

pytestmark = pytest.mark.gpu

DT = {"f32": torch.float32, "bf16": torch.bfloat16}
HALF = {"f32": 2.0 ** -24, "bf16": 2.0 ** -8}              # a rounding to the stored type, relative
STEP = 2.0 ** -24                                          # a rounding in fp32, relative


@pytest.fixture(scope="module")
def rs3():
    from paper_2608_22526_gb300 import rs3
    return rs3


def gen(seed):
    return torch.Generator(device="cuda").manual_seed(seed)


def status():
    return torch.zeros(1, dtype=torch.int32, device="cuda")


def bits(t):
    return t.contiguous().view(torch.int16 if t.dtype == torch.bfloat16 else torch.int32)


# ---------------------------------------------------------------------------
# rotary positions
# ---------------------------------------------------------------------------
def frequencies(pairs, base, factor, context, fast, slow):
    out = []
    for n in pairs:
        for i in range(n):
            f = base ** (-i / n)
            g = 0.0 if context == 0 else min(1.0, max(0.0, (context * f / (2 * math.pi) - slow) / (fast - slow)))
            out.append(f * (g + (1 - g) / factor))
    return torch.tensor(out, dtype=torch.float64, device="cuda")


def angles(pos, pairs, freq):
    axis = torch.tensor([a for a, n in enumerate(pairs) for _ in range(n)], device="cuda")
    return pos.double().view(-1, len(pairs))[:, axis] * freq


def rope_ref(x, H, d, rot, layout, ang, magnitude=1.0, inverse=False):
    """(value, |x0| + |x1| of its pair) in 64 bits; x [rows, H * d], ang [rows, rot / 2]."""
    h = x.double().view(-1, H, d)
    out, size = h.clone(), torch.zeros_like(h)
    half = rot // 2
    p = torch.arange(half, device="cuda")
    i, j = (2 * p, 2 * p + 1) if layout == "pairs" else (p, p + half)
    z = torch.complex(h[..., i], h[..., j]) * torch.polar(torch.full_like(ang, magnitude), -ang if inverse else ang)[:, None]
    out[..., i], out[..., j] = z.real, z.imag
    size[..., i] = size[..., j] = h[..., i].abs() + h[..., j].abs()
    return out.view(x.shape), size.view(x.shape)


def check_rope(got, ref, size, dtype, ang):
    # the angle: 2^-53 of it in the frequency, taken twice, and as much in this test's own product; t = rest * step takes
    # three roundings of |t| <= pi / 4 (2.4 half-steps), its sine or cosine 1.5 more of values up to 1, the magnitude
    # and the two products and sum three: under 8 half-steps of |x0| + |x1|; then the rounding to the stored type
    far = float(ang.abs().max()) * 2.0 ** -50 if ang.numel() else 0.0
    tol = HALF[dtype] * ref.abs() + (8 * STEP + far) * size * (1 + HALF[dtype])
    err = (got.double() - ref).abs()
    assert (err <= tol + 1e-42).all(), float((err - tol).max())


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("layout", ["pairs", "halves"])
@pytest.mark.parametrize("d,rot,pairs", [(8, 2, (1,)), (16, 16, (8,)), (64, 64, (16, 16)), (64, 48, (8, 8, 8)), (80, 46, (7, 16)),
                                         (128, 6, (1, 1, 1)), (256, 256, (43, 43, 42)), (256, 250, (125,)), (24, 24, (0, 12))])
@pytest.mark.parametrize("rows,Hq,Hk", [(1, 1, 1), (37, 3, 1), (1200, 1, 5)])
def test_rows_match_64_bits(rs3, dtype, layout, d, rot, pairs, rows, Hq, Hk):
    g = gen(d + rot + rows)
    q = (torch.randn((rows, Hq * d), generator=g, device="cuda") * 3).to(DT[dtype])
    k = torch.randn((2 * rows, Hk * d), generator=g, device="cuda").to(DT[dtype])
    pos = [torch.randint(-9, 1000, (n, len(pairs)), generator=g, device="cuda").to(torch.int32) for n in (rows, 2 * rows)]
    long = dict(factor=4.0, context=512.0, beta_fast=20.0, beta_slow=0.5) if rows == 37 else {}
    spec = rs3.rope_spec(rot, pairs, layout, base=5000.0, **long)
    freq = frequencies(pairs, 5000.0, long.get("factor", 1.0), long.get("context", 0), 20.0, 0.5)
    qo, ko = torch.zeros_like(q), torch.zeros_like(k)
    rs3.rs3_rope_rows(q, qo, pos[0], k, ko, pos[1], dtype, Hq, Hk, d, spec)
    for x, y, p, H in ((q, qo, pos[0], Hq), (k, ko, pos[1], Hk)):
        ang = angles(p, pairs, freq)
        check_rope(y, *rope_ref(x, H, d, rot, layout, ang), dtype, ang)
    rest = torch.arange(d, device="cuda") >= rot                       # copied bit for bit
    assert torch.equal(bits(qo.view(-1, d)[:, rest]), bits(q.view(-1, d)[:, rest]))
    # in place: the same bits
    rs3.rs3_rope_rows(q, q, pos[0], k, k, pos[1], dtype, Hq, Hk, d, spec)
    assert torch.equal(bits(q), bits(qo)) and torch.equal(bits(k), bits(ko))


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("layout,rot", [("pairs", 34), ("pairs", 32), ("halves", 32), ("halves", 22), ("halves", 6)])
def test_elements_that_do_not_turn_keep_their_bits(rs3, dtype, layout, rot):
    """Whatever they are: infinities, NaN of any payload."""
    d, H, rows = 64, 3, 40
    g = gen(rot)
    raw = torch.randint(-2 ** 31, 2 ** 31 - 1, (rows, H * d), generator=g, device="cuda").to(torch.int32)
    x = (raw.to(torch.int16) if dtype == "bf16" else raw).view(DT[dtype]).clone()
    x.view(rows, H, d)[..., :rot] = 1.0
    x.view(rows, H, d)[:, 0, rot:rot + 2] = math.inf
    pos = torch.arange(rows, dtype=torch.int32, device="cuda")[:, None]
    y = torch.zeros_like(x)
    rs3.rs3_rope_rows(x, y, pos, None, None, None, dtype, H, 0, d, rs3.rope_spec(rot, layout=layout))
    assert torch.equal(bits(y).view(rows, H, d)[..., rot:], bits(x).view(rows, H, d)[..., rot:])
    assert y.view(rows, H, d)[..., :rot].isfinite().all()


@pytest.mark.parametrize("layout", ["pairs", "halves"])
def test_far_positions(rs3, layout):
    """The whole range of positions: whole turns drop out."""
    d, rows = 64, 200
    g = gen(3)
    pos = torch.randint(-2 ** 31, 2 ** 31 - 1, (rows, 1), generator=g, device="cuda").to(torch.int32)
    pos[0], pos[1], pos[2] = 0, -2 ** 31, 2 ** 31 - 1
    x = torch.randn((rows, d), generator=g, device="cuda")
    y = torch.zeros_like(x)
    spec = rs3.rope_spec(d, layout=layout, factor=3.0)
    rs3.rs3_rope_rows(x, y, pos, None, None, None, "f32", 1, 0, d, spec)
    ang = angles(pos, (32,), frequencies((32,), 10000.0, 3.0, 0, 32, 1))
    check_rope(y, *rope_ref(x, 1, d, d, layout, ang), "f32", ang)
    assert torch.equal(y[0], x[0])


def test_one_rotation_undoes_another(rs3):
    """Back with `inverse`: the transpose, which is the gradient (against differences, too)."""
    d, rows = 32, 50
    g = gen(4)
    pos = torch.randint(0, 5000, (rows, 1), generator=g, device="cuda").to(torch.int32)
    x, w = (torch.randn((rows, d), generator=g, device="cuda") for _ in range(2))
    there, back = rs3.rope_spec(24, layout="halves", magnitude=1.5), rs3.rope_spec(24, layout="halves", magnitude=1.5, inverse=True)

    def turn(v, spec):
        o = torch.zeros_like(v)
        rs3.rs3_rope_rows(v, o, pos, None, None, None, "f32", 1, 0, d, spec)
        return o

    grad = turn(w, back)                                     # of sum(w * turn(x))
    ang = angles(pos, (12,), frequencies((12,), 10000.0, 1.0, 0, 32, 1))
    check_rope(grad, *(t * (1.5 if i else 1.0) for i, t in enumerate(rope_ref(w, 1, d, 24, "halves", ang, 1.5, True))), "f32", ang)
    # differences of a linear function, exact but for its roundings: f(x + e) - f(x) over e = 2^-3 along each element
    # in turn; the values reach 8 * 1.5 and the sum of two products of w, each with 11 half-steps of its terms
    for at in (0, 5, 12, 23, 24, 31):
        e = torch.zeros_like(x)
        e[:, at] = 0.125
        slope = ((turn(x + e, there).double() - turn(x, there).double()) * w.double()).sum(1) / 0.125
        size = ((turn(x.abs() + e, there).double().abs() + 3 * x.double().abs() + 1) * w.double().abs()).sum(1)
        assert ((slope - grad[:, at].double()).abs() <= 8 * 2 * 12 * STEP * 2 * size).all()


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("layout,rot", [("pairs", 64), ("halves", 64), ("halves", 44)])
def test_packed_rows_with_masks(rs3, dtype, layout, rot):
    """Queries, keys and values side by side, in place; rows that the mask leaves hold NaN and keep their bits."""
    G, mn, H, d = 3, 45, 2, 64
    x = torch.randn((G, mn, 3 * H * d), generator=gen(5), device="cuda").to(DT[dtype])
    keep = (torch.rand((G, mn), generator=gen(6), device="cuda") < 0.5).to(torch.uint8)
    keep[1] = 0
    x[keep == 0, H * d:2 * H * d] = math.nan
    before = x.clone()
    pos = torch.randint(0, 100, (G, mn, 1), generator=gen(7), device="cuda").to(torch.int32)
    q, k = x[..., :H * d], x[..., H * d:2 * H * d]
    rs3.rs3_rope_rows(q, q, pos, k, k, pos, dtype, H, H, d, rs3.rope_spec(rot, layout=layout), k_keep=keep)
    ang = angles(pos, (rot // 2,), frequencies((rot // 2,), 10000.0, 1.0, 0, 32, 1))
    flat = before.view(-1, 3 * H * d)
    check_rope(q.reshape(-1, H * d), *rope_ref(flat[:, :H * d], H, d, rot, layout, ang), dtype, ang)
    on = keep.view(-1) != 0
    check_rope(k.reshape(-1, H * d)[on], *rope_ref(flat[on, H * d:2 * H * d], H, d, rot, layout, ang[on]), dtype, ang)
    same = torch.ones_like(x, dtype=torch.bool)
    same[..., :H * d] = False
    same[..., H * d:2 * H * d] = (keep == 0)[..., None]
    assert torch.equal(bits(x)[same], bits(before)[same])


@pytest.mark.parametrize("rot,pairs", [(16, (8,)), (64, (16, 16)), (6, (1, 1, 1)), (256, (43, 43, 42))])
def test_table_matches_64_bits_and_the_calls_that_take_one(rs3, rot, pairs):
    mn = 143
    g = gen(8)
    pos = torch.randint(0, 300, (mn, len(pairs)), generator=g, device="cuda").to(torch.int32)
    spec = rs3.rope_spec(rot, pairs, factor=2.0, context=100.0, magnitude=1.25)
    table = torch.full((mn, rot // 2, 2), 9.0, device="cuda")
    rs3.rs3_rope_table(pos, spec, table)
    ang = angles(pos, pairs, frequencies(pairs, 10000.0, 2.0, 100.0, 32, 1))
    ref = 1.25 * torch.stack([ang.cos(), ang.sin()], -1)
    assert ((table.double() - ref).abs() <= 1.25 * (5 * STEP + float(ang.max()) * 2.0 ** -50)).all()
    if rot % 8 == 0:
        # the table's rotation inside the head norms (which scale by 1 here) is the rows' own
        x = torch.randn((mn, rot), generator=g, device="cuda")
        x = x / x.square().mean(1, keepdim=True).sqrt()
        a, b = torch.zeros_like(x), torch.zeros_like(x)
        rs3.rs3_qk_norm_rope(x, a, None, None, "f32", mn, 1, 0, rot, eps=0.0, rope=table)
        rs3.rs3_rope_rows(x, b, pos, None, None, None, "f32", 1, 0, rot, spec)
        assert torch.allclose(a, b, rtol=0, atol=64 * STEP * 1.25 * 2 * float(x.abs().max()))


def test_rope_takes_no_rows_and_keeps_what_lies_around(rs3):
    d = 64
    x = torch.randn((6, d), generator=gen(9), device="cuda")
    y = torch.full((8, d), 7.0, device="cuda")
    pos = torch.arange(6, dtype=torch.int32, device="cuda")[:, None]
    spec = rs3.rope_spec(d, layout="halves")
    rs3.rs3_rope_rows(x[:0], y[:0], pos[:0], None, None, None, "f32", 1, 0, d, spec)
    rs3.rs3_rope_table(pos[:0], spec, y)
    assert (y == 7).all()
    rs3.rs3_rope_rows(x, y[1:7], pos, None, None, None, "f32", 1, 0, d, spec)
    assert (y[0] == 7).all() and (y[7] == 7).all() and not (y[1:7] == 7).any()
    with pytest.raises(ValueError):
        rs3.rs3_rope_rows(x, y[:6], pos[:5], None, None, None, "f32", 1, 0, d, spec)
    with pytest.raises(rs3.RS3Error):                      # rows that lie over their operand's
        rs3.rs3_rope_rows(y[:6], y[1:7], pos, None, None, None, "f32", 1, 0, d, spec)


# ---------------------------------------------------------------------------
# norms around a block
# ---------------------------------------------------------------------------
def norm_ref(kind, v, e, w, b, eps):
    """(value, bound of its error before rounding) of a norm in 64 bits; v [rows, C] is off by at most e [rows, 1] per
    element.  A sum over a row takes at most 32 adds of one lane, five over a warp and eight over a CTA, so 48
    half-steps of the values' sizes; half of that is left of a sum of squares after the root, with its
    mean, the root's own four and the product under 32."""
    one = torch.ones_like(v)
    if kind != "none":
        if kind == "layer":
            e = 2 * e + 50 * STEP * v.abs().mean(1, keepdim=True) + STEP * v.abs().amax(1, keepdim=True)
            v = v - v.mean(1, keepdim=True)
        r = (v.square().mean(1, keepdim=True) + eps).rsqrt()
        n = v * r
        e = e * r * (1 + n.abs()) + 32 * STEP * n.abs()
    else:
        n = v
        e = e * one
    w = one if w is None else w.double()
    b = torch.zeros_like(v) if b is None else b.double()
    y = n * w + b
    return y, e * w.abs() + 3 * STEP * ((n * w).abs() + b.abs())


def block_ref(y, x, post, pre, gate, alpha, eps):
    """(x', bound), (h, bound) of rows [rows, C]; post, pre: (kind, weight, bias)."""
    v = alpha * x.double()
    e = 2 * STEP * v.abs()
    if y is not None:
        t, te = norm_ref(post[0], y.double(), torch.zeros((y.shape[0], 1), device="cuda", dtype=torch.float64), post[1], post[2], eps)
        g = torch.ones_like(t) if gate is None else gate.double()
        v = v + g * t
        e = e + te * g.abs() + 4 * STEP * (g * t).abs()
    h, he = norm_ref(pre[0], v, e.amax(1, keepdim=True), pre[1], pre[2], eps)
    return (v, e), (h, he)


def check(got, ref, bound, dtype):
    tol = bound + HALF[dtype] * (ref.abs() + bound)
    err = (got.double() - ref).abs()
    assert (err <= tol + 1e-42).all(), float((err - tol).max())


def vectors(U, C, per_unit, seed):
    g = gen(seed)
    return [s + 0.3 * torch.randn((U, C) if p else (C,), generator=g, device="cuda") for s, p in
            ((1.0, False), (0.0, per_unit), (0.5, per_unit), (1.0, per_unit), (0.0, False))]


def rows_of(t, u):
    return None if t is None else (t if t.dim() == 1 else t[u])


def run_block(rs3, dtype, U, mn, C, kept, post="rms", pre="rms", gate=True, alpha=0.75, with_y=True, per_unit=False, seed=0, scale=1.0, eps=1e-6):
    g = gen(seed + C)
    y = (torch.randn((U, mn, C), generator=g, device="cuda") * scale).to(DT[dtype])
    x = (torch.randn((U, mn, C), generator=g, device="cuda") * 2 + 0.3).to(DT[dtype])
    pw, pb, ga, w, b = vectors(U, C, per_unit, seed)
    idx = count = None
    if kept is not None:
        idx = torch.stack([torch.randperm(mn, generator=g, device="cuda")[:max(1, max(kept))].sort().values for _ in range(U)]).to(torch.int32)
        count = torch.tensor(kept, dtype=torch.int32, device="cuda")
    xo, ho = torch.full_like(x, 7.0), torch.full_like(x, 9.0)
    st = status()
    args = dict(idx=idx, count=count, post=post, post_weight=pw, post_bias=pb, gate=ga if gate else None, alpha=alpha, pre=pre,
                pre_weight=w, pre_bias=b, eps=eps, status=st)
    rs3.rs3_norm_residual(y if with_y else None, x, xo, ho, dtype, **args)
    assert int(st) == 0
    for u in range(U):
        cells = torch.arange(mn, device="cuda") if idx is None else idx[u, :kept[u]].long()
        if cells.numel():
            vx, vh = block_ref(y[u, cells] if with_y else None, x[u, cells], (post, pw, rows_of(pb, u)), (pre, rows_of(w, u), b),
                               rows_of(ga, u) if gate else None, alpha, eps)
            check(xo[u, cells], *vx, dtype)
            check(ho[u, cells], *vh, dtype)
        left = torch.ones(mn, dtype=torch.bool, device="cuda")
        left[cells] = False
        assert (xo[u, left] == 7).all() and (ho[u, left] == 9).all()
    # in place over the operands: the same bits
    xi, yi = x.clone(), y.clone()
    rs3.rs3_norm_residual(yi if with_y else None, xi, xi, yi, dtype, **args)
    for u in range(U):
        cells = torch.arange(mn, device="cuda") if idx is None else idx[u, :kept[u]].long()
        assert torch.equal(bits(xi[u, cells]), bits(xo[u, cells]))
        assert torch.equal(bits(yi[u, cells]), bits(ho[u, cells]))
    return xo, ho


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("C", [8, 24, 64, 200, 256, 264, 512, 1000, 1024, 2056, 4096])
@pytest.mark.parametrize("post,pre", [("rms", "rms"), ("layer", "layer"), ("none", "layer")])
def test_block_matches_64_bits(rs3, dtype, C, post, pre):
    run_block(rs3, dtype, 2, 37, C, None, post, pre, per_unit=C % 3 == 0)
    run_block(rs3, dtype, 3, 50, C, [50, 0, 13], post, pre, gate=False, alpha=1.0, per_unit=C % 3 == 1)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_block_of_one_cell_and_of_many(rs3, dtype):
    run_block(rs3, dtype, 1, 1, 64, None)
    run_block(rs3, dtype, 1, 1, 64, [1], with_y=False, pre="layer")
    run_block(rs3, dtype, 1, 16384, 64, [16384])
    run_block(rs3, dtype, 300, 5, 16, None, per_unit=True)
    run_block(rs3, dtype, 2, 9000, 256, [9000, 4001], "layer", "rms", per_unit=True)


def test_block_results_one_at_a_time_and_rows_without_spread(rs3):
    x = torch.full((1, 4, 64), 3.0, device="cuda")
    x[0, 1] = 0.0
    x[0, 2] = torch.randn(64, generator=gen(1), device="cuda") * 1e-20
    x[0, 3] = torch.randn(64, generator=gen(2), device="cuda") * 1e15
    h, xo = torch.zeros_like(x), torch.zeros_like(x)
    rs3.rs3_norm_residual(None, x, None, h, "f32", pre="layer")
    for i in range(4):
        check(h[0, i:i + 1], *block_ref(None, x[0, i:i + 1], ("none", None, None), ("layer", None, None), None, 1.0, 1e-6)[1], "f32")
    assert (h[0, 1] == 0).all()
    rs3.rs3_norm_residual(x, x, xo, None, "f32", post="rms", alpha=-2.0)
    check(xo[0], *block_ref(x[0], x[0], ("rms", None, None), ("none", None, None), None, -2.0, 1e-6)[0], "f32")


def test_block_bad_counts_and_cells_are_latched_and_skipped(rs3):
    U, mn, C = 4, 10, 32
    x = torch.randn((U, mn, C), generator=gen(1), device="cuda")
    idx = torch.arange(5, dtype=torch.int32, device="cuda").repeat(U, 1)
    idx[2, 1], idx[2, 3] = -1, mn
    count = torch.tensor([6, -1, 5, 2], dtype=torch.int32, device="cuda")
    out, st = torch.full_like(x, 7.0), status()
    rs3.rs3_norm_residual(None, x, out, None, "f32", idx=idx, count=count, status=st)
    assert int(st) == rs3.RS3_EINVAL
    want = torch.full_like(x, 7.0)
    for u, cells in ((2, [0, 2, 4]), (3, [0, 1])):
        want[u, cells] = x[u, cells]
    assert torch.equal(out, want)


def test_layer_calls_captured_and_on_another_stream(rs3):
    """Both calls, replayed on other values, and on a stream that is not the current one."""
    U, mn, C = 2, 60, 128
    x, y = (torch.randn((U, mn, C), generator=gen(i), device="cuda") for i in range(2))
    pos = torch.arange(U * mn, dtype=torch.int32, device="cuda")[:, None].contiguous()
    spec = rs3.rope_spec(64, layout="halves")
    xo, ho, ro = torch.zeros_like(x), torch.zeros_like(x), torch.zeros_like(x)

    def call(stream=None):
        rs3.rs3_norm_residual(y, x, xo, ho, "f32", post="rms", pre="layer", stream=stream)
        rs3.rs3_rope_rows(ho, ro, pos, None, None, None, "f32", 2, 0, 64, spec, stream=stream)

    call()
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        call()
    x.mul_(1.5)
    y.add_(0.25)
    for t in (xo, ho, ro):
        t.zero_()
    graph.replay()
    torch.cuda.synchronize()
    got = [t.clone() for t in (xo, ho, ro)]
    for t in (xo, ho, ro):
        t.zero_()
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    call(side)
    side.synchronize()
    assert all(torch.equal(a, b) for a, b in zip(got, (xo, ho, ro))) and (ro != 0).any()
