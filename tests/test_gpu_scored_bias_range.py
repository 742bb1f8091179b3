"""Scored readouts whose cap bounds the scores, with biases that set frames further apart than scores do: what has been
summed against a low bias may weigh more than all that follows against a high one."""
import math

import pytest
import torch

from test_gpu_long_bank import DT, Built, bits, gen
from test_gpu_more_readouts import frames_of, keep_sets, reference, run_scored, scored_rows, spoil

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def rs3():
    from paper_2608_22526_gb300 import rs3
    return rs3


def saturated(rs3, dtype, U, H, d, m, ring_frames, seed, high):
    """A bank whose rows of the frames in `high` (ages, F: conditioning, F + 1: pointers) have scores at the cap, all others
    at minus the cap, and queries for it."""
    b = Built(rs3, U=U, H=H, d=d, dtype=dtype, m=m, n=m, window=-1, ring_frames=ring_frames, commits=ring_frames, n_ptr=9, seed=seed)
    F = b.bank.max_frames
    high = [F if h == "cond" else F + 1 if h == "ptr" else h for h in high]
    for u in range(U):
        at, slot = frames_of(b, u)
        sign = torch.where(torch.isin(slot, torch.tensor(high, device="cuda")), 1.0, -1.0)
        b.bank.k_store[u, at] = (sign[:, None] * 60.0 * (0.5 + b.bank.k_store[u, at].float().abs())).to(DT[dtype])
    spoil(b, None)
    # 60 * 0.5 * 0.5 * sqrt(16) is above the largest cap here, at the narrowest heads
    q = (0.5 + torch.randn((1, b.mn, H * d), generator=gen(seed + 1), device="cuda").abs()).to(DT[dtype])
    return b, q


def check(rs3, b, q, counts, cap, bias):
    idx, count = keep_sets(b.U, b.mn, max(counts), counts, 7)
    group = torch.zeros(b.U, dtype=torch.int32, device="cuda")
    out = torch.full((b.U, b.mn, b.D), math.nan, dtype=DT[b.dtype], device="cuda")
    want, tol = reference(b.dtype, b.H, b.d, q, idx, counts, group, None, b.d ** -0.5, None, out.shape, scored_rows(b, None), cap,
                          lambda u, h: bias[h])
    run_scored(rs3, b, q, 1, idx, count, group, cap, bias, None, None, 0.0, None, out)
    assert int(b.st) == 0
    err = (out.double() - want).abs()
    assert (err <= tol).all(), (float((err - tol).max()), float(err.max()))
    return out


# few queries over short banks (a unit's rows in few pieces), over long ones (in many), and much work (whole groups; heads
# of 64 and 128 by two query tiles)
SHAPES = [("bf16", 2, 1, 256, 16, 4, [30, 9]), ("bf16", 1, 1, 256, 32, 20, [40]), ("bf16", 8, 4, 256, 24, 3, [300, 576, 9, 129, 400, 1, 0, 64]),
          ("bf16", 2, 1, 64, 16, 4, [30, 9]), ("bf16", 1, 1, 64, 32, 20, [40]), ("bf16", 2, 8, 64, 64, 4, [2500, 1200]),
          ("bf16", 1, 2, 128, 32, 20, [40]), ("bf16", 2, 4, 128, 64, 8, [2500, 1200]), ("bf16", 1, 1, 32, 16, 6, [100]),
          ("f32", 1, 1, 64, 16, 6, [100]), ("f32", 1, 1, 128, 16, 6, [100])]


@pytest.mark.parametrize("dtype,U,H,d,m,ring_frames,counts", SHAPES)
@pytest.mark.parametrize("cap,sunk", [(55.0, -90.0), (55.0, -105.0), (50.0, -90.0), (40.0, -79.0), (55.0, -180.0)])
@pytest.mark.parametrize("order", ["sunk first", "sunk last", "sunk between"])
def test_frames_of_low_bias_and_high_scores_weigh_what_they_should(rs3, dtype, U, H, d, m, ring_frames, counts, cap, sunk, order):
    """Scores of twice the cap above the others' make up for a bias of less than that, whichever is read first."""
    F = ring_frames
    where = {"sunk first": ["cond", F - 1], "sunk last": ["ptr", 0], "sunk between": [F // 2]}[order]
    b, q = saturated(rs3, dtype, U, H, d, m, ring_frames, 5, where)
    bias = torch.zeros((H, F + 2), device="cuda")
    for w in where:
        bias[:, F if w == "cond" else F + 1 if w == "ptr" else w] = sunk
    check(rs3, b, q, counts, cap, bias)


@pytest.mark.parametrize("dtype,U,H,d,m,ring_frames,counts", SHAPES)
@pytest.mark.parametrize("cap", [20.0, 55.0])
def test_biases_that_climb_step_by_step(rs3, dtype, U, H, d, m, ring_frames, counts, cap):
    """A reference that moves by less than fp32's range, by more, and by a little in every frame, both ways."""
    b, q = saturated(rs3, dtype, U, H, d, m, ring_frames, 6, range(0, ring_frames, 2))
    age = torch.arange(ring_frames + 2, device="cuda").float()
    for slope in (-5.4, -40.0, -100.0, 5.4, 40.0):
        bias = (slope * age).repeat(H, 1)
        bias[:, ring_frames] = slope * ring_frames
        bias[:, ring_frames + 1] = 0.0
        check(rs3, b, q, counts, cap, bias.contiguous())


@pytest.mark.parametrize("H,d,m,counts", [(1, 256, 16, [30]), (1, 64, 16, [30]), (8, 64, 64, [2500])])
def test_values_as_large_as_the_limit_allows(rs3, H, d, m, counts):
    """Rows times values times e^cap just below the limit, with biases that rise by less than moves a reference."""
    b, q = saturated(rs3, "bf16", 1, H, d, m, 3, 8, ["cond", 0, 1, 2, "ptr"])
    at, _ = frames_of(b, 0)
    b.bank.v_store[0, at] = b.bank.v_store[0, at].float().sign().bfloat16() * (0.9e36 / (len(at) * math.exp(55.0)))
    bias = torch.tensor([0.0, -1.8, -3.6, -5.4, -0.1], device="cuda").repeat(H, 1).contiguous()
    out = check(rs3, b, q, counts, 55.0, bias)
    assert out[0].isfinite().any()


@pytest.mark.parametrize("dtype,U,H,d,m,ring_frames,counts", SHAPES[:8])
@pytest.mark.parametrize("offset", [-1e9, -1e5, 12345.0, 1e9])
def test_an_offset_of_all_biases_changes_nothing(rs3, dtype, U, H, d, m, ring_frames, counts, offset):
    """All frames masked by the same finite number, scores at either end of the cap: the weights are the scores' own."""
    b, q = saturated(rs3, dtype, U, H, d, m, ring_frames, 9, range(0, ring_frames, 3))
    idx, count = keep_sets(U, b.mn, max(counts), counts, 7)
    group = torch.zeros(U, dtype=torch.int32, device="cuda")
    outs = []
    for value in (0.0, offset):
        bias = torch.full((H, ring_frames + 2), value, device="cuda")
        outs.append(torch.zeros((U, b.mn, b.D), dtype=DT[dtype], device="cuda"))
        run_scored(rs3, b, q, 1, idx, count, group, 55.0, bias, None, None, 0.0, None, outs[-1])
    assert int(b.st) == 0
    assert torch.equal(bits(outs[0]), bits(outs[1])) and (outs[0] != 0).any()


@pytest.mark.parametrize("dtype,U,H,d,m,ring_frames,counts", SHAPES)
@pytest.mark.parametrize("value", [math.inf, math.nan])
def test_a_bias_that_is_no_number_makes_its_queries_none(rs3, dtype, U, H, d, m, ring_frames, counts, value):
    """Plus infinity and NaN reach the result from whichever piece they are in, of the head and unit that they belong to."""
    b, q = saturated(rs3, dtype, U, H, d, m, ring_frames, 10, [0])
    idx, count = keep_sets(U, b.mn, max(counts), counts, 7)
    group = torch.zeros(U, dtype=torch.int32, device="cuda")
    for frame in (0, ring_frames // 2, ring_frames, ring_frames + 1):
        bias = torch.zeros((U, H, ring_frames + 2), device="cuda")
        bias[0, H - 1, frame] = value
        bias[:, :, 1] = -math.inf
        out = torch.zeros((U, b.mn, b.D), dtype=DT[dtype], device="cuda")
        run_scored(rs3, b, q, 1, idx, count, group, 55.0, bias, None, None, 0.0, None, out)
        assert int(b.st) == 0
        cells = idx[0, :counts[0]].long()
        # (of three frames, the middle one's value gives way to minus infinity)
        assert out[0, cells, (H - 1) * d:].isnan().all() == (frame != 1), frame
        out[0, cells, (H - 1) * d:] = 0.0
        assert out.isfinite().all(), frame
