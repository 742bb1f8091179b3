"""Readouts whose scores climb from tile to tile, so that what has been summed is scaled down again and again, against
64 bits.  The scaled sums have to be in place before the next tile's product is added to them."""
import math

import pytest
import torch

from test_gpu_long_bank import DT, bits, gen
from test_gpu_more_readouts import built, frames_of, keep_sets, reference, run_scored, run_shared, scored_rows, shared_rows

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def rs3():
    from paper_2608_22526_gb300 import rs3
    return rs3


def climbing(rs3, U, H, d, seed, first=0.0, step=0.11, frames=12):
    """A bank whose keys lie along a head's direction, further out from frame to frame; (bank, directions)."""
    b = built(rs3, U=U, H=H, d=d, dtype="bf16", m=16, n=16, window=-1, ring_frames=frames, commits=frames, n_ptr=0, n_cond=0, seed=seed)
    g = gen(11)
    u = torch.randint(0, 2, (H * d,), generator=g, device="cuda").float() * 2 - 1
    for i in range(U):
        at, age = frames_of(b, i)
        out = first + step * (16.0 / math.sqrt(d)) * (frames - 1 - age).float()
        noise = 0.1 * torch.randn((len(at), H * d), generator=g, device="cuda")
        b.bank.k_store[i, at] = (out[:, None] * u + noise).bfloat16()
    return b, u


# one query tile: heads of 256 at any number of queries, of 64 and 128 where a unit has at most one
SHAPES = [(8, 4, 256, [256, 200, 130, 1, 256, 129, 128, 0]), (16, 4, 128, [128 - 5 * i for i in range(16)]),
          (16, 4, 64, [128 - 5 * i for i in range(16)]), (1, 1, 256, [9])]


@pytest.mark.parametrize("U,H,d,counts", SHAPES)
@pytest.mark.parametrize("call", ["memory", "scored", "capped", "shared"])
def test_sums_follow_scores_that_climb(rs3, U, H, d, counts, call):
    b, u = climbing(rs3, U, H, d, 2)
    D, mn = H * d, b.mn
    g = gen(5)
    # a step of a frame is some 5 to 12 in the log2 domain
    q = (4.0 * (0.6 + 0.8 * torch.rand((1, mn, 1), generator=g, device="cuda")) * u).bfloat16()
    idx, count = keep_sets(U, mn, max(counts), counts, 7)
    group = torch.zeros(U, dtype=torch.int32, device="cuda")
    outs = [torch.full((U, mn, D), math.nan, dtype=DT["bf16"], device="cuda") for _ in range(3)]
    rows, cap, bias = scored_rows(b, None), 0.0, None
    if call == "shared":
        p, _ = climbing(rs3, 1, H, d, 3, first=0.4)
        prefix = torch.zeros(U, dtype=torch.int32, device="cuda")
        rows = shared_rows(b, p, [0] * U)
    elif call != "memory":
        cap = 60.0 if call == "capped" else 0.0
        bias = -0.5 * torch.arange(b.bank.max_frames + 2, device="cuda").float().repeat(H, 1)
    for out in outs:
        if call == "shared":
            run_shared(rs3, b, p, q, 1, idx, count, group, prefix, None, 0.0, None, out)
        elif call == "memory":
            ws = torch.empty(rs3.rs3_readout_workspace_bytes(U, H, d, max(counts), "bf16"), dtype=torch.uint8, device="cuda")
            rs3.rs3_memory_readout(q, "bf16", 1, mn, H, d, group, idx, count, max(counts), b.bank, None, None, out, 0.0, ws, b.st)
        else:
            run_scored(rs3, b, q, 1, idx, count, group, cap, bias, None, None, 0.0, None, out)
    assert int(b.st) == 0
    want, tol = reference("bf16", H, d, q, idx, counts, group, None, d ** -0.5, None, outs[0].shape, rows, cap,
                          None if bias is None else lambda _, h: bias[h])
    err = (outs[0].double() - want).abs()
    assert (err <= tol).all(), (float((err - tol).max()), float(err.max()))
    assert tol.max() < 0.2
    for out in outs[1:]:
        assert torch.equal(bits(out), bits(outs[0]))
