"""fp32 heads of 128: the readouts stay inside the workspace that they ask for, with few queries and with many."""
import math

import pytest
import torch

from test_gpu_long_bank import bits
from test_gpu_more_readouts import biases, built, run_scored, run_shared, scored_case, shared_case

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def rs3():
    from paper_2608_22526_gb300 import rs3
    return rs3


@pytest.mark.parametrize("U,H,m,counts", [(1, 1, 16, [1]), (3, 2, 16, [256, 100, 3]), (8, 4, 40, [1600] * 8)])
def test_readouts_of_heads_of_128_stay_inside_their_workspaces(rs3, U, H, m, counts):
    b = built(rs3, U=U, H=H, d=128, dtype="f32", m=m, n=m, window=3, commits=4, n_ptr=5, seed=2)
    p = built(rs3, U=1, H=H, d=128, dtype="f32", m=m, n=m, window=3, commits=4, n_ptr=0, seed=3)
    bias = biases(b, "unit")
    q, idx, count, group, table, out, _ = scored_case(rs3, b, counts, [0] * U, 1, 6.0, bias)
    n = rs3.rs3_scored_readout_workspace_bytes(b.bank, idx.shape[1])
    ws = torch.full((n + 65536,), 77, dtype=torch.uint8, device="cuda")
    again = torch.full_like(out, math.nan)
    run_scored(rs3, b, q, 1, idx, count, group, 6.0, bias, None, table, 0.0, None, again, ws[:n])
    assert torch.equal(bits(again), bits(out)) and (ws[n:] == 77).all()
    q, idx, count, group, prefix_unit, table, out = shared_case(rs3, b, p, counts, [0] * U, [0] * U, 1)
    n = rs3.rs3_shared_readout_workspace_bytes(b.bank, p.bank, idx.shape[1])
    ws = torch.full((n + 65536,), 77, dtype=torch.uint8, device="cuda")
    again = torch.full_like(out, math.nan)
    run_shared(rs3, b, p, q, 1, idx, count, group, prefix_unit, table, 0.0, None, again, ws[:n])
    assert torch.equal(bits(again), bits(out)) and (ws[n:] == 77).all()
    assert int(b.st) == 0
