"""fp32 heads of 128 in the scored and shared readouts: the one kernel that their calls take is what their workspace is for.
CPU only."""
import ctypes

import pytest

from test_long_bank_abi import _bank


@pytest.fixture(scope="module")
def rs3():
    from paper_2608_22526_gb300 import _build
    _build.build()
    from paper_2608_22526_gb300 import rs3
    return rs3


@pytest.mark.parametrize("k_max", [0, 1, 20, 64])
def test_workspace_of_heads_of_128(rs3, k_max):
    bank = _bank(rs3, U=1, H=1, d=128, dtype="f32")
    prefix = _bank(rs3, U=1, H=1, d=128, dtype="f32", k=1 << 41, v=1 << 42, meta=1 << 43)
    # two slots for each of two CTAs an SM (148 to 160 of them) of 32 rows, with their (m, l); lists and tables of this small
    # bank in half a megabyte.  Tiles of 128 rows, a CTA an SM, would need twice as much.
    one = 2 * 2 * 160 * 32 * (128 + 2) * 4 + (1 << 19)
    assert rs3.lib.rs3_scored_readout_workspace_bytes(ctypes.byref(bank), k_max) <= one
    # (the shared readout has a slot for each of its few groups besides)
    assert rs3.lib.rs3_shared_readout_workspace_bytes(ctypes.byref(bank), ctypes.byref(prefix), k_max) <= 2 * one
