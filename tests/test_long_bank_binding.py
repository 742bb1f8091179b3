"""The binding of the long-bank calls refuses tensors that are not on the device of the call before the library
sees them.  CPU only: tensors say that they are on a device, and nothing may reach the library."""
import types

import pytest
import torch


class There(torch.Tensor):
    """A CPU tensor that calls itself one of device 0."""

    def get_device(self):
        return 0


def there(*shape, dtype=torch.int32):
    return torch.zeros(shape, dtype=dtype).as_subclass(There)


U, H, D, MN, K, TOP, BLOCK, ROWS = 2, 1, 64, 16, 4, 3, 32, 64


@pytest.fixture()
def calls(monkeypatch):
    """(rs3, calls): calls[name](**changes) makes a call whose tensors are on device 0, the current one."""
    from paper_2608_22526_gb300 import _build
    _build.build()
    from paper_2608_22526_gb300 import rs3

    class Lib:
        def __getattr__(self, name):
            return lambda *a: reached.append(name) or 0

    reached = []
    monkeypatch.setattr(rs3, "lib", Lib())
    monkeypatch.setattr(torch.cuda, "current_device", lambda: 0)
    monkeypatch.setattr(rs3, "_stream", lambda s: 0)
    store = there(U, ROWS, H * D, dtype=torch.bfloat16)
    bank = types.SimpleNamespace(U=U, H=H, d=D, D=H * D, dtype="bf16", mn=MN, rows_per_unit=ROWS, desc=rs3.BankDesc(), k_store=store,
                                 v_store=store, meta=there(64, dtype=torch.int64))
    nb, st, ws = ROWS // BLOCK, there(1), there(256, dtype=torch.uint8)
    grid = there(1, MN, H * D, dtype=torch.bfloat16)
    read = (grid, "bf16", 1, MN, H, D, there(U), there(U, K), there(U), K)
    dig, step, sel = there(U, H, nb, D, dtype=torch.int8), there(U, H, nb, dtype=torch.float32), there(U, H, K, TOP)
    out = there(U, MN, H * D, dtype=torch.bfloat16)
    keep = there(U, ROWS, dtype=torch.uint8)
    return rs3, reached, types.SimpleNamespace(
        rs3_bank_copy=lambda bank=bank, dst=None, keep=keep, ws=ws: rs3.rs3_bank_copy(dst or bank, bank, there(U), keep, ws, st),
        rs3_bank_drop_frames=lambda bank=bank: rs3.rs3_bank_drop_frames(bank, there(U), None, st),
        rs3_bank_digest=lambda bank=bank: rs3.rs3_bank_digest(bank, BLOCK, -1, dig, step, st),
        rs3_block_select=lambda bank=bank, ws=ws: rs3.rs3_block_select(*read, bank, BLOCK, dig, step, None, TOP, sel, ws, st),
        rs3_sparse_readout=lambda bank=bank, ws=ws: rs3.rs3_sparse_readout(*read, bank, BLOCK, sel, TOP, None, None, out, 0.0, ws, st)), bank


ALL = ["rs3_bank_copy", "rs3_bank_drop_frames", "rs3_bank_digest", "rs3_block_select", "rs3_sparse_readout"]


@pytest.mark.parametrize("name", ALL)
def test_calls_on_one_device_reach_the_library(calls, name):
    _, reached, make, _ = calls
    getattr(make, name)()
    assert reached == [name]


@pytest.mark.parametrize("name", ["rs3_bank_copy", "rs3_block_select", "rs3_sparse_readout"])
def test_a_workspace_elsewhere_is_refused(calls, name):
    _, reached, make, _ = calls
    with pytest.raises(ValueError, match="workspace"):
        getattr(make, name)(ws=torch.zeros(256, dtype=torch.uint8))
    assert not reached
    getattr(make, name)(ws=None)                           # (the library's to refuse, or not to need)
    assert reached == [name]


def test_a_copy_without_a_mask_takes_an_empty_workspace_from_anywhere(calls):
    _, reached, make, _ = calls
    make.rs3_bank_copy(keep=None, ws=torch.zeros(0, dtype=torch.uint8))
    assert reached == ["rs3_bank_copy"]


@pytest.mark.parametrize("name", ALL)
def test_a_bank_elsewhere_is_refused(calls, name):
    _, reached, make, bank = calls
    other = types.SimpleNamespace(**{**vars(bank), **{part: torch.zeros(4) for part in ("k_store", "v_store", "meta")}})
    for args in ([dict(bank=other), dict(dst=other)] if name == "rs3_bank_copy" else [dict(bank=other)]):
        with pytest.raises(ValueError, match="bank"):
            getattr(make, name)(**args)
    assert not reached
