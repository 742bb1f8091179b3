"""Refusals of rs3_scored_readout and rs3_shared_readout on the host, and what the binding and the pipeline check or do
before the library sees a call.  CPU only: no call here reaches a kernel."""
import contextlib
import ctypes
import types

import pytest
import torch

from test_long_bank_abi import ODD, ONE, _bank


@pytest.fixture(scope="module")
def b():
    from paper_2608_22526_gb300 import _build
    _build.build()
    from paper_2608_22526_gb300 import rs3
    return rs3


FAR = dict(k=1 << 41, v=1 << 42, meta=1 << 43)
BIG = 1 << 40                                              # bytes of a workspace that is large enough


def read_args(**over):
    a = dict(q=ONE, dtype=1, G=1, mn=64, H=4, d=64, group=ONE, idx=ONE, count=ONE, k_max=20)
    a.update({k: v for k, v in over.items() if k in a})
    return a


READ_REFUSALS = [(dict(q=None), "EINVAL"), (dict(q=ODD), "EINVAL"), (dict(group=None), "EINVAL"), (dict(idx=None), "EINVAL"),
                 (dict(count=None), "EINVAL"), (dict(dtype=0), "EINVAL"), (dict(dtype=7), "EINVAL"), (dict(H=2), "EINVAL"),
                 (dict(d=128), "EINVAL"), (dict(G=0), "EINVAL"), (dict(mn=0), "EINVAL"), (dict(k_max=-1), "EINVAL"),
                 (dict(out=None), "EINVAL"), (dict(out=ODD), "EINVAL"), (dict(residual=ODD), "EINVAL"), (dict(rope=ODD), "EINVAL"),
                 (dict(ws=None), "EINVAL"), (dict(ws=ODD), "EINVAL"), (dict(status=None), "EINVAL")]


def scored(b, bank=None, cap=0.0, bias=None, bias_stride=0, keep=None, rope=None, residual=None, out=ONE, scale=0.0, ws=ONE, n=BIG, status=ONE,
           **over):
    bank = _bank(b) if bank is None else bank
    return b.lib.rs3_scored_readout(*read_args(**over).values(), ctypes.byref(bank), cap, bias, bias_stride, keep, rope, residual, out, scale,
                                    ws, n, status, None)


@pytest.mark.parametrize("over,code", READ_REFUSALS + [
    (dict(cap=-1.0), "EINVAL"), (dict(cap=float("nan")), "EINVAL"), (dict(cap=float("inf")), "EINVAL"), (dict(cap=2.0 ** -11), "EINVAL"),
    (dict(cap=2.0 ** 11), "EINVAL"), (dict(bias=ctypes.c_void_p(18)), "EINVAL"), (dict(bias=ONE, bias_stride=-4), "EINVAL"),
    (dict(bias=ONE, bias_stride=4 * 22 - 1), "EINVAL"), (dict(n=0), "ECAPACITY")])
def test_scored_refusals(b, over, code):
    assert scored(b, **over) == getattr(b, "RS3_" + code)


def test_scored_sizes(b):
    assert scored(b, bank=b.BankDesc()) == b.RS3_EINVAL
    need = b.lib.rs3_scored_readout_workspace_bytes(ctypes.byref(_bank(b)), 20)
    assert scored(b, n=need - 1) == b.RS3_ECAPACITY
    assert b.lib.rs3_scored_readout_workspace_bytes(ctypes.byref(b.BankDesc()), 20) == 0
    assert b.lib.rs3_scored_readout_workspace_bytes(None, 20) == 0
    assert b.lib.rs3_scored_readout_workspace_bytes(ctypes.byref(_bank(b)), -1) == 0
    sizes = [b.lib.rs3_scored_readout_workspace_bytes(ctypes.byref(_bank(b)), k) for k in range(0, 65, 4)]
    assert sizes == sorted(sizes)
    assert scored(b, bank=_bank(b, d=48), d=48) == b.RS3_EUNSUPPORTED
    assert scored(b, bank=_bank(b, U=2049, ring=1 << 20)) == b.RS3_EUNSUPPORTED     # 2^31 rows


def shared(b, bank=None, prefix=None, of=ONE, rope=None, residual=None, out=ONE, scale=0.0, ws=ONE, n=BIG, status=ONE, **over):
    bank, prefix = _bank(b) if bank is None else bank, _bank(b, **FAR) if prefix is None else prefix
    return b.lib.rs3_shared_readout(*read_args(**over).values(), ctypes.byref(bank), ctypes.byref(prefix), of, rope, residual, out, scale, ws,
                                    n, status, None)


@pytest.mark.parametrize("over,code", READ_REFUSALS + [(dict(of=None), "EINVAL"), (dict(k_max=65), "EINVAL"), (dict(mn=65), "EINVAL"),
                                                       (dict(n=0), "ECAPACITY")])
def test_shared_refusals(b, over, code):
    assert shared(b, **over) == getattr(b, "RS3_" + code)


def test_shared_banks(b):
    assert shared(b, bank=b.BankDesc()) == b.RS3_EINVAL and shared(b, prefix=b.BankDesc()) == b.RS3_EINVAL
    for other in (dict(H=2), dict(d=32), dict(dtype="f32"), dict(mn=32)):
        assert shared(b, prefix=_bank(b, **FAR, **other)) == b.RS3_EINVAL
    need = b.lib.rs3_shared_readout_workspace_bytes(ctypes.byref(_bank(b)), ctypes.byref(_bank(b, **FAR)), 20)
    assert shared(b, n=need - 1) == b.RS3_ECAPACITY
    assert shared(b, bank=_bank(b, U=5000)) == b.RS3_EUNSUPPORTED and shared(b, prefix=_bank(b, U=5000, **FAR)) == b.RS3_EUNSUPPORTED
    known, none = ctypes.byref(_bank(b)), ctypes.byref(b.BankDesc())
    assert [b.lib.rs3_shared_readout_workspace_bytes(*a) for a in ((none, known, 5), (known, none, 5), (None, known, 5), (known, known, -1))] == [0] * 4
    sizes = [b.lib.rs3_shared_readout_workspace_bytes(known, known, k) for k in range(0, 65, 4)]
    assert sizes == sorted(sizes)


# ---------------------------------------------------------------------------
# the binding
# ---------------------------------------------------------------------------
class There(torch.Tensor):
    """A CPU tensor that calls itself one of device 0."""

    def get_device(self):
        return 0


def there(*shape, dtype=torch.int32):
    return torch.zeros(shape, dtype=dtype).as_subclass(There)


U, H, D, MN, K, F = 2, 2, 64, 16, 4, 3
bf, f32, u8 = torch.bfloat16, torch.float32, torch.uint8


@pytest.fixture()
def calls(b, monkeypatch):
    """(rs3, reached, make): make.name(**changes) calls the binding with tensors of the current device."""
    class Lib:
        def __getattr__(self, name):
            return (lambda *a: None) if name == "rs3_default_rope_spec" else lambda *a: reached.append(name) or 0

    reached = []
    monkeypatch.setattr(b, "lib", Lib())
    monkeypatch.setattr(torch.cuda, "current_device", lambda: 0)
    monkeypatch.setattr(b, "_stream", lambda s: 0)

    def bank():
        store = there(U, 32, H * D, dtype=bf)
        return types.SimpleNamespace(U=U, H=H, d=D, D=H * D, dtype="bf16", mn=MN, rows_per_unit=32, max_frames=F, desc=b.BankDesc(), k_store=store,
                                     v_store=store, meta=there(64, dtype=torch.int64))

    grid, st, out = there(1, MN, H * D, dtype=bf), there(1), there(U, MN, H * D, dtype=bf)
    read = (grid, "bf16", 1, MN, H, D, there(U), there(U, K), there(U), K)
    vec = there(H * D, dtype=f32)

    def scored(bank=bank(), bias=there(H, F + 2, dtype=f32), keep=there(U, F + 2, dtype=u8), res=None, out=out, ws=there(8, dtype=u8)):
        b.rs3_scored_readout(*read, bank, 5.0, bias, keep, None, res, out, 0.0, ws, st)

    def shared(bank=bank(), prefix=bank(), of=there(U), res=None, out=out, ws=there(8, dtype=u8)):
        b.rs3_shared_readout(*read, bank, prefix, of, None, res, out, 0.0, ws, st)

    def rows(q=grid, pos=there(MN, 1), keep=there(MN, dtype=u8), q_out=there(1, MN, H * D, dtype=bf)):
        b.rs3_rope_rows(q, q_out, pos, None, None, None, "bf16", H, 0, D, b.rope_spec(D), q_keep=keep)

    def table(pos=there(MN, 1), to=there(MN, D // 2, 2, dtype=f32)):
        b.rs3_rope_table(pos, b.rope_spec(D), to)

    def block(x=out, y=there(U, MN, H * D, dtype=bf), idx=there(U, K), count=there(U), gate=vec, status=st, h=there(U, MN, H * D, dtype=bf), **kw):
        b.rs3_norm_residual(y, x, None, h, "bf16", idx=idx, count=count, gate=gate, status=status, **kw)

    return b, reached, types.SimpleNamespace(rs3_scored_readout=scored, rs3_shared_readout=shared, rs3_rope_rows=rows, rs3_rope_table=table,
                                             rs3_norm_residual=block), bank


def test_calls_on_one_device_reach_the_library(calls):
    _, reached, make, _ = calls
    for name, call in vars(make).items():
        call()
        assert reached.pop() == name
    make.rs3_scored_readout(bias=None, keep=None, res=there(U, MN, H * D, dtype=bf))
    make.rs3_scored_readout(bias=there(U, H, F + 2, dtype=f32))
    make.rs3_norm_residual(idx=None, count=None, status=None, gate=there(U, H * D, dtype=f32), pre="layer", post="rms")
    make.rs3_rope_rows(keep=None)
    assert len(reached) == 4


@pytest.mark.parametrize("name,change", [
    ("rs3_scored_readout", dict(bias=torch.zeros(H, F + 2))), ("rs3_scored_readout", dict(bias=there(H, F + 1, dtype=f32))),
    ("rs3_scored_readout", dict(bias=there(3, H, F + 2, dtype=f32))), ("rs3_scored_readout", dict(bias=there(H, F + 2, dtype=torch.float64))),
    ("rs3_scored_readout", dict(keep=there(U, F, dtype=u8))), ("rs3_scored_readout", dict(keep=there(U, F + 2))),
    ("rs3_scored_readout", dict(keep=torch.zeros((U, F + 2), dtype=u8))), ("rs3_scored_readout", dict(ws=torch.zeros(8, dtype=u8))),
    ("rs3_scored_readout", dict(res=there(1, MN, H * D, dtype=bf))), ("rs3_scored_readout", dict(out=None)),
    ("rs3_shared_readout", dict(of=None)), ("rs3_shared_readout", dict(of=there(1))), ("rs3_shared_readout", dict(of=there(U, dtype=torch.int64))),
    ("rs3_shared_readout", dict(of=torch.zeros(U, dtype=torch.int32))), ("rs3_shared_readout", dict(ws=torch.zeros(8, dtype=u8))),
    ("rs3_shared_readout", dict(out=there(U, MN, H * D, dtype=f32))),
    ("rs3_rope_rows", dict(pos=there(MN - 1, 1))), ("rs3_rope_rows", dict(pos=None)), ("rs3_rope_rows", dict(pos=there(MN, 1, dtype=torch.int64))),
    ("rs3_rope_rows", dict(keep=there(MN - 1, dtype=u8))), ("rs3_rope_rows", dict(q=torch.zeros((1, MN, H * D), dtype=bf))),
    ("rs3_rope_rows", dict(q_out=there(1, MN - 1, H * D, dtype=bf))),
    ("rs3_rope_table", dict(pos=torch.zeros((MN, 1), dtype=torch.int32))), ("rs3_rope_table", dict(to=there(MN - 1, D // 2, 2, dtype=f32))),
    ("rs3_norm_residual", dict(x=there(MN, H * D, dtype=bf))), ("rs3_norm_residual", dict(y=there(1, MN, H * D, dtype=bf))),
    ("rs3_norm_residual", dict(gate=there(1, dtype=f32))), ("rs3_norm_residual", dict(gate=there(H * D, dtype=bf))),
    ("rs3_norm_residual", dict(gate=torch.zeros(H * D))), ("rs3_norm_residual", dict(idx=None)), ("rs3_norm_residual", dict(count=None)),
    ("rs3_norm_residual", dict(status=None)), ("rs3_norm_residual", dict(h=torch.zeros((U, MN, H * D), dtype=bf))),
    ("rs3_norm_residual", dict(pre_weight=there(3, H * D, dtype=f32)))])
def test_tensors_of_other_sizes_types_or_devices_are_refused(calls, name, change):
    _, reached, make, _ = calls
    with pytest.raises(ValueError):
        getattr(make, name)(**change)
    assert not reached


def test_banks_elsewhere_are_refused(calls):
    _, reached, make, bank = calls
    other = bank()
    other.k_store = torch.zeros(4)
    for call in (lambda: make.rs3_scored_readout(bank=other), lambda: make.rs3_shared_readout(bank=other), lambda: make.rs3_shared_readout(prefix=other)):
        with pytest.raises(ValueError, match="bank"):
            call()
    assert not reached


def test_a_prefix_on_another_stream_is_waited_for_and_waits(b, monkeypatch):
    from paper_2608_22526_gb300 import pipeline
    log = []

    class Stream:
        def __init__(self, name):
            self.name = name

        def __eq__(self, other):
            return self.name == other.name

        def wait_stream(self, other):
            log.append((self.name, "waits for", other.name))

    def pipe(stream):
        p = pipeline.Pipeline.__new__(pipeline.Pipeline)
        p.w = types.SimpleNamespace(dtype="bf16", G=1, mn=4, H=1, d=64)
        p.device, p.stream, p.bank, p.k_max = torch.device("cpu"), stream, types.SimpleNamespace(desc=None), 2
        p.unit_group = p.idx = p.count = p.status = None
        return p

    monkeypatch.setattr(torch.cuda, "stream", lambda s: contextlib.nullcontext())
    monkeypatch.setattr(pipeline.rs3, "rs3_shared_readout_workspace_bytes", lambda bank, prefix, k: 16)
    monkeypatch.setattr(pipeline.rs3, "rs3_shared_readout", lambda *a: log.append("call"))
    a, c = pipe(Stream("a")), pipe(Stream("c"))
    a.share(c, None)
    a.readout_shared(None, None, None)
    assert log == [("a", "waits for", "c"), "call", ("c", "waits for", "a")]
    log.clear()
    a.share(pipe(Stream("a")), None)
    a.readout_shared(None, None, None)
    assert log == ["call"]
