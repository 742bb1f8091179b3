"""Refusals of rs3_rope_table, rs3_rope_rows and rs3_norm_residual on the host.  CPU only: no call here reaches a kernel."""
import ctypes

import pytest

P = 0x10000                                                # an aligned address that nothing reads


@pytest.fixture(scope="module")
def rs3():
    from paper_2608_22526_gb300 import _build
    _build.build()
    from paper_2608_22526_gb300 import rs3
    return rs3


def rope(rs3, spec, q=P, rows=4, stride=64, H=1, pos=P, out=2 * P, out_stride=64, dtype=0, d=64):
    return rs3.lib.rs3_rope_rows(q, rows, stride, H, pos, None, out, out_stride, None, 0, 0, 0, None, None, None, 0, dtype, d,
                                 ctypes.byref(spec), None)


def test_struct_sizes_match_the_header(rs3):
    assert ctypes.sizeof(rs3.RopeSpec) == 72
    assert ctypes.sizeof(rs3.Norm) == 40


def test_rope_spec_defaults(rs3):
    s = rs3.rope_spec(64)
    assert (s.layout, s.rot, s.axes, list(s.pairs), s.inverse) == (0, 64, 1, [32, 0, 0], 0)
    assert (s.base, s.factor, s.context, s.beta_fast, s.beta_slow, s.magnitude) == (10000.0, 1.0, 0.0, 32.0, 1.0, 1.0)
    for bad in ([], [1, 1, 1, 1]):
        with pytest.raises(ValueError):
            rs3.rope_spec(8, bad)
    with pytest.raises(KeyError):
        rs3.rope_spec(8, layout="quarters")


@pytest.mark.parametrize("change", [dict(rot=0), dict(rot=3), dict(rot=66), dict(axes=0), dict(axes=4), dict(layout=2), dict(base=0.5),
                                    dict(base=float("nan")), dict(factor=0.5), dict(factor=float("inf")), dict(context=-1.0),
                                    dict(magnitude=float("nan")), dict(context=10.0, beta_fast=1.0, beta_slow=1.0)])
def test_rope_specs_that_are_none(rs3, change):
    s = rs3.rope_spec(64)
    for k, v in change.items():
        setattr(s, k, v)
    assert rope(rs3, s) == rs3.RS3_EINVAL


@pytest.mark.parametrize("pairs", [[31], [33], [40, -8], [16, 8]])
def test_rope_pairs_that_do_not_add_up(rs3, pairs):
    assert rope(rs3, rs3.rope_spec(64, pairs)) == rs3.RS3_EINVAL


@pytest.mark.parametrize("change", [dict(q=None), dict(out=None), dict(pos=None), dict(q=P + 8), dict(out=2 * P + 4), dict(pos=P + 2), dict(rows=-1),
                                    dict(H=0), dict(stride=60), dict(stride=66), dict(out_stride=63), dict(out=P, out_stride=128),
                                    dict(out=P + 256), dict(d=66), dict(dtype=2), dict(d=0)])
def test_rope_refuses(rs3, change):
    assert rope(rs3, rs3.rope_spec(64 if change.get("d", 64) >= 64 else 2), **change) == rs3.RS3_EINVAL


def test_rope_heads_that_are_too_wide(rs3):
    assert rope(rs3, rs3.rope_spec(64), d=264, stride=264, out_stride=264) == rs3.RS3_EUNSUPPORTED
    assert rope(rs3, rs3.rope_spec(264), d=264, stride=264, out_stride=264) == rs3.RS3_EUNSUPPORTED
    assert rs3.lib.rs3_rope_table(P, 4, ctypes.byref(rs3.rope_spec(264)), P, None) == rs3.RS3_EUNSUPPORTED


def test_rope_table_refuses(rs3):
    s = ctypes.byref(rs3.rope_spec(64))
    for a in ((None, 4, s, P), (P, 4, s, None), (P + 2, 4, s, P), (P, 4, s, P + 8), (P, -1, s, P), (P, 4, None, P)):
        assert rs3.lib.rs3_rope_table(*a, None) == rs3.RS3_EINVAL


def test_nothing_to_do_is_fine(rs3):
    s = rs3.rope_spec(64)
    assert rope(rs3, s, q=None, rows=0, out=None, pos=None) == rs3.RS3_OK
    assert rs3.lib.rs3_rope_table(None, 0, ctypes.byref(s), None, None) == rs3.RS3_OK
    assert block(rs3, idx=P, count=P, k_max=0, status=P) == rs3.RS3_OK


def block(rs3, y=P, x=4 * P, dtype=0, U=2, mn=16, C=64, idx=None, count=None, k_max=0, post=None, gate=None, gate_stride=0, alpha=1.0,
          pre=None, x_out=8 * P, h_out=12 * P, status=None):
    n = [None if v is None else ctypes.byref(v) for v in (post, pre)]
    return rs3.lib.rs3_norm_residual(y, x, dtype, U, mn, C, idx, count, k_max, n[0], gate, gate_stride, alpha, n[1], x_out, h_out,
                                     status, None)


def norm(rs3, kind=1, eps=1e-6, weight=None, bias=None, weight_stride=0, bias_stride=0):
    return rs3.Norm(kind, eps, weight, bias, weight_stride, bias_stride)


@pytest.mark.parametrize("change", [
    dict(x=None), dict(x_out=None, h_out=None), dict(U=0), dict(mn=0), dict(C=0), dict(C=66), dict(dtype=3), dict(x=4 * P + 8), dict(y=P + 4),
    dict(x_out=8 * P + 8), dict(h_out=12 * P + 8), dict(idx=P), dict(count=P), dict(idx=P, count=P, k_max=-1, status=P),
    dict(idx=P, count=P, k_max=17, status=P), dict(idx=P, count=P, k_max=4), dict(alpha=float("nan")), dict(alpha=float("inf")),
    dict(gate=P + 8), dict(gate=P, gate_stride=32), dict(gate=P, gate_stride=66),
    # results that lie over an operand or each other
    dict(x_out=4 * P + 256), dict(h_out=P + 256), dict(x_out=8 * P, h_out=8 * P), dict(h_out=8 * P + 256)])
def test_block_refuses(rs3, change):
    assert block(rs3, **change) == rs3.RS3_EINVAL


@pytest.mark.parametrize("change", [dict(kind=3), dict(kind=-1), dict(eps=-1.0), dict(eps=float("nan")), dict(weight=P + 8),
                                    dict(bias=P, bias_stride=32), dict(weight=P, weight_stride=65)])
def test_block_norms_that_are_none(rs3, change):
    assert block(rs3, post=norm(rs3, **change)) == rs3.RS3_EINVAL
    assert block(rs3, pre=norm(rs3, **change)) == rs3.RS3_EINVAL


def test_block_sizes_past_the_limits(rs3):
    for change in (dict(C=4104), dict(mn=16385), dict(U=65536)):
        assert block(rs3, **{**dict(U=1, mn=1, C=8), **change}) == rs3.RS3_EUNSUPPORTED
