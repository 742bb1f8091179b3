"""The limits of a rotation's description, as the header has them.  CPU only: no call here reaches a kernel."""
import ctypes
import os

import pytest

HEADER = os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "include", "rs3.h")


@pytest.fixture(scope="module")
def rs3():
    from paper_2608_22526_gb300 import _build
    _build.build()
    from paper_2608_22526_gb300 import rs3
    return rs3


LIMITS = [("base", 1.0, 0.99), ("base", 1e12, 1.01e12), ("factor", 1.0, 0.99), ("factor", 1e9, 1.01e9), ("context", 0.0, -1.0), ("context", 1e12, 1.01e12),
          ("beta_fast", 1e12, 1.01e12), ("magnitude", 9.9e29, 1e30), ("magnitude", -9.9e29, -1e30), ("beta_slow", 0.0, -0.1)]


@pytest.mark.parametrize("field,last,past", LIMITS)
def test_the_last_value_is_taken_and_the_next_refused(rs3, field, last, past):
    for value, code in ((last, rs3.RS3_OK), (past, rs3.RS3_EINVAL)):
        s = rs3.rope_spec(64, context=100.0)
        setattr(s, field, value)
        assert rs3.lib.rs3_rope_table(None, 0, ctypes.byref(s), None, None) == code


def test_the_header_names_them():
    with open(HEADER) as f:
        spec = f.read().split("How a head turns.")[1].split("} rs3_rope_spec;")[0]
    for limit in ("1 <= base <= 1e12", "1 <= factor <= 1e9", "0 <= context <= 1e12", "0 <= slow < fast <= 1e12", "|magnitude| < 1e30"):
        assert limit in spec, limit
