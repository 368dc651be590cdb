"""Arguments of the sequence operators that only a conversion or a launch would find out: refused on the host, without a GPU."""
import ctypes as C

import pytest

from paper_2510_23498_amd import binding as rb

P = C.c_void_p(1 << 20)  # (aligned, never touched: every call below is refused)


@pytest.fixture(scope="module")
def lib():
    return rb.load_library()


@pytest.mark.parametrize("bad", [dict(eps=1e-60), dict(eps=1e39), dict(alpha=1e300), dict(alpha=-4e38)])
def test_join_parameters_that_fp32_does_not_hold(lib, bad):
    """eps = 0 makes a row of zeros 0 * inf, alpha = inf one of dropped elements"""
    kw = {**dict(alpha=1.0, eps=1e-6), **bad}
    j = C.byref(rb._Join(4, 8, rb.BF16, kw["alpha"], kw["eps"], 0.0, 0, 0, 0, 0, 0))
    assert lib.rampde_join_workspace_bytes(j) == 0
    assert lib.rampde_join_fwd(j, *[P] * 9, None) == rb.EINVAL
    assert lib.rampde_join_bwd(j, *[P] * 16, 1 << 40, None) == rb.EINVAL
