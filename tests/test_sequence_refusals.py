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


def test_launches_of_more_threads_than_an_axis_has(lib):
    """2^32 threads along the axis: refused as unsupported before the launch, not reported as an error of it"""
    room = 1 << 60
    q, m = lib.rampde_fp8_quantize, lib.rampde_fp8_matmul
    assert q(rb.F32, 0, 1 << 28, 1, P, 0, P, P, None, None, None) == rb.EUNSUPPORTED          # 2^24 workgroups of 256
    assert q(rb.F32, 0, 1, 1 << 26, P, 0, P, P, None, None, None) == rb.EUNSUPPORTED          # (the other axis: 65535 workgroups)
    for mode, t in ((1, None), (2, P)):
        assert q(rb.F32, mode, 1, 1 << 30, P, 0, P, P, t, t, None) == rb.EUNSUPPORTED         # 2^23 workgroups of 512
        assert q(rb.F32, mode, 1 << 23, 1, P, 0, P, P, t, t, None) == rb.EUNSUPPORTED
    assert m(4, 1 << 26, 1, P, P, P, P, rb.F32, 0, P, 0, P, room, None) == rb.EUNSUPPORTED    # 2^22 workgroups of 1024
    assert m(1 << 20, 1 << 20, 1, P, P, P, P, rb.F32, 0, P, 0, P, room, None) == rb.EUNSUPPORTED
    r = rb._Recurrence(1 << 10, 1 << 11, 1 << 17, 1, rb.BF16)                                 # 2^20 blocks, 16 tiles each, of 512
    assert lib.rampde_recurrence_workspace_bytes(C.byref(r)) == 0
    assert lib.rampde_recurrence_fwd(C.byref(r), P, P, P, P, P, P, P, P, room, None) == rb.EUNSUPPORTED
    r = rb._Recurrence(1 << 10, 1, 1 << 17, 1, rb.BF16)                                       # (as many samples of one step fit)
    assert lib.rampde_recurrence_workspace_bytes(C.byref(r)) == 256


@pytest.mark.parametrize("D,gates", [(6, 2), (96, 2), (80, 1), (256, 1)])
def test_gates_of_other_numbers_of_channels_say_so(D, gates):
    torch = pytest.importorskip("torch")
    with pytest.raises(rb.RampdeError, match="power of two, at most 128") as e:
        rb._recurrence_plan(torch.bfloat16, (2, 3, D), (3 * D, D, 1), (2, 3, gates), (3 * gates, gates, 1), None)
    assert e.value.code == rb.EUNSUPPORTED


def test_rejected_arguments_come_with_the_reason():
    torch = pytest.importorskip("torch")
    with pytest.raises(rb.RampdeError) as e:   # (steps past 2^30)
        rb._recurrence_plan(torch.bfloat16, (1, 1 << 31, 2), (1 << 32, 2, 1), (1, 1 << 31, 2), (1 << 32, 2, 1), None)
    assert e.value.code == rb.EUNSUPPORTED
    lib = rb.load_library()
    for kw, code in ((dict(cols=16385), rb.EUNSUPPORTED), (dict(cols=0), rb.EINVAL)):
        j = C.byref(rb._Join(4, kw["cols"], rb.BF16, 1.0, 1e-6))
        with pytest.raises(rb.RampdeError) as e:
            rb._needed(int(lib.rampde_join_workspace_bytes(j)), lib.rampde_join_fwd, j)
        assert e.value.code == code


def test_unknown_modes_and_gradients_of_nothing():
    torch = pytest.importorskip("torch")
    with pytest.raises(ValueError, match="rows, cols, blocks"):
        rb._quantize_plan((2, 3), (3, 1), "diagonal")
    with pytest.raises(ValueError, match="dgate"):
        rb._like_of(None, torch.zeros(2, 3), None, "dgate")
    assert rb._like_of(None, None, None, "dgate") is None
