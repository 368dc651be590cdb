"""Calls go to the GPU of their tensors, whichever is current."""
import contextlib
import types

import numpy as np
import pytest

torch = pytest.importorskip("torch")

from paper_2510_23498_amd import binding as rb  # noqa: E402


def test_the_tensors_gpu_is_current_during_a_call(monkeypatch):
    current = [0]

    @contextlib.contextmanager
    def device(d):
        before, current[0] = current[0], d.index
        yield
        current[0] = before
    monkeypatch.setattr(torch._C, "_cuda_getDevice", lambda: current[0], raising=False)
    monkeypatch.setattr(torch.cuda, "device", device)
    for index in (0, 1):
        assert rb._on(torch.device("cuda", index), lambda a, b: (a, b, current[0]), 5, 6) == (5, 6, index)
        assert current[0] == 0


def test_streams_are_those_of_the_tensors_gpu(monkeypatch):
    monkeypatch.setattr(torch._C, "_cuda_getCurrentRawStream", lambda index: 100 + index, raising=False)
    one = torch.device("cuda", 1)
    assert rb._stream_of(None, one) == 101
    assert rb._stream_of(types.SimpleNamespace(device=one, cuda_stream=7), one) == 7
    with pytest.raises(ValueError):
        rb._stream_of(types.SimpleNamespace(device=torch.device("cuda", 0), cuda_stream=7), one)


@pytest.mark.gpu
def test_every_call_is_made_on_the_tensors_gpu(monkeypatch):
    """With another GPU said to be current, each call still finds its own: launches under a guard, results as ever"""
    rb.load_library()
    calls, device = [], torch.device("cuda", 0)
    x = torch.ones(2, 5, 8, dtype=torch.bfloat16, device=device)
    y, b = torch.ones(4, 8, device=device), torch.ones(4, 8, dtype=torch.bfloat16, device=device)
    vel, tab, pol = rb.Velocity.mlp((8, 16, 8)), rb.Tableau([[0]], [1.0], [0]), rb.Policy(low="bf16")
    theta = torch.full((rb.rampde_num_params(vel),), 0.01, device=device)
    grid = np.linspace(0, 1, 3)

    def work():
        _, hT, states = rb.rampde_recurrence_fwd(x, x, save_states=True)
        dx = rb.rampde_recurrence_bwd(x, x, states, x)[0]
        y2, _, rstd = rb.rampde_join_fwd(rb.Join(), y, b, save_rstd=True)
        g = rb.rampde_join_bwd(rb.Join(), y2, b, rstd, y, b)
        q = rb.rampde_fp8_quantize(rb.rampde_dropout(b, 0.5, 1))
        p, short = rb.rampde_fp8_matmul(q, q), rb.rampde_fp8_matmul(q, q, short_sums=True)
        yN, ckpt = rb.rampde_odeint_fwd(vel, theta, y, grid, tab, pol)
        static = rb.rampde_odeint_fwd_static(vel, theta, y, grid, tab, pol, torch.empty_like(ckpt), torch.empty_like(yN))[0]
        back = rb.rampde_odeint_bwd(vel, theta, grid, tab, pol, ckpt, y)[0]
        back2, _, gt, _ = rb.rampde_odeint_bwd_tgrid(vel, theta, grid, tab, pol, ckpt, y)
        return [hT, dx, y2, g.db, p, short, yN, static, back, back2, gt]

    want = work()
    on, entered = rb._on, []

    class Guard(torch.cuda.device):
        def __init__(self, d):
            super().__init__(d)
            entered.append(d)
    monkeypatch.setattr(rb, "_on", lambda d, fn, *a: (calls.append((d, fn.__name__)), on(d, fn, *a))[1])
    monkeypatch.setattr(torch._C, "_cuda_getDevice", lambda: 1)
    monkeypatch.setattr(torch.cuda, "device", Guard)
    got = work()
    monkeypatch.undo()
    names = {n for _, n in calls}
    assert names == {n for n in rb.EXPORTS if n.endswith(("_fwd", "_bwd", "_tgrid", "dropout", "quantize", "matmul", "matmul_short"))} | \
        {"rampde_odeint_fwd_static"}
    assert all(d == device for d, _ in calls) and entered == [device] * len(calls)
    for u, v in zip(want, got):
        assert torch.equal(u, v)
