"""The recurrence's state carried in place, over chains of several tiles."""
import numpy as np
import pytest

import sequence_reference as ref

torch = pytest.importorskip("torch")
pytestmark = pytest.mark.gpu

LOW = {"bf16": torch.bfloat16, "f16": torch.float16, "f32": torch.float32}


@pytest.fixture(scope="module")
def rb():
    from paper_2510_23498_amd import binding
    binding.load_library()
    return binding


def _normal(rng, shape, dtype, std=1.0, mean=0.0):
    return torch.from_numpy((rng.standard_normal(shape) * std + mean).astype(np.float32)).to(dtype).cuda()


# tiles of 128 steps in windows of 16: two tiles, one window (whole, and one step more), several; channels by pairs and by ones
@pytest.mark.parametrize("T", [129, 200, 1000, 2048, 2049, 5000])
@pytest.mark.parametrize("B,D,share,low", [(2, 640, 1, "bf16"), (3, 131, 1, "f16"), (1, 256, 32, "f32")])
def test_state_and_its_gradient_in_place(rb, B, T, D, share, low):
    """The last tile of a chain writes hT over h0 (dh0 over dhT) while others run: what the first tile read is what all go by.  Gates
    that hold on to the state for thousands of steps, so that the state shows in every tile."""
    rng = np.random.default_rng(T + D)
    x, z = _normal(rng, (B, T, D), LOW[low]), _normal(rng, (B, T, D // share), LOW[low], 0.5, -8.0)
    h0, dh, dhT = _normal(rng, (B, D), torch.float32), _normal(rng, (B, T, D), LOW[low], 1e-3), _normal(rng, (B, D), torch.float32)
    h, hT, states = rb.rampde_recurrence_fwd(x, z, h0=h0, save_states=True)
    back = rb.rampde_recurrence_bwd(x, z, states, dh, dhT=dhT, h0=h0)
    want = ref.recurrence(*(t.double().cpu().numpy() for t in (x, z, h0)), None, dh.double().cpu().numpy(), dhT.double().cpu().numpy())
    for got, w, name, lo in ((h, want[0], "h", low), (hT, want[1], "hT", "f32"), (back[0], want[2], "dx", low), (back[2], want[4], "dh0", "f32")):
        # (thousands of steps that hardly contract: fp32 roundings of the state add up like their square root)
        ref.close(got.double().cpu().numpy(), w, lo, 16 * T, name)
    for _ in range(4):
        state, grad = h0.clone(), dhT.clone()
        again = rb.rampde_recurrence_fwd(x, z, h0=state, hT=state, save_states=True)
        assert again[1] is state
        for a, b in zip(again, (h, hT, states)):
            assert torch.equal(a, b)
        again = rb.rampde_recurrence_bwd(x, z, states, dh, dhT=grad, dh0=grad)
        assert again[2] is grad
        for a, b in zip(again, back):
            assert torch.equal(a, b)


@pytest.mark.parametrize("B,T,D,share,low", [(4, 1, 96, 1, "bf16"), (3, 70, 33, 1, "f16"), (2, 900, 256, 64, "f32")])
def test_last_state_alone(rb, B, T, D, share, low):
    """Without h, the other outputs have the same bits; a given h is written all the same"""
    rng = np.random.default_rng(T)
    x, z = _normal(rng, (B, T, D), LOW[low]), _normal(rng, (B, T, D // share), LOW[low])
    n = torch.tensor([T, 0, T // 2, T][:B], dtype=torch.int32, device="cuda")
    h, hT, states = rb.rampde_recurrence_fwd(x, z, lengths=n, save_states=True)
    none, hT2, states2 = rb.rampde_recurrence_fwd(x, z, lengths=n, save_states=True, want_h=False)
    assert none is None and torch.equal(hT, hT2) and torch.equal(states, states2)
    out = torch.zeros_like(h)
    assert rb.rampde_recurrence_fwd(x, z, lengths=n, h=out, want_h=False)[0] is out and torch.equal(out, h)
