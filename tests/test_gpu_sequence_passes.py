"""Sequence operators where a kernel goes round more than once, and where offsets pass 32 bits."""
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
    return torch.from_numpy((rng.standard_normal(shape, dtype=np.float32) * np.float32(std) + np.float32(mean))).to(dtype).cuda()


def _np(t):
    return None if t is None else t.double().cpu().numpy()


def _mask(n, p, seed, offset):
    """ref.mask, all counters at a time"""
    word, s32 = np.uint64(0xFFFFFFFF), np.uint64(32)
    ctr = np.arange((n + 7) // 8, dtype=np.uint64) + np.uint64(offset)
    c = [ctr & word, ctr >> s32, np.zeros_like(ctr), np.zeros_like(ctr)]
    k = [seed & 0xFFFFFFFF, seed >> 32 & 0xFFFFFFFF]
    for _ in range(10):
        p0, p1 = np.uint64(0xD2511F53) * c[0], np.uint64(0xCD9E8D57) * c[2]
        c = [(p1 >> s32) ^ c[1] ^ np.uint64(k[0]), p1 & word, (p0 >> s32) ^ c[3] ^ np.uint64(k[1]), p0 & word]
        k = [(k[0] + 0x9E3779B9) & 0xFFFFFFFF, (k[1] + 0xBB67AE85) & 0xFFFFFFFF]
    halves = np.stack([w >> np.uint64(s) & np.uint64(0xFFFF) for w in c for s in (0, 16)], 1).ravel()[:n]
    drop = int(round(p * 65536))
    return np.where(halves >= drop, 65536.0 / (65536 - drop), 0.0)


def test_the_mask_of_these_tests():
    for n, p, seed, offset in ((1, 0.3, 1, 0), (1001, 0.25, 77 << 33, (1 << 32) - 5)):
        assert np.array_equal(_mask(n, p, seed, offset), ref.mask(n, p, seed, offset))


# The backward pass has at most 512 workgroups: more than 512 times their rows, the last turn incomplete; rows of 8, 16, 32 and 64 lanes and of
# 2, 4, 8 and 16 wavefronts.  The last one: more rows than the forward pass's 65536 workgroups take at a time, too.
PASSES = [(40003, 50, "bf16", 0.0), (20001, 100, "f16", 0.1), (10001, 250, "bf16", 0.1), (5001, 300, "f32", 0.2), (5000, 513, "bf16", 0.1),
          (1500, 2048, "bf16", 0.1), (700, 4096, "f16", 0.1), (1025, 4100, "bf16", 0.0), (600, 9001, "bf16", 0.1), (2100001, 5, "f32", 0.0)]


@pytest.mark.parametrize("rows,cols,low,p", PASSES)
def test_join_of_more_rows_than_one_turn_takes(rb, rows, cols, low, p):
    rng = np.random.default_rng(rows)
    y, b, gate = _normal(rng, (rows, cols), torch.float32, 2.0), _normal(rng, (rows, cols), LOW[low]), _normal(rng, (rows, cols), LOW[low])
    par = {k: _normal(rng, (cols,), torch.float32, 0.3, 1.0) for k in ("w_post", "scale", "w_pre")}
    dy_out, dx = _normal(rng, (rows, cols), torch.float32), _normal(rng, (rows, cols), LOW[low])
    # (rows of few columns that happen to be small have large gradients, which would be all that the tolerance looks at)
    y += torch.sign(y)
    b += torch.sign(b)
    j = rb.Join(alpha=0.5, eps=1e-5, p=p, seed=77 << 33, offset=(1 << 32) - 5)
    y2, x, rstd = rb.rampde_join_fwd(j, y, b, gate=gate, **par, save_rstd=True)
    g = rb.rampde_join_bwd(j, y2, b, rstd, dy_out, dx, gate=gate, **par)
    k = _mask(rows * cols, p, 77 << 33, (1 << 32) - 5).reshape(rows, cols) if p else None
    wy, wx, wr, wg = ref.join(_np(y), _np(b), _np(gate), *(_np(par[n]) for n in ("w_post", "scale", "w_pre")), 0.5, 1e-5, k, _np(dy_out),
                              _np(dx))
    ref.close(_np(y2), wy, "f32", cols, "y'")
    ref.close(_np(x), wx, low, cols, "x")
    ref.close(_np(rstd), wr, "f32", cols, "rstd")
    for name, w in wg.items():
        ref.close(_np(getattr(g, name)), w, low if name in ("db", "dgate") else "f32", cols + (rows if name.startswith("dw") or name == "dscale" else 0),
                  name)


@pytest.mark.parametrize("low", ["bf16", "f32"])
def test_dropout_of_more_elements_than_one_turn_takes(rb, low):
    """4096 workgroups of 2048 elements at a time: 8388608"""
    n = 9000003
    x = _normal(np.random.default_rng(3), (n,), LOW[low])
    k = torch.from_numpy(_mask(n, 0.25, 5 << 34, (1 << 32) - 9)).cuda()
    out = rb.rampde_dropout(x, 0.25, 5 << 34, (1 << 32) - 9)
    # (a factor of 4 / 3 in fp32, rounded, and the product, rounded, to fp32 and then to the type)
    want = x.double() * k
    assert torch.equal(out == 0, want == 0)
    assert ((out.double() - want).abs() <= (ref.UNIT[low] + 2.0 ** -22) * want.abs()).all()


@pytest.mark.parametrize("D,share", [(64, 1), (33, 1), (96, 32)])
@pytest.mark.parametrize("low,apart", [("bf16", 1 << 31), ("f16", 1 << 30), ("f32", 1 << 30)])
def test_samples_far_apart(rb, low, apart, D, share):
    """Samples from 2^31 bytes to 2^32 bytes behind one another, x, z and their gradients alike, forward and backward: the results of
    neighbouring ones, to rounding"""
    B, T = 2, 150
    rng = np.random.default_rng(D + share)
    apart += 64

    def far(shape):
        return torch.empty(B * apart, dtype=LOW[low], device="cuda").as_strided(shape, (apart, shape[2], 1))
    x0, z0, dh = _normal(rng, (B, T, D), LOW[low]), _normal(rng, (B, T, D // share), LOW[low]), _normal(rng, (B, T, D), LOW[low])
    h0, dhT = _normal(rng, (B, D), torch.float32), _normal(rng, (B, D), torch.float32)
    n = torch.tensor([T, 70], dtype=torch.int32, device="cuda")
    h, hT, states = rb.rampde_recurrence_fwd(x0, z0, h0=h0, lengths=n, save_states=True)
    back = rb.rampde_recurrence_bwd(x0, z0, states, dh, dhT=dhT, lengths=n, h0=h0)
    x, z, dx, dz = far(x0.shape), far(z0.shape), far(x0.shape), far(z0.shape)
    x.copy_(x0)
    z.copy_(z0)
    again = rb.rampde_recurrence_fwd(x, z, h0=h0, lengths=n, save_states=True)
    for u, v, name, lo in zip(again, (h, hT, states), ("h", "hT", "states"), (low, "f32", "f32")):
        ref.close(_np(u), _np(v), lo, 16, name)
    rb.rampde_recurrence_bwd(x, z, states, dh, dhT=dhT, lengths=n, h0=h0, dx=dx, dz=dz)
    for u, v, name in ((dx, back[0], "dx"), (dz, back[1], "dz")):
        ref.close(_np(u), _np(v), low, 16 * share, name)


@pytest.mark.parametrize("low,apart,share", [("bf16", 1 << 27, 1), ("f32", 1 << 26, 2)])
def test_steps_far_apart(rb, low, apart, share):
    """Sixteen steps over more than 2^31 bytes, with time as the slowest index"""
    B, T, D = 3, 20, 10
    rng = np.random.default_rng(share)

    def far(last):
        return torch.empty(T * apart, dtype=LOW[low], device="cuda").as_strided((B, T, last), (last, apart, 1))
    x0, z0, dh = _normal(rng, (B, T, D), LOW[low]), _normal(rng, (B, T, D // share), LOW[low]), _normal(rng, (B, T, D), LOW[low])
    x, z, dx, dz = far(D), far(D // share), far(D), far(D // share)
    x.copy_(x0)
    z.copy_(z0)
    want = ref.recurrence(_np(x0), _np(z0), None, None, _np(dh))
    h, hT, states = rb.rampde_recurrence_fwd(x, z, save_states=True)
    rb.rampde_recurrence_bwd(x, z, states, dh, dx=dx, dz=dz)
    for got, w, name, lo in ((h, want[0], "h", low), (hT, want[1], "hT", "f32"), (dx, want[2], "dx", low), (dz, want[3], "dz", low)):
        ref.close(_np(got), w, lo, 16 * share, name)
