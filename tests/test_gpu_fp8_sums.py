"""Sums of the 8-bit product: in fp32 whatever the result's type, short ones only where the caller asks for them."""
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


def _np(t):
    return t.double().cpu().numpy()


def _operands(rb, M, N, K, seed):
    rng = np.random.default_rng(seed)
    a = torch.from_numpy((rng.standard_normal((M, K)) * np.exp(rng.standard_normal((M, 1)))).astype(np.float32)).cuda()
    b = torch.from_numpy((rng.standard_normal((N, K)) * 0.05).astype(np.float32)).cuda()
    return rb.rampde_fp8_quantize(a), rb.rampde_fp8_quantize(b, "blocks")[0]


# few rows, small tiles (in pieces, whole, of more than one turn of workgroups) and large ones: two blocks of the contraction, ten with a
# remainder, and eight, so that the scales' words and both slots come round again
SIZES = [(5, 70, 4200), (17, 130, 129), (129, 257, 1000), (1000, 1000, 520), (128, 16384, 2300), (2100, 4100, 200), (2100, 4100, 1200),
         (2304, 4096, 1024)]


@pytest.mark.parametrize("low", ["bf16", "f16", "f32"])
@pytest.mark.parametrize("M,N,K", SIZES)
def test_product_is_a_sum_in_fp32(rb, M, N, K, low):
    """Rounding of the result, and of fp32 sums in any order: 127 additions in a block of 128 products, one more for every block"""
    a, b = _operands(rb, M, N, K, M + N + K)
    da, db = _np(a.dequantize()), _np(b.dequantize())
    want, size = da @ db.T, np.abs(da) @ np.abs(db).T
    sums = 2.0 ** -24 * (K / 128 + 128) * size
    got = rb.rampde_fp8_matmul(a, b, dtype=LOW[low])
    assert (np.abs(_np(got) - want) <= ref.UNIT[low] * np.abs(want) + sums).all()
    assert torch.equal(got, rb.rampde_fp8_matmul(a, b, dtype=LOW[low]))
    if low == "f32":
        acc = torch.full((M, N), 3.0, device="cuda")
        rb.rampde_fp8_matmul(a, b, out=acc, accumulate=True)
        assert (np.abs(_np(acc) - want - 3) <= 2.0 ** -23 * (3 + np.abs(want)) + sums).all()


@pytest.mark.parametrize("low", ["bf16", "f16"])
@pytest.mark.parametrize("M,N,K", [(20, 3000, 512), (600, 500, 512), (2304, 4096, 512)])
def test_results_of_16_bits_are_the_nearest_ones(rb, M, N, K, low):
    """Of the results that are at least their root mean square r, those that are not nearest to the exact sum: it lies within the
    error e of the sum of a tie, and ties are u |v| >= u r apart, u the unit of the type, so a share of 2 e / (u r) of them at most.
    Sums in fp32 of K products are off by e = 2^-24 sqrt(K) r; short sums by 1.5e-5 r, a share seven times as large."""
    a, b = _operands(rb, M, N, K, 7 * M + N)
    a.scales.fill_(127)   # (rows of one size, so that r is one number)
    want = _np(a.dequantize()) @ _np(b.dequantize()).T
    r = np.sqrt(np.mean(want ** 2))
    big = np.abs(want) >= r
    near = _np(torch.from_numpy(want).to(LOW[low]))   # (fp64 to 16 bits, nearest even)
    got = _np(rb.rampde_fp8_matmul(a, b, dtype=LOW[low]))
    share = np.mean(got[big] != near[big])
    assert share <= 2 * 2.0 ** -24 * np.sqrt(K) / ref.UNIT[low], share


@pytest.mark.parametrize("low", ["bf16", "f16"])
def test_no_place_of_a_group_is_dropped(rb, low):
    """Two products of 2^8 that cancel, and one of 2^(8 - m - n) beside them, at every distance along the contraction"""
    def operand(t):
        values = t.to(torch.float8_e4m3fn)
        assert (values.float() == t).all()
        return rb.Fp8(values.view(torch.uint8).cuda(), torch.full((t.shape[0], 4), 127, dtype=torch.uint8).cuda(), 128)
    for rows in (16, 64):
        for at in (1, 2, 7, 8, 39, 41, 47, 100):
            a, b = torch.zeros(rows, 128), torch.ones(8, 128)
            a[:, 0], a[:, 40], a[:, at] = 256, -256, 2.0 ** (8 - torch.arange(rows).clamp(max=15).float())
            b[:, at] = 2.0 ** -torch.arange(8).float()
            got = rb.rampde_fp8_matmul(operand(a), operand(b), dtype=LOW[low]).float().cpu()
            m, n = torch.arange(rows).clamp(max=15)[:, None], torch.arange(8)[None]
            assert torch.equal(got, 2.0 ** (8 - m - n).float())


@pytest.mark.parametrize("low", ["bf16", "f16"])
@pytest.mark.parametrize("M,N,K", [(5, 33, 200), (31, 70, 4200), (129, 257, 1000), (1000, 1000, 520), (2100, 4100, 200), (2100, 4100, 1200)])
def test_short_sums_stay_within_what_the_instruction_drops(rb, M, N, K, low):
    """The 8-bit matrix instructions align 8 successive products to the largest and keep 13 binary places below its leading one: each of
    the other 7 loses less than 2^-13 of the largest.  Sums of the groups and blocks are fp32, cut off rather than rounded."""
    a, b = _operands(rb, M, N, K, M + N + K + 1)
    da, db = a.dequantize(), b.dequantize()
    tops = torch.zeros(M, N, device="cuda")
    for k in range(0, K, 8):
        tops += torch.stack([da[:, i, None].abs() * db[None, :, i].abs() for i in range(k, min(k + 8, K))]).amax(0)
    want, size = _np(da) @ _np(db).T, np.abs(_np(da)) @ np.abs(_np(db)).T
    sums = 7 * 2.0 ** -13 * _np(tops) * (1 + 1e-5) + 2.0 ** -23 * (K / 8 + 8) * size
    out = torch.full((M, N + 5), 7.0, dtype=LOW[low], device="cuda")
    got = rb.rampde_fp8_matmul(a, b, out=out[:, 2:2 + N], short_sums=True)
    assert (out[:, :2] == 7).all() and (out[:, 2 + N:] == 7).all()
    assert (np.abs(_np(got) - want) <= ref.UNIT[low] * np.abs(want) + (1 + ref.UNIT[low]) * sums + 2.0 ** -25).all()
    assert torch.equal(got, rb.rampde_fp8_matmul(a, b, dtype=LOW[low], short_sums=True))


def test_short_sums_keep_13_places(rb):
    """What the precision notes say of the 8-bit matrix instructions, on products 2^-j of two that cancel"""
    def operand(t):
        return rb.Fp8(t.to(torch.float8_e4m3fn).view(torch.uint8).cuda(), torch.full((t.shape[0], 4), 127, dtype=torch.uint8).cuda(), 128)
    for rows in (16, 64):
        for at, places in ((2, 13), (7, 13), (8, 23), (100, 23)):
            a, b = torch.zeros(rows, 128), torch.ones(8, 128)
            a[:, 0], a[:, 40], a[:, at] = 256, -256, 2.0 ** (8 - torch.arange(rows).clamp(max=15).float())
            b[:, at] = 2.0 ** -torch.arange(8).float()
            got = rb.rampde_fp8_matmul(operand(a), operand(b), dtype=torch.bfloat16, short_sums=True).float().cpu()
            for m in range(min(rows, 16)):
                for n in range(8):
                    assert (got[m, n] == 2.0 ** (8 - m - n)) == (m + n <= places), (at, m, n)


def test_short_sums_of_fp32_results_are_refused(rb):
    a, b = _operands(rb, 4, 5, 6, 0)
    for kw in (dict(dtype=torch.float32), dict(out=torch.zeros(4, 5, device="cuda"), accumulate=True)):
        with pytest.raises(ValueError):
            rb.rampde_fp8_matmul(a, b, short_sums=True, **kw)


@pytest.mark.parametrize("low", ["bf16", "f16", "f32"])
@pytest.mark.parametrize("M,N", [(16, 40), (29, 70), (127, 20), (300, 200), (2100, 4100)])
def test_scales_at_both_ends_of_their_range(rb, low, M, N):
    """Every scale that a block can have, against one that brings the product back to about 1: two products of 4 x 4 places a result, whose
    sum is exact where fp32 holds it, and off by a unit of the larger product's last place where they are further apart.  Few rows,
    small and large tiles, either operand."""
    rng = np.random.default_rng(M)
    every = torch.arange(127, dtype=torch.uint8)   # all finite values from 0 up

    def operand(rows, scales, values):
        v = torch.zeros(rows, 256, dtype=torch.uint8)
        v[:, 3], v[:, 200] = values, values.flip(0)
        s = torch.full((rows, 4), 127, dtype=torch.uint8)
        s[:, 0], s[:, 1] = scales, scales
        return rb.Fp8(v.cuda(), s.cuda(), 256)
    for scale in (0, 1, 2, 3, 4, 60, 244, 246, 247, 248, 254):
        a = torch.full((M,), 127, dtype=torch.uint8)
        a[rng.integers(0, M, max(1, M // 40))] = scale   # (a few rows of many)
        b = torch.full((N,), 127, dtype=torch.uint8)
        b[rng.integers(0, N, max(1, N // 40))] = 254 - scale
        va, vb = every[torch.arange(M) % 127], every[(torch.arange(N) * 5 + 64) % 127]
        x, y = operand(M, a, va), operand(N, b, vb)
        for p, q in ((x, y), (y, x)):
            d = [t.values.view(torch.float8_e4m3fn).double()[:, [3, 200]] * torch.exp2(t.scales[:, :1].double() - 127) for t in (p, q)]
            want = d[0] @ d[1].T
            keep = want.abs() < 2.0 ** 127   # (infinite, or on the way there, otherwise)
            got = rb.rampde_fp8_matmul(p, q, dtype=LOW[low])
            top = (d[0][:, :1] * d[1][:, 0]).abs().maximum((d[0][:, 1:] * d[1][:, 1]).abs())
            exact = keep & ((low != "f32") | (want.float().double() == want))
            assert torch.equal(got[exact], want.float().to(LOW[low])[exact]), scale
            assert ((got.double() - want).abs() <= 2.0 ** -23 * top)[keep & ~exact].all(), scale
            if low != "f32":
                assert torch.equal(rb.rampde_fp8_matmul(p, q, dtype=LOW[low], short_sums=True)[keep], got[keep]), scale
        assert not torch.isnan(rb.rampde_fp8_matmul(x, y, dtype=LOW[low])).any()


def test_rows_of_the_smallest_and_largest_numbers(rb):
    """Quantised from fp32: rows of 2^-135 and of 3.4e38 (which rounds to 2^128) against columns that bring them back"""
    x = torch.zeros(40, 130, device="cuda")
    x[:, 0], x[:, 129] = 1.0, 1.0
    x[3, 0], x[3, 129], x[17, 0], x[17, 129] = 2.0 ** -135, 2.0 ** -134, 3.4e38, 3.4e38
    w = torch.zeros(50, 130, device="cuda")
    w[:, 0], w[:, 129] = 1.0, 2.0
    w[5, 0], w[6, 0] = 2.0 ** 120, 2.0 ** -120
    got = rb.rampde_fp8_matmul(rb.rampde_fp8_quantize(x), rb.rampde_fp8_quantize(w), dtype=torch.float32)
    assert got[3, 5] == 2.0 ** -15 + 2.0 ** -133 and got[17, 6] == float("inf") and got[0, 5] == 2.0 ** 120
    assert got[3, 0] == 2.0 ** -135 + 2.0 ** -133 and (got[[0, 1, 2, 4, 39]][:, :5] == 3.0).all()
    w[:, 129] = 0
    got = rb.rampde_fp8_matmul(rb.rampde_fp8_quantize(x), rb.rampde_fp8_quantize(w), dtype=torch.float32)
    assert got[17, 6] == 2.0 ** 8 and got[17, 0] == float("inf") and got[17, 5] == float("inf")


@pytest.mark.parametrize("M,N", [(16, 40), (29, 70), (300, 200), (2100, 4100)])
def test_sums_up_to_the_largest_number(rb, M, N):
    """One product of ones against powers of two, up to 2^127, and sums past it"""
    x, w = torch.zeros(M, 256, device="cuda"), torch.zeros(N, 256, device="cuda")
    x[:, 7], x[:, 250] = 1.0, 1.0
    e = torch.arange(N, device="cuda") % 16 + 112.0   # 2^112 to 2^127
    w[:, 7] = torch.exp2(e)
    got = rb.rampde_fp8_matmul(rb.rampde_fp8_quantize(x), rb.rampde_fp8_quantize(w), dtype=torch.float32)
    assert (got == torch.exp2(e)).all()
    w[:, 250] = w[:, 7]
    got = rb.rampde_fp8_matmul(rb.rampde_fp8_quantize(x), rb.rampde_fp8_quantize(w), dtype=torch.bfloat16)
    assert (got.float() == torch.exp2(e + 1)).all()   # (infinite for 2^128)
    w[:, 250] = -w[:, 7]
    got = rb.rampde_fp8_matmul(rb.rampde_fp8_quantize(x), rb.rampde_fp8_quantize(w), dtype=torch.float32)
    assert (got == 0).all()
    x[3, 9] = float("nan")
    got = rb.rampde_fp8_matmul(rb.rampde_fp8_quantize(x), rb.rampde_fp8_quantize(w), dtype=torch.float32)
    assert torch.isnan(got[3]).all() and (got[[i for i in range(M) if i != 3]] == 0).all()
