"""Rotations by far angles, against cosine and sine of many digits: up to 2^47 the nearest fp32 numbers, NaN beyond."""
import ctypes
import decimal
import math

import numpy as np
import pytest

from oracle import kv_cache as kvo

import paged

torch = pytest.importorskip("torch")
FAR = 2.0 ** 47
HALF = 2.0 ** -24          # half a step of fp32, relative


def _pi():
    """pi to 90 digits by Machin's formula, in whole numbers."""
    one = 10 ** 100

    def arctan_inverse(x):
        term, total, n, sign = one // x, 0, 1, 1
        while term:
            total, term, n, sign = total + sign * (term // n), term // (x * x), n + 2, -sign
        return total
    with decimal.localcontext() as c:
        c.prec = 90
        return decimal.Decimal(4 * (4 * arctan_inverse(5) - arctan_inverse(239))) / one


def cos_sin(theta):
    """(cos, sin) of a float of any size, as decimals of 40 digits behind the point at least."""
    with decimal.localcontext() as c:
        c.prec = 80
        quarter = _PI / 2
        x = decimal.Decimal(theta)
        k = (x / quarter).to_integral_value()
        r = x - k * quarter
        terms, total = [decimal.Decimal(1)], [decimal.Decimal(0), decimal.Decimal(0)]
        for n in range(1, 60):
            terms.append(terms[-1] * r / n)
        for n, t in enumerate(terms):
            total[n & 1] += -t if n & 2 else t
        cos, sin = total
        return ((cos, sin), (-sin, cos), (-cos, -sin), (sin, -cos))[int(k) % 4]


_PI = _pi()


def test_the_reference_itself():
    assert str(_PI).startswith("3.14159265358979323846264338327950288419716939937510582097494459")
    for x in (0.0, 1.0, -2.5, 3.0, 100.0, -12345.678, 1e6):
        c, s = cos_sin(x)
        assert abs(float(c) - math.cos(x)) < 1e-15 and abs(float(s) - math.sin(x)) < 1e-15
        with decimal.localcontext() as digits:
            digits.prec = 80
            assert abs(c * c + s * s - 1) < decimal.Decimal(10) ** -60


def test_frequencies_that_are_no_number():
    import paper_2304_01089_amd as rp
    lib = rp.load_library()
    freqs, amplitude = np.zeros(512), ctypes.c_double()
    call = lambda base, scaling=0, factor=1.0: lib.rptq_rope_freqs(1024, base, scaling, factor, 4096.0, 1.0, 32.0, freqs.ctypes.data_as(ctypes.c_void_p), ctypes.byref(amplitude))     # noqa: E731
    assert call(5e-324) == -6 and call(5e-324, 3, 2.0) == -6
    assert call(1e-300) == 0 and np.isfinite(freqs).all() and freqs[-1] > 1e298
    assert call(5e-324, 1, 1e300) in (0, -6) and call(1e308, 2, 1.0) == 0


FREQS = np.array([2.0 ** 16, np.nextafter(2.0 ** 16, 0), 65535.9, 54321.0987654321, np.pi * 2 ** 14, 12345.678, 32768.0, 1e3, 25.0, 1.0, 1e-3, 1e-9, -777.7, -65536.0, 0.5 * np.pi, 4e4])


@pytest.mark.gpu
@pytest.mark.parametrize("interleaved", [False, True])
def test_cosines_and_sines_of_far_angles(interleaved):
    import paper_2304_01089_amd as rp
    rng = np.random.default_rng(5)
    positions = np.concatenate([[2 ** 31 - 1, -2 ** 31, -(2 ** 31 - 1), 2 ** 30 + 12345], rng.integers(-2 ** 31, 2 ** 31, 60)]).astype(np.int32)
    T, pairs = len(positions), len(FREQS)
    j = np.arange(pairs)
    first, second = (2 * j, 2 * j + 1) if interleaved else (j, j + pairs)
    x = np.zeros((T, 2 * pairs), np.float32)
    x[:, first] = 1.0                                             # (a pair becomes its cosine and sine)
    rot = rp.Rotary(2 * pairs, torch.from_numpy(FREQS).cuda(), interleaved=interleaved)
    got = rp.rope(rot, torch.from_numpy(x).cuda(), torch.from_numpy(positions).cuda(), 2 * pairs).double().cpu().numpy()
    for t, p in enumerate(positions):
        for i, f in enumerate(FREQS):
            theta = float(p) * f
            assert abs(theta) <= FAR
            for at, want in zip((first[i], second[i]), cos_sin(theta)):
                # (half a step of fp32, and what the 64-bit number before it was off by)
                near = abs(want) * decimal.Decimal(HALF * (1 + 2.0 ** -26)) + decimal.Decimal(2.0 ** -62)
                assert abs(decimal.Decimal(float(got[t, at])) - want) <= near, (p, f)


@pytest.mark.gpu
@pytest.mark.parametrize("interleaved", [False, True])
def test_angles_beyond_become_nan(interleaved):
    """Alone and in front of the cache; nothing else of the rows does."""
    import paper_2304_01089_amd as rp
    H, hd, bits, page, pairs = 2, 64, 4, 16, 16
    positions = np.array([-2 ** 31, 2 ** 31 - 1, 0, 1], np.int32)
    freqs = np.full(pairs, 0.25)
    freqs[:6] = [2.0 ** 16, np.nextafter(2.0 ** 16, 1e9), 1e20, np.inf, np.nan, -2.0 ** 200]
    with np.errstate(invalid="ignore"):
        far = ~(np.abs(positions.astype(np.float64)[:, None] * freqs) <= FAR)
    assert far[0].sum() == 5 and far[2].sum() == 2 and far[3].sum() == 4
    j = np.arange(pairs)
    first, second = (2 * j, 2 * j + 1) if interleaved else (j, j + pairs)
    none = np.zeros((4, hd), bool)
    none[:, first], none[:, second] = far, far
    none = np.tile(none, (1, H))
    hc, lo, hi = paged.clusters(H, hd, bits, 3, 4)
    table = torch.from_numpy(paged.table_rows(hc)).cuda()
    k = torch.from_numpy(paged.values(np.random.default_rng(1), lo, hi, 4)).cuda().bfloat16()
    rot, near = (rp.Rotary(2 * pairs, torch.from_numpy(f).cuda(), interleaved=interleaved) for f in (freqs, np.where(far.any(0), 0.0, freqs)))
    pos = torch.from_numpy(positions).cuda()
    turned = rp.rope(rot, k.float(), pos, hd).cpu().numpy()
    plain = rp.rope(near, k.float(), pos, hd).cpu().numpy()
    assert np.array_equal(np.isnan(turned), none)
    whole = np.tile(np.isin(np.arange(hd), np.concatenate([first[far.any(0)], second[far.any(0)]])), H)
    assert np.array_equal(turned[:, ~whole], plain[:, ~whole])
    cache = rp.paged_cache(1, page, H, hd, bits, table, table)
    q = rp.rope_quant_paged(cache, rot, k, k, k, pos, torch.arange(4, device="cuda"))
    assert np.array_equal(np.isnan(q.float().cpu().numpy()), none)
    assert np.array_equal(q.float().cpu().numpy()[~none], kvo.round_to_bf16(turned)[~none])
    codes = kvo.kv_quant(np.where(none, 0.0, turned).astype(np.float32), hc, 0, bits)
    back = kvo.kv_dequant(codes, hc, 0, original_order=True)
    got = rp.kv_dequant_paged(cache, torch.arange(4, device="cuda"))[0].float().cpu().numpy()
    assert np.array_equal(got[~none], back[~none])
