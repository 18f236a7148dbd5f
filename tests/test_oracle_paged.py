"""Pins of the attention oracle, and of the test-side page layout.  No GPU."""
from fractions import Fraction

import numpy as np
import pytest

from oracle import kv_cache as kvo

import packfmt
import paged


def _case(bits=4, H=2, hd=32, T=9, seed=3):
    hk, lo, hi = paged.clusters(H, hd, bits, 3, seed)
    hv, lov, hiv = paged.clusters(H, hd, bits, 3, seed + 50)
    rng = np.random.default_rng(seed)
    k, v = kvo.kv_quant(paged.values(rng, lo, hi, T), hk, 0, bits), kvo.kv_quant(paged.values(rng, lov, hiv, T), hv, 0, bits)
    return hk, hv, k, v, rng


def test_scores_and_weights_by_exact_arithmetic():
    hk, hv, k, v, rng = _case()
    n_q, hd = 4, 32
    q = kvo.round_to_bf16(rng.standard_normal(n_q * hd).astype(np.float32) * np.float32(0.1))
    out, lse = kvo.attend(q, k, v, hk, 0, hv, 0, n_q, 0.25)
    s, _, z = kvo.position_tables(hk, 0)
    sv, _, zv = kvo.position_tables(hv, 0)
    for h in (0, 3):
        kv = h // 2
        a = []
        for t in range(len(k)):
            total = Fraction(0)
            for j in range(kv * hd, (kv + 1) * hd):
                c = int(hk.perm[j]) - kv * hd
                total += Fraction(float(q[h * hd + c])) * Fraction(float(s[j])) * (int(k[t, j]) - int(z[j]))
            a.append(float(total / 4))
        p = np.exp(np.array(a) - max(a))
        assert abs(lse[h] - (max(a) + np.log(p.sum()))) < 1e-12
        for j in range(kv * hd, (kv + 1) * hd):
            want = sum(p[t] * float(sv[j]) * (int(v[t, j]) - int(zv[j])) for t in range(len(k))) / p.sum()
            assert abs(out[h * hd + int(hv.perm[j]) - kv * hd] - want) < 1e-12 * (1 + abs(want))


def test_the_same_from_de_quantized_tensors_in_channel_order():
    hk, hv, k, v, rng = _case(bits=8, T=40)
    n_q, hd, H = 2, 32, 2
    s, _, z = kvo.position_tables(hk, 0)
    sv, _, zv = kvo.position_tables(hv, 0)
    kh, vh = np.empty(k.shape), np.empty(v.shape)
    kh[:, hk.perm] = s.astype(np.float64) * (k - z)
    vh[:, hv.perm] = sv.astype(np.float64) * (v - zv)
    q = rng.standard_normal(n_q * hd)
    out, lse = kvo.attend(q, k, v, hk, 0, hv, 0, n_q, 0.1)
    a = 0.1 * np.einsum("hj,thj->ht", q.reshape(H, hd), kh.reshape(-1, H, hd))
    p = np.exp(a - a.max(1, keepdims=True))
    p /= p.sum(1, keepdims=True)
    assert np.allclose(out.reshape(H, hd), np.einsum("ht,thj->hj", p, vh.reshape(-1, H, hd)), rtol=1e-12, atol=1e-12)
    assert np.allclose(lse, np.log(np.exp(a - a.max()).sum(1)) + a.max(), rtol=1e-12)


def test_one_token_none_and_equal_scores():
    hk, hv, k, v, rng = _case()
    sv, _, zv = kvo.position_tables(hv, 0)
    q = rng.standard_normal(64)
    out, lse = kvo.attend(q, k[:0], v[:0], hk, 0, hv, 0, 2, 1.0)
    assert (out == 0).all() and (lse == -np.inf).all()
    one, _ = kvo.attend(q, k[:1], v[:1], hk, 0, hv, 0, 2, 1.0)
    want = np.empty(64)
    want[hv.perm] = sv.astype(np.float64) * (v[0] - zv)
    assert np.allclose(one, want, rtol=1e-14)
    flat, lse = kvo.attend(q * 0, k, v, hk, 0, hv, 0, 2, 1.0)
    want[hv.perm] = (sv.astype(np.float64) * (v - zv)).mean(0)
    assert np.allclose(flat, want, rtol=1e-12) and np.allclose(lse, np.log(9))


@pytest.mark.parametrize("bits", [3, 4, 8])
def test_page_rows_are_the_dense_rows_cut_in_blocks(bits):
    rng = np.random.default_rng(bits)
    codes = rng.integers(-(1 << (bits - 1)), 1 << (bits - 1), (5, 256))
    rows = paged.page_rows(codes, bits)
    assert rows.shape == (5, 2, 16 * bits)
    assert np.array_equal(rows.reshape(5, -1), packfmt.pack_groups(codes, bits))
    assert np.array_equal(packfmt.unpack_groups(rows[:, 1], 128, bits), codes[:, 128:])
    pages = np.zeros((3, 2, 16, 16 * bits), np.uint8)
    paged.put(pages, [17, -1, 48, 47, 0], rows, 16)
    assert np.array_equal(pages[1, :, 1], rows[0]) and np.array_equal(pages[2, :, 15], rows[3]) and np.array_equal(pages[0, :, 0], rows[4])
    assert (pages[0, :, 1:] == 0).all() and (pages[1, :, 2:] == 0).all()
