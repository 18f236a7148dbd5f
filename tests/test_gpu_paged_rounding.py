"""How exactly attention over the pages computes a weight and the logarithm of the sum where scores are small: a number far from
them (the fixed point's power of two) must not be added before a rounding.  Every tolerance counts the roundings of fp32 that the
formula cannot do without, on inputs where few are left."""
import numpy as np
import pytest

from oracle import kv_cache as kvo

import packfmt

pytestmark = pytest.mark.gpu
torch = pytest.importorskip("torch")

U = 2.0 ** -24          # half a step of fp32, relative


@pytest.fixture(scope="module")
def rp():
    import paper_2304_01089_amd as rp_
    rp_.load_library()
    assert torch.cuda.is_available()
    return rp_


def dev(a, dtype=None):
    return torch.from_numpy(np.ascontiguousarray(a if dtype is None else np.asarray(a, dtype))).cuda()


def records(s, z):
    """A position table that leaves every channel where it is."""
    s = np.asarray(s, np.float32)
    inv = (1.0 / s.astype(np.float64)).astype(np.float32)
    return dev(np.stack([np.arange(len(s), dtype=np.int32), inv.view(np.int32), s.view(np.int32), np.asarray(z, np.int32)], axis=1))


def one_page(rp, hd, bits, k_codes, v_codes, k_table, v_table):
    """A cache of one key/value head and one page of 16 tokens, which every sequence reads."""
    def rows(codes):
        full = np.zeros((16, hd), np.int64)
        full[:len(codes)] = codes
        return dev(packfmt.pack_groups(full, bits).reshape(16, hd // 128, 16 * bits).transpose(1, 0, 2)[None])

    return rp.PagedCache(1, hd, bits, 16, rows(k_codes), rows(v_codes), k_table, v_table)


def attend(rp, cache, q, tokens, scale, wide):
    B, share, hd = q.shape
    table = torch.full((B, 400 if wide else 1), -1, dtype=torch.int32, device="cuda")       # (wide: sequences may be cut)
    table[:, 0] = 0
    out = torch.full((B, share * hd), float("nan"), device="cuda")
    bits = torch.from_numpy(q.astype(np.float32).reshape(B, -1)).cuda().bfloat16()
    assert np.array_equal(bits.float().cpu().numpy().reshape(q.shape), q)
    _, lse = rp.attend_paged(cache, bits, table, torch.full((B,), tokens, dtype=torch.int32, device="cuda"), scale=scale, out=out, want_lse=True)
    return out.double().cpu().numpy().reshape(q.shape), lse.double().cpu().numpy()


@pytest.mark.parametrize("wide", [False, True])
@pytest.mark.parametrize("bits", [3, 4, 8])
@pytest.mark.parametrize("hd,share", [(128, 1), (128, 8), (128, 16), (256, 4), (256, 8)])
def test_two_tokens_whose_weights_are_close(rp, hd, share, bits, wide):
    """Keys 0 and -1 in one channel, queries q there: scores 0 and -q exactly but for q' = q log2(e), so w = exp(-q) is all that there
    is: out = c w / (1 + w) for value codes 0 and c, lse = log(1 + w).

    q' takes three roundings of half a step (the constant log2(e), its product with q, the score's conversion to fp32) and 2^-30 in
    its fixed point, which move w by a relative 3 U q + 2^-30 q; 2^x has one step (2 U).  A weight above 1/2 has all its bits in
    the fixed point.  1 + w, the conversion of c w and the quotient round once each.  lse: 1 + w moves by w / (1 + w) of w's error
    and its own rounding, log2 has one step, ln 2 and the product with it a half each."""
    k, v = np.zeros((2, hd), np.int64), np.zeros((2, hd), np.int64)
    k[1, 0] = -1
    v[1] = 1 + np.arange(hd) % 3
    plain = records(np.ones(hd), np.zeros(hd))
    cache = one_page(rp, hd, bits, k, v, plain, plain)
    rng = np.random.default_rng(hd + share)
    q = np.zeros((256, share, hd))
    q[..., 0] = kvo.round_to_bf16(np.exp(rng.uniform(np.log(2.0 ** -7), np.log(0.6), q.shape[:2])).astype(np.float32))
    out, lse = attend(rp, cache, q, 2, 1.0, wide)
    x = q[..., 0]
    w = np.exp(-x)
    e = (3 * U + 2.0 ** -30) * x + 2 * U
    want = w / (1 + w)
    tol = want * (e / (1 + w) + 3 * U) * (1 + 1e-6)
    off = np.abs(out - want[..., None] * v[1])
    assert (off <= tol[..., None] * v[1]).all(), (off / (tol[..., None] * v[1])).max()
    tol = (e * w / (1 + w) + U + 4 * U * np.log1p(w)) * (1 + 1e-6)
    off = np.abs(lse - np.log1p(w))
    assert (off <= tol).all(), (off / tol).max()


@pytest.mark.parametrize("wide", [False, True])
@pytest.mark.parametrize("size", [0.002, 0.05])
@pytest.mark.parametrize("hd,share,bits", [(128, 1, 4), (128, 12, 8), (256, 4, 3), (256, 8, 8)])
def test_the_logarithm_of_one_token(rp, hd, share, bits, size, wide):
    """One token: lse is its score, log2 of the sum being 0 exactly.

    q' takes four roundings (q s, the constant, its product with the scale, their product), relative to the sums S1 of |q' c| and Sz
    of |q' z|; the fixed point half a unit per code, of 2^-29 of the largest |q'| at most, and a 2^-4 of that for the lower half's conversion; the
    score's conversion two U of S1 and its upper half's one; the sum over the zero points, in 64 bits, one; their difference one of it.
    Then ln 2 and the product with it."""
    rng = np.random.default_rng(hd + share + bits)
    top = 1 << (bits - 1)
    s, z = rng.uniform(0.5, 1.0, hd).astype(np.float32), rng.integers(-3, 4, hd)
    k = rng.integers(-top, top, (1, hd))
    cache = one_page(rp, hd, bits, k, k, records(s, z), records(s, z))
    scale = float(np.float32(hd ** -0.5))
    q = kvo.round_to_bf16((rng.standard_normal((256, share, hd)) * size).astype(np.float32)).astype(np.float64)
    out, lse = attend(rp, cache, q, 1, scale, wide)
    qp = q * s.astype(np.float64) * scale * np.log2(np.e)
    want = np.log(2) * (qp * (k[0] - z)).sum(-1)
    s1, sz = np.abs(qp * k[0]).sum(-1), np.abs(qp * z).sum(-1)
    fixed = 2.0 ** -30 * (1 + 2.0 ** -4) * np.abs(qp).max(-1) * np.abs(k[0]).sum()
    tol = (np.log(2) * (7 * U * s1 + 5 * U * sz + U * (s1 + sz) + fixed) + 2 * U * np.abs(want)) * (1 + 1e-6)
    off = np.abs(lse - want)
    assert (off <= tol).all(), (off / tol).max()
    assert np.abs(out - s.astype(np.float64) * (k[0] - z)).max() <= 3 * U * top * 4
