"""Test-side view of the paged cache, written from include/rptq.h alone: packing codes into pages, building sites and
tables, and how far an fp32 attention may be from the float64 one."""
import numpy as np

from oracle import kv_cache as kvo

import packfmt

U = 2.0 ** -24          # half a step of fp32, relative


def clusters(H, hd, bits, g, seed, away=2.0):
    """Per-head clustering of channels whose ranges differ in width and lie away from zero: (HeadClusters, min, max)."""
    rng = np.random.default_rng(seed)
    d = H * hd
    width = np.exp(rng.normal(0, 1, d))
    mid = rng.normal(0, away, d) * width
    lo, hi = (mid - 3 * width).astype(np.float32), (mid + 3 * width).astype(np.float32)
    return kvo.cluster_heads([lo], [hi], H, min(g, hd), bits, seed), lo, hi


def values(rng, lo, hi, T):
    """bf16 rows that fill the channels' ranges and sometimes leave them."""
    x = (lo + hi) / 2 + (hi - lo) / 6 * rng.standard_normal((T, len(lo)))
    return kvo.round_to_bf16(x.astype(np.float32))


def table_rows(hc, tensor=0):
    """The position table's records, [D, 4] int32."""
    s, inv, z = kvo.position_tables(hc, tensor)
    return np.stack([hc.perm.astype(np.int32), inv.view(np.int32), s.view(np.int32), z.astype(np.int32)], axis=1)


def page_rows(codes, bits):
    """Codes [T, D] in cluster order -> a token's rows in the blocks of a page, [T, D / 128, 16 * bits] bytes."""
    T, d = codes.shape
    return packfmt.pack_groups(codes, bits).reshape(T, d // 128, 16 * bits)


def put(pages, slots, rows, page_size):
    """Rows into pages [n, D / 128, page_size, 16 * bits] at the slots that exist."""
    for t, slot in enumerate(np.asarray(slots)):
        if 0 <= slot < pages.shape[0] * page_size:
            pages[slot // page_size, :, slot % page_size] = rows[t]


def attend_bounds(q, k_codes, hc_k, hc_v, n_q, scale, bits, out64, lse64, tensor_k=0, tensor_v=0):
    """How far an fp32 evaluation of one sequence's attention may be from the float64 one: (per output, per head's lse).

    With q' = q s scale log2(e) (four roundings: s and scale log2(e) fold in three products, one rounded constant) and exact
    sums of q' times codes, rounded a few times at the end, a score in units of log2 is off by at most 8 U S1, where
    S1 = max_t sum_j |q'_j c_tj|.  2^x adds a relative 2 U and its argument's own rounding is in the 8.  A weight is then off
    by a relative e = ln 2 * 8 U S1 + 4 U, the sums of n weights by another (n / 64 + 40) U (exact within 64 tokens,
    added up in fp32 beyond, joined over waves and parts).  A mean of codes c with |c| <= 2^(bits - 1) moves by at most
    2 e 2^(bits - 1) from the weights, and both sums' relative errors apply to it once more; s (mean - z) adds three
    roundings of what it is made of."""
    H, dh = hc_k.n_heads, hc_k.d_head
    share = n_q // H
    s_k, _, z_k = kvo.position_tables(hc_k, tensor_k)
    s_v, _, z_v = kvo.position_tables(hc_v, tensor_v)
    n = len(k_codes)
    top = 2.0 ** (bits - 1)
    q = np.asarray(q, dtype=np.float64).reshape(n_q, dh)
    out, lse = np.zeros((n_q, dh)), np.zeros(n_q)
    for h in range(n_q):
        kv = h // share
        sl = slice(kv * dh, (kv + 1) * dh)
        qp = np.abs(q[h][hc_k.perm[sl] - kv * dh] * s_k[sl].astype(np.float64) * scale * np.log2(np.e))
        s1 = float((np.abs(np.asarray(k_codes)[:, sl]) @ qp).max()) if n else 0.0
        sz = float(qp @ np.abs(z_k[sl]))
        e = np.log(2) * 8 * U * s1 + 4 * U
        sums = (n / 64 + 40) * U
        cols = hc_v.perm[sl] - kv * dh
        s, z = s_v[sl].astype(np.float64), np.abs(z_v[sl].astype(np.float64))
        out[h][cols] = s * top * (2 * e + 2 * sums) + 3 * U * s * (top + z) + U * np.abs(out64.reshape(n_q, dh)[h][cols])
        finite = abs(lse64[h]) if n else 0.0
        # (m + log2 l - z term, each rounded, then times ln 2: the z term takes the roundings of q')
        lse[h] = np.log(2) * (8 * U * s1 + 6 * U * sz) + e + sums + 4 * U * (finite + s1 + sz)
    return out.reshape(-1), lse
