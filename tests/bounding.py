"""Plain forms of the rotary and cache-bounding operators in 64 bits, written from include/rptq.h, and how far fp32 may be off."""
import numpy as np

from oracle import kv_cache as kvo

U = 2.0 ** -24          # half a step of fp32, relative


def pairs(rot, interleaved):
    j = np.arange(rot // 2)
    return (2 * j, 2 * j + 1) if interleaved else (j, j + rot // 2)


def turns(positions, freqs, amplitude):
    """cos and sin per row and pair, float64."""
    theta = np.asarray(positions, np.float64)[:, None] * freqs
    return amplitude * np.cos(theta), amplitude * np.sin(theta)


def rope64(x, positions, hd, rot, interleaved, freqs, amplitude=1.0):
    """(rows turned in float64, bound of an fp32 evaluation with cos and sin rounded to fp32): a product of two rounded factors' is
    off by two half steps (the factor's, its own), the sum by one of the result."""
    x = np.asarray(x, np.float64).reshape(len(x), -1, hd)
    c, s = (t[:, None] for t in turns(positions, freqs, amplitude))
    a, b = pairs(rot, interleaved)
    y, tol = x.copy(), np.zeros_like(x)
    y[..., a], y[..., b] = c * x[..., a] - s * x[..., b], c * x[..., b] + s * x[..., a]
    for u, v in ((a, b), (b, a)):
        parts = np.abs(c * x[..., u]) + np.abs(s * x[..., v])
        tol[..., u] = 2.01 * U * parts + U * (np.abs(y[..., u]) + 2.01 * U * parts)
    return y.reshape(len(x), -1), tol.reshape(len(x), -1)


def rope32(x, positions, hd, rot, interleaved, freqs, amplitude=1.0):
    """The documented roundings, step by step: fp32 bits."""
    x = np.asarray(x, np.float32).reshape(len(x), -1, hd)
    c, s = (t.astype(np.float32)[:, None] for t in turns(positions, freqs, amplitude))
    a, b = pairs(rot, interleaved)
    y = x.copy()
    y[..., a], y[..., b] = x[..., a] * c - x[..., b] * s, x[..., b] * c + x[..., a] * s
    return y.reshape(len(x), -1)


def weights64(q, lse, k_codes, at, n, hc, n_q, scale, queries, tensor=0):
    """What the tokens at indices `at` (k_codes: their rows) of a sequence of n got of `queries` queries: (sums [H, len(at)], bound).

    In units of log2 a score's error is at most 8 U (S1 + SZ), with every step in fp32: q' has four roundings, which count once for the codes' sum
    (S1 = sum |q'_j c_j|) and once for the zero points' (SZ = sum |q'_j z_j|), its fixed point half a unit 30 bits below the largest, the digits'
    sums two half steps, the difference from lse one; lse in these units one of its own, one as it joins the zero points' term
    and one in the difference.  2^x adds a step, the sum over p pairs (p / 4 + 6) half steps."""
    H, dh = hc.n_heads, hc.d_head
    share = n_q // H
    s, _, z = kvo.position_tables(hc, tensor)
    q = np.asarray(q, np.float64).reshape(queries, n_q, dh)
    got, tol = np.zeros((H, len(at))), np.zeros((H, len(at)))
    for h in range(H):
        sl = slice(h * dh, (h + 1) * dh)
        codes, ss, zz = np.asarray(k_codes)[:, sl].astype(np.float64), s[sl].astype(np.float64), z[sl].astype(np.float64)
        for i in range(queries):
            sees = np.asarray(at) < n - (queries - 1 - i)
            for g in range(h * share, (h + 1) * share):
                qp = q[i, g][hc.perm[sl] - h * dh] * ss * scale
                with np.errstate(all="ignore"):
                    p = np.where(sees, np.exp(codes @ qp - zz @ qp - np.float64(lse[i, g])), 0.0)
                off = np.log2(np.e) * (np.abs(codes) @ np.abs(qp) + np.abs(zz) @ np.abs(qp)) * 8 + 3 * abs(lse[i, g] * np.log2(np.e))
                got[h] += p
                with np.errstate(invalid="ignore"):                 # (a query that sees nothing has no finite lse)
                    tol[h] += np.where(sees, p * U * (np.log(2) * off + 2), 0.0)
    return got, tol + (share * queries / 4 + 6) * U * got


def evict(weights, positions, budget, first, recent):
    """(token that every place below the budget holds afterwards) of one head of n tokens."""
    n = len(weights)
    if n <= budget:
        return np.arange(n)
    p = np.asarray(positions, np.int64)
    safe = (p < first) | (p > p.max() - recent)
    w = np.asarray(weights, np.float64)
    # (safe tokens are all alike: should they be more than the budget, the first of them stay)
    order = sorted(range(n), key=lambda t: (not safe[t], not (safe[t] or np.isnan(w[t])), 0.0 if safe[t] or np.isnan(w[t]) else -w[t], t))
    keep = np.zeros(n, bool)
    keep[order[:budget]] = True
    src = np.arange(budget)
    src[~keep[:budget]] = np.flatnonzero(keep[budget:]) + budget
    return src
