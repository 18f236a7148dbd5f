"""Buffer management around the C entry points: allocates the device tensors a site and
its linear layers need (torch is used for memory only) and calls the library."""
from __future__ import annotations

from dataclasses import dataclass
from typing import List, Optional

import numpy as np

from . import binding as B


@dataclass
class Calibration:
    """Host result of rptq_calibrate for one site, plus device copies the kernels read."""
    d: int
    bits: int
    ch_min: np.ndarray
    ch_max: np.ndarray
    assign: np.ndarray
    perm: np.ndarray
    cluster_off: np.ndarray
    s: np.ndarray
    inv_s: np.ndarray
    z: np.ndarray
    g_eff: int
    k_padded: int
    perm_pad: object = None          # device int32 [K_p]
    perm_pad_host: np.ndarray = None
    gamma_pad: object = None
    beta_pad: object = None


@dataclass
class FoldedLinear:
    N: int
    Wq: object
    sW: object
    zW: object
    wsum: object
    colterm: object


def calibrate_site(x_batches, gamma, beta, eps, relu, g, bits, seed=0, max_iter=100) -> Calibration:
    import torch
    res = B.rptq_calibrate(x_batches, gamma, beta, eps, relu, g, bits, seed, max_iter)
    d = x_batches[0].shape[1]
    cal = Calibration(d=d, bits=bits, k_padded=B.rptq_padded_k(res["cluster_off"]), **res)
    dev = x_batches[0].device
    cal.perm_pad = torch.empty(cal.k_padded, dtype=torch.int32, device=dev)
    if gamma is not None:
        cal.gamma_pad = torch.empty(cal.k_padded, dtype=torch.float32, device=dev)
        cal.beta_pad = torch.empty(cal.k_padded, dtype=torch.float32, device=dev)
    B.rptq_fold_reorder(gamma, beta, d, cal.perm, cal.cluster_off, None, None, None, 0, d, None,
                        cal.perm_pad, cal.gamma_pad, cal.beta_pad, None, None, None, None, None)
    cal.perm_pad_host = cal.perm_pad.cpu().numpy()
    return cal


def identity_site(cal: Calibration) -> Calibration:
    """The same site for an input that already arrives in its cluster order (the output of a
    linear layer whose rows were permuted offline by this site's reorder index): the gather
    is the identity; clusters, parameters and padding are unchanged.  No LayerNorm."""
    import copy
    import torch
    out = copy.copy(cal)
    ident = np.arange(cal.d, dtype=np.int32)
    out.perm = ident
    out.perm_pad = torch.empty_like(cal.perm_pad)
    out.gamma_pad = None
    out.beta_pad = None
    B.rptq_fold_reorder(None, None, cal.d, ident, cal.cluster_off, None, None, None, 0, cal.d, None,
                        out.perm_pad, None, None, None, None, None, None, None)
    out.perm_pad_host = out.perm_pad.cpu().numpy()
    return out


def fold_linear(cal: Calibration, W, perm_out=None, next_site: Optional[Calibration] = None) -> FoldedLinear:
    """perm_out: reorder index of the layer's output (rows of W), a host array.  next_site: lay the rows out
    as that site's padded cluster-order positions instead (pad rows are zero), which is what
    cluster_gemm_quant needs; the layer then has next_site.k_padded outputs."""
    import torch
    N, K = W.shape
    if next_site is not None:
        perm_out = next_site.perm_pad_host
        N = next_site.k_padded
    dev = W.device
    out = FoldedLinear(
        N=N,
        Wq=torch.empty(B.rptq_weight_bytes(N, cal.k_padded), dtype=torch.uint8, device=dev),
        sW=torch.empty(N, dtype=torch.float32, device=dev),
        zW=torch.empty(N, dtype=torch.int32, device=dev),
        wsum=torch.empty((N, cal.g_eff), dtype=torch.int32, device=dev),
        colterm=torch.empty(N, dtype=torch.float32, device=dev))
    B.rptq_fold_reorder(None, None, cal.d, cal.perm, cal.cluster_off, cal.s, cal.z, W, N, K, perm_out,
                        cal.perm_pad, None, None, out.Wq, out.sW, out.zW, out.wsum, out.colterm)
    return out


def ln_quant(cal: Calibration, x, eps=1e-5, relu=False, codes=None, xsum=None, rowterm=None, want_xsum=False):
    M = x.shape[0]
    if codes is None or rowterm is None or (xsum is None and want_xsum):
        import torch
        dev = x.device
        if codes is None:
            codes = torch.empty(B.rptq_codes_bytes(M, cal.k_padded, cal.bits), dtype=torch.uint8, device=dev)
        if rowterm is None:
            rowterm = torch.empty(M, dtype=torch.float32, device=dev)
        if xsum is None and want_xsum:
            xsum = torch.empty((M, cal.g_eff), dtype=torch.int32, device=dev)
    B.rptq_ln_quant(x, M, cal.d, cal.gamma_pad, cal.beta_pad, eps, relu, cal.perm_pad, cal.cluster_off,
                    cal.s, cal.inv_s, cal.z, cal.bits, codes, xsum, rowterm)
    return codes, xsum, rowterm


def cluster_gemm(cal: Calibration, lin: FoldedLinear, codes, rowterm, M, y=None, dtype=None):
    if y is None:
        import torch
        y = torch.empty((M, lin.N), dtype=dtype or torch.bfloat16, device=codes.device)
    B.rptq_cluster_gemm(codes, M, cal.bits, lin.Wq, lin.N, cal.cluster_off, cal.s, lin.sW, lin.zW, lin.colterm,
                        rowterm, y)
    return y


def cluster_gemm_quant(cal: Calibration, lin: FoldedLinear, codes, rowterm, M, next_site: Calibration, relu=True,
                       next_codes=None, next_rowterm=None, workspace=None):
    """The product of `lin` (folded with next_site=...) quantized for `next_site` in the output stage."""
    if next_codes is None or next_rowterm is None or workspace is None:
        import torch
        dev = codes.device
        if next_codes is None:
            next_codes = torch.empty(B.rptq_codes_bytes(M, next_site.k_padded, next_site.bits), dtype=torch.uint8, device=dev)
        if next_rowterm is None:
            next_rowterm = torch.empty(M, dtype=torch.float32, device=dev)
        if workspace is None:
            workspace = torch.empty(max(16, B.rptq_cluster_gemm_quant_workspace_bytes(M, lin.N)), dtype=torch.uint8, device=dev)
    B.rptq_cluster_gemm_quant(codes, M, cal.bits, lin.Wq, lin.N, cal.cluster_off, cal.s, lin.sW, lin.zW, lin.colterm,
                              rowterm, relu, next_site.cluster_off, next_site.s, next_site.inv_s, next_site.z,
                              next_site.bits, next_codes, next_rowterm, workspace)
    return next_codes, next_rowterm


# ---- weights with one parameter pair per (output channel, input cluster): App. A.4 as printed ----
@dataclass
class FoldedLinearCw:
    N: int
    Wq: object
    sW: object            # [N, g]
    zW: object            # [N, g]
    wsum: object          # [N, g]
    scale_tab: object     # [g, N_p]
    cross_tab: object     # [N_p, 32]
    colterm: object       # [N]


def fold_linear_cw(cal: Calibration, W, perm_out=None) -> FoldedLinearCw:
    import torch
    N, K = (W.shape[0] if perm_out is None else len(perm_out)), W.shape[1]
    dev, g = W.device, cal.g_eff
    out = FoldedLinearCw(
        N=N,
        Wq=torch.empty(B.rptq_weight_bytes(N, cal.k_padded), dtype=torch.uint8, device=dev),
        sW=torch.empty((N, g), dtype=torch.float32, device=dev),
        zW=torch.empty((N, g), dtype=torch.int32, device=dev),
        wsum=torch.empty((N, g), dtype=torch.int32, device=dev),
        scale_tab=torch.empty(B.rptq_cw_scale_bytes(N, g) // 4, dtype=torch.float32, device=dev),
        cross_tab=torch.empty(B.rptq_cw_cross_bytes(N, g) // 4, dtype=torch.float32, device=dev),
        colterm=torch.empty(N, dtype=torch.float32, device=dev))
    B.rptq_fold_reorder_cw(cal.perm, cal.cluster_off, cal.s, cal.z, W, N, K, perm_out, cal.perm_pad, out.Wq, out.sW,
                           out.zW, out.wsum, out.scale_tab, out.cross_tab, out.colterm)
    return out


def cluster_rowsums(cal: Calibration, codes, M, rowsums=None):
    if rowsums is None:
        import torch
        rowsums = torch.empty(max(4, B.rptq_cw_rowsum_bytes(M, cal.g_eff) // 4), dtype=torch.float32, device=codes.device)
    B.rptq_cluster_rowsums(codes, M, cal.bits, cal.cluster_off, cal.s, cal.z, rowsums)
    return rowsums


def cluster_gemm_cw(cal: Calibration, lin: FoldedLinearCw, codes, rowsums, M, y=None, dtype=None):
    if y is None:
        import torch
        y = torch.empty((M, lin.N), dtype=dtype or torch.bfloat16, device=codes.device)
    B.rptq_cluster_gemm_cw(codes, M, cal.bits, lin.Wq, lin.N, cal.cluster_off, lin.scale_tab, lin.cross_tab, lin.colterm,
                           rowsums, y)
    return y


# ---- the key/value cache in pages ------------------------------------------------------------------
@dataclass
class PagedCache:
    """Keys and values of one layer: pages of codes, and the position tables (rptq_kv_tables, of n_heads heads) they are written and
    read by.  The pages have to have the shape that the sizes name: it is compared at the first call after any of them was set."""
    n_heads: int
    head_dim: int
    bits: int
    page_size: int
    k_pages: object       # uint8 [n_pages, d / 128, page_size, 16 * bits]
    v_pages: object
    k_table: object
    v_table: object
    _compared = False     # (no field)

    def __setattr__(self, name, value):
        object.__setattr__(self, name, value)
        object.__setattr__(self, "_compared", False)

    def compare(self):
        """Refuses pages of another shape than the sizes name: the codes would be taken for other tokens' or channels'."""
        _page_bytes(self.n_heads * self.head_dim, self.page_size, self.bits)
        want = (self.n_heads * self.head_dim // 128, self.page_size, 16 * self.bits)
        for name, pages in (("k_pages", self.k_pages), ("v_pages", self.v_pages)):
            if pages.dim() != 4 or tuple(pages.shape[1:]) != want:
                raise ValueError("%s: expected shape [pages, %d, %d, %d], got %s" % ((name,) + want + (tuple(pages.shape),)))
        object.__setattr__(self, "_compared", True)


def _page_bytes(d: int, page_size: int, bits: int) -> int:
    n = B.rptq_kv_page_bytes(d, page_size, bits)
    if n == 0:
        raise B.RptqError(-3 if bits not in (3, 4, 8) else -2, "rptq_kv_page_bytes")
    return n


def paged_cache(n_pages: int, page_size: int, n_heads: int, head_dim: int, bits: int, k_table, v_table) -> PagedCache:
    """A cache with room for n_pages * page_size tokens.  (What no token was written to holds no values: no call reads it but
    for a token that a page table and a length claim.)"""
    import torch
    d = n_heads * head_dim
    _page_bytes(d, page_size, bits)
    pages = [torch.zeros((n_pages, d // 128, page_size, 16 * bits), dtype=torch.uint8, device=k_table.device) for _ in range(2)]
    return PagedCache(n_heads, head_dim, bits, page_size, pages[0], pages[1], k_table, v_table)


def kv_quant_paged(cache: PagedCache, k, v, slots):
    """Keys and values [T, d] of new tokens into the cache; a negative slot: that row is stored nowhere."""
    cache._compared or cache.compare()
    B.rptq_kv_quant_paged(k, v, slots, cache.k_table, cache.v_table, cache.bits, cache.k_pages, cache.v_pages, cache.page_size)


def kv_dequant_paged(cache: PagedCache, slots, k=None, v=None):
    """The rows at these slots, bf16 in the original channel order; where a slot is none, zeros, or what a given tensor held."""
    cache._compared or cache.compare()
    if k is None or v is None:
        import torch
        shape = (slots.shape[0], cache.n_heads * cache.head_dim)
        if k is None:
            k = torch.zeros(shape, dtype=torch.bfloat16, device=slots.device)
        if v is None:
            v = torch.zeros(shape, dtype=torch.bfloat16, device=slots.device)
    B.rptq_kv_dequant_paged(cache.k_pages, cache.v_pages, cache.page_size, cache.bits, slots, cache.k_table, cache.v_table, k, v)
    return k, v


def attend_paged_workspace(cache: PagedCache, batch: int, n_q_heads: int):
    """Device memory for attend_paged calls of that many sequences, one call at a time."""
    import torch
    return torch.empty(max(16, B.rptq_attend_paged_workspace_bytes(batch, n_q_heads, cache.n_heads, cache.head_dim)),
                       dtype=torch.uint8, device=cache.k_pages.device)


def attend_paged(cache: PagedCache, q, page_table, lens, scale=None, out=None, lse=None, want_lse=False, workspace=None):
    """Attention of one new token of every sequence over the cache.  q: [B, n_q_heads * head_dim]; scale: 1 / sqrt(head_dim)
    unless given.  Returns (out, lse); lse is None unless given or wanted."""
    cache._compared or cache.compare()
    n_q_heads = q.shape[1] // cache.head_dim
    if out is None or (lse is None and want_lse) or workspace is None:
        import torch
        if out is None:
            out = torch.empty(tuple(q.shape), dtype=torch.bfloat16, device=q.device)
        if lse is None and want_lse:
            lse = torch.empty((q.shape[0], n_q_heads), dtype=torch.float32, device=q.device)
        if workspace is None:
            workspace = attend_paged_workspace(cache, q.shape[0], n_q_heads)
    B.rptq_attend_paged(q, n_q_heads, cache.n_heads, cache.head_dim, cache.head_dim ** -0.5 if scale is None else scale,
                        cache.k_table, cache.v_table, cache.bits, cache.k_pages, cache.v_pages, cache.page_size, page_table,
                        lens, out, lse, workspace)
    return out, lse


# ---- rotary positions in front of the cache ------------------------------------------------------------
@dataclass
class Rotary:
    """How a model turns its queries and keys: frequencies (float64, radians per position, one per pair, on the device), what the
    turned channels are multiplied by, and whether a pair is channels (2 j, 2 j + 1) or (j, j + rotary_dim / 2) of a head."""
    rotary_dim: int
    freqs: object
    amplitude: float = 1.0
    interleaved: bool = False


def rotary(rotary_dim: int, base: float = 10000.0, interleaved: bool = False, scaling=None, factor: float = 1.0, trained: float = 0.0,
           slow: float = 1.0, fast: float = 32.0, device="cuda") -> Rotary:
    """Frequencies base^(-2 j / rotary_dim), for contexts longer than the trained one scaled as rptq_rope_freqs says ("linear", "base",
    "parts").  "parts" comes with an amplitude of 0.1 log(factor) + 1; a model that has another one sets the result's."""
    import torch
    freqs, amplitude = B.rptq_rope_freqs(rotary_dim, base, scaling, factor, trained, slow, fast)
    return Rotary(rotary_dim, torch.from_numpy(freqs).to(device), amplitude, interleaved)


def rope(rot: Rotary, x, positions, head_dim: int, out=None):
    """Rows x [T, n_heads * head_dim] turned by their positions (int32 [T]); out may be x, or of another type."""
    if out is None:
        import torch
        out = torch.empty(tuple(x.shape), dtype=x.dtype, device=x.device)
    B.rptq_rope(x, out, positions, head_dim, rot.rotary_dim, rot.interleaved, rot.freqs, rot.amplitude)
    return out


def rope_quant_paged(cache: PagedCache, rot: Rotary, q, k, v, positions, slots, q_out=None):
    """kv_quant_paged of turned keys, and the same tokens' queries turned (q None: no queries), in one launch.  Returns the
    queries; q_out may be q."""
    cache._compared or cache.compare()
    if q is not None and q_out is None:
        import torch
        q_out = torch.empty(tuple(q.shape), dtype=torch.bfloat16, device=q.device)
    B.rptq_rope_quant_paged(q, q_out, k, v, positions, slots, cache.head_dim, rot.rotary_dim, rot.interleaved, rot.freqs, rot.amplitude,
                            cache.k_table, cache.v_table, cache.bits, cache.k_pages, cache.v_pages, cache.page_size)
    return q_out


# ---- bounding the cache by accumulated attention weight --------------------------------------------------
@dataclass
class CacheTrack:
    """A record of every token of a batch: what each key/value head's queries gave it, and where in the text it stands."""
    weights: object       # fp32 [B, n_heads, capacity]
    positions: object     # int32 [B, n_heads, capacity]


def cache_track(cache: PagedCache, batch: int, capacity: int) -> CacheTrack:
    """Records of up to `capacity` tokens of each of `batch` sequences; attend_weights_paged fills in a token's when it is fresh."""
    import torch
    shape, dev = (batch, cache.n_heads, capacity), cache.k_pages.device
    return CacheTrack(torch.zeros(shape, dtype=torch.float32, device=dev), torch.zeros(shape, dtype=torch.int32, device=dev))


def attend_weights_paged_workspace(cache: PagedCache, batch: int, n_q_heads: int, queries: int):
    """Device memory for attend_weights_paged calls of such sizes, one call at a time; None where they need none."""
    size = B.rptq_attend_weights_paged_workspace_bytes(batch, queries, n_q_heads, cache.n_heads, cache.head_dim)
    if size == 0:
        return None
    import torch
    return torch.empty(size, dtype=torch.uint8, device=cache.k_pages.device)


def attend_weights_paged(cache: PagedCache, q, page_table, lens, lse, track: CacheTrack, positions=None, queries: int = 1, fresh: int = 1,
                         scale=None, workspace=None):
    """Adds what the last `queries` tokens of every sequence gave each of its tokens to the records.  q: [B * queries, n_q_heads *
    head_dim]; lse: what attend_paged left for these rows; the newest `fresh` tokens' records start here, the newest one's
    position being positions[b] (its index where None).  scale: attend_paged's."""
    cache._compared or cache.compare()
    n_q_heads = q.shape[1] // cache.head_dim
    if workspace is None and queries * n_q_heads > 4 * cache.n_heads:          # (up to four queries of a key/value head need none)
        workspace = attend_weights_paged_workspace(cache, lens.shape[0], n_q_heads, queries)
    B.rptq_attend_weights_paged(q, queries, n_q_heads, cache.n_heads, cache.head_dim,
                                cache.head_dim ** -0.5 if scale is None else scale, cache.k_table, cache.bits, cache.k_pages, cache.page_size,
                                page_table, lens, lse, positions, fresh, track.weights, track.positions, workspace)


def evict_paged_workspace(cache: PagedCache, batch: int, capacity: int, budget: int):
    """Device memory for evict_paged calls of such sizes, one call at a time."""
    import torch
    return torch.empty(max(16, B.rptq_evict_paged_workspace_bytes(batch, cache.n_heads, capacity, budget)), dtype=torch.uint8,
                       device=cache.k_pages.device)


def evict_paged(cache: PagedCache, page_table, lens, track: CacheTrack, budget: int, first: int = 0, recent: int = 0, out=None,
                lens_out=None, workspace=None):
    """Every head of every sequence of more than `budget` tokens keeps that many: the ones at positions below `first`, the newest
    `recent`, then the heaviest.  Rows move in place, records too unless `out` is another track.  Returns the new lengths."""
    cache._compared or cache.compare()
    if lens_out is None or workspace is None:
        import torch
        if lens_out is None:
            lens_out = torch.empty(tuple(lens.shape), dtype=torch.int32, device=lens.device)
        if workspace is None:
            workspace = evict_paged_workspace(cache, lens.shape[0], track.weights.shape[2], budget)
    out = track if out is None else out
    B.rptq_evict_paged(cache.n_heads, cache.head_dim, cache.bits, cache.k_pages, cache.v_pages, cache.page_size, page_table, lens,
                       track.weights, track.positions, budget, first, recent, out.weights, out.positions, lens_out, workspace)
    return lens_out
