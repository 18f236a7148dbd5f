"""The cache in pages on the GPU against the oracle: codes and read-back bit for bit, attention within the bound that its
fp32 arithmetic allows, and everything that a call must leave alone."""
import numpy as np
import pytest

import workloads as w
from oracle import kv_cache as kvo

import paged

pytestmark = pytest.mark.gpu
torch = pytest.importorskip("torch")


@pytest.fixture(scope="module")
def rp():
    import paper_2304_01089_amd as rp_
    rp_.load_library()
    assert torch.cuda.is_available()
    return rp_


def dev_bf16(x):
    return torch.from_numpy(w.bf16_bits(np.ascontiguousarray(x)).view(np.int16)).cuda().view(torch.bfloat16)


def dev(a, dtype=None):
    return torch.from_numpy(np.ascontiguousarray(a if dtype is None else np.asarray(a, dtype))).cuda()


_SITES = {}


def site(H, hd, bits, g=3):
    """Clusterings and tables of a key and a value tensor (made once per shape)."""
    key = (H, hd, bits, g)
    if key not in _SITES:
        seed = H * 1000 + hd + bits
        k, v = paged.clusters(H, hd, bits, g, seed), paged.clusters(H, hd, bits, g, seed + 500)
        _SITES[key] = k, v, dev(paged.table_rows(k[0])), dev(paged.table_rows(v[0]))
    return _SITES[key]


def test_the_table_is_the_documented_one(rp):
    hc, lo, hi = paged.clusters(4, 64, 4, 3, 9)
    table = torch.zeros(rp.rptq_kv_table_bytes(256), dtype=torch.uint8, device="cuda")
    rp.rptq_kv_tables(hc.perm, hc.cluster_off, hc.s[0], hc.inv_s[0], hc.z[0], 256, 4, 3, table)
    assert np.array_equal(table.view(torch.int32).view(256, 4).cpu().numpy(), paged.table_rows(hc))


# ---- writing and reading ---------------------------------------------------------------------------------
ROWS = [
    (1, 1, 128, 16), (3, 2, 64, 16), (17, 9, 128, 32), (33, 6, 256, 64), (5, 4, 32, 4096), (200, 12, 64, 128), (130, 40, 128, 64),
    (1000, 3, 128, 256),
]


def slots_for(rng, T, n_pages, page):
    """Distinct slots in no order; some rows have none (below, at and far beyond the ends)."""
    slots = rng.permutation(n_pages * page)[:T].astype(np.int64)
    if T > 4:
        slots[rng.permutation(T)[:4]] = [-1, n_pages * page, -2 ** 62, 2 ** 40]
    return slots


@pytest.mark.parametrize("bits", [3, 4, 8])
@pytest.mark.parametrize("T,H,hd,page", ROWS)
def test_rows_written_and_read_bit_for_bit(rp, T, H, hd, page, bits):
    (hk, klo, khi), (hv, vlo, vhi), kt, vt = site(H, hd, bits)
    d = H * hd
    rng = np.random.default_rng(T + d + page + bits)
    n_pages = (T + page - 1) // page + 2
    slots = slots_for(rng, T, n_pages, page)
    k, v = paged.values(rng, klo, khi, T), paged.values(rng, vlo, vhi, T)
    want = [np.full((n_pages, d // 128, page, 16 * bits), 0xA5, np.uint8) for _ in range(2)]
    codes = kvo.kv_quant(k, hk, 0, bits), kvo.kv_quant(v, hv, 0, bits)
    for p, c in zip(want, codes):
        paged.put(p, slots, paged.page_rows(c, bits), page)
    # keys and values as columns of one tensor, and each a tensor of its own
    wide = torch.full((T, 3 * d + 8), float("nan"), dtype=torch.bfloat16, device="cuda")
    wide[:, d:2 * d], wide[:, 2 * d:3 * d] = dev_bf16(k), dev_bf16(v)
    for kk, vv in ((wide[:, d:2 * d], wide[:, 2 * d:3 * d]), (dev_bf16(k), dev_bf16(v))):
        pool = torch.full((2, n_pages + 1, d // 128, page, 16 * bits), 0xA5, dtype=torch.uint8, device="cuda")
        cache = rp.PagedCache(H, hd, bits, page, pool[0, :n_pages], pool[1, :n_pages], kt, vt)
        rp.kv_quant_paged(cache, kk, vv, dev(slots))
        torch.cuda.synchronize()
        for p, q in zip(want, pool.cpu().numpy()):
            assert np.array_equal(q[:n_pages], p) and (q[n_pages] == 0xA5).all()
    # read back, into columns of a wider tensor too; rows without a slot stay
    back = [kvo.kv_dequant(c, h, 0, original_order=True) for c, h in zip(codes, (hk, hv))]
    there = (slots >= 0) & (slots < n_pages * page)
    for kk, vv in ((wide[:, d:2 * d], wide[:, 2 * d:3 * d]), (torch.empty(2, T, d, dtype=torch.bfloat16, device="cuda"))):
        wide.fill_(7.0)
        kk.fill_(7.0), vv.fill_(7.0)
        rp.kv_dequant_paged(cache, dev(slots), k=kk, v=vv)
        torch.cuda.synchronize()
        for got, ref in ((kk, back[0]), (vv, back[1])):
            got = got.float().cpu().numpy()
            assert np.array_equal(got[there], ref[there]) and (got[~there] == 7.0).all()
        assert (wide[:, :d] == 7.0).all() and (wide[:, 3 * d:] == 7.0).all()
    # a slot several times, and the allocating form
    twice = np.concatenate([slots[there][::-1], slots[there][:1]])
    kk, vv = rp.kv_dequant_paged(cache, dev(twice))
    at = np.concatenate([np.flatnonzero(there)[::-1], np.flatnonzero(there)[:1]])
    assert np.array_equal(kk.float().cpu().numpy(), back[0][at]) and np.array_equal(vv.float().cpu().numpy(), back[1][at])


def test_values_that_are_not_finite_stay_in_their_channel(rp):
    H, hd, bits, page = 2, 128, 4, 16
    (hk, lo, hi), _, kt, vt = site(H, hd, bits)
    rng = np.random.default_rng(5)
    x = paged.values(rng, lo, hi, 3)
    bad = x.copy()
    bad[1, 40], bad[1, 200], bad[2, 7] = np.nan, np.inf, -np.inf
    outs = []
    for rows in (x, bad):
        cache = rp.paged_cache(1, page, H, hd, bits, kt, vt)
        rp.kv_quant_paged(cache, dev_bf16(rows), dev_bf16(rows), dev([4, 9, 2], np.int64))
        outs.append(rp.kv_dequant_paged(cache, dev([4, 9, 2], np.int64))[0].float().cpu().numpy())
    same = outs[0] == outs[1]
    assert same[np.isfinite(bad)].all()


def test_pages_beyond_32_bits(rp):
    """Slots whose bytes lie past 4 GiB (and element counts past 2^31)."""
    H, hd, bits, page = 64, 128, 8, 256
    _, _, kt, vt = site(H, hd, bits)
    d = H * hd
    size = rp.rptq_kv_page_bytes(d, page, bits)
    n_pages = (5 << 30) // size
    if torch.cuda.mem_get_info()[0] < 24 << 30:
        pytest.skip("not enough free memory")
    cache = rp.paged_cache(n_pages, page, H, hd, bits, kt, vt)
    (hk, klo, khi), (hv, vlo, vhi) = site(H, hd, bits)[:2]
    rng = np.random.default_rng(1)
    k, v = paged.values(rng, klo, khi, 40), paged.values(rng, vlo, vhi, 40)
    slots = (n_pages - 1) * page + np.arange(40)
    rp.kv_quant_paged(cache, dev_bf16(k), dev_bf16(v), dev(slots))
    kc, vc = kvo.kv_quant(k, hk, 0, bits), kvo.kv_quant(v, hv, 0, bits)
    got = rp.kv_dequant_paged(cache, dev(slots))[0].float().cpu().numpy()
    assert np.array_equal(got, kvo.kv_dequant(kc, hk, 0, original_order=True))
    assert not cache.k_pages[: n_pages - 1].any() and not cache.v_pages[: n_pages - 1].any()
    q = kvo.round_to_bf16((rng.standard_normal((1, d)) * 0.02).astype(np.float32))
    table = dev([[n_pages - 1]], np.int32)
    out = rp.attend_paged(cache, dev_bf16(q), table, dev([40], np.int32), out=torch.empty(1, d, device="cuda"))[0]
    want, lse = kvo.attend(q[0], kc, vc, hk, 0, hv, 0, H, hd ** -0.5)
    tol, _ = paged.attend_bounds(q[0], kc, hk, hv, H, hd ** -0.5, bits, want, lse)
    assert (np.abs(out[0].double().cpu().numpy() - want) <= tol).all()


# ---- attention ----------------------------------------------------------------------------------------------
class Batch:
    """Sequences in shuffled pages, with the codes that every one of them sees."""

    def __init__(self, rp, lens, H, hd, bits, page, holes=(), seed=0, extra_pages=2):
        (self.hk, _, _), (self.hv, _, _), kt, vt = site(H, hd, bits)
        self.lens, self.H, self.hd, self.bits = lens, H, hd, bits
        rng = self.rng = np.random.default_rng(seed + H + hd + bits + page)
        d = H * hd
        top = 1 << (bits - 1)
        need = [(max(n, 0) + page - 1) // page for n in lens]
        width = max(need + [1])
        n_pages = sum(need) + extra_pages
        ids = rng.permutation(n_pages)
        # entries behind a sequence's end, and pages that are not there, are no page numbers
        nonsense = [-1, n_pages, 2 ** 31 - 1, -2 ** 31]
        self.table = rng.choice(nonsense, (len(lens), width)).astype(np.int64)
        # everything in the pages that is no token of a sequence is there to be seen if it is read
        pages = [rng.integers(0, 256, (n_pages, d // 128, page, 16 * bits)).astype(np.uint8) for _ in range(2)]
        self.k, self.v, at = [], [], 0
        for b, n in enumerate(lens):
            n = max(n, 0)
            mine, at = ids[at:at + need[b]], at + need[b]
            codes = rng.integers(-top, top, (2, n, d))
            slots = mine[np.arange(n) // page] * page + np.arange(n) % page
            for p, c in zip(pages, codes):
                paged.put(p, slots, paged.page_rows(c, bits), page)
            self.table[b, :need[b]] = mine
            there = np.ones(n, bool)
            for hole in holes:
                if hole < need[b]:
                    self.table[b, hole] = nonsense[(b + hole) % 4]
                    there[hole * page:(hole + 1) * page] = False
            self.k.append(codes[0][there])
            self.v.append(codes[1][there])
        self.cache = rp.PagedCache(H, hd, bits, page, dev(pages[0]), dev(pages[1]), kt, vt)
        self.page_table, self.dev_lens = dev(self.table, np.int32), dev(lens, np.int32)

    def queries(self, n_q, sharp=1.0):
        s, _, _ = kvo.position_tables(self.hk, 0)
        norm = np.sqrt((s.reshape(self.H, self.hd) ** 2).sum(1)) * 2.0 ** self.bits / 3.5
        t = sharp * 2.0 * np.sqrt(self.hd) / np.repeat(norm, n_q // self.H)
        q = self.rng.standard_normal((len(self.lens), n_q, self.hd)) * t[None, :, None]
        return kvo.round_to_bf16(q.astype(np.float32)).reshape(len(self.lens), -1)

    def check(self, q, n_q, scale, out, lse=None):
        """`out` (device, fp32 or bf16) and lse against the oracle."""
        got = out.double().cpu().numpy()
        for b in range(len(self.lens)):
            want, wl = kvo.attend(q[b], self.k[b], self.v[b], self.hk, 0, self.hv, 0, n_q, scale)
            tol, tl = paged.attend_bounds(q[b], self.k[b], self.hk, self.hv, n_q, scale, self.bits, want, wl)
            if out.dtype == torch.bfloat16:
                tol = tol + 2.0 ** -8 * (np.abs(want) + tol)
            worst = (np.abs(got[b] - want) / np.maximum(tol, 1e-300)).max() if len(self.k[b]) else 0.0
            assert (np.abs(got[b] - want) <= tol).all(), (b, self.lens[b], worst)
            if not len(self.k[b]):
                assert (got[b] == 0).all()
            if lse is not None:
                mine = lse[b].double().cpu().numpy()
                if len(self.k[b]):
                    assert (np.abs(mine - wl) <= tl).all(), (b, self.lens[b], (np.abs(mine - wl) / tl).max())
                else:
                    assert (mine == -np.inf).all()


def run(rp, batch, q, n_q, dtype=torch.float32, lse=True, scale=None, workspace=None):
    out = torch.full((q.shape[0], q.shape[1]), float("nan"), dtype=dtype, device="cuda")
    r = rp.attend_paged(batch.cache, dev_bf16(q), batch.page_table, batch.dev_lens, scale=scale, out=out, want_lse=lse,
                        workspace=workspace)
    torch.cuda.synchronize()
    return r


EDGES = [0, 1, 2, 15, 16, 17, 31, 33, 63, 64, 65, 127, 129, 255, 256, 257, 300, 513, 1000]


@pytest.mark.parametrize("bits", [3, 4, 8])
@pytest.mark.parametrize("H,share,hd,page", [(4, 1, 32, 16), (2, 1, 64, 16), (2, 3, 64, 32), (1, 1, 128, 16), (1, 4, 128, 64),
                                             (2, 5, 128, 16), (1, 8, 128, 128), (1, 1, 256, 16), (1, 6, 256, 32)])
def test_lengths_around_every_edge(rp, H, share, hd, page, bits):
    b = Batch(rp, EDGES, H, hd, bits, page)
    n_q = H * share
    q = b.queries(n_q)
    out, lse = run(rp, b, q, n_q)
    b.check(q, n_q, hd ** -0.5, out, lse)


@pytest.mark.parametrize("H,share,hd,bits,page,lens", [
    (1, 16, 128, 4, 16, [700, 3]),               # as many query heads on one as a workgroup takes
    (1, 17, 64, 8, 64, None), (2, 17, 64, 3, 64, [129, 50]), (1, 32, 128, 3, 32, [333, 64]), (1, 71, 128, 4, 16, [90]),
    (4, 9, 32, 4, 16, [200, 7]), (2, 24, 256, 4, 64, [77, 400]), (3, 1, 256, 8, 16, [50]), (96, 1, 128, 3, 64, [70, 1]),
    (12, 1, 64, 8, 4096, [5000, 4096, 4097]), (16, 2, 32, 3, 1024, [1025, 2]),
])
def test_head_layouts(rp, H, share, hd, bits, page, lens):
    if lens is None:                                          # (64 channels are no whole block)
        _, _, kt, vt = site(2, 64, bits)
        cache = rp.paged_cache(2, page, 2, hd, bits, kt, vt)
        cache.n_heads = 1
        with pytest.raises(rp.RptqError):
            rp.attend_paged(cache, torch.zeros(1, 64 * share, dtype=torch.bfloat16, device="cuda"), dev([[0]], np.int32), dev([1], np.int32))
        return
    b = Batch(rp, lens, H, hd, bits, page)
    n_q = H * share
    q = b.queries(n_q)
    for dtype in (torch.float32, torch.bfloat16):
        out, lse = run(rp, b, q, n_q, dtype)
        b.check(q, n_q, hd ** -0.5, out, lse)


@pytest.mark.parametrize("bits", [3, 4, 8])
@pytest.mark.parametrize("H,share,hd", [(1, 6, 128), (1, 12, 128), (1, 16, 128), (1, 17, 128), (2, 7, 64), (4, 4, 32), (1, 8, 256), (1, 11, 256)])
def test_many_heads_of_a_workgroup(rp, H, share, hd, bits):
    """Page tables for so many tokens that a workgroup takes as many heads as it can."""
    b = Batch(rp, EDGES, H, hd, bits, 16)
    b.page_table = torch.cat([b.page_table, torch.full((len(EDGES), 1500), -1, dtype=torch.int32, device="cuda")], 1)
    n_q = H * share
    q = b.queries(n_q)
    out, lse = run(rp, b, q, n_q)
    b.check(q, n_q, hd ** -0.5, out, lse)


@pytest.mark.parametrize("bits,page,lens", [(4, 16, [9001]), (3, 64, [20011, 5]), (8, 256, [4096, 7000, 0, 12345]),
                                            (4, 128, [33000])])
def test_long_sequences(rp, bits, page, lens):
    b = Batch(rp, lens, 1, 128, bits, page)
    q = b.queries(4)
    out, lse = run(rp, b, q, 4)
    b.check(q, 4, 128 ** -0.5, out, lse)


def test_many_sequences(rp):
    lens = [int(n) for n in np.random.default_rng(3).integers(0, 200, 300)]
    b = Batch(rp, lens, 2, 64, 4, 16)
    q = b.queries(2)
    out, lse = run(rp, b, q, 2)
    b.check(q, 2, 64 ** -0.5, out, lse)


def test_many_sequences_some_of_them_long(rp):
    """More sequences than a wave has lanes, a few of them cut, and heads that are joined several at a time."""
    lens = [int(n) for n in np.random.default_rng(5).integers(0, 500, 140)]
    lens[3], lens[77], lens[139] = 6000, 2500, 5999
    b = Batch(rp, lens, 1, 128, 4, 64)
    q = b.queries(33)
    for dtype in (torch.float32, torch.bfloat16):
        out, lse = run(rp, b, q, 33, dtype)
        b.check(q, 33, 128 ** -0.5, out, lse)


@pytest.mark.parametrize("B", [1, 2, 63, 64, 65, 128, 129])
def test_batches_around_a_wave_of_lengths(rp, B):
    """Page tables for more than any sequence has, so that every sequence may be cut: one that is, wherever it stands, among short
    and empty ones; and nothing at all."""
    for long_one in sorted({0, B // 2, B - 1}):
        lens = [(7 * i + B) % 90 * (i % 5 != 0) for i in range(B)]
        lens[long_one] = 4000
        b = Batch(rp, lens, 1, 128, 3, 64, seed=B)
        b.page_table = torch.cat([b.page_table, torch.full((B, 100), -1, dtype=torch.int32, device="cuda")], 1)
        q = b.queries(2)
        out, lse = run(rp, b, q, 2)
        b.check(q, 2, 128 ** -0.5, out, lse)
    b.dev_lens = torch.zeros(B, dtype=torch.int32, device="cuda")
    out, lse = run(rp, b, q, 2)
    assert (out == 0).all() and (lse == -float("inf")).all()


@pytest.mark.parametrize("bits", [3, 4])
@pytest.mark.parametrize("H,share,hd", [(32, 1, 128), (32, 5, 128), (16, 1, 256)])
def test_pools_beyond_the_last_level_cache(rp, H, share, hd, bits):
    """More than 256 MiB of codes within reach of the page table, few of them taken."""
    b = Batch(rp, [300, 0, 65, 700], H, hd, bits, 64, extra_pages=1400)
    width = torch.full((4, 400), -1, dtype=torch.int32, device="cuda")
    width[:, :b.page_table.shape[1]] = b.page_table
    b.page_table = width
    assert 1400 * 2 * rp.rptq_kv_page_bytes(H * hd, 64, bits) > 1 << 28
    n_q = H * share
    q = b.queries(n_q)
    out, lse = run(rp, b, q, n_q)
    b.check(q, n_q, hd ** -0.5, out, lse)


def test_more_tiles_than_32_bits_count(rp):
    """Sequences of 2^27 tokens whose pages are there at the start and the end only: 2^31 tiles of 64 in the batch."""
    B, page, n_q = 1040, 4096, 2
    b = Batch(rp, [4 * page], 1, 128, 4, page, extra_pages=0)
    ids = b.table[0]
    q1 = b.queries(n_q)
    lens = (1 << 27) - 1000 * np.arange(B)
    width = (1 << 27) // page
    assert ((lens + 63) // 64).sum() > 1 << 31
    table = torch.full((B, width), -1, dtype=torch.int32, device="cuda")
    last = (lens - 1) // page
    first_id, last_id = ids[np.arange(B) % 3], ids[3]
    table[:, 0] = dev(first_id, np.int32)
    table[torch.arange(B, device="cuda"), dev(last, np.int64)] = int(last_id)
    b.page_table, b.dev_lens = table, dev(lens, np.int32)
    q = np.tile(q1, (B, 1))
    out, lse = run(rp, b, q, n_q)
    at = {int(i): n for n, i in enumerate(ids)}                # where a page's codes are in the sequence of four pages
    for row in (0, 1, 2, 500, 1038, 1039):
        tail = int(lens[row]) - int(last[row]) * page
        tokens = np.r_[at[int(first_id[row])] * page + np.arange(page), at[int(last_id)] * page + np.arange(tail)]
        k, v = b.k[0][tokens], b.v[0][tokens]
        want, wl = kvo.attend(q[row], k, v, b.hk, 0, b.hv, 0, n_q, 128 ** -0.5)
        tol, tl = paged.attend_bounds(q[row], k, b.hk, b.hv, n_q, 128 ** -0.5, 4, want, wl)
        assert (np.abs(out[row].double().cpu().numpy() - want) <= tol).all(), row
        assert (np.abs(lse[row].double().cpu().numpy() - wl) <= tl).all(), row
    assert torch.isfinite(out).all() and torch.isfinite(lse).all()


def test_the_largest_batch(rp):
    """As many sequences and query heads as there may be at once."""
    if torch.cuda.mem_get_info()[0] < 24 << 30:
        pytest.skip("not enough free memory")
    B, n_q, hd = 32768, 1024, 32
    b = Batch(rp, [300, 2, 0, 65], 4, hd, 4, 16)
    few = b.queries(n_q)
    kind = torch.arange(B, device="cuda") % 4
    q = dev_bf16(few)[kind]
    out = torch.full((B, n_q * hd), float("nan"), dtype=torch.bfloat16, device="cuda")
    _, lse = rp.attend_paged(b.cache, q, b.page_table[kind], b.dev_lens[kind], out=out, want_lse=True)
    b.check(few, n_q, hd ** -0.5, out[:4], lse[:4])
    assert torch.equal(out.view(-1, 4, n_q * hd), out[:4].expand(B // 4, -1, -1))
    assert torch.equal(lse.view(-1, 4, n_q), lse[:4].expand(B // 4, -1, -1))


@pytest.mark.parametrize("page,holes", [(16, (0,)), (16, (1, 2, 3, 5)), (64, (0, 2)), (32, tuple(range(64))), (16, tuple(range(0, 80, 3)))])
def test_pages_that_are_not_there(rp, page, holes):
    """Tokens of a page that is not there take no part, wherever it lies, and a sequence may lose all of its pages."""
    b = Batch(rp, [1, 40, 64, 130, 700, 1100], 2, 64, 4, page, holes=holes)
    q = b.queries(4)
    out, lse = run(rp, b, q, 4)
    b.check(q, 4, 64 ** -0.5, out, lse)


def test_lengths_outside_the_table_are_clamped(rp):
    b = Batch(rp, [64, 64, 64, 10], 1, 128, 4, 16)
    q = b.queries(2)
    want, want_lse = run(rp, b, q, 2)
    b.dev_lens = dev([64, 65, 2 ** 31 - 1, 10], np.int32)
    out, lse = run(rp, b, q, 2)
    assert torch.equal(out[:3], want[:3]) and torch.equal(lse[:3], want_lse[:3])
    b.dev_lens = dev([64, -1, -2 ** 31, 10], np.int32)
    out, lse = run(rp, b, q, 2)
    assert (out[1:3] == 0).all() and (lse[1:3] == -float("inf")).all()


@pytest.mark.parametrize("sharp", [0.0, 1e-30, 30.0, 3000.0])
def test_flat_and_sharp_scores(rp, sharp):
    """From all weights equal to one weight only, and scores of thousands."""
    b = Batch(rp, [500, 1, 77], 2, 128, 4, 16)
    q = b.queries(4, sharp)
    out, lse = run(rp, b, q, 4)
    b.check(q, 4, 128 ** -0.5, out, lse)


def test_a_weight_beside_many_small_ones(rp):
    """One token far above 20000 others whose weights only matter together."""
    H, hd, bits, page, n = 1, 128, 4, 64, 20000
    b = Batch(rp, [n], H, hd, bits, page)
    s, _, _ = kvo.position_tables(b.hk, 0)
    codes = np.zeros((n, hd), np.int64)
    codes[:, 0] = -1
    codes[7777, 0] = 7
    codes[:, 1] = np.random.default_rng(0).integers(-2, 2, n)
    pages = np.zeros((n // page + 3, 1, page, 16 * bits), np.uint8)
    slots = b.table[0][np.arange(n) // page] * page + np.arange(n) % page
    paged.put(pages, slots, paged.page_rows(codes, bits), page)
    b.cache.k_pages = dev(pages[:b.cache.k_pages.shape[0]])
    b.k = [codes]
    q = np.zeros((1, hd), np.float32)
    q[0, b.hk.perm[0]] = 1.7 / s[0]                           # 8 codes apart: 13.6 / ln 2 = 2^19.6
    q[0, b.hk.perm[1]] = 0.3 / s[1]
    q = kvo.round_to_bf16(q)
    out, lse = run(rp, b, q, 1, scale=1.0)
    b.check(q, 1, 1.0, out, lse)


def test_scale_and_equal_keys(rp):
    b = Batch(rp, [100, 260], 2, 64, 8, 16)
    q = b.queries(2)
    for scale in (1.0, -0.3, 0.0):
        out, lse = run(rp, b, q, 2, scale=scale)
        b.check(q, 2, scale, out, lse)


def test_queries_that_are_not_finite_touch_their_head_only(rp):
    b = Batch(rp, [100, 260, 0], 2, 64, 4, 16)
    q = b.queries(4)
    want, want_lse = run(rp, b, q, 4)
    bad = q.copy().reshape(3, 4, 64)
    bad[0, 1, 5], bad[1, 0, 0], bad[1, 3, 63] = np.nan, np.inf, -np.inf
    out, lse = run(rp, b, bad.reshape(3, -1), 4)
    hit = torch.zeros(3, 4, dtype=torch.bool, device="cuda")
    hit[0, 1] = hit[1, 0] = hit[1, 3] = True
    out, want = out.view(3, 4, 64), want.view(3, 4, 64)
    assert torch.equal(out[~hit], want[~hit]) and torch.equal(lse[~hit], want_lse[~hit])
    assert out[hit].isnan().all() and lse[hit].isnan().all()


def test_strides_and_what_lies_around(rp):
    """q, out and the page table as parts of wider tensors; what lies beside the outputs stays."""
    b = Batch(rp, [100, 260, 0, 17], 2, 64, 4, 16)
    q = b.queries(4)
    want, want_lse = run(rp, b, q, 4)
    n = q.shape[1]
    wide_q = torch.full((4, 3 * n + 8), float("nan"), dtype=torch.bfloat16, device="cuda")
    wide_q[:, 8:8 + n] = dev_bf16(q)
    wide_out = torch.full((6, 2 * n), 5.0, device="cuda")
    lse = torch.full((6, 4), 5.0, device="cuda")
    wide_table = torch.full((4, b.page_table.shape[1] + 3), 2 ** 30, dtype=torch.int32, device="cuda")
    wide_table[:, 1:-2] = b.page_table
    rp.attend_paged(b.cache, wide_q[:, 8:8 + n], wide_table[:, 1:-2], b.dev_lens, out=wide_out[1:5, n:], lse=lse[1:5])
    torch.cuda.synchronize()
    assert torch.equal(wide_out[1:5, n:], want) and torch.equal(lse[1:5], want_lse)
    assert (wide_out[:, :n] == 5.0).all() and (wide_out[[0, 5]] == 5.0).all() and (lse[[0, 5]] == 5.0).all()
    # the workspace's size is kept to
    need = rp.rptq_attend_paged_workspace_bytes(4, 4, 2, 64)
    ws = torch.full((need + 4096,), 0x5A, dtype=torch.uint8, device="cuda")
    out, lse = run(rp, b, q, 4, workspace=ws[:need])
    assert torch.equal(out, want) and (ws[need:] == 0x5A).all()
    with pytest.raises(rp.RptqError, match="-7"):
        run(rp, b, q, 4, workspace=ws[:need - 1])


def test_the_same_bits_every_time(rp):
    b = Batch(rp, [3000, 1, 700, 64], 2, 128, 4, 64)
    q = b.queries(8)
    first, first_lse = run(rp, b, q, 8)
    for _ in range(5):
        out, lse = run(rp, b, q, 8)
        assert torch.equal(out, first) and torch.equal(lse, first_lse)


def test_other_streams(rp):
    b = Batch(rp, [3000, 1, 700, 64], 2, 128, 4, 64)
    q = b.queries(8)
    want, _ = run(rp, b, q, 8)
    streams = [torch.cuda.Stream() for _ in range(2)]
    qs, outs = dev_bf16(q), [torch.zeros_like(want) for _ in streams]
    work = [rp.attend_paged_workspace(b.cache, 4, 8) for _ in streams]
    torch.cuda.synchronize()
    for _ in range(10):
        for s, o, ws in zip(streams, outs, work):
            with torch.cuda.stream(s):
                o.zero_()
                rp.attend_paged(b.cache, qs, b.page_table, b.dev_lens, out=o, workspace=ws)
    torch.cuda.synchronize()
    assert all(torch.equal(o, want) for o in outs)


def test_recorded_steps_replay(rp):
    """A decoding step (write, attend, read back) recorded once and replayed as the sequences grow: lengths, slots and pages
    are read on the device.  Two graphs share a workspace."""
    H, hd, bits, page, B, n_q = 2, 64, 4, 16, 3, 4
    (hk, klo, khi), (hv, vlo, vhi), kt, vt = site(H, hd, bits)
    d, steps = H * hd, 40
    cache = rp.paged_cache(16, page, H, hd, bits, kt, vt)
    eager = rp.paged_cache(16, page, H, hd, bits, kt, vt)
    rng = np.random.default_rng(4)
    table = dev(rng.permutation(16)[:12].reshape(3, 4), np.int32)
    k, v = (torch.zeros(B, d, dtype=torch.bfloat16, device="cuda") for _ in range(2))
    q = torch.zeros(B, n_q * hd, dtype=torch.bfloat16, device="cuda")
    lens, slots = torch.zeros(B, dtype=torch.int32, device="cuda"), torch.full((B,), -1, dtype=torch.int64, device="cuda")
    ws = rp.attend_paged_workspace(cache, B, n_q)

    def step(cache):
        rp.kv_quant_paged(cache, k, v, slots)
        out, lse = rp.attend_paged(cache, q, table, lens, want_lse=True, workspace=ws)
        return (out, lse) + rp.kv_dequant_paged(cache, slots)

    step(eager)
    torch.cuda.synchronize()
    graphs, results = [], []
    for _ in range(2):
        g = torch.cuda.CUDAGraph()
        with torch.cuda.graph(g):
            results.append(step(cache))
        graphs.append(g)
    for i in range(steps):
        have = lens.cpu().numpy()
        grow = np.array([1, i % 2, 1 if i > 20 else 0])
        at = table.cpu().numpy()[np.arange(3), have // page] * page + have % page
        slots.copy_(dev(np.where(grow, at, -1), np.int64))
        lens.copy_(dev(have + grow, np.int32))
        k.copy_(dev_bf16(paged.values(rng, klo, khi, B)))
        v.copy_(dev_bf16(paged.values(rng, vlo, vhi, B)))
        q.copy_(dev_bf16((rng.standard_normal((B, n_q * hd)) * 0.05).astype(np.float32)))
        graphs[i % 2].replay()
        torch.cuda.synchronize()
        replayed = [t.clone() for t in results[i % 2]]
        for a, b in zip(replayed, step(eager)):
            assert torch.equal(a, b)
        assert torch.equal(cache.k_pages, eager.k_pages) and torch.equal(cache.v_pages, eager.v_pages)
    assert lens.tolist() == [40, 20, 19]


def test_a_decoding_layer(rp):
    """The operators as they are used: an RPTQ projection gives queries, keys and values, the new tokens go into the cache and
    attention answers, step after step, against the oracle on the tensors that the projection gave."""
    d_model, H, n_q, hd, bits, page, B, steps = 256, 2, 4, 64, 4, 16, 3, 21
    rng = np.random.default_rng(8)
    gen = torch.Generator(device="cuda").manual_seed(8)
    cal = [torch.randn(64, d_model, generator=gen, device="cuda").bfloat16() for _ in range(2)]
    gamma, beta = torch.ones(d_model, device="cuda"), torch.zeros(d_model, device="cuda")
    at = rp.calibrate_site(cal, gamma, beta, 1e-5, False, 8, 8, seed=1)
    W = torch.randn((n_q + 2 * H) * hd, d_model, generator=gen, device="cuda") * 0.06
    lin = rp.fold_linear(at, W)

    def project(x):
        codes, _, rowterm = rp.ln_quant(at, x)
        return rp.cluster_gemm(at, lin, codes, rowterm, x.shape[0])

    seen = torch.cat([project(x) for x in cal]).float().cpu().numpy()
    nq, d = n_q * hd, H * hd
    sites, tables = [], []
    for x in (seen[:, nq:nq + d], seen[:, nq + d:]):
        hc = kvo.cluster_heads([x.min(0)], [x.max(0)], H, 4, bits, 2)
        table = torch.empty(rp.rptq_kv_table_bytes(d), dtype=torch.uint8, device="cuda")
        rp.rptq_kv_tables(hc.perm, hc.cluster_off, hc.s[0], hc.inv_s[0], hc.z[0], d, H, 4, table)
        sites.append(hc)
        tables.append(table)
    cache = rp.paged_cache(8, page, H, hd, bits, *tables)
    ids = rng.permutation(8)[:6].reshape(3, 2)
    page_table = dev(ids, np.int32)
    past = [[], []]
    for i in range(steps):
        qkv = project(torch.randn(B, d_model, generator=gen, device="cuda").bfloat16())
        q, k, v = qkv[:, :nq], qkv[:, nq:nq + d], qkv[:, nq + d:]
        rp.kv_quant_paged(cache, k, v, dev(ids[:, i // page] * page + i % page, np.int64))
        out, lse = rp.attend_paged(cache, q, page_table, dev([i + 1] * B, np.int32), out=torch.empty(B, nq, device="cuda"), want_lse=True)
        for p, x, hc in zip(past, (k, v), sites):
            p.append(kvo.kv_quant(x.float().cpu().numpy(), hc, 0, bits))
        for b in range(B):
            kc, vc = np.stack([c[b] for c in past[0]]), np.stack([c[b] for c in past[1]])
            qb = q[b].float().cpu().numpy()
            want, wl = kvo.attend(qb, kc, vc, sites[0], 0, sites[1], 0, n_q, hd ** -0.5)
            tol, tl = paged.attend_bounds(qb, kc, sites[0], sites[1], n_q, hd ** -0.5, bits, want, wl)
            assert (np.abs(out[b].double().cpu().numpy() - want) <= tol).all()
            assert (np.abs(lse[b].double().cpu().numpy() - wl) <= tl).all()


def test_refusals(rp):
    b = Batch(rp, [10, 20], 2, 64, 4, 16)
    c, q = b.cache, torch.zeros(2, 128, dtype=torch.bfloat16, device="cuda")
    x, slots = torch.zeros(3, 128, dtype=torch.bfloat16, device="cuda"), torch.zeros(3, dtype=torch.int64, device="cuda")
    with pytest.raises(ValueError, match="dtype"):
        rp.kv_quant_paged(c, x.float(), x, slots)
    with pytest.raises(ValueError, match="dtype"):
        rp.kv_quant_paged(c, x, x, slots.int())
    with pytest.raises(ValueError, match="one per row"):
        rp.kv_quant_paged(c, x, x, slots[:2])
    with pytest.raises(ValueError, match="T, d"):
        rp.kv_quant_paged(c, x, x[:, :64], slots)
    with pytest.raises(ValueError, match="contiguous rows"):
        rp.kv_quant_paged(c, x.t().contiguous().t(), x, slots)
    with pytest.raises(ValueError, match="table"):
        rp.rptq_kv_quant_paged(x, x, slots, c.k_table[:100], c.v_table, 4, c.k_pages, c.v_pages, 16)
    with pytest.raises(ValueError, match="pages"):
        rp.rptq_kv_quant_paged(x, x, slots, c.k_table, c.v_table, 4, c.k_pages[:1], c.v_pages, 16)
    with pytest.raises(ValueError, match="pages"):
        rp.rptq_kv_dequant_paged(c.k_pages.view(-1)[:-16], c.v_pages.view(-1)[:-16], 16, 4, slots, c.k_table, c.v_table, x, x)
    with pytest.raises(rp.RptqError, match="-2"):
        rp.rptq_kv_quant_paged(x, x, slots, c.k_table, c.v_table, 4, c.k_pages, c.v_pages, 24)
    with pytest.raises(rp.RptqError, match="-3"):
        rp.rptq_kv_quant_paged(x, x, slots, c.k_table, c.v_table, 5, c.k_pages, c.v_pages, 16)
    with pytest.raises(rp.RptqError, match="-2"):                    # one row's columns are another's
        rp.kv_quant_paged(c, x[:1].expand(3, 128), x, slots)
    with pytest.raises(rp.RptqError, match="-4"):
        rp.kv_quant_paged(c, torch.zeros(3, 136, dtype=torch.bfloat16, device="cuda")[:, 4:132], x, slots)
    with pytest.raises(ValueError, match="bf16 or fp32"):
        rp.attend_paged(c, q, b.page_table, b.dev_lens, out=q.half())
    with pytest.raises(ValueError, match="shape"):
        rp.attend_paged(c, q, b.page_table, b.dev_lens, out=q[:1])
    with pytest.raises(ValueError, match="lens"):
        rp.attend_paged(c, q, b.page_table, b.dev_lens[:1])
    with pytest.raises(ValueError, match="dtype"):
        rp.attend_paged(c, q, b.page_table.long(), b.dev_lens)
    with pytest.raises(ValueError, match="lse"):
        rp.attend_paged(c, q, b.page_table, b.dev_lens, lse=torch.zeros(3, device="cuda"))
    with pytest.raises(rp.RptqError, match="-6"):
        rp.attend_paged(c, q, b.page_table, b.dev_lens, scale=float("inf"))
    with pytest.raises(rp.RptqError, match="-2"):                    # three query heads on two
        rp.attend_paged(c, torch.zeros(2, 192, dtype=torch.bfloat16, device="cuda"), b.page_table, b.dev_lens)
    with pytest.raises(ValueError, match="device"):
        rp.attend_paged(c, q.cpu(), b.page_table, b.dev_lens, out=q, workspace=c.k_pages)


def test_calls_of_nothing(rp):
    b = Batch(rp, [10, 20], 2, 64, 4, 16)
    x, slots = torch.zeros(0, 128, dtype=torch.bfloat16, device="cuda"), torch.zeros(0, dtype=torch.int64, device="cuda")
    before = b.cache.k_pages.clone()
    rp.kv_quant_paged(b.cache, x, x, slots)
    k, v = rp.kv_dequant_paged(b.cache, slots)
    assert k.shape == v.shape == (0, 128) and torch.equal(b.cache.k_pages, before)
    out, lse = rp.attend_paged(b.cache, x, b.page_table[:0], b.dev_lens[:0], want_lse=True)
    assert out.shape == (0, 128) and lse.shape == (0, 2)


def test_native_and_python_marshalling(rp, monkeypatch):
    """Ordinary arguments are taken natively, with the results that the Python marshalling leads to; an argument out of the
    ordinary, whichever it is, is not (None, and nothing written)."""
    from paper_2304_01089_amd import binding
    b = Batch(rp, [100, 37], 2, 64, 4, 16)
    c, gen = b.cache, torch.Generator(device="cuda").manual_seed(1)
    wide = torch.randn(3, 400, generator=gen, device="cuda").bfloat16()
    k, v, slots = wide[:, :128], wide[:, 128:256], torch.tensor([3, 70, -1], device="cuda")
    pages = c.k_pages.clone(), c.v_pages.clone()
    back = torch.zeros(2, 3, 128, dtype=torch.bfloat16, device="cuda")
    q, out, lse = wide[:2, 136:392], torch.zeros(2, 256, device="cuda"), torch.zeros(2, 4, device="cuda")
    ws = rp.attend_paged_workspace(c, 2, 4)
    calls = [
        ("kv_quant_paged", (k, v, slots, c.k_table, c.v_table, 4) + pages + (16, None), pages),
        ("kv_dequant_paged", pages + (16, 4, slots, c.k_table, c.v_table, back[0], back[1], None), (back,)),
        ("attend_paged", (q, 4, 2, 64, 0.125, c.k_table, c.v_table, 4, c.k_pages, c.v_pages, 16, b.page_table, b.dev_lens, out, lse, ws, None),
         (out, lse)),
        ("attend_paged", (q, 4, 2, 64, 0.125, c.k_table, c.v_table, 4, c.k_pages, c.v_pages, 16, b.page_table, b.dev_lens, out.bfloat16(), None,
                          ws, None), ()),
    ]
    for name, args, outs in calls:
        native, entry = getattr(binding._CALLS, name), getattr(rp, "rptq_" + name)
        start = [t.clone() for t in outs]
        assert native(*args) == 0, name
        got = [t.clone() for t in outs]
        assert not outs or any(not torch.equal(a, s) for a, s in zip(got, start))
        for t, s in zip(outs, start):
            t.copy_(s)
        with monkeypatch.context() as m:
            m.setattr(binding, "_CALLS", None)
            m.setattr(binding, "_CALLS_SOUGHT", True)
            entry(*args)
        assert all(torch.equal(a, t) for a, t in zip(got, outs)), name
        for t in outs:
            t.view(torch.uint8).fill_(0x3c)
        torch.cuda.synchronize()
        for i, a in enumerate(args):
            if isinstance(a, torch.Tensor):
                odd = [a.cpu(), a.to(torch.float64 if a.dtype != torch.float64 else torch.int8), 1, a[None], a.reshape(-1)[:1]]
                if a is not lse:
                    odd.append(None)
                if a is ws or a is c.k_table or a is c.v_table:            # (bytes of any type, as long as there are enough)
                    odd = [a.cpu(), 1, None] + ([a.reshape(-1)[:8]] if a is not ws else [])
                elif a is lse or a.dtype == torch.uint8:                   # (any shape)
                    odd = odd[:3] + odd[4:]
                if a is pages[0] or a is pages[1] or a is c.k_pages or a is c.v_pages:
                    odd.append(a[:-1])
            elif a is None:
                odd = [torch.cuda.current_stream()] if i == len(args) - 1 else [1]
            elif isinstance(a, float):
                odd = [1, np.float32(0.1)]
            else:
                odd = [float(a), np.int64(a), 1 << 80, 0, -a]
            for o in odd:
                assert native(*args[:i], o, *args[i + 1:]) is None, (name, i, o)
        assert native(*args[:-1]) is None and native(*args, None) is None, name
        torch.cuda.synchronize()
        assert all((t.view(torch.uint8) == 0x3c).all() for t in outs), name


@pytest.mark.parametrize("lens", [[3], [16], [16, 5], [1, 0, 7]])
def test_tables_of_one_page_are_marshalled_natively(rp, lens):
    from paper_2304_01089_amd import binding
    b = Batch(rp, lens, 2, 64, 4, 16)
    assert b.page_table.shape[1] == 1
    q = b.queries(4)
    out, ws = torch.full((len(lens), 256), float("nan"), device="cuda"), rp.attend_paged_workspace(b.cache, len(lens), 4)
    c = b.cache
    assert binding._CALLS.attend_paged(dev_bf16(q), 4, 2, 64, 0.125, c.k_table, c.v_table, 4, c.k_pages, c.v_pages, 16, b.page_table,
                                       b.dev_lens, out, None, ws, None) == 0
    torch.cuda.synchronize()
    b.check(q, 4, 0.125, out)
