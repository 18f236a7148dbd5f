"""Attention weights added up per token of the paged cache, and eviction by them, on the GPU against plain forms in 64 bits; then
everything together as a serving loop runs it."""
import numpy as np
import pytest

from oracle import kv_cache as kvo

import bounding
import paged
from test_gpu_paged import Batch, dev, dev_bf16, site

pytestmark = pytest.mark.gpu
torch = pytest.importorskip("torch")


@pytest.fixture(scope="module")
def rp():
    import paper_2304_01089_amd as rp_
    rp_.load_library()
    assert torch.cuda.is_available()
    return rp_


def there(batch, b):
    """Indices of the tokens of sequence b whose pages are there (batch.k[b]'s rows)."""
    n = max(int(batch.lens[b]), 0)
    page = batch.cache.page_size
    ids = batch.table[b][np.arange(n) // page]
    return np.flatnonzero((ids >= 0) & (ids < batch.cache.k_pages.shape[0]))


def window(rp, batch, n_q, queries, sharp=1.0):
    """Queries [B * queries, n_q hd] for the last tokens of every sequence, and what the attention leaves as lse (float32)."""
    s, _, _ = kvo.position_tables(batch.hk, 0)
    H, hd = batch.H, batch.hd
    norm = np.sqrt((s.reshape(H, hd) ** 2).sum(1)) * 2.0 ** batch.bits / 3.5
    t = sharp * 2.0 * np.sqrt(hd) / np.repeat(norm, n_q // H)
    B = len(batch.lens)
    q = kvo.round_to_bf16((batch.rng.standard_normal((B * queries, n_q, hd)) * t[None, :, None]).astype(np.float32)).reshape(B * queries, -1)
    lse = np.full((B * queries, n_q), -np.inf)
    for b in range(B):
        at = there(batch, b)
        for i in range(queries):
            sees = at < max(int(batch.lens[b]), 0) - (queries - 1 - i)
            lse[b * queries + i] = kvo.attend(q[b * queries + i], batch.k[b][sees], batch.v[b][sees], batch.hk, 0, batch.hv, 0, n_q, hd ** -0.5)[1]
    return q, lse.astype(np.float32)


def accumulate(rp, batch, n_q, queries, fresh, capacity, positions=True, seed=0, q_lse=None):
    """One call against the plain form; returns the track."""
    rng = np.random.default_rng(seed)
    B, H = len(batch.lens), batch.H
    q, lse = window(rp, batch, n_q, queries) if q_lse is None else q_lse
    w0 = rng.random((B, H, capacity)).astype(np.float32)
    p0 = rng.integers(0, 1000, (B, H, capacity)).astype(np.int32)
    newest = rng.integers(5000, 6000, B).astype(np.int32)
    track = rp.CacheTrack(dev(w0), dev(p0))
    rp.attend_weights_paged(batch.cache, dev_bf16(q), batch.page_table, batch.dev_lens, dev(lse), track, positions=dev(newest) if positions else None,
                            queries=queries, fresh=fresh)
    torch.cuda.synchronize()
    got, gp = track.weights.double().cpu().numpy(), track.positions.cpu().numpy()
    for b in range(B):
        n = min(max(int(batch.lens[b]), 0), capacity, batch.table.shape[1] * batch.cache.page_size)
        at = there(batch, b)
        at, codes = at[at < n], batch.k[b][at < n]
        sums, tol = bounding.weights64(q[b * queries:(b + 1) * queries], lse[b * queries:(b + 1) * queries], codes, at, n, batch.hk, n_q, batch.hd ** -0.5, queries)
        start = max(0, n - fresh)
        old = w0[b].astype(np.float64)
        old[:, start:n] = 0.0
        want, near = old.copy(), np.zeros_like(old)
        want[:, at] += sums
        near[:, at] = tol + bounding.U * (old[:, at] + sums) * (queries * n_q // H // 64 + 2)
        assert (np.abs(got[b] - want) <= near).all(), (b, n, (np.abs(got[b] - want) / np.maximum(near, 1e-300)).max())
        t = np.arange(start, n)
        want_p = p0[b].copy()
        want_p[:, start:n] = newest[b] - (n - 1 - t) if positions else t
        assert np.array_equal(gp[b], want_p), b
    return track


EDGES = [0, 1, 2, 15, 17, 63, 64, 65, 127, 255, 256, 257, 300, 513]


@pytest.mark.parametrize("bits", [3, 4, 8])
@pytest.mark.parametrize("H,share,hd,page", [(4, 1, 32, 16), (8, 2, 32, 32), (4, 3, 32, 16), (2, 1, 64, 16), (2, 2, 64, 16), (4, 5, 64, 32), (1, 1, 128, 16), (2, 4, 128, 64),
                                             (1, 7, 128, 128), (1, 1, 256, 16), (2, 6, 256, 32)])
def test_lengths_around_every_edge(rp, H, share, hd, page, bits):
    accumulate(rp, Batch(rp, EDGES, H, hd, bits, page), H * share, 1, 1, 530)


@pytest.mark.parametrize("queries,fresh", [(1, 0), (2, 2), (3, 1000), (5, 0), (17, 40), (64, 1 << 30)])
@pytest.mark.parametrize("H,share,hd,bits", [(4, 1, 32, 4), (2, 1, 64, 8), (1, 4, 128, 3), (1, 3, 256, 4), (2, 2, 64, 4)])
def test_windows_of_queries(rp, H, share, hd, bits, queries, fresh):
    """Several queries of a sequence, more of them than tokens in some; more row tiles than are held at a time."""
    accumulate(rp, Batch(rp, [0, 1, 3, 40, 64, 300], H, hd, bits, 16), H * share, queries, fresh, 300, positions=queries != 3)


def test_many_heads_on_one(rp):
    accumulate(rp, Batch(rp, [700, 5], 1, 128, 4, 64), 96, 3, 10, 1000)


@pytest.mark.parametrize("holes", [(0,), (1, 2), (0, 1, 2, 3)])
def test_pages_that_are_not_there(rp, holes):
    accumulate(rp, Batch(rp, [0, 16, 17, 64, 200], 2, 64, 4, 16, holes=holes), 4, 3, 70, 200)


def test_records_shorter_than_the_sequences(rp):
    b = Batch(rp, [100, 300, 37], 2, 64, 4, 16)
    q, lse = window(rp, b, 2, 1)
    b.lens = [100, 100, 37]                                           # (what a capacity of 100 makes of them)
    b.k, b.v = [k[:100] for k in b.k], [v[:100] for v in b.v]
    accumulate(rp, b, 2, 1, 5, 100, q_lse=(q, lse))


def test_lengths_outside_the_table(rp):
    b = Batch(rp, [32, 48], 2, 64, 4, 16)
    q, lse = window(rp, b, 2, 1)
    b.dev_lens = dev([-7, 2 ** 31 - 1], np.int32)
    b.lens, b.k, b.v = [0, 48], [b.k[0][:0], b.k[1]], [b.v[0][:0], b.v[1]]
    accumulate(rp, b, 2, 1, 5, 64, q_lse=(q, lse))


@pytest.mark.parametrize("bits", [3, 4])
def test_long_sequences(rp, bits):
    """More tiles than there are parts, the sums of a sequence's weights near the number of its query heads."""
    b = Batch(rp, [20000, 777, 9000], 1, 128, bits, 64)
    track = accumulate(rp, b, 4, 1, 1 << 29, 20000)
    total = track.weights.double().sum(-1).cpu().numpy()[:, 0]
    assert np.allclose(total[0], 4.0, atol=1e-4)


def test_the_attention_that_left_the_sums(rp):
    """lse from attend_paged itself: the weights of a sequence's tokens add up to one per query head."""
    H, share, hd, bits = 2, 3, 64, 4
    b = Batch(rp, [1000, 64, 1, 333], H, hd, bits, 16)
    q = b.queries(H * share)
    _, lse = rp.attend_paged(b.cache, dev_bf16(q), b.page_table, b.dev_lens, want_lse=True)
    track = rp.cache_track(b.cache, 4, 1000)
    rp.attend_weights_paged(b.cache, dev_bf16(q), b.page_table, b.dev_lens, lse, track, fresh=1000)
    total = track.weights.double().sum(-1).cpu().numpy()
    # (every weight's error bound, and the logarithm's own)
    assert np.abs(total - share).max() < 2e-4
    assert torch.equal(track.positions[0, 0], torch.arange(1000, dtype=torch.int32, device="cuda"))


def test_queries_that_are_not_finite(rp):
    b = Batch(rp, [50, 20], 2, 64, 4, 16)
    q, lse = window(rp, b, 4, 1)
    clean, bad = (rp.cache_track(b.cache, 2, 64) for _ in range(2))
    rp.attend_weights_paged(b.cache, dev_bf16(q), b.page_table, b.dev_lens, dev(lse), clean, fresh=64)
    q[0, 3 * 64 + 5] = np.nan                                          # query head 3: key/value head 1
    rp.attend_weights_paged(b.cache, dev_bf16(q), b.page_table, b.dev_lens, dev(lse), bad, fresh=64)
    assert torch.isnan(bad.weights[0, 1, :50]).all() and (bad.weights[0, 1, 50:] == 0).all()
    assert torch.equal(bad.weights[0, 0], clean.weights[0, 0]) and torch.equal(bad.weights[1], clean.weights[1])


# ---- eviction --------------------------------------------------------------------------------------------------
def evicted(rp, batch, budget, first, recent, weights, positions, capacity, in_place, garbage=0):
    """One call against the plain form, every byte of the pages compared."""
    c, H, hd, bits, page = batch.cache, batch.H, batch.hd, batch.bits, batch.cache.page_size
    before = [t.cpu().numpy().copy() for t in (c.k_pages, c.v_pages)]
    want = [t.copy() for t in before]
    track = rp.CacheTrack(dev(weights), dev(positions))
    out = track if in_place else rp.CacheTrack(torch.full_like(track.weights, 7.5), torch.full_like(track.positions, -9))
    start = [t.cpu().numpy().copy() for t in (out.weights, out.positions)]
    workspace = rp.evict_paged_workspace(c, len(batch.lens), capacity, budget).fill_(0xA5)
    lens = rp.evict_paged(c, batch.page_table, batch.dev_lens, track, budget, first=first, recent=recent, out=None if in_place else out, workspace=workspace)
    torch.cuda.synchronize()
    n_pages, row = before[0].shape[0], hd * bits // 8
    for b in range(len(batch.lens)):
        n = min(max(int(batch.lens[b]), 0), capacity, batch.table.shape[1] * page)
        used = batch.table[b][:(n + page - 1) // page]
        cut = n > budget and ((used >= 0) & (used < n_pages)).all()
        left = budget if cut else n
        assert lens[b].item() == left, b
        for h in range(H):
            src = bounding.evict(weights[b, h, :n], positions[b, h, :n], budget, first, recent) if cut else np.arange(n)
            start[0][b, h, :left], start[1][b, h, :left] = weights[b, h][src], positions[b, h][src]
            for t in np.flatnonzero(src != np.arange(left)):
                for p, q in zip(want, before):
                    a, z = (batch.table[b][i // page] for i in (t, src[t]))
                    for part in range(max(1, hd // 128)):
                        blk, off = (h * hd + part * 128) // 128, (h * hd + part * 128) % 128 * bits // 8
                        size = min(row, 16 * bits)
                        p[a, blk, t % page, off:off + size] = q[z, blk, src[t] % page, off:off + size]
    for got, p in zip((c.k_pages, c.v_pages), want):
        assert np.array_equal(got.cpu().numpy(), p)
    assert np.array_equal(out.weights.cpu().numpy().view(np.int32), start[0].view(np.int32)) and np.array_equal(out.positions.cpu().numpy(), start[1])
    if not in_place:
        assert torch.equal(track.weights.view(torch.int32), dev(weights).view(torch.int32)) and torch.equal(track.positions, dev(positions))
    return lens, out


def records(rng, B, H, capacity, ties=False):
    w = np.exp(2.0 * rng.standard_normal((B, H, capacity))).astype(np.float32)
    if ties:
        w = np.round(w * 2) / 2
    w[rng.random(w.shape) < 0.05] = 0.0
    p = np.stack([np.stack([rng.permutation(2 * capacity)[:capacity] for _ in range(H)]) for _ in range(B)]).astype(np.int32)
    return w.astype(np.float32), p


@pytest.mark.parametrize("in_place", [True, False])
@pytest.mark.parametrize("bits", [3, 4, 8])
@pytest.mark.parametrize("H,hd,page,budget,first,recent", [(4, 32, 16, 60, 0, 0), (2, 64, 16, 17, 4, 13), (3, 128, 32, 100, 3, 20), (2, 256, 16, 1, 0, 1), (2, 256, 64, 250, 0, 250),
                                                           (1, 128, 16, 299, 0, 0), (8, 32, 128, 128, 128, 0)])
def test_heads_keep_their_heaviest(rp, H, hd, page, budget, first, recent, bits, in_place):
    lens = [0, 1, budget - 1, budget, budget + 1, 300, 257, 64]
    b = Batch(rp, lens, H, hd, bits, page)
    w, p = records(np.random.default_rng(budget + hd), len(lens), H, 310, ties=budget == 100)
    evicted(rp, b, budget, first, recent, w, p, 310, in_place)


@pytest.mark.parametrize("n,budget", [(2049, 2048), (4096, 1), (8192, 5000), (8193, 4000), (32768, 16384), (32769, 16000), (33000, 32999), (70001, 300), (40000, 20001)])
def test_long_sequences_cut(rp, n, budget):
    """Every way of holding the keys and of moving the rows, at its ends."""
    b = Batch(rp, [n, n // 3, n - 1], 1, 128, 3, 64)
    w, p = records(np.random.default_rng(n), 3, 1, n, ties=n % 2 == 0)
    evicted(rp, b, budget, 4, min(100, budget - 4) if budget > 4 else 0, w, p, n, n % 3 == 0) if budget > 4 else \
        evicted(rp, b, budget, 0, 0, w, p, n, True)


@pytest.mark.parametrize("n,budget", [(8300, 8200), (8400, 5000), (10000, 2)])
def test_many_heads_of_long_sequences(rp, n, budget):
    """As many heads as fill the chip with a workgroup each."""
    b = Batch(rp, [n, n - 1, 64], 44, 32, 3, 128)
    w, p = records(np.random.default_rng(n), 3, 44, n)
    evicted(rp, b, budget, 0, budget // 3, w, p, n, n == 8400)


@pytest.mark.parametrize("what", ["all equal", "all zero", "zeros of both signs", "infinities and nan", "negative", "ends of the range", "steps of the last bit", "steps of the last bits", "safe ones first"])
def test_orders_of_weights(rp, what):
    rng = np.random.default_rng(6)
    n, budget = 500, 123
    w, p = records(rng, 2, 2, n)
    if what == "all equal":
        w[:] = 0.375
    elif what == "all zero":
        w[:] = 0.0
    elif what == "zeros of both signs":
        w[:] = np.where(rng.random(w.shape) < 0.5, -0.0, 0.0)
    elif what == "infinities and nan":
        w[rng.random(w.shape) < 0.1] = np.inf
        w[rng.random(w.shape) < 0.1] = np.nan
        w[rng.random(w.shape) < 0.1] = -np.inf
        w.view(np.int32)[rng.random(w.shape) < 0.02] = -1                # (a NaN with its sign bit set)
    elif what == "negative":
        w = -w
    elif what == "ends of the range":
        w = rng.choice(np.array([np.finfo(np.float32).max, np.finfo(np.float32).tiny, 1e-45, 0.0, 3e38], np.float32), w.shape)
    elif what == "steps of the last bit":
        w = (np.float32(1.0).view(np.int32) + rng.integers(0, 300, w.shape).astype(np.int32)).view(np.float32)
    elif what == "steps of the last bits":
        w = (np.float32(1.0).view(np.int32) + rng.integers(0, 1 << 14, w.shape).astype(np.int32)).view(np.float32)
    else:
        w = -np.arange(n, dtype=np.float32) * np.ones((2, 2, 1), np.float32)
        p[:] = np.arange(n)
    b = Batch(rp, [n, 300], 2, 64, 4, 16)
    evicted(rp, b, budget, 10, 40, w, p, n, True)
    # the same tokens behind many others, in long sequences, and in sequences whose keys do not fit on the chip
    for m in (12000, 34000):
        more, where = records(rng, 1, 2, m)
        more[0, :, -n:], where[0, :, -n:] = w[0], p[0]
        if what == "all equal":
            more[:] = 0.375
        evicted(rp, Batch(rp, [m], 2, 64, 4, 128), m - 300, 10, 40, more, where, m, False)


def test_positions_at_the_ends_of_their_type(rp):
    rng = np.random.default_rng(2)
    w, p = records(rng, 1, 2, 100)
    p[0, 0, :10], p[0, 1, :3] = -2 ** 31, 2 ** 31 - 1
    p[0, 0, 10:] = -2 ** 31 + rng.permutation(90) + 1
    evicted(rp, Batch(rp, [100], 2, 64, 4, 16), 50, 0, 50, w, p, 100, False)
    w, p = records(rng, 1, 2, 100)
    p[:] = 7                                                            # (more at one position than may be safe)
    evicted(rp, Batch(rp, [100], 2, 64, 4, 16), 50, 8, 1, w, p, 100, False)


@pytest.mark.parametrize("holes", [(0,), (1,), (3,), (7,)])
def test_sequences_with_pages_elsewhere_stay(rp, holes):
    b = Batch(rp, [0, 17, 100, 50, 128], 2, 64, 4, 16, holes=holes)
    w, p = records(np.random.default_rng(1), 5, 2, 128)
    evicted(rp, b, 20, 2, 5, w, p, 128, False)


def test_records_of_another_length_than_the_tables(rp):
    b = Batch(rp, [100, 300, 37], 2, 64, 4, 16)
    w, p = records(np.random.default_rng(1), 3, 2, 80)
    evicted(rp, b, 50, 0, 10, w, p, 80, True)                            # (tokens behind the records do not count)
    b = Batch(rp, [100, 300, 37], 2, 64, 4, 16)
    w, p = records(np.random.default_rng(1), 3, 2, 1000)
    b.dev_lens = dev([100, 2 ** 31 - 1, -5], np.int32)
    b.lens = [100, 304, 0]
    evicted(rp, b, 50, 0, 10, w, p, 1000, True)


def test_many_heads_of_many_sequences(rp):
    lens = [int(n) for n in np.random.default_rng(5).integers(0, 90, 600)]
    b = Batch(rp, lens, 4, 32, 4, 16)
    w, p = records(np.random.default_rng(3), 600, 4, 96)
    evicted(rp, b, 40, 2, 8, w, p, 96, True)


# ---- together ----------------------------------------------------------------------------------------------------
def test_attention_over_what_is_kept(rp):
    """Attention after an eviction is attention over the kept tokens: the plain form over each head's rows."""
    H, hd, bits, n_q, budget = 2, 64, 4, 6, 40
    b = Batch(rp, [200, 41, 90], H, hd, bits, 16)
    w, p = records(np.random.default_rng(8), 3, H, 200)
    k, v = [x.copy() for x in b.k], [x.copy() for x in b.v]
    lens, _ = evicted(rp, b, budget, 1, 5, w, p, 200, True)
    for s in range(3):
        kk, vv = np.zeros((budget, H * hd), int), np.zeros((budget, H * hd), int)
        for h in range(H):
            n = len(k[s])
            src = bounding.evict(w[s, h, :n], p[s, h, :n], budget, 1, 5)
            sl = slice(h * hd, (h + 1) * hd)
            kk[:, sl], vv[:, sl] = k[s][src][:, sl], v[s][src][:, sl]
        b.k[s], b.v[s] = kk, vv
    b.lens = [budget] * 3
    q = b.queries(n_q)
    out, lse = rp.attend_paged(b.cache, dev_bf16(q), b.page_table, lens, out=torch.empty(3, n_q * hd, device="cuda"), want_lse=True)
    b.check(q, n_q, hd ** -0.5, out, lse)


def serve(rp, caches, rot, x, steps, budget, H, hd, n_q, page, bits, recorded):
    """Decoding with a bounded cache: rotate and write, attend, add up the weights, evict; eagerly or recorded once and replayed."""
    cache, table, B = caches
    d, cap = H * hd, table.shape[1] * page
    qkv = torch.zeros(B, (n_q + 2 * H) * hd, dtype=torch.bfloat16, device="cuda")
    pos = torch.zeros(B, dtype=torch.int32, device="cuda")
    lens, grown = torch.zeros(B, dtype=torch.int32, device="cuda"), torch.zeros(B, dtype=torch.int32, device="cuda")
    slots = torch.full((B,), -1, dtype=torch.int64, device="cuda")
    track = rp.cache_track(cache, B, cap)
    att, ev = rp.attend_paged_workspace(cache, B, n_q), rp.evict_paged_workspace(cache, B, cap, budget)
    out, lse = torch.empty(B, n_q * hd, device="cuda"), torch.empty(B, n_q, device="cuda")
    q_out = torch.empty(B, n_q * hd, dtype=torch.bfloat16, device="cuda")

    def step():
        q, k, v = qkv[:, :n_q * hd], qkv[:, n_q * hd:n_q * hd + d], qkv[:, n_q * hd + d:]
        rp.rope_quant_paged(cache, rot, q, k, v, pos, slots, q_out=q_out)
        rp.attend_paged(cache, q_out, table, grown, out=out, lse=lse, workspace=att)
        rp.attend_weights_paged(cache, q_out, table, grown, lse, track, positions=pos)
        rp.evict_paged(cache, table, grown, track, budget, first=2, recent=6, lens_out=lens, workspace=ev)

    graph = None
    outs = []
    for i in range(steps):
        have = lens.cpu().numpy()
        grow = np.array([1] * (B - 1) + [i % 2])                         # (the last sequence only every other step)
        slots.copy_(dev(np.where(grow, table.cpu().numpy()[np.arange(B), have // page] * page + have % page, -1).astype(np.int64)))
        grown.copy_(dev((have + grow).astype(np.int32)))
        pos.copy_(dev(np.array([i] * (B - 1) + [i // 2], np.int32)))
        qkv.copy_(x[i])
        if recorded and i == 3:
            torch.cuda.synchronize()
            graph = torch.cuda.CUDAGraph()
            with torch.cuda.graph(graph):
                step()
        if graph is not None:
            graph.replay()
        else:
            step()
        torch.cuda.synchronize()
        outs.append([t.clone() for t in (out, lse, q_out, lens, track.weights, track.positions)])
    return outs, track


def test_a_serving_loop_with_a_bounded_cache(rp):
    """Rotate and write, attend, add up, evict, step after step: the recorded loop's bits are the eager one's, and every step is the
    plain form of itself."""
    H, hd, bits, n_q, page, B, budget, steps = 2, 64, 4, 4, 16, 3, 24, 60
    (hk, klo, khi), (hv, vlo, vhi), kt, vt = site(H, hd, bits)
    rng = np.random.default_rng(12)
    d = H * hd
    x = np.concatenate([rng.standard_normal((steps * B, n_q * hd)).astype(np.float32) * 0.02, paged.values(rng, klo, khi, steps * B),
                        paged.values(rng, vlo, vhi, steps * B)], axis=1)
    x = kvo.round_to_bf16(x)
    xd = dev_bf16(x).reshape(steps, B, -1)
    table = dev(rng.permutation(8)[:6].reshape(3, 2), np.int32)
    rot = rp.rotary(32, interleaved=True)
    freqs = rot.freqs.cpu().numpy()
    runs = []
    for recorded in (False, True):
        cache = rp.paged_cache(8, page, H, hd, bits, kt, vt)
        runs.append(serve(rp, (cache, table, B), rot, xd, steps, budget, H, hd, n_q, page, bits, recorded)[0])
    for a, b in zip(*runs):
        assert all(torch.equal(s, t) for s, t in zip(a, b))
    # the plain loop, with the weights that the kernels found (so that the same tokens leave)
    x = x.reshape(steps, B, -1)
    kept_k, kept_v = [[np.zeros((0, d), int) for _ in range(B)] for _ in range(2)]
    w = np.zeros((B, H, 2 * page))
    p = np.zeros((B, H, 2 * page), np.int64)
    for i in range(steps):
        out, lse, q_out, lens, tw, tp = (t.double().cpu().numpy() for t in runs[0][i])
        for b in range(B):
            pos = i if b < B - 1 else i // 2
            grows = b < B - 1 or i % 2
            row = x[i, b][None]
            q = kvo.round_to_bf16(bounding.rope32(row[:, :n_q * hd], [pos], hd, 32, True, freqs))
            assert np.array_equal(q[0], q_out[b])
            if grows:
                kc = kvo.kv_quant(bounding.rope32(row[:, n_q * hd:n_q * hd + d], [pos], hd, 32, True, freqs), hk, 0, bits)
                kept_k[b], kept_v[b] = np.concatenate([kept_k[b], kc]), np.concatenate([kept_v[b], kvo.kv_quant(row[:, n_q * hd + d:], hv, 0, bits)])
            n = len(kept_k[b])
            want, wl = kvo.attend(q[0], kept_k[b], kept_v[b], hk, 0, hv, 0, n_q, hd ** -0.5)
            tol, tl = paged.attend_bounds(q[0], kept_k[b], hk, hv, n_q, hd ** -0.5, bits, want, wl)
            assert (np.abs(out[b] - want) <= tol).all()
            if n == 0:
                continue
            assert (np.abs(lse[b] - wl) <= tl).all()
            got, near = bounding.weights64(q, lse[b][None], kept_k[b], np.arange(n), n, hk, n_q, hd ** -0.5, 1)
            w[b, :, n - 1] = 0.0                                          # (the newest token starts here, whether it was there the step before or not)
            w[b, :, :n] += got
            p[b, :, n - 1] = pos
            for h in range(H):
                # tokens leave by the kernel's weights: what it kept has to be the heaviest up to its own rounding
                src = np.arange(n) if n <= budget else bounding.evict(w[b, h, :n].astype(np.float32), p[b, h, :n], budget, 2, 6)
                kept = tp[b, h, :len(src)].astype(int)
                assert np.array_equal(p[b, h][src], kept), (i, b, h)
                sl = slice(h * hd, (h + 1) * hd)
                for rows in (kept_k, kept_v):
                    rows[b][:len(src), sl] = rows[b][src][:, sl]
                w[b, h, :len(src)], p[b, h, :len(src)] = w[b, h][src], p[b, h][src]
                assert np.allclose(tw[b, h, :len(src)], w[b, h, :len(src)], rtol=1e-4, atol=0)
                w[b, h, :len(src)] = tw[b, h, :len(src)]
            kept_k[b], kept_v[b] = kept_k[b][:len(src)], kept_v[b][:len(src)]
            assert lens[b] == len(src)


def test_other_streams(rp):
    """Two streams at once, each with records and a workspace of its own."""
    b = Batch(rp, [900, 40, 333], 2, 64, 4, 16)
    q, lse = window(rp, b, 4, 2)
    qd, ld = dev_bf16(q), dev(lse)
    w, p = records(np.random.default_rng(1), 3, 2, 900)
    pages = [b.cache.k_pages.clone(), b.cache.v_pages.clone()]
    caches = [rp.PagedCache(2, 64, 4, 16, pages[0].clone(), pages[1].clone(), b.cache.k_table, b.cache.v_table) for _ in range(3)]
    tracks = [rp.CacheTrack(dev(w), dev(p)) for _ in caches]
    work = [rp.evict_paged_workspace(c, 3, 900, 100) for c in caches]
    lens = [torch.zeros(3, dtype=torch.int32, device="cuda") for _ in caches]

    def go(i):
        rp.attend_weights_paged(caches[i], qd, b.page_table, b.dev_lens, ld, tracks[i], queries=2)
        rp.evict_paged(caches[i], b.page_table, b.dev_lens, tracks[i], 100, recent=10, lens_out=lens[i], workspace=work[i])

    go(0)
    torch.cuda.synchronize()
    streams = [torch.cuda.Stream() for _ in range(2)]
    for _ in range(5):
        for i, s in enumerate(streams, 1):
            with torch.cuda.stream(s):
                for dst, src in zip((caches[i].k_pages, caches[i].v_pages, tracks[i].weights, tracks[i].positions), pages + [dev(w), dev(p)]):
                    dst.copy_(src)
                go(i)
    torch.cuda.synchronize()
    for i in (1, 2):
        assert torch.equal(caches[i].k_pages, caches[0].k_pages) and torch.equal(caches[i].v_pages, caches[0].v_pages)
        assert torch.equal(tracks[i].weights, tracks[0].weights) and torch.equal(tracks[i].positions, tracks[0].positions) and torch.equal(lens[i], lens[0])


def test_refusals(rp):
    b = Batch(rp, [10, 20], 2, 64, 4, 16)
    c, q, lse = b.cache, torch.zeros(2, 128, dtype=torch.bfloat16, device="cuda"), torch.zeros(2, 2, device="cuda")
    t = rp.cache_track(c, 2, 32)
    add = lambda q=q, lse=lse, track=t, lens=b.dev_lens, table=b.page_table, **more: rp.attend_weights_paged(c, q, table, lens, lse, track, **more)     # noqa: E731
    cut = lambda track=t, budget=5, lens=b.dev_lens, table=b.page_table, **more: rp.evict_paged(c, table, lens, track, budget, **more)                # noqa: E731
    small = rp.CacheTrack(t.weights[:, :, :30], t.positions)
    one = rp.cache_track(c, 1, 32)
    for match, call in (
            ("dtype", lambda: add(q=q.float())), ("shape", lambda: add(q=q[:1])), ("lse", lambda: add(lse=lse[:, :1])), ("dtype", lambda: add(lse=lse.double())),
            ("capacity", lambda: add(track=small)), ("capacity", lambda: add(track=one)), ("lens", lambda: add(lens=b.dev_lens[:1])), ("dtype", lambda: add(table=b.page_table.long())),
            ("dtype", lambda: add(positions=b.dev_lens.long())), ("one per row", lambda: add(positions=b.dev_lens[:1])), ("shape", lambda: add(queries=2)),
            ("contiguous", lambda: add(track=rp.CacheTrack(torch.zeros(2, 2, 64, device="cuda")[:, :, ::2], t.positions))),
            ("dtype", lambda: add(track=rp.CacheTrack(t.weights.double(), t.positions))),
            ("capacity", lambda: cut(track=small)), ("shape", lambda: cut(out=rp.cache_track(c, 2, 40))), ("sequence", lambda: cut(lens_out=b.dev_lens[:1])),
            ("dtype", lambda: cut(lens_out=torch.zeros(2, dtype=torch.int64, device="cuda"))), ("device", lambda: cut(lens=b.dev_lens.cpu(), lens_out=b.dev_lens))):
        with pytest.raises(ValueError, match=match):
            call()
    for status, call in (
            (-2, lambda: add(fresh=-1)), (-6, lambda: add(scale=float("nan"))), (-2, lambda: cut(budget=0)), (-2, lambda: cut(first=3, recent=3)),
            (-2, lambda: cut(recent=-1)), (-2, lambda: cut(lens_out=b.dev_lens)), (-7, lambda: cut(track=rp.cache_track(c, 2, 9000), budget=4000, workspace=t.weights))):
        with pytest.raises(rp.RptqError, match="status %d" % status):
            call()
    assert not t.weights.any() and not t.positions.any()


def test_calls_of_nothing(rp):
    b = Batch(rp, [10, 20], 2, 64, 4, 16)
    c = b.cache
    none = torch.zeros(0, 128, dtype=torch.bfloat16, device="cuda")
    rp.attend_weights_paged(c, none, b.page_table[:0], b.dev_lens[:0], torch.zeros(0, 2, device="cuda"), rp.cache_track(c, 0, 32))
    assert rp.evict_paged(c, b.page_table[:0], b.dev_lens[:0], rp.cache_track(c, 0, 32), 5).shape == (0,)


@pytest.mark.parametrize("entry", ["rope", "rope_quant_paged", "attend_weights_paged", "evict_paged"])
def test_native_and_python_marshalling(rp, monkeypatch, entry):
    """Ordinary arguments are taken natively, with the results that the Python marshalling leads to; an argument out of the
    ordinary, whichever it is, is not (None, and nothing written)."""
    from paper_2304_01089_amd import binding
    b = Batch(rp, [100, 37], 2, 64, 4, 16)
    c, gen = b.cache, torch.Generator(device="cuda").manual_seed(1)
    wide = torch.randn(3, 704, generator=gen, device="cuda").bfloat16()
    k, v, q, slots = wide[:, :128], wide[:, 128:256], wide[:, 256:512], torch.tensor([3, 70, -1], device="cuda")
    pos, freqs = torch.tensor([3, 500, 7], dtype=torch.int32, device="cuda"), rp.rotary(32).freqs
    pages = c.k_pages.clone(), c.v_pages.clone()
    q_out, y = torch.zeros(3, 256, dtype=torch.bfloat16, device="cuda"), torch.zeros(3, 256, device="cuda")
    w, p = records(np.random.default_rng(1), 2, 2, 112)
    tw, tp, lse = dev(w), dev(p), torch.full((2, 4), 5.0, device="cuda")
    ow, op, lens_out = torch.zeros_like(tw), torch.zeros_like(tp), torch.zeros(2, dtype=torch.int32, device="cuda")
    ws = rp.evict_paged_workspace(c, 2, 112, 20)
    args, outs = {
        "rope": ((q, y, pos, 64, 32, True, freqs, 1.5, None), (y,)),
        "rope_quant_paged": ((q, q_out, k, v, pos, slots, 64, 32, False, freqs, 1.5, c.k_table, c.v_table, 4) + pages + (16, None), (q_out,) + pages),
        "attend_weights_paged": ((q[:2], 1, 4, 2, 64, 0.125, c.k_table, 4, c.k_pages, 16, b.page_table, b.dev_lens, lse, b.dev_lens.clone(), 1, tw, tp, None, None), (tw, tp)),
        "evict_paged": ((2, 64, 4) + pages + (16, b.page_table, b.dev_lens, dev(w), dev(p), 20, 2, 5, ow, op, lens_out, ws, None), pages + (ow, op, lens_out)),
    }[entry]
    native, plain = getattr(binding._CALLS, entry), getattr(rp, "rptq_" + entry)
    start = [t.clone() for t in outs]
    assert native(*args) == 0
    got = [t.clone() for t in outs]
    assert all(not torch.equal(a, s) for a, s in zip(got, start))
    for t, s in zip(outs, start):
        t.copy_(s)
    with monkeypatch.context() as m:
        m.setattr(binding, "_CALLS", None)
        m.setattr(binding, "_CALLS_SOUGHT", True)
        plain(*args)
    assert all(torch.equal(a, t) for a, t in zip(got, outs))
    for t in outs:
        t.view(torch.uint8).fill_(0x3c)
    torch.cuda.synchronize()
    for i, a in enumerate(args):
        if isinstance(a, torch.Tensor):
            odd = [a.cpu(), 1]
            if a is not ws and a is not c.k_table and a is not c.v_table:
                odd.append(a.to(torch.float64 if a.dtype != torch.float64 else torch.int8))
                odd.append(a.reshape(-1)[:1] if a.dtype != torch.uint8 else a.reshape(-1)[:100])
            if not (entry == "attend_weights_paged" and i == 13):
                odd.append(None)
        elif a is None:
            odd = [torch.cuda.current_stream()] if i == len(args) - 1 else [1, c.k_pages.cpu()]
        elif isinstance(a, bool):
            odd = [1, 0, None]
        elif isinstance(a, float):
            odd = [1, np.float32(0.1)]
        else:
            odd = [float(a), np.int64(a), 1 << 80]
        for o in odd:
            assert native(*args[:i], o, *args[i + 1:]) is None, (i, o)
    assert native(*args[:-1]) is None and native(*args, None) is None
    torch.cuda.synchronize()
    assert all((t.view(torch.uint8) == 0x3c).all() for t in outs)
