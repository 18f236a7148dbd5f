"""Attention weights of windows of many queries, up to whole prompts: the error of a sum does not grow with the number of queries."""
import numpy as np
import pytest

from oracle import kv_cache as kvo

import bounding
from test_gpu_paged import Batch, dev, dev_bf16

pytestmark = pytest.mark.gpu
torch = pytest.importorskip("torch")

# Half steps of fp32 that a sum may be off by, relative to itself: a pass adds up to 16 row tiles and joins four rows, 18 in all; passes are added
# up exactly but for errors of errors (passes^2 2^-48: 0.3 of a half step for 2048 passes); one more as the sum is rounded at last.
SUM = 19.3


@pytest.fixture(scope="module")
def rp():
    import paper_2304_01089_amd as rp_
    rp_.load_library()
    assert torch.cuda.is_available()
    return rp_


def queries_for(batch, n):
    """bf16 [n, H hd] whose scores have a standard deviation of about two, float32 values."""
    s, _, _ = kvo.position_tables(batch.hk, 0)
    H, hd = batch.H, batch.hd
    t = 2.0 * np.sqrt(hd) / (np.sqrt((s.reshape(H, hd) ** 2).sum(1)) * 2.0 ** batch.bits / 3.5)
    return torch.randn(n, H, hd, generator=torch.Generator(device="cuda").manual_seed(n), device="cuda").mul_(dev(t, np.float32)[:, None]).bfloat16().reshape(n, H * hd)


@pytest.mark.parametrize("H,hd", [(4, 32), (2, 64), (1, 128), (1, 256)])
def test_whole_prompts_of_queries_alike(rp, H, hd):
    """Queries of zeros: every weight of a query head is exp(-lse), which is where rounded sums drift.  2^x twice, each within a step, is four
    half steps more."""
    n, share = 16384, 8
    b = Batch(rp, [n], H, hd, 4, 64)
    lse = (3.5 + 0.37 * np.arange(H * share)).astype(np.float32)
    track = rp.cache_track(b.cache, 1, n)
    q = torch.zeros(n, H * share * hd, dtype=torch.bfloat16, device="cuda")
    rp.attend_weights_paged(b.cache, q, b.page_table, b.dev_lens, dev(np.tile(lse, (n, 1))), track, queries=n, fresh=n)
    got = track.weights[0].double().cpu().numpy()
    want = np.exp(-lse.astype(np.float64)).reshape(H, share).sum(1)[:, None] * (n - np.arange(n))
    off = np.abs(got - want) / want
    assert off.max() <= (SUM + 4) * bounding.U, off.max() / bounding.U
    assert torch.equal(track.positions[0, 0], torch.arange(n, dtype=torch.int32, device="cuda"))


def check(batch, b, q, lse, n, queries, got, w0):
    """Sequence number b's weights against 64 bits; every sequence has the first one's tokens."""
    sums, tol = bounding.weights64(q, lse, batch.k[0], np.arange(n), n, batch.hk, q.shape[1] // batch.hd, batch.hd ** -0.5, queries)
    share = q.shape[1] // batch.hd // batch.H
    tol -= (share * queries / 4 + 6) * bounding.U * sums               # (what a sum in one row would be off by)
    near = tol + (SUM + 1) * bounding.U * (sums + w0)
    assert (np.abs(got - (w0 + sums)) <= near).all(), (b, (np.abs(got - (w0 + sums)) / near).max())


@pytest.mark.parametrize("H,hd,n,queries,bits", [(4, 32, 1300, 1540, 4), (2, 64, 1500, 1600, 8), (1, 128, 2900, 1540, 3), (1, 256, 2900, 772, 4)])
def test_many_tokens_of_a_workgroup(rp, H, hd, n, queries, bits):
    """As many sequences as leave one workgroup to each, all over the same pages: more tiles of tokens than sums are kept of."""
    B = 2048
    if torch.cuda.mem_get_info()[0] < 24 << 30:
        pytest.skip("not enough free memory")
    b = Batch(rp, [n], H, hd, bits, 16)
    q = queries_for(b, B * queries)
    gen = torch.Generator(device="cuda").manual_seed(1)
    lse = 5.0 + 0.3 * torch.randn(B * queries, H, generator=gen, device="cuda")
    w0 = torch.rand(B, H, n, generator=gen, device="cuda")
    track = rp.CacheTrack(w0.clone(), torch.full((B, H, n), 7, dtype=torch.int32, device="cuda"))
    lens, table = b.dev_lens.repeat(B), b.page_table.repeat(B, 1)
    rp.attend_weights_paged(b.cache, q, table, lens, lse, track, queries=queries, fresh=0)
    for i in (0, 777, B - 1):
        rows = slice(i * queries, (i + 1) * queries)
        check(b, i, q[rows].float().cpu().numpy(), lse[rows].cpu().numpy(), n, queries, track.weights[i].double().cpu().numpy(), w0[i].double().cpu().numpy())
    assert (track.positions == 7).all()


@pytest.mark.parametrize("queries", [511, 512, 513, 700])
def test_around_as_many_queries_as_sums_are_kept_of(rp, queries):
    """Up to 24 passes are rounded, half a step each; the lengths around the window's."""
    H, hd, share = 2, 64, 3
    lens = [queries + 40, queries, queries - 7, 1, 0]
    b = Batch(rp, lens, H, hd, 4, 16)
    rng = np.random.default_rng(queries)
    q = queries_for(b, len(lens) * queries * share).reshape(len(lens) * queries, -1)
    lse = (5.0 + 0.3 * rng.standard_normal((len(lens) * queries, H * share))).astype(np.float32)
    w0 = rng.random((len(lens), H, queries + 50)).astype(np.float32)
    track = rp.CacheTrack(dev(w0), dev(np.zeros(w0.shape, np.int32)))
    rp.attend_weights_paged(b.cache, q, b.page_table, b.dev_lens, dev(lse), track, queries=queries, fresh=9)
    got, qn = track.weights.double().cpu().numpy(), q.float().cpu().numpy()
    for i, n in enumerate(lens):
        old = w0[i].astype(np.float64)
        old[:, max(0, n - 9):n] = 0.0
        rows = slice(i * queries, (i + 1) * queries)
        sums, tol = bounding.weights64(qn[rows], lse[rows], b.k[i], np.arange(n), n, b.hk, H * share, hd ** -0.5, queries)
        tol += (SUM + 1 + 24 - (share * queries / 4 + 6)) * bounding.U * sums
        assert (np.abs(got[i, :, :n] - old[:, :n] - sums) <= tol + 25 * bounding.U * old[:, :n]).all(), n
        assert np.array_equal(got[i, :, n:], old[:, n:])


def test_sums_that_are_not_finite(rp):
    """What is kept of a sum is nothing where it is infinite or NaN; others keep theirs."""
    H, hd, n, queries = 2, 64, 1600, 1540
    b = Batch(rp, [n], H, hd, 4, 16)
    lse = torch.full((queries, H), 5.0, device="cuda")
    q = queries_for(b, queries)
    clean = rp.cache_track(b.cache, 1, n)
    rp.attend_weights_paged(b.cache, q, b.page_table, b.dev_lens, lse, clean, queries=queries, fresh=0)
    track = rp.cache_track(b.cache, 1, n)
    track.weights[0, 0, 3], track.weights[0, 0, 4], track.weights[0, 1, 5] = float("inf"), float("nan"), float("-inf")
    rp.attend_weights_paged(b.cache, q, b.page_table, b.dev_lens, lse, track, queries=queries, fresh=0)
    assert track.weights[0, 0, 3] == float("inf") and torch.isnan(track.weights[0, 0, 4]) and track.weights[0, 1, 5] == float("-inf")
    same = torch.ones(H, n, dtype=torch.bool, device="cuda")
    same[0, 3:5], same[1, 5] = False, False
    assert torch.equal(track.weights[0][same], clean.weights[0][same])


def test_the_attention_of_a_window_leaves_its_sums(rp):
    """lse from attend_paged: a row per query of the window, over the tokens that it sees.  What a sequence's tokens get of a query head adds up
    to the number of queries that see any."""
    H, share, hd, n = 2, 3, 64, 7
    lens = [1000, 64, 1, 333, 0, 7]
    b = Batch(rp, lens, H, hd, 4, 16)
    q = queries_for(b, len(lens) * n * share).reshape(len(lens) * n, -1)
    back = torch.arange(n - 1, -1, -1, dtype=torch.int32, device="cuda")
    seen = (b.dev_lens[:, None] - back).reshape(-1).contiguous()
    _, lse = rp.attend_paged(b.cache, q, b.page_table.repeat_interleave(n, 0), seen, want_lse=True)
    track = rp.cache_track(b.cache, len(lens), 1000)
    rp.attend_weights_paged(b.cache, q, b.page_table, b.dev_lens, lse, track, queries=n, fresh=1000)
    got, ls, qn = track.weights.double().cpu().numpy(), lse.cpu().numpy(), q.float().cpu().numpy()
    for i, length in enumerate(lens):
        rows = slice(i * n, (i + 1) * n)
        sums, tol = bounding.weights64(qn[rows], ls[rows], b.k[i], np.arange(length), length, b.hk, H * share, hd ** -0.5, n)
        assert (np.abs(got[i, :, :length] - sums) <= tol).all()
        # (every weight's error bound, and the logarithm's own, as where one query's weights add up)
        assert np.abs(got[i].sum(-1) - share * min(n, length)).max() < 2e-4 * n
        assert (got[i, :, length:] == 0).all()
