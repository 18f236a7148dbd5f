"""Calls of the cache-bounding operators that their documentation allows and a program may come to: recorded graphs that share their
workspaces, a process's first call, recorded, records half in place, rows and tables inside larger tensors, one token, token numbers at the
limit."""
import os
import subprocess
import sys

import numpy as np
import pytest

import bounding
from test_gpu_bounding import evicted, records, window
from test_gpu_paged import Batch, dev, dev_bf16

pytestmark = pytest.mark.gpu
torch = pytest.importorskip("torch")
TOP = 1 << 29
ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))

PROGRAM = r"""
import sys
sys.path.insert(0, "tests")
import numpy as np, torch
import paper_2304_01089_amd as rp
from test_gpu_bounding import records
from test_gpu_paged import Batch, dev, dev_bf16
n, budget, queries = (int(a) for a in sys.argv[1:])
b = Batch(rp, [n, 30], 2, 64, 4, 16)
w, p = records(np.random.default_rng(0), 2, 2, n)
q = dev_bf16(b.queries(4)).repeat_interleave(queries, 0)
lse = torch.full((2 * queries, 4), 3.0, device="cuda")
start = [b.cache.k_pages.clone(), b.cache.v_pages.clone(), dev(w), dev(p)]
track, lens = rp.CacheTrack(dev(w), dev(p)), torch.zeros(2, dtype=torch.int32, device="cuda")
work = rp.attend_weights_paged_workspace(b.cache, 2, 4, queries), rp.evict_paged_workspace(b.cache, 2, n, budget)

def go():
    rp.attend_weights_paged(b.cache, q, b.page_table, b.dev_lens, lse, track, queries=queries, workspace=work[0])
    rp.evict_paged(b.cache, b.page_table, b.dev_lens, track, budget, recent=9, lens_out=lens, workspace=work[1])

state = [b.cache.k_pages, b.cache.v_pages, track.weights, track.positions]
def restore():
    for t, s in zip(state, start):
        t.copy_(s)

torch.cuda.synchronize()
graph = torch.cuda.CUDAGraph()
with torch.cuda.graph(graph):
    go()
outs = []
for _ in range(3):
    restore()
    graph.replay()
    torch.cuda.synchronize()
    outs.append([t.clone() for t in state + [lens]])
restore()
go()
torch.cuda.synchronize()
for o in outs:
    assert all(torch.equal(x.view(torch.uint8), y.view(torch.uint8)) for x, y in zip(o, state + [lens]))
print("ok")
"""


@pytest.fixture(scope="module")
def rp():
    import paper_2304_01089_amd as rp_
    rp_.load_library()
    assert torch.cuda.is_available()
    return rp_


def test_graphs_that_share_their_workspaces(rp):
    """A window of many queries and a long cut, both of which need their workspaces, of two batches: recorded apart, replayed in turn."""
    queries, budget, cap = 40, 2500, 5200
    work, sides = None, []
    for seed in (0, 1):
        b = Batch(rp, [5100, 3000, 60], 1, 128, 4, 64, seed=seed)
        q, lse = window(rp, b, 4, queries)
        w, p = records(np.random.default_rng(seed), 3, 1, cap)
        start = [b.cache.k_pages.clone(), b.cache.v_pages.clone(), dev(w), dev(p)]
        track = rp.CacheTrack(start[2].clone(), start[3].clone())
        if work is None:
            work = (rp.attend_weights_paged_workspace(b.cache, 3, 4, queries), rp.evict_paged_workspace(b.cache, 3, cap, budget))
            assert work[0] is not None
        sides.append((b, dev_bf16(q), dev(lse), track, torch.zeros(3, dtype=torch.int32, device="cuda"), start))

    def go(side):
        b, q, lse, track, lens, _ = side
        rp.attend_weights_paged(b.cache, q, b.page_table, b.dev_lens, lse, track, queries=queries, fresh=queries, workspace=work[0])
        rp.evict_paged(b.cache, b.page_table, b.dev_lens, track, budget, first=4, recent=64, lens_out=lens, workspace=work[1])

    def state(side):
        b, _, _, track, lens, _ = side
        return [b.cache.k_pages, b.cache.v_pages, track.weights, track.positions, lens]

    def restore(side):
        for t, s in zip(state(side), side[5]):
            t.copy_(s)
        side[4].zero_()

    want, graphs = [], []
    for side in sides:
        go(side)
        torch.cuda.synchronize()
        want.append([t.clone() for t in state(side)])
        assert side[4].tolist() == [budget, budget, 60]
    for side in sides:
        restore(side)
        torch.cuda.synchronize()
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph):
            go(side)
        graphs.append(graph)
    for turn in range(3):
        for side in sides:
            restore(side)
        for work_bytes in work:
            work_bytes.fill_(0xFF if turn else 0)
        graphs[turn % 2].replay()
        graphs[1 - turn % 2].replay()
        torch.cuda.synchronize()
        for side, w in zip(sides, want):
            assert all(torch.equal(a, b) for a, b in zip(state(side), w)), turn


@pytest.mark.parametrize("n,budget,queries", [(300, 100, 1), (6000, 5999, 3), (9000, 4200, 12), (33000, 700, 1)])
def test_recording_the_first_calls_of_a_process(n, budget, queries):
    r = subprocess.run([sys.executable, "-u", "-c", PROGRAM, str(n), str(budget), str(queries)], cwd=ROOT, capture_output=True, text=True, timeout=100)
    assert r.returncode == 0 and r.stdout.strip().endswith("ok"), r.stdout + r.stderr


@pytest.mark.parametrize("n,budget", [(300, 100), (9000, 4200)])
@pytest.mark.parametrize("weights_apart", [False, True])
def test_records_half_in_place(rp, n, budget, weights_apart):
    b = Batch(rp, [n, 50], 2, 64, 4, 16)
    w, p = records(np.random.default_rng(2), 2, 2, n)
    track = rp.CacheTrack(dev(w), dev(p))
    out = rp.CacheTrack(torch.zeros_like(track.weights) if weights_apart else track.weights, track.positions if weights_apart else torch.zeros_like(track.positions))
    lens = rp.evict_paged(b.cache, b.page_table, b.dev_lens, track, budget, recent=7, out=out)
    assert lens.tolist() == [budget, 50]
    for s, left in enumerate(lens.tolist()):
        for h in range(2):
            src = bounding.evict(w[s, h, :[n, 50][s]], p[s, h, :[n, 50][s]], budget, 0, 7)
            assert np.array_equal(out.weights[s, h, :left].cpu().numpy(), w[s, h][src]) and np.array_equal(out.positions[s, h, :left].cpu().numpy(), p[s, h][src])


@pytest.mark.parametrize("queries", [1, 6, 20])
def test_rows_and_tables_inside_larger_tensors(rp, queries):
    b = Batch(rp, [100, 333, 2], 2, 64, 4, 16)
    q, lse = window(rp, b, 6, queries)
    wide = torch.full((3 * queries, 6 * 64 + 24), float("nan"), dtype=torch.bfloat16, device="cuda")
    wide[:, 8:8 + 6 * 64] = dev_bf16(q)
    table = torch.full((3, b.page_table.shape[1] + 5), -1, dtype=torch.int32, device="cuda")
    table[:, 3:3 + b.page_table.shape[1]] = b.page_table
    views = wide[:, 8:8 + 6 * 64], table[:, 3:3 + b.page_table.shape[1]]
    tracks = [rp.cache_track(b.cache, 3, 340) for _ in range(2)]
    rp.attend_weights_paged(b.cache, dev_bf16(q), b.page_table, b.dev_lens, dev(lse), tracks[0], queries=queries, fresh=400)
    rp.attend_weights_paged(b.cache, views[0], views[1], b.dev_lens, dev(lse), tracks[1], queries=queries, fresh=400)
    assert torch.equal(tracks[0].weights, tracks[1].weights) and torch.equal(tracks[0].positions, tracks[1].positions)
    assert tracks[0].weights[1, :, :330].gt(0).any()
    other = rp.PagedCache(2, 64, 4, 16, b.cache.k_pages.clone(), b.cache.v_pages.clone(), b.cache.k_table, b.cache.v_table)
    a = rp.evict_paged(b.cache, b.page_table, b.dev_lens, tracks[0], 40)
    z = rp.evict_paged(other, views[1], b.dev_lens, tracks[1], 40)
    assert torch.equal(a, z) and torch.equal(b.cache.k_pages, other.k_pages) and torch.equal(b.cache.v_pages, other.v_pages)
    assert torch.equal(tracks[0].weights, tracks[1].weights) and torch.equal(tracks[0].positions, tracks[1].positions)


def test_one_token(rp):
    b = Batch(rp, [1, 1], 2, 64, 4, 16)
    q, lse = window(rp, b, 2, 1)
    track = rp.cache_track(b.cache, 2, 1)
    rp.attend_weights_paged(b.cache, dev_bf16(q), b.page_table, b.dev_lens, dev(lse), track, positions=dev([70, 5], np.int32))
    # (one token has the whole of the attention; its score and the logarithm are off by eight half steps of their terms' sum, below 200 here)
    assert (track.weights - 1).abs().max() < 1e-4 and track.positions.flatten().tolist() == [70, 70, 5, 5]
    assert rp.evict_paged(b.cache, b.page_table, b.dev_lens, track, 1, recent=1).tolist() == [1, 1]


def long_cache(rp, seed=0):
    """Two pages of 4096 tokens, in turn, as a sequence of 2^29 (to read, or to move a row in)."""
    if torch.cuda.mem_get_info()[0] < 24 << 30:
        pytest.skip("not enough free memory")
    b = Batch(rp, [8192], 1, 128, 4, 4096, seed=seed, extra_pages=0)
    return b, b.page_table.repeat(1, TOP // 8192).contiguous(), dev([TOP], np.int32)


@pytest.mark.parametrize("queries", [1, 21])
def test_weights_of_as_many_tokens_as_there_may_be(rp, queries):
    b, table, lens = long_cache(rp)
    q, lse = window(rp, b, 1, queries)
    short, long = rp.cache_track(b.cache, 1, 8192), rp.cache_track(b.cache, 1, TOP)
    rp.attend_weights_paged(b.cache, dev_bf16(q), b.page_table, b.dev_lens, dev(lse), short, queries=queries, fresh=0)
    rp.attend_weights_paged(b.cache, dev_bf16(q), table, lens, dev(lse), long, queries=queries, fresh=5)
    torch.cuda.synchronize()
    w = long.weights.view(-1, 8192)
    assert torch.equal(w[-1], short.weights.view(-1))
    whole = w[0].clone()                                               # (the last tokens are seen by every query here)
    assert torch.equal(whole[:8192 - queries + 1], short.weights.view(-1)[:8192 - queries + 1])
    assert (w[:-1] == whole).all()
    assert long.positions[0, 0, -6:].tolist() == [0] + list(range(TOP - 5, TOP)) and not long.positions[0, 0, :-5].any()


def test_eviction_from_as_many_tokens_as_there_may_be(rp):
    b, table, lens = long_cache(rp)
    hole = TOP - (1 << 20) + 77
    w = torch.rand(1, 1, TOP, generator=torch.Generator(device="cuda").manual_seed(1), device="cuda")
    w[0, 0, hole] = -1.0
    track = rp.CacheTrack(w, torch.arange(TOP, dtype=torch.int32, device="cuda").view(1, 1, TOP))
    want = [w.clone().view(-1), track.positions.clone().view(-1)]
    for t in want:
        t[hole] = t[-1]
    before = [b.cache.k_pages.clone(), b.cache.v_pages.clone()]
    got = rp.evict_paged(b.cache, table, lens, track, TOP - 1, first=1, recent=1)
    torch.cuda.synchronize()
    assert got.tolist() == [TOP - 1]
    assert torch.equal(track.weights.view(-1), want[0]) and torch.equal(track.positions.view(-1), want[1])
    ids = b.page_table[0].tolist()
    for now, was in zip((b.cache.k_pages, b.cache.v_pages), before):
        was[ids[hole // 4096 % 2], :, hole % 4096] = was[ids[1], :, 4095].clone()
        assert torch.equal(now, was)


@pytest.mark.parametrize("what", ["random", "ties", "all equal", "the last one", "nan and infinities", "all safe", "none safe"])
@pytest.mark.parametrize("n", [2, 65, 700, 4097, 8193, 20000, 32769])
def test_one_token_leaves(rp, n, what):
    """A batch at its budget and a token more, for every way of holding the keys: the smallest weight's leaves, of equal ones the last."""
    b = Batch(rp, [n, n - 1, n], 2, 64, 3, 64)
    rng = np.random.default_rng(n)
    w, p = records(rng, 3, 2, n + 3, ties=what == "ties")
    first, recent = (0, n // 2) if n > 2 else (0, 1)
    if what == "all equal":
        w[:] = 0.25
    elif what == "the last one":
        w[:, :, n - 1] = -1.0
        first = recent = 0
    elif what == "nan and infinities":
        w[:] = rng.choice(np.array([np.nan, np.inf, -np.inf, 0.0, -0.0], np.float32), w.shape)
    elif what == "all safe":
        p[:] = np.arange(n + 3)
        first, recent = 0, n - 1
        p[:, 1, 0] = n                                                  # (the second head: the one that is not safe is another)
    elif what == "none safe":
        first = recent = 0
    evicted(rp, b, n - 1, first, recent, w, p, n + 3, what in ("random", "all equal"))
