"""Pools of many GiB: pages on both sides of 2, 4, 6 and 8 GiB hold the same tokens with the same results as those of a small pool."""
import numpy as np
import pytest

from test_gpu_bounding import records, window
from test_gpu_paged import Batch, dev, dev_bf16

pytestmark = pytest.mark.gpu
torch = pytest.importorskip("torch")
H, HD, PAGE = 8, 128, 256


@pytest.fixture(scope="module")
def rp():
    import paper_2304_01089_amd as rp_
    rp_.load_library()
    assert torch.cuda.is_available()
    return rp_


def far(rp, bits):
    """(a batch in a small pool, the same in one of 8.3 GiB a tensor, that one's page table, its pages' numbers and the small one's)."""
    if torch.cuda.mem_get_info()[0] < 40 << 30:
        pytest.skip("not enough free memory")
    b = Batch(rp, [900, 256, 1500, 3], H, HD, bits, PAGE)
    size = rp.rptq_kv_page_bytes(H * HD, PAGE, bits)
    used = sorted({int(i) for s, n in enumerate(b.lens) for i in b.table[s][:(n + PAGE - 1) // PAGE]})
    gib = [1.0, 1.999, 2.0, 2.5, 3.0, 3.5, 3.999, 4.0, 5.0, 6.0, 7.0, 8.2]
    ids = [int(g * 2 ** 30) // size for g in gib]
    assert len(set(ids)) == len(used) == len(ids)
    n_pages = int(8.3 * 2 ** 30) // size
    pages = [torch.zeros((n_pages,) + tuple(t.shape[1:]), dtype=torch.uint8, device="cuda") for t in (b.cache.k_pages, b.cache.v_pages)]
    for big, small in zip(pages, (b.cache.k_pages, b.cache.v_pages)):
        for i, j in zip(ids, used):
            big[i] = small[j]
    cache = rp.PagedCache(H, HD, bits, PAGE, *pages, b.cache.k_table, b.cache.v_table)
    moved = dict(zip(used, ids))
    table = np.array([[moved.get(int(i), -1) for i in row] for row in b.table])
    return b, cache, dev(table, np.int32), ids, used


@pytest.mark.parametrize("bits", [3, 4, 8])
def test_attention(rp, bits):
    b, cache, table, _, _ = far(rp, bits)
    q = b.queries(2 * H)
    got, lse = rp.attend_paged(cache, dev_bf16(q), table, b.dev_lens, out=torch.empty(4, 2 * H * HD, device="cuda"), want_lse=True)
    b.check(q, 2 * H, HD ** -0.5, got, lse)


@pytest.mark.parametrize("queries", [1, 9])
@pytest.mark.parametrize("bits", [3, 4, 8])
def test_accumulated_weights(rp, bits, queries):
    b, cache, table, _, _ = far(rp, bits)
    q, lse = window(rp, b, 2 * H, queries)
    tracks = [rp.cache_track(cache, 4, 1500) for _ in range(2)]
    for c, t, track in ((b.cache, b.page_table, tracks[0]), (cache, table, tracks[1])):
        rp.attend_weights_paged(c, dev_bf16(q), t, b.dev_lens, dev(lse), track, queries=queries, fresh=10)
    assert torch.equal(tracks[0].weights, tracks[1].weights) and torch.equal(tracks[0].positions, tracks[1].positions)
    assert tracks[0].weights[2].gt(0).any()


@pytest.mark.parametrize("budget", [255, 400])
@pytest.mark.parametrize("bits", [3, 4, 8])
def test_eviction(rp, bits, budget):
    b, cache, table, ids, used = far(rp, bits)
    w, p = records(np.random.default_rng(budget), 4, H, 1500)
    tracks = [rp.CacheTrack(dev(w), dev(p)) for _ in range(2)]
    lens = [rp.evict_paged(c, t, b.dev_lens, track, budget, first=1, recent=20) for c, t, track in ((b.cache, b.page_table, tracks[0]), (cache, table, tracks[1]))]
    assert torch.equal(lens[0], lens[1]) and torch.equal(tracks[0].weights, tracks[1].weights) and torch.equal(tracks[0].positions, tracks[1].positions)
    for big, small in ((cache.k_pages, b.cache.k_pages), (cache.v_pages, b.cache.v_pages)):
        assert torch.equal(big[ids], small[used])
        big[ids] = 0
        assert not big.any()


@pytest.mark.parametrize("bits", [3, 8])
def test_rotated_writes(rp, bits):
    b, cache, _, ids, used = far(rp, bits)
    n = len(ids) * 3
    rng = np.random.default_rng(7)
    k, v = (dev_bf16(rng.standard_normal((n, H * HD)).astype(np.float32)) for _ in range(2))
    pos = torch.arange(n, dtype=torch.int32, device="cuda")
    off = np.tile([0, 17, PAGE - 1], len(ids))
    rot = rp.rotary(HD)
    for c, numbers in ((b.cache, used), (cache, ids)):
        rp.rope_quant_paged(c, rot, None, k, v, pos, dev((np.repeat(numbers, 3) * PAGE + off).astype(np.int64)))
    for big, small in ((cache.k_pages, b.cache.k_pages), (cache.v_pages, b.cache.v_pages)):
        assert torch.equal(big[ids], small[used])
        big[ids] = 0
        assert not big.any()
