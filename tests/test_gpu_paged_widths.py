"""Keys, values and heads of another width than the cache's tables: refused, whichever way a call is marshalled, with everything
left as it was.  (The narrower ones divide the pool into a whole number of pages, so that the sizes alone would fit.)"""
import numpy as np
import pytest

import paged

pytestmark = pytest.mark.gpu
torch = pytest.importorskip("torch")

H, HD, BITS, PAGE = 4, 64, 4, 16


@pytest.fixture(scope="module")
def rp():
    import paper_2304_01089_amd as rp_
    rp_.load_library()
    assert torch.cuda.is_available()
    return rp_


@pytest.fixture
def cache(rp):
    tables = [torch.from_numpy(paged.table_rows(paged.clusters(H, HD, BITS, 3, seed)[0])).cuda() for seed in (1, 2)]
    c = rp.paged_cache(6, PAGE, H, HD, BITS, *tables)
    c.k_pages.fill_(0x5A), c.v_pages.fill_(0xA5)
    return c


def untouched(c):
    torch.cuda.synchronize()
    return bool((c.k_pages == 0x5A).all()) and bool((c.v_pages == 0xA5).all())


def both_ways(monkeypatch, call):
    from paper_2304_01089_amd import binding
    call()
    with monkeypatch.context() as m:
        m.setattr(binding, "_CALLS", None)
        m.setattr(binding, "_CALLS_SOUGHT", True)
        call()


@pytest.mark.parametrize("width", [128, 512])
def test_rows_of_another_width(rp, cache, monkeypatch, width):
    slots = torch.tensor([0, 17, 40], device="cuda")
    wide = torch.full((3, width + 256), 7.0, dtype=torch.bfloat16, device="cuda")
    k, v = wide[:, :width], torch.full((3, width), 7.0, dtype=torch.bfloat16, device="cuda")

    def refused():
        with pytest.raises(ValueError, match="k_table"):
            rp.kv_quant_paged(cache, k, v, slots)
        with pytest.raises(ValueError, match="k_table"):
            rp.kv_dequant_paged(cache, slots, k=k, v=v)
        flat = cache.k_pages.view(-1), cache.v_pages.view(-1)
        with pytest.raises(ValueError, match="k_table"):
            rp.rptq_kv_quant_paged(k, v, slots, cache.k_table, cache.v_table, BITS, *flat, PAGE)
        with pytest.raises(ValueError, match="k_table"):
            rp.rptq_kv_dequant_paged(*flat, PAGE, BITS, slots, cache.k_table, cache.v_table, k, v)
        with pytest.raises(ValueError, match="v_table"):
            rp.rptq_kv_quant_paged(k, v, slots, cache.k_table.repeat(2, 1)[:width].contiguous(), cache.v_table, BITS, *flat, PAGE)

    both_ways(monkeypatch, refused)
    assert untouched(cache) and (wide == 7.0).all() and (v == 7.0).all()


def test_heads_of_another_width(rp, cache, monkeypatch):
    q = torch.ones(2, 8 * HD, dtype=torch.bfloat16, device="cuda")
    out = torch.full((2, 8 * HD), 5.0, device="cuda")
    table, lens = torch.zeros(2, 1, dtype=torch.int32, device="cuda"), torch.ones(2, dtype=torch.int32, device="cuda")
    ws = rp.attend_paged_workspace(cache, 2, 16)

    def refused():
        for heads in (2, 8):
            with pytest.raises(ValueError, match="k_table"):
                rp.rptq_attend_paged(q, 8, heads, HD, 1.0, cache.k_table, cache.v_table, BITS, cache.k_pages.view(-1),
                                     cache.v_pages.view(-1), PAGE, table, lens, out, None, ws)

    both_ways(monkeypatch, refused)
    assert untouched(cache) and (out == 5.0).all()


def test_the_cache_s_own_width_is_taken(rp, cache, monkeypatch):
    slots = torch.tensor([0, 17, 40], device="cuda")
    x = torch.randn(3, 256, generator=torch.Generator(device="cuda").manual_seed(3), device="cuda").bfloat16()
    seen = []

    def taken():
        rp.kv_quant_paged(cache, x, x, slots)
        seen.append(torch.stack(rp.kv_dequant_paged(cache, slots)))

    both_ways(monkeypatch, taken)
    assert torch.equal(seen[0], seen[1]) and not untouched(cache)
