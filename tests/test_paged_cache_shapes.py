"""A paged cache's pages have to be the pages that its sizes name, whichever call takes them: refused on the host alone, before
any tensor is looked up on a device."""
import pytest

import paper_2304_01089_amd as rp

torch = pytest.importorskip("torch")

H, HD, BITS, PAGE = 4, 64, 4, 16          # 256 channels: [pages, 2, 16, 64]


def pages(*shape):
    return torch.zeros(*shape, dtype=torch.uint8)


def cache(**change):
    sizes = dict(n_heads=H, head_dim=HD, bits=BITS, page_size=PAGE, k_pages=pages(6, 2, 16, 64), v_pages=pages(6, 2, 16, 64),
                 k_table=torch.zeros(256, 4, dtype=torch.int32), v_table=torch.zeros(256, 4, dtype=torch.int32))
    return rp.PagedCache(**dict(sizes, **change))


def calls(c):
    """Every call that takes a cache's pages, for 256 channels."""
    k, slots, one = torch.zeros(3, 256, dtype=torch.bfloat16), torch.zeros(3, dtype=torch.int64), torch.ones(3, dtype=torch.int32)
    ws = pages(1 << 16)
    return (lambda: rp.kv_quant_paged(c, k, k, slots), lambda: rp.kv_dequant_paged(c, slots, k=k, v=k),
            lambda: rp.attend_paged(c, k, one[:, None], one, out=k, workspace=ws))


# every one of these holds a whole number of pages of the sizes named
WRONG = [
    dict(page_size=32), dict(page_size=64, k_pages=pages(8, 2, 16, 64), v_pages=pages(8, 2, 16, 64)), dict(bits=8), dict(n_heads=2),
    dict(n_heads=8), dict(head_dim=128), dict(k_pages=pages(3, 2, 32, 64)), dict(v_pages=pages(12, 1, 16, 64)), dict(k_pages=pages(6, 16, 2, 64)),
    dict(k_pages=pages(6 * 2 * 16 * 64)), dict(v_pages=pages(2, 3, 2, 16, 64)),
]


@pytest.mark.parametrize("change", WRONG, ids=lambda c: ",".join("%s=%s" % (n, v if isinstance(v, int) else "x".join(map(str, v.shape))) for n, v in c.items()))
def test_other_pages_are_refused(change):
    for call in calls(cache(**change)):
        with pytest.raises(ValueError, match=r"_pages: expected shape \[pages, "):
            call()


def test_sizes_that_change_after_a_call_are_looked_at_again():
    c = cache()
    for call in calls(c):
        with pytest.raises(ValueError, match="device"):          # (its own pages: it gets as far as the device)
            call()
    c.page_size = 32
    for call in calls(c):
        with pytest.raises(ValueError, match=r"k_pages: expected shape \[pages, 2, 32, 64\]"):
            call()
    c.page_size, c.v_pages = 16, pages(6, 2, 8, 128)
    for call in calls(c):
        with pytest.raises(ValueError, match=r"v_pages: expected shape \[pages, 2, 16, 64\]"):
            call()


def test_sizes_that_no_cache_has():
    for change, status in ((dict(n_heads=1), -2), (dict(page_size=24), -2), (dict(bits=5), -3)):
        for call in calls(cache(**change)):
            with pytest.raises(rp.RptqError, match="status %d" % status):
                call()


def test_a_cache_whose_fields_came_past_the_constructor_is_looked_at():
    """(As unpickling and copying bring them.)"""
    c = rp.PagedCache.__new__(rp.PagedCache)
    c.__dict__.update({n: v for n, v in cache(page_size=32).__dict__.items() if not n.startswith("_")})
    for call in calls(c):
        with pytest.raises(ValueError, match=r"k_pages: expected shape \[pages, 2, 32, 64\]"):
            call()
