"""What the paged entry points refuse, on the host alone: every refusal comes before any HIP call, so no address here is real."""
import ctypes
import os

import pytest

import paper_2304_01089_amd as rp

F = ctypes.c_void_p(4096)          # (some 16-byte-aligned address; never followed)
ODD = ctypes.c_void_p(4100)
NULL, SHAPE, BITS, ALIGN, RANGE, WORKSPACE = -1, -2, -3, -4, -6, -7


@pytest.fixture(scope="module")
def lib():
    if not os.path.exists(rp.library_path()):
        from paper_2304_01089_amd.build import build_library
        build_library()
    return rp.load_library()


def test_sizes(lib):
    assert rp.rptq_kv_page_bytes(128, 16, 4) == 16 * 64
    assert rp.rptq_kv_page_bytes(12288, 64, 3) == 64 * 4608
    assert rp.rptq_kv_page_bytes(256, 4096, 8) == 4096 * 256
    for d, page, bits in ((64, 16, 4), (192, 16, 4), (128, 8, 4), (128, 24, 4), (128, 8192, 4), (128, 0, 4), (128, -16, 4),
                          (0, 16, 4), (-128, 16, 4), (32896, 16, 4), (128, 16, 5)):
        assert rp.rptq_kv_page_bytes(d, page, bits) == 0
    assert rp.rptq_attend_paged_workspace_bytes(4, 8, 2, 128) >= 0
    for B, n_q, n_kv, hd in ((-1, 8, 2, 128), (4, 7, 2, 128), (4, 8, 0, 128), (4, 0, 2, 128), (4, 8, 2, 80), (4, 8, 2, 512), (4, 1, 1, 64),
                             (4, 512, 1, 128), (1 << 21, 8, 2, 128)):
        assert rp.rptq_attend_paged_workspace_bytes(B, n_q, n_kv, hd) == 0


ROWS = dict(k=F, ld_k=128, v=F, ld_v=128, T=4, d=128, k_table=F, v_table=F, bits=4, slots=F, k_pages=F, v_pages=F, n_pages=2,
            page_size=16, stream=None)
BAD_ROWS = [(name, None, NULL) for name in ("k", "v", "k_table", "v_table", "slots", "k_pages", "v_pages")]
BAD_ROWS += [(name, ODD, ALIGN) for name in ("k", "v", "k_table", "v_table", "slots", "k_pages", "v_pages")]
BAD_ROWS += [("bits", 5, BITS), ("bits", 0, BITS), ("T", -1, SHAPE), ("d", 64, SHAPE), ("d", 192, SHAPE), ("d", 0, SHAPE), ("d", 65536, SHAPE),
             ("ld_k", 120, SHAPE), ("ld_v", 127, SHAPE), ("ld_k", 132, SHAPE), ("ld_v", -128, SHAPE), ("n_pages", 0, SHAPE), ("n_pages", -1, SHAPE),
             ("n_pages", 1 << 31, SHAPE), ("page_size", 8, SHAPE), ("page_size", 48, SHAPE), ("page_size", 8192, SHAPE), ("page_size", 0, SHAPE)]


@pytest.mark.parametrize("name,value,status", BAD_ROWS)
def test_rows_refused(lib, name, value, status):
    a = dict(ROWS, **{name: value})
    assert lib.rptq_kv_quant_paged(a["k"], a["ld_k"], a["v"], a["ld_v"], a["T"], a["d"], a["k_table"], a["v_table"], a["bits"],
                                   a["slots"], a["k_pages"], a["v_pages"], a["n_pages"], a["page_size"], None) == status
    assert lib.rptq_kv_dequant_paged(a["k_pages"], a["v_pages"], a["n_pages"], a["page_size"], a["bits"], a["slots"], a["T"], a["d"],
                                     a["k_table"], a["v_table"], a["k"], a["ld_k"], a["v"], a["ld_v"], None) == status


ATTEND = dict(q=F, ld_q=1024, B=4, n_q=8, n_kv=2, hd=128, scale=0.1, k_table=F, v_table=F, bits=4, k_pages=F, v_pages=F, n_pages=9,
              page_size=16, page_table=F, ld_pt=3, per_seq=3, lens=F, out=F, ld_out=1024, dtype=rp.DTYPE_BF16, lse=None, workspace=F,
              ws_bytes=1 << 30)
BAD_ATTEND = [(name, None, NULL) for name in ("q", "k_table", "v_table", "k_pages", "v_pages", "page_table", "lens", "out", "workspace")]
BAD_ATTEND += [(name, ODD, ALIGN) for name in ("q", "k_table", "v_table", "k_pages", "v_pages", "out", "workspace")]
BAD_ATTEND += [(name, ctypes.c_void_p(4098), ALIGN) for name in ("page_table", "lens", "lse")]
BAD_ATTEND += [("bits", 2, BITS), ("B", -1, SHAPE), ("B", 32769, SHAPE), ("n_q", 7, SHAPE), ("n_q", 0, SHAPE), ("n_kv", 0, SHAPE), ("n_kv", -2, SHAPE), ("hd", 80, SHAPE),
               ("hd", 16, SHAPE), ("hd", 0, SHAPE), ("n_q", 512, SHAPE), ("ld_q", 1016, SHAPE), ("ld_q", 1028, SHAPE), ("ld_out", 0, SHAPE),
               ("per_seq", 0, SHAPE), ("ld_pt", 2, SHAPE), ("dtype", 2, SHAPE), ("n_pages", 0, SHAPE), ("page_size", 20, SHAPE),
               ("scale", float("nan"), RANGE), ("scale", float("inf"), RANGE), ("ws_bytes", 0, WORKSPACE)]


def attend(lib, a):
    return lib.rptq_attend_paged(a["q"], a["ld_q"], a["B"], a["n_q"], a["n_kv"], a["hd"], a["scale"], a["k_table"], a["v_table"], a["bits"],
                                 a["k_pages"], a["v_pages"], a["n_pages"], a["page_size"], a["page_table"], a["ld_pt"], a["per_seq"], a["lens"],
                                 a["out"], a["ld_out"], a["dtype"], a["lse"], a["workspace"], a["ws_bytes"], None)


@pytest.mark.parametrize("name,value,status", BAD_ATTEND)
def test_attention_refused(lib, name, value, status):
    assert attend(lib, dict(ATTEND, **{name: value})) == status


def test_tokens_of_a_sequence_fit_32_bits(lib):
    assert attend(lib, dict(ATTEND, page_size=4096, per_seq=(1 << 17) + 1, ld_pt=1 << 20)) == SHAPE


def test_tensors_that_are_not_on_the_device_are_refused():
    torch = pytest.importorskip("torch")
    t = torch.zeros(4, 128, dtype=torch.bfloat16)
    pages = torch.zeros(2, 1, 16, 64, dtype=torch.uint8)
    cache = rp.PagedCache(2, 64, 4, 16, pages, pages, t, t)
    slots = torch.zeros(4, dtype=torch.int64)
    for call in (lambda: rp.kv_quant_paged(cache, t, t, slots), lambda: rp.kv_dequant_paged(cache, slots),
                 lambda: rp.attend_paged(cache, t, slots[:, None].int(), slots.int(), out=t, workspace=pages)):
        with pytest.raises(ValueError, match="device"):
            call()
