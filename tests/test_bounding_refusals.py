"""What the rotary and the cache-bounding entry points refuse, on the host alone: every refusal comes before any HIP call, so no
address here is real.  And the frequencies, which are made on the host."""
import ctypes
import math
import os

import numpy as np
import pytest

import paper_2304_01089_amd as rp

F, G = ctypes.c_void_p(4096), ctypes.c_void_p(8192)     # (some 16-byte-aligned addresses; never followed)
OFF8, OFF2, OFF1 = ctypes.c_void_p(4104), ctypes.c_void_p(4098), ctypes.c_void_p(4097)
NULL, SHAPE, BITS, ALIGN, RANGE, WORKSPACE = -1, -2, -3, -4, -6, -7


@pytest.fixture(scope="module")
def lib():
    if not os.path.exists(rp.library_path()):
        from paper_2304_01089_amd.build import build_library
        build_library()
    return rp.load_library()


def refused(call, good, bad):
    for name, value, status in bad:
        assert call(dict(good, **{name: value})) == status, (name, value)


def test_rotations_refused(lib):
    good = dict(x=F, xd=0, ld_x=1024, y=G, yd=0, ld_y=1024, pos=F, T=5, heads=8, hd=128, rot=128, inter=0, freqs=F, amp=1.0)
    bad = [(n, None, NULL) for n in ("x", "y", "pos", "freqs")]
    bad += [("x", OFF1, ALIGN), ("y", OFF1, ALIGN), ("pos", OFF2, ALIGN), ("freqs", ctypes.c_void_p(4100), ALIGN)]
    bad += [("xd", 2, SHAPE), ("yd", -1, SHAPE), ("T", -1, SHAPE), ("T", 1 << 41, SHAPE), ("heads", 0, SHAPE), ("heads", 513, SHAPE), ("hd", 0, SHAPE),
            ("hd", 1025, SHAPE), ("rot", 0, SHAPE), ("rot", 63, SHAPE), ("rot", 130, SHAPE), ("rot", -2, SHAPE), ("ld_x", 1023, SHAPE),
            ("ld_y", 0, SHAPE), ("amp", math.nan, RANGE), ("amp", math.inf, RANGE)]

    def call(a):
        return lib.rptq_rope(a["x"], a["xd"], a["ld_x"], a["y"], a["yd"], a["ld_y"], a["pos"], a["T"], a["heads"], a["hd"], a["rot"], a["inter"],
                             a["freqs"], a["amp"], None)

    refused(call, good, bad)
    refused(call, dict(good, xd=1, yd=1), [("x", OFF2, ALIGN), ("y", OFF2, ALIGN)])
    refused(call, dict(good, y=F), [("ld_y", 1032, SHAPE), ("yd", 1, SHAPE)])          # x itself, at another stride or of another type


ROWS = dict(q=F, ld_q=1024, q_out=G, ld_out=1024, n_q=8, k=F, ld_k=256, v=F, ld_v=256, T=4, n_kv=2, hd=128, pos=F, rot=64, inter=1, freqs=F,
            amp=1.0, k_table=F, v_table=F, bits=4, slots=F, k_pages=F, v_pages=F, n_pages=2, page=16)


def test_rotated_writes_refused(lib):
    bad = [(n, None, NULL) for n in ("q", "q_out", "k", "v", "pos", "freqs", "k_table", "v_table", "slots", "k_pages", "v_pages")]
    bad += [(n, OFF8, ALIGN) for n in ("q", "q_out", "k", "v", "k_table", "v_table", "k_pages", "v_pages")]
    bad += [("pos", OFF2, ALIGN), ("freqs", ctypes.c_void_p(4100), ALIGN), ("slots", ctypes.c_void_p(4100), ALIGN), ("bits", 2, BITS), ("T", -1, SHAPE), ("n_kv", 0, SHAPE),
            ("n_kv", 257, SHAPE), ("n_q", 0, SHAPE), ("n_q", 257, SHAPE), ("hd", 80, SHAPE), ("hd", 512, SHAPE), ("rot", 24, SHAPE), ("rot", 144, SHAPE),
            ("rot", 0, SHAPE), ("rot", 15, SHAPE), ("ld_q", 1020, SHAPE), ("ld_out", 1028, SHAPE), ("ld_k", 248, SHAPE), ("ld_v", 260, SHAPE), ("n_pages", 0, SHAPE),
            ("page", 24, SHAPE), ("amp", math.nan, RANGE)]

    def call(a):
        return lib.rptq_rope_quant_paged(a["q"], a["ld_q"], a["q_out"], a["ld_out"], a["n_q"], a["k"], a["ld_k"], a["v"], a["ld_v"], a["T"], a["n_kv"], a["hd"],
                                         a["pos"], a["rot"], a["inter"], a["freqs"], a["amp"], a["k_table"], a["v_table"], a["bits"], a["slots"],
                                         a["k_pages"], a["v_pages"], a["n_pages"], a["page"], None)

    refused(call, ROWS, bad)
    refused(call, dict(ROWS, q_out=F), [("ld_out", 1032, SHAPE)])


def test_accumulations_refused(lib):
    good = dict(q=F, ld_q=1024, B=4, queries=3, n_q=8, n_kv=2, hd=128, scale=0.1, k_table=F, bits=4, k_pages=F, n_pages=9, page=16, table=F, ld_pt=3,
                per_seq=3, lens=F, lse=F, pos=F, fresh=1, weights=F, tpos=F, cap=48, ws=None, ws_bytes=0)
    bad = [(n, None, NULL) for n in ("q", "k_table", "k_pages", "table", "lens", "lse", "weights", "tpos")]
    bad += [(n, OFF8, ALIGN) for n in ("q", "k_table", "k_pages")] + [(n, OFF2, ALIGN) for n in ("table", "lens", "lse", "pos", "weights", "tpos")]
    bad += [("bits", 5, BITS), ("B", -1, SHAPE), ("B", 32769, SHAPE), ("queries", 0, SHAPE), ("queries", 65537, SHAPE), ("n_q", 7, SHAPE), ("n_kv", 0, SHAPE),
            ("hd", 48, SHAPE), ("ld_q", 1016, SHAPE), ("ld_q", 1028, SHAPE), ("per_seq", 0, SHAPE), ("ld_pt", 2, SHAPE), ("cap", 0, SHAPE), ("cap", (1 << 29) + 1, SHAPE),
            ("fresh", -1, SHAPE), ("n_pages", 0, SHAPE), ("page", 40, SHAPE), ("scale", math.nan, RANGE)]

    def call(a):
        return lib.rptq_attend_weights_paged(a["q"], a["ld_q"], a["B"], a["queries"], a["n_q"], a["n_kv"], a["hd"], a["scale"], a["k_table"], a["bits"], a["k_pages"],
                                             a["n_pages"], a["page"], a["table"], a["ld_pt"], a["per_seq"], a["lens"], a["lse"], a["pos"], a["fresh"], a["weights"],
                                             a["tpos"], a["cap"], a["ws"], a["ws_bytes"], None)

    refused(call, good, bad)
    refused(call, dict(good, page=4096, ld_pt=1 << 20), [("per_seq", (1 << 17) + 1, SHAPE)])
    refused(call, dict(good, queries=100, ws=F, ws_bytes=1 << 30), [("ws", None, WORKSPACE), ("ws_bytes", 1000, WORKSPACE), ("ws", OFF8, ALIGN)])


def test_evictions_refused(lib):
    good = dict(B=4, n_kv=2, hd=128, bits=4, k_pages=F, v_pages=G, n_pages=9, page=16, table=F, ld_pt=3, per_seq=3, lens=F, w=F, p=F, cap=48, budget=10,
                first=2, recent=8, w_out=F, p_out=F, lens_out=G, ws=F, ws_bytes=1 << 20)
    bad = [(n, None, NULL) for n in ("k_pages", "v_pages", "table", "lens", "w", "p", "w_out", "p_out", "lens_out", "ws")]
    bad += [(n, OFF8, ALIGN) for n in ("k_pages", "v_pages", "ws")] + [(n, OFF2, ALIGN) for n in ("table", "lens", "w", "p", "w_out", "p_out", "lens_out")]
    bad += [("bits", 6, BITS), ("B", -1, SHAPE), ("B", 32769, SHAPE), ("n_kv", 0, SHAPE), ("n_kv", 3000, SHAPE), ("hd", 48, SHAPE), ("cap", 0, SHAPE),
            ("cap", 1 << 30, SHAPE), ("budget", 0, SHAPE), ("budget", -5, SHAPE), ("first", -1, SHAPE), ("first", 3, SHAPE), ("recent", -1, SHAPE), ("recent", 9, SHAPE),
            ("recent", 2 ** 31 - 1, SHAPE), ("lens_out", F, SHAPE), ("v_pages", F, SHAPE), ("per_seq", 0, SHAPE), ("ld_pt", 2, SHAPE), ("n_pages", 0, SHAPE), ("page", 8, SHAPE),
            ("ws_bytes", 31, WORKSPACE)]

    def call(a):
        return lib.rptq_evict_paged(a["B"], a["n_kv"], a["hd"], a["bits"], a["k_pages"], a["v_pages"], a["n_pages"], a["page"], a["table"], a["ld_pt"], a["per_seq"],
                                    a["lens"], a["w"], a["p"], a["cap"], a["budget"], a["first"], a["recent"], a["w_out"], a["p_out"], a["lens_out"], a["ws"], a["ws_bytes"], None)

    refused(call, good, bad)
    refused(call, dict(good, B=32768, n_kv=65), [("ws_bytes", 0, SHAPE)])              # more heads than there may be


def test_workspaces(lib):
    assert rp.rptq_attend_weights_paged_workspace_bytes(4, 1, 8, 2, 128) == 0
    assert rp.rptq_attend_weights_paged_workspace_bytes(4, 32, 8, 2, 128) >= 4 * 32 * 8 * 4 * 128       # (four digits of every query's value)
    assert rp.rptq_attend_weights_paged_workspace_bytes(32768, 65536, 128, 1, 256) > 1 << 47
    for a in ((-1, 1, 8, 2, 128), (4, 0, 8, 2, 128), (4, 65537, 8, 2, 128), (4, 1, 7, 2, 128), (4, 1, 8, 2, 100)):
        assert rp.rptq_attend_weights_paged_workspace_bytes(*a) == 0
    assert rp.rptq_evict_paged_workspace_bytes(4, 2, 48, 10) >= 4 * 8
    assert rp.rptq_evict_paged_workspace_bytes(4, 2, 4096, 16) < 1 << 10
    few, many = (rp.rptq_evict_paged_workspace_bytes(400, 2, 100000, n) for n in (16, 50000))
    assert few < 1 << 13 and many >= 4 * 800 * 2 * 50000
    for a in ((-1, 2, 48, 10), (4, 0, 48, 10), (4, 2, 0, 10), (4, 2, 48, 0), (32768, 65, 48, 10)):
        assert rp.rptq_evict_paged_workspace_bytes(*a) == 0


@pytest.mark.parametrize("rot", [2, 4, 20, 64, 128, 1024])
def test_frequencies(lib, rot):
    j = np.arange(rot // 2)
    plain = 10000.0 ** (-2.0 * j / rot)
    f, a = rp.rptq_rope_freqs(rot)
    assert f.dtype == np.float64 and a == 1.0 and np.allclose(f, plain, rtol=1e-13)
    f, a = rp.rptq_rope_freqs(rot, 500000.0, "linear", 4.0)
    assert a == 1.0 and np.allclose(f, 500000.0 ** (-2.0 * j / rot) / 4, rtol=1e-13)
    f, a = rp.rptq_rope_freqs(rot, 10000.0, "base", 4.0)
    assert a == 1.0 and f[0] == 1.0 and (rot == 2 or math.isclose(f[-1], plain[-1] / 4, rel_tol=1e-12))     # (the slowest pair is slowed by the whole factor)
    f, a = rp.rptq_rope_freqs(rot, 10000.0, "parts", 8.0, trained=4096.0, slow=1.0, fast=32.0)
    turns = plain * 4096 / (2 * math.pi)
    assert math.isclose(a, 0.1 * math.log(8.0) + 1) and np.allclose(f[turns >= 32], plain[turns >= 32], rtol=1e-13)
    assert np.allclose(f[turns <= 1], plain[turns <= 1] / 8, rtol=1e-13)
    between = (turns > 1) & (turns < 32)
    assert ((f[between] < plain[between]) & (f[between] > plain[between] / 8)).all() and (np.diff(f) < 0).all()


def test_frequencies_refused(lib):
    for args, status in (((3,), SHAPE), ((0,), SHAPE), ((-2,), SHAPE), ((1026,), SHAPE), ((64, 0.0), RANGE), ((64, -1.0), RANGE), ((64, math.nan), RANGE),
                         ((64, 1e4, "linear", 0.5), RANGE), ((64, 1e4, "base", math.inf), RANGE), ((64, 1e4, "parts", 2.0), RANGE),
                         ((64, 1e4, "parts", 2.0, 4096.0, 5.0, 5.0), RANGE), ((64, 1e4, "parts", 2.0, 4096.0, -1.0, 5.0), RANGE)):
        with pytest.raises(rp.RptqError, match="status %d" % status):
            rp.rptq_rope_freqs(*args)
    with pytest.raises(ValueError, match="scaling"):
        rp.rptq_rope_freqs(64, 1e4, "other")


def test_tensors_that_are_not_on_the_device_are_refused(lib):
    torch = pytest.importorskip("torch")
    x, pos = torch.zeros(4, 128, dtype=torch.bfloat16), torch.zeros(4, dtype=torch.int32)
    pages = torch.zeros(2, 1, 16, 64, dtype=torch.uint8)
    cache = rp.PagedCache(2, 64, 4, 16, pages, pages, x, x)
    rot = rp.rotary(64, device="cpu")
    assert rot.freqs.dtype == torch.float64 and rot.freqs.shape == (32,) and rot.amplitude == 1.0 and not rot.interleaved
    track = rp.cache_track(cache, 4, 20)
    assert track.weights.shape == track.positions.shape == (4, 2, 20)
    for call in (lambda: rp.rope(rot, x, pos, 64), lambda: rp.rope_quant_paged(cache, rot, x, x, x, pos, pos.long()),
                 lambda: rp.attend_weights_paged(cache, x, pos[:, None], pos, torch.zeros(4, 2), track),
                 lambda: rp.evict_paged(cache, pos[:, None], pos, track, 3)):
        with pytest.raises(ValueError, match="device"):
            call()


def test_pages_of_another_shape_are_refused():
    torch = pytest.importorskip("torch")
    x, pos = torch.zeros(4, 128, dtype=torch.bfloat16), torch.zeros(4, dtype=torch.int32)
    pages = torch.zeros(2, 1, 32, 64, dtype=torch.uint8)
    cache = rp.PagedCache(2, 64, 4, 16, pages, pages, x, x)
    rot, track = rp.rotary(64, device="cpu"), rp.CacheTrack(torch.zeros(4, 2, 20), torch.zeros(4, 2, 20, dtype=torch.int32))
    for call in (lambda: rp.rope_quant_paged(cache, rot, x, x, x, pos, pos.long()),
                 lambda: rp.attend_weights_paged(cache, x, pos[:, None], pos, torch.zeros(4, 2), track),
                 lambda: rp.evict_paged(cache, pos[:, None], pos, track, 3)):
        with pytest.raises(ValueError, match=r"k_pages: expected shape \[pages, 1, 16, 64\]"):
            call()
