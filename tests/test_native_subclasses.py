"""Tensors of a program's own class: their attributes are read as they are, and not asked for one by one through __torch_function__."""
import numpy as np
import pytest

torch = pytest.importorskip("torch")
ASKED = []


class Named(torch.Tensor):
    """Counts what goes through it."""

    @classmethod
    def __torch_function__(cls, func, types, args=(), kwargs=None):
        ASKED.append(func)
        return super().__torch_function__(func, types, args, kwargs or {})


def named(t):
    return t.as_subclass(Named) if isinstance(t, torch.Tensor) else t


def test_refused_without_being_asked():
    """On the host a tensor's device is the first thing that is wrong with it."""
    import os
    import paper_2304_01089_amd as rp
    if not os.path.exists(rp.library_path()):
        pytest.skip("librptq.so is not built")
    rp.load_library()
    x, bytes_, ints, rows = (named(torch.zeros(4, 128, dtype=t)) for t in (torch.bfloat16, torch.uint8, torch.int32, torch.float32))
    freqs, off, one = named(torch.zeros(32, dtype=torch.float64)), np.array([0, 128], np.int32), np.ones(1, np.float32)
    zero = np.zeros(1, np.int32)
    pages, table = named(torch.zeros(1024, dtype=torch.uint8)), named(torch.zeros(2048, dtype=torch.uint8))
    slots, lens = named(torch.zeros(4, dtype=torch.int64)), named(torch.zeros(4, dtype=torch.int32))
    track = named(torch.zeros(4, 2, 16)), named(torch.zeros(4, 2, 16, dtype=torch.int32))
    calls = [
        lambda: rp.rptq_ln_quant(x, 4, 128, None, None, 1e-5, False, ints, off, one, one, zero, 4, bytes_),
        lambda: rp.rptq_cluster_gemm(bytes_, 4, 4, bytes_, 128, off, one, rows, ints, rows, rows, rows),
        lambda: rp.rptq_cluster_rowsums(bytes_, 4, 4, off, one, zero, rows),
        lambda: rp.rptq_cluster_gemm_cw(bytes_, 4, 4, bytes_, 128, off, rows, rows, rows, rows, rows),
        lambda: rp.rptq_kv_quant(x, 4, 128, bytes_, 4, bytes_),
        lambda: rp.rptq_kv_dequant(bytes_, 4, 128, bytes_, 4, x),
        lambda: rp.rptq_kv_quant_paged(x, x, slots, table, table, 4, pages, pages, 16),
        lambda: rp.rptq_kv_dequant_paged(pages, pages, 16, 4, slots, table, table, x, x),
        lambda: rp.rptq_attend_paged(x, 2, 2, 64, 0.1, table, table, 4, pages, pages, 16, ints, lens, x, None, bytes_),
        lambda: rp.rptq_rope(x, x, lens, 64, 64, False, freqs, 1.0),
        lambda: rp.rptq_rope_quant_paged(x, x, x, x, lens, slots, 64, 64, False, freqs, 1.0, table, table, 4, pages, pages, 16),
        lambda: rp.rptq_attend_weights_paged(x, 1, 2, 2, 64, 0.1, table, 4, pages, 16, ints, lens, rows, None, 1, *track),
        lambda: rp.rptq_evict_paged(2, 64, 4, pages, pages, 16, ints, lens, *track, 5, 0, 0, *track, lens, bytes_),
    ]
    for i, call in enumerate(calls):
        del ASKED[:]
        with pytest.raises(ValueError):
            call()
        assert not ASKED, (i, ASKED)


@pytest.mark.gpu
def test_the_same_results():
    """A step of a bounded cache, through the layer's functions."""
    import paper_2304_01089_amd as rp
    from oracle import kv_cache as kvo
    import paged
    rp.load_library()
    H, hd, bits, page, B, n_q = 2, 64, 4, 16, 3, 4
    hc, lo, hi = paged.clusters(H, hd, bits, 3, 7)
    table = torch.from_numpy(paged.table_rows(hc)).cuda()
    x = torch.from_numpy(kvo.round_to_bf16(paged.values(np.random.default_rng(3), lo, hi, 60))).cuda().bfloat16()
    pages = torch.arange(6, dtype=torch.int32, device="cuda").reshape(B, 2)
    slots = torch.arange(60, device="cuda") // 20 * 32 + torch.arange(60, device="cuda") % 20
    positions = (torch.arange(60, device="cuda") % 20).int()
    lens = torch.full((B,), 20, dtype=torch.int32, device="cuda")
    q = torch.randn(B, n_q * hd, generator=torch.Generator(device="cuda").manual_seed(2), device="cuda").bfloat16()
    rot = rp.rotary(hd)

    def step(of):
        cache = rp.paged_cache(6, page, H, hd, bits, table, table)
        cache.k_pages.fill_(0x21), cache.v_pages.fill_(0x43)
        cache.k_pages, cache.v_pages = of(cache.k_pages), of(cache.v_pages)
        track = rp.cache_track(cache, B, 32)
        track.weights, track.positions = of(track.weights), of(track.positions)
        turned = torch.empty_like(q)
        rp.rope(rot, of(q), of(lens), hd, out=of(turned))
        rp.rope_quant_paged(cache, rot, None, of(x), of(x), of(positions), of(slots))
        out, lse = torch.empty(B, n_q * hd, device="cuda"), torch.empty(B, n_q, device="cuda")
        workspace = rp.attend_paged_workspace(cache, B, n_q)
        rp.attend_paged(cache, of(turned), of(pages), of(lens), out=of(out), lse=of(lse), workspace=of(workspace))
        rp.attend_weights_paged(cache, of(turned), of(pages), of(lens), of(lse), track, fresh=20)
        left = torch.zeros_like(lens)
        rp.evict_paged(cache, of(pages), of(lens), track, 11, first=1, recent=3, lens_out=of(left), workspace=rp.evict_paged_workspace(cache, B, 32, 11))
        return [t.as_subclass(torch.Tensor) for t in (turned, out, lse, left, cache.k_pages, cache.v_pages, track.weights, track.positions)]

    for a, b in zip(step(lambda t: t), step(named)):
        assert torch.equal(a, b)
    x2, y, pos = named(q), named(torch.empty_like(q)), named(lens)
    del ASKED[:]
    rp.rptq_rope(x2, y, pos, hd, hd, False, named(rot.freqs), 1.0)
    assert not ASKED
