"""Thousands of sequences whose page tables could hold far more than they have, so that every workgroup finds its part among all
of them: some cut, most of them short or empty."""
import pytest

from test_gpu_paged import Batch, dev_bf16

pytestmark = pytest.mark.gpu
torch = pytest.importorskip("torch")


@pytest.fixture(scope="module")
def rp():
    import paper_2304_01089_amd as rp_
    rp_.load_library()
    assert torch.cuda.is_available()
    return rp_


@pytest.mark.parametrize("H,share,hd,bits", [(1, 2, 128, 4), (2, 4, 64, 3), (1, 5, 256, 8)])
@pytest.mark.parametrize("B", [3001, 8195])
def test_thousands_of_sequences_some_of_them_cut(rp, B, H, share, hd, bits):
    """Five kinds of sequences in turn: the first five against the oracle, the others like the first of their kind, to the bit (all
    of a kind are cut alike)."""
    lens = [300, 2, 0, 65, 2600]
    b = Batch(rp, lens, H, hd, bits, 64)
    n_q = H * share
    few = b.queries(n_q)
    kind = torch.arange(B, device="cuda") % len(lens)
    table = torch.full((B, 100), -1, dtype=torch.int32, device="cuda")
    table[:, :b.page_table.shape[1]] = b.page_table[kind]
    out = torch.full((B, n_q * hd), float("nan"), device="cuda")
    _, lse = rp.attend_paged(b.cache, dev_bf16(few)[kind], table, b.dev_lens[kind].contiguous(), out=out, want_lse=True)
    torch.cuda.synchronize()
    b.check(few, n_q, hd ** -0.5, out[:5], lse[:5])
    assert torch.equal(out, out[kind]) and torch.equal(lse, lse[kind])
