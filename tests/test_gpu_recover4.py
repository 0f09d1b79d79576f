"""The 4-bit serving example: prompts, decode, a checkpoint and a recovery
through the library's operators."""
import pytest
import torch

from paper_2606_17787_amd import recover4

pytestmark = pytest.mark.gpu

LENS = (37, 300, 5, 1100, 64)


@pytest.mark.parametrize("order,block_size", [("NHD", 16), ("HND", 32)])
@pytest.mark.parametrize("kept", [LENS, (0,) * 5])
def test_a_recovered_worker_decodes_the_same_bits(kept, order, block_size):
    """From a checkpoint of everything and from none at all, the cache holds
    the same bits in other pages, and decode reads them in the same order."""
    want, got = recover4.run(LENS, kept, order=order, block_size=block_size)
    assert torch.isfinite(want.float()).all()
    assert torch.equal(want, got)


@pytest.mark.parametrize("group,head_dim", [(4, 128), (1, 64)])
def test_a_suffix_behind_a_restored_prefix(group, head_dim):
    """The first worker's prompts saw their keys and values unrounded, the
    recovered one's suffixes see the prefix as 4-bit rows: at most half of one
    of 15 steps off, of a spread that is about 4 standard deviations of a
    quarter's 32 (16) elements.  That moves a hidden state by no more than the
    same part of the attention's share of it, 4 / 30; four layers' worth is
    the bound."""
    want, got = recover4.run(LENS, group=group, head_dim=head_dim)
    off = (got - want).float().norm() / want.float().norm()
    assert 0 < float(off) < 4 * 4 / 30
