"""The 4-bit serving example's library calls on the GPU against their
definitions, one by one."""
import pytest

import recover_ref
from paper_2606_17787_amd import recover4

pytestmark = pytest.mark.gpu

LENS = (37, 300, 5, 1100, 64)


@pytest.mark.parametrize("order,block_size", [("NHD", 16), ("HND", 32)])
@pytest.mark.parametrize("group,head_dim", [(4, 128), (1, 64)])
@pytest.mark.parametrize("kept", [(36, 282, 0, 1048, 0), (37, 0, 3, 1, 64),
                                  (0, 0, 0, 0, 0)])
def test_every_attention_of_a_recovery(monkeypatch, kept, group, head_dim,
                                       order, block_size):
    """Each attention of both workers against the definitions, over the keys
    and values of the request's own tokens: the restored prefix bit for bit.
    (What mistakes this catches: test_recover4.py.)"""
    record = recover_ref.Record(monkeypatch)
    recover4.run(LENS, kept, 3, block_size, order, group=group,
                 head_dim=head_dim)
    recover_ref.check(record, 2, LENS, kept, 3)
