"""The 4-bit serving example's library calls on the GPU against their
definitions, one by one."""
import pytest
import torch

import recover_ref
from paper_2606_17787_amd import attn, recover4

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


def test_layers_do_not_wait_for_the_device(monkeypatch):
    """From a step's first append on, its layers are enqueued without a wait
    for the device (prompts, suffixes behind a prefix and decode)."""
    append, step = attn.lumen_attn_append4, recover4.Worker.step

    def watched_append(*args, **kw):
        torch.cuda.set_sync_debug_mode("error")
        append(*args, **kw)

    def watched_step(*args):
        try:
            return step(*args)
        finally:
            torch.cuda.set_sync_debug_mode("default")
    monkeypatch.setattr(attn, "lumen_attn_append4", watched_append)
    monkeypatch.setattr(recover4.Worker, "step", watched_step)
    want, got = recover4.run(LENS, (36, 282, 0, 1048, 0), 1)
    assert torch.isfinite(got.float()).all()
