"""The check of the 4-bit serving example's calls, on the CPU with plain calls
in the library's place: it passes what is right and fails what is not."""
import pytest
import torch

import recover_ref
from paper_2606_17787_amd import attn, recover4

LENS, KEPT, STEPS = (37, 70, 5, 100, 20), (30, 70, 0, 83, 1), 2


def run(monkeypatch, kept=KEPT, order="NHD"):
    record = recover_ref.Record(monkeypatch)
    recover4.run(LENS, kept, STEPS, 16, order, head_dim=64, device="cpu")
    return record


@pytest.mark.parametrize("order", ["NHD", "HND"])
@pytest.mark.parametrize("kept", [KEPT, (0,) * 5])
def test_plain_calls_pass(monkeypatch, kept, order):
    recover_ref.use_plain_calls(monkeypatch)
    recover_ref.check(run(monkeypatch, kept, order), 2, LENS, kept, STEPS)


def zeroed(k, v):
    k.zero_(), v.zero_()


def swapped(k, v):
    both = k.clone()
    k.copy_(v), v.copy_(both)


def misordered(k, v):
    for x in (k, v):
        x[:30] = x[:30].flip(0)


def one_request_dropped(k, v):
    k[:37], v[:37] = 0, 0


def one_bit_off(k, v):
    v[3, 0, 5] = torch.nextafter(v[3, 0, 5], torch.tensor(
        9.0, dtype=v.dtype))


@pytest.mark.parametrize("mistake", [zeroed, swapped, misordered,
                                     one_request_dropped, one_bit_off])
def test_a_wrong_prefix_fails(monkeypatch, mistake):
    """Mistakes planted in the plain read-back of the prefix."""
    recover_ref.use_plain_calls(monkeypatch)

    def read4(shape, nb, layer, cache, slots, k, v, status):
        recover_ref.read4(shape, nb, layer, cache, slots, k, v, status)
        mistake(k, v)
    monkeypatch.setattr(attn, "lumen_attn_read4", read4)
    with pytest.raises(AssertionError, match="keys|values"):
        recover_ref.check(run(monkeypatch), 2, LENS, KEPT, STEPS)


@pytest.mark.parametrize("mistake", ["not restored", "shifted", "swapped"])
def test_a_wrong_restore_fails(monkeypatch, mistake):
    """Mistakes planted in the plain checkpoint."""
    recover_ref.use_plain_calls(monkeypatch)

    def unpack(shape, nb, cache, table, start, end, ckpt, status):
        rows = ckpt.view(-1, shape.num_layers, 2, shape.num_kv_heads,
                         shape.head_dim)
        rows = {"not restored": torch.zeros_like(rows),
                "shifted": rows.roll(1, 0), "swapped": rows.flip(2)}[mistake]
        recover_ref.unpack_ranges(shape, nb, cache, table, start, end,
                                  rows.contiguous(), status)
    monkeypatch.setattr(recover4.kv, "lumen_kv_ckpt_unpack_ranges", unpack)
    with pytest.raises(AssertionError, match="keys|values"):
        recover_ref.check(run(monkeypatch), 2, LENS, KEPT, STEPS)


def test_wrong_decode_attention_fails(monkeypatch):
    """A key too few in a plain decode."""
    recover_ref.use_plain_calls(monkeypatch)

    def decode4(shape, nb, layer, cache, table, lens, q, out, ws, status):
        recover_ref.decode4(shape, nb, layer, cache, table, lens - 1, q, out,
                            ws, status)
    monkeypatch.setattr(attn, "lumen_attn_decode4", decode4)
    with pytest.raises(AssertionError, match="decode"):
        recover_ref.check(run(monkeypatch), 2, LENS, KEPT, STEPS)
