"""The operators of the 16-bit paged cache together, as a worker uses them: each
call against its definition, and a recovered worker against the one that failed."""
import numpy as np
import pytest
import torch

import paged_ref as ref
from attn_ref import UNIT
from paper_2606_17787_amd import budget, paged
from test_gpu_paged import close

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("places,order,bs", [(64, "NHD", 16), (128, "HND", 8),
                                             (96, "NHD", 24), (1024, "HND", 32)])
def test_a_recovered_worker_goes_on_as_the_first_would_have(places, order, bs):
    want, got = budget.run(budget=places, order=order, block_size=bs)
    assert torch.isfinite(want).all()
    assert torch.equal(got, want)


def test_a_budget_that_nothing_passes_changes_nothing():
    """Without evictions the worker decodes the same whatever its pages hold."""
    a, _ = budget.run(lens=(20, 45), budget=512, chunk=64, steps=3)
    b, _ = budget.run(lens=(20, 45), budget=256, chunk=64, steps=3)
    assert torch.equal(a, b)


@pytest.mark.parametrize("order", ["NHD", "HND"])
def test_each_call_of_a_run_against_its_definition(monkeypatch, order):
    seen = dict(append=0, attend=0, weigh=0, evict=0, release=0)
    real = {n: getattr(paged, f"lumen_paged_{n}") for n in seen}

    def host(t):
        return t.cpu().numpy()

    def append(shape, nb, layer, cache, k, v, slots, status, ledger, positions):
        want, words = cache.clone(), ledger.clone()
        rows = ref.by_slot(want, shape, nb)[layer]
        b, o = slots // shape.block_size, slots % shape.block_size
        rows[0, b, o], rows[1, b, o] = k, v
        words[layer, 0, b, :, o] = 0
        words[layer, 1, b, :, o] = positions[:, None].expand(
            -1, shape.num_kv_heads)
        real["append"](shape, nb, layer, cache, k, v, slots, status,
                       ledger=ledger, positions=positions)
        assert torch.equal(cache.view(torch.int16), want.view(torch.int16))
        assert torch.equal(ledger, words)
        seen["append"] += 1

    def attend(shape, nb, layer, cache, table, lens, cu, q, out, status,
               max_new, lse):
        real["attend"](shape, nb, layer, cache, table, lens, cu, q, out, status,
                       max_new=max_new, lse=lse)
        want, slack, wl, lslack, written, code = ref.attended(
            q, cache, shape, nb, host(table), host(lens), host(cu), None, layer,
            max_new)
        assert written.all() and code == 0
        close(out, want, slack, UNIT[out.dtype], "attend")
        close(lse, wl, lslack, 0.0, "lse")
        seen["attend"] += 1

    def weigh(shape, nb, layer, cache, table, lens, cu, q, lse, ledger, status,
              max_new):
        want, slack = ref.weighed(q, lse, cache, shape, nb, host(table),
                                  host(lens), host(cu),
                                  paged.weights_of(ledger)[layer].clone(), None,
                                  layer, max_new)
        real["weigh"](shape, nb, layer, cache, table, lens, cu, q, lse, ledger,
                      status, max_new=max_new)
        close(paged.weights_of(ledger)[layer], want, slack, 0.0, "weigh")
        seen["weigh"] += 1

    def evict(shape, nb, cache, ledger, table, lens, keep, frm, left, ws,
              status, sinks):
        want, words = cache.cpu(), host(ledger).copy()
        rest, code = ref.evicted(want, words, shape, nb, host(table),
                                 host(lens), host(keep), host(frm), sinks)
        real["evict"](shape, nb, cache, ledger, table, lens, keep, frm, left, ws,
                      status, sinks=sinks)
        assert code == 0 and np.array_equal(host(left), rest)
        assert np.array_equal(host(ledger), words)
        assert torch.equal(cache.cpu().view(torch.int16),
                           want.view(torch.int16))
        seen["evict"] += int((rest < host(lens)).any())

    def release(lens, have, table, bs, nb, free, count, now, status):
        want, n, code = ref.released(host(lens), host(have), host(table), bs, nb,
                                     host(free), int(count))
        real["release"](lens, have, table, bs, nb, free, count, now, status)
        assert code == 0 and int(now) == n
        assert np.array_equal(host(free), want)
        # no block is on the list twice, or on it and held
        held = [t for r, h in enumerate(host(lens))
                for t in host(table)[r, :-(-int(h) // bs)]]
        ids = list(want[:n]) + held
        assert len(set(ids)) == len(ids) == nb
        seen["release"] += 1

    for name, f in dict(append=append, attend=attend, weigh=weigh, evict=evict,
                        release=release).items():
        monkeypatch.setattr(paged, f"lumen_paged_{name}", f)
    budget.run(lens=(37, 150, 5, 90), budget=48, chunk=64, steps=6, every=3,
               order=order, head_dim=64)
    assert min(seen.values()) > 3, seen
