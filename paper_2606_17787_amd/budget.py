"""A worker that serves from a 16-bit paged cache held to a budget, fails, and is
recovered.

    python -m paper_2606_17787_amd.budget

recover4's small attention-only model with random weights; the cache, its ledger,
its pages and every attention go through the library:

  step      slots -> per layer: append, attend, weigh (prompts in chunks, then a
            token a request)
  shrink    evict over all layers -> release of the pages behind what is left
  failure   the rows of every place, and the ledger's pages, packed as a checkpoint
  recovery  on a fresh worker: slots -> unpack of both; then it goes on

The run compares what the recovered worker decodes with what the first one would
have decoded: equal, bit for bit, with what each later step evicts.
"""
from __future__ import annotations

import numpy as np
import torch

from . import attn
from . import kvckpt as kv
from . import paged
from .recover4 import Model
from .workloads import CacheShape


class Worker:
    """One GPU's 16-bit cache and the requests on it, each held to `budget`
    places: it may pass them by `slack` between two evictions."""

    def __init__(self, model: Model, requests: int, budget: int, slack: int,
                 sinks: int = 4, recent: int = 16, block_size: int = 16,
                 order: str = "NHD", seed: int = 0, device="cuda"):
        self.m, self.R, self.bs, self.device = model, requests, block_size, device
        self.sinks, self.recent = sinks, recent
        self.shape = CacheShape(model.layers, model.H, model.D, block_size,
                                order, 2)
        cols = -(-(budget + slack) // block_size)
        self.nb = requests * cols
        self.cache = torch.empty(self.shape.pool_elems(self.nb),
                                 dtype=torch.bfloat16, device=device)
        self.ledger = paged.new_ledger(self.shape, self.nb, device)
        self.table = torch.full((requests, cols), -1, dtype=torch.int32,
                                device=device)
        ids = np.random.default_rng(seed).permutation(self.nb)
        self.free = torch.from_numpy(ids.astype(np.int32)).to(device)
        self.free_count = torch.tensor([self.nb], device=device)
        self.now = torch.empty_like(self.free_count)
        self.keep = torch.full((requests,), budget, dtype=torch.int32,
                               device=device)
        # places, tokens seen, and places whose pages the table holds
        self.lens = torch.zeros(requests, dtype=torch.int32, device=device)
        self.seen, self.have = (torch.zeros_like(self.lens) for _ in range(2))
        self.left = torch.empty_like(self.lens)
        self.status = torch.zeros(1, dtype=torch.int32, device=device)
        self.ws = paged.new_evict_workspace(self.shape, requests, cols, device)

    def pages(self, end, count: int):
        """Pages for the places from lens to `end`, `count` in all: their slots
        and the sums of their numbers."""
        slots = torch.empty(count, dtype=torch.int64, device=self.device)
        cu = torch.empty(self.R + 1, dtype=torch.int32, device=self.device)
        attn.lumen_attn_slots(self.lens, end, self.table, self.bs, self.nb,
                              self.free, self.free_count, slots, cu, self.left,
                              self.now, self.status, have=self.have)
        self.free_count.copy_(self.now)
        self.have = torch.maximum(self.have, end)
        return slots, cu

    def step(self, tokens: torch.Tensor, new: torch.Tensor,
             max_new: int) -> torch.Tensor:
        """new[r] tokens of every request, packed, through the model."""
        x = self.m.embed[tokens]
        end = self.lens + new
        slots, cu = self.pages(end, tokens.numel())
        at = torch.arange(tokens.numel(), dtype=torch.int32, device=self.device)
        r = torch.searchsorted(cu, at, right=True) - 1
        positions = self.seen[r] + at - cu[r]
        for layer in range(self.m.layers):
            q, k, v = self.m.project(layer, x)
            paged.lumen_paged_append(self.shape, self.nb, layer, self.cache, k,
                                     v, slots, self.status, ledger=self.ledger,
                                     positions=positions)
            out = torch.empty(q.shape, dtype=q.dtype, device=self.device)
            lse = torch.empty(q.shape[:2], device=self.device)
            paged.lumen_paged_attend(self.shape, self.nb, layer, self.cache,
                                     self.table, end, cu, q, out, self.status,
                                     max_new=max_new, lse=lse)
            paged.lumen_paged_weigh(self.shape, self.nb, layer, self.cache,
                                    self.table, end, cu, q, lse, self.ledger,
                                    self.status, max_new=max_new)
            x = self.m.add(layer, x, out)
        self.lens, self.seen = end, self.seen + new
        return x

    def shrink(self) -> None:
        """Every request to its budget; the pages behind go back."""
        paged.lumen_paged_evict(self.shape, self.nb, self.cache, self.ledger,
                                self.table, self.lens, self.keep,
                                self.seen - self.recent, self.left, self.ws,
                                self.status, sinks=self.sinks)
        paged.lumen_paged_release(self.left, self.have, self.table, self.bs,
                                  self.nb, self.free, self.free_count, self.now,
                                  self.status)
        self.free_count.copy_(self.now)
        self.lens = self.left.clone()
        self.have = torch.minimum(self.have, self.lens)

    def _ranges(self):
        """Zero, and the requests' places and pages."""
        return torch.zeros_like(self.lens), self.lens, \
            (self.lens + self.bs - 1) // self.bs

    def checkpoint(self):
        """The rows of all places, the ledger's pages, and how far each request
        is."""
        zero, places, pages = self._ranges()
        led = paged.ledger_shape(self.shape)
        rows = torch.empty(int(places.sum()) * self.shape.token_row_elems,
                           dtype=torch.bfloat16, device=self.device)
        words = torch.empty(int(pages.sum()) * led.token_row_elems,
                            dtype=torch.int32, device=self.device)
        kv.lumen_kv_ckpt_pack_ranges(self.shape, self.nb, self.cache,
                                     self.table, zero, places, rows, self.status)
        kv.lumen_kv_ckpt_pack_ranges(led, self.nb, self.ledger, self.table, zero,
                                     pages, words, self.status)
        return rows, words, self.lens.clone(), self.seen.clone()

    def restore(self, checkpoint) -> None:
        """A checkpoint into fresh pages."""
        rows, words, lens, seen = checkpoint
        self.pages(lens, int(lens.sum()))
        self.lens, self.seen = lens.clone(), seen.clone()
        zero, places, pages = self._ranges()
        kv.lumen_kv_ckpt_unpack_ranges(self.shape, self.nb, self.cache,
                                       self.table, zero, places, rows,
                                       self.status)
        kv.lumen_kv_ckpt_unpack_ranges(paged.ledger_shape(self.shape), self.nb,
                                       self.ledger, self.table, zero, pages,
                                       words, self.status)

    def check(self) -> None:
        code = int(self.status)
        if code != kv.LUMEN_OK:
            raise RuntimeError(kv.lumen_kv_ckpt_strerror(code))


def run(lens=(37, 300, 5, 700, 64), budget: int = 128, chunk: int = 96,
        steps: int = 12, every: int = 4, block_size: int = 16,
        order: str = "NHD", layers: int = 2, kv_heads: int = 2, group: int = 4,
        head_dim: int = 128, seed: int = 0, device="cuda"):
    """Prompts in chunks of at most `chunk` tokens, an eviction after each, then
    single tokens with one every `every` of them.  Returns the hidden states that
    the first worker and the one recovered after the prompts decode."""
    model = Model(layers, kv_heads, group, head_dim, seed=seed, device=device)
    R, rng = len(lens), np.random.default_rng(seed)
    prompts = [rng.integers(0, 512, n) for n in lens]
    answers = rng.integers(0, 512, (steps, R))

    def worker(number):
        return Worker(model, R, budget, max(chunk, every),
                      block_size=block_size, order=order, seed=number,
                      device=device)

    def words(x, dtype=torch.int32):
        return torch.as_tensor(np.asarray(x), dtype=dtype, device=device)

    def decode(w):
        out, one = [], words([1] * R)
        for s in range(steps):
            out.append(w.step(words(answers[s], torch.int64), one, 1))
            if (s + 1) % every == 0:
                w.shrink()
        w.check()
        return torch.stack(out)

    first = worker(1)
    for at in range(0, max(lens), chunk):
        part = [p[at:at + chunk] for p in prompts]
        first.step(words(np.concatenate(part), torch.int64),
                   words([len(p) for p in part]), chunk)
        first.shrink()
    saved = first.checkpoint()
    want = decode(first)
    second = worker(2)
    second.restore(saved)
    return want, decode(second)


def main() -> None:
    for budget in (64, 128, 1024):
        want, got = run(budget=budget)
        print(f"{budget} places a request: decoded states "
              f"{'equal' if torch.equal(got, want) else 'differ'}")


if __name__ == "__main__":
    main()
