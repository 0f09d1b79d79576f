"""A worker that serves from a 4-bit paged cache, fails, and is recovered.

    python -m paper_2606_17787_amd.recover4

A small attention-only model with random weights stands in for a real one; the
cache, its pages and every attention go through the library:

  prompts   slots -> per layer: append4, prompt
  decode    slots -> per layer: append4, decode4
  failure   the first `kept` tokens of each request were packed as a checkpoint
  recovery  on a fresh worker: slots -> unpack (whole 4-bit rows), then the rest
            of the tokens: slots -> per layer: append4, read4 of the prefix and
            prompt over the prefix and the tokens' own keys; then decode goes on

The run compares what the recovered worker decodes with what the first one
would have decoded.
"""
from __future__ import annotations

import numpy as np
import torch

from . import attn
from . import kvckpt as kv


class Model:
    """Residual attention layers without norms or an MLP: x + attention(x) W."""

    def __init__(self, layers: int, kv_heads: int, group: int, head_dim: int,
                 vocab: int = 512, seed: int = 0, device="cuda"):
        g = torch.Generator().manual_seed(seed)
        self.layers, self.H, self.D = layers, kv_heads, head_dim
        self.Hq = kv_heads * group
        width = self.Hq * head_dim

        def weights(*dims):
            w = torch.randn(*dims, generator=g) * dims[-2] ** -0.5
            return w.to(torch.bfloat16).to(device)
        self.embed = weights(vocab, width) * vocab ** 0.5
        self.qkv = [weights(width, (self.Hq + 2 * kv_heads) * head_dim)
                    for _ in range(layers)]
        self.out = [weights(width, width) for _ in range(layers)]

    def project(self, layer: int, x: torch.Tensor):
        """q, k and v of tokens x: slices of one product."""
        y = torch.mm(x, self.qkv[layer]).view(
            x.shape[0], self.Hq + 2 * self.H, self.D)
        return y[:, :self.Hq], y[:, self.Hq:self.Hq + self.H], \
            y[:, self.Hq + self.H:]

    def add(self, layer: int, x: torch.Tensor, a: torch.Tensor):
        return x + torch.mm(a.reshape(x.shape), self.out[layer])


class Worker:
    """One GPU's 4-bit cache and the requests on it."""

    def __init__(self, model: Model, requests: int, tokens: int,
                 block_size: int = 16, order: str = "NHD", seed: int = 0,
                 device="cuda"):
        self.m, self.R, self.bs, self.device = model, requests, block_size, device
        self.shape = attn.cache_shape4(model.layers, model.H, model.D,
                                       block_size, order)
        cols = -(-tokens // block_size)
        self.nb = requests * cols
        self.cache = torch.empty(self.shape.pool_elems(self.nb),
                                 dtype=torch.uint8, device=device)
        self.table = torch.full((requests, cols), -1, dtype=torch.int32,
                                device=device)
        ids = np.random.default_rng(seed).permutation(self.nb)
        self.free = torch.from_numpy(ids.astype(np.int32)).to(device)
        self.free_count = torch.tensor([self.nb], device=device)
        self.free_left = torch.empty_like(self.free_count)
        self.have = torch.zeros(requests, dtype=torch.int32, device=device)
        self.lens = torch.empty_like(self.have)
        self.status = torch.zeros(1, dtype=torch.int32, device=device)
        self.ws = attn.new_decode4_workspace(self.shape, requests, model.Hq,
                                             device)

    def pages(self, start, end, count: int):
        """Pages for tokens [start, end) of every request, `count` in all:
        their slots and the sums of their numbers."""
        slots = torch.empty(count, dtype=torch.int64, device=self.device)
        cu = torch.empty(self.R + 1, dtype=torch.int32, device=self.device)
        attn.lumen_attn_slots(start, end, self.table, self.bs, self.nb,
                              self.free, self.free_count, slots, cu, self.lens,
                              self.free_left, self.status, have=self.have)
        self.free_count.copy_(self.free_left)
        self.have = torch.maximum(self.have, end)
        return slots, cu

    def step(self, tokens: torch.Tensor, start, end) -> torch.Tensor:
        """Tokens [start, end) of every request, packed, through the model; the
        keys and values before `start` are in the cache."""
        x = self.m.embed[tokens]
        slots, cu = self.pages(start, end, tokens.numel())
        single = bool((end - start == 1).all())
        before = 0 if single else int(start.sum())
        if before:
            # every token's slot, which of the packed keys are old ones, and where
            # the new ones go (by arithmetic: no wait for the device)
            zero = torch.zeros_like(start)
            all_slots, cu_k = self.pages(zero, end, before + tokens.numel())
            at = torch.arange(all_slots.numel(), device=self.device)
            r = torch.searchsorted(cu_k, at, right=True) - 1
            old = at - cu_k[r] < start[r]
            new = torch.arange(tokens.numel(), device=self.device)
            r = torch.searchsorted(cu, new, right=True) - 1
            new = new - cu[r] + start[r] + cu_k[r]
        for layer in range(self.m.layers):
            q, k, v = self.m.project(layer, x)
            attn.lumen_attn_append4(self.shape, self.nb, layer, self.cache, k,
                                    v, slots, self.status)
            out = torch.empty(q.shape, dtype=q.dtype, device=self.device)
            if single:
                attn.lumen_attn_decode4(self.shape, self.nb, layer, self.cache,
                                        self.table, self.lens, q, out, self.ws,
                                        self.status)
            elif not before:
                attn.lumen_attn_prompt(q, k, v, out, cu, self.status)
            else:
                ka, va = (torch.empty((at.numel(),) + k.shape[1:],
                                      dtype=k.dtype, device=self.device)
                          for _ in range(2))
                attn.lumen_attn_read4(
                    self.shape, self.nb, layer, self.cache,
                    torch.where(old, all_slots, -1), ka, va, self.status)
                ka.index_copy_(0, new, k)
                va.index_copy_(0, new, v)
                attn.lumen_attn_prompt(q, ka, va, out, cu, self.status,
                                       cu_k=cu_k)
            x = self.m.add(layer, x, out)
        return x

    def checkpoint(self, kept: torch.Tensor) -> torch.Tensor:
        """The 4-bit rows of the first `kept` tokens of every request."""
        n = int(kept.sum())
        ckpt = torch.empty(n * self.shape.token_row_elems, dtype=torch.uint8,
                           device=self.device)
        kv.lumen_kv_ckpt_pack_ranges(self.shape, self.nb, self.cache,
                                     self.table, torch.zeros_like(kept), kept,
                                     ckpt, self.status)
        return ckpt

    def restore(self, ckpt: torch.Tensor, kept: torch.Tensor) -> None:
        """A checkpoint into fresh pages."""
        zero = torch.zeros_like(kept)
        self.pages(zero, kept, int(kept.sum()))
        kv.lumen_kv_ckpt_unpack_ranges(self.shape, self.nb, self.cache,
                                       self.table, zero, kept, ckpt,
                                       self.status)

    def check(self) -> None:
        code = int(self.status)
        if code != kv.LUMEN_OK:
            raise RuntimeError(kv.lumen_kv_ckpt_strerror(code))


def run(lens=(37, 300, 5, 1100, 64), kept=None, steps: int = 4,
        block_size: int = 16, order: str = "NHD", layers: int = 2,
        kv_heads: int = 2, group: int = 4, head_dim: int = 128, seed: int = 0,
        device="cuda"):
    """Returns the hidden states that the first worker and the recovered one
    decode, [steps, R, width] each.  kept: tokens of each request that the
    checkpoint holds (None: all but the last few)."""
    model = Model(layers, kv_heads, group, head_dim, seed=seed, device=device)
    R, rng = len(lens), np.random.default_rng(seed)
    prompts = [rng.integers(0, 512, n) for n in lens]
    answers = rng.integers(0, 512, (steps, R))
    most = max(lens) + steps
    if kept is None:
        kept = [max(0, n - 1 - 17 * i) for i, n in enumerate(lens)]

    def words(x, dtype=torch.int32):
        return torch.as_tensor(np.asarray(x), dtype=dtype, device=device)

    def decode(worker):
        n, out = words(lens), []
        for s in range(steps):
            out.append(worker.step(words(answers[s], torch.int64), n, n + 1))
            n = n + 1
        worker.check()
        return torch.stack(out)

    first = Worker(model, R, most, block_size, order, 1, device)
    first.step(words(np.concatenate(prompts), torch.int64),
               words([0] * R), words(lens))
    ckpt = first.checkpoint(words(kept))
    want = decode(first)

    second = Worker(model, R, most, block_size, order, 2, device)
    second.restore(ckpt, words(kept))
    rest = [p[k:] for p, k in zip(prompts, kept)]
    if sum(map(len, rest)):
        second.step(words(np.concatenate(rest), torch.int64), words(kept),
                    words(lens))
    return want, decode(second)


def main() -> None:
    lens = (37, 300, 5, 1100, 64)
    for what, kept in (("all of the prompts", lens), ("most of them", None),
                       ("nothing", (0,) * len(lens))):
        want, got = run(lens, kept)
        off = (got - want).float().norm() / want.float().norm()
        print(f"checkpoint of {what}: decoded states "
              f"{'equal' if torch.equal(got, want) else f'off by {off:.2e}'}")


if __name__ == "__main__":
    main()
