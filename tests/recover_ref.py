"""What the 4-bit serving example has to compute, for its tests: a plain form of
the library calls it makes (CPU tensors), and a record of its calls that is
checked against the definitions, token by token, without its block tables."""
from __future__ import annotations

import numpy as np
import torch

import attn_ref as ref
from paper_2606_17787_amd import attn
from paper_2606_17787_amd import kvckpt as kv

NAMES = ("lumen_attn_slots", "lumen_attn_append4", "lumen_attn_read4",
         "lumen_attn_decode4", "lumen_attn_prompt")


def stored(x: torch.Tensor) -> torch.Tensor:
    """The values (float64) that a 4-bit cache holds of x."""
    v = ref.values(*ref.quantise(x.float().cpu().numpy()))
    return torch.from_numpy(v.astype(np.float64)).to(x.device)


# ------------------------------------------------------- plain library calls

def _rows(shape, nb, layer, cache):
    c = cache.view(shape.pool_dims(nb))[layer]
    return c if shape.order == "NHD" else c.transpose(2, 3)


def slots(start, end, table, bs, nb, free, count, out, cu, lens, left, status,
          have=None, stream=None):
    got = ref.slots(start.numpy(), end.numpy(), table.numpy(), bs, nb,
                    free.numpy(), int(count), out.numel(),
                    None if have is None else have.numpy())
    for t, x in zip((table, out, cu, lens), got):
        t.copy_(torch.from_numpy(x))
    left.fill_(int(got[4]))
    status.clamp_(max=got[5])


def append4(shape, nb, layer, cache, k, v, slots, status, stream=None):
    rows, bs = _rows(shape, nb, layer, cache), shape.block_size
    for i, x in enumerate((k, v)):
        r = torch.from_numpy(ref.to_rows(*ref.quantise(x.float().numpy())))
        live = slots >= 0
        rows[i, slots[live] // bs, slots[live] % bs] = r[live]


def read4(shape, nb, layer, cache, slots, k, v, status, stream=None):
    rows, bs = _rows(shape, nb, layer, cache), shape.block_size
    for i, x in enumerate((k, v)):
        val = ref.from_rows(rows[i, slots.clamp(min=0) // bs, slots % bs])
        x.copy_(torch.where((slots >= 0)[:, None, None], val, 0.0))


def decode4(shape, nb, layer, cache, table, lens, q, out, ws, status,
            scale=None, stream=None):
    rows, bs = _rows(shape, nb, layer, cache), shape.block_size
    for r, n in enumerate(lens.tolist()):
        t = torch.arange(n)
        k, v = (ref.from_rows(rows[i, table[r, t // bs].long(), t % bs])
                for i in (0, 1))
        out[r:r + 1] = attend(q[r:r + 1], k, v, 0.0)[0].to(out.dtype)


def prompt(q, k, v, out, cu_q, status, cu_k=None, scale=None, workspace=None,
           stream=None):
    cu_k = cu_q if cu_k is None else cu_k
    for s in range(len(cu_q) - 1):
        a, b, e, f = *cu_q[s:s + 2].tolist(), *cu_k[s:s + 2].tolist()
        out[a:b] = attend(q[a:b], k[e:f], v[e:f], 0.0)[0].to(out.dtype)


def _tokens(shape, nb, cache, table, start, end):
    """The pool as [tokens of all requests, layer, 2, H, row] indices."""
    c, bs = cache.view(shape.pool_dims(nb)), shape.block_size
    c = c if shape.order == "NHD" else c.transpose(3, 4)
    for r, (s, e) in enumerate(zip(start.tolist(), end.tolist())):
        for t in range(s, e):
            yield c[:, :, int(table[r, t // bs]), t % bs]


def pack_ranges(shape, nb, cache, table, start, end, ckpt, status):
    rows = ckpt.view(-1, shape.num_layers, 2, shape.num_kv_heads,
                     shape.head_dim)
    for i, x in enumerate(_tokens(shape, nb, cache, table, start, end)):
        rows[i] = x


def unpack_ranges(shape, nb, cache, table, start, end, ckpt, status):
    rows = ckpt.view(-1, shape.num_layers, 2, shape.num_kv_heads,
                     shape.head_dim)
    for i, x in enumerate(_tokens(shape, nb, cache, table, start, end)):
        x.copy_(rows[i])


def use_plain_calls(monkeypatch):
    for name, fn in zip(NAMES, (slots, append4, read4, decode4, prompt)):
        monkeypatch.setattr(attn, name, fn)
    monkeypatch.setattr(kv, "lumen_kv_ckpt_pack_ranges", pack_ranges)
    monkeypatch.setattr(kv, "lumen_kv_ckpt_unpack_ranges", unpack_ranges)


# ------------------------------------------------------------------ the record

class Record(list):
    """(name, arguments as they are after the call) of the example's library
    calls."""

    def __init__(self, monkeypatch):
        super().__init__()
        for name in NAMES:
            monkeypatch.setattr(attn, name, self._wrap(name))

    def _wrap(self, name):
        fn = getattr(attn, name)

        def held(x):
            if not torch.is_tensor(x):
                return x
            # caches are told apart by their place, and not copied
            return x.data_ptr() if x.dtype == torch.uint8 else x.clone()

        def call(*args, **kw):
            fn(*args, **kw)
            self.append((name[len("lumen_attn_"):], [held(x) for x in args],
                         {a: held(x) for a, x in kw.items()}))
        return call


def attend(q, k, v, p_unit):
    """(out, slack) of queries [n, Hq, D] at the ends of keys [m, H, D]."""
    n, m, G = q.shape[0], k.shape[0], q.shape[1] // k.shape[1]
    i = torch.arange(n, device=q.device)[:, None] + m - n
    seen = torch.arange(m, device=q.device)[None] <= i
    heads = [ref.attend(q[:, h].double(), k[:, h // G].double(),
                        v[:, h // G].double(), q.shape[2] ** -0.5, seen, p_unit)
             for h in range(q.shape[1])]
    return (torch.stack([o for o, _ in heads], 1),
            torch.stack([s for _, s in heads], 1))


def check(record, layers, lens, kept, steps):
    """Every attention of a run over requests of `lens` tokens, of which the
    second worker gets the first `kept` from the checkpoint, against the
    definitions: keys and values are what earlier appends of the same request
    put there, in 4 bits, except a prompt's own, which are as projected.  The
    prefix rows have to be equal bit for bit, the outputs within the error of
    a kernel that rounds its weights (attn_ref.attend)."""
    R = len(lens)
    own = [n - k for n, k in zip(lens, kept)]
    caches = [a[3] for name, a, _ in record if name == "append4"]
    first, second = dict.fromkeys(caches)  # in the order of their first use
    calls = {c: [[] for _ in range(layers)] for c in (first, second)}
    cache = None
    for name, a, kw in record:
        if name in ("append4", "read4", "decode4"):
            cache, layer = a[3], a[2]
        if name != "slots":  # a prompt is of the append before it
            calls[cache][layer].append((name, a, kw))
    for layer in range(layers):
        held = {}
        for c, new in ((first, lens), (second, own)):
            at = iter(calls[c][layer])
            name, a, _ = next(at)
            assert name == "append4"
            cu = np.cumsum([0] + list(new))
            mine = [x.split(list(new)) for x in a[4:6]]
            past = [[torch.empty((0,) + a[4].shape[1:], dtype=torch.float64,
                                 device=a[4].device)] * R] * 2
            if c == second:
                past = [[held[r][i][:kept[r]] for r in range(R)]
                        for i in (0, 1)]
            name, a, kw = next(at)
            if name == "read4":
                assert c == second
                name, a, kw = next(at)
            assert name == "prompt" and a[4].tolist() == cu.tolist()
            cu_k = cu
            if c == second and any(kept):
                cu_k = np.cumsum([0] + list(lens))
                assert kw["cu_k"].tolist() == cu_k.tolist()
            q, ka, va, out = a[:4]
            for r in range(R):
                s = slice(int(cu[r]), int(cu[r + 1]))
                k, v = (torch.cat([past[i][r].to(q.dtype), mine[i][r]])
                        for i in (0, 1))
                e = slice(int(cu_k[r]), int(cu_k[r + 1]))
                assert torch.equal(ka[e], k), f"keys, request {r}"
                assert torch.equal(va[e], v), f"values, request {r}"
                want, slack = attend(q[s], k, v, ref.UNIT[q.dtype])
                ref.assert_close(out[s], want, slack, q.dtype, f"prompt {r}")
            rows = [[torch.cat([past[i][r], stored(mine[i][r])])
                     for i in (0, 1)] for r in range(R)]
            if c == first:
                held = {r: list(rows[r]) for r in range(R)}
            for _ in range(steps):
                name, a, _ = next(at)
                assert name == "append4"
                for r in range(R):
                    for i in (0, 1):
                        rows[r][i] = torch.cat([rows[r][i],
                                                stored(a[4 + i][r:r + 1])])
                name, a, _ = next(at)
                assert name == "decode4"
                q, out = a[6], a[7]
                for r in range(R):
                    want, slack = attend(q[r:r + 1], *rows[r], 2.0 ** -11)
                    ref.assert_close(out[r:r + 1], want, slack, q.dtype,
                                     f"decode {r}")
            assert next(at, None) is None
