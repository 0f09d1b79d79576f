"""Plain references of the 16-bit paged cache's operators for the tests: the
definitions of include/lumen_paged.h in 64 bits (attention and weights) and in
Python loops (eviction, released pages)."""
from __future__ import annotations

import math

import numpy as np
import torch

from attn_ref import UNIT

RANGE, BLOCK_ID, CAPACITY = -5, -6, -7


def by_slot(cache, shape, nb):
    """A view of a cache as [layers, 2, blocks, block size, heads, head dim]."""
    x = cache.view(shape.pool_dims(nb))
    return x if shape.order == "NHD" else x.transpose(3, 4)


def tables(rng, lens, bs, spare=3, cols=None):
    """Block tables of pages in a random order, -1 past them, and the number of
    blocks."""
    pages = [-(-max(0, int(n)) // bs) for n in lens]
    nb = sum(pages) + spare
    ids = rng.permutation(nb).astype(np.int32)
    table = np.full((len(lens), max([1] + pages) if cols is None else cols),
                    -1, np.int32)
    at = 0
    for r, p in enumerate(pages):
        table[r, :min(p, table.shape[1])] = ids[at:at + p][:table.shape[1]]
        at += p
    return table, nb


def places(table_row, n, bs, nb):
    """(blocks, slots in them, whether they count) of a request's n places."""
    j = np.arange(max(0, n))
    page = j // bs
    there = page < len(table_row)
    block = np.where(there, table_row[np.minimum(page, len(table_row) - 1)], -1) \
        if len(table_row) else np.full(len(j), -1)
    live = (block >= 0) & (block < nb)
    return np.where(live, block, 0), j % bs, live


def attend(q, k, v, scale, seen, p_unit):
    """Attention of q [m, D] over k, v [n, D] in 64 bits with places seen [m, n]:
    (out, its slack, lse, its slack, weights, their slack, relative).

    A score is a sum of D products, each rounding at most 2^-24 of the sum of
    magnitudes: its error is at most e = 2 D 2^-24 scale sum |q||k| (the 2 for
    scaling and the maximum).  lse moves by at most e, the sum's own roundings
    (2^-14 allows a thousand of 2^-24 in a row) and the two of its log and its
    factor.  out's weights move by a factor of e in numerator and denominator
    and are rounded to p_unit.  A weight exp(s - lse) with an lse given moves by
    e, by roundings of s and lse (2^-23 of each, times log2(e) and back) and by the
    exponential's own, 2^-22."""
    m, n = seen.shape
    zero = torch.zeros(m, q.shape[1], dtype=torch.float64, device=q.device)
    if m == 0 or n == 0:
        none = torch.full((m,), -math.inf, dtype=torch.float64, device=q.device)
        return zero, zero, none, torch.zeros_like(none), seen.double(), \
            seen.double()
    s = torch.matmul(q, k.t().contiguous()) * scale
    mag = torch.matmul(q.abs(), k.abs().t().contiguous()) * scale
    s = s.masked_fill(~seen, -math.inf)
    mag = torch.where(s == -math.inf, 0.0, mag)  # exact: no weight at all
    none = ~seen.any(-1)
    top = s.amax(-1)
    # as the formula has it: NaN for a score of NaN or +infinity, or where all are
    # -infinity; a row that sees nothing has no weights
    p = torch.exp(s - top[:, None])
    total = p.sum(-1)
    lse = torch.where((top == -math.inf), top, top + total.log())
    p = torch.where(none[:, None], 0.0, p / total[:, None])
    live = torch.where(seen.any(0)[:, None], v, 0.0)
    out, size = torch.matmul(p, live), torch.matmul(p, live.abs())
    e = 2 * q.shape[-1] * 2.0 ** -24 * mag
    top = e.amax(-1)  # of a row
    lse_slack = top + 2.0 ** -14 + 2.0 ** -22 * lse.abs().nan_to_num(0, 0, 0)
    p_slack = e + 2.0 ** -22 + 2.0 ** -22 * (
        s.abs().nan_to_num(0, 0, 0) + lse.abs().nan_to_num(0, 0, 0)[:, None])
    return out, size * (p_unit + 2 * top[:, None] + 2.0 ** -14), lse, \
        lse_slack, p, p_slack


def request_rows(r, q, cache, shape, nb, table, lens, cu, layer, most_new):
    """(first query, new tokens, k [n, H, D], v, seen [m, n], blocks, slots) of
    request r in 64 bits, or None where it is skipped."""
    a, b = int(cu[r]), int(cu[r + 1])
    if a < 0 or b < a or b > q.shape[0] or b - a > most_new:
        return None
    n, m, bs = max(0, int(lens[r])), b - a, shape.block_size
    block, at, live = places(table[r], n, bs, nb)
    rows = by_slot(cache, shape, nb)[layer]
    k, v = (rows[i, block, at].double() for i in (0, 1))
    j, i = torch.arange(n, device=q.device), torch.arange(m, device=q.device)
    seen = (j[None] <= i[:, None] + n - m) & \
        torch.tensor(live, device=q.device)[None]
    return a, m, k, v, seen, block, at


def attended(q, cache, shape, nb, table, lens, cu, scale=None, layer=0,
             most_new=None):
    """(out, slack, lse, slack, written rows, status) of a call in 64 bits."""
    T, Hq, D = q.shape
    scale = D ** -0.5 if scale is None else scale
    most_new = T if most_new is None else most_new
    G = Hq // shape.num_kv_heads
    out = torch.zeros(T, Hq, D, dtype=torch.float64, device=q.device)
    slack, lse = torch.zeros_like(out), torch.zeros_like(out[..., 0])
    lse_slack = torch.zeros_like(lse)
    written = torch.zeros(T, dtype=torch.bool, device=q.device)
    status = 0
    for r in range(len(lens)):
        x = request_rows(r, q, cache, shape, nb, table, lens, cu, layer, most_new)
        if x is None or lens[r] < 0 or \
                lens[r] > table.shape[1] * shape.block_size:
            status = min(status, RANGE)
        if x is None:
            continue
        a, m, k, v, seen, block, at = x
        written[a:a + m] = True
        n = seen.shape[1]
        _, _, live = places(table[r], min(n, table.shape[1] * shape.block_size),
                            shape.block_size, nb)
        if m and not live.all():
            status = min(status, BLOCK_ID)
        for h in range(Hq):
            o = attend(q[a:a + m, h].double(), k[:, h // G], v[:, h // G],
                       scale, seen, UNIT[q.dtype])
            out[a:a + m, h], slack[a:a + m, h] = o[0], o[1]
            lse[a:a + m, h], lse_slack[a:a + m, h] = o[2], o[3]
    return out, slack, lse, lse_slack, written, status


def weighed(q, lse, cache, shape, nb, table, lens, cu, weights, scale=None,
            layer=0, most_new=None):
    """(weights, slack) of the layer's places after a call, [nb, H, bs].  Sums run
    over the rows 32 at a time, then over 32 lanes, then onto what was there."""
    T, Hq, D = q.shape
    scale = D ** -0.5 if scale is None else scale
    most_new = T if most_new is None else most_new
    H = shape.num_kv_heads
    G = Hq // H
    want, slack = weights.double().clone(), torch.zeros_like(weights.double())
    for r in range(len(lens)):
        x = request_rows(r, q, cache, shape, nb, table, lens, cu, layer, most_new)
        if x is None:
            continue
        a, m, k, v, seen, block, at = x
        if m == 0 or seen.shape[1] == 0:
            continue
        block, at = torch.tensor(block, device=q.device), \
            torch.tensor(at, device=q.device)
        any_ = seen.any(0)
        roundings = (m * G / 32 + 8) * 2.0 ** -24
        for h in range(H):
            total = torch.zeros(seen.shape[1], dtype=torch.float64,
                                device=q.device)
            room = torch.zeros_like(total)
            for g in range(h * G, (h + 1) * G):
                s = torch.matmul(q[a:a + m, g].double(),
                                 k[:, h].t().contiguous()) * scale
                s = s.masked_fill(~seen, -math.inf)
                given = lse[a:a + m, g].double()
                p = torch.where(given[:, None] == -math.inf, 0.0,
                                torch.exp(s - given[:, None]))
                p_slack = attend(q[a:a + m, g].double(), k[:, h], v[:, h],
                                 scale, seen, 0.0)[5]
                total += p.sum(0)
                room += (p * p_slack).sum(0)
            b, o, t = block[any_], at[any_], total[any_]
            want[b, h, o] += t
            slack[b, h, o] += room[any_] + t * roundings + \
                2.0 ** -23 * want[b, h, o].abs()
    return want, slack


def rank_order(weights, pos, sinks, recent_from):
    """Places in the order in which they are kept."""
    def key(j):
        w = float(weights[j])
        first = pos[j] < sinks or pos[j] >= recent_from
        nan = math.isnan(w)
        return (not first, nan, 0.0 if nan else -w, j)
    return sorted(range(len(weights)), key=key)


def evicted(cache, ledger, shape, nb, table, lens, keep, recent_from, sinks,
            first_layer=0, layers=None):
    """(left, status); cache (a host tensor) and ledger (numpy int32) changed in
    place."""
    bs, H = shape.block_size, shape.num_kv_heads
    layers = shape.num_layers - first_layer if layers is None else layers
    rows = by_slot(cache, shape, nb)
    left, status = np.array(lens, np.int32), 0
    for r, n in enumerate(int(x) for x in lens):
        b = int(keep[r])
        if n < 0 or b < 0 or n > table.shape[1] * bs:
            status = min(status, RANGE)
            continue
        if n <= b:
            continue
        block, at, live = places(table[r], n, bs, nb)
        if not live.all():
            status = min(status, BLOCK_ID)
            continue
        left[r] = b
        for layer in range(first_layer, first_layer + layers):
            for h in range(H):
                w = ledger[layer, 0, block, h, at].view(np.float32)
                p = ledger[layer, 1, block, h, at]
                kept = set(rank_order(w, p, sinks, int(recent_from[r]))[:b])
                holes = [j for j in range(b) if j not in kept]
                src = [j for j in range(b, n) if j in kept]
                assert len(holes) == len(src)
                for to, frm in zip(holes, src):
                    rows[layer, :, block[to], at[to], h] = \
                        rows[layer, :, block[frm], at[frm], h]
                    ledger[layer, :, block[to], h, at[to]] = \
                        ledger[layer, :, block[frm], h, at[frm]]
    return left, status


def released(lens, have, table, bs, nb, free, count):
    """(free, count now, status)."""
    free, status = free.copy(), 0
    at = max(0, min(int(count), len(free)))
    for r, (n, h) in enumerate(zip(lens, have)):
        n, h = int(n), int(h)
        if n < 0 or h < 0:
            status = min(status, RANGE)
            continue
        first, last = -(-n // bs), -(-h // bs)
        if last <= first:
            continue
        if last > table.shape[1]:
            status = min(status, RANGE)
            continue
        for p in range(first, last):
            if at >= len(free):
                status = min(status, CAPACITY)
                break
            if not 0 <= table[r, p] < nb:
                status = min(status, BLOCK_ID)
            free[at] = table[r, p]
            at += 1
    return free, at, status
