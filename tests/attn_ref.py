"""Plain references of the serving operators for the tests: the definitions of
include/lumen_attn.h in Python loops (slots) and in 64 bits (attention), and
the 4-bit row format in numpy."""
from __future__ import annotations

import numpy as np
import torch

RANGE, BLOCK_ID, CAPACITY = -5, -6, -7


def slots(start, end, table, bs, nb, free, count, num_slots, have=None):
    """(table, slots, cu, lens, left, status) of one step."""
    table = table.copy()
    R, cols = table.shape
    count = max(0, min(int(count), len(free)))
    status, base, cu, lens = 0, 0, [0], []
    out = np.full(num_slots, -1, np.int64)
    left = count
    for r in range(R):
        s, e = int(start[r]), int(end[r])
        h = s if have is None else int(have[r])
        if s < 0 or e < s or h < 0:
            status = min(status, RANGE)
            cu.append(cu[-1])
            lens.append(s)
            continue
        cu.append(cu[-1] + e - s)
        first, last = -(-h // bs), -(-e // bs)
        if last > cols:
            status = min(status, RANGE)
            lens.append(s)
            continue
        need = max(0, last - first)
        if need and base + need > count:
            status = min(status, CAPACITY)
            base += need
            lens.append(s)
            continue
        pages = list(table[r])
        for j in range(need):
            b = int(free[count - 1 - base - j])
            pages[first + j] = b
            if 0 <= b < nb:
                table[r, first + j] = b
            else:
                status = min(status, BLOCK_ID)
        base += need
        if need:
            left = count - base
        lens.append(e)
        for t in range(s, e):
            i = cu[-2] + t - s
            if i >= num_slots:
                break
            b = int(pages[t // bs])
            if 0 <= b < nb:
                out[i] = b * bs + t % bs
            else:
                status = min(status, BLOCK_ID)
    if cu[-1] > num_slots:
        status = min(status, CAPACITY)
    return table, out, np.array(cu, np.int32), np.array(lens, np.int32), \
        left, status


# ---------------------------------------------------------- the 4-bit rows

KV4_MAX = 6848.0


def quantise(x: np.ndarray):
    """(codes uint8 [..., D], A, B float16 [..., 4]) of x [..., D] in the
    32-bit arithmetic the format states."""
    D = x.shape[-1]
    y = np.clip(x.astype(np.float32), -KV4_MAX, KV4_MAX)
    y = y.reshape(x.shape[:-1] + (4, D // 4))
    lo, hi = y.min(-1), y.max(-1)  # NaN propagates
    nan = np.isnan(lo)
    third = np.float32(1.0 / 15.0)
    with np.errstate(all="ignore"):
        A = ((hi - lo) * third).astype(np.float16)
        Af = A.astype(np.float32)
        B = (lo - np.float32(64) * Af).astype(np.float16)
        first = B.astype(np.float32) + np.float32(64) * Af
        inv = np.where(Af > 0, np.float32(1) / Af, np.float32(0))
        q = np.clip(np.rint((y - first[..., None]) *
                            inv.astype(np.float32)[..., None]), 0, 15)
    q = np.where(nan[..., None], 0, q).astype(np.uint8)
    A = np.where(nan, np.float16("nan"), A)
    B = np.where(nan, np.float16("nan"), B)
    return q.reshape(x.shape), A, B


def values(codes, A, B):
    """Values the codes stand for (float16)."""
    D = codes.shape[-1]
    q = codes.reshape(codes.shape[:-1] + (4, D // 4)).astype(np.float64)
    x = A.astype(np.float64)[..., None] * (64 + q) + \
        B.astype(np.float64)[..., None]
    return x.astype(np.float16).reshape(codes.shape)


def to_rows(codes, A, B) -> np.ndarray:
    """Row bytes [..., D/2 + 16]."""
    packed = codes[..., 0::2] | codes[..., 1::2] << 4
    ab = np.stack([A, B], -1).astype(np.float16)
    ab = np.ascontiguousarray(ab.reshape(A.shape[:-1] + (8,))).view(np.uint8)
    return np.concatenate([packed, ab], -1)


def from_rows(rows: torch.Tensor) -> torch.Tensor:
    """Values (float64) of row bytes [..., D/2 + 16]."""
    D = 2 * (rows.shape[-1] - 16)
    codes = torch.stack([rows[..., :D // 2] & 15, rows[..., :D // 2] >> 4], -1)
    codes = codes.reshape(rows.shape[:-1] + (4, D // 4)).double()
    ab = rows[..., D // 2:].contiguous().view(torch.float16).double()
    ab = ab.reshape(rows.shape[:-1] + (4, 2))
    x = ab[..., 0:1] * (64 + codes) + ab[..., 1:2]
    return x.half().double().reshape(rows.shape[:-1] + (D,))


# ------------------------------------------------------------ attention

# Unit roundoff of the output types: half a unit in the last of 8 and of 11
# significant bits.
UNIT = {torch.bfloat16: 2.0 ** -8, torch.float16: 2.0 ** -11}


def attend(q, k, v, scale, seen, p_unit):
    """Attention of q [n, D] over k, v [m, D] in 64 bits with keys seen
    [n, m].  Returns (out, slack): slack bounds the error of a kernel that
    sums in 32 bits and rounds its weights to p_unit before the products with
    v; it leaves out the output's own rounding.

    A score is a sum of D products, each rounding at most 2^-24 of the sum of
    magnitudes: its error is at most 2 D 2^-24 scale sum |q||k| (the 2 for
    scaling and the maximum).  It moves a weight by that factor, numerator and
    denominator alike, so twice in the quotient.  The sums over keys add
    roundings of 2^-24 each, of which 2^-14 allows a thousand in a row."""
    if q.shape[0] == 0 or k.shape[0] == 0:
        return torch.zeros_like(q), torch.zeros_like(q)
    s = torch.matmul(q, k.transpose(0, 1).contiguous()) * scale
    mag = torch.matmul(q.abs(), k.abs().transpose(0, 1).contiguous()) * scale
    mag = torch.where(seen, mag, torch.zeros_like(mag))
    s = s.masked_fill(~seen, float("-inf"))
    top = s.amax(-1, keepdim=True)
    p = torch.exp(s - torch.where(torch.isfinite(top), top, 0.0))
    total = p.sum(-1, keepdim=True)
    p = torch.where(total > 0, p / total, torch.zeros_like(p))
    live = torch.where(seen.any(0)[:, None], v, torch.zeros_like(v))
    out = torch.matmul(p, live)
    size = torch.matmul(p, live.abs())
    err = 2 * q.shape[-1] * 2.0 ** -24 * mag.amax(-1, keepdim=True)
    return out, size * (p_unit + 2 * err + 2.0 ** -14)


def assert_close(got, want, slack, dtype, what=""):
    """|got - want| within slack and the output type's rounding."""
    got = got.double()
    assert torch.isfinite(got).all(), f"{what}: not finite"
    tiny = 2.0 ** -24 if dtype == torch.float16 else 2.0 ** -126
    room = slack + UNIT[dtype] * (want.abs() + slack) + tiny
    off = (got - want).abs()
    if not bool((off <= room).all()):
        at = (off / room).argmax()
        raise AssertionError(
            f"{what}: off by {off.reshape(-1)[at]:.3g} where "
            f"{room.reshape(-1)[at]:.3g} is allowed, at {int(at)} of "
            f"{off.numel()}; {int((off > room).sum())} are too far")
