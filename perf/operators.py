"""What the serving operators cost: block tables and slot maps, the 4-bit paged
cache's append and read-back, decode attention over it, and prompt attention.

run() goes through one operator in its plain form (elementary torch operations
in 32 bits, rounded once at the end) or, where `own` is true, through the
framework's kernels.  exact() is the same from the definitions in 64 bits.

A row of the 4-bit cache (one token, one KV head, K or V) holds head_dim / 2
bytes of codes, element 2i in the low half of byte i and 2i + 1 in the high
half, and then four pairs of 16-bit floats (A, B), one for each quarter of the
row's elements.  Code q stands for A * (64 + q) + B, rounded to 16 bits.  For a
quarter from lo to hi, A is (hi - lo) / 15 and B is lo - 64 * A, each rounded to
16 bits, and an element's code is the nearest.  Elements are held to +-6848, so
that B stays in range.
"""
import math

import numpy as np
import torch

own = False

DT = {"bf16": torch.bfloat16, "fp16": torch.float16}


# ------------------------------------------------------------------- the cases

def listed():
    return [
        # A decode step of a tiny deployment: one new token for each of 8
        # requests.  Latency is all there is.
        dict(name="slots-step-8", op="slots", R=8, median=216, sigma=0.5, new=1, cols=32, bs=16),
        # 1,024 prompts admitted at once into fresh pages.
        dict(name="slots-prompts-1024", op="slots", R=1024, median=0, sigma=0.75, new=512, cols=512, bs=32),
        # The new tokens of a 256-request decode step, one layer of a
        # Llama-3-8B-shaped cache.
        dict(name="append-step-256", op="append", T=256, H=8, D=128, bs=16, order="NHD", dtype="bf16"),
        # A batch of prompts written into one layer (an odd number of tokens).
        dict(name="append-prompts-16411", op="append", T=16411, H=8, D=128, bs=16, order="NHD", dtype="bf16"),
        # Decode over the tiny cache: 8 requests of a few hundred tokens.
        dict(name="decode-tiny-8", op="decode", R=8, H=2, G=2, D=64, bs=16, order="NHD", dtype="bf16", median=216, sigma=0.5, clip=432),
        # The ordinary step: 256 requests around 2,048 tokens, 32 query heads
        # over 8 KV heads.
        dict(name="decode-256", op="decode", R=256, H=8, G=4, D=128, bs=16, order="NHD", dtype="bf16", median=2048, sigma=0.75, clip=16384),
        # Three long contexts, head-major pages of 32 tokens: few rows, so the
        # keys have to be split.
        dict(name="decode-long-3", op="decode", R=3, H=8, G=4, D=128, bs=32, order="HND", dtype="fp16", median=100003, sigma=0.3, clip=131072),
        # One tensor-parallel rank of a 70B-shaped model: one KV head, 8 query
        # heads, 512 requests around 4,096 tokens.
        dict(name="decode-tp8-512", op="decode", R=512, H=1, G=8, D=128, bs=16, order="NHD", dtype="bf16", median=4096, sigma=0.75, clip=32768),
        # Prompts of the tiny deployment: 8 of a few hundred tokens.
        dict(name="prompt-tiny-8", op="prompt", R=8, H=2, G=2, D=64, dtype="fp16", median=216, sigma=0.5, clip=432, prefix=0),
        # A batch of packed prompts of very different lengths.
        dict(name="prompt-packed-24", op="prompt", R=24, H=8, G=4, D=128, dtype="bf16", median=384, sigma=0.75, clip=4096, prefix=0),
        # One long prompt.
        dict(name="prompt-16384", op="prompt", R=1, H=8, G=4, D=128, dtype="bf16", median=16384, sigma=0.0, clip=16384, prefix=0),
        # Suffixes behind restored prefixes on one tensor-parallel rank: the
        # recovery of requests whose checkpoint holds most of their prompt.
        dict(name="prompt-suffix-tp8-5", op="prompt", R=5, H=1, G=8, D=128, dtype="bf16", median=1237, sigma=0.5, clip=4096, prefix=11003),
    ]


def _log(rng, lo, hi):
    """A whole number spread over the logarithm of [lo, hi], odd ones too."""
    return min(hi, max(lo, int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))))


def draw(rng):
    op = rng.choice(["slots", "append", "decode", "decode", "prompt", "prompt"])
    bs = rng.choice([8, 16, 16, 32, 64])
    order = rng.choice(["NHD", "HND"])
    dtype = rng.choice(["bf16", "fp16"])
    if op == "slots":
        R = _log(rng, 1, 1024)
        return dict(op=op, R=R, median=rng.choice([0, _log(rng, 1, 4096)]), sigma=0.6, new=rng.choice([1, _log(rng, 1, 512)]), cols=16384 // bs, bs=bs)
    if op == "append":
        H = rng.choice([1, 2, 4, 8])
        return dict(op=op, T=_log(rng, 1, 16384), H=H, D=rng.choice([64, 128, 128, 256]), bs=bs, order=order, dtype=dtype)
    if op == "decode":
        H, G, D = rng.choice([1, 2, 4, 8]), rng.choice([1, 2, 3, 4, 7, 8]), rng.choice([64, 128, 128, 256])
        R = _log(rng, 1, 256)
        most = 600_000 * 8 * 128 // (R * H * D * 3)  # the padded plain form stays inside the largest listed case
        median = _log(rng, 1, max(2, min(32768, most // 4)))
        return dict(op=op, R=R, H=H, G=G, D=D, bs=bs, order=order, dtype=dtype, median=median, sigma=0.6, clip=4 * median)
    H, G, D = rng.choice([1, 2, 4, 8]), rng.choice([1, 2, 3, 4, 7, 8]), rng.choice([64, 128, 128])
    R = _log(rng, 1, 16)
    most = math.sqrt(32 * 16384.0 * 16384.0 / (H * G)) / R  # tokens a request at the largest listed case's cost
    prefix = rng.choice([0, 0, _log(rng, 1, max(2, int(min(16384, most / 2))))])
    median = _log(rng, 1, max(2, int(min(16384, most / 1.5 - prefix))))
    return dict(op=op, R=R, H=H, G=G, D=D, dtype=dtype, median=median, sigma=0.5, clip=2 * median, prefix=prefix)


def _lengths(median, sigma, n, hi):
    """n lengths at the quantiles of a lognormal distribution, in a mixed order
    that is the same every time; at least 1, at most hi; odd ones among them."""
    z = np.array([_normal_quantile((i + 0.5) / n) for i in range(n)])
    x = np.clip(np.rint(median * np.exp(sigma * z)), 1, hi).astype(np.int64)
    return x[np.random.RandomState(n).permutation(n)]


def _normal_quantile(p):
    """The standard normal distribution's quantile, by bisection on erf."""
    lo, hi = -8.0, 8.0
    for _ in range(60):
        mid = (lo + hi) / 2
        lo, hi = (mid, hi) if 0.5 * (1 + math.erf(mid / math.sqrt(2))) < p else (lo, mid)
    return (lo + hi) / 2


# -------------------------------------------------------------------- the work

def _slots_lengths(c):
    start = _lengths(c["median"], c["sigma"], c["R"], 8192) if c["median"] else np.zeros(c["R"], np.int64)
    new = np.ones(c["R"], np.int64) if c["new"] == 1 else _lengths(c["new"], c["sigma"], c["R"], 8192)
    return start, start + new


def _prompt_lengths(c):
    nq = _lengths(c["median"], c["sigma"], c["R"], c["clip"])
    # every third request has no prefix, the others different ones
    nk = nq + (np.arange(c["R"]) % 3 > 0) * (c["prefix"] * (1 + np.arange(c["R"])) // c["R"])
    return nq, nk


def work(case):
    c = case
    if c["op"] == "slots":
        s, e = _slots_lengths(c)
        pages, old = -(-e // c["bs"]), -(-s // c["bs"])
        touched, fresh = int((pages - s // c["bs"]).sum()), int((pages - old).sum())
        return {"bytes": 8 * c["R"] + 8 * fresh + 4 * (touched - fresh) + 8 * int((e - s).sum()) + 8 * c["R"], "flops": int((e - s).sum())}
    if c["op"] == "append":
        n, row = 2 * c["T"] * c["H"], c["D"] // 2 + 16
        return {"bytes": n * (4 * c["D"] + 2 * row) + 8 * c["T"], "flops": 8 * n * c["D"]}
    if c["op"] == "decode":
        total = int(_lengths(c["median"], c["sigma"], c["R"], c["clip"]).sum())
        return {"bytes": 2 * total * c["H"] * (c["D"] // 2 + 16) + 4 * c["R"] * c["H"] * c["G"] * c["D"], "flops": 4 * total * c["H"] * c["G"] * c["D"]}
    nq, nk = _prompt_lengths(c)
    pairs = int((nq * nk - nq * (nq - 1) // 2).sum())
    return {"bytes": 4 * c["D"] * c["H"] * (c["G"] * int(nq.sum()) + int(nk.sum())), "flops": 4 * pairs * c["H"] * c["G"] * c["D"]}


# ------------------------------------------------------------------ the inputs

def _tables(rows, bs, seed, spare=1.05):
    """Block tables of fragmented pages for contexts of `rows` tokens, -1 past
    them, the number of blocks, and the blocks that stay free."""
    pages = -(-rows // bs)
    nb = int(pages.sum() * spare) + 8
    perm = np.random.RandomState(seed % (1 << 31)).permutation(nb).astype(np.int32)
    cols = max(1, int(pages.max()))
    bt = np.full((len(rows), cols), -1, np.int32)
    at = 0
    for r, p in enumerate(pages):
        bt[r, :p] = perm[at:at + p]
        at += p
    return bt, nb, perm[at:]


def _dims(c, nb):
    row = c["D"] // 2 + 16
    return (1, 2, nb, c["bs"], c["H"], row) if c["order"] == "NHD" else (1, 2, nb, c["H"], c["bs"], row)


def _by_slot(cache, order):
    """A view of the cache as [2, blocks, block size, heads, row]."""
    return cache[0] if order == "NHD" else cache[0].transpose(2, 3)


def _shape(c):
    from paper_2606_17787_amd import attn
    return attn.cache_shape4(1, c["H"], c["D"], c["bs"], c["order"])


def prepare(case, seed):
    c, dev = case, "cuda"
    g = torch.Generator(device=dev)
    g.manual_seed(seed)
    status = torch.zeros(1, dtype=torch.int32, device=dev)
    st = {"case": c, "status": status}
    if c["op"] == "slots":
        start, end = _slots_lengths(c)
        bt, nb, _ = _tables(start, c["bs"], seed)
        pages = -(-end // c["bs"])
        nb += int(pages.sum())
        table = np.full((c["R"], max(c["cols"], int(pages.max()))), -1, np.int32)
        table[:, :bt.shape[1]] = bt
        free = np.setdiff1d(np.arange(nb, dtype=np.int32), bt[bt >= 0])
        free = free[np.random.RandomState((seed + 1) % (1 << 31)).permutation(len(free))]
        total = int((end - start).sum())
        st |= {"start": torch.tensor(start, dtype=torch.int32, device=dev), "end": torch.tensor(end, dtype=torch.int32, device=dev),
               "table": torch.tensor(table, device=dev), "free": torch.tensor(free, device=dev), "nb": nb,
               "count": torch.tensor([len(free)], dtype=torch.int64, device=dev), "T": total}
        if own:
            from paper_2606_17787_amd import attn
            st |= {"slots": torch.empty(total, dtype=torch.int64, device=dev), "cu": torch.empty(c["R"] + 1, dtype=torch.int32, device=dev),
                   "lens": torch.empty(c["R"], dtype=torch.int32, device=dev), "left": torch.empty(1, dtype=torch.int64, device=dev)}
            st["call"] = attn.prepare_slots(st["start"], st["end"], st["table"], c["bs"], nb, st["free"], st["count"], st["slots"],
                                            st["cu"], st["lens"], st["left"], status)
        return st
    if c["op"] == "append":
        nb = -(-c["T"] * 5 // (4 * c["bs"])) + 4
        slots = torch.randperm(nb * c["bs"], generator=g, device=dev)[:c["T"]]
        # values with a few heavier channels, as keys have them
        heavy = 1 + 5 * (torch.arange(c["D"], device=dev) % 29 == 3)
        kv = [(torch.randn(c["T"], c["H"], c["D"], generator=g, device=dev) * heavy).to(DT[c["dtype"]]) for _ in range(2)]
        cache = torch.randint(0, 256, _dims(c, nb), generator=g, device=dev, dtype=torch.uint8)
        st |= {"cache": cache, "k": kv[0], "v": kv[1], "slots": slots, "nb": nb}
        if own:
            from paper_2606_17787_amd import attn
            st["out"] = [torch.empty(c["T"], c["H"], c["D"], dtype=torch.float16, device=dev) for _ in range(2)]
            sh = _shape(c)
            st["call"] = attn.prepare_append4(sh, nb, 0, cache, kv[0], kv[1], slots, status)
            st["read"] = attn.prepare_read4(sh, nb, 0, cache, slots, st["out"][0], st["out"][1], status)
        return st
    if c["op"] == "decode":
        lens = _lengths(c["median"], c["sigma"], c["R"], c["clip"])
        bt, nb, _ = _tables(lens, c["bs"], seed)
        cache = torch.randint(0, 256, _dims(c, nb), generator=g, device=dev, dtype=torch.uint8)
        rows = _by_slot(cache, c["order"])
        # pairs (A, B) of groups around zero, a few wider ones among them
        dims = rows.shape[:-1] + (4,)
        A = (0.15 + 0.25 * torch.rand(dims, generator=g, device=dev)).half()
        B = (-(64 + 7.5 + 2 * torch.randn(dims, generator=g, device=dev)) * A).half()
        pairs = torch.stack([A, B], -1).reshape(rows.shape[:-1] + (8,))
        # slots past a context's end hold what was there before: here NaN
        bt_d = torch.tensor(bt, device=dev)
        tail = torch.tensor(lens % c["bs"], device=dev)
        last = bt_d[torch.arange(c["R"], device=dev), torch.tensor(-(-lens // c["bs"]) - 1, device=dev)].long()
        stale = (torch.arange(c["bs"], device=dev)[None] >= tail[:, None]) & (tail[:, None] > 0)
        pairs[:, last] = pairs[:, last].masked_fill(stale[None, :, :, None, None], float("nan"))
        rows[..., c["D"] // 2:] = pairs.view(torch.uint8)
        q = torch.randn(c["R"], c["H"] * c["G"], c["D"], generator=g, device=dev).to(DT[c["dtype"]])
        st |= {"cache": cache, "table": bt_d, "lens": torch.tensor(lens, dtype=torch.int32, device=dev), "q": q, "nb": nb, "most": int(lens.max())}
        if own:
            from paper_2606_17787_amd import attn
            sh = _shape(c)
            st["out"] = torch.empty_like(q)
            st["ws"] = attn.new_decode4_workspace(sh, c["R"], c["H"] * c["G"], dev)
            st["call"] = attn.prepare_decode4(sh, nb, 0, cache, bt_d, st["lens"], q, st["out"], st["ws"], status)
        return st
    nq, nk = _prompt_lengths(c)
    cu = [torch.tensor(np.concatenate([[0], np.cumsum(n)]), dtype=torch.int32, device=dev) for n in (nq, nk)]
    # q, k and v as one projection writes them: q and the new tokens' k and v
    # are read in place, through their strides, where there is no prefix
    Hq, H = c["H"] * c["G"], c["H"]
    if c["prefix"]:
        q = torch.randn(int(nq.sum()), Hq, c["D"], generator=g, device=dev).to(DT[c["dtype"]])
        k, v = ((torch.randn(int(nk.sum()), H, c["D"], generator=g, device=dev)).to(DT[c["dtype"]]) for _ in range(2))
    else:
        qkv = torch.randn(int(nq.sum()), Hq + 2 * H, c["D"], generator=g, device=dev).to(DT[c["dtype"]])
        q, k, v = qkv[:, :Hq], qkv[:, Hq:Hq + H], qkv[:, Hq + H:]
    st |= {"q": q, "k": k, "v": v, "cu_q": cu[0], "cu_k": cu[1]}
    if own:
        from paper_2606_17787_amd import attn
        st["out"] = torch.empty(q.shape, dtype=q.dtype, device=dev)
        st["call"] = attn.prepare_prompt(q, k, v, st["out"], cu[0], status, cu_k=cu[1] if c["prefix"] else None)
    return st


# ------------------------------------------------------------- the plain forms

def _values(rows, D):
    """The values that rows of the 4-bit cache stand for, in 32 bits."""
    codes = rows[..., :D // 2]
    q = torch.stack([codes & 15, codes >> 4], -1).reshape(rows.shape[:-1] + (4, D // 4)).float()
    ab = rows[..., D // 2:].contiguous().view(torch.float16).float().reshape(rows.shape[:-1] + (4, 2))
    x = ab[..., 0:1] * (q + 64) + ab[..., 1:2]
    return x.half().float().reshape(rows.shape[:-1] + (D,))


def _quantised(x):
    """Rows of the 4-bit cache for x [..., D]."""
    D = x.shape[-1]
    y = x.float().clamp(-6848.0, 6848.0).reshape(x.shape[:-1] + (4, D // 4))
    lo, hi = y.amin(-1, keepdim=True), y.amax(-1, keepdim=True)
    A = ((hi - lo) * (1 / 15)).half().float()
    B = (lo - 64 * A).half().float()
    q = ((y - (B + 64 * A)) * (1 / torch.where(A > 0, A, torch.ones_like(A)))).round().clamp(0, 15)
    q = (q * (A > 0)).to(torch.uint8).reshape(x.shape)
    codes = q[..., 0::2] | (q[..., 1::2] << 4)
    ab = torch.stack([A, B], -1).half().reshape(x.shape[:-1] + (8,)).view(torch.uint8)
    return torch.cat([codes, ab], -1)


def _plain_slots(st):
    bs, R = st["case"]["bs"], st["case"]["R"]
    start, end, table, free = st["start"].long(), st["end"].long(), st["table"], st["free"]
    n = end - start
    cu = torch.cat([n.new_zeros(1), n.cumsum(0)])
    first, last = (start + bs - 1) // bs, (end + bs - 1) // bs
    need = last - first
    base = need.cumsum(0) - need
    granted = (need == 0) | (base + need <= st["count"])
    j = torch.arange(table.shape[1], device=table.device)[None] - first[:, None]
    fresh = (j >= 0) & (j < need[:, None]) & granted[:, None]
    at = (st["count"] - 1 - base[:, None] - j).clamp(0, len(free) - 1)
    table = torch.where(fresh, free[at], table)
    tok = torch.arange(st["T"], device=table.device)
    req = torch.searchsorted(cu[1:].contiguous(), tok, right=True).clamp(max=R - 1)
    pos = start[req] + tok - cu[req]
    slots = torch.where(granted[req], table[req, pos // bs].long() * bs + pos % bs, -1)
    lens = torch.where(granted, end, start)
    return {"table": table, "slots": slots, "cu": cu.int(), "lens": lens.int(), "left": st["count"] - (need * granted).sum()}


def _plain_append(st):
    c = st["case"]
    rows = _by_slot(st["cache"], c["order"])
    block, at = st["slots"] // c["bs"], st["slots"] % c["bs"]
    out = {}
    for i, name in enumerate(("k", "v")):
        rows[i, block, at] = _quantised(st[name])
        out[name] = _values(rows[i, block, at], c["D"]).half()
    return out


def _plain_decode(st):
    c = st["case"]
    rows = _by_slot(st["cache"], c["order"])
    pos = torch.arange(st["most"], device=rows.device)
    live = pos[None] < st["lens"][:, None]
    block = torch.where(live, st["table"][:, pos // c["bs"]], 0).long()
    at = (pos % c["bs"])[None].expand_as(block)
    q = st["q"].float().reshape(c["R"], c["H"], c["G"], c["D"]) * c["D"] ** -0.5
    k = _values(rows[0, block, at], c["D"]).permute(0, 2, 3, 1).contiguous()
    s = torch.matmul(q, k).masked_fill(~live[:, None, None], float("-inf"))
    del k
    p = torch.exp(s - s.amax(-1, keepdim=True))
    v = _values(rows[1, block, at], c["D"]).masked_fill(~live[:, :, None, None], 0.0)
    o = torch.matmul(p, v.transpose(1, 2).contiguous()) / p.sum(-1, keepdim=True)
    return o.reshape(st["q"].shape).to(st["q"].dtype)


def _plain_prompt(st):
    c = st["case"]
    q, k, v = (st[n].float().transpose(0, 1) for n in ("q", "k", "v"))
    k, v = (x.repeat_interleave(c["G"], 0) for x in (k, v))
    cu_q, cu_k = st["cu_q"].long(), st["cu_k"].long()
    i, j = (torch.arange(x.shape[1], device=x.device) for x in (q, k))
    seq_i, seq_j = torch.searchsorted(cu_q[1:], i, right=True), torch.searchsorted(cu_k[1:], j, right=True)
    # a query sees the keys of its sequence up to its own, from the end
    behind_i, behind_j = cu_q[1:][seq_i] - i, cu_k[1:][seq_j] - j
    hidden = (seq_i[:, None] != seq_j[None]) | (behind_j[None] < behind_i[:, None])
    s = torch.matmul(q * c["D"] ** -0.5, k.transpose(1, 2).contiguous()).masked_fill_(hidden, float("-inf"))
    p = s.sub_(s.amax(-1, keepdim=True)).exp_()
    o = torch.matmul(p, v) / p.sum(-1, keepdim=True)
    return o.transpose(0, 1).to(st["q"].dtype)


_PLAIN = {"slots": _plain_slots, "append": _plain_append, "decode": _plain_decode, "prompt": _plain_prompt}


def run(state):
    op = state["case"]["op"]
    if not own:
        return _PLAIN[op](state)
    state["call"]()
    if op == "slots":
        return {n: state[n] for n in ("table", "slots", "cu", "lens", "left")}
    if op == "append":
        state["read"]()
        return {"k": state["out"][0], "v": state["out"][1]}
    return state["out"]


# ------------------------------------------------------------------ in 64 bits

def _exact_values(rows, D):
    lo, hi = rows[..., :D // 2] % 16, rows[..., :D // 2] // 16
    q = torch.empty(rows.shape[:-1] + (D,), dtype=torch.float64, device=rows.device)
    q[..., 0::2], q[..., 1::2] = lo.double(), hi.double()
    ab = rows[..., D // 2:].contiguous().view(torch.float16).double()
    x = ab[..., 0::2].repeat_interleave(D // 4, -1) * (64 + q) + ab[..., 1::2].repeat_interleave(D // 4, -1)
    return x.half().double()


def _attend(q, k, v, scale, hidden=None):
    """Attention of q [..., n, D] over k and v [..., m, D] in 64 bits."""
    s = torch.matmul(q, k.transpose(-1, -2)) * scale
    if hidden is not None:
        s[..., hidden] = -math.inf
    s = torch.exp(s - s.max(-1, keepdim=True).values)
    return torch.matmul(s, v) / s.sum(-1, keepdim=True)


def exact(case, seed):
    c, st = case, prepare(case, seed)
    if c["op"] == "slots":
        return None  # whole numbers only
    if c["op"] == "append":
        out = {}
        for name in ("k", "v"):
            x = st[name].double().clamp(-6848, 6848).reshape(c["T"], c["H"], 4, -1)
            low, high = x.min(-1).values, x.max(-1).values
            A = ((high - low) / 15).half().double()
            B = (low - 64 * A).half().double()
            first = (B + 64 * A)[..., None]
            q = torch.where(A[..., None] > 0, ((x - first) / A[..., None]).round(), 0.0).clamp(0, 15)
            out[name] = (A[..., None] * (64 + q) + B[..., None]).half().double().reshape(c["T"], c["H"], c["D"])
        return out
    if c["op"] == "decode":
        rows, out = _by_slot(st["cache"], c["order"]), []
        for r, n in enumerate(st["lens"].tolist()):
            t = torch.arange(n, device=rows.device)
            block, at = st["table"][r, t // c["bs"]].long(), t % c["bs"]
            k, v = (_exact_values(rows[i][block, at], c["D"]).transpose(0, 1) for i in (0, 1))
            o = _attend(st["q"][r].double().reshape(c["H"], c["G"], c["D"]), k, v, c["D"] ** -0.5)
            out.append(o.reshape(-1, c["D"]))
        return torch.stack(out)
    out = torch.empty(st["q"].shape, dtype=torch.float64, device=st["q"].device)
    cu_q, cu_k = st["cu_q"].tolist(), st["cu_k"].tolist()
    for r in range(c["R"]):
        a, b, e, f = cu_q[r], cu_q[r + 1], cu_k[r], cu_k[r + 1]
        row = torch.arange(b - a, device=out.device) + (f - e) - (b - a)
        hidden = torch.arange(f - e, device=out.device)[None] > row[:, None]
        for h in range(c["H"]):
            for n in range(h * c["G"], (h + 1) * c["G"]):
                out[a:b, n] = _attend(st["q"][a:b, n].double(), st["k"][e:f, h].double(), st["v"][e:f, h].double(), c["D"] ** -0.5, hidden)
    return out
