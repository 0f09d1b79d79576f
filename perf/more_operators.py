"""What the operators of 16-bit paged caches cost: K and V into their pages,
attention of new tokens over a paged cache (single tokens, a few, whole chunks),
the weights that places of the cache gather, and eviction down to a budget.

run() goes through one operator in its plain form (elementary torch operations
in 32 bits, rounded once at the end) or, where `own` is true, through the
framework's kernels.  exact() is the same from the definitions in 64 bits.

A request's places 0 .. n - 1 are the slots that its block table names, in order;
its m new tokens are the last m of them, and a new token sees the places up to its
own.  The ledger holds two words for every layer, block, head and slot of a block:
the weight that the place has gathered (a 32-bit float) and the position of its
token in the text.  Eviction keeps, for every layer, request and head, the `keep`
places that rank first: those with a position under `sinks` or not under `recent_from`
before all others, then by weight, then the lower place.  A kept place behind the
first `keep` moves into a place that was given up among them, both in their order.
"""
import math

import numpy as np
import torch

own = False

DT = {"bf16": torch.bfloat16, "fp16": torch.float16}


# ------------------------------------------------------------------- the cases

def listed():
    return [
        # The new tokens of a 256-request decode step, one layer of a
        # Llama-3-8B-shaped cache.
        dict(name="append-step-256", op="append", T=256, H=8, D=128, bs=16, order="NHD", dtype="bf16"),
        # A batch of prompts written into one layer (an odd number of tokens).
        dict(name="append-prompts-16411", op="append", T=16411, H=8, D=128, bs=16, order="NHD", dtype="bf16"),
        # Decode over a tiny cache: 8 requests of a few hundred tokens.
        # Latency is all there is.
        dict(name="attend-tiny-8", op="attend", R=8, H=2, G=2, D=64, bs=16, order="NHD", dtype="fp16", before=216, sigma=0.5, new=1, every=1),
        # The ordinary decode step: 256 requests around 2,048 tokens, 32 query
        # heads over 8 KV heads.
        dict(name="attend-step-256", op="attend", R=256, H=8, G=4, D=128, bs=16, order="NHD", dtype="bf16", before=2048, sigma=0.75, new=1, every=1),
        # Five drafted tokens a request checked at once, head-major pages of 32.
        dict(name="attend-drafts-64", op="attend", R=64, H=8, G=4, D=128, bs=32, order="HND", dtype="fp16", before=4096, sigma=0.5, new=5, every=1),
        # One tensor-parallel rank of a 70B-shaped model (one KV head, 8 query
        # heads): chunks of 512 prompt tokens beside the single tokens of the
        # other requests.
        dict(name="attend-mixed-tp8-96", op="attend", R=96, H=1, G=8, D=128, bs=16, order="NHD", dtype="bf16", before=2048, sigma=0.6, new=512, every=8),
        # A chunk of one long prompt behind what is in the cache already.
        dict(name="attend-chunk-2048", op="attend", R=1, H=8, G=4, D=128, bs=16, order="NHD", dtype="bf16", before=14336, sigma=0.0, new=2048, every=1),
        # The weights of a decode step's tokens.
        dict(name="weigh-step-256", op="weigh", R=256, H=8, G=4, D=128, bs=16, order="NHD", dtype="bf16", before=2048, sigma=0.75, new=1, every=1),
        # The last 32 queries of 16 prompts weigh the prompts' places.
        dict(name="weigh-window-16", op="weigh", R=16, H=8, G=4, D=128, bs=16, order="NHD", dtype="bf16", before=4096, sigma=0.5, new=32, every=1),
        # A chunk of a prompt weighs what is before it and itself.
        dict(name="weigh-chunk-2048", op="weigh", R=1, H=8, G=4, D=128, bs=16, order="NHD", dtype="bf16", before=6144, sigma=0.0, new=2048, every=1),
        # 64 requests at a budget of 2,048 places, 16 tokens over it, four
        # layers of a Llama-3-8B-shaped cache.
        dict(name="evict-steps-64", op="evict", L=4, R=64, H=8, D=128, bs=16, order="NHD", dtype="bf16", median=2064, sigma=0.0, keep=2048, sinks=4, recent=256),
        # 16 prompts around 8,192 tokens cut down to 1,024 places.
        dict(name="evict-prompts-16", op="evict", L=2, R=16, H=8, D=128, bs=16, order="NHD", dtype="bf16", median=8192, sigma=0.5, keep=1024, sinks=4, recent=64),
    ]


def _log(rng, lo, hi):
    """A whole number spread over the logarithm of [lo, hi], odd ones too."""
    return min(hi, max(lo, int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))))


def draw(rng):
    op = rng.choice(["append", "attend", "attend", "attend", "weigh", "weigh", "evict"])
    bs = rng.choice([8, 16, 16, 24, 32, 64])
    order = rng.choice(["NHD", "HND"])
    dtype = rng.choice(["bf16", "fp16"])
    if op == "append":
        H = rng.choice([1, 2, 4, 8])
        return dict(op=op, T=_log(rng, 1, 16384), H=H, D=rng.choice([64, 128, 128, 256]), bs=bs, order=order, dtype=dtype)
    if op == "evict":
        L, H, D = rng.choice([1, 2, 4]), rng.choice([1, 2, 4, 8]), rng.choice([64, 128, 128, 256])
        R = _log(rng, 1, 64)
        most = 500_000 * 8 * 128 // (L * R * H * D * 2)  # places of a request at the largest listed case's cost
        median = _log(rng, 2, max(3, min(32768, most)))
        keep = _log(rng, 1, median)
        return dict(op=op, L=L, R=R, H=H, D=D, bs=bs, order=order, dtype=dtype, median=median, sigma=0.5, keep=keep, sinks=rng.choice([0, 4]), recent=_log(rng, 1, keep))
    H, G, D = rng.choice([1, 2, 4, 8]), rng.choice([1, 2, 3, 4, 7, 8]), rng.choice([64, 128, 128])
    R = _log(rng, 1, 256)
    # the padded plain form and the products stay inside the largest listed cases
    most = 500_000 * 8 * 128 // (R * H * D * 3)
    before = _log(rng, 1, max(2, min(32768, most // 4)))
    room = 1_000_000_000 // (R * H * G * 3 * before)
    new = rng.choice([1, _log(rng, 1, max(2, min(32, room))), _log(rng, 1, max(2, min(2048, room, before)))])
    return dict(op=op, R=R, H=H, G=G, D=D, bs=bs, order=order, dtype=dtype, before=before, sigma=0.5, new=new, every=rng.choice([1, 1, 4]))


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


def _sizes(c):
    """(new tokens, places with them) of every request."""
    m = np.where(np.arange(c["R"]) % c["every"] == 0, c["new"], 1)
    return m, m + _lengths(c["before"], c["sigma"], c["R"], 4 * c["before"])


# -------------------------------------------------------------------- the work

def work(case):
    c = case
    if c["op"] == "append":
        n = c["T"] * c["H"]
        return {"bytes": 8 * n * c["D"] + 12 * c["T"] + 8 * n, "flops": 2 * n * c["D"]}
    if c["op"] == "evict":
        n = _lengths(c["median"], c["sigma"], c["R"], 4 * c["median"])
        given = np.maximum(n - c["keep"], 0)
        # what moves: about the kept share of the places behind the budget, and the last ones
        moved = np.minimum(given, np.minimum(given, c["recent"]) + np.maximum(given - c["recent"], 0) * c["keep"] // n)
        sets = c["L"] * c["H"]
        return {"bytes": sets * (8 * int(n[given > 0].sum()) + (8 * c["D"] + 16) * int(moved.sum())) + 16 * c["R"], "flops": sets * int(n.sum())}
    m, n = _sizes(c)
    pairs, rows = int((m * n - m * (m - 1) // 2).sum()), c["H"] * c["G"] * int(m.sum())
    if c["op"] == "attend":
        return {"bytes": 4 * c["D"] * (c["H"] * int(n.sum()) + rows) + 4 * rows, "flops": 4 * pairs * c["H"] * c["G"] * c["D"]}
    return {"bytes": c["H"] * int(n.sum()) * (2 * c["D"] + 8) + rows * (2 * c["D"] + 4), "flops": 2 * pairs * c["H"] * c["G"] * c["D"]}


# ------------------------------------------------------------------ the inputs

def _tables(rows, bs, seed, spare=1.05):
    """Block tables of fragmented pages for contexts of `rows` tokens, -1 past
    them, the number of blocks, and the blocks that stay free."""
    pages = -(-rows // bs)
    nb = int(pages.sum() * spare) + 8
    perm = np.random.RandomState(seed % (1 << 31)).permutation(nb).astype(np.int32)
    bt = np.full((len(rows), max(1, int(pages.max()))), -1, np.int32)
    at = 0
    for r, p in enumerate(pages):
        bt[r, :p] = perm[at:at + p]
        at += p
    return bt, nb, perm[at:]


def _cache(c, nb, g):
    L = c.get("L", 1)
    dims = (L, 2, nb, c["bs"], c["H"], c["D"]) if c["order"] == "NHD" else (L, 2, nb, c["H"], c["bs"], c["D"])
    x = torch.empty(dims, dtype=DT[c["dtype"]], device="cuda")
    for layer in range(L):
        for i in range(2):
            x[layer, i] = torch.randn(dims[2:], generator=g, device="cuda")
    return x


def _by_slot(cache, order):
    """A view of the cache as [layers, 2, blocks, block size, heads, head dim]."""
    return cache if order == "NHD" else cache.transpose(3, 4)


def _shape(c):
    from paper_2606_17787_amd.workloads import CacheShape
    return CacheShape(c.get("L", 1), c["H"], c["D"], c["bs"], c["order"], 2)


def _mass(g, dims):
    """Gathered weights: most places little, a few much, and equal ones among
    them (places that nothing has looked at yet hold 0)."""
    x = torch.exp(2 * torch.randn(dims, generator=g, device="cuda") - 4)
    x = torch.where(torch.rand(dims, generator=g, device="cuda") < 0.2, (x * 64).round() / 64, x)
    return x.masked_fill(torch.rand(dims, generator=g, device="cuda") < 0.05, 0.0)


def prepare(case, seed):
    c, dev = case, "cuda"
    g = torch.Generator(device=dev)
    g.manual_seed(seed)
    status = torch.zeros(1, dtype=torch.int32, device=dev)
    st = {"case": c, "status": status}
    if c["op"] == "append":
        nb = -(-c["T"] * 5 // (4 * c["bs"])) + 4
        slots = torch.randperm(nb * c["bs"], generator=g, device=dev)[:c["T"]]
        # k and v as one projection writes them: read in place, through their strides
        kv = torch.randn(c["T"], 2 * c["H"], c["D"], generator=g, device=dev).to(DT[c["dtype"]])
        k, v = kv[:, :c["H"]], kv[:, c["H"]:]
        pos = torch.randint(0, 1 << 20, (c["T"],), generator=g, device=dev, dtype=torch.int32)
        ledger = torch.randint(0, 1 << 20, (1, 2, nb, c["H"], c["bs"]), generator=g, device=dev, dtype=torch.int32)
        st |= {"cache": _cache(c, nb, g), "ledger": ledger, "k": k, "v": v, "slots": slots, "pos": pos, "nb": nb}
        if own:
            from paper_2606_17787_amd import paged
            st["call"] = paged.prepare_append(_shape(c), nb, 0, st["cache"], k, v, slots, status, ledger=ledger, positions=pos)
        return st
    if c["op"] == "evict":
        n = _lengths(c["median"], c["sigma"], c["R"], 4 * c["median"])
        bt, nb, free = _tables(n, c["bs"], seed)
        bt_d = torch.tensor(bt, device=dev)
        dims = (c["L"], nb, c["H"], c["bs"])
        fresh = torch.empty((c["L"], 2) + dims[1:], dtype=torch.int32, device=dev)
        fresh[:, 0] = _mass(g, dims).view(torch.int32)
        # positions of the tokens: in order, and mixed where eviction went before
        place = torch.arange(bt.shape[1] * c["bs"], device=dev)
        sign = torch.rand((c["L"], c["R"], c["H"], len(place)), generator=g, device=dev)
        sign = torch.where((place >= c["keep"]) | (place < c["sinks"]), place / len(place) + 2.0 * (place >= c["keep"]) - (place < c["sinks"]) * 1.0, sign)
        pos = torch.argsort(torch.argsort(sign, -1), -1).int()
        live = torch.tensor(bt >= 0, device=dev)
        pos = pos.reshape(c["L"], c["R"], c["H"], bt.shape[1], c["bs"]).transpose(2, 3)
        fresh[:, 1] = 0
        fresh[:, 1, bt_d[live].long()] = pos[:, live]
        lens = torch.tensor(n, dtype=torch.int32, device=dev)
        keep = torch.full((c["R"],), c["keep"], dtype=torch.int32, device=dev)
        room = torch.zeros(nb, dtype=torch.int32, device=dev)
        room[:len(free)] = torch.tensor(free, device=dev)
        st |= {"cache": _cache(c, nb, g), "fresh": fresh, "ledger": torch.empty_like(fresh), "table": bt_d, "lens": lens, "keep": keep,
               "recent_from": lens - c["recent"], "nb": nb, "free": room, "count": torch.tensor([len(free)], dtype=torch.int64, device=dev), "most": int(n.max())}
        if own:
            from paper_2606_17787_amd import paged
            sh = _shape(c)
            st["left"], st["now"] = torch.empty_like(lens), torch.empty_like(st["count"])
            st["ws"] = paged.new_evict_workspace(sh, c["R"], bt.shape[1], dev)
            st["call"] = paged.prepare_evict(sh, nb, st["cache"], st["ledger"], bt_d, lens, keep, st["recent_from"], st["left"], st["ws"], status, sinks=c["sinks"])
            st["back"] = paged.prepare_release(st["left"], lens, bt_d, c["bs"], nb, room, st["count"], st["now"], status)
        return st
    m, n = _sizes(c)
    bt, nb, _ = _tables(n, c["bs"], seed)
    cache = _cache(c, nb, g)
    bt_d = torch.tensor(bt, device=dev)
    # slots past a context's end hold what was there before: here NaN
    slots = _by_slot(cache, c["order"])
    tail = torch.tensor(n % c["bs"], device=dev)
    last = bt_d[torch.arange(c["R"], device=dev), torch.tensor(-(-n // c["bs"]) - 1, device=dev)].long()
    stale = (torch.arange(c["bs"], device=dev)[None] >= tail[:, None]) & (tail[:, None] > 0)
    slots[0][:, last] = slots[0][:, last].masked_fill(stale[None, :, :, None, None], float("nan"))
    # q as one projection writes it, beside k and v: read in place
    qkv = torch.randn(int(m.sum()), c["H"] * (c["G"] + 2), c["D"], generator=g, device=dev).to(DT[c["dtype"]])
    q = qkv[:, :c["H"] * c["G"]]
    cu = torch.tensor(np.concatenate([[0], np.cumsum(m)]), dtype=torch.int32, device=dev)
    lens = torch.tensor(n, dtype=torch.int32, device=dev)
    st |= {"cache": cache, "table": bt_d, "lens": lens, "cu": cu, "q": q, "nb": nb, "most": int(n.max()), "most_new": int(m.max())}
    if c["op"] == "weigh":
        # what the attention of these tokens gave beside its output
        st["lse"] = _plain_attend(st, values=False)
        st["ledger"] = torch.zeros(1, 2, nb, c["H"], c["bs"], dtype=torch.int32, device=dev)
        st["ledger"][:, 0] = _mass(g, (1, nb, c["H"], c["bs"])).view(torch.int32)
    if own:
        from paper_2606_17787_amd import paged
        sh = _shape(c)
        if c["op"] == "attend":
            st["out"] = torch.empty(q.shape, dtype=q.dtype, device=dev)
            st["lse"] = torch.empty(q.shape[:2], dtype=torch.float32, device=dev)
            st["call"] = paged.prepare_attend(sh, nb, 0, cache, bt_d, lens, cu, q, st["out"], status, max_new=st["most_new"], lse=st["lse"])
        else:
            st["call"] = paged.prepare_weigh(sh, nb, 0, cache, bt_d, lens, cu, q, st["lse"], st["ledger"], status, max_new=st["most_new"])
    return st


# ------------------------------------------------------------- the plain forms

def _plain_append(st):
    c = st["case"]
    rows = _by_slot(st["cache"], c["order"])[0]
    block, at = st["slots"] // c["bs"], st["slots"] % c["bs"]
    rows[0, block, at], rows[1, block, at] = st["k"], st["v"]
    st["ledger"][0, 0, block, :, at] = 0
    st["ledger"][0, 1, block, :, at] = st["pos"][:, None].expand(-1, c["H"])
    return {"cache": st["cache"], "ledger": st["ledger"]}


def _padded(st):
    """The requests side by side, padded to the longest: queries [R, H, m * G, D]
    in 32 bits, blocks and places in them [R, n], the packed token of each query
    [R, m], whether there is one, and the pairs that see each other [R, m, n]."""
    c = st["case"]
    cu, lens = st["cu"].long(), st["lens"].long()
    i, j = (torch.arange(x, device=cu.device) for x in (st["most_new"], st["most"]))
    m = cu[1:] - cu[:-1]
    there = i[None] < m[:, None]
    token = torch.where(there, cu[:-1, None] + i[None], 0)
    sees = (j[None, None] <= (i[None] + (lens - m)[:, None])[:, :, None]) & there[:, :, None]
    block = torch.where(j[None] < lens[:, None], st["table"][:, j // c["bs"]], 0).long()
    q = st["q"][token].float().reshape(c["R"], len(i), c["H"], c["G"], c["D"])
    q = q.permute(0, 2, 1, 3, 4).reshape(c["R"], c["H"], -1, c["D"])
    return q, block, (j % c["bs"])[None].expand_as(block), token, there, sees


def _plain_scores(st, q, block, at, sees):
    """Scores [R, H, m, G, n], -infinity where a query does not see a place."""
    c = st["case"]
    k = _by_slot(st["cache"], c["order"])[0, 0][block, at].float()
    k = k.permute(0, 2, 3, 1).contiguous()
    s = torch.matmul(q * c["D"] ** -0.5, k).reshape(c["R"], c["H"], sees.shape[1], c["G"], -1)
    return s.masked_fill_(~sees[:, None, :, None], float("-inf"))


def _packed(x, token, there):
    """[R, H, m, G, ...] back to packed tokens [T, H * G, ...]."""
    x = x.permute(0, 2, 1, 3, *range(4, x.dim()))[there]
    return x.reshape((x.shape[0], -1) + x.shape[3:])


def _plain_attend(st, values=True):
    c = st["case"]
    q, block, at, token, there, sees = _padded(st)
    s = _plain_scores(st, q, block, at, sees)
    top = s.amax(-1, keepdim=True)
    top = torch.where(torch.isfinite(top), top, 0.0)
    p = s.sub_(top).exp_()
    total = p.sum(-1, keepdim=True)
    lse = _packed((top + total.log())[..., 0], token, there)
    if not values:
        return lse
    v = _by_slot(st["cache"], c["order"])[0, 1][block, at].float()
    v = v.masked_fill_(~sees.any(1)[:, :, None, None], 0.0).transpose(1, 2).contiguous()
    o = torch.matmul(p.reshape(c["R"], c["H"], -1, p.shape[-1]), v).reshape(p.shape[:-1] + (c["D"],)) / total
    return {"out": _packed(o, token, there).to(st["q"].dtype), "lse": lse}


def _plain_weigh(st):
    c = st["case"]
    q, block, at, token, there, sees = _padded(st)
    s = _plain_scores(st, q, block, at, sees)
    lse = st["lse"][token].reshape(c["R"], -1, c["H"], c["G"]).transpose(1, 2)
    p = s.sub_(lse[..., None]).exp_().sum((2, 3))  # [R, H, n]
    mass = st["ledger"][0, 0].view(torch.float32)
    live = sees.any(1)
    b, o = block[live], at[live]
    mass[b, :, o] = mass[b, :, o] + p.transpose(1, 2)[live]
    return {"ledger": st["ledger"]}


def _plain_evict(st):
    c = st["case"]
    lens, keep, table = st["lens"].long(), st["keep"].long(), st["table"]
    j = torch.arange(st["most"], device=lens.device)
    live = j[None] < lens[:, None]
    block, at = torch.where(live, table[:, j // c["bs"]], 0).long(), (j % c["bs"])[None].expand(c["R"], -1)
    led = st["ledger"][:, :, block, :, at].permute(2, 3, 0, 4, 1)  # [L, 2, R, H, n]
    mass, pos = led[:, 0].contiguous().view(torch.float32), led[:, 1]
    # the order: protected places, the other ones by weight, those past the end
    first = (pos < c["sinks"]) | (pos >= st["recent_from"][None, :, None, None])
    kind = torch.where(live[None, :, None], torch.where(first, 0, 1), 2)
    order = torch.sort(mass, dim=-1, descending=True, stable=True).indices
    order = torch.gather(order, -1, torch.sort(torch.gather(kind, -1, order), dim=-1, stable=True).indices)
    rank = torch.empty_like(order).scatter_(-1, order, j.expand_as(order).contiguous())
    left = torch.minimum(lens, keep)
    kept = (rank < left[None, :, None, None]) & live[None, :, None]
    inside = j[None] < left[:, None]
    hole, source = ~kept & inside[None, :, None], kept & ~inside[None, :, None]
    to, frm = hole.nonzero(as_tuple=True), source.nonzero(as_tuple=True)  # in the same order, as many
    layer, r, h = to[:3]
    rows = _by_slot(st["cache"], c["order"])
    tb, ta, fb, fa = block[r, to[3]], at[r, to[3]], block[r, frm[3]], at[r, frm[3]]
    rows[layer, 0, tb, ta, h], rows[layer, 1, tb, ta, h] = rows[layer, 0, fb, fa, h], rows[layer, 1, fb, fa, h]
    st["ledger"][layer, :, tb, h, ta] = st["ledger"][layer, :, fb, h, fa]
    # the pages behind what is left
    first_page, end_page = -(-left // c["bs"]), -(-lens // c["bs"])
    p = torch.arange(table.shape[1], device=lens.device)
    back = table[(p[None] >= first_page[:, None]) & (p[None] < end_page[:, None])]
    free = st["free"].clone()
    place = st["count"] + torch.arange(len(back), device=lens.device)
    free[place] = back
    return {"cache": st["cache"], "ledger": st["ledger"], "left": left.int(), "free": free, "now": st["count"] + len(back)}


_PLAIN = {"append": _plain_append, "attend": _plain_attend, "weigh": _plain_weigh, "evict": _plain_evict}


def run(state):
    op = state["case"]["op"]
    if op == "evict":  # the weights and positions that the step has left
        state["ledger"].copy_(state["fresh"])
    if not own:
        out = _PLAIN[op](state)
    else:
        state["call"]()
        if op == "append":
            out = {n: state[n] for n in ("cache", "ledger")}
        elif op == "attend":
            out = {n: state[n] for n in ("out", "lse")}
        elif op == "weigh":
            out = {"ledger": state["ledger"]}
        else:
            state["back"]()
            out = {n: state[n] for n in ("cache", "ledger", "left", "free", "now")}
    if op in ("weigh", "evict"):  # the two halves of the ledger, each of its type
        led = out.pop("ledger")
        out["mass"], out["pos"] = led[:, 0].view(torch.float32), led[:, 1]
    return out


# ------------------------------------------------------------------ in 64 bits

def exact(case, seed):
    c = case
    if c["op"] in ("append", "evict"):
        return None  # words that move as they are, and whole numbers
    st = prepare(case, seed)
    cu, rows = st["cu"].tolist(), _by_slot(st["cache"], c["order"])[0]
    scale, G = c["D"] ** -0.5, c["G"]
    if c["op"] == "attend":
        out = torch.empty(st["q"].shape, dtype=torch.float64, device=st["q"].device)
        lse = torch.empty(st["q"].shape[:2], dtype=torch.float64, device=st["q"].device)
    else:
        mass = st["ledger"][:, 0].view(torch.float32).double()
    for r, n in enumerate(st["lens"].tolist()):
        a, b = cu[r], cu[r + 1]
        t = torch.arange(n, device=rows.device)
        block, at = st["table"][r, t // c["bs"]].long(), t % c["bs"]
        hidden = t[None] > torch.arange(b - a, device=rows.device)[:, None] + n - (b - a)
        for h in range(c["H"]):
            k, v = (rows[i][block, at, h].double() for i in (0, 1))
            for x in range(h * G, (h + 1) * G):
                s = torch.mm(st["q"][a:b, x].double(), k.t().contiguous()) * scale
                s[hidden] = -math.inf
                if c["op"] == "weigh":
                    mass[0, block, h, at] += torch.exp(s - st["lse"][a:b, x, None].double()).sum(0)
                else:
                    lse[a:b, x] = torch.logsumexp(s, -1)
                    out[a:b, x] = torch.mm(torch.exp(s - lse[a:b, x, None]), v)
    return {"out": out, "lse": lse} if c["op"] == "attend" else {"mass": mass, "pos": None}
