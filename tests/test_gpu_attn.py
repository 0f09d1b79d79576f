"""The serving operators on the GPU against plain references: slot maps, the
4-bit cache's append and read, decode and prompt attention."""
import math

import numpy as np
import pytest
import torch

import attn_ref as ref
import paper_2606_17787_amd.kvckpt as kv
from paper_2606_17787_amd import attn
from gpu_util import dev

pytestmark = pytest.mark.gpu

BF, FP = torch.bfloat16, torch.float16


def word(value=0):
    return torch.full((1,), value, dtype=torch.int32, device=dev())


def i32(a):
    return torch.tensor(np.asarray(a, np.int32), device=dev())


# ------------------------------------------------------------------ slots

def run_slots(start, end, table, bs, nb, free, count, num_slots, have=None):
    R = len(start)
    status = word()
    t = i32(table)
    cu, lens = i32(np.full(R + 1, -9)), i32(np.full(R, -9))
    left = torch.full((1,), -9, dtype=torch.int64, device=dev())
    out = torch.full((num_slots,), -9, dtype=torch.int64, device=dev())
    attn.lumen_attn_slots(
        i32(start), i32(end), t, bs, nb, i32(free),
        torch.tensor([count], dtype=torch.int64, device=dev()), out, cu, lens,
        left, status, have=None if have is None else i32(have))
    return (t.cpu().numpy(), out.cpu().numpy(), cu.cpu().numpy(),
            lens.cpu().numpy(), int(left), int(status))


def check_slots(*args, **kw):
    got, want = run_slots(*args, **kw), ref.slots(*args, **kw)
    for name, g, w in zip(("table", "slots", "cu", "lens", "left", "status"),
                          got, want):
        assert np.array_equal(g, w), name
    return want


def step(rng, R, bs, most_old, most_new, spare=0):
    start = rng.integers(0, most_old + 1, R)
    end = start + rng.integers(0, most_new + 1, R)
    pages = -(-start // bs)
    need = -(-end // bs) - pages
    nb = int(pages.sum() + need.sum()) + spare + 3
    ids = rng.permutation(nb).astype(np.int32)
    cols = int((-(-end // bs)).max(initial=0)) + 2
    table = np.full((R, cols), -1, np.int32)
    at = 0
    for r in range(R):
        table[r, :pages[r]] = ids[at:at + pages[r]]
        at += pages[r]
    return start, end, table, nb, ids[at:], int((end - start).sum())


@pytest.mark.parametrize("R", [1, 2, 63, 64, 65, 257, 1000, 4096])
@pytest.mark.parametrize("bs", [1, 16, 24])
def test_slots_random_steps(R, bs):
    rng = np.random.default_rng(100 * R + bs)
    old, new = (300, 40) if R <= 300 else (40, 9)
    start, end, table, nb, free, T = step(rng, R, bs, old, new)
    want = check_slots(start, end, table, bs, nb, free, len(free), T)
    assert want[5] == 0


def test_slots_single_tokens_and_none():
    rng = np.random.default_rng(5)
    start, end, table, nb, free, T = step(rng, 40, 16, 100, 0)
    assert T == 0
    check_slots(start, end, table, 16, nb, free, len(free), 0)
    check_slots(start, start + 1, np.pad(table, ((0, 0), (0, 1)),
                                         constant_values=-1), 16, nb + 64,
                np.concatenate([free, np.arange(nb, nb + 64)]), len(free) + 64,
                40)


def test_slots_padding_and_no_requests():
    rng = np.random.default_rng(6)
    start, end, table, nb, free, T = step(rng, 9, 16, 50, 30)
    check_slots(start, end, table, 16, nb, free, len(free), T + 1000)
    got = run_slots([], [], np.zeros((0, 4)), 16, 8, [1, 2], 2, 5)
    assert got[2].tolist() == [0] and got[4] == 2 and got[5] == 0
    assert got[1].tolist() == [-1] * 5


def test_slots_too_few_blocks_refuses_in_order():
    rng = np.random.default_rng(7)
    start, end, table, nb, free, T = step(rng, 300, 16, 60, 60)
    for count in (0, 1, 100, len(free) // 2, len(free) - 4):
        want = check_slots(start, end, table, 16, nb, free, count, T)
        assert want[5] == ref.CAPACITY


def test_slots_counts_outside_the_list_are_held():
    rng = np.random.default_rng(8)
    start, end, table, nb, free, T = step(rng, 20, 16, 60, 60)
    check_slots(start, end, table, 16, nb, free, 1 << 40, T)
    check_slots(start, end, table, 16, nb, free, -3, T)


def test_slots_bad_requests():
    rng = np.random.default_rng(9)
    start, end, table, nb, free, T = step(rng, 120, 16, 60, 60)
    start[3], end[7] = -1, start[7] - 2
    end[11] = 16 * table.shape[1] + 1  # past the table
    T = int(np.where((start >= 0) & (end >= start), end - start, 0).sum())
    want = check_slots(start, end, table, 16, nb, free, len(free), T)
    assert want[5] == ref.RANGE
    free = free.copy()
    free[-2], free[-5] = nb, -4
    table[20, 0] = -1
    start[20] = 0
    end[20] = 30
    have = np.maximum(start, 0)
    have[20] = 16  # its first page is said to be there, and is not
    T = int(np.where((start >= 0) & (end >= start), end - start, 0).sum())
    want = check_slots(start, end, table, 16, nb, free, len(free), T,
                       have=have)
    assert want[5] == ref.BLOCK_ID


def test_slots_have():
    """Slots of tokens whose pages are all there: nothing is taken."""
    rng = np.random.default_rng(10)
    start, end, table, nb, free, _ = step(rng, 50, 16, 200, 0)
    zero = np.zeros_like(start)
    T = int(start.sum())
    want = check_slots(zero, start, table, 16, nb, free, len(free), T,
                       have=start)
    assert want[5] == 0 and want[4] == len(free)
    # pages ahead of the first new token are taken with it
    check_slots(start, start + 40, np.pad(table, ((0, 0), (0, 4)),
                                          constant_values=-1), 16, nb + 999,
                np.arange(nb, nb + 900), 900, 2000, have=start // 2)


def test_slots_total_past_int32_is_held():
    big = np.full(4, (1 << 30) + 7)
    got = run_slots(np.zeros(4), big, np.zeros((4, 2)), 16, 8, [1], 1, 3)
    assert got[5] == ref.CAPACITY
    assert got[2].tolist() == [0, (1 << 30) + 7] + [(1 << 31) - 1] * 3
    assert got[1].tolist() == [-1] * 3


# --------------------------------------------------------- append and read

def caches(shape, nb, rng):
    """A cache of random bytes, and a [2, nb, bs, H, row] view of layer l."""
    n = shape.pool_elems(nb)
    cache = torch.from_numpy(rng.integers(0, 256, n, dtype=np.uint8)).to(dev())

    def rows(layer):
        c = cache.view(shape.pool_dims(nb))[layer]
        return c if shape.order == "NHD" else c.transpose(2, 3)
    return cache, rows


def some_kv(rng, T, H, D, dtype, seed_scale=1.0):
    x = torch.from_numpy(rng.standard_normal((T, H, D)).astype(np.float32))
    return (x * seed_scale).to(dtype).to(dev())


@pytest.mark.parametrize("dtype", [BF, FP])
@pytest.mark.parametrize("order", ["NHD", "HND"])
@pytest.mark.parametrize("T,H,D,bs", [(1, 1, 64, 16), (7, 3, 128, 16),
                                      (33, 2, 256, 8), (257, 8, 128, 1),
                                      (130, 5, 64, 24)])
def test_append_and_read_bit_exact(T, H, D, bs, order, dtype):
    rng = np.random.default_rng(T * D + H)
    nb = -(-T // bs) * 2 + 3
    sh = attn.cache_shape4(2, H, D, bs, order)
    cache, rows = caches(sh, nb, rng)
    before = cache.clone()
    k, v = some_kv(rng, T, H, D, dtype), some_kv(rng, T, H, D, dtype, 40.0)
    k[0, 0, :D // 4] = 1.25        # a quarter of one value: A is 0
    v[0, 0, D // 4:D // 2] = 0.0
    slots = torch.from_numpy(rng.permutation(nb * bs)[:T].astype(np.int64))
    slots = slots.to(dev())
    if T > 5:
        slots[5] = -1              # a padding token
    status = word()
    attn.lumen_attn_append4(sh, nb, 1, cache, k, v, slots, status)
    assert int(status) == 0
    live = (slots >= 0).cpu().numpy()
    block, pos = slots // bs, slots % bs
    got = rows(1)
    want = before.view(sh.pool_dims(nb)).clone()
    w1 = want[1] if order == "NHD" else want[1].transpose(2, 3)
    for i, x in enumerate((k, v)):
        q, A, B = ref.quantise(x.float().cpu().numpy())
        r = torch.from_numpy(ref.to_rows(q, A, B)).to(dev())
        w1[i, block[live], pos[live]] = r[live]
    # the rows are the format's, and nothing else of the cache has changed
    assert torch.equal(cache, want.reshape(-1))
    del got
    for odt in (FP, BF):
        ko, vo = (torch.full((T, H, D), 9.0, dtype=odt, device=dev())
                  for _ in range(2))
        attn.lumen_attn_read4(sh, nb, 1, cache, slots, ko, vo, status)
        assert int(status) == 0
        for o, x in ((ko, k), (vo, v)):
            q, A, B = ref.quantise(x.float().cpu().numpy())
            val = torch.from_numpy(ref.values(q, A, B)).to(dev())
            val[~torch.from_numpy(live).to(dev())] = 0
            assert torch.equal(o, val.to(odt))


def test_append_error_is_half_a_step():
    """Each value is within half a step of its quarter (and the 16-bit
    roundings of A, B and the value) of the element it stands for."""
    rng = np.random.default_rng(3)
    for dtype, scale in ((BF, 1.0), (FP, 1e-3), (BF, 900.0)):
        x = some_kv(rng, 200, 4, 128, dtype, scale)
        sh = attn.cache_shape4(1, 4, 128, 16)
        cache, _ = caches(sh, 13, rng)
        status = word()
        slots = torch.arange(200, device=dev())
        attn.lumen_attn_append4(sh, 13, 0, cache, x, x, slots, status)
        o = torch.empty_like(x, dtype=FP)
        attn.lumen_attn_read4(sh, 13, 0, cache, slots, o, o.clone(), status)
        y = x.double().reshape(200, 4, 4, 32)
        wide = y.amax(-1, keepdim=True) - y.amin(-1, keepdim=True)
        big = y.abs().amax(-1, keepdim=True)
        # half a step; A's rounding over 15 steps and 64 of B's, B's own
        # (it is at most 64 A + |lo|), and the value's
        step = wide / 15
        room = step / 2 + 2.0 ** -11 * (15 * step + 64 * step + big) + \
            2.0 ** -11 * big + 16 * 2.0 ** -25
        off = (o.double().reshape(y.shape) - y).abs()
        assert bool((off <= room).all())


def test_append_special_values():
    """Infinities saturate, elements past the limit too, a NaN makes its
    quarter NaN and no other, subnormal spreads collapse to one value."""
    sh = attn.cache_shape4(1, 1, 128, 16)
    cache = torch.zeros(sh.pool_elems(2), dtype=torch.uint8, device=dev())
    x = torch.randn(4, 1, 128, generator=torch.Generator().manual_seed(1))
    x[0, 0, 3], x[0, 0, 40] = float("inf"), float("-inf")
    x[1, 0, 70] = float("nan")
    x[2, 0, :32] *= 1e30
    x[3, 0] = torch.linspace(0, 1e-9, 128)
    x = x.to(BF).to(dev())
    status, slots = word(), torch.arange(4, device=dev())
    attn.lumen_attn_append4(sh, 2, 0, cache, x, x, slots, status)
    o = torch.empty(4, 1, 128, dtype=FP, device=dev())
    attn.lumen_attn_read4(sh, 2, 0, cache, slots, o, o.clone(), status)
    q, A, B = ref.quantise(x.float().cpu().numpy())
    want = torch.from_numpy(ref.values(q, A, B))
    o = o.cpu()
    assert torch.equal(torch.isnan(o), torch.isnan(want))
    assert torch.isnan(o[1, 0, 64:96]).all()
    assert int(torch.isnan(o).sum()) == 32
    assert torch.equal(torch.nan_to_num(o), torch.nan_to_num(want))
    assert abs(float(o[0, 0, 3]) - ref.KV4_MAX) <= 8
    assert int(status) == 0


def test_append_slots_past_the_pool():
    rng = np.random.default_rng(4)
    sh = attn.cache_shape4(1, 2, 64, 16)
    cache, _ = caches(sh, 4, rng)
    before = cache.clone()
    x = some_kv(rng, 3, 2, 64, BF)
    slots = torch.tensor([64, 1 << 40, -(1 << 40)], device=dev())
    status = word()
    attn.lumen_attn_append4(sh, 4, 0, cache, x, x, slots, status)
    assert int(status) == ref.BLOCK_ID and torch.equal(cache, before)
    status, o = word(), torch.ones(3, 2, 64, dtype=BF, device=dev())
    p = torch.ones_like(o)
    attn.lumen_attn_read4(sh, 4, 0, cache, slots, o, p, status)
    assert int(status) == ref.BLOCK_ID
    assert not o.any() and not p.any()


def test_append_strided_rows():
    """K and V as slices of one fused projection, and read back into slices."""
    rng = np.random.default_rng(11)
    sh = attn.cache_shape4(1, 4, 128, 16)
    cache, _ = caches(sh, 8, rng)
    qkv = some_kv(rng, 50, 24, 128, BF)
    k, v = qkv[:, 16:20], qkv[:, 20:]
    slots = torch.arange(100, 50, -1, device=dev())
    status = word()
    attn.lumen_attn_append4(sh, 8, 0, cache, k, v, slots, status)
    both = torch.zeros(50, 8, 128, dtype=FP, device=dev())
    attn.lumen_attn_read4(sh, 8, 0, cache, slots, both[:, :4], both[:, 4:],
                          status)
    for o, x in ((both[:, :4], k), (both[:, 4:], v)):
        want = ref.values(*ref.quantise(x.float().cpu().numpy()))
        assert np.array_equal(o.cpu().numpy(), want)


# --------------------------------------------------------------- decode

def decode_case(rng, lens, H, G, D, bs, order, dtype, layers=1, layer=0,
                nan_tail=True, scale=1.0):
    """Random 4-bit pages under a random table; the rest of the pool holds
    random bytes, among them NaN pairs."""
    lens = np.asarray(lens, np.int64)
    pages = -(-lens // bs)
    nb = int(pages.sum()) + 3
    ids = rng.permutation(nb)
    cols = max(1, int(pages.max(initial=0)))
    table = np.full((len(lens), cols), -1, np.int32)
    at = 0
    for r, p in enumerate(pages):
        table[r, :p] = ids[at:at + p]
        at += p
    sh = attn.cache_shape4(layers, H, D, bs, order)
    cache, rows = caches(sh, nb, rng)
    live = rows(layer)
    g = torch.Generator(device=dev()).manual_seed(int(rng.integers(1 << 30)))
    dims = live.shape[:-1] + (4,)
    A = (0.05 + 0.3 * torch.rand(dims, generator=g, device=dev())).half()
    B = ((torch.randn(dims, generator=g, device=dev()) - 71.5) * A).half()
    pairs = torch.stack([A, B], -1).reshape(live.shape[:-1] + (8,))
    if nan_tail:
        for r, n in enumerate(lens):
            if n % bs:
                pairs[:, table[r, n // bs], n % bs:] = float("nan")
    live[..., D // 2:] = pairs.view(torch.uint8)
    q = torch.randn(len(lens), H * G, D, generator=g, device=dev()) * scale
    return sh, nb, cache, rows, i32(table), i32(lens), q.to(dtype)


def decode_want(rows, table, lens, q, H, bs, scale, dtype):
    G, D = q.shape[1] // H, q.shape[2]
    out = torch.zeros(q.shape, dtype=torch.float64, device=dev())
    slack = torch.zeros_like(out)
    # weights rounded to no fewer bits than a 16-bit float's
    for r, n in enumerate(lens.tolist()):
        if n <= 0:
            continue
        t = torch.arange(n, device=dev())
        block, pos = table[r, t // bs].long(), t % bs
        for h in range(H):
            k, v = (ref.from_rows(rows[i][block, pos, h]) for i in (0, 1))
            o, s = ref.attend(q[r, h * G:(h + 1) * G].double(), k, v, scale,
                              torch.ones(G, n, dtype=torch.bool,
                                         device=dev()), 2.0 ** -11)
            out[r, h * G:(h + 1) * G] = o
            slack[r, h * G:(h + 1) * G] = s
    return out, slack


def check_decode(rng, lens, H, G, D, bs, order, dtype, scale=None, **kw):
    sh, nb, cache, rows, table, dl, q = decode_case(rng, lens, H, G, D, bs,
                                                    order, dtype, **kw)
    layer = kw.get("layer", 0)
    out = torch.full_like(q, 7.0)
    status = word()
    ws = attn.new_decode4_workspace(sh, len(lens), H * G)
    sc = D ** -0.5 if scale is None else scale
    want, slack = decode_want(rows(layer), table, dl, q, H, bs, sc, dtype)
    for _ in range(2):  # the workspace is ready for the next call
        attn.lumen_attn_decode4(sh, nb, layer, cache, table, dl, q, out, ws,
                                status, scale=scale)
        assert int(status) == 0
        ref.assert_close(out, want, slack, dtype)
    return sh, nb, cache, rows, table, dl, q, out


LENS = [0, 1, 2, 15, 16, 17, 31, 32, 33, 63, 64, 65, 127, 128, 129, 300, 1025]


@pytest.mark.parametrize("dtype", [BF, FP])
@pytest.mark.parametrize("order", ["NHD", "HND"])
@pytest.mark.parametrize("D", [64, 128, 256])
@pytest.mark.parametrize("H,G,bs", [(2, 2, 16), (1, 8, 32), (3, 1, 8),
                                    (2, 7, 24)])
def test_decode_lengths(H, G, bs, D, order, dtype):
    rng = np.random.default_rng(H * 100 + G * 10 + D)
    check_decode(rng, LENS, H, G, D, bs, order, dtype)


@pytest.mark.parametrize("G", [1, 3, 4, 12, 16, 17, 32, 71])
def test_decode_groups(G):
    rng = np.random.default_rng(G)
    check_decode(rng, [5, 100, 0, 64], 2, G, 128, 16, "NHD", BF)


@pytest.mark.parametrize("bs", [1, 2, 16, 48, 64, 128, 1000])
def test_decode_page_sizes(bs):
    rng = np.random.default_rng(bs)
    check_decode(rng, [1, 999, 1000, 1001, 77], 2, 4, 128, bs, "HND", FP)


@pytest.mark.parametrize("lens", [[20000], [1, 30011, 2], [5000] * 40,
                                  [3000, 1] * 100])
def test_decode_long_and_many(lens):
    """Keys split over workgroups, and more requests than workgroups."""
    rng = np.random.default_rng(len(lens))
    check_decode(rng, lens, 2, 4, 128, 16, "NHD", BF)


@pytest.mark.parametrize("order", ["NHD", "HND"])
@pytest.mark.parametrize("H", [3, 5, 6, 7, 9, 11, 12, 16, 24])
def test_decode_head_counts(H, order):
    """Workgroups of every number of heads that lie together, and head counts
    of which a workgroup takes a part."""
    rng = np.random.default_rng(H)
    check_decode(rng, [1, 700, 33, 1290, 0, 128], H, 2, 128, 16, order, BF)
    check_decode(rng, [40, 515], H, 1, 64, 24, order, FP)
    check_decode(rng, [300, 1, 77], H, 3, 256, 8, order, BF)


def test_decode_one_long_request_of_one_head():
    rng = np.random.default_rng(77)
    check_decode(rng, [120001], 1, 8, 64, 32, "HND", FP)


def test_decode_many_requests():
    rng = np.random.default_rng(78)
    lens = rng.integers(0, 40, 4096)
    check_decode(rng, lens, 1, 2, 64, 16, "NHD", BF)


def test_decode_layers_scale_and_sharp_scores():
    """A layer of several, a scale of its own, and queries so large that one
    key takes almost all of the weight."""
    rng = np.random.default_rng(12)
    check_decode(rng, [100, 1000], 2, 4, 128, 16, "HND", BF, layers=3, layer=2,
                 scale=0.02)
    check_decode(rng, [100, 1000], 2, 4, 128, 16, "NHD", BF, scale=3.0)


def test_decode_strided_queries():
    rng = np.random.default_rng(13)
    sh, nb, cache, rows, table, dl, q = decode_case(
        rng, [40, 300, 7], 2, 4, 128, 16, "NHD", BF)
    fused = torch.randn(3, 12, 128, device=dev()).to(BF)
    fused[:, :8] = q
    out, status = torch.empty_like(q), word()
    ws = attn.new_decode4_workspace(sh, 3, 8)
    attn.lumen_attn_decode4(sh, nb, 0, cache, table, dl, fused[:, :8], out,
                            ws, status)
    want, slack = decode_want(rows(0), table, dl, q, 2, 16, 128 ** -0.5, BF)
    ref.assert_close(out, want, slack, BF)


def test_decode_device_errors_leave_tokens_out():
    """Pages past the table and ids outside the pool are left out of the sum
    and recorded; a negative length is a request without tokens."""
    rng = np.random.default_rng(14)
    lens = [100, 90, 80, 64]
    sh, nb, cache, rows, table, dl, q = decode_case(
        rng, lens, 2, 4, 128, 16, "NHD", BF, nan_tail=False)
    ws = attn.new_decode4_workspace(sh, 4, 8)
    sc = 128 ** -0.5

    def want_without(r, dead):
        n = lens[r]
        t = torch.arange(n, device=dev())
        t = t[~torch.isin(t // 16, torch.tensor(dead, device=dev()))]
        block, pos = table[r, t // 16].long(), t % 16
        o = [ref.attend(q[r, h * 4:h * 4 + 4].double(),
                        *(ref.from_rows(rows(0)[i][block, pos, h])
                          for i in (0, 1)), sc,
                        torch.ones(4, len(t), dtype=torch.bool, device=dev()),
                        2.0 ** -11) for h in range(2)]
        return (torch.cat([x[0] for x in o]), torch.cat([x[1] for x in o]))

    bad = table.clone()
    bad[0, 2], bad[1, 0] = nb, -1
    bad[3, :] = -1
    out, status = torch.full_like(q, 7.0), word()
    attn.lumen_attn_decode4(sh, nb, 0, cache, bad, dl, q, out, ws, status)
    assert int(status) == ref.BLOCK_ID
    for r, dead in ((0, [2]), (1, [0]), (2, [])):
        ref.assert_close(out[r], *want_without(r, dead), BF)
    assert not out[3].any()
    # lengths past the table, and a negative one
    long = dl.clone()
    long[2], long[3] = 100000, -5
    out, status = torch.full_like(q, 7.0), word()
    attn.lumen_attn_decode4(sh, nb, 0, cache, table[:, :5].contiguous(), long,
                            q, out, ws, status)
    assert int(status) == ref.RANGE
    ref.assert_close(out[2], *want_without(2, []), BF)
    ref.assert_close(out[0], *want_without(0, [5, 6]), BF)
    assert not out[3].any()


def test_decode_offsets_past_32_bits():
    """A layer whose pages lie more than 4 GiB apart."""
    rng = np.random.default_rng(15)
    H, D, bs, nb = 8, 128, 16, 450_000
    sh = attn.cache_shape4(1, H, D, bs, "HND")
    assert sh.pool_elems(nb) // 2 > 1 << 32
    cache = torch.empty(sh.pool_elems(nb), dtype=torch.uint8, device=dev())
    n = 100
    ids = np.array([[nb - 1, 0, nb - 2, 449_000, 3, 440_001, nb - 7]])
    table, lens = i32(ids), i32([n])
    t = torch.arange(n, device=dev())
    slots = table[0, t // bs].long() * bs + t % bs
    k, v = some_kv(rng, n, H, D, BF), some_kv(rng, n, H, D, BF)
    status = word()
    attn.lumen_attn_append4(sh, nb, 0, cache, k, v, slots, status)
    ko, vo = torch.empty_like(k), torch.empty_like(v)
    attn.lumen_attn_read4(sh, nb, 0, cache, slots, ko, vo, status)
    for o, x in ((ko, k), (vo, v)):
        want = ref.values(*ref.quantise(x.float().cpu().numpy()))
        assert torch.equal(o, torch.from_numpy(want).to(dev()).to(BF))
    q = some_kv(rng, 1, 16, D, BF)
    out, ws = torch.empty_like(q), attn.new_decode4_workspace(sh, 1, 16)
    attn.lumen_attn_decode4(sh, nb, 0, cache, table, lens, q, out, ws, status)
    assert int(status) == 0
    rows = cache.view(sh.pool_dims(nb))[0].transpose(2, 3)
    want, slack = decode_want(rows, table, lens, q, H, bs, D ** -0.5, BF)
    ref.assert_close(out, want, slack, BF)


# --------------------------------------------------------------- prompt

def prompt_want(q, k, v, cu_q, cu_k, scale, p_unit):
    G = q.shape[1] // k.shape[1]
    out = torch.full(q.shape, 7.0, dtype=torch.float64, device=dev())
    slack = torch.zeros_like(out)
    for s in range(len(cu_q) - 1):
        a, b, e, f = cu_q[s], cu_q[s + 1], cu_k[s], cu_k[s + 1]
        i = torch.arange(b - a, device=dev())[:, None] + (f - e) - (b - a)
        seen = torch.arange(f - e, device=dev())[None] <= i
        for h in range(q.shape[1]):
            out[a:b, h], slack[a:b, h] = ref.attend(
                q[a:b, h].double(), k[e:f, h // G].double(),
                v[e:f, h // G].double(), scale, seen, p_unit)
    return out, slack


def check_prompt(nq, nk, H, G, D, dtype, scale=None, gap=0, seed=0,
                 fused=False, q_scale=1.0):
    """Sequences of nq queries and nk keys (None: the queries' tokens), with
    `gap` foreign tokens before each, NaN in the keys and values of those."""
    g = torch.Generator(device=dev()).manual_seed(seed)
    own = nk is None
    nk = nq if own else nk

    def spans(n):
        at, cu = 0, []
        for x in n:
            cu.append((at + gap, at + gap + x))
            at += gap + x
        return cu, at + gap
    sq, tq = spans(nq)
    sk, tk = spans(nk)
    if fused:
        x = torch.randn(tq, H * (G + 2), D, generator=g, device=dev()).to(dtype)
        q, k, v = x[:, :H * G], x[:, H * G:H * G + H], x[:, H * G + H:]
    else:
        q = (torch.randn(tq, H * G, D, generator=g, device=dev()) *
             q_scale).to(dtype)
        k, v = (torch.randn(tk, H, D, generator=g, device=dev()).to(dtype)
                for _ in range(2))
    out, status = torch.full(q.shape, 7.0, dtype=dtype, device=dev()), word()
    sc = D ** -0.5 if scale is None else scale
    p_unit = ref.UNIT[dtype]
    want = torch.full(q.shape, 7.0, dtype=torch.float64, device=dev())
    slack = torch.zeros_like(want)
    inside_k = torch.zeros(tk, dtype=torch.bool, device=dev())
    for a, b in sk:
        inside_k[a:b] = True
    if gap:
        k[~inside_k] = float("nan")
        v[~inside_k] = float("inf")
    for (a, b), (e, f) in zip(sq, sk):
        o, s = prompt_want(q[a:b], k[e:f], v[e:f], [0, b - a], [0, f - e], sc,
                           p_unit)
        want[a:b], slack[a:b] = o, s
    if gap:
        for (a, b), (e, f) in zip(sq, sk):
            attn.lumen_attn_prompt(q, k, v, out, i32([a, b]), status,
                                   cu_k=i32([e, f]), scale=scale)
    else:
        cu_q = [a for a, _ in sq] + [tq]
        cu_k = [a for a, _ in sk] + [tk]
        attn.lumen_attn_prompt(q, k, v, out, i32(cu_q), status,
                               cu_k=None if own else i32(cu_k), scale=scale)
    assert int(status) == 0
    ref.assert_close(out, want, slack, dtype)
    return out


SEQS = [1, 2, 0, 15, 16, 17, 31, 32, 33, 63, 64, 65, 127, 128, 129, 255, 256,
        257, 0, 300]


@pytest.mark.parametrize("dtype", [BF, FP])
@pytest.mark.parametrize("D", [64, 128])
@pytest.mark.parametrize("H,G", [(2, 1), (2, 2), (1, 3), (2, 4), (1, 7),
                                 (1, 8), (1, 12), (1, 16)])
def test_prompt_lengths(H, G, D, dtype):
    check_prompt(SEQS, None, H, G, D, dtype, seed=G)


@pytest.mark.parametrize("G", [1, 4, 8])
@pytest.mark.parametrize("nq,nk", [
    ([1, 1, 1], [1, 64, 1000]), ([5, 40, 130], [70, 41, 2000]),
    ([64, 32, 1], [0, 31, 0]), ([100, 257], [33, 200]),
    ([256, 0, 3], [4096, 9, 3])])
def test_prompt_suffixes_and_rows_that_see_nothing(nq, nk, G):
    check_prompt(nq, nk, 2, G, 128, BF, seed=G)
    check_prompt(nq, nk, 1, G, 64, FP, seed=G + 1)


@pytest.mark.parametrize("n", [1000, 2049, 4096])
def test_prompt_longer(n):
    check_prompt([n], None, 2, 4, 128, BF, seed=n)
    check_prompt([n, n // 3], None, 1, 1, 64, FP, seed=n)


def test_prompt_fused_projection():
    check_prompt([77, 300, 1, 128], None, 2, 4, 128, BF, fused=True)


def test_prompt_foreign_tokens_do_not_leak():
    """NaN and infinities in tokens beside a sequence's own, before and after
    it, leave its outputs alone, and no other row is written."""
    check_prompt([5, 64, 130], None, 1, 4, 128, BF, gap=40)
    check_prompt([5, 64, 130], [100, 64, 133], 2, 1, 64, FP, gap=3)


def test_prompt_scale_and_sharp_scores():
    check_prompt([300, 10], None, 2, 2, 128, BF, scale=0.013)
    check_prompt([300, 10], None, 2, 2, 128, BF, scale=2.0)
    # scores that rise along the keys, so that the running maximum moves
    check_prompt([700], None, 1, 4, 64, FP, q_scale=9.0)


def test_prompt_many_sequences():
    rng = np.random.default_rng(4)
    check_prompt([int(x) for x in rng.integers(0, 9, 700)], None, 1, 2, 64, BF)


def test_prompt_eight_wavefronts():
    """Long sequences of many heads, which take the larger workgroups: a mean
    of 2,048 queries and 131,072 rows."""
    check_prompt([2048], None, 16, 4, 64, BF, seed=1)
    check_prompt([2100, 0, 5500], [2200, 0, 5500], 2, 12, 128, FP, seed=2)


@pytest.mark.parametrize("nq,nk,H,G,D", [
    ([3], [9000], 1, 1, 128),          # one tile, many parts
    ([40, 1, 90], [5000, 2100, 0], 2, 4, 128),
    ([17, 64], [20011, 70], 1, 8, 64),
    ([1] * 70 + [33], [64] * 70 + [8000], 2, 3, 64)])
@pytest.mark.parametrize("dtype", [BF, FP])
def test_prompt_few_rows_of_long_keys(nq, nk, H, G, D, dtype):
    """Tiles whose keys are cut into parts, and joined."""
    check_prompt(nq, nk, H, G, D, dtype, seed=len(nq))


@pytest.mark.parametrize("H,G,D,dtype", [(2, 1, 64, BF), (1, 4, 128, FP),
                                         (2, 8, 128, BF), (1, 2, 64, FP)])
@pytest.mark.parametrize("nq,nk", [([70, 200], [70, 200]), ([33], [150]),
                                   ([5, 130], [6000, 130])])
def test_prompt_values_that_are_not_finite(H, G, D, dtype, nq, nk):
    """NaN and infinities among a sequence's own values reach the queries that
    see them, in their elements, and nothing else."""
    g = torch.Generator(device=dev()).manual_seed(sum(nk))
    q = torch.randn(sum(nq), H * G, D, generator=g, device=dev()).to(dtype)
    k, v = (torch.randn(sum(nk), H, D, generator=g, device=dev()).to(dtype)
            for _ in range(2))
    cu_q, cu_k = np.cumsum([0] + nq), np.cumsum([0] + nk)
    want, slack = prompt_want(q, k, v, cu_q, cu_k, D ** -0.5, ref.UNIT[dtype])
    # (sequence, key from its end, head, element, value)
    bad = [(s, back, h, e, x) for s in range(len(nq)) for h in range(H)
           for back, e, x in ((1, 3, "nan"), (2, 40, "inf"), (30, 63, "-inf"),
                              (31, 0, "nan"), (nk[s], D - 1, "inf"))
           if back <= nk[s]]
    for s, back, h, e, x in bad:
        key = nk[s] - back
        v[cu_k[s] + key, h, e] = float(x)
        first = max(0, key - (nk[s] - nq[s]))  # query that sees it
        rows = slice(int(cu_q[s]) + first, int(cu_q[s + 1]))
        heads = slice(h * G, h * G + G)
        want[rows, heads, e] += float(x)
    out, status = torch.full_like(q, 7.0), word()
    attn.lumen_attn_prompt(q, k, v, out, i32(cu_q), status, cu_k=i32(cu_k))
    assert int(status) == 0
    got, fine = out.double(), torch.isfinite(want)
    assert torch.equal(torch.isnan(got), torch.isnan(want))
    inf = torch.isinf(want)
    assert torch.equal(torch.isinf(got), inf)
    assert torch.equal(got[inf], want[inf])
    zero = torch.zeros_like(want)
    ref.assert_close(torch.where(fine, got, zero), torch.where(fine, want, zero),
                     torch.where(fine, slack, zero), dtype)


def test_prompt_many_small_weights():
    """One key far above 70,000 others whose weights are 2^-25 of it each: in
    fp16 they would round to 0."""
    n, D = 70001, 64
    q = torch.zeros(1, 1, D, dtype=FP, device=dev())
    k = torch.zeros(n, 1, D, dtype=FP, device=dev())
    v = torch.ones(n, 1, D, dtype=FP, device=dev())
    q[..., 0], k[7, :, 0], v[7] = 1.0, 25 * math.log(2), -1.0
    out, status = torch.empty_like(q), word()
    cu_q, cu_k = [0, 1], [0, n]
    attn.lumen_attn_prompt(q, k, v, out, i32(cu_q), status, cu_k=i32(cu_k),
                           scale=1.0)
    want, slack = prompt_want(q, k, v, cu_q, cu_k, 1.0, ref.UNIT[FP])
    assert int(status) == 0
    ref.assert_close(out, want, slack, FP)


def test_prompt_bad_bounds():
    g = torch.Generator(device=dev()).manual_seed(0)
    q = torch.randn(100, 4, 64, generator=g, device=dev()).to(BF)
    k, v = (torch.randn(100, 2, 64, generator=g, device=dev()).to(BF)
            for _ in range(2))
    want, slack = prompt_want(q[:20], k[:20], v[:20], [0, 20], [0, 20], 0.125,
                              ref.UNIT[BF])
    for cu in ([0, 20, 101], [0, 20, 10], [0, 20, -4], [0, 20, 1 << 30]):
        out, status = torch.full_like(q, 7.0), word()
        attn.lumen_attn_prompt(q, k, v, out, i32(cu), status)
        assert int(status) == ref.RANGE, cu
        ref.assert_close(out[:20], want, slack, BF)
        assert bool((out[20:] == 7.0).all())
    status = word()
    attn.lumen_attn_prompt(q, k, v, q.clone(), i32([0, 20]), status,
                           cu_k=i32([90, 101]))
    assert int(status) == ref.RANGE


def test_prompt_sequences_that_share_queries():
    """Bounds that go back and forth: more tiles than queries have room for.
    Every row is a sequence's or not written."""
    g = torch.Generator(device=dev()).manual_seed(3)
    n, m, H, G, D = 200, 9000, 1, 8, 64
    q = torch.randn(n, H * G, D, generator=g, device=dev()).to(BF)
    k, v = (torch.randn(m, H, D, generator=g, device=dev()).to(BF)
            for _ in range(2))
    want, slack = prompt_want(q, k, v, [0, n], [0, m], D ** -0.5, ref.UNIT[BF])
    out, status = torch.full_like(q, 7.0), word()
    attn.lumen_attn_prompt(q, k, v, out, i32([0, n] * 600), status,
                           cu_k=i32([0, m] * 600))
    assert int(status) == ref.RANGE
    written = (out != 7.0).any(-1, keepdim=True).expand_as(out)
    assert bool(written.any())
    seven, zero = torch.full_like(want, 7.0), torch.zeros_like(want)
    ref.assert_close(out, torch.where(written, want, seven),
                     torch.where(written, slack, zero), BF)


# ------------------------------------------------- streams, graphs, together

def test_calls_on_another_stream_and_in_a_graph():
    """One step (slots, append, decode) on a side stream and captured in a
    graph; each replay follows eager work that changes its inputs."""
    rng = np.random.default_rng(21)
    H, G, D, bs, R = 2, 4, 128, 16, 12
    sh = attn.cache_shape4(1, H, D, bs)
    start, end, table, nb, free, _ = step(rng, R, bs, 700, 0)
    table = np.pad(table, ((0, 0), (0, 2)), constant_values=-1)
    nb += 64
    free = np.concatenate([free, np.arange(nb - 64, nb, dtype=np.int32)])
    cache, rows = caches(sh, nb, rng)
    old = i32(start)
    dt, status = i32(table), word()
    ids, count = i32(free), torch.tensor([len(free)], device=dev())
    kv_in = [some_kv(rng, int(start.sum()), H, D, BF) for _ in range(2)]
    slots0 = torch.empty(int(start.sum()), dtype=torch.int64, device=dev())
    cu, lens = i32(np.zeros(R + 1)), i32(np.zeros(R))
    left = torch.zeros(1, dtype=torch.int64, device=dev())
    attn.lumen_attn_slots(i32(np.zeros(R)), old, dt, bs, nb, ids, count,
                          slots0, cu, lens, left, status, have=old)
    attn.lumen_attn_append4(sh, nb, 0, cache, *kv_in, slots0, status)
    new_end = old + 1
    slots1 = torch.empty(R, dtype=torch.int64, device=dev())
    k, v = (torch.zeros(R, H, D, dtype=BF, device=dev()) for _ in range(2))
    q = torch.zeros(R, H * G, D, dtype=BF, device=dev())
    out, ws = torch.empty_like(q), attn.new_decode4_workspace(sh, R, H * G)

    def one():
        attn.lumen_attn_slots(old, new_end, dt, bs, nb, ids, count, slots1,
                              cu, lens, left, status)
        attn.lumen_attn_append4(sh, nb, 0, cache, k, v, slots1, status)
        attn.lumen_attn_decode4(sh, nb, 0, cache, dt, lens, q, out, ws, status)

    def refill():
        for t in (k, v, q):
            t.copy_(torch.randn(t.shape, device=dev()))
        out.fill_(7.0)
        torch.cuda.synchronize()

    def check():
        torch.cuda.synchronize()
        assert int(status) == 0
        want, slack = decode_want(rows(0), dt, lens, q, H, bs, D ** -0.5, BF)
        ref.assert_close(out, want, slack, BF)

    side = torch.cuda.Stream()
    refill()
    with torch.cuda.stream(side):
        one()
    check()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        one()
    for _ in range(4):
        refill()
        graph.replay()
        check()


def test_prompt_in_a_graph():
    g = torch.Generator(device=dev()).manual_seed(3)
    cu = i32([0, 100, 100, 333])
    q = torch.zeros(333, 8, 128, dtype=BF, device=dev())
    k, v = (torch.zeros(333, 2, 128, dtype=BF, device=dev()) for _ in range(2))
    out, status = torch.empty_like(q), word()
    attn.lumen_attn_prompt(q, k, v, out, cu, status)
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        attn.lumen_attn_prompt(q, k, v, out, cu, status)
    for _ in range(3):
        for t in (q, k, v):
            t.copy_(torch.randn(t.shape, generator=g, device=dev()))
        out.fill_(7.0)
        torch.cuda.synchronize()
        graph.replay()
        torch.cuda.synchronize()
        want, slack = prompt_want(q, k, v, [0, 100, 100, 333],
                                  [0, 100, 100, 333], 128 ** -0.5,
                                  ref.UNIT[BF])
        ref.assert_close(out, want, slack, BF)
        assert int(status) == 0


def test_checkpoint_moves_a_4bit_cache():
    """pack and unpack move 4-bit rows into fresh pages, and decode over the
    restored cache gives the same bits."""
    rng = np.random.default_rng(31)
    lens = [1, 100, 333, 16]
    sh, nb, cache, rows, table, dl, q = decode_case(
        rng, lens, 2, 4, 128, 16, "NHD", BF, layers=2)
    ws = attn.new_decode4_workspace(sh, 4, 8)
    a, b, status = torch.empty_like(q), torch.empty_like(q), word()
    attn.lumen_attn_decode4(sh, nb, 0, cache, table, dl, q, a, ws, status)
    ck = torch.empty(sum(lens) * sh.token_row_elems, dtype=torch.uint8,
                     device=dev())
    zero = torch.zeros_like(dl)
    kv.lumen_kv_ckpt_pack_ranges(sh, nb, cache, table, zero, dl, ck, status)
    fresh = torch.full_like(cache, 255)
    moved = torch.where(table >= 0, (table + 5) % nb, table)
    kv.lumen_kv_ckpt_unpack_ranges(sh, nb, fresh, moved, zero, dl, ck, status)
    attn.lumen_attn_decode4(sh, nb, 0, fresh, moved, dl, q, b, ws, status)
    assert int(status) == 0 and torch.equal(a, b)
