"""The 16-bit paged cache's operators on the GPU against their definitions
(tests/paged_ref.py): append, attend, weigh, evict, release."""
import math

import numpy as np
import pytest
import torch

import paged_ref as ref
from attn_ref import UNIT
from paper_2606_17787_amd import paged
from paper_2606_17787_amd.workloads import CacheShape, HND, NHD
from gpu_util import dev

pytestmark = pytest.mark.gpu

BF, FP = torch.bfloat16, torch.float16


def word(value=0):
    return torch.full((1,), value, dtype=torch.int32, device=dev())


def i32(a):
    return torch.tensor(np.asarray(a, np.int32), device=dev())


def gen(seed):
    g = torch.Generator(device=dev())
    g.manual_seed(seed)
    return g


def new_cache(shape, nb, dtype, g):
    return torch.randn(shape.pool_elems(nb), generator=g,
                       device=dev()).to(dtype)


# ----------------------------------------------------------------- append

@pytest.mark.parametrize("D", [64, 128, 256])
@pytest.mark.parametrize("order,bs,H", [(NHD, 16, 8), (HND, 24, 3), (NHD, 1, 1),
                                        (HND, 32, 2)])
@pytest.mark.parametrize("T", [1, 37, 1000])
@pytest.mark.parametrize("ledger", [True, False])
def test_append(D, order, bs, H, T, ledger):
    g = gen(T * 7 + D)
    dtype = BF if T % 2 else FP
    sh = CacheShape(2, H, D, bs, order)
    nb = T // bs + 3
    cache = new_cache(sh, nb, dtype, g)
    led = torch.randint(-2 ** 31, 2 ** 31 - 1, paged.ledger_dims(sh, nb),
                        generator=g, device=dev(), dtype=torch.int32)
    kv = torch.randn(T, 2 * H + 1, D, generator=g, device=dev()).to(dtype)
    k, v = kv[:, :H], kv[:, H + 1:]
    slots = torch.randperm(nb * bs, generator=g, device=dev())[:T]
    if T > 4:
        slots[3] = -1
    pos = torch.randint(0, 2 ** 31 - 1, (T,), generator=g, device=dev(),
                        dtype=torch.int32)
    want, wl = cache.clone(), led.clone()
    rows = ref.by_slot(want, sh, nb)[1]
    at = slots >= 0
    b, o = slots[at] // bs, slots[at] % bs
    rows[0, b, o], rows[1, b, o] = k[at], v[at]
    if ledger:
        wl[1, 0, b, :, o] = 0
        wl[1, 1, b, :, o] = pos[at][:, None].expand(-1, H)
    status = word()
    paged.lumen_paged_append(sh, nb, 1, cache, k, v, slots, status,
                             ledger=led if ledger else None,
                             positions=pos if ledger else None)
    assert torch.equal(cache.view(torch.int16), want.view(torch.int16))
    assert torch.equal(led, wl)
    assert int(status) == 0


def test_append_slots_past_the_pool_and_no_tokens():
    sh = CacheShape(1, 2, 64, 16, NHD)
    cache = new_cache(sh, 2, BF, gen(1))
    want = cache.clone()
    k = torch.ones(3, 2, 64, dtype=BF, device=dev())
    status = word()
    paged.lumen_paged_append(sh, 2, 0, cache, k, k,
                             torch.tensor([32, 1 << 40, -5], device=dev()), status)
    assert torch.equal(cache, want) and int(status) == ref.BLOCK_ID
    status = word()
    paged.lumen_paged_append(sh, 2, 0, cache, k[:0], k[:0],
                             torch.zeros(0, dtype=torch.int64, device=dev()),
                             status)
    assert torch.equal(cache, want) and int(status) == 0


# ----------------------------------------------------------------- attend

class Case:
    """A cache with requests of n places, m of them new."""

    def __init__(self, n, m, H, G, D, bs=16, order=NHD, dtype=BF, seed=0,
                 spare=3, layers=1, cols=None, stale=True):
        rng, g = np.random.default_rng(seed), gen(seed)
        self.n, self.m = list(n), list(m)
        self.sh = CacheShape(layers, H, D, bs, order)
        self.table, self.nb = ref.tables(rng, self.n, bs, spare, cols)
        self.cache = new_cache(self.sh, self.nb, dtype, g)
        self.layer = layers - 1
        if stale:  # what no request's places hold is NaN
            used = np.zeros((self.nb, bs), bool)
            for r, x in enumerate(self.n):
                b, o, live = ref.places(self.table[r], x, bs, self.nb)
                used[b[live], o[live]] = True
            rows = ref.by_slot(self.cache, self.sh, self.nb)
            rows[:, :, torch.tensor(~used, device=dev())] = float("nan")
        T = int(sum(max(0, x) for x in self.m))
        qkv = torch.randn(T, H * G + 2 * H, D, generator=g, device=dev())
        self.q = qkv.to(dtype)[:, :H * G]
        self.cu = np.concatenate([[0], np.cumsum(self.m)]).astype(np.int32)

    def attend(self, max_new=None, scale=None, lse=True, **kw):
        status = word()
        out = torch.full(self.q.shape, 7.0, dtype=self.q.dtype, device=dev())
        l = torch.full(self.q.shape[:2], 7.0, device=dev()) if lse else None
        paged.lumen_paged_attend(
            self.sh, self.nb, self.layer, self.cache, i32(self.table),
            i32(self.n), i32(self.cu), self.q, out, status, max_new=max_new,
            lse=l, scale=scale, **kw)
        return out, l, int(status)

    def check(self, max_new=None, scale=None, what="", **kw):
        out, lse, status = self.attend(max_new, scale, **kw)
        want, slack, wl, lslack, written, ws = ref.attended(
            self.q, self.cache, self.sh, self.nb, self.table, self.n, self.cu,
            scale, self.layer, max_new)
        assert status == ws, what
        assert (out[~written] == 7.0).all() and (lse[~written] == 7.0).all()
        close(out[written], want[written], slack[written], UNIT[out.dtype], what)
        close(lse[written], wl[written], lslack[written], 0.0, what + " lse")
        return out, lse


def close(got, want, slack, unit, what=""):
    """Not finite where the definition is not, and else within slack and the
    output's own rounding (2^-24: fp16's subnormals)."""
    got = got.double()
    fine = torch.isfinite(want)
    assert torch.equal(torch.isnan(got), torch.isnan(want)), what
    both = ~fine & ~torch.isnan(want)
    assert torch.equal(got[both], want[both]), what
    room = slack + unit * (want.abs() + slack) + 2.0 ** -24
    off = (got - want).abs()
    bad = fine & ~(off <= room)
    assert not bool(bad.any()), (
        f"{what}: {int(bad.sum())} of {bad.numel()} too far: off by "
        f"{off[bad].max():.3g} where {room[bad].max():.3g} is allowed")


@pytest.mark.parametrize("dtype", [BF, FP])
@pytest.mark.parametrize("D", [64, 128])
@pytest.mark.parametrize("H,G,bs,order", [(8, 4, 16, NHD), (2, 1, 8, HND),
                                          (1, 8, 64, NHD), (3, 7, 24, HND),
                                          (2, 3, 1, NHD), (1, 2, 5, HND)])
def test_attend_single_tokens(dtype, D, H, G, bs, order):
    n = [1, 2, 15, 16, 17, 63, 64, 65, 100, 0, 255, 256, 257, 700]
    Case(n, [1] * len(n), H, G, D, bs, order, dtype, seed=G + bs).check(max_new=1)


@pytest.mark.parametrize("dtype", [BF, FP])
@pytest.mark.parametrize("D", [64, 128])
@pytest.mark.parametrize("H,G,bs,order", [(8, 4, 16, NHD), (2, 1, 8, HND),
                                          (1, 8, 64, NHD), (3, 7, 24, HND),
                                          (2, 3, 1, NHD), (1, 2, 5, HND)])
def test_attend_chunks(dtype, D, H, G, bs, order):
    """Whole prompts, suffixes, a few tokens, none, and more tokens than
    places."""
    n = [1, 40, 300, 129, 64, 0, 500, 3, 200, 1000, 31]
    m = [1, 40, 100, 128, 5, 0, 1, 9, 0, 33, 31]
    c = Case(n, m, H, G, D, bs, order, dtype, seed=G + bs)
    c.check()
    c.check(max_new=128)


@pytest.mark.parametrize("m", [1, 2, 3, 4, 5, 7, 8, 9, 16, 31, 32, 33])
@pytest.mark.parametrize("G", [1, 4, 8])
def test_attend_few_tokens(m, G):
    n = [m, m + 1, 64, 100 + m, 777, 1500]
    m = [min(m, x) for x in n]
    Case(n, m, 2, G, 128, seed=m[-1]).check(max_new=max(m))


@pytest.mark.parametrize("m", [1, 3, 100])
@pytest.mark.parametrize("R", [1, 2, 65, 300])
def test_attend_many_requests(R, m):
    rng = np.random.default_rng(R)
    n = rng.integers(0, 600 if R < 100 else 150, R)
    new = np.minimum(rng.integers(0, m + 1, R), n)
    Case(n, new, 2, 2, 64, seed=R, dtype=FP).check(max_new=m)


@pytest.mark.parametrize("n,m", [([20000], [1]), ([20000], [4]), ([9000], [300]),
                                 ([9000, 5, 4000], [1, 1, 1]),
                                 ([9000, 700, 4000, 3000], [1, 200, 2, 70]),
                                 ([3000], [3000])])
@pytest.mark.parametrize("H,G", [(1, 8), (8, 4)])
def test_attend_long(n, m, H, G):
    """Places that are cut into parts, which are joined."""
    Case(n, m, H, G, 128, seed=n[0]).check(max_new=max(m))


@pytest.mark.parametrize("max_new", [1, 60])
def test_attend_bad_requests_and_pages(max_new):
    c = Case([300, 200, 100, 80, 50, 400, 90, 64, 128], [1] * 9, 2, 4, 128,
             seed=5, cols=20, dtype=FP)
    c.n[1] = -3  # counts as 0
    c.table[2, 1] = -1
    c.table[2, 3] = c.nb
    c.table[3] = -1  # no place of it counts
    c.n[5] = 400  # past the 20 pages of a table row
    c.check(max_new=max_new)
    c.table[:] = -1
    c.check(max_new=max_new)


@pytest.mark.parametrize("m", [1, 9, 70])
@pytest.mark.parametrize("dead", [(2,), (3,), (2, 3), (0, 3), (1,), (4, 7, 11)])
@pytest.mark.parametrize("bs", [16, 8, 5])
def test_attend_and_weigh_with_dead_pages_anywhere(m, dead, bs):
    """Places of every part of a step left out, and counted ones around them."""
    c = Case([200, 130], [m, m], 2, 4, 128, bs, seed=5, dtype=FP)
    for page in dead:
        c.table[0, page * 16 // bs] = -1
        c.table[1, page % 8 * 16 // bs] = c.nb + 7
    c.check(max_new=m)
    check_weigh(c, max_new=m)


def test_attend_skips_requests_with_bad_bounds():
    c = Case([300, 200, 100, 80, 50], [3, 60, 7, 0, 4], 2, 4, 128, seed=6)
    c.check(max_new=59)  # the second has too many: skipped
    for at, value in ((1, -1), (2, 1000), (3, 2)):
        d = Case([300, 200, 100, 80, 50], [3, 60, 7, 0, 4], 2, 4, 128, seed=6)
        d.cu[at] = value
        out, lse, status = d.attend()
        assert status == ref.RANGE
    c = Case([10, 20], [2, 3], 2, 4, 128, seed=6)
    c.cu[:] = [1, 3, 4]  # the first and last tokens are in no request
    c.check()


def test_attend_without_lse_without_requests_or_tokens():
    c = Case([300, 20], [5, 1], 2, 4, 128, seed=7)
    want, _, _ = c.attend()
    assert torch.equal(c.attend(lse=False)[0], want)
    Case([], [], 2, 4, 128).check()
    Case([5, 9], [0, 0], 2, 4, 128).check()
    # no pages at all
    c = Case([0, 0], [2, 1], 2, 4, 128)
    c.table = np.zeros((2, 0), np.int32)
    c.check()


@pytest.mark.parametrize("n,m,H,G", [([5000], [4100], 16, 1),
                                     ([2100, 2300], [2100, 2200], 16, 2),
                                     ([9000], [2050], 4, 8)])
@pytest.mark.parametrize("dtype", [BF, FP])
def test_attend_large_tiles(n, m, H, G, dtype):
    """Rows enough for workgroups of eight wavefronts."""
    Case(n, m, H, G, 128, seed=n[0], dtype=dtype).check(max_new=max(m))


@pytest.mark.parametrize("dtype", [BF, FP])
def test_attend_large_tiles_with_values_that_are_not_finite(dtype):
    c = Case([4200], [4100], 16, 1, 128, dtype=dtype, seed=2)
    base, _, _ = c.attend()
    rows = ref.by_slot(c.cache, c.sh, c.nb)
    j = 3000  # seen by the last 1,200 queries
    rows[0, 1, int(c.table[0, j // 16]), j % 16, 3, 9] = float("inf")
    got, _, _ = c.attend()
    want = base.clone()
    want[j - 100:, 3, 9] = float("inf")
    assert torch.equal(got, want)


@pytest.mark.parametrize("dtype", [BF, FP])
@pytest.mark.parametrize("m", [1, 5, 70])
def test_attend_hidden_values_that_are_not_finite(dtype, m):
    """Infinities and NaN in places after a query's own do not reach it."""
    n = [200, 90, 64]
    c = Case(n, [m] * 3 if m < 64 else [70, 70, 64], 2, 4, 128, dtype=dtype,
             seed=8)
    base, base_lse, _ = c.attend()
    rows = ref.by_slot(c.cache, c.sh, c.nb)
    for r, x in enumerate(n):
        for back, bad in ((1, "nan"), (2, "inf"), (4, "-inf"), (40, "nan")):
            if back > c.m[r]:
                continue
            j = x - back
            b, o = int(c.table[r, j // 16]), j % 16
            rows[0, :, b, o] = float(bad)  # K and V
    got, got_lse, _ = c.attend()
    for r, x in enumerate(n):
        a = c.cu[r]
        first = min([b for b in (40, 4, 2, 1) if b <= c.m[r]][:1] or [0])
        clean = c.m[r] - first
        assert torch.equal(got[a:a + clean], base[a:a + clean])
        assert torch.equal(got_lse[a:a + clean], base_lse[a:a + clean])
        assert torch.isnan(got[a + clean:a + c.m[r]]).all()


@pytest.mark.parametrize("dtype", [BF, FP])
@pytest.mark.parametrize("m", [1, 6, 50])
@pytest.mark.parametrize("bad", ["inf", "-inf", "nan"])
def test_attend_seen_values_that_are_not_finite(dtype, m, bad):
    """A value that is not finite reaches every query that sees it, in its own
    element alone."""
    c = Case([150, 3000], [m, m], 2, 2, 64, dtype=dtype, seed=9)
    base, _, _ = c.attend()
    rows = ref.by_slot(c.cache, c.sh, c.nb)
    hit = 150 - (m + 1) // 2  # seen from the middle of the new tokens on
    rows[0, 1, int(c.table[0, hit // 16]), hit % 16, 1, 5] = float(bad)
    rows[0, 1, int(c.table[1, 3]), 2, 0, 63] = float(bad)
    got, _, _ = c.attend()
    want = base.clone()
    first = max(0, hit - (150 - m))
    want[first:m, 2:, 5] = float(bad)
    want[m:, :2, 63] = float(bad)
    assert torch.equal(got.isnan(), want.isnan())
    assert torch.equal(got.nan_to_num(9e3), want.nan_to_num(9e3))


@pytest.mark.parametrize("dtype", [BF, FP])
@pytest.mark.parametrize("m,n", [(1, 40), (1, 3000), (40, 40), (40, 3000)])
def test_attend_scores_that_are_not_finite(dtype, m, n):
    """NaN where the formula has it: a score of NaN or +infinity, or none but
    -infinity."""
    for value, rest in (("inf", 1.0), ("nan", 1.0), ("-inf", 1.0),
                        ("-inf", float("-inf"))):
        c = Case([n], [m], 1, 2, 64, dtype=dtype, seed=10)
        c.q[:] = c.q.abs() + 0.5  # an infinite key gives an infinite score
        rows = ref.by_slot(c.cache, c.sh, c.nb)
        for j in range(n):
            b, o = int(c.table[0, j // 16]), j % 16
            if j == n // 3:
                rows[0, 0, b, o, 0, 7] = float(value)
            elif rest != 1.0:
                rows[0, 0, b, o, 0, 7] = rest
        c.check(what=f"{value}, {rest}")


@pytest.mark.parametrize("scale", [1e-45, 1e-9, 1.0, 2e38])
@pytest.mark.parametrize("m", [1, 40])
def test_attend_of_zero_queries_is_the_mean(scale, m):
    c = Case([200, 1500], [m, m], 2, 2, 64, seed=11, dtype=FP)
    c.q[:] = 0
    c.check(scale=scale)


@pytest.mark.parametrize("m", [1, 40])
def test_attend_means_of_large_values_stay_finite(m):
    c = Case([1200], [m], 1, 4, 64, seed=12)
    c.q[:] = 0
    ref.by_slot(c.cache, c.sh, c.nb)[:, 1] = 2e36
    out, _, _ = c.attend()
    assert torch.isfinite(out).all()
    assert ((out.double() - 2e36).abs() <= 2e36 * 2.0 ** -7).all()


def test_attend_large_scores():
    """Scores of hundreds: one place has all the weight, and rising maxima."""
    c = Case([900, 70], [40, 3], 2, 4, 128, seed=13, dtype=FP)
    c.q *= 30
    c.check()


@pytest.mark.parametrize("dtype", [BF, FP])
@pytest.mark.parametrize("m", [1, 3, 60])
@pytest.mark.parametrize("n", [400, 16000])
@pytest.mark.parametrize("down", [9, 21, 23, 30])
def test_attend_many_small_weights_beside_a_large_one(dtype, m, n, down):
    """One place's score is `down` powers of two over all the others': their
    weights, some of which round to subnormals, count in the sum as in the
    products.  (The others' values are ones, the large one's are zeros.)"""
    c = Case([n], [m], 1, 2, 64, dtype=dtype, seed=1)
    c.q[:] = 0
    c.q[:, :, 0] = 1
    rows = ref.by_slot(c.cache, c.sh, c.nb)
    keep = rows.isfinite()
    rows[0, 0] = torch.where(keep[0, 0], 0.0, rows[0, 0])
    rows[0, 1] = torch.where(keep[0, 1], 1.0, rows[0, 1])
    b, o = int(c.table[0, 5]), 3
    rows[0, 0, b, o, 0, 0] = down
    rows[0, 1, b, o] = 0
    out, lse, _ = c.attend(scale=math.log(2.0))
    last = out[-1].double()
    rest = (n - 1) * 2.0 ** -down
    want = rest / (1 + rest)
    # a weight of 2^-down of the largest has an absolute rounding of at most
    # 2^-25 in fp16's subnormals, at 2^7 of them or more for the largest one
    lost = 2.0 ** (down - 32) if dtype == FP else 0.0
    assert ((last / want - 1).abs() <= 2 * UNIT[dtype] + lost + 2.0 ** -14).all()
    full = math.log(2.0) * down + math.log1p(rest)
    assert ((lse[-1].double() - full).abs() <= 2.0 ** -14 + 2.0 ** -22 * full).all()


def test_attend_repeats_itself():
    c = Case([4000, 3000, 100, 900, 7], [200, 1, 100, 3, 7], 2, 4, 128, seed=14)
    a, la, _ = c.attend()
    for _ in range(3):
        b, lb, _ = c.attend()
        assert torch.equal(a, b) and torch.equal(la, lb)


def test_attend_requests_share_pages():
    c = Case([300, 300], [5, 5], 2, 4, 128, seed=15, stale=False)
    c.table[1] = c.table[0]
    c.check()


# ------------------------------------------------------------------ weigh

def check_weigh(c, max_new=None, scale=None, window=None):
    """Weights of a call on a ledger with some; window: the last queries of
    each request alone."""
    H, bs = c.sh.num_kv_heads, c.sh.block_size
    _, lse, _ = c.attend(scale=scale)
    q, cu = c.q, c.cu
    if window:
        at = np.concatenate([np.arange(max(a, b - window), b)
                             for a, b in zip(cu[:-1], cu[1:])] or [[]])
        sel = torch.tensor(at.astype(np.int64), device=dev())
        q, lse = q[sel], lse[sel]
        cu = np.concatenate([[0], np.cumsum(np.minimum(np.diff(cu), window))])
    led = paged.new_ledger(c.sh, c.nb, dev())
    led.copy_(torch.rand(led.shape, generator=gen(3), device=dev())
              .view(torch.int32))
    before = led.clone()
    status = word()
    paged.lumen_paged_weigh(c.sh, c.nb, c.layer, c.cache, i32(c.table), i32(c.n),
                            i32(cu), q, lse, led, status, max_new=max_new,
                            scale=scale)
    start = paged.weights_of(before)[c.layer]
    want, slack = ref.weighed(q, lse, c.cache, c.sh, c.nb, c.table, c.n, cu,
                              start, scale, c.layer, max_new)
    got = paged.weights_of(led)[c.layer]
    close(got, want, slack, 0.0, "weights")
    same = slack == 0
    assert torch.equal(got[same & want.isfinite()],
                       start[same & want.isfinite()])
    led[c.layer, 0] = before[c.layer, 0]
    assert torch.equal(led, before)
    return int(status)


@pytest.mark.parametrize("dtype", [BF, FP])
@pytest.mark.parametrize("D", [64, 128])
@pytest.mark.parametrize("H,G,bs,order", [(8, 4, 16, NHD), (2, 1, 8, HND),
                                          (1, 8, 64, NHD), (3, 7, 24, HND),
                                          (2, 3, 1, NHD), (1, 2, 5, HND)])
def test_weigh(dtype, D, H, G, bs, order):
    n = [1, 40, 300, 129, 64, 0, 500, 3, 200, 1000, 31, 256, 257]
    m = [1, 40, 100, 128, 5, 0, 1, 9, 0, 33, 31, 1, 2]
    c = Case(n, m, H, G, D, bs, order, dtype, seed=G + bs)
    assert check_weigh(c) == 0
    assert check_weigh(c, max_new=8, window=8) == 0
    assert check_weigh(c, max_new=1, window=1) == 0


@pytest.mark.parametrize("n,m,H,G", [([5000], [1], 1, 8), ([3000], [900], 2, 4),
                                     ([1500], [1500], 1, 4),
                                     ([2000, 100], [64, 100], 8, 1)])
def test_weigh_long(n, m, H, G):
    check_weigh(Case(n, m, H, G, 128, seed=n[0]))


def test_weigh_single_tokens():
    rng = np.random.default_rng(4)
    n = rng.integers(0, 300, 130)
    check_weigh(Case(n, np.minimum(n, 1), 2, 4, 128, seed=4), max_new=1)


def test_weigh_bad_requests_and_pages():
    c = Case([300, 200, 100, 80, 50, 400, 90], [1, 30, 20, 5, 50, 1, 2], 2, 4,
             128, seed=5, cols=20)
    c.n[1] = -3
    c.table[2, 1] = -1
    c.table[2, 3] = c.nb
    c.table[3] = -1
    assert check_weigh(c) == ref.BLOCK_ID
    assert check_weigh(c, max_new=29) == ref.BLOCK_ID
    c = Case([300, 20], [3, 4], 2, 4, 128, seed=5)
    c.cu[2] = 1000
    led = paged.new_ledger(c.sh, c.nb, dev())
    status = word()
    lse = torch.zeros(c.q.shape[:2], device=dev())
    paged.lumen_paged_weigh(c.sh, c.nb, 0, c.cache, i32(c.table), i32(c.n),
                            i32(c.cu), c.q, lse, led, status)
    assert int(status) == ref.RANGE


def test_weigh_of_rows_that_saw_nothing_and_of_nan():
    c = Case([3, 100, 60], [5, 2, 1], 1, 2, 64, seed=6)
    check_weigh(c)  # the first two queries of the first request see nothing
    _, lse, _ = c.attend()
    lse[5, 0] = float("nan")
    led = paged.new_ledger(c.sh, c.nb, dev())
    paged.lumen_paged_weigh(c.sh, c.nb, 0, c.cache, i32(c.table), i32(c.n),
                            i32(c.cu), c.q, lse, led, word())
    w = paged.weights_of(led)[0]
    b, o, _ = ref.places(c.table[1], 100, 16, c.nb)
    nan = torch.zeros_like(w, dtype=torch.bool)
    nan[torch.tensor(b[:99]), 0, torch.tensor(o[:99])] = True
    assert torch.equal(w.isnan(), nan)


def test_weights_of_a_query_sum_to_one():
    c = Case([333], [1], 2, 4, 128, seed=7)
    _, lse, _ = c.attend()
    led = paged.new_ledger(c.sh, c.nb, dev())
    paged.lumen_paged_weigh(c.sh, c.nb, 0, c.cache, i32(c.table), i32(c.n),
                            i32(c.cu), c.q, lse, led, word())
    total = paged.weights_of(led).double().sum((0, 1, 3))
    # of a head's four queries: each weight is off by the errors of two scores at
    # most (attend's, in lse, and weigh's), some 2 D 2^-24 times the size of a score
    assert ((total - 4).abs() < 4 * 2.0 ** -12).all()


# ------------------------------------------------------------------ evict

class Evict:
    def __init__(self, n, keep, H=2, D=64, bs=16, order=NHD, layers=1, seed=0,
                 dtype=BF, sinks=2, recent=8, cols=None, kind="mixed"):
        rng, g = np.random.default_rng(seed), gen(seed)
        self.n, self.keep = list(n), list(keep)
        self.sh = CacheShape(layers, H, D, bs, order)
        self.table, self.nb = ref.tables(rng, self.n, bs, 3, cols)
        self.cache = new_cache(self.sh, self.nb, dtype, g)
        dims = (layers, self.nb, H, bs)
        w = rng.exponential(size=dims).astype(np.float32)
        if kind == "ties":
            w = np.floor(w * 2).astype(np.float32) * np.where(
                rng.random(dims) < 0.5, 1, -1).astype(np.float32)
        elif kind == "odd":
            w[rng.random(dims) < 0.2] = np.nan
            w[rng.random(dims) < 0.1] = np.inf
            w[rng.random(dims) < 0.1] = -np.inf
            w[rng.random(dims) < 0.1] = -0.0
            w[rng.random(dims) < 0.1] = 0.0
            w[rng.random(dims) < 0.1] *= -1
            w.reshape(-1)[::17] = -np.float32("nan")
        elif kind == "same":
            w[:] = 0
        self.led = np.zeros((layers, 2) + dims[1:], np.int32)
        self.led[:, 0] = w.view(np.int32)
        for r, x in enumerate(self.n):
            b, o, live = ref.places(self.table[r], x, bs, self.nb)
            for layer in range(layers):
                for h in range(H):
                    p = np.arange(len(b))
                    rng.shuffle(p)
                    self.led[layer, 1, b[live], h, o[live]] = p[live]
        self.sinks = sinks
        self.frm = np.array([x - recent for x in self.n], np.int32)

    def check(self, first=0, layers=None):
        want, wl = self.cache.cpu(), self.led.copy()
        left, ws = ref.evicted(want, wl, self.sh, self.nb, self.table, self.n,
                               self.keep, self.frm, self.sinks, first, layers)
        cache, led = self.cache.clone(), torch.tensor(self.led, device=dev())
        got, status = i32(np.full(len(self.n), -9)), word()
        paged.lumen_paged_evict(
            self.sh, self.nb, cache, led, i32(self.table), i32(self.n),
            i32(self.keep), i32(self.frm), got,
            paged.new_evict_workspace(self.sh, len(self.n),
                                      self.table.shape[1], dev()),
            status, sinks=self.sinks, first_layer=first, num_layers=layers)
        assert np.array_equal(got.cpu().numpy(), left)
        assert int(status) == ws
        assert np.array_equal(led.cpu().numpy(), wl)
        assert torch.equal(cache.cpu().view(torch.int16),
                           want.view(torch.int16))
        return ws


@pytest.mark.parametrize("kind", ["mixed", "ties", "odd", "same"])
@pytest.mark.parametrize("H,D,bs,order", [(2, 64, 16, NHD), (3, 128, 8, HND),
                                          (1, 256, 24, NHD), (2, 64, 1, HND)])
def test_evict(kind, H, D, bs, order):
    n = [100, 65, 64, 63, 1, 0, 300, 129, 40, 200, 17]
    keep = [50, 64, 64, 64, 0, 5, 1, 128, 39, 0, 3]
    Evict(n, keep, H, D, bs, order, seed=H + bs, kind=kind).check()


@pytest.mark.parametrize("sinks,recent", [(0, 0), (0, 1), (4, 30), (0, 1000),
                                          (1000, 0), (50, 60), (-3, -5)])
def test_evict_protected_places(sinks, recent):
    Evict([200, 90, 130], [60, 80, 4], seed=3, sinks=sinks,
          recent=recent).check()


def test_evict_layers():
    e = Evict([100, 40], [30, 20], layers=4, seed=4)
    e.check()
    e.check(first=1, layers=2)
    e.check(first=3)


@pytest.mark.parametrize("n,keep", [([5000], [4096]), ([5000], [4999]),
                                    ([9000, 100, 4500], [700, 90, 4400]),
                                    ([20000], [9000]), ([40000], [30000]),
                                    ([33000, 100], [5, 90]),
                                    ([2048], [2047]), ([4096], [1]),
                                    ([8192], [8000]), ([32768], [32767])])
@pytest.mark.parametrize("kind", ["mixed", "ties", "odd"])
def test_evict_long(n, keep, kind):
    Evict(n, keep, H=1, seed=5, kind=kind).check()


@pytest.mark.parametrize("D", [64, 128, 256])
@pytest.mark.parametrize("H,long", [(1, 120), (2, 120), (2, 3000), (2, 7000),
                                    (2, 20000)])
def test_evict_many_requests(H, long, D):
    """Few and many (layer, request, head), whose workgroups then move their
    places themselves; one of the requests longer than the others."""
    rng = np.random.default_rng(6)
    R = 300 if D == 64 else 256
    n = rng.integers(0, 120, R)
    n[7] = long
    keep = rng.integers(0, 100, R)
    keep[7] = long // 3
    Evict(n, keep, H=H, D=D, seed=6).check()


def test_evict_bad_requests():
    e = Evict([100, 60, 80, 50, 90, 70], [50, 20, 30, 10, 95, 20], seed=7,
              cols=6, recent=4)
    e.n[1] = -1
    e.keep[3] = -1
    assert e.check() == ref.RANGE
    e.table[2, 4] = -1
    e.table[4, 0] = e.nb  # of a request within its budget: not looked at
    assert e.check() == ref.BLOCK_ID
    e = Evict([100, 60], [50, 20], seed=8, cols=6)
    e.n[0] = 97  # past six pages of 16
    assert e.check() == ref.RANGE


def test_evict_twice_gives_what_once_gives():
    """What is left after a first call is all of a second one's budget."""
    e = Evict([300, 200], [100, 120], layers=2, seed=9)
    cache, led = e.cache.clone(), torch.tensor(e.led, device=dev())
    ws = paged.new_evict_workspace(e.sh, 2, e.table.shape[1], dev())
    left, again, status = i32([0, 0]), i32([0, 0]), word()
    paged.lumen_paged_evict(e.sh, e.nb, cache, led, i32(e.table), i32(e.n),
                            i32(e.keep), i32(e.frm), left, ws, status)
    c, l = cache.clone(), led.clone()
    paged.lumen_paged_evict(e.sh, e.nb, cache, led, i32(e.table), left,
                            i32(e.keep), i32(e.frm), again, ws, status)
    assert torch.equal(cache.view(torch.int16), c.view(torch.int16))
    assert torch.equal(led, l) and torch.equal(again, left)


# ---------------------------------------------------------------- release

def check_release(lens, have, table, bs, nb, free, count):
    want, now, ws = ref.released(lens, have, table, bs, nb, free, count)
    f, status = i32(free), word()
    got = torch.full((1,), -9, dtype=torch.int64, device=dev())
    paged.lumen_paged_release(
        i32(lens), i32(have), i32(table), bs, nb, f,
        torch.tensor([count], dtype=torch.int64, device=dev()), got, status)
    assert np.array_equal(f.cpu().numpy(), want)
    assert int(got) == now and int(status) == ws
    return ws


@pytest.mark.parametrize("R", [0, 1, 3, 64, 65, 300, 4096])
@pytest.mark.parametrize("bs", [1, 16, 24])
def test_release(R, bs):
    rng = np.random.default_rng(R + bs)
    have = rng.integers(0, 200 if R < 1000 else 60, R)
    lens = rng.integers(0, 200 if R < 1000 else 60, R)
    table, nb = ref.tables(rng, have, bs)
    free = np.full(nb + 5, -7, np.int32)
    assert check_release(lens, have, table, bs, nb, free, 5) == 0


def test_release_past_the_list_and_bad_requests():
    rng = np.random.default_rng(1)
    have = rng.integers(50, 200, 40)
    lens = have // 3
    table, nb = ref.tables(rng, have, 16)
    for cap in (0, 1, 50):
        assert check_release(lens, have, table, 16, nb,
                             np.zeros(cap, np.int32), 1) == ref.CAPACITY
    for count in (-5, 1 << 40):
        check_release(lens, have, table, 16, nb, np.zeros(1000, np.int32), count)
    lens[3], have[7] = -1, -2
    have[9] = table.shape[1] * 16 + 1
    assert check_release(lens, have, table, 16, nb, np.zeros(1000, np.int32),
                         4) == ref.RANGE
    table[20, 8], table[21, 8] = -1, nb
    have[20] = have[21] = 150
    lens[20] = lens[21] = 20
    assert check_release(lens, have, table, 16, nb, np.zeros(1000, np.int32),
                         4) == ref.BLOCK_ID


# ----------------------------------- weigh: rows that a wavefront holds, keys

@pytest.mark.parametrize("dtype", [BF, FP])
@pytest.mark.parametrize("D", [64, 128])
@pytest.mark.parametrize("G,window", [(1, 65), (4, 17), (3, 32), (1, 127),
                                      (4, 32), (8, 16), (1, 129), (3, 43)])
@pytest.mark.parametrize("bs,order", [(16, NHD), (5, HND)])
def test_weigh_up_to_and_past_128_rows(dtype, D, G, window, bs, order):
    """Every tile of rows that a wavefront holds, part-filled and full, and the
    first count of rows that it does not hold."""
    w = window
    n = [w, w + 1, 64 + w, 300, 1500, 0, w + 3, 1100]
    m = [w, w, w, w - 1, w, 0, 1, w // 2]
    c = Case(n, m, 2, G, D, bs, order, dtype, seed=G + w)
    assert check_weigh(c, max_new=w) == 0


@pytest.mark.parametrize("dtype", [BF, FP])
@pytest.mark.parametrize("m", [1, 6, 30, 70])
@pytest.mark.parametrize("D", [64, 128])
@pytest.mark.parametrize("whole", [True, False])
def test_weigh_keys_that_are_not_finite(dtype, m, D, whole):
    """NaN and infinities among the keys (a whole row, or one element, whose
    scores are then infinite): a query with a score of NaN or +infinity makes the
    places that it sees NaN, and no others; a score of -infinity weighs 0."""
    n, G = [200, 90, 150, 1300], 4
    c = Case(n, [m] * 4, 2, G, D, dtype=dtype, seed=m)
    rows = ref.by_slot(c.cache, c.sh, c.nb)
    for r, (back, bad) in enumerate(((1, "nan"), ((m + 1) // 2, "inf"),
                                     ((m + 2) // 3, "-inf"), (700, "-inf"))):
        j = n[r] - back
        at = rows[0, 0, int(c.table[r, j // 16]), j % 16]
        if whole:
            at[0] = float(bad)
        else:
            at[0, 3] = float(bad)
    _, lse, _ = c.attend()
    led = paged.new_ledger(c.sh, c.nb, dev())
    led.copy_(torch.rand(led.shape, generator=gen(3), device=dev())
              .view(torch.int32))
    want = paged.weights_of(led)[0].double()
    slack = torch.zeros_like(want)
    for r, x in enumerate(n):
        a, _, k, v, seen, block, at = ref.request_rows(
            r, c.q, c.cache, c.sh, c.nb, c.table, c.n, c.cu, 0, m)
        block, at = (torch.tensor(t, device=dev()) for t in (block, at))
        for g in range(2 * G):
            q, given = c.q[a:a + m, g].double(), lse[a:a + m, g].double()
            s = torch.matmul(q, k[:, g // G].t().contiguous()) * D ** -0.5
            p = torch.where(seen, torch.exp(s - given[:, None]), 0.0)
            room = ref.attend(q, k[:, g // G], v[:, g // G], D ** -0.5, seen,
                              0.0)[5]
            want[block, g // G, at] += p.sum(0)
            slack[block, g // G, at] += torch.where(p > 0, p * room, 0.0).sum(0)
    # the sums' own roundings, as weighed() counts them
    slack += want.abs().nan_to_num(0) * ((m * G / 32 + 8) * 2.0 ** -24
                                         + 2.0 ** -23)
    status = word()
    paged.lumen_paged_weigh(c.sh, c.nb, 0, c.cache, i32(c.table), i32(c.n),
                            i32(c.cu), c.q, lse, led, status, max_new=m)
    got = paged.weights_of(led)[0]
    assert int(status) == 0
    # places that no NaN reaches, of every request and head, are among those checked
    assert want.isnan().any() and want.isfinite().any()
    close(got, want, slack, 0.0, "weights")
