"""The 16-bit paged cache's operators at their edges: streams, prepared calls,
graphs, strides, caches past 32 bits, and calls whose results must not change."""
import numpy as np
import pytest
import torch

import paged_ref as ref
from attn_ref import UNIT
from gpu_util import dev
from paper_2606_17787_amd import paged
from paper_2606_17787_amd.workloads import CacheShape, HND, NHD
from test_gpu_paged import BF, FP, Case, Evict, check_weigh, close, gen, i32, \
    new_cache, word

pytestmark = pytest.mark.gpu


class Calls:
    """One call of each operator on tensors of its own, and what they wrote."""

    def __init__(self, m=3, seed=0):
        n = [700, 33, 1500, 64]
        self.c = Case(n, [m] * 4, 2, 4, 128, seed=seed, layers=2, stale=False)
        c = self.c
        self.table, self.lens, self.cu = i32(c.table), i32(c.n), i32(c.cu)
        self.status = word()
        T = c.q.shape[0]
        self.out = torch.zeros(c.q.shape, dtype=c.q.dtype, device=dev())
        self.lse = torch.zeros(c.q.shape[:2], device=dev())
        self.ledger = paged.new_ledger(c.sh, c.nb, dev())
        g = gen(seed + 1)
        self.k, self.v = (torch.randn(T, 2, 128, generator=g, device=dev())
                          .to(BF) for _ in range(2))
        self.slots = torch.tensor(
            [int(c.table[r, j // 16]) * 16 + j % 16
             for r in range(4) for j in range(n[r] - m, n[r])], device=dev())
        self.pos = torch.arange(T, dtype=torch.int32, device=dev())
        self.keep, self.frm = i32([300, 20, 800, 64]), i32([690, 30, 1400, 60])
        self.left = i32([0] * 4)
        self.ws = paged.new_evict_workspace(c.sh, 4, c.table.shape[1], dev())
        self.free = i32(np.full(c.nb, -1))
        self.count, self.now = (torch.zeros(1, dtype=torch.int64, device=dev())
                                for _ in range(2))
        self.start = [t.clone() for t in self.written()]

    def written(self):
        return [self.c.cache, self.ledger, self.out, self.lse, self.left,
                self.free, self.now, self.status]

    def reset(self):
        for t, s in zip(self.written(), self.start):
            t.copy_(s)

    def args(self):
        c = self.c
        head = (c.sh, c.nb, 1, c.cache)
        return [("append", head + (self.k, self.v, self.slots, self.status),
                 dict(ledger=self.ledger, positions=self.pos)),
                ("attend", head + (self.table, self.lens, self.cu, c.q,
                                   self.out, self.status),
                 dict(max_new=max(c.m), lse=self.lse)),
                ("weigh", head + (self.table, self.lens, self.cu, c.q, self.lse,
                                  self.ledger, self.status),
                 dict(max_new=max(c.m))),
                ("evict", (c.sh, c.nb, c.cache, self.ledger, self.table,
                           self.lens, self.keep, self.frm, self.left, self.ws,
                           self.status), dict(sinks=2)),
                ("release", (self.left, self.lens, self.table, 16, c.nb,
                             self.free, self.count, self.now, self.status),
                 dict())]

    def call(self, **kw):
        for name, a, k in self.args():
            getattr(paged, f"lumen_paged_{name}")(*a, **k, **kw)

    def prepared(self):
        return [getattr(paged, f"prepare_{name}")(*a, **k)
                for name, a, k in self.args()]

    def results(self):
        torch.cuda.synchronize()
        return [t.clone() for t in self.written()]


def same(a, b):
    for x, y in zip(a, b):
        assert torch.equal(x.view(torch.int16) if x.dtype == BF else x,
                           y.view(torch.int16) if y.dtype == BF else y)


@pytest.mark.parametrize("m", [1, 3, 33])
def test_calls_take_a_stream(m):
    x = Calls(m)
    x.call()
    want = x.results()
    x.reset()
    torch.cuda.synchronize()
    stream = torch.cuda.Stream()
    x.call(stream=stream)
    stream.synchronize()
    same(x.results(), want)
    assert int(x.status) == 0


@pytest.mark.parametrize("m", [1, 3, 33])
def test_prepared_calls_are_the_calls(m):
    x = Calls(m)
    x.call()
    want = x.results()
    calls = x.prepared()
    stream = torch.cuda.Stream()
    for s in (None, None, stream):
        x.reset()
        torch.cuda.synchronize()
        for f in calls:
            f(s)
        same(x.results(), want)


@pytest.mark.parametrize("m", [1, 33])
def test_two_graphs_of_the_calls(m):
    """Captured with workspaces of their own and replayed side by side, with
    eager work and new lengths between."""
    xs = [Calls(m, seed) for seed in (0, 1)]
    want, shorter = [], []
    for x in xs:
        x.call()
        want.append(x.results())
        x.reset()
        x.lens.sub_(17)
        x.call()
        shorter.append(x.results())
        x.lens.add_(17)
        x.reset()
    torch.cuda.synchronize()
    held, graphs = [], []
    for x in xs:
        calls = x.prepared()
        for f in calls:  # first uses are not captured
            f()
        x.reset()
        torch.cuda.synchronize()
        g = torch.cuda.CUDAGraph()
        with torch.cuda.graph(g):
            for f in calls:
                f()
        held.append(calls)
        graphs.append(g)
    for turn in range(4):
        for x in xs:
            x.reset()
            if turn % 2:
                x.lens.sub_(17)
        streams = [torch.cuda.Stream() for _ in xs]
        torch.cuda.synchronize()
        for s, g in zip(streams, graphs):
            with torch.cuda.stream(s):
                g.replay()
        torch.cuda.synchronize()
        for x, w in zip(xs, shorter if turn % 2 else want):
            same(x.results(), w)
            if turn % 2:
                x.lens.add_(17)
        torch.randn(1000, 1000, device=dev()).sum().item()


def test_a_prepared_attends_own_workspace_outlives_its_last_call():
    """The object goes while its call is under way on another stream: its
    workspace is not given to what is allocated next."""
    c = Case([9000] * 8, [1] * 8, 2, 4, 128, seed=3)
    want, _, _ = c.attend(max_new=1)
    out = torch.zeros_like(want)
    stream = torch.cuda.Stream()
    args = (c.sh, c.nb, 0, c.cache, i32(c.table), i32(c.n), i32(c.cu), c.q, out,
            word())
    torch.cuda.synchronize()
    for _ in range(20):
        f = paged.prepare_attend(*args, max_new=1)
        size = f._workspace.numel()
        f(stream)
        del f
        torch.full((size,), 255, dtype=torch.uint8, device=dev())
    torch.cuda.synchronize()
    assert torch.equal(out, want)


@pytest.mark.parametrize("m", [1, 40])
def test_queries_stored_head_by_head(m):
    c = Case([300, 90], [m, m], 2, 3, 64, dtype=FP, seed=4)
    want, wl, _ = c.attend()
    c.q = c.q.transpose(0, 1).contiguous().transpose(0, 1)
    assert c.q.stride(1) > c.q.stride(0) or m * 2 == 1
    got, gl, _ = c.attend()
    assert torch.equal(got, want) and torch.equal(gl, wl)
    check_weigh(c)


@pytest.mark.parametrize("order", [NHD, HND])
def test_caches_past_32_bits(order):
    """Blocks at both ends of a cache whose keys alone pass 2^32 bytes."""
    sh = CacheShape(1, 1, 128, 16, order)
    nb = (1 << 20) + 4000  # of 4 KB each for K and V
    cache = torch.empty(sh.pool_elems(nb), dtype=BF, device=dev())
    n = [90, 50]
    table = np.array([[0, nb - 1, 7, nb - 2, 1 << 20, nb - 5],
                      [nb - 3, 3, (1 << 20) + 9, 11, -1, -1]], np.int32)
    c = Case(n, [5, 40], 1, 4, 128, seed=5, stale=False)
    small = c.cache.view(c.sh.pool_dims(c.nb))
    big = cache.view(sh.pool_dims(nb))
    rows = ref.by_slot(cache, sh, nb)
    ledger = torch.zeros(paged.ledger_dims(sh, nb), dtype=torch.int32,
                         device=dev())
    T = sum(n)
    slots = torch.tensor([int(table[r, j // 16]) * 16 + j % 16
                          for r in range(2) for j in range(n[r])], device=dev())
    g = gen(6)
    k, v = (torch.randn(T, 1, 128, generator=g, device=dev()).to(BF)
            for _ in range(2))
    pos = torch.cat([torch.arange(x, dtype=torch.int32) for x in n]).to(dev())
    status = word()
    paged.lumen_paged_append(sh, nb, 0, cache, k, v, slots, status,
                             ledger=ledger, positions=pos)
    b, o = slots // 16, slots % 16
    assert torch.equal(rows[0, 0][b, o], k) and torch.equal(rows[0, 1][b, o], v)
    assert torch.equal(ledger[0, 1][b, 0, o], pos)
    c.sh, c.nb, c.cache, c.table = sh, nb, cache, table
    out, lse = c.check()
    want, slack = ref.weighed(c.q, lse, cache, sh, nb, table, n, c.cu,
                              paged.weights_of(ledger)[0].clone())
    paged.lumen_paged_weigh(sh, nb, 0, cache, i32(table), i32(n), i32(c.cu),
                            c.q, lse, ledger, status)
    close(paged.weights_of(ledger)[0], want, slack, 0.0, "weights")
    del want, slack
    weights = paged.weights_of(ledger)[0][b, 0, o].cpu().numpy()
    left = i32([0, 0])
    paged.lumen_paged_evict(
        sh, nb, cache, ledger, i32(table), i32(n), i32([40, 30]),
        i32([80, 48]), left, paged.new_evict_workspace(sh, 2, 6, dev()), status,
        sinks=2)
    at = 0
    for r, keep in enumerate((40, 30)):
        frm = (80, 48)[r]
        kept = set(ref.rank_order(weights[at:at + n[r]], np.arange(n[r]), 2,
                                  frm)[:keep])
        src = [j for j in range(keep, n[r]) if j in kept]
        order_now = [j if j in kept else src.pop(0) for j in range(keep)]
        blk = torch.tensor(table[r, np.arange(keep) // 16], device=dev()).long()
        off = torch.arange(keep, device=dev()) % 16
        assert ledger[0, 1][blk, 0, off].tolist() == order_now
        assert torch.equal(rows[0, 0][blk, off], k[at + torch.tensor(order_now)])
        assert torch.equal(rows[0, 1][blk, off], v[at + torch.tensor(order_now)])
        at += n[r]
    assert left.tolist() == [40, 30] and int(status) == 0


@pytest.mark.parametrize("m", [2, 200])
def test_tables_of_as_many_places_as_32_bits_count(m):
    """2,048 pages of 2^20 places each, of which one is there."""
    sh = CacheShape(1, 1, 64, 1 << 20, NHD)
    cache = torch.zeros(sh.pool_elems(1), dtype=BF, device=dev())
    n, cu = 2500, [0, m]
    g = gen(8)
    k, v = (torch.randn(n, 1, 64, generator=g, device=dev()).to(BF)
            for _ in range(2))
    q = torch.randn(m, 2, 64, generator=g, device=dev()).to(BF)
    ledger = torch.zeros(paged.ledger_dims(sh, 1), dtype=torch.int32,
                         device=dev())
    status, out = word(), torch.empty_like(q)
    lse = torch.empty(m, 2, device=dev())
    table = np.full((1, 2048), -1, np.int32)
    table[0, 0] = 0
    every = torch.arange(n, device=dev())
    paged.lumen_paged_append(sh, 1, 0, cache, k, v, every, status,
                             ledger=ledger, positions=every.to(torch.int32))
    args = (sh, 1, 0, cache, i32(table), i32([n]), i32(cu), q)
    paged.lumen_paged_attend(*args, out, status, lse=lse)
    paged.lumen_paged_weigh(*args, lse, ledger, status)
    # the definitions, over a cache of pages of 25 that holds the same
    small = CacheShape(1, 1, 64, 25, NHD)
    pool = torch.zeros(small.pool_elems(100), dtype=BF, device=dev())
    rows = ref.by_slot(pool, small, 100)
    rows[0, 0] = k.view(100, 25, 1, 64)
    rows[0, 1] = v.view(100, 25, 1, 64)
    places = np.arange(100, dtype=np.int32)[None]
    want, slack = ref.weighed(q, lse, pool, small, 100, places, [n], cu,
                              torch.zeros(100, 1, 25, device=dev()))
    close(paged.weights_of(ledger)[0, 0, 0, :n], want.flatten(),
          slack.flatten(), 0.0, "weights")
    assert int(status) == 0 and not paged.weights_of(ledger)[0, 0, 0, n:].any()


def test_more_requests_than_lanes_and_errors_among_the_last():
    for max_new in (1, 4):
        n = [20] * 200
        c = Case(n, [1] * 200, 1, 2, 64, seed=7)
        c.n[150] = -1
        c.table[190, 1] = c.nb
        c.check(max_new=max_new)
        check_weigh(c, max_new=max_new)


def test_a_pool_without_blocks():
    sh = CacheShape(1, 2, 64, 16, NHD)
    cache = torch.empty(0, dtype=BF, device=dev())
    led = paged.new_ledger(sh, 0, dev())
    table = i32(np.full((2, 4), 0))
    q = torch.ones(2, 4, 64, dtype=BF, device=dev())
    out, lse = torch.full_like(q, 7), torch.full((2, 4), 7.0, device=dev())
    status = word()
    cu = i32([0, 1, 2])
    paged.lumen_paged_attend(sh, 0, 0, cache, table, i32([9, 0]), cu, q, out,
                             status, lse=lse)
    assert (out == 0).all() and torch.isinf(lse).all()
    assert int(status) == ref.BLOCK_ID
    status = word()
    paged.lumen_paged_weigh(sh, 0, 0, cache, table, i32([9, 0]), cu, q, lse, led,
                            status)
    assert int(status) == ref.BLOCK_ID
    status, left = word(), i32([0, 0])
    paged.lumen_paged_evict(sh, 0, cache, led, table, i32([9, 3]), i32([4, 4]),
                            i32([0, 0]), left,
                            paged.new_evict_workspace(sh, 2, 4, dev()), status)
    assert left.tolist() == [9, 3] and int(status) == ref.BLOCK_ID


@pytest.mark.parametrize("m", [1, 70])
def test_one_block_for_every_page(m):
    """A table may name a block more than once: it is read as often."""
    c = Case([200], [m], 2, 4, 128, seed=8, stale=False)
    c.table[0, :] = 2
    c.check()


def test_evictions_repeat_themselves():
    e = Evict([3000, 500, 20000], [700, 499, 9000], layers=2, seed=9, kind="ties")
    ws = paged.new_evict_workspace(e.sh, 3, e.table.shape[1], dev())
    results = []
    for _ in range(3):
        cache, led = e.cache.clone(), torch.tensor(e.led, device=dev())
        left = i32([0] * 3)
        ws.random_(0, 256)  # what it holds does not matter
        paged.lumen_paged_evict(e.sh, e.nb, cache, led, i32(e.table), i32(e.n),
                                i32(e.keep), i32(e.frm), left, ws, word(),
                                sinks=e.sinks)
        results.append((cache, led, left))
    for r in results[1:]:
        same(r, results[0])


def test_what_a_workspace_holds_does_not_matter():
    c = Case([4000, 300, 9000], [200, 1, 3], 2, 4, 128, seed=10)
    want, wl, _ = c.attend(max_new=200)
    ws = paged.new_attend_workspace(c.sh, i32(c.table), i32(c.n), c.q, 200)
    for _ in range(3):
        ws.random_(0, 256)
        got, gl, status = c.attend(max_new=200, workspace=ws)
        assert torch.equal(got, want) and torch.equal(gl, wl) and status == 0


def test_requests_past_a_narrow_table_repeat_themselves():
    """A request with many more places than the table's 8,192: those that there are
    count, and all tiles of rows that see every one of them are computed alike."""
    pages, tiles = 512, 780
    T = tiles * 128
    c = Case([pages * 16], [128], 1, 1, 64, seed=11, dtype=FP)
    c.q = c.q[:128].repeat(tiles, 1, 1)  # each tile's rows are the same ones
    c.n, c.m, c.cu = [T], [T], np.array([0, T], np.int32)
    out, lse, status = c.attend()
    assert status == ref.RANGE
    flat = slice(pages * 16 // 128, tiles)  # tiles whose rows see all places
    out, lse = out.view(tiles, 128, 64)[flat], lse.view(tiles, 128)[flat]
    k, v = (ref.by_slot(c.cache, c.sh, c.nb)[0, i, torch.tensor(
        c.table[0], device=dev()).long()].reshape(-1, 64).double()
        for i in (0, 1))
    seen = torch.ones(128, pages * 16, dtype=torch.bool, device=dev())
    want, slack, wl, lslack = ref.attend(c.q[:128, 0].double(), k, v, 0.125,
                                         seen, UNIT[FP])[:4]
    close(out[0], want, slack, UNIT[FP])
    close(lse[0], wl, lslack, 0.0)
    assert bool((out == out[:1]).all()) and bool((lse == lse[:1]).all())


@pytest.mark.parametrize("n,m,H,G,D", [
    ([300, 20, 64], [1, 1, 1], 2, 4, 128), ([300, 90, 64], [9, 90, 3], 2, 3, 64),
    ([9000, 700, 4000], [1, 200, 2], 2, 8, 128), ([5000], [4100], 16, 1, 128)])
@pytest.mark.parametrize("dtype", [BF, FP])
def test_attend_in_the_queries_place(n, m, H, G, D, dtype):
    """Whole tiles, tiles in parts, and workgroups of eight wavefronts."""
    c = Case(n, m, H, G, D, dtype=dtype, seed=12)
    c.q = c.q.contiguous()
    want, wl, _ = c.attend(max_new=max(m))
    args = (i32(c.table), i32(c.n), i32(c.cu))
    for _ in range(3):
        q, lse, status = c.q.clone(), torch.zeros_like(wl), word()
        paged.lumen_paged_attend(c.sh, c.nb, 0, c.cache, *args, q, q, status,
                                 max_new=max(m), lse=lse)
        assert torch.equal(q, want) and torch.equal(lse, wl)
        assert int(status) == 0


def test_append_of_rows_of_the_cache():
    """Tokens of one request into slots of another, in the same layer."""
    sh = CacheShape(1, 3, 64, 8, NHD)
    cache = new_cache(sh, 20, BF, gen(13))
    rows = cache.view(2, 160, 3, 64)
    want = cache.clone().view(2, 160, 3, 64)
    want[:, 100:150] = want[:, 10:60]
    status = word()
    paged.lumen_paged_append(sh, 20, 0, cache, rows[0, 10:60], rows[1, 10:60],
                             torch.arange(100, 150, device=dev()), status)
    assert torch.equal(rows, want) and int(status) == 0


@pytest.mark.parametrize("dtype", [BF, FP])
@pytest.mark.parametrize("m", [1, 60])
@pytest.mark.parametrize("down", [10, 40, 200])
def test_infinite_values_with_the_smallest_weights(dtype, m, down):
    """Where a weight is too small for its type an infinite value still shows, in
    its own element alone."""
    c = Case([400, 70], [m, m], 1, 2, 64, dtype=dtype, seed=14)
    rows = ref.by_slot(c.cache, c.sh, c.nb)[0]
    c.q[:] = 0
    c.q[:, :, 0] = 1
    keys = rows[0]
    keys[keys.isfinite()] = 0
    keys[int(c.table[0, 4]), 7, 0, 0] = -down  # seen by all, not in a last step
    base, lse, _ = c.attend(scale=0.6931471805599453)
    rows[1, int(c.table[0, 4]), 7, 0, 9] = float("inf")
    got, again, status = c.attend(scale=0.6931471805599453)
    assert status == 0 and torch.equal(lse, again)
    hit = torch.zeros_like(got, dtype=torch.bool)
    hit[:m, :, 9] = True
    assert torch.equal(got[~hit], base[~hit]) and base.isfinite().all()
    assert not (got[hit].isfinite() | (got[hit] == float("-inf"))).any()
    if down < 20:
        assert (got[hit] == float("inf")).all()


@pytest.mark.parametrize("G", [16, 33, 64, 96, 130, 200])
@pytest.mark.parametrize("m", [1, 5, 40])
def test_many_query_heads_of_one(G, m):
    """More heads than a tile of rows has, and counts that divide none."""
    n = [m, 300, 130, 1700]
    c = Case(n, [m] * 4, 1, G, 64 if G % 2 else 128, dtype=FP, seed=G)
    c.check(max_new=m)
    assert check_weigh(c, max_new=m) == 0
