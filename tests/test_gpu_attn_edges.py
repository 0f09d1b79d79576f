"""The serving operators at the ends of their inputs' ranges, against plain
references: values and scales that 32 bits or 16 hold badly, rows that see
only infinities, sizes past 2^31, streams and forms of a call."""
import numpy as np
import pytest
import torch

import attn_ref as ref
from paper_2606_17787_amd import attn
from gpu_util import dev
from test_gpu_attn import (BF, FP, decode_case, decode_want, i32, prompt_want,
                           word)

pytestmark = pytest.mark.gpu


def run_decode(sh, nb, cache, table, lens, q, scale=None):
    out, status = torch.full_like(q, 7.0), word()
    ws = attn.new_decode4_workspace(sh, lens.numel(), q.shape[1])
    attn.lumen_attn_decode4(sh, nb, 0, cache, table, lens, q, out, ws, status,
                            scale=scale)
    assert int(status) == 0
    return out


def run_prompt(q, k, v, cu_q, cu_k=None, scale=None):
    out, status = torch.full_like(q, 7.0), word()
    attn.lumen_attn_prompt(q, k, v, out, i32(cu_q), status,
                           cu_k=None if cu_k is None else i32(cu_k),
                           scale=scale)
    assert int(status) == 0
    return out


# ------------------------------------------- scales at the ends of the range

@pytest.mark.parametrize("scale", [1e-45, 1e-9, 1.0, 2e38])
@pytest.mark.parametrize("dtype", [BF, FP])
def test_decode_of_zero_queries_is_the_mean(dtype, scale):
    """A row of zeros has scores of 0 under any scale, masked keys beside the
    seen ones in its last block or not."""
    rng = np.random.default_rng(1)
    sh, nb, cache, rows, table, lens, q = decode_case(
        rng, [1, 31, 32, 45, 500], 2, 4, 128, 16, "NHD", dtype)
    q[:, 1::2] = 0
    q[:, ::2] *= min(1.0, 1 / scale)
    want, slack = decode_want(rows(0), table, lens, q, 2, 16, scale, dtype)
    ref.assert_close(run_decode(sh, nb, cache, table, lens, q, scale), want,
                     slack, dtype)


@pytest.mark.parametrize("scale", [1e-45, 1e-9, 2e38])
@pytest.mark.parametrize("dtype", [BF, FP])
def test_prompt_of_zero_queries_is_the_mean(dtype, scale):
    g = torch.Generator(device=dev()).manual_seed(2)
    q = torch.zeros(150, 4, 64, dtype=dtype, device=dev())
    k, v = (torch.randn(150, 2, 64, generator=g, device=dev()).to(dtype)
            for _ in range(2))
    cu = [0, 1, 70, 150]
    want, slack = prompt_want(q, k, v, cu, cu, scale, ref.UNIT[dtype])
    ref.assert_close(run_prompt(q, k, v, cu, scale=scale), want, slack, dtype)


# ----------------------------------------------------------- large values

@pytest.mark.parametrize("value", [2e36, -2e36])
@pytest.mark.parametrize("H", [1, 64])
def test_prompt_means_of_large_values_stay_finite(H, value):
    """64 keys of score 0 and 64 whose weights are 2^7.9 of theirs, all of one
    value: the sum of the weights under the true maximum times it is below
    3.4e38.  (64 heads of 2,048 queries take the larger workgroups.)"""
    n = 2048 if H == 64 else 1
    q = torch.zeros(n, H, 64, dtype=BF, device=dev())
    k = torch.zeros(128, 1, 64, dtype=BF, device=dev())
    v = torch.full((128, 1, 64), value, dtype=BF, device=dev())
    q[..., 0], k[64:, :, 0] = 1.0, 7.9 * 0.6931
    # every query sees all keys: they are the ends of sequences of one query
    out = torch.full_like(q, 7.0)
    if n == 1:
        out = run_prompt(q, k, v, [0, 1], [0, 128], scale=1.0)
    else:
        k = torch.cat([k, torch.full((n - 1, 1, 64), -9.0, dtype=BF,
                                     device=dev())])
        v = torch.cat([v, torch.zeros(n - 1, 1, 64, dtype=BF, device=dev())])
        out = run_prompt(q, k, v, [0, n], [0, 127 + n], scale=1.0)
    top = v[0, 0, 0].double()
    # the later keys' weights are 2^-20 of the others', 2,047 of them
    room = float(top.abs()) * (2 * ref.UNIT[BF] + 2.0 ** -9)
    assert torch.isfinite(out).all()
    assert float((out.double() - top).abs().max()) <= room


# ------------------------------------------- scores that are not finite

# Lengths of one key, of part of a block, of several workgroups' shares.
@pytest.mark.parametrize("lens", [[1, 20, 33, 700, 0], [9000]])
@pytest.mark.parametrize("H,order", [(2, "NHD"), (1, "NHD"), (2, "HND")])
@pytest.mark.parametrize("dtype", [BF, FP])
def test_decode_scores_that_are_not_finite(lens, H, order, dtype):
    """Infinite and NaN queries: a row whose scores are all -infinity or that
    has one of +infinity is NaN, as is one with a NaN; the rows beside it and
    requests without keys are as ever."""
    rng = np.random.default_rng(4)
    D, G, bs = 128, 4, 16
    sh, nb, cache, rows, table, dl, q = decode_case(rng, lens, H, G, D, bs,
                                                    order, dtype)
    # element 0 of every key is negative: its quarter's B is, by far
    pairs = rows(0)[0][..., D // 2:D // 2 + 4].contiguous()
    half = pairs.view(torch.float16)
    half[..., 1] = -200.0
    half[..., 0] = 0.5
    stale = torch.zeros_like(half[..., 0], dtype=torch.bool)
    for r, n in enumerate(lens):
        if n % bs:
            stale[table[r, n // bs].long(), n % bs:] = True
    half[stale] = float("nan")
    rows(0)[0][..., D // 2:D // 2 + 4] = half.view(torch.uint8)
    zero = torch.zeros_like(q[:, 0])
    first = zero.clone()
    first[:, 0] = 1
    heads = range(0, H * G, 4)
    for h in heads:
        q[:, h] = torch.where(first > 0, float("inf"), zero)       # all -inf
        q[:, h + 1] = torch.where(first > 0, float("-inf"), zero)  # all +inf
        q[:, h + 2, 5] = float("nan")
    want, slack = decode_want(rows(0), table, dl, torch.nan_to_num(q), H, bs,
                              D ** -0.5, dtype)
    out = run_decode(sh, nb, cache, table, dl, q).double()
    some = (dl > 0)[:, None, None]
    bad = torch.zeros_like(want, dtype=torch.bool)
    for h in heads:
        bad[:, h:h + 3] = some
    assert torch.equal(torch.isnan(out), bad)
    z = torch.zeros_like(want)
    ref.assert_close(torch.where(bad, z, out), torch.where(bad, z, want),
                     torch.where(bad, z, slack), dtype)


def formula(q, k, v, scale, seen, dtype):
    """(out, slack) of one head in 64 bits, with no special case for rows whose
    scores are all -infinity; zeros for rows that see no key.  slack is that of
    the finite rows, whose keys of score -infinity have no weight."""
    s = (torch.matmul(q, k.transpose(0, 1).contiguous()) * scale)
    s = s.masked_fill(~seen, float("-inf"))
    p = torch.exp(s - s.amax(-1, keepdim=True))
    out = torch.matmul(p / p.sum(-1, keepdim=True), v)
    out[~seen.any(-1)] = 0.0
    weighed = seen & torch.isfinite(s)
    _, slack = ref.attend(torch.nan_to_num(q, 0.0, 0.0, 0.0),
                          torch.nan_to_num(k, 0.0, 0.0, 0.0), v, scale,
                          weighed, ref.UNIT[dtype])
    return out, slack


@pytest.mark.parametrize("nq,nk,H,G,D", [
    ([70, 130], [70, 130], 2, 2, 64), ([33, 5], [150, 3], 1, 4, 128),
    ([40, 3], [6000, 70], 1, 8, 128), ([2100], [2100], 8, 8, 64)])
@pytest.mark.parametrize("dtype", [BF, FP])
def test_prompt_scores_that_are_not_finite(nq, nk, H, G, D, dtype):
    """Infinities and NaN in keys and queries: rows that see a score of NaN or
    +infinity, or none but -infinity, are NaN; a score of -infinity among
    others has no weight; rows that see no such key are as ever."""
    g = torch.Generator(device=dev()).manual_seed(sum(nk))
    q = torch.randn(sum(nq), H * G, D, generator=g, device=dev())
    k, v = (torch.randn(sum(nk), H, D, generator=g, device=dev()).to(dtype)
            for _ in range(2))
    cu_q, cu_k = np.cumsum([0] + nq), np.cumsum([0] + nk)
    q[..., 1] = q[..., 1].abs() + 0.5
    q[::3, :, 1] *= -1  # an infinite element of a key is +infinity for others
    q = q.to(dtype)
    for s, n in enumerate(nk):
        first = max(0, n - nq[s])  # the last key of the first query
        k[cu_k[s], 0, 1] = float("-inf")        # every query sees it
        if n > 9:
            k[cu_k[s] + n // 2 + 1, 0, 1] = float("-inf")
            k[cu_k[s + 1] - 2, 0, 1] = float("inf")   # the last two queries
            k[cu_k[s + 1] - 1, 0, 7] = float("nan")   # the last one
        q[cu_q[s + 1] - 3, G - 1, 9] = float("nan")
        q[cu_q[s], :, 2] = float("inf")
        k[cu_k[s]:cu_k[s] + first + 1, :, 2] = -1.0   # all of its scores
    out = run_prompt(q, k, v, cu_q, cu_k).double()
    nans = 0
    for s in range(len(nq)):
        a, b, e, f = cu_q[s], cu_q[s + 1], cu_k[s], cu_k[s + 1]
        i = torch.arange(b - a, device=dev())[:, None] + (f - e) - (b - a)
        seen = torch.arange(f - e, device=dev())[None] <= i
        for h in range(H * G):
            want, slack = formula(q[a:b, h].double(), k[e:f, h // G].double(),
                                  v[e:f, h // G].double(), D ** -0.5, seen,
                                  dtype)
            bad = torch.isnan(want)
            nans += int(bad.any(-1).sum())
            z = torch.zeros_like(want)
            assert torch.equal(torch.isnan(out[a:b, h]), bad), (s, h)
            ref.assert_close(torch.where(bad, z, out[a:b, h]),
                             torch.where(bad, z, want),
                             torch.where(bad, z, slack), dtype, f"{s} {h}")
    assert 0 < nans < sum(nq) * H * G


# -------------------------------------------------- every pair that a row holds

@pytest.mark.parametrize("D", [64, 128, 256])
def test_read_rounds_a_value_once(D):
    """Pairs of any size, whose value may need more bits than 32-bit arithmetic
    holds: rounded to 16 bits once.  1986 * 2^-17 * 66 + 4000 is 2^-15 above the
    middle of two 16-bit values."""
    rng = np.random.default_rng(6)
    H, bs, nb = 2, 16, 64
    T = nb * bs
    codes = rng.integers(0, 16, (2, T, H, D)).astype(np.uint8)
    A = (rng.uniform(0.5, 1, (2, T, H, 4)) *
         2.0 ** rng.integers(-20, 8, (2, T, H, 4))).astype(np.float16)
    B = (rng.uniform(-1, 1, (2, T, H, 4)) *
         2.0 ** rng.integers(-10, 13, (2, T, H, 4))).astype(np.float16)
    A[:, 0], B[:, 0], codes[:, 0, :, ::3] = 1986 * 2.0 ** -17, 4000.0, 2
    A[:, 1], B[:, 1] = 0.0, 5.0
    A[:, 2], B[:, 2] = 2.0 ** -24, 2.0 ** -24  # subnormal
    sh = attn.cache_shape4(1, H, D, bs)
    cache = torch.from_numpy(ref.to_rows(codes, A, B)).to(dev()).reshape(-1)
    want = ref.values(codes, A, B)
    assert want[0, 0, 0, 0] == 4002.0
    slots, status = torch.arange(T, device=dev()), word()
    for dtype in (FP, BF):
        k, v = (torch.empty(T, H, D, dtype=dtype, device=dev())
                for _ in range(2))
        attn.lumen_attn_read4(sh, nb, 0, cache, slots, k, v, status)
        assert int(status) == 0
        for got, w in ((k, want[0]), (v, want[1])):
            assert torch.equal(got.cpu(), torch.from_numpy(w).to(dtype))


# ------------------------------------------------------- what a NaN costs

def test_one_nan_does_not_slow_a_prompt_down_many_times():
    """A NaN in an early value, key or a query makes the tiles that see it run
    once more, with a look at each value: about two passes more, of which 8 are
    allowed for."""
    n, H, G, D = 8192, 2, 8, 128
    g = torch.Generator(device=dev()).manual_seed(1)
    q, k, v = (torch.randn(n, h, D, generator=g, device=dev()).to(BF)
               for h in (H * G, H, H))
    out, status = torch.empty_like(q), word()
    call = attn.prepare_prompt(q, k, v, out, i32([0, n]), status)

    def time():
        call()
        at = [torch.cuda.Event(enable_timing=True) for _ in range(6)]
        for e in at:
            e.record()
            call()
        torch.cuda.synchronize()
        return min(a.elapsed_time(b) for a, b in zip(at, at[1:]))

    clean = time()
    for t, row in ((v, 5), (k, 5), (q, n - 7)):
        was = t[row].clone()
        t[row, :, 9] = float("nan")
        assert time() < 8 * clean
        assert torch.isnan(out).any() and torch.isfinite(out).any()
        t[row] = was
    call()
    assert torch.isfinite(out).all() and int(status) == 0


# ------------------------------------------------------------ sizes past 2^31

def test_slots_from_a_free_list_of_more_than_2_to_the_31_places():
    """Pages come from the list's end, wherever that is."""
    n = (1 << 31) + 5
    free = torch.zeros(n, dtype=torch.int32, device=dev())
    free[-6:] = i32([11, 12, 13, 14, 15, 16])
    count, left = (torch.tensor([n], device=dev()) for _ in range(2))
    table, status = i32(np.full((2, 4), -1)), word()
    slots = torch.empty(50, dtype=torch.int64, device=dev())
    cu, lens = i32(np.zeros(3)), i32(np.zeros(2))
    attn.lumen_attn_slots(i32([0, 0]), i32([20, 30]), table, 16, 20, free,
                          count, slots, cu, lens, left, status)
    assert int(status) == 0 and int(left) == n - 4
    assert table.tolist() == [[16, 15, -1, -1], [14, 13, -1, -1]]
    assert slots[[0, 16, 20, 36]].tolist() == [256, 240, 224, 208]
    assert lens.tolist() == [20, 30]


# ------------------------------------------------------------------- streams

def test_a_prepared_prompts_own_workspace_outlives_its_last_call():
    """The object may go while another stream still runs its call: its
    workspace is not given away before that has ended."""
    g = torch.Generator(device=dev()).manual_seed(8)
    q, k, v = (torch.randn(3000, h, 64, generator=g, device=dev()).to(BF)
               for h in (4, 2, 2))
    out, status, cu = torch.empty_like(q), word(), i32([0, 3000])
    call = attn.prepare_prompt(q, k, v, out, cu, status)
    workspace = call._keep[1][-1]
    at, n = workspace.data_ptr(), workspace.numel()
    assert n > 0
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        torch.cuda._sleep(100_000_000)
    call(side)
    del workspace, call
    others = [torch.empty(n, dtype=torch.uint8, device=dev()) for _ in range(3)]
    still = not side.query()
    assert at not in [t.data_ptr() for t in others] and still
    side.synchronize()
    want, slack = prompt_want(q, k, v, [0, 3000], [0, 3000], 0.125,
                              ref.UNIT[BF])
    assert int(status) == 0
    ref.assert_close(out, want, slack, BF)


class Step:
    """One call of each operator: inputs, outputs and a twin of each output."""

    def __init__(self, seed):
        rng = np.random.default_rng(seed)
        self.H, self.G, self.D, self.bs, self.R = 2, 4, 128, 16, 5
        lens = [40, 700, 1, 5000, 33]
        (self.sh, self.nb, self.cache, self.rows, self.table, self.lens,
         self.q) = decode_case(rng, lens, self.H, self.G, self.D, self.bs,
                               "NHD", BF)
        self.start, self.end = self.lens, self.lens + 3
        self.new_table = torch.nn.functional.pad(self.table, (0, 2), value=-1)
        g = torch.Generator(device=dev()).manual_seed(seed)
        self.k, self.v = (torch.randn(3 * self.R, self.H, self.D, generator=g,
                                      device=dev()).to(BF) for _ in range(2))
        self.free = torch.arange(self.nb, self.nb + 20, dtype=torch.int32,
                                 device=dev())
        self.big_nb = self.nb + 20
        self.big = torch.zeros(self.sh.pool_elems(self.big_nb),
                               dtype=torch.uint8, device=dev())
        self.count = torch.tensor([20], device=dev())
        self.ws = attn.new_decode4_workspace(self.sh, self.R, self.H * self.G)
        # 3,000 queries behind 6,000 keys: planned and cut
        self.pq = torch.randn(3000, 8, 128, generator=g, device=dev()).to(BF)
        self.pk, self.pv = (torch.randn(6000, 2, 128, generator=g,
                                        device=dev()).to(BF) for _ in range(2))
        self.cu_q, self.cu_k = i32([0, 2990, 3000]), i32([0, 2990, 6000])
        self.pws = attn.new_prompt_workspace(self.pq, self.pk, 2)
        assert self.pws is not None

    def outputs(self):
        return dict(
            table=self.new_table.clone(), cache=self.big.clone(),
            slots=torch.full((15,), -9, dtype=torch.int64, device=dev()),
            cu=i32(np.zeros(self.R + 1)), lens=i32(np.zeros(self.R)),
            left=torch.zeros(1, dtype=torch.int64, device=dev()),
            k=torch.zeros_like(self.k), v=torch.zeros_like(self.v),
            out=torch.full_like(self.q, 7.0),
            prompt=torch.full_like(self.pq, 7.0), status=word())

    def arguments(self, o, workspace=True):
        """(name, arguments, keywords) of the calls, in their order."""
        st = o["status"]
        return [
            ("slots", (self.start, self.end, o["table"], self.bs, self.big_nb,
                       self.free, self.count, o["slots"], o["cu"], o["lens"],
                       o["left"], st), {}),
            ("append4", (self.sh, self.big_nb, 0, o["cache"], self.k, self.v,
                         o["slots"], st), {}),
            ("read4", (self.sh, self.big_nb, 0, o["cache"], o["slots"], o["k"],
                       o["v"], st), {}),
            ("decode4", (self.sh, self.nb, 0, self.cache, self.table,
                         self.lens, self.q, o["out"], self.ws, st), {}),
            ("prompt", (self.pq, self.pk, self.pv, o["prompt"], self.cu_q, st),
             dict(cu_k=self.cu_k, workspace=self.pws if workspace else None)),
        ]

    def call(self, o, **kw):
        for name, args, more in self.arguments(o):
            getattr(attn, "lumen_attn_" + name)(*args, **more, **kw)

    def check(self, o):
        torch.cuda.synchronize()
        assert int(o["status"]) == 0
        want, slack = decode_want(self.rows(0), self.table, self.lens, self.q,
                                  self.H, self.bs, self.D ** -0.5, BF)
        ref.assert_close(o["out"], want, slack, BF, "decode")
        want, slack = prompt_want(self.pq, self.pk, self.pv,
                                  self.cu_q.tolist(), self.cu_k.tolist(),
                                  128 ** -0.5, ref.UNIT[BF])
        ref.assert_close(o["prompt"], want, slack, BF, "prompt")
        got = ref.slots(self.start.cpu().numpy(), self.end.cpu().numpy(),
                        self.new_table.cpu().numpy(), self.bs, self.big_nb,
                        self.free.cpu().numpy(), 20, 15)
        for name, g in zip(("table", "slots", "cu", "lens"), got):
            assert np.array_equal(o[name].cpu().numpy(), g), name
        for name, x in (("k", self.k), ("v", self.v)):
            val = ref.values(*ref.quantise(x.float().cpu().numpy()))
            assert torch.equal(o[name].cpu(), torch.from_numpy(val).to(BF))


def same(a, b):
    for name in a:
        assert torch.equal(a[name], b[name]), name


def test_calls_take_a_stream():
    """stream= runs a call there, in its order, and gives the current stream's
    results; so does a current stream that is not the default one."""
    s = Step(41)
    here = s.outputs()
    s.call(here)
    s.check(here)
    side = torch.cuda.Stream()
    for inside in (False, True):
        o = s.outputs()
        side.wait_stream(torch.cuda.current_stream())
        with torch.cuda.stream(side):
            torch.cuda._sleep(100_000_000)
        if inside:
            with torch.cuda.stream(side):
                s.call(o)
        else:
            s.call(o, stream=side)
        assert not side.query()  # nothing ran elsewhere, ahead of it
        early = bool((o["out"][3] == 7.0).all())
        side.synchronize()
        assert early
        same(o, here)


def test_a_prompt_on_a_stream_of_its_own_and_a_workspace_of_the_calls():
    s = Step(42)
    here = s.outputs()
    s.call(here)
    side = torch.cuda.Stream()
    o = s.outputs()
    side.wait_stream(torch.cuda.current_stream())
    for _ in range(3):
        attn.lumen_attn_prompt(s.pq, s.pk, s.pv, o["prompt"], s.cu_q,
                               o["status"], cu_k=s.cu_k, stream=side)
    side.synchronize()
    assert int(o["status"]) == 0
    assert torch.equal(o["prompt"], here["prompt"])


@pytest.mark.parametrize("workspace", [True, False])
def test_prepared_calls_are_the_calls(workspace):
    s = Step(43)
    here, o = s.outputs(), s.outputs()
    s.call(here)
    calls = [getattr(attn, "prepare_" + name)(*args, **kw)
             for name, args, kw in s.arguments(o, workspace)]
    for c in calls:
        c()
    torch.cuda.synchronize()
    s.check(o)
    same(o, here)
    # again, on another stream, over other outputs
    side = torch.cuda.Stream()
    for name, x in s.outputs().items():
        o[name].copy_(x)
    side.wait_stream(torch.cuda.current_stream())
    for c in calls:
        c(side)
    side.synchronize()
    same(o, here)


@pytest.mark.parametrize("workspace", [True, False])
def test_a_planned_prompt_in_a_graph(workspace):
    """Plan, cut tiles and join, replayed between eager work that changes the
    inputs, each replay against the eager result."""
    s = Step(44)
    o = s.outputs()
    ws = s.pws if workspace else None

    def one(out):
        attn.lumen_attn_prompt(s.pq, s.pk, s.pv, out, s.cu_q, o["status"],
                               cu_k=s.cu_k, workspace=ws)
    one(o["prompt"])
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        one(o["prompt"])
    bounds = [([0, 2990, 3000], [0, 2990, 6000]),
              ([0, 1, 3000], [0, 3000, 6000]), ([0, 1500, 1500], [0, 10, 10]),
              ([0, 2990, 3000], [0, 2990, 6000])]
    for cu_q, cu_k in bounds:
        for t in (s.pq, s.pk, s.pv):
            t.copy_(torch.randn(t.shape, device=dev()))
        s.cu_q.copy_(i32(cu_q))
        s.cu_k.copy_(i32(cu_k))
        eager = torch.full_like(s.pq, 7.0)
        one(eager)
        o["prompt"].fill_(7.0)
        torch.cuda.synchronize()
        graph.replay()
        torch.cuda.synchronize()
        assert torch.equal(o["prompt"], eager)
        n = cu_q[-1]
        want, slack = prompt_want(s.pq[:n], s.pk, s.pv, cu_q, cu_k,
                                  128 ** -0.5, ref.UNIT[BF])
        ref.assert_close(eager[:n], want, slack, BF)
        assert bool((eager[n:] == 7.0).all()) and int(o["status"]) == 0


# -------------------------------------------------------- strides and values

def by_head(x):
    """x [tokens, heads, D] stored head by head, with a gap between them."""
    T, H, D = x.shape
    room = torch.full((H, T + 3, D + 8), float("nan"), dtype=x.dtype,
                      device=x.device)
    view = room[:, 1:T + 1, :D].transpose(0, 1)
    view.copy_(x)
    assert view.stride(1) > view.stride(0)
    return view


def test_rows_stored_head_by_head():
    s = Step(45)
    here, o = s.outputs(), s.outputs()
    s.call(here)
    st = o["status"]
    s.call(o)
    o["cache"].copy_(s.big)
    k, v = by_head(torch.zeros_like(s.k)), by_head(torch.zeros_like(s.v))
    attn.lumen_attn_append4(s.sh, s.big_nb, 0, o["cache"], by_head(s.k),
                            by_head(s.v), o["slots"], st)
    attn.lumen_attn_read4(s.sh, s.big_nb, 0, o["cache"], o["slots"], k, v, st)
    attn.lumen_attn_decode4(s.sh, s.nb, 0, s.cache, s.table, s.lens,
                            by_head(s.q), o["out"], s.ws, st)
    attn.lumen_attn_prompt(by_head(s.pq), by_head(s.pk), by_head(s.pv),
                           o["prompt"], s.cu_q, st, cu_k=s.cu_k,
                           workspace=s.pws)
    same(o, here)
    assert torch.equal(k, here["k"]) and torch.equal(v, here["v"])
    # the gaps between the rows are as they were
    assert torch.isnan(k._base[:, 0]).all() and torch.isnan(v._base[:, -1]).all()


@pytest.mark.parametrize("size,scale", [(1e30, 1e-31), (1e-30, 1e29),
                                        (1e5, 1e-6), (3e38, 1e-40)])
def test_decode_bf16_queries_of_any_size(size, scale):
    rng = np.random.default_rng(16)
    sh, nb, cache, rows, table, lens, q = decode_case(
        rng, [70, 1, 600], 2, 4, 128, 16, "NHD", BF)
    q = (q.float().clamp(-1, 1) * size).to(BF)
    want, slack = decode_want(rows(0), table, lens, q, 2, 16, scale, BF)
    ref.assert_close(run_decode(sh, nb, cache, table, lens, q, scale), want,
                     slack, BF)


@pytest.mark.parametrize("dtype", [BF, FP])
def test_decode_queries_with_elements_of_very_different_sizes(dtype):
    """One element far above the others, over keys that are 0 there: what is
    left of the others is all there is."""
    rng = np.random.default_rng(17)
    sh, nb, cache, rows, table, lens, q = decode_case(
        rng, [70, 1, 600], 2, 4, 128, 16, "NHD", dtype)
    q[..., 3] = 2.0 ** 15
    # the first quarter of every key: codes of 0 under A = 0 and B = 0
    first = rows(0)[0]
    first[..., :16] = 0
    first[..., 64:68] = 0
    want, slack = decode_want(rows(0), table, lens, q, 2, 16, 128 ** -0.5,
                              dtype)
    ref.assert_close(run_decode(sh, nb, cache, table, lens, q), want, slack,
                     dtype)


# --------------------------------------------------------- forms of a prompt

@pytest.mark.parametrize("R", [65, 128, 129, 200])
@pytest.mark.parametrize("bad", [False, True])
def test_more_sequences_than_lanes_without_a_plan(R, bad):
    """Tiles that find themselves in a second round of sequences, also behind
    bounds that are refused."""
    g = torch.Generator(device=dev()).manual_seed(R)
    n = np.random.default_rng(R).integers(1, 6, R)
    cu = np.concatenate([[0], np.cumsum(n)])
    T, H, G = int(cu[-1]), 1, 4
    q = torch.randn(T, H * G, 64, generator=g, device=dev()).to(BF)
    k, v = (torch.randn(T, H, 64, generator=g, device=dev()).to(BF)
            for _ in range(2))
    assert attn.new_prompt_workspace(q, k, R) is None
    want, slack = prompt_want(q, k, v, cu, cu, 0.125, ref.UNIT[BF])
    out, status, bounds = torch.full_like(q, 7.0), word(), cu.copy()
    if bad:
        bounds[64] = T + 1  # the 64th sequence and the one after it
        gone = slice(int(cu[63]), int(cu[65]))
        want[gone], slack[gone] = 7.0, 0.0
    attn.lumen_attn_prompt(q, k, v, out, i32(bounds), status)
    assert int(status) == (ref.RANGE if bad else 0)
    ref.assert_close(out, want, slack, BF)


@pytest.mark.parametrize("R", [65, 200])
def test_bad_bounds_past_the_first_lanes_are_recorded(R):
    """In the last sequence of all, which no tile looks for."""
    T = 2 * R
    q = torch.zeros(T, 4, 64, dtype=BF, device=dev())
    k = torch.zeros(T, 1, 64, dtype=BF, device=dev())
    cu = np.arange(0, T + 1, 2)
    cu[-1] = T + 1
    out, status = torch.full_like(q, 7.0), word()
    attn.lumen_attn_prompt(q, k, k, out, i32(cu), status)
    assert int(status) == ref.RANGE
    assert bool((out[:-2] == 0).all()) and bool((out[-2:] == 7.0).all())


@pytest.mark.parametrize("dtype,H,G,D", [(BF, 16, 4, 64), (FP, 2, 32, 128)])
def test_values_that_are_not_finite_in_larger_workgroups(dtype, H, G, D):
    """Eight wavefronts, four tiles in turn: some early, some late and some
    neighbouring values are NaN or infinite."""
    n = 2048
    g = torch.Generator(device=dev()).manual_seed(18)
    q = torch.randn(n, H * G, D, generator=g, device=dev()).to(dtype)
    k, v = (torch.randn(n, H, D, generator=g, device=dev()).to(dtype)
            for _ in range(2))
    want, slack = prompt_want(q, k, v, [0, n], [0, n], D ** -0.5,
                              ref.UNIT[dtype])
    for key, h, e, x in ((0, 0, 1, "inf"), (700, 1, 5, "nan"),
                         (701, 1, 5, "inf"), (702, 1, 6, "-inf"),
                         (703, 1, 6, "inf"), (1151, 0, D - 1, "-inf"),
                         (1152, 0, D - 2, "nan"), (n - 1, 1, 0, "inf")):
        v[key, h, e] = float(x)
        want[key:, h * G:h * G + G, e] += float(x)
    out = run_prompt(q, k, v, [0, n]).double()
    z, fine, inf = torch.zeros_like(want), want.isfinite(), want.isinf()
    assert torch.equal(out.isnan(), want.isnan())
    assert torch.equal(out.isinf(), inf) and torch.equal(out[inf], want[inf])
    ref.assert_close(torch.where(fine, out, z), torch.where(fine, want, z),
                     torch.where(fine, slack, z), dtype)


def test_a_prepared_prompt_with_its_own_workspace_in_a_graph():
    """Captured on a stream that is not the workspace's, and replayed between
    eager work."""
    s = Step(46)
    o, here = s.outputs(), s.outputs()
    call = attn.prepare_prompt(s.pq, s.pk, s.pv, o["prompt"], s.cu_q,
                               o["status"], cu_k=s.cu_k)
    call()
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        call()
    for _ in range(3):
        for t in (s.pq, s.pk, s.pv):
            t.copy_(torch.randn(t.shape, device=dev()))
        attn.lumen_attn_prompt(s.pq, s.pk, s.pv, here["prompt"], s.cu_q,
                               here["status"], cu_k=s.cu_k, workspace=s.pws)
        o["prompt"].fill_(7.0)
        torch.cuda.synchronize()
        graph.replay()
        torch.cuda.synchronize()
        assert torch.equal(o["prompt"], here["prompt"])
        assert int(o["status"]) == 0


def test_slots_of_an_empty_map():
    """A map without room for the tokens there are is an error; None is not."""
    for slots, tokens, want in ((0, 3, ref.CAPACITY), (0, 0, 0), (None, 3, 0)):
        table, status = i32(np.full((1, 2), -1)), word()
        cu, lens, left = i32([0, 0]), i32([0]), torch.zeros(
            1, dtype=torch.int64, device=dev())
        if slots is not None:
            slots = torch.empty(0, dtype=torch.int64, device=dev())
        attn.lumen_attn_slots(i32([0]), i32([tokens]), table, 16, 9,
                              i32([3, 4]), torch.tensor([2], device=dev()),
                              slots, cu, lens, left, status)
        assert int(status) == want
        assert cu.tolist() == [0, tokens] and lens.tolist() == [tokens]
        assert table[0, 0] == (4 if tokens else -1)
