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
