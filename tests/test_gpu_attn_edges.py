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
