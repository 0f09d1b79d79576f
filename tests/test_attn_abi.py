"""The serving operators' C ABI without a GPU: exports, refusals before any
HIP call (the fake pointers are never dereferenced) and the binding's checks;
and the 4-bit row format's own properties."""
import ctypes
import re

import numpy as np
import pytest
import torch

import attn_ref as ref
import paper_2606_17787_amd.kvckpt as kv
from paper_2606_17787_amd import attn

FAKE = 0x7F0000000000
ODD = FAKE + 2
OK_OR_HIP = (kv.LUMEN_OK, kv.LUMEN_ERR_HIP)


@pytest.fixture(scope="module")
def lib():
    return attn._lib()


def rows(base=FAKE, token=512, head=128):
    return ctypes.byref(attn.lumen_attn_rows(base, token, head))


def layout(**kw):
    d = dict(num_layers=2, num_kv_heads=2, head_dim=80, block_size=16,
             num_blocks=8, elem_bytes=1, cache_order=kv.LUMEN_CACHE_NHD)
    d.update(kw)
    return ctypes.byref(kv.lumen_kv_layout(**d))


def test_exports_every_declared_entry_point(lib):
    names = attn.exported_names()
    assert set(names) == {"lumen_attn_slots", "lumen_attn_append4",
                          "lumen_attn_read4", "lumen_attn_decode4",
                          "lumen_attn_decode4_workspace_bytes",
                          "lumen_attn_prompt",
                          "lumen_attn_prompt_workspace_bytes"}
    for n in names:
        assert hasattr(lib, n), n


def test_binding_constants_match_the_header():
    text = open(attn.HEADER).read()
    defines = dict(re.findall(r"^#define (LUMEN_ATTN_\w+) (\d+)$", text, re.M))
    names = [n for n in dir(attn) if n.startswith("LUMEN_ATTN_")]
    assert set(names) == set(defines)
    for n in names:
        assert getattr(attn, n) == int(defines[n])


def test_slots_refusals(lib):
    def call(s=FAKE, e=FAKE, have=None, R=2, bt=FAKE, cols=4, bs=16, nb=8,
             free=FAKE, count=FAKE, cap=8, slots=FAKE, n=10, cu=FAKE,
             lens=FAKE, left=FAKE, status=FAKE):
        return lib.lumen_attn_slots(s, e, have, R, bt, cols, bs, nb, free,
                                    count, cap, slots, n, cu, lens, left,
                                    status, None)
    bad = kv.LUMEN_ERR_INVALID_ARG
    for kw in (dict(R=-1), dict(cols=-1), dict(bs=0), dict(nb=-1),
               dict(cap=-1), dict(n=-1), dict(s=None), dict(e=None),
               dict(bt=None), dict(free=None), dict(count=None),
               dict(slots=None), dict(cu=None), dict(lens=None),
               dict(left=None), dict(status=None)):
        assert call(**kw) == bad, kw
    assert call(R=attn.LUMEN_ATTN_MAX_REQS + 1) == kv.LUMEN_ERR_TOO_MANY
    for kw in (dict(status=ODD), dict(slots=FAKE + 4), dict(count=FAKE + 4),
               dict(left=FAKE + 4), dict(s=ODD), dict(e=ODD), dict(have=ODD),
               dict(bt=ODD), dict(free=ODD), dict(cu=ODD), dict(lens=ODD)):
        assert call(**kw) == kv.LUMEN_ERR_MISALIGNED, kw


LAYOUT_BAD = [dict(num_layers=0), dict(num_kv_heads=0), dict(block_size=0),
              dict(num_blocks=-1), dict(num_blocks=1 << 60)]
LAYOUT_UNSUPPORTED = [dict(elem_bytes=2), dict(head_dim=64),
                      dict(head_dim=96), dict(cache_order=2),
                      dict(block_size=1 << 30)]


@pytest.mark.parametrize("fn", ["append4", "read4"])
def test_append_and_read_refusals(lib, fn):
    def call(lay=None, layer=0, cache=FAKE, k=None, v=None, dtype=0,
             slots=FAKE, n=3, status=FAKE):
        lay = layout() if lay is None else lay
        k = rows() if k is None else k
        v = rows() if v is None else v
        if fn == "append4":
            return lib.lumen_attn_append4(lay, layer, cache, k, v, dtype,
                                          slots, n, status, None)
        return lib.lumen_attn_read4(lay, layer, cache, slots, n, k, v, dtype,
                                    status, None)
    for kw in LAYOUT_BAD:
        assert call(lay=layout(**kw)) == kv.LUMEN_ERR_INVALID_ARG, kw
    for kw in LAYOUT_UNSUPPORTED:
        assert call(lay=layout(**kw)) == kv.LUMEN_ERR_UNSUPPORTED, kw
    for kw in (dict(layer=-1), dict(layer=2), dict(cache=None),
               dict(slots=None), dict(n=-1), dict(status=None),
               dict(k=rows(None)), dict(v=rows(None)),
               dict(k=rows(token=-8)), dict(v=rows(head=-8))):
        assert call(**kw) == kv.LUMEN_ERR_INVALID_ARG, kw
    assert call(dtype=2) == kv.LUMEN_ERR_UNSUPPORTED
    for kw in (dict(cache=FAKE + 8), dict(slots=FAKE + 4), dict(status=ODD),
               dict(k=rows(FAKE + 8)), dict(v=rows(token=4)),
               dict(k=rows(head=12))):
        assert call(**kw) == kv.LUMEN_ERR_MISALIGNED, kw
    assert call(n=0, cache=None, slots=None, k=rows(None),
                v=rows(None)) == kv.LUMEN_OK


def test_decode_refusals(lib):
    def call(lay=None, layer=0, cache=FAKE, bt=FAKE, cols=4, lens=FAKE, R=2,
             q=None, dtype=0, hq=8, scale=0.1, out=FAKE, ws=FAKE,
             wsb=1 << 40, status=FAKE):
        lay = layout() if lay is None else lay
        q = rows() if q is None else q
        return lib.lumen_attn_decode4(lay, layer, cache, bt, cols, lens, R, q,
                                      dtype, hq, scale, out, ws, wsb, status,
                                      None)
    for kw in LAYOUT_BAD:
        assert call(lay=layout(**kw)) == kv.LUMEN_ERR_INVALID_ARG, kw
    for kw in LAYOUT_UNSUPPORTED:
        assert call(lay=layout(**kw)) == kv.LUMEN_ERR_UNSUPPORTED, kw
    need = lib.lumen_attn_decode4_workspace_bytes(layout(), 2, 8)
    assert need > 0
    for kw in (dict(layer=2), dict(cache=None), dict(bt=None), dict(cols=-1),
               dict(lens=None), dict(R=-1), dict(q=rows(None)), dict(hq=0),
               dict(hq=3), dict(scale=0.0), dict(scale=-1.0),
               dict(scale=float("nan")), dict(scale=float("inf")),
               dict(out=None), dict(ws=None), dict(wsb=need - 1),
               dict(status=None), dict(q=rows(token=-8))):
        assert call(**kw) == kv.LUMEN_ERR_INVALID_ARG, kw
    assert call(dtype=-1) == kv.LUMEN_ERR_UNSUPPORTED
    assert call(R=attn.LUMEN_ATTN_MAX_REQS + 1) == kv.LUMEN_ERR_TOO_MANY
    for kw in (dict(cache=FAKE + 8), dict(bt=ODD), dict(lens=ODD),
               dict(out=FAKE + 8), dict(ws=FAKE + 8), dict(status=ODD),
               dict(q=rows(FAKE + 8)), dict(q=rows(head=4))):
        assert call(**kw) == kv.LUMEN_ERR_MISALIGNED, kw
    assert call(R=0, lens=None, bt=None, out=None, ws=None, wsb=0,
                q=rows(None)) == kv.LUMEN_OK


def test_decode_workspace_bytes(lib):
    f = lib.lumen_attn_decode4_workspace_bytes
    assert f(layout(), -1, 8) == 0 and f(layout(), 2, 3) == 0
    assert f(layout(head_dim=64), 2, 8) == 0 and f(None, 2, 8) == 0
    assert f(layout(), attn.LUMEN_ATTN_MAX_REQS + 1, 8) == 0
    for R in (0, 1, 100, 4096):
        assert 0 < f(layout(), R, 8) < 1 << 31


def test_prompt_refusals(lib):
    def call(q=None, k=None, v=None, dtype=0, cu_q=FAKE, cu_k=FAKE, S=2,
             tq=10, tk=10, hq=8, h=2, d=128, scale=0.1, out=FAKE,
             status=FAKE, ws=None, wsb=0):
        q, k, v = (rows() if x is None else x for x in (q, k, v))
        return lib.lumen_attn_prompt(q, k, v, dtype, cu_q, cu_k, S, tq, tk,
                                     hq, h, d, scale, out, ws, wsb, status,
                                     None)
    for kw in (dict(S=-1), dict(tq=-1), dict(tk=-1), dict(hq=0), dict(h=0),
               dict(h=3), dict(scale=0.0), dict(scale=float("nan")),
               dict(scale=float("inf")), dict(cu_q=None), dict(out=None),
               dict(status=None), dict(q=rows(None)), dict(k=rows(None)),
               dict(v=rows(None)), dict(k=rows(token=-8)),
               dict(cu_k=None, tk=11)):
        assert call(**kw) == kv.LUMEN_ERR_INVALID_ARG, kw
    for kw in (dict(dtype=2), dict(d=256), dict(d=96), dict(tq=1 << 31),
               dict(tk=1 << 31)):
        assert call(**kw) == kv.LUMEN_ERR_UNSUPPORTED, kw
    far = rows(token=(1 << 24) + 8)
    assert call(k=far) == kv.LUMEN_ERR_UNSUPPORTED
    assert call(v=far) == kv.LUMEN_ERR_UNSUPPORTED
    assert call(S=0, tq=1, tk=1, k=far, v=far) == kv.LUMEN_OK
    assert call(S=attn.LUMEN_ATTN_MAX_REQS + 1) == kv.LUMEN_ERR_TOO_MANY
    for kw in (dict(cu_q=ODD), dict(cu_k=ODD), dict(out=FAKE + 8),
               dict(status=ODD), dict(q=rows(FAKE + 8)),
               dict(v=rows(head=4))):
        assert call(**kw) == kv.LUMEN_ERR_MISALIGNED, kw
    assert call(S=0, cu_q=None, tq=0, tk=0, out=None, q=rows(None),
                k=rows(None), v=rows(None)) == kv.LUMEN_OK


def test_prompt_workspace(lib):
    f = lib.lumen_attn_prompt_workspace_bytes
    assert f(2, 10, 10, 8, 2, 128) == 0 and f(2, 10, 9000, 8, 2, 96) == 0
    assert f(2, 10, 9000, 8, 3, 128) == 0 and f(-1, 10, 9000, 8, 2, 128) == 0
    most = 0
    for s, tq, tk in ((1, 1, 5000), (3, 100, 100000), (9, 1 << 27, 1 << 27)):
        n = f(s, tq, tk, 8, 2, 128)
        assert 0 < n < 1 << 28 and n >= most
        most = n


def test_workspace_of_refused_sizes(lib):
    """0 for every size that the call itself refuses."""
    f = lib.lumen_attn_decode4_workspace_bytes
    assert f(layout(num_kv_heads=1), 2, 65535) > 0
    assert f(layout(num_kv_heads=1), 2, 65536) == 0
    g = lib.lumen_attn_prompt_workspace_bytes
    assert g(1, 1 << 27, 1 << 27, 8, 8, 128) > 0
    # 2^27 tokens of 4,096 heads: more workgroups than a launch takes
    assert g(1, 1 << 27, 1 << 27, 4096, 4096, 128) == 0
    assert lib.lumen_attn_prompt(
        rows(), rows(), rows(), 0, FAKE, FAKE, 1, 1 << 27, 1 << 27, 4096,
        4096, 128, 0.1, FAKE, FAKE, 1 << 40, FAKE, None) < 0


def test_binding_refuses_host_tensors_and_shapes():
    sh = attn.cache_shape4(1, 2, 128, 16)
    with pytest.raises(ValueError, match="head_dim 96"):
        attn.cache_shape4(1, 2, 96, 16)
    cache = torch.zeros(sh.pool_elems(2), dtype=torch.uint8)
    x = torch.zeros(3, 2, 128, dtype=torch.bfloat16)
    slots = torch.zeros(3, dtype=torch.int64)
    status = torch.zeros(1, dtype=torch.int32)
    with pytest.raises(ValueError):
        attn.lumen_attn_append4(sh, 2, 0, cache, x, x, slots, status)
    with pytest.raises(ValueError, match="one row per slot"):
        attn.lumen_attn_append4(sh, 2, 0, cache, x[:2], x, slots, status)
    with pytest.raises(ValueError, match="the layout needs"):
        attn.lumen_attn_append4(sh, 3, 0, cache, x, x, slots, status)
    with pytest.raises(ValueError, match="k and v differ"):
        attn.lumen_attn_prompt(x, x, x[:, :1], x, torch.zeros(2), status)
    assert attn.head_dim4(sh) == 128 and sh.head_dim == 80


def test_row_format_round_trip():
    """Codes of values the format holds come back as they were, and a quarter
    covers its range within half a step."""
    rng = np.random.default_rng(1)
    x = rng.standard_normal((50, 128)).astype(np.float32)
    q, A, B = ref.quantise(x)
    v = ref.values(q, A, B).astype(np.float32)
    back = ref.from_rows(torch.from_numpy(ref.to_rows(q, A, B)))
    assert np.array_equal(back.numpy(), v.astype(np.float64))
    step = A.astype(np.float32).repeat(32, -1)
    assert (np.abs(v - x) <= step * (0.5 + 79 * 2.0 ** -11) + 2.0 ** -8).all()
    # the extreme elements take the extreme codes
    y = x.reshape(50, 4, 32)
    lowest = q.reshape(50, 4, 32)[y == y.min(-1, keepdims=True)]
    assert (lowest == 0).all()
    assert (q.reshape(50, 4, 32)[y == y.max(-1, keepdims=True)] == 15).all()


def test_scales_past_the_range_of_the_exponent(lib):
    """A scale that times log2(e) is infinite makes every score infinite or
    NaN: refused."""
    def decode(scale):  # of no requests
        return lib.lumen_attn_decode4(layout(), 0, FAKE, FAKE, 4, FAKE, 0,
                                      rows(), 0, 8, scale, FAKE, FAKE, 0, FAKE,
                                      None)

    def prompt(scale):  # of no sequences
        return lib.lumen_attn_prompt(rows(), rows(), rows(), 0, FAKE, FAKE, 0,
                                     10, 10, 8, 2, 128, scale, FAKE, None, 0,
                                     FAKE, None)
    for call in (decode, prompt):
        assert call(2e38) == kv.LUMEN_OK
        for scale in (2.4e38, 3.4e38):
            assert call(scale) == kv.LUMEN_ERR_INVALID_ARG


def test_prompt_refuses_more_threads_than_a_launch_takes(lib):
    """Heads so many that a few sequences need 2^32 threads: refused before
    anything is enqueued, and without a workspace."""
    g = lib.lumen_attn_prompt_workspace_bytes

    def call(heads):
        return lib.lumen_attn_prompt(
            rows(), rows(), rows(), 0, FAKE, FAKE, 3, 3, 3, heads, heads, 64,
            0.1, FAKE, FAKE, 1 << 40, FAKE, None)
    # three tiles of 256 threads a head
    assert g(3, 3, 3, 5592405, 5592405, 64) > 0
    for heads in (5592406, 1 << 25, (1 << 31) - 1):
        assert g(3, 3, 3, heads, heads, 64) == 0
        assert call(heads) == kv.LUMEN_ERR_UNSUPPORTED
