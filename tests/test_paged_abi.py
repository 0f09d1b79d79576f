"""The 16-bit paged cache's C ABI without a GPU: exports, refusals before any HIP
call (the fake pointers are never dereferenced), workspace sizes and the binding's
checks; and the compiled text of the loads into LDS."""
import ctypes
import os
import re
import subprocess

import numpy as np
import pytest
import torch

import paged_ref as ref
import paper_2606_17787_amd.kvckpt as kv
from paper_2606_17787_amd import attn, build, paged
from paper_2606_17787_amd.workloads import CacheShape, HND, NHD

FAKE = 0x7F0000000000
ODD = FAKE + 2
BAD, UNSUPPORTED = kv.LUMEN_ERR_INVALID_ARG, kv.LUMEN_ERR_UNSUPPORTED


@pytest.fixture(scope="module")
def lib():
    return paged._lib()


def rows(base=FAKE, token=512, head=128):
    return ctypes.byref(attn.lumen_attn_rows(base, token, head))


def layout(**kw):
    d = dict(num_layers=2, num_kv_heads=2, head_dim=128, block_size=16,
             num_blocks=8, elem_bytes=2, cache_order=kv.LUMEN_CACHE_NHD)
    d.update(kw)
    return ctypes.byref(kv.lumen_kv_layout(**d))


def test_exports_every_declared_entry_point(lib):
    names = paged.exported_names()
    assert set(names) == {
        "lumen_paged_append", "lumen_paged_attend",
        "lumen_paged_attend_workspace_bytes", "lumen_paged_weigh",
        "lumen_paged_weigh_workspace_bytes", "lumen_paged_evict",
        "lumen_paged_evict_workspace_bytes", "lumen_paged_release"}
    for n in names:
        assert hasattr(lib, n), n


def test_binding_constants_match_the_header():
    text = open(paged.HEADER).read()
    defines = dict(re.findall(r"^#define (LUMEN_PAGED_\w+) (\d+)$", text, re.M))
    names = [n for n in dir(paged) if n.startswith("LUMEN_PAGED_")]
    assert set(names) == set(defines)
    for n in names:
        assert getattr(paged, n) == int(defines[n])


LAYOUT_BAD = [dict(num_layers=0), dict(num_kv_heads=0), dict(block_size=0),
              dict(num_blocks=-1), dict(num_blocks=1 << 60)]
LAYOUT_UNSUPPORTED = [dict(elem_bytes=1), dict(elem_bytes=4), dict(head_dim=96),
                      dict(head_dim=80), dict(cache_order=2),
                      dict(block_size=1 << 28)]


def test_append_refusals(lib):
    def call(lay=None, layer=0, cache=FAKE, k=None, v=None, slots=FAKE,
             pos=FAKE, n=3, ledger=FAKE, status=FAKE):
        return lib.lumen_paged_append(
            layout() if lay is None else lay, layer, cache,
            rows() if k is None else k, rows() if v is None else v, slots, pos,
            n, ledger, status, None)
    for kw in LAYOUT_BAD:
        assert call(lay=layout(**kw)) == BAD, kw
    for kw in LAYOUT_UNSUPPORTED:
        assert call(lay=layout(**kw)) == UNSUPPORTED, kw
    for kw in (dict(layer=-1), dict(layer=2), dict(cache=None),
               dict(slots=None), dict(n=-1), dict(status=None), dict(pos=None),
               dict(ledger=None), dict(k=rows(None)), dict(v=rows(None)),
               dict(k=rows(token=-8)), dict(v=rows(head=-8))):
        assert call(**kw) == BAD, kw
    for kw in (dict(cache=FAKE + 8), dict(slots=FAKE + 4), dict(status=ODD),
               dict(pos=ODD), dict(ledger=ODD), dict(k=rows(FAKE + 8)),
               dict(v=rows(token=4)), dict(k=rows(head=12))):
        assert call(**kw) == kv.LUMEN_ERR_MISALIGNED, kw
    assert call(n=0, cache=None, slots=None, k=rows(None), v=rows(None),
                pos=None, ledger=None) == kv.LUMEN_OK


@pytest.mark.parametrize("fn", ["attend", "weigh"])
def test_attend_and_weigh_refusals(lib, fn):
    size = getattr(lib, f"lumen_paged_{fn}_workspace_bytes")

    def call(lay=None, layer=0, cache=FAKE, bt=FAKE, cols=400, lens=FAKE,
             cu=FAKE, R=2, q=None, T=10, new=10, dtype=0, hq=8, scale=0.1,
             out=FAKE, lse=FAKE, ledger=FAKE, ws=FAKE, wsb=1 << 40,
             status=FAKE):
        lay = layout() if lay is None else lay
        q = rows() if q is None else q
        last = (ws, wsb, status, None)
        if fn == "attend":
            return lib.lumen_paged_attend(lay, layer, cache, bt, cols, lens,
                                          cu, R, q, T, new, dtype, hq, scale,
                                          out, lse, *last)
        return lib.lumen_paged_weigh(lay, layer, cache, bt, cols, lens, cu, R,
                                     q, T, new, dtype, hq, scale, lse, ledger,
                                     *last)
    for kw in LAYOUT_BAD:
        assert call(lay=layout(**kw)) == BAD, kw
    for kw in LAYOUT_UNSUPPORTED + [dict(head_dim=256)]:
        assert call(lay=layout(**kw)) == UNSUPPORTED, kw
    need = size(layout(), 400, 2, 10, 10, 8)
    bad = [dict(layer=2), dict(layer=-1), dict(cache=None), dict(bt=None),
           dict(cols=-1), dict(lens=None), dict(cu=None), dict(R=-1),
           dict(q=rows(None)), dict(T=-1), dict(new=-1), dict(hq=0),
           dict(hq=3), dict(scale=0.0), dict(scale=-1.0),
           dict(scale=float("nan")), dict(scale=float("inf")),
           dict(scale=2.4e38), dict(status=None), dict(q=rows(token=-8))]
    if fn == "attend":
        assert need > 0
        bad += [dict(out=None), dict(ws=None), dict(wsb=need - 1)]
    else:
        bad += [dict(lse=None), dict(ledger=None)]
    for kw in bad:
        assert call(**kw) == BAD, kw
    for kw in (dict(dtype=2), dict(T=1 << 31, new=1), dict(T=1 << 29)):
        assert call(**kw) == UNSUPPORTED, kw
    assert call(R=attn.LUMEN_ATTN_MAX_REQS + 1) == kv.LUMEN_ERR_TOO_MANY
    odd = [dict(cache=FAKE + 8), dict(bt=ODD), dict(lens=ODD), dict(cu=ODD),
           dict(ws=FAKE + 8), dict(lse=ODD), dict(status=ODD),
           dict(q=rows(FAKE + 8)), dict(q=rows(head=4))]
    odd.append(dict(out=FAKE + 8) if fn == "attend" else dict(ledger=ODD))
    for kw in odd:
        assert call(**kw) == kv.LUMEN_ERR_MISALIGNED, kw
    nothing = dict(lens=None, cu=None, bt=None, out=None, lse=None, ledger=None,
                   ws=None, wsb=0, cache=None)
    assert call(R=0, **nothing) == kv.LUMEN_OK
    assert call(T=0, q=rows(None), **nothing) == kv.LUMEN_OK


def test_attend_workspace(lib):
    f = lib.lumen_paged_attend_workspace_bytes
    assert f(layout(), 400, -1, 10, 10, 8) == 0
    assert f(layout(), 400, 2, 10, 10, 3) == 0
    assert f(layout(head_dim=256), 400, 2, 10, 10, 8) == 0
    assert f(None, 400, 2, 10, 10, 8) == 0
    assert f(layout(), 4, 2, 10, 10, 8) == 0  # nothing to cut or to plan
    for R, T in ((1, 1), (100, 100), (4096, 4096), (9, 1 << 20)):
        assert 0 < f(layout(), 10000, R, T, T, 8) < 1 << 30
    # as many threads as a launch takes, and more
    many = layout(num_kv_heads=1 << 20, head_dim=64, block_size=1)
    assert f(many, 1, 15, 15, 1, 1 << 20) >= 0
    assert lib.lumen_paged_attend(
        many, 0, FAKE, FAKE, 1, FAKE, FAKE, 17, rows(), 17, 1, 0, 1 << 20, 0.1,
        FAKE, None, FAKE, 1 << 40, FAKE, None) == UNSUPPORTED


def test_evict_refusals(lib):
    def call(lay=None, first=0, layers=2, cache=FAKE, ledger=FAKE, bt=FAKE,
             cols=4, lens=FAKE, keep=FAKE, frm=FAKE, sinks=0, R=2, left=FAKE,
             ws=FAKE, wsb=1 << 40, status=FAKE):
        return lib.lumen_paged_evict(
            layout() if lay is None else lay, first, layers, cache, ledger, bt,
            cols, lens, keep, frm, sinks, R, left, ws, wsb, status, None)
    for kw in LAYOUT_BAD:
        assert call(lay=layout(**kw)) == BAD, kw
    for kw in LAYOUT_UNSUPPORTED:
        assert call(lay=layout(**kw)) == UNSUPPORTED, kw
    need = lib.lumen_paged_evict_workspace_bytes(layout(), 2, 4, 2)
    assert need > 0
    for kw in (dict(first=-1), dict(first=1), dict(layers=0), dict(layers=3),
               dict(layers=-1), dict(cache=None), dict(ledger=None),
               dict(bt=None), dict(cols=-1), dict(lens=None), dict(keep=None),
               dict(frm=None), dict(R=-1), dict(left=None), dict(ws=None),
               dict(wsb=need - 1), dict(status=None)):
        assert call(**kw) == BAD, kw
    most = paged.LUMEN_PAGED_MAX_PLACES // 16
    assert call(cols=most + 1) == UNSUPPORTED
    assert lib.lumen_paged_evict_workspace_bytes(layout(), 2, most + 1, 2) == 0
    assert lib.lumen_paged_evict_workspace_bytes(layout(), 2, most, 2) > 0
    assert call(R=attn.LUMEN_ATTN_MAX_REQS + 1) == kv.LUMEN_ERR_TOO_MANY
    many = layout(num_layers=200, num_kv_heads=16)
    assert call(lay=many, layers=200, R=4096) == UNSUPPORTED
    for kw in (dict(cache=FAKE + 8), dict(ledger=ODD), dict(bt=ODD),
               dict(lens=ODD), dict(keep=ODD), dict(frm=ODD), dict(left=ODD),
               dict(ws=FAKE + 8), dict(status=ODD)):
        assert call(**kw) == kv.LUMEN_ERR_MISALIGNED, kw
    assert call(R=0, cache=None, ledger=None, bt=None, lens=None, keep=None,
                frm=None, left=None, ws=None, wsb=0) == kv.LUMEN_OK


def test_release_refusals(lib):
    def call(lens=FAKE, have=FAKE, R=2, bt=FAKE, cols=4, bs=16, nb=8,
             free=FAKE, count=FAKE, cap=8, now=FAKE, status=FAKE):
        return lib.lumen_paged_release(lens, have, R, bt, cols, bs, nb, free,
                                       count, cap, now, status, None)
    for kw in (dict(R=-1), dict(cols=-1), dict(bs=0), dict(nb=-1),
               dict(cap=-1), dict(lens=None), dict(have=None), dict(bt=None),
               dict(free=None), dict(count=None), dict(now=None),
               dict(status=None)):
        assert call(**kw) == BAD, kw
    assert call(R=attn.LUMEN_ATTN_MAX_REQS + 1) == kv.LUMEN_ERR_TOO_MANY
    for kw in (dict(lens=ODD), dict(have=ODD), dict(bt=ODD), dict(free=ODD),
               dict(count=FAKE + 4), dict(now=FAKE + 4), dict(status=ODD)):
        assert call(**kw) == kv.LUMEN_ERR_MISALIGNED, kw


def apart(*names):
    return {name: FAKE + (i << 20) for i, name in enumerate(names)}


@pytest.mark.parametrize("name,bytes_", [("lens", 8), ("keep", 8), ("frm", 8),
                                         ("bt", 32)])
@pytest.mark.parametrize("by", ["all", "first", "last"])
def test_evict_refuses_results_among_its_inputs(lib, name, bytes_, by):
    """Other workgroups read the inputs while d_left is written."""
    at = apart("cache", "ledger", "bt", "lens", "keep", "frm", "left", "ws",
               "status")
    at["left"] = at[name] + {"all": 0, "first": -4, "last": bytes_ - 4}[by]
    assert lib.lumen_paged_evict(
        layout(), 0, 2, at["cache"], at["ledger"], at["bt"], 4, at["lens"],
        at["keep"], at["frm"], 0, 2, at["left"], at["ws"], 1 << 16,
        at["status"], None) == BAD


@pytest.mark.parametrize("name,bytes_", [("lens", 8), ("have", 8),
                                         ("count", 8), ("bt", 32),
                                         ("free", 64)])
def test_release_refuses_its_count_among_its_inputs(lib, name, bytes_):
    at = apart("lens", "have", "bt", "free", "count", "now", "status")
    for now in (at[name], at[name] + bytes_ - 8):
        assert lib.lumen_paged_release(
            at["lens"], at["have"], 2, at["bt"], 4, 16, 8, at["free"],
            at["count"], 16, now, at["status"], None) == BAD


@pytest.mark.parametrize("result,bytes_", [("free", 64), ("now", 8),
                                           ("status", 4)])
@pytest.mark.parametrize("name,size", [("lens", 8), ("have", 8), ("count", 8),
                                       ("bt", 32), ("free", 64), ("now", 8),
                                       ("status", 4)])
def test_release_refuses_results_that_overlap(lib, result, bytes_, name, size):
    """Its workgroups read the inputs while they write the list, its count and
    the status word."""
    if result == name:
        return
    need = {"free": 4, "now": 8, "status": 4}[result]
    for to in (0, 4 - bytes_, size - 4):
        at = apart("lens", "have", "bt", "free", "count", "now", "status")
        at[result] = at[name] + (to if to % need == 0 else 0)
        assert lib.lumen_paged_release(
            at["lens"], at["have"], 2, at["bt"], 4, 16, 8, at["free"],
            at["count"], 16, at["now"], at["status"], None) == BAD


@pytest.mark.parametrize("result,bytes_", [("left", 8), ("status", 4)])
@pytest.mark.parametrize("name,size", [("lens", 8), ("keep", 8), ("frm", 8),
                                       ("bt", 32), ("cache", 1 << 18),
                                       ("ledger", 1 << 12), ("ws", 256),
                                       ("left", 8), ("status", 4)])
def test_evict_refuses_results_that_overlap(lib, result, bytes_, name, size):
    if result == name:
        return
    for to in (0, 4 - bytes_, size - 4):
        at = apart("cache", "ledger", "bt", "lens", "keep", "frm", "left", "ws",
                   "status")
        at[result] = at[name] + to
        assert lib.lumen_paged_evict(
            layout(), 0, 2, at["cache"], at["ledger"], at["bt"], 4, at["lens"],
            at["keep"], at["frm"], 0, 2, at["left"], at["ws"], 1 << 16,
            at["status"], None) == BAD


def wide_apart():
    names = ("cache", "bt", "lens", "cu", "q", "out", "lse", "status", "ledger",
             "ws")
    return {name: FAKE + (i << 26) for i, name in enumerate(names)}


@pytest.mark.parametrize("result,bytes_", [("out", 20480), ("lse", 320),
                                           ("ws", 256), ("status", 4)])
@pytest.mark.parametrize("name,size", [("cache", 1 << 17), ("bt", 3200),
                                       ("lens", 8), ("cu", 12), ("q", 20480),
                                       ("out", 20480), ("lse", 320),
                                       ("ws", 256), ("status", 4)])
def test_attend_refuses_results_that_overlap(lib, result, bytes_, name, size):
    """Among the plan of the workspace, or what other workgroups read.  (Two
    layers' cache, of which the second is attended to.)"""
    if result == name:
        return
    need = {"out": 16, "ws": 16}.get(result, 4)
    for to in (need, need - bytes_, size - need):
        if to % need or to >= size:
            continue
        at = wide_apart()
        at[result] = at[name] + to + (name == "cache") * (1 << 17)
        assert lib.lumen_paged_attend(
            layout(), 1, at["cache"], at["bt"], 400, at["lens"], at["cu"], 2,
            rows(at["q"], 1024, 128), 10, 10, 0, 8, 0.1, at["out"], at["lse"],
            at["ws"], 1 << 26, at["status"], None) == BAD, to


@pytest.mark.parametrize("result,bytes_", [("ledger", 2048), ("status", 4)])
@pytest.mark.parametrize("name,size", [("cache", 1 << 17), ("bt", 3200),
                                       ("lens", 8), ("cu", 12), ("q", 20480),
                                       ("lse", 320), ("ledger", 2048),
                                       ("status", 4)])
def test_weigh_refuses_results_that_overlap(lib, result, bytes_, name, size):
    if result == name:
        return
    for to in (0, 4 - bytes_, size - 4):
        at = wide_apart()
        # the second layer's words and rows
        at[result] = at[name] + to + {"cache": 1 << 17, "ledger": 2048}.get(
            name, 0) - 2048 * (result == "ledger")
        assert lib.lumen_paged_weigh(
            layout(), 1, at["cache"], at["bt"], 400, at["lens"], at["cu"], 2,
            rows(at["q"], 1024, 128), 10, 10, 0, 8, 0.1, at["lse"],
            at["ledger"], None, 0, at["status"], None) == BAD, to


@pytest.mark.parametrize("result,bytes_", [("cache", 1 << 17), ("ledger", 2048),
                                           ("status", 4)])
@pytest.mark.parametrize("name,size", [("slots", 24), ("pos", 12),
                                       ("ledger", 2048), ("status", 4),
                                       ("cache", 1 << 17)])
def test_append_refuses_results_that_overlap(lib, result, bytes_, name, size):
    if result == name:
        return
    need = {"cache": 16}.get(result, 4)
    for to in (0, need - bytes_, size - need):
        if to % need or to >= size:
            continue
        at = apart("cache", "k", "v", "slots", "pos", "ledger", "status")
        layer = {"cache": 1 << 17, "ledger": 2048}  # from a layer to the next
        at[result] = at[name] + to + layer.get(name, 0) - layer.get(result, 0)
        assert lib.lumen_paged_append(
            layout(), 1, at["cache"], rows(at["k"], 256), rows(at["v"], 256),
            at["slots"], at["pos"], 3, at["ledger"], at["status"], None) == BAD


def test_binding_refuses_host_tensors_and_shapes():
    sh = CacheShape(2, 2, 128, 16, NHD)
    cache = torch.zeros(sh.pool_elems(2), dtype=torch.bfloat16)
    x = torch.zeros(3, 2, 128, dtype=torch.bfloat16)
    slots = torch.zeros(3, dtype=torch.int64)
    word = torch.zeros(1, dtype=torch.int32)
    led = torch.zeros(paged.ledger_dims(sh, 2), dtype=torch.int32)
    with pytest.raises(ValueError, match="device tensor"):
        paged.lumen_paged_append(sh, 2, 0, cache, x, x, slots, word)
    with pytest.raises(ValueError, match="one row per slot"):
        paged.lumen_paged_append(sh, 2, 0, cache, x[:2], x, slots, word)
    with pytest.raises(ValueError, match="as the cache"):
        paged.lumen_paged_append(sh, 2, 0, cache, x.half(), x, slots, word)
    with pytest.raises(ValueError, match="come together"):
        paged.lumen_paged_append(sh, 2, 0, cache, x, x, slots, word, ledger=led)
    with pytest.raises(ValueError, match="the layout needs"):
        paged.lumen_paged_append(sh, 3, 0, cache, x, x, slots, word)
    lens, table = torch.zeros(2, dtype=torch.int32), torch.zeros(2, 4)
    for kw, match in ((dict(cu=lens), "num_reqs"), (dict(q=x[0]), "q must be"),
                      (dict(q=x.half()), "as the cache"),
                      (dict(table=table[:1]), "block_tables")):
        with pytest.raises(ValueError, match=match):
            paged.lumen_paged_attend(
                sh, 2, 0, cache, kw.get("table", table), lens,
                kw.get("cu", torch.zeros(3)), kw.get("q", x), x, word)
    with pytest.raises(ValueError, match="keep must have"):
        paged.lumen_paged_evict(sh, 2, cache, led, table, lens, lens[:1], lens,
                                lens, word, word)
    with pytest.raises(ValueError, match="have must have"):
        paged.lumen_paged_release(lens, lens[:1], table, 16, 2, word, slots[:1],
                                  slots[:1], word)
    assert paged.ledger_dims(sh, 5) == (2, 2, 5, 2, 16)
    assert paged.ledger_shape(sh).pool_elems(5) == 2 * 2 * 5 * 2 * 16
    with pytest.raises(ValueError, match="multiple of 4 words"):
        paged.ledger_shape(CacheShape(1, 1, 64, 3, HND))


def test_the_order_in_which_places_are_kept():
    """The definition that eviction is checked against, by hand."""
    nan, inf = np.float32("nan"), np.float32("inf")
    w = np.array([1, 3, nan, 3, -0.0, 0.0, inf, -inf, 2], np.float32)
    pos = np.arange(9)
    assert ref.rank_order(w, pos, 0, 99) == [6, 1, 3, 8, 0, 4, 5, 7, 2]
    assert ref.rank_order(w, pos, 1, 7) == [8, 0, 7, 6, 1, 3, 4, 5, 2]
    assert ref.rank_order(w, pos, 3, 99) == [1, 0, 2, 6, 3, 8, 4, 5, 7]


HIPCC = os.path.join(os.environ.get("ROCM_PATH", "/opt/rocm"), "bin", "hipcc")


def scalars(operand):
    m = re.match(r"s\[(\d+):(\d+)\]|s(\d+)$", operand)
    if not m:
        return {operand} if operand == "m0" else set()
    return {int(m[3])} if m[3] else set(range(int(m[1]), int(m[2]) + 1))


@pytest.mark.skipif(not os.path.exists(HIPCC), reason="no hipcc")
@pytest.mark.parametrize("source", ["lumen_paged_attend", "lumen_paged_weigh"])
def test_no_load_into_lds_reads_a_register_written_just_before(source):
    """The compiler does not look into the text of these loads for the five cycles
    that a scalar register written by a vector instruction needs."""
    flags = [f for f in build.HIPCC_FLAGS if f not in ("-shared", "-Werror")]
    text = subprocess.run(
        [HIPCC, *flags, "-I", build.INCLUDE, "--cuda-device-only", "-S",
         os.path.join(build.PKG, "csrc", source + ".hip"), "-o", "-"],
        capture_output=True, text=True, check=True).stdout
    lines = [l.strip() for l in text.splitlines()]
    lines = [l for l in lines if l and not l.startswith((";", "."))
             and not l.endswith(":")]
    loads = 0
    for i, l in enumerate(lines):
        if not l.startswith("global_load_lds"):
            continue
        loads += 1
        need = {"m0"}.union(*(scalars(o.strip().split()[0])
                              for o in l.split(None, 1)[1].split(",")))
        wait, j = 0, i - 1
        while wait < 5:
            if lines[j].startswith("s_nop"):
                wait += int(lines[j].split()[1], 0) + 1
            else:
                if lines[j].startswith("v_"):
                    to = lines[j].split(None, 1)[1].split(",")
                    written = set().union(*(scalars(o.strip())
                                            for o in to[:2]))
                    # (the second operand is a result of some instructions)
                    assert not written & need, lines[j:i + 1]
                wait += 1
            j -= 1
    assert loads > 20
