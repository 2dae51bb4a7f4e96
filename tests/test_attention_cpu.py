"""The attention calls without a GPU: what is refused, workspace sizes, and -- compiled for the host -- the arithmetic by which the
kernels find rows in a cache, which is all that stands between a wrong slot, page or length and the memory behind the cache."""
import ctypes
import math
import os
import subprocess

import pytest
import torch

import paper_2506_22694_amd as vt
from paper_2506_22694_amd import attention, binding

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
NULL, SHAPE, DTYPE, ALIGN, WORKSPACE = 1, 2, 3, 4, 5
A, ODD = 0x10000, 0x10004      # device addresses that are never followed


@pytest.fixture(scope="module")
def lib():
    if not os.path.exists(binding.LIB_PATH):
        from paper_2506_22694_amd import build
        build.build_library()
    return binding.load_library()


def _cache(**kw):
    c = attention._CacheStruct(A, A, A, A, 2, 10, 8, 64, 128)
    for name, value in kw.items():
        setattr(c, name, value)
    return c


def _norm(**kw):
    a = dict(type=1, n=4, hq=8, hk=2, D=64, wq=A, wk=A, eps=1e-6, table=A, rows=100, rot=64, style=0, pos=A, pos_type=1)
    a.update(kw)
    return list(a.values())


def test_norm_and_rotation_refuse(lib):
    def call(q=A, qs=512, k=A, ks=128, qo=A, qos=512, ko=A, kos=128, **kw):
        return lib.vt_qk_norm_rope(q, qs, k, ks, *_norm(**kw), qo, qos, ko, kos, None)
    for kw in ({"type": 2}, {"type": 7}, {"pos_type": 2}):
        assert call(**kw) == DTYPE, kw
    for kw in ({"n": -1}, {"n": 1 << 31}, {"hq": -1}, {"hq": 0, "hk": 0}, {"hq": 1024, "hk": 1}, {"D": 0}, {"D": 264}, {"eps": 0.0}, {"eps": math.nan},
               {"eps": math.inf}, {"rot": 0}, {"rot": 72}, {"rows": 0}, {"style": 2}, {"qs": 511}, {"ks": 64}, {"qos": 504}, {"kos": 0}, {"qs": -512}):
        assert call(**kw) == SHAPE, kw
    for kw in ({"q": None}, {"k": None}, {"qo": None}, {"ko": None}, {"wq": None}, {"wk": None}, {"pos": None}):
        assert call(**kw) == NULL, kw
    for kw in ({"q": ODD}, {"k": ODD}, {"qo": ODD}, {"ko": ODD}, {"qs": 516}, {"kos": 132}, {"wq": ODD}, {"table": ODD}, {"pos": ODD}, {"rot": 60},
               {"D": 60, "rot": 56}):
        assert call(**kw) == ALIGN, kw
    assert call(n=0, q=None, k=None, pos=None) == 0 and call(n=0, q=ODD) == 0


def test_gradients_refuse(lib):
    ws = lib.vt_qk_norm_rope_backward_ws_bytes(4, 64)
    assert ws >= 4 * 2 * 64 * 4 and ws % 256 == 0
    assert lib.vt_qk_norm_rope_backward_ws_bytes(-1, 64) == 0 == lib.vt_qk_norm_rope_backward_ws_bytes(4, 257)
    sizes = [lib.vt_qk_norm_rope_backward_ws_bytes(n, 64) for n in (0, 1, 4, 1000, 5000, 1 << 30)]
    assert sizes == sorted(sizes) and sizes[-1] < 1 << 24

    def call(gq=A, gqs=512, gk=A, gks=128, q=A, qs=512, k=A, ks=128, dq=A, dqs=512, dk=A, dks=128, dqw=A, dkw=A, w=A, wsb=ws, **kw):
        return lib.vt_qk_norm_rope_backward(gq, gqs, gk, gks, q, qs, k, ks, *_norm(**kw), dq, dqs, dk, dks, dqw, dkw, w, wsb, None)
    assert call(type=3) == DTYPE and call(n=-1) == SHAPE and call(D=300) == SHAPE
    for name in ("gq", "gk", "q", "k", "dq", "dk", "dqw", "dkw"):
        assert call(**{name: None}) == NULL, name
    for name in ("gq", "gk", "q", "k", "dq", "dk"):
        assert call(**{name: ODD}) == ALIGN, name
    for name in ("gqs", "gks", "qs", "ks", "dqs", "dks"):
        assert call(**{name: 8}) == SHAPE, name
    assert call(w=None) == WORKSPACE == call(wsb=ws - 1) == call(w=ODD)
    assert call(n=0, wq=None, wk=None, q=None, k=None, w=None, wsb=0, pos=None) == 0


def test_cache_writes_and_reads_refuse(lib):
    def write(q=A, qs=1024, k=A, ks=1024, v=A, vs=1024, qo=A, qos=1024, slots=A, slot_type=1, cache=None, **kw):
        a = _norm(**{"D": 128, "rot": 128, **kw})
        del a[3:5]      # (kv heads and head size are the cache's)
        c = _cache(**(cache or {}))
        return lib.vt_qkv_to_cache(q, qs, k, ks, v, vs, *a, qo, qos, ctypes.addressof(c), slots, slot_type, None)

    def read(k=A, v=A, n=4, slots=A, slot_type=1, out=1, cache=None):
        c = _cache(**(cache or {}))
        return lib.vt_kv_cache_read(ctypes.addressof(c), slots, slot_type, n, k, v, out, None)
    for f in (write, read):
        for kw in ({"type": 0}, {"type": 3}):
            assert f(cache=kw) == DTYPE, kw
        for kw in ({"pages": 0}, {"heads": 0}, {"heads": 1025}, {"head_dim": 8}, {"head_dim": 272}, {"page_size": 8}, {"page_size": 48}, {"page_size": 0},
                   {"page_size": 131072}):
            assert f(cache=kw) == SHAPE, kw
        for kw in ({"k": None}, {"v": None}, {"k_scale": None}, {"v_scale": None}):
            assert f(cache=kw) == NULL, kw
        for kw in ({"k": ODD}, {"v": ODD}, {"head_dim": 72}, {"k_scale": 0x10001}):
            assert f(cache=kw) == ALIGN, kw
        assert f(slot_type=2) == DTYPE and f(slots=None) == NULL and f(slots=ODD) == ALIGN
        assert f(n=-1) == SHAPE and f(n=0, slots=None, k=None) == 0
    for kw in ({"q": None}, {"k": None}, {"v": None}, {"qo": None}):
        assert write(**kw) == NULL, kw
    assert write(vs=1023) == SHAPE and write(v=ODD) == ALIGN and write(type=2) == DTYPE
    assert read(out=2) == DTYPE and read(v=None) == NULL and read(k=ODD) == ALIGN
    assert lib.vt_kv_cache_read(None, A, 1, 4, A, A, 1, None) == NULL


def test_attention_refuses(lib):
    big = 1 << 30

    def call(q=A, qs=4096, type=1, n=3, hq=32, pt=A, pages=40, lengths=A, requests=3, start=None, max_rows=1, mask=None, most=2000, scale=0.1, out=A, os=4096,
             lse=None, ws=A, wsb=big, cache=None):
        c = _cache(**(cache or {}))
        return lib.vt_paged_attention(q, qs, type, n, hq, ctypes.addressof(c), pt, pages, lengths, requests, start, max_rows, mask, most, scale, out, os, lse,
                                      ws, wsb, None)
    assert call(type=2) == DTYPE and call(cache={"type": 0}) == DTYPE
    for kw in ({"n": -1}, {"n": 2}, {"requests": 4}, {"requests": -1}, {"hq": 0}, {"hq": 33}, {"hq": 2048}, {"pages": 0}, {"max_rows": 0}, {"max_rows": 2},
               {"n": 7, "start": A, "max_rows": 2}, {"most": -1}, {"most": big + 1}, {"scale": math.inf}, {"scale": math.nan}, {"qs": 4088}, {"os": 8},
               {"cache": {"heads": 5}}, {"n": 1 << 22, "requests": 1 << 22}):
        assert call(**kw) == SHAPE, kw
    for kw in ({"q": None}, {"pt": None}, {"lengths": None}, {"out": None}):
        assert call(**kw) == NULL, kw
    for kw in ({"q": ODD}, {"out": ODD}, {"pt": 0x10002}, {"lengths": 0x10001}, {"start": 0x10002}, {"mask": ODD}, {"lse": 0x10002}, {"qs": 4100}):
        assert call(**kw) == ALIGN, kw
    assert call(ws=None) == WORKSPACE == call(ws=ODD) == call(wsb=256)
    assert call(n=0, requests=0, q=None) == 0 and call(n=0, start=A, q=None, lengths=None) == 0


def test_workspace_for_the_largest_call_serves_all_below(lib):
    size = lib.vt_paged_attention_ws_bytes
    assert size(1, 32, 8, 128, 1, 1, 128) == 0 == size(9, 32, 8, 128, 70000, 1, 1 << 20) and size(1, 32, 7, 128, 1, 1, 1 << 20) == 0 and size(3, 32, 8, 128, 2, 1, 1 << 20) == 0
    import random
    rng = random.Random(3)
    for _ in range(3000):
        hk = rng.choice([1, 2, 8])
        hq, D = hk * rng.choice([1, 3, 4, 8]), rng.choice([64, 80, 128, 256])
        requests, rows, most = rng.randint(1, 80), rng.randint(1, 20), rng.choice([rng.randint(0, 2000), rng.randint(0, 200000)])
        whole = size(requests * rows, hq, hk, D, requests, rows, most)
        r, m, t = rng.randint(1, requests), rng.randint(1, rows), rng.randint(0, most)
        n = rng.randint(1, r * m)
        c = _cache(heads=hk, head_dim=D)
        assert size(n, hq, hk, D, r, m, t) <= whole
        for type in (0, 1):      # (the alignment of the log-sum-exps is looked at last, after the workspace's size)
            assert lib.vt_paged_attention(A, hq * D, type, n, hq, ctypes.addressof(c), A, 1, A, r, A, m, None, t, 1.0, A, hq * D, 0x10002, A,
                                          whole, None) == ALIGN


def test_binding_refuses():
    x = torch.zeros(2, 4, 64)
    with pytest.raises(ValueError):
        vt.qk_norm_rope(x, x)
    with pytest.raises(ValueError):
        vt.KVCache(2, 64, 4, 64, device="cpu")
    with pytest.raises(TypeError):
        vt.KVCache(2, 64, 4, 64, dtype=torch.float32, device="cpu")
    with pytest.raises(ValueError):
        vt.rope_table(4, 8, device="cpu", frequencies=torch.ones(3))


def test_table_keeps_the_angles_of_far_positions():
    t = vt.rope_table(200001, 8, 500000.0, device="cpu")
    for i in range(4):
        angle = 200000 * 500000.0 ** (-2 * i / 8)
        assert abs(t[200000, i].item() - math.cos(angle)) < 1e-7 and abs(t[200000, 4 + i].item() - math.sin(angle)) < 1e-7
    assert torch.equal(vt.rope_table(9, 4, device="cpu", frequencies=torch.tensor([1.0, 0.0]))[:, 1], torch.ones(9))


# ------------------------------------------------------------------ the kernels' own arithmetic, on the host
_CELLS = r"""
#include "vt_cells.h"
extern "C" {
int64_t slot(int64_t s, int64_t pages, int heads, int head, int shift) { return vt::row_of_slot(s, pages, heads, head, shift); }
int64_t page(int p, int64_t pages, int heads, int head, int shift) { return vt::row_of_page(p, pages, heads, head, shift); }
int tokens(int length, int most) { return vt::tokens_of(length, most); }
int rows(const int32_t *start, int b, int n, int max_rows, int *first) { return vt::rows_of(start, b, n, max_rows, *first); }
int steps(int tokens, int rows, int step) { return vt::steps_of(tokens, rows, step); }
int share(int all, int places, int place, int *per, int *start) { return vt::share_steps(all, places, place, *per, *start); }
int exponent(float x) { uint32_t u; __builtin_memcpy(&u, &x, 4); return vt::scale_exponent(u); }
}
"""


@pytest.fixture(scope="module")
def cells(tmp_path_factory):
    at = tmp_path_factory.mktemp("cells")
    (at / "cells.cpp").write_text(_CELLS)
    subprocess.run(["g++", "-std=c++17", "-O1", "-fsanitize=undefined", "-fno-sanitize-recover=all", "-shared", "-fPIC", "-static-libubsan", "-I",
                    os.path.join(ROOT, "paper_2506_22694_amd", "csrc"), str(at / "cells.cpp"), "-o", str(at / "cells.so")], check=True)
    L = ctypes.CDLL(str(at / "cells.so"))
    i64, i32 = ctypes.c_int64, ctypes.c_int32
    L.slot.argtypes, L.slot.restype = [i64, i64, i32, i32, i32], i64
    L.page.argtypes, L.page.restype = [i32, i64, i32, i32, i32], i64
    L.tokens.argtypes = [i32, i32]
    L.rows.argtypes = [ctypes.c_void_p, i32, i32, i32, ctypes.POINTER(i32)]
    L.share.argtypes = [i32, i32, i32, ctypes.POINTER(i32), ctypes.POINTER(i32)]
    L.exponent.argtypes = [ctypes.c_float]
    return L


def test_slots_and_pages_outside_the_cache_have_no_row(cells):
    for pages, heads, shift in ((1, 1, 4), (7, 3, 5), (1 << 31, 8, 16)):
        size = 1 << shift
        for s in (0, 1, size - 1, size, pages * size - 1):
            if s < pages * size:
                for head in (0, heads - 1):
                    assert cells.slot(s, pages, heads, head, shift) == (s // size * heads + head) * size + s % size < pages * heads * size
        for s in (-1, -size, -(1 << 63), pages * size, pages * size + 1, (1 << 63) - 1):
            assert cells.slot(s, pages, heads, 0, shift) == -1, s
        for p in (0, pages - 1):
            if p < 1 << 31:
                assert cells.page(p, pages, heads, heads - 1, shift) == (p * heads + heads - 1) * size
        for p in (-1, -(1 << 31), pages, (1 << 31) - 1):
            if p < 0 or pages <= p < 1 << 31:
                assert cells.page(p, pages, heads, 0, shift) == -1, p


def test_lengths_and_rows_stay_within_what_there_is(cells):
    assert [cells.tokens(x, 100) for x in (-(1 << 31), -1, 0, 1, 100, 101, (1 << 31) - 1)] == [0, 0, 0, 1, 100, 100, 100]
    assert cells.tokens((1 << 31) - 1, 1 << 30) == 1 << 30
    first = ctypes.c_int32()
    assert cells.rows(None, 5, 6, 1, ctypes.byref(first)) == 1 and first.value == 5
    start = (ctypes.c_int32 * 9)(0, 3, 3, 10, 9, -4, 2, 50, 60)
    got = []
    for b in range(8):
        rows = cells.rows(start, b, 12, 5, ctypes.byref(first))
        assert rows == 0 or (first.value == start[b] >= 0 and first.value + rows <= 12)
        got.append(rows)
    assert got == [3, 0, 5, 0, 0, 0, 5, 0]


def test_shares_cover_every_step_once(cells):
    assert [cells.steps(t, 1, 128) for t in (0, 1, 128, 129, 256, 257, 1 << 30)] == [1, 1, 1, 2, 2, 3, 1 << 23] and cells.steps(500, 0, 128) == 0
    per, start = ctypes.c_int32(), ctypes.c_int32()
    for all_ in (0, 1, 5, 64, 65, 1000, (1 << 30) - 1, 1 << 30):
        for places in (1, 2, 7, 64, 512):
            upto = 0
            for place in range(places):
                left = cells.share(all_, places, place, ctypes.byref(per), ctypes.byref(start))
                assert left >= 0 and (left == 0 or start.value == upto) and left <= per.value
                upto += left
            assert upto == all_


def _shared_out(cells, tokens, rows, places, step):
    """What the workgroups of one kv head do with requests of `tokens` cached tokens and `rows` new rows, in the kernel's order: parts written
    {(place, number there): (request, first step, steps)}, where the join is told to look {request: (place, parts, number)}, by place too."""
    steps = [cells.steps(t, r, step) for t, r in zip(tokens, rows)]
    written, by_request, by_place = {}, {}, {}
    whole = []
    per, start = ctypes.c_int32(), ctypes.c_int32()
    for place in range(places):
        left = cells.share(sum(steps), places, place, ctypes.byref(per), ctypes.byref(start))
        if left == 0:
            by_place[place] = (place, 1, 0, 0)
            continue
        b, before = 0, 0
        while start.value >= before + steps[b]:
            before += steps[b]
            b += 1
        at, segment = start.value - before, 0
        while left > 0:
            take = min(left, steps[b] - at)
            complete = take == steps[b]
            left -= take
            parts = (place, 1 if complete else 1 + -(-(steps[b] - take) // per.value), int(segment != 0), b)
            begins = take > 0 and at == 0
            by_place[place] = parts if begins else (place, 1, 0, b)
            if begins:
                by_request[b] = parts
            if take > 0 and complete:
                whole.append(b)
            elif take > 0:
                assert (place, int(segment != 0)) not in written
                written[place, int(segment != 0)] = (b, at, take)
            b, at, segment = b + 1, 0, segment + 1
    return steps, written, by_request, by_place, whole


def test_the_join_finds_every_part_of_every_request(cells):
    import random
    rng = random.Random(7)
    for _ in range(400):
        n = rng.choice([1, 2, 5, 30, 200])
        tokens = [rng.choice([0, 1, 128, rng.randint(0, 3000), rng.randint(0, 300)]) for _ in range(n)]
        rows = [rng.choice([0, 1, 1, 4]) for _ in range(n)]
        places = rng.choice([1, 2, 7, 64, 256])
        steps, written, by_request, by_place, whole = _shared_out(cells, tokens, rows, places, 128)
        assert set(by_place) == set(range(places))
        assert set(by_request) == {b for b in range(n) if rows[b] > 0}
        begun = {p[3]: p for p in by_place.values() if p[1] > 1}
        for b in range(n):
            if rows[b] == 0:
                assert b not in begun and b not in whole
                continue
            place, parts, number, _ = by_request[b]
            assert (parts == 1) == (b in whole) and (parts == 1 or begun[b] == by_request[b]) and (parts > 1 or b not in begun)
            if parts > 1:
                at = 0
                for i in range(parts):
                    of, first, took = written.pop((place + i, number if i == 0 else 0))
                    assert of == b and first == at
                    at += took
                assert at == steps[b]
        assert not written


def test_scales_are_the_smallest_that_hold_the_maximum(cells):
    import random
    rng = random.Random(1)
    values = [448.0, 448.0 * (1 + 2 ** -23), 449.0, 1.75, 1.7500002, 3.4028234e38, 1e-30, 2.0 ** -126, 0.0, 2.0 ** -149] + [
        rng.uniform(1, 2) * 2.0 ** rng.randint(-126, 127) for _ in range(2000)]
    for x in values:
        x = ctypes.c_float(x).value
        e = cells.exponent(x)
        assert 1 <= e <= 254 and x <= 448 * 2.0 ** (e - 127)
        assert e == 1 or x > 448 * 2.0 ** (e - 128)


def test_build_rejects_attention_kernels_with_accumulation_registers():
    from paper_2506_22694_amd import build
    remarks = "\n".join([
        "a.h:1:1: remark: Function Name: kernel_a [-Rpass-analysis=kernel-resource-usage]",
        "a.h:1:1: remark:     VGPRs: 200 [-Rpass-analysis=kernel-resource-usage]",
        "a.h:1:1: remark:     AGPRs: 0 [-Rpass-analysis=kernel-resource-usage]",
        "a.h:1:1: remark: Function Name: kernel_b [-Rpass-analysis=kernel-resource-usage]",
        "a.h:1:1: remark:     AGPRs: 12 [-Rpass-analysis=kernel-resource-usage]",
    ])
    assert build._accumulation_users(remarks) == [("kernel_b", 12)]
    assert all(os.path.basename(s).startswith(build.NO_ACCUMULATION) for s in build._sources() if "vt_attend_d" in s)
