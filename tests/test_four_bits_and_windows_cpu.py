"""The 4-bit cache's and the windowed attention's calls without a GPU: what is refused, and -- compiled for the host -- the arithmetic by which the
kernels find a scale, and which tokens of a request they read."""
import ctypes
import math
import os
import random
import subprocess

import pytest
import torch

import paper_2506_22694_amd as vt
from test_attention_cpu import A, ALIGN, DTYPE, NULL, ODD, SHAPE, WORKSPACE, _cache, _norm, lib  # noqa: F401

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
FOUR = {"type": 4}


def test_four_bit_caches_are_refused_where_their_sizes_do_not_fit(lib):      # noqa: F811
    def write(cache, n=4):
        a = _norm(D=128, rot=128, n=n)
        del a[3:5]
        c = _cache(**FOUR, **cache)
        return lib.vt_qkv_to_cache(A, 1024, A, 1024, A, 1024, *a, A, 1024, ctypes.addressof(c), A, 1, None)

    def read(cache, n=4):
        c = _cache(**FOUR, **cache)
        return lib.vt_kv_cache_read(ctypes.addressof(c), A, 1, n, A, A, 1, None)

    def attend(cache, n=1):
        c = _cache(**FOUR, **cache)
        return lib.vt_paged_attention(A, 4096, 1, n, 32, ctypes.addressof(c), A, 40, A, n, None, 1, None, 2000, 0.1, A, 4096, None, A, 1 << 30, None)
    for f in (write, read, attend):
        for kw in ({"head_dim": 48}, {"head_dim": 80}, {"head_dim": 16}, {"k": ODD}, {"v": ODD}, {"k_scale": 0x10002}, {"v_scale": 0x10001}):
            assert f(kw) == ALIGN, kw
        for kw in ({"k": None}, {"v": None}, {"k_scale": None}, {"v_scale": None}):
            assert f(kw) == NULL, kw
        for kw in ({"pages": 0}, {"head_dim": 288}, {"head_dim": 8}, {"page_size": 24}):
            assert f(kw) == SHAPE, kw
        assert f({}, n=0) == 0


def test_windowed_attention_refuses(lib):      # noqa: F811
    big = 1 << 30

    def call(q=A, qs=4096, type=1, n=3, hq=32, pt=A, pages=40, lengths=A, requests=3, start=None, max_rows=1, mask=None, positions=None, pos_type=1, window=100,
             sinks=4, most=2000, scale=0.1, out=A, os=4096, lse=None, ws=A, wsb=big, cache=None):
        c = _cache(**(cache or {}))
        return lib.vt_paged_attention_window(q, qs, type, n, hq, ctypes.addressof(c), pt, pages, lengths, requests, start, max_rows, mask, positions, pos_type,
                                             window, sinks, most, scale, out, os, lse, ws, wsb, None)
    assert call(type=2) == DTYPE and call(cache={"type": 0}) == DTYPE and call(mask=A, positions=A, pos_type=2) == DTYPE
    for kw in ({"window": 0}, {"window": -1}, {"window": big + 1}, {"sinks": -1}, {"sinks": big + 1}, {"positions": A}, {"n": 2}, {"max_rows": 0},
               {"max_rows": 2}, {"most": -1}, {"most": big + 1}, {"scale": math.inf}, {"qs": 4088}, {"hq": 33}, {"pages": 0},
               {"requests": 65535, "n": 65535, "most": big}):
        assert call(**kw) == SHAPE, kw
    for kw in ({"q": None}, {"pt": None}, {"lengths": None}, {"out": None}):
        assert call(**kw) == NULL, kw
    for kw in ({"q": ODD}, {"pt": 0x10002}, {"mask": ODD}, {"mask": A, "positions": 0x10004}, {"mask": A, "positions": 0x10002, "pos_type": 0}, {"lse": 0x10002}):
        assert call(**kw) == ALIGN, kw
    assert call(n=0, requests=0, q=None, pt=None) == 0
    # a workspace of the size of a call without a window is enough: none where a window keeps the tokens few
    wide = {"window": 1500, "start": A, "max_rows": 8, "n": 20}
    assert call(ws=None, **wide) == WORKSPACE == call(wsb=100, **wide) == call(ws=0x10010, **wide)


def test_windows_need_no_more_than_the_workspace_of_a_call_without():
    rng = random.Random(5)
    lib_ = vt.load_library()
    for _ in range(300):
        requests, rows, hk = rng.choice([1, 3, 64, 700]), rng.choice([1, 5, 64, 1000]), rng.choice([1, 8])
        hq, D, most = hk * rng.choice([1, 4]), rng.choice([32, 64, 128, 256]), rng.choice([1, 300, 385, 5000, 131072])
        n = requests * rows
        if n * hq > 1 << 23:
            continue
        size = lib_.vt_paged_attention_ws_bytes(n, hq, hk, D, requests, rows, most)
        for window in (1, 100, 500, 4096, 1 << 30):
            for sinks in (0, 4, 1000):
                c = _cache(type=1, heads=hk, head_dim=D, k_scale=None, v_scale=None)
                # (a misaligned out_lse is the last thing that is looked at: nothing is launched)
                status = lib_.vt_paged_attention_window(A, hq * D, 1, n, hq, ctypes.addressof(c), A, 9000, A, requests, A, rows, None, None, 0, window, sinks, most,
                                                        0.1, A, hq * D, 0x10002, A, size, None)
                assert status == ALIGN, (requests, rows, hq, D, most, window, sinks, status)


@pytest.mark.parametrize("held,scales", [(1, None), (2, A), (4, A)])
def test_any_split_of_any_cache_fits_the_workspace(held, scales):
    rng = random.Random(held)
    lib_ = vt.load_library()
    for _ in range(600):
        requests, rows, hk = rng.choice([1, 2, 5, 17, 64]), rng.choice([1, 2, 8, 17, 40, 130]), rng.choice([1, 2, 4, 8, 32])
        hq, D, most = hk * rng.choice([1, 2, 4, 7]), rng.choice([32, 64, 96, 128, 160, 256]), rng.choice([385, 520, 1000, 5000, 20000, 131072])
        n = requests * rows
        size = lib_.vt_paged_attention_ws_bytes(n, hq, hk, D, requests, rows, most)
        c = _cache(type=held, heads=hk, head_dim=D, k_scale=scales, v_scale=scales)
        for less in (1, 2, 7):      # (of a workspace for more rows or longer requests than there are)
            for window in (0, 100, 1000, 4096, 1 << 30):
                m, length = max(1, rows // less), most // less
                for mask in (None, A):
                    status = lib_.vt_paged_attention_window(A, hq * D, 1, requests * m, hq, ctypes.addressof(c), A, 9000, A, requests, A, m, mask, None, 0, window, 4 if window else 0,
                                                            length, 0.1, A, hq * D, 0x10002, A, size, None) if window else \
                        lib_.vt_paged_attention(A, hq * D, 1, requests * m, hq, ctypes.addressof(c), A, 9000, A, requests, A, m, mask, length, 0.1, A, hq * D, 0x10002, A, size, None)
                    assert status == ALIGN, (requests, m, hq, hk, D, length, window, mask, status)


def test_python_refuses_before_anything_is_sent():
    q = torch.ones(1, 2, 64)
    with pytest.raises(ValueError):
        vt.KVCache(1, 16, 2, 40, dtype=torch.float4_e2m1fn_x2, device="cpu")
    with pytest.raises((ValueError, TypeError)):
        vt.KVCache(1, 16, 2, 64, dtype=torch.float16, device="cpu")
    assert q.shape == (1, 2, 64)


# ---------------------------------------------------------------------------------------------- on the host
@pytest.fixture(scope="module")
def cells(tmp_path_factory):
    d = tmp_path_factory.mktemp("cells")
    (d / "c.cpp").write_text('''#include "vt_cells.h"
extern "C" {
int64_t scale_at(int64_t row, int groups, int group, int shift) { return vt::scale_of_row(row, groups, group, shift); }
int exponent(float x) { uint32_t u; __builtin_memcpy(&u, &x, 4); return vt::scale_exponent_of_four(u); }
int gap(int tokens, int back, int window, int sinks) { return vt::window_gap(tokens, back, window, sinks); }
int round16(int x) { return vt::round16(x); }
int last(int tokens, int rows, int i) { return vt::last_position(tokens, rows, i); }
int given(int tokens, int64_t p) { return vt::given_position(tokens, p); }
}''')
    subprocess.run(["g++", "-O1", "-shared", "-fPIC", "-Wall", "-I" + os.path.join(ROOT, "paper_2506_22694_amd", "csrc"), str(d / "c.cpp"), "-o",
                    str(d / "c.so")], check=True)
    c = ctypes.CDLL(str(d / "c.so"))
    c.scale_at.restype, c.scale_at.argtypes = ctypes.c_int64, [ctypes.c_int64, ctypes.c_int, ctypes.c_int, ctypes.c_int]
    c.exponent.argtypes = [ctypes.c_float]
    c.given.argtypes = [ctypes.c_int, ctypes.c_int64]
    return c


def test_every_group_of_a_row_has_a_scale_of_its_own(cells):
    for pages, heads, shift, groups in ((3, 2, 4, 1), (2, 3, 5, 4), (1, 1, 6, 8)):
        size = 1 << shift
        seen = {}
        for row in range(pages * heads * size):
            for group in range(groups):
                at = cells.scale_at(row, groups, group, shift)
                page_head, place = divmod(row, size)
                assert at == (page_head * groups + group) * size + place and at not in seen
                seen[at] = row
        assert sorted(seen) == list(range(pages * heads * size * groups))
    assert cells.scale_at((1 << 40) + 3, 8, 7, 16) == (((1 << 24) * 8 + 7) << 16) + 3


def test_scales_are_the_smallest_that_hold_the_maximum(cells):
    rng = random.Random(1)
    for x in [6.0, 6.0 * (1 + 2 ** -23), 6.5, 1.5, 1.5000002, 3.4028234e38, 1e-30, 2.0 ** -126, 0.0, 2.0 ** -149, 3.0, 4.0] + [
            rng.uniform(1, 2) * 2.0 ** rng.randint(-126, 127) for _ in range(2000)]:
        x = ctypes.c_float(x).value
        e = cells.exponent(x)
        assert 1 <= e <= 253 and x <= 6 * 2.0 ** (e - 127)
        assert e == 1 or x > 6 * 2.0 ** (e - 128)


def test_the_gap_holds_no_token_that_a_row_sees_and_begins_and_ends_at_the_first_of_sixteen(cells):
    rng = random.Random(2)
    for _ in range(4000):
        tokens = rng.choice([0, 1, 15, 16, 17, rng.randint(0, 400), 1 << 30])
        window, sinks = rng.choice([1, 2, 15, 16, 17, rng.randint(1, 300), 1 << 30]), rng.choice([0, 1, 15, 16, 17, rng.randint(0, 200), 1 << 30])
        rows, given = rng.choice([1, 2, 8, rng.randint(1, 200), 1 << 22]), rng.random() < 0.3
        back = 64 if given else rows
        gap = cells.gap(tokens, back, window, sinks)
        begin = cells.round16(sinks)
        assert gap >= 0 and gap % 16 == 0 and (gap == 0 or gap <= tokens)
        if gap:
            assert begin + gap <= tokens + 15 and begin >= sinks
            lowest = cells.given(tokens, -(1 << 62)) if given else cells.last(tokens, rows, 0)
            assert begin + gap <= max(0, lowest - window + 1)            # the first token of the lowest row's window
            assert lowest - window + 1 - (begin + gap) < 16                # ... and no more than 15 ahead of it
        # what is left to read
        assert tokens - gap <= sinks + 15 + window + 15 + back


def test_positions_are_those_of_the_tail_or_the_last_tokens(cells):
    assert [cells.last(100, 5, i) for i in range(5)] == [95, 96, 97, 98, 99] and cells.last(3, 5, 0) == -2
    assert cells.given(100, 36) == 36 and cells.given(100, 35) == 36 and cells.given(100, -(1 << 63)) == 36
    assert cells.given(100, 1000) == 1000 and cells.given(100, (1 << 63) - 1) == (1 << 31) - 1 and cells.given(0, -70) == -64
