"""Attention with a sliding window and sinks over a paged cache, against 64 bits by the definition: single tokens, tree levels, chunks of prompts.

Tolerances: a score is a sum of D products in fp32, off by up to sqrt(D) / 2 + 8 half steps of the sum of their sizes; a weight is off by that much,
absolute in the exponent, and by exp2's and the sums' few.  Chunks of bf16 rows hold their weights in 16 bits (half a step 2^-17).  out is a mean of values, so
off by its weights' relative error times the mean size of its values, then rounded once."""
import math

import pytest
import torch

import paper_2506_22694_amd as vt
import test_gpu_four_bits as four
from paper_2506_22694_amd import binding
from test_gpu_attention import BF16, E4M3, F32, HALF, _case, _gen, _outcome, _randn, _values, close

pytestmark = pytest.mark.gpu

E2M1 = four.E2M1
CACHES = [BF16, E4M3, E2M1]


def case(g, held, dtype, hq, hk, D, page, lengths, rows=None, gain=1.5):
    if held == E2M1:
        return four.case(g, dtype, hq, hk, D, page, lengths, rows, gain)
    return _case(g, held, dtype, hq, hk, D, page, lengths, rows, gain=gain)


def sees(length, rows, window, sinks, mask=None, positions=None):
    """[rows, length]: by the definition."""
    t = torch.arange(length, device="cuda")[None]
    p = length - rows + torch.arange(rows, device="cuda")[:, None] if positions is None else positions.long()[:, None].clamp(min=length - 64)
    see = (t > p - window) | (t < sinks)
    if mask is None:
        return see & (t <= p)
    bits = (mask[:, None] >> (t - (length - 64)).clamp(0, 63)) & 1
    return see & ((t < length - 64) | (bits == 1))


def attend64(q, k, v, see, scale):
    """q [rows, hq, D], k and v [tokens, hk, D], see [rows, tokens]: out, lse and the mean size of the values."""
    rows, hq, D = q.shape
    hk = k.shape[1]
    x = q.double().view(rows, hk, -1, D).permute(1, 2, 0, 3)                      # [hk, G, rows, D]
    k, v = (y.double().transpose(0, 1).contiguous() for y in (k, v))              # [hk, tokens, D]
    if k.shape[1] == 0:
        return torch.zeros(rows, hq, D, dtype=torch.float64, device="cuda"), torch.full((rows, hq), -math.inf, dtype=torch.float64, device="cuda"), torch.zeros(
            rows, hq, D, dtype=torch.float64, device="cuda")
    s = torch.matmul(x, k.transpose(-1, -2).contiguous()[:, None]) * scale
    s = s.masked_fill(~see, -math.inf)
    lse = torch.logsumexp(s, -1)
    w = torch.exp(s - torch.where(lse == -math.inf, 0.0, lse)[..., None])
    w = torch.where(see, w, 0.0)

    def mean(v):
        out = torch.matmul(w, torch.where(v.isfinite(), v, 0.0)[:, None])
        # what a row sees of NaN and infinities
        nan, up, down = (torch.matmul(see.double(), odd.double())[:, None] > 0 for odd in (v.isnan(), v == math.inf, v == -math.inf))
        out = torch.where(nan | (up & down), math.nan, torch.where(up, math.inf, torch.where(down, -math.inf, out)))
        return out.permute(2, 0, 1, 3).reshape(rows, hq, D)
    return mean(v), lse.permute(2, 0, 1).reshape(rows, hq), mean(torch.where(v.isfinite(), v.abs(), 0.0))


def check(cache, table, lengths, q, starts, window, sinks, mask=None, positions=None, scale=None, readable=None, **kw):
    n, hq, D = q.shape
    scale = D ** -0.5 if scale is None else scale
    max_rows = 1 if starts is None else max(1, int(starts.diff().max()))
    out, lse = vt.paged_attention(q, cache, table, lengths, row_start=starts, max_rows=max_rows, tail_mask=mask, scale=scale, return_lse=True, window=window,
                                  sinks=sinks, positions=positions, **kw)
    assert out.dtype == q.dtype and lse.dtype == F32
    first = list(range(n + 1)) if starts is None else starts.tolist()
    for b, length in enumerate(lengths.tolist()):
        rows = slice(first[b], first[b + 1])
        if first[b] == first[b + 1]:
            continue
        k, v = _values(cache, table if readable is None else readable, b, length)
        see = sees(length, first[b + 1] - first[b], window, sinks, None if mask is None else mask[rows], None if positions is None else positions[rows])
        want, want_lse, spread = attend64(q[rows], k, v, see, scale)
        kk = torch.where(k.isfinite(), k, 0.0).abs()
        most = (q[rows].double().abs().amax() * kk.sum(-1).amax() * abs(scale)).item() if length else 0.0
        fine = most * (math.sqrt(D) / 2 + 8) * 2.0 ** -24 + 40 * 2.0 ** -24
        weight = fine + (2.0 ** -16 if q.dtype == BF16 else 0.0)
        close(out[rows], want, HALF[q.dtype], weight * 2 * spread)
        close(lse[rows], want_lse, 2.0 ** -23, fine * 2)
    return out, lse


# Chunks of enough work go through a kernel of their own: layouts of many kv heads reach it with few rows and tokens, heads of every kernel's size among them
WIDE = [(128, 128, 64), (96, 48, 128), (224, 32, 96), (64, 64, 32), (64, 32, 256), (120, 40, 160)]
LAYOUTS = [(4, 2, 64), (32, 8, 128), (7, 1, 128), (6, 3, 256), (20, 1, 96), (3, 3, 32), (5, 1, 160)]
WINDOWS = [(1, 0), (15, 1), (16, 16), (17, 4), (64, 0), (100, 33), (128, 200), (1 << 30, 0), (1, 1 << 30)]


@pytest.mark.parametrize("hq,hk,D", LAYOUTS)
@pytest.mark.parametrize("held", CACHES)
@pytest.mark.parametrize("dtype", [BF16, F32])
def test_single_tokens(hq, hk, D, held, dtype):
    g = _gen(hq * D)
    a = case(g, held, dtype, hq, hk, D, 16, [1, 0, 17, 31, 32, 33, 64, 65, 127, 128, 129, 300, 1500])
    b = case(g, held, dtype, hq, hk, D, 64, [4099])
    for window, sinks in WINDOWS:
        check(*a, window, sinks)
        check(*b, window, sinks)


@pytest.mark.parametrize("held", CACHES)
def test_single_tokens_of_long_windows_split_and_joined(held):
    g = _gen(2)
    for lengths in ([9001], [5000, 0, 130, 2600, 777]):
        a = case(g, held, BF16, 8, 2, 128, 64, lengths)
        for window, sinks in ((4096, 4), (1000, 500), (513, 0), (385, 1)):
            check(*a, window, sinks)


def test_a_window_of_everything_is_attention_without_one():
    g = _gen(3)
    for held in CACHES:
        cache, table, lengths, q, _ = case(g, held, BF16, 8, 2, 64, 16, [300, 20, 0, 4000])
        want = vt.paged_attention(q, cache, table, lengths, return_lse=True)
        got = vt.paged_attention(q, cache, table, lengths, return_lse=True, window=1 << 30)
        assert torch.equal(want[0], got[0]) and torch.equal(want[1], got[1])


@pytest.mark.parametrize("hq,hk,D,rows", [(4, 2, 64, [3, 1, 0, 5]), (32, 8, 128, [8, 8, 1, 4]), (8, 8, 128, [16, 2, 7, 33]), (4, 1, 256, [8, 1, 2, 9]),
                                          (12, 3, 96, [6, 6, 6, 6]), (64, 1, 64, [2, 3, 1, 2])])
@pytest.mark.parametrize("held", CACHES)
@pytest.mark.parametrize("dtype", [BF16, F32])
def test_tree_levels(hq, hk, D, rows, held, dtype):
    g = _gen(hq + D)
    for lengths in ([40, 1, 64, 63], [200, 129, 65, 500], [700, 3, 1300, 90]):
        a = case(g, held, dtype, hq, hk, D, 32, lengths, rows=rows)
        mask = torch.randint(-(1 << 63), (1 << 63) - 1, (sum(rows),), generator=g, device="cuda")
        mask[0], mask[1], mask[-1] = 0, -1, -(1 << 63)
        base = torch.repeat_interleave(a[2].long(), torch.tensor(rows, device="cuda"))
        positions = base - 40 + torch.randint(-30, 50, (sum(rows),), generator=g, device="cuda")      # some below the tail, some past the end
        for window, sinks in ((1, 0), (20, 3), (100, 16), (150, 40), (1 << 30, 0)):
            check(*a, window, sinks, mask=mask, positions=positions)
            check(*a, window, sinks, mask=mask, positions=positions.int())
            check(*a, window, sinks, mask=mask)


@pytest.mark.parametrize("hq,hk,D,rows", [(32, 8, 128, 8), (20, 4, 96, 5), (64, 32, 64, 9), (28, 4, 64, 16), (28, 4, 64, 40)])
@pytest.mark.parametrize("held", CACHES)
def test_levels_of_many_requests(hq, hk, D, rows, held):
    """As much to read that workgroups have two or four tiles of query rows."""
    g = _gen(hq + D + rows)
    n = 40
    lengths = [3500] + [[64, 1, 700, 63, 0, 130, 333][i % 7] for i in range(n - 2)] + [3073]
    counts = [[rows, 1, 0, 3, 2][i % 5] for i in range(n)]
    a = case(g, held, BF16, hq, hk, D, 32, lengths, rows=counts)
    mask = torch.randint(-(1 << 63), (1 << 63) - 1, (sum(counts),), generator=g, device="cuda")
    mask[0], mask[1], mask[-1] = 0, -1, -(1 << 63)
    base = torch.repeat_interleave(a[2].long(), torch.tensor(counts, device="cuda"))
    positions = base - 40 + torch.randint(-30, 50, (sum(counts),), generator=g, device="cuda")
    for window, sinks in ((3000, 20), (100, 3000), (1 << 30, 0)):
        check(*a, window, sinks, mask=mask, positions=positions, max_length=1 << 16)
        check(*a, window, sinks, mask=mask, max_length=1 << 16)
    check(*a, 3000, 4, max_length=1 << 16)
    if held == E2M1:
        four._check_attention(*a, mask=mask, max_length=1 << 16)


@pytest.mark.parametrize("hq,hk,D", LAYOUTS)
@pytest.mark.parametrize("held", CACHES)
@pytest.mark.parametrize("dtype", [BF16, F32])
def test_chunks_of_prompts(hq, hk, D, held, dtype):
    g = _gen(hq + D)
    # rows of no cached token of their own, of all, of the last ones; requests without rows and without tokens
    a = case(g, held, dtype, hq, hk, D, 16, [40, 1, 0, 200, 333, 130, 64], rows=[40, 1, 3, 77, 150, 0, 70])
    for window, sinks in ((1, 0), (7, 2), (16, 16), (33, 0), (100, 20), (129, 4), (1 << 30, 0), (3, 1 << 30)):
        check(*a, window, sinks)


@pytest.mark.parametrize("hq,hk,D", WIDE)
@pytest.mark.parametrize("held", CACHES)
def test_chunks_of_many_heads(hq, hk, D, held):
    g = _gen(hq + D)
    for page, lengths, rows in ((16, [40, 1, 0, 200, 333, 130, 64, 500], [40, 1, 3, 77, 150, 0, 70, 130]), (64, [400, 390, 700, 70, 65], [200, 1, 97, 70, 100])):
        a = case(g, held, BF16, hq, hk, D, page, lengths, rows=rows)
        for window, sinks in ((1, 0), (7, 2), (16, 16), (33, 0), (100, 20), (129, 4), (1 << 30, 0), (3, 1 << 30)):
            check(*a, window, sinks)
        for scale in (0.0, -0.2):
            check(*a, 100, 4, scale=scale)


@pytest.mark.parametrize("held", CACHES)
@pytest.mark.parametrize("hq,hk,D", [(16, 4, 128), (6, 2, 64), (5, 1, 256)])
def test_chunks_in_shares(held, hq, hk, D):
    """Long windows of few heads and rows: a chunk's tokens are cut into shares, some of them of no tokens."""
    g = _gen(hq)
    a = case(g, held, BF16, hq, hk, D, 64, [9000, 300, 0, 5003], rows=[130, 140, 2, 77])
    for window, sinks in ((8000, 4), (5000, 700), (1 << 30, 0)):
        out, lse = check(*a, window, sinks)
        again = vt.paged_attention(a[3], *a[:3], row_start=a[4], max_rows=140, window=window, sinks=sinks, return_lse=True)
        assert torch.equal(out, again[0]) and torch.equal(lse, again[1])


@pytest.mark.parametrize("held", CACHES)
@pytest.mark.parametrize("hq,hk,D", [(32, 8, 128), (14, 2, 64), (4, 4, 256), (9, 1, 128)])
def test_longer_chunks(held, hq, hk, D):
    g = _gen(hq)
    a = case(g, held, BF16, hq, hk, D, 64, [1500, 900, 3], rows=[700, 900, 1])
    for window, sinks in ((256, 4), (1000, 17), (1 << 30, 0)):
        check(*a, window, sinks)


@pytest.mark.parametrize("held", CACHES)
@pytest.mark.parametrize("rows", [None, 3, 40])
def test_more_requests_than_shares(held, rows):
    g = _gen(30)
    n = 90
    lengths = [[1490, 0, 130, 128, 1, 700, 90, 260, 64][i * 7 % 9] for i in range(n)]
    counts = None if rows is None else [i * 5 % (rows + 1) for i in range(n)]
    a = case(g, held, BF16, 8, 8, 64, 16, lengths, rows=counts)
    for window, sinks in ((100, 4), (600, 0), (1000, 300)):
        check(*a, window, sinks, max_length=1504)


@pytest.mark.parametrize("held", CACHES)
@pytest.mark.parametrize("kind", ["token", "tree", "prompt", "wide"])
@pytest.mark.parametrize("D", [64, 128, 256])
def test_what_no_row_sees_may_be_anything(held, kind, D):
    """Pages between the sinks and the windows are out of the cache, other places that no row sees hold NaN, infinities and any scale."""
    g = _gen(D)
    hk, page = 64 if kind == "wide" else 2, 16
    lengths, rows = [900, 45, 333, 0, 16], {"token": None, "tree": [3, 2, 5, 1, 2]}.get(kind, [200, 45, 9, 2, 16])
    cache, table, lengths, q, starts = case(g, held, BF16, 2 * hk, hk, D, page, lengths, rows=rows)
    mask = torch.full((q.shape[0],), -1, device="cuda") if kind == "tree" else None
    if mask is not None:
        mask[0] = ~(1 << 10)
    counts = rows or [1] * 5
    for window, sinks in ((50, 20), (17, 0), (130, 3)):
        readable, hidden = table.clone(), table.clone()
        first = 0
        bad_k, bad_v = [t.clone() for t in (cache.k, cache.v)], None
        seen = torch.zeros(cache.pages, page, dtype=torch.bool, device="cuda")
        for b, length in enumerate(lengths.tolist()):
            see = sees(length, counts[b], window, sinks, None if mask is None else mask[first:first + counts[b]]).any(0)
            first += counts[b]
            for i in range(-(-length // page)):
                here = see[16 * i:16 * i + 16]
                if here.any():
                    seen[table[b, i].long(), :here.numel()] = here
                elif i % 2:
                    hidden[b, i] = (-1, cache.pages, 1 << 30)[i % 3]
        keep = [t.view(torch.uint8).clone() for t in (cache.k, cache.v)] + [s.clone() if s is not None else None for s in (cache.k_scale, cache.v_scale)]
        for i, x in enumerate((cache.k, cache.v)):
            if held == BF16:
                x.transpose(1, 2)[~seen] = math.nan if i else math.inf
            elif held == E4M3:
                x.view(torch.uint8).transpose(1, 2)[~seen] = 0x7F
                (cache.v_scale if i else cache.k_scale).transpose(1, 2)[~seen] = 255
            else:
                (cache.v_scale if i else cache.k_scale).permute(0, 3, 1, 2)[~seen] = 255 if i else 254
        out, lse = check(cache, hidden, lengths, q, starts, window, sinks, mask=mask, readable=readable)
        assert out.isfinite().all() and not lse.isnan().any()
        for t, was in zip((cache.k, cache.v), keep):
            t.view(torch.uint8).copy_(was)
        for s, was in zip((cache.k_scale, cache.v_scale), keep[2:]):
            if s is not None:
                s.copy_(was)
        del bad_k, bad_v


@pytest.mark.parametrize("held", CACHES)
@pytest.mark.parametrize("hq,D", [(16, 64), (8, 64), (16, 128)])
def test_hidden_nan_and_infinities_reach_only_the_rows_that_see_them(held, hq, D):
    """Five nodes whose heads fill two or four tiles (requests may be long)."""
    g = _gen(hq + D)
    cache, table, lengths, q, starts = case(g, held, BF16, hq, 2, D, 16, [100], rows=[5])
    for token, value in ((80, math.inf), (90, math.nan)):
        page, place = table[0, token // 16].long(), token % 16
        if held == BF16:
            cache.v[page, 1, place, token % 17] = value
        elif held == E4M3:
            cache.v.view(torch.uint8)[page, 1, place, token % 17] = 0x7F
        else:
            cache.v_scale[page, 1, token // 10 % (D // 32), place] = 255
    page, place = table[0, 85 // 16].long(), 85 % 16
    if held == E2M1:
        cache.k_scale[page, 0, 0, place] = 255
    elif held == E4M3:
        cache.k.view(torch.uint8)[page, 0, place, 3] = 0x7F
    else:
        cache.k[page, 0, place, 3] = math.nan
    hidden = (1 << 64) - 1
    for token in (80, 85, 90):
        hidden &= ~(1 << (token - 100 + 64))
    masks = [hidden | 1 << (80 - 36), hidden, hidden | 1 << (90 - 36), hidden | 1 << (85 - 36), hidden]
    mask = torch.tensor([m - (1 << 64) if m >> 63 else m for m in masks], device="cuda")
    for kw in ({}, {"max_length": 1 << 22}):
        out, lse = check(cache, table, lengths, q, starts, 1 << 29, 0, mask=mask, **kw)
        assert out[1].isfinite().all() and out[4].isfinite().all() and lse[1].isfinite().all()
        assert not out[0].isfinite().all() and not out[2].isfinite().all() and lse[3].isnan().any()
        if held == E2M1:
            four._check_attention(cache, table, lengths, q, starts, mask=mask, **kw)


@pytest.mark.parametrize("held", CACHES)
@pytest.mark.parametrize("dtype", [BF16, F32])
@pytest.mark.parametrize("hk,D", [(2, 64), (2, 128), (2, 256), (512, 64), (300, 128), (200, 256), (500, 32)])
def test_nan_and_infinities_reach_only_the_rows_that_see_them(held, dtype, hk, D):
    g = _gen(D)
    cache, table, lengths, q, starts = case(g, held, dtype, 2 * hk, hk, D, 16, [150], rows=[100])

    def spot(token):
        return table[0, token // 16].long(), token % 16
    for token, value in ((70, math.nan), (90, math.inf), (120, -math.inf)):
        page, place = spot(token)
        if held == BF16:
            cache.v[page, 1, place, 7 + token % 3] = value
        elif held == E4M3:
            cache.v.view(torch.uint8)[page, 1, place, 7 + token % 3] = 0x7F
        else:
            cache.v_scale[page, 1, 0, place] = 255
    page, place = spot(100)
    if held == E2M1:
        cache.k_scale[page, 0, 0, place] = 255
    elif held == E4M3:
        cache.k.view(torch.uint8)[page, 0, place, 3] = 0x7F
    else:
        cache.k[page, 0, place, 3] = math.nan
    for window, sinks in ((10, 0), (40, 4), (3, 75)):
        if held == BF16 or sinks < 70:
            out, lse = check(cache, table, lengths, q, starts, window, sinks)
            assert out[:20].isfinite().all()


def test_rows_and_lengths_that_say_more_than_there_is():
    g = _gen(9)
    for max_rows in (2, 100):
        cache, table, lengths, q, _ = case(g, BF16, BF16, 4, 2, 64, 16, [48, 48, 48, 48])
        out, lse = torch.full_like(q, 7.0), torch.full((4, 4), 7.0, device="cuda")
        starts = torch.tensor([0, 2, 1, 3, 90], dtype=torch.int32, device="cuda")
        wrong = torch.tensor([48, 1 << 30, -5, (1 << 31) - 1], dtype=torch.int32, device="cuda")
        vt.paged_attention(q, cache, table, wrong, row_start=starts, max_rows=max_rows, out=out, out_lse=lse, window=20, sinks=2)
        assert out.isfinite().all() and out[0].ne(7.0).any() and out[3].ne(7.0).any()
        assert out[2].eq(0).all() and lse[2].eq(-math.inf).all()      # (of no tokens; the row before it is two requests')
    # rows that belong to no request stay as they are
    out = torch.full_like(q, 7.0)
    vt.paged_attention(q, cache, table, lengths, row_start=torch.tensor([1, 2, 3, 3, 3], dtype=torch.int32, device="cuda"), max_rows=70, out=out, window=5)
    assert out[0].eq(7.0).all() and out[3].eq(7.0).all() and out[1].ne(7.0).any() and out[2].ne(7.0).any()


@pytest.mark.parametrize("rows", [[3, 2], [130, 70], [290, 1200]])
def test_rows_apart_in_place_and_on_another_stream(rows):
    g = _gen(12)
    cache, table, lengths, q, starts = case(g, BF16, BF16, 8, 2, 64, 16, [300, 4000], rows=rows)
    kw = dict(row_start=starts, max_rows=max(rows), window=2000, sinks=3)
    want = vt.paged_attention(q, cache, table, lengths, **kw)
    wide = torch.zeros(sum(rows), 10 * 64, device="cuda", dtype=BF16)
    wide[:, 64:9 * 64] = q.flatten(1)
    apart = wide[:, 64:9 * 64].unflatten(1, (8, 64))
    stream = torch.cuda.Stream()
    stream.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(stream):
        got = vt.paged_attention(apart, cache, table, lengths, out=apart, **kw)
    torch.cuda.current_stream().wait_stream(stream)
    assert torch.equal(got, want) and wide[:, :64].eq(0).all() and wide[:, 9 * 64:].eq(0).all()


def test_a_cache_beyond_32_bits():
    hk, D, page = 8, 128, 64
    pages = (5 << 30) // (hk * D * page * 2)
    cache = vt.KVCache(pages, page, hk, D)
    g = _gen(13)
    table = torch.tensor([[pages - 1, 5, pages - 2, 3]], dtype=torch.int32, device="cuda")
    k, v = _randn(g, 250, hk, D).to(BF16), _randn(g, 250, hk, D).to(BF16)
    vt.kv_cache_write(cache, k, v, cache.slots(table, torch.zeros(250, dtype=torch.int64, device="cuda"), torch.arange(250, device="cuda")))
    length = torch.tensor([250], dtype=torch.int32, device="cuda")
    check(cache, table, length, _randn(g, 1, 8, D).to(BF16), None, 100, 10)
    for hq in (8, 1000):
        check(cache, table, length, _randn(g, 200, hq, D).to(BF16), torch.tensor([0, 200], dtype=torch.int32, device="cuda"), 100, 10)


@pytest.mark.parametrize("rows", [[1, 1], [4, 2], [150, 90], [600, 90]])
def test_captured_in_a_graph(rows):
    g = _gen(14)
    cache, table, lengths, q, starts = case(g, E2M1, BF16, 32, 8, 64, 16, [2500, 410], rows=rows)
    mask = torch.randint(-(1 << 62), 1 << 62, (sum(rows),), generator=g, device="cuda") if rows[0] == 4 else None
    ws = vt.AttentionWorkspace(sum(rows), 32, 8, 64, 2, max(rows), 2500, "cuda")
    out = torch.empty_like(q)
    call = lambda: vt.paged_attention(q, cache, table, lengths, row_start=starts, max_rows=max(rows), tail_mask=mask, max_length=2500, ws=ws, out=out,      # noqa: E731
                                      window=1200, sinks=4)
    call()
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        call()
    for i in range(4):
        q.copy_(_randn(g, *q.shape))
        lengths.copy_(torch.tensor([2500 - 300 * i, 410 - 100 * i], device="cuda"))
        graph.replay()
        torch.cuda.synchronize()
        got = out.clone()
        out.zero_()
        call()
        assert torch.equal(got, out)


def test_the_same_every_time():
    g = _gen(15)
    for rows in (None, [200, 100, 1]):
        cache, table, lengths, q, starts = case(g, BF16, BF16, 64, 16, 128, 64, [3000, 700, 90], rows=rows)
        kw = dict(row_start=starts, max_rows=200 if rows else None, window=1024, sinks=4, return_lse=True)
        want = vt.paged_attention(q, cache, table, lengths, **kw)
        for _ in range(5):
            got = vt.paged_attention(q, cache, table, lengths, **kw)
            assert torch.equal(got[0], want[0]) and torch.equal(got[1], want[1])


def _calls():
    g = _gen(20)
    cache, table, lengths, rows, starts = case(g, E4M3, BF16, 4, 2, 64, 16, [400, 30], rows=[3, 2])
    ws = vt.AttentionWorkspace(5, 4, 2, 64, 2, 3, 512, "cuda")
    mask = torch.randint(-(1 << 62), 1 << 62, (5,), generator=g, device="cuda")
    plain = dict(q=rows, cache=cache, page_table=table, lengths=lengths, row_start=starts, max_rows=3, max_length=512, ws=ws, return_lse=True)
    return [dict(plain, window=50, sinks=2), dict(plain, window=50, sinks=0, tail_mask=mask), dict(plain, window=9, sinks=5, tail_mask=mask, positions=mask % 400)]


def test_the_native_way_and_pythons_give_the_same(monkeypatch):
    vt.load_library()
    native = binding._bind
    assert native is not None
    for args in _calls():
        cases = [args]
        for key in ("window", "sinks"):
            cases += [dict(args, **{key: v}) for v in (0, -1, 1 << 30, (1 << 30) + 1, 1 << 40, 2.5, math.nan, "1", None)]
        if "positions" in args:
            p = args["positions"]
            cases += [dict(args, positions=v) for v in (p.int(), p.cpu(), p.double(), p[:-1].contiguous(), 3, None)] + [dict(args, tail_mask=None), dict(args, window=None)]
        for changed in cases:
            both = []
            for way in (native, None):
                monkeypatch.setattr(binding, "_bind", way)
                both.append(_outcome(vt.paged_attention, changed))
            assert type(both[0]) is type(both[1]), (both, changed["window"], changed["sinks"])
            if isinstance(both[0], list):
                for x, y in zip(*both):
                    assert torch.equal(x, y)
            else:
                assert both[0] == both[1]


def test_plain_calls_take_the_native_way(monkeypatch):
    asked = []

    class Spy:
        def __getattr__(self, name):
            def call(*a):
                got = getattr(native, name)(*a)
                asked.append(got is not None)
                return got
            return call
    vt.load_library()
    native = binding._bind
    monkeypatch.setattr(binding, "_bind", Spy())
    for args in _calls():
        vt.paged_attention(**args)
    assert asked == [True] * 3


def test_refusals():
    cache = vt.KVCache(2, 16, 2, 64)
    q = torch.ones(2, 4, 64, device="cuda", dtype=BF16)
    table, lengths = torch.zeros(2, 2, dtype=torch.int32, device="cuda"), torch.ones(2, dtype=torch.int32, device="cuda")
    mask, at = torch.zeros(2, dtype=torch.int64, device="cuda"), torch.zeros(2, dtype=torch.int64, device="cuda")
    for kw in ({"sinks": 4}, {"positions": at}, {"positions": at, "window": 5}, {"window": 5, "tail_mask": mask, "positions": at[:1]}):
        with pytest.raises(ValueError):
            vt.paged_attention(q, cache, table, lengths, **kw)
    with pytest.raises(TypeError):
        vt.paged_attention(q, cache, table, lengths, window=5, tail_mask=mask, positions=at.double())
    with pytest.raises(ValueError):
        vt.paged_attention(q.clone().requires_grad_(), cache, table, lengths, window=5)
    for kw in ({"window": 0}, {"window": -3}, {"window": (1 << 30) + 1}, {"window": 5, "sinks": -1}):
        with pytest.raises(vt.VocabTrimError) as e:
            vt.paged_attention(q, cache, table, lengths, **kw)
        assert e.value.status == 2
