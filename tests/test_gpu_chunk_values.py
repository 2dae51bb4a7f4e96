"""Chunks of prompts over values where sums of bf16 terms can go wrong: infinities that every row sees, several tiles inside the window, met with weights
whose lower bits are zero.  Against 64 bits by the definition, with the tolerances of test_gpu_window_attention.py."""
import math

import pytest
import torch

import paper_2506_22694_amd as vt
from test_gpu_attention import BF16, E4M3, _gen
from test_gpu_four_bits import E2M1
from test_gpu_window_attention import WIDE, case, check

pytestmark = pytest.mark.gpu

# Chunks of enough work go through a kernel of their own: over 8 and 4 bits, heads past 128 values do with many kv heads
PAST_128 = [(512, 512, 256), (320, 320, 160), (448, 224, 192)]


def hold(cache, table, token, head, d, value, b=0):
    """An infinity (4 bits: a group of zeros beside it, 6 or -6 at a scale of 2^127) or NaN as value d of a token's row."""
    page, place = table[b, token // cache.page_size].long(), token % cache.page_size
    if cache.v.dtype == BF16:
        cache.v[page, head, place, d] = value
        return
    codes = cache.v.view(torch.uint8)[page, head, place]
    if cache.v.dtype == E4M3:
        assert math.isnan(value)
        codes[d] = 0x7F
        return
    group = d // 32
    codes[16 * group:16 * group + 16] = 0
    codes[d // 2] = (0xF if value < 0 else 7) << 4 * (d % 2)
    cache.v_scale[page, head, group, place] = 255 if math.isnan(value) else 254


@pytest.mark.parametrize("held", [BF16, E2M1])
@pytest.mark.parametrize("hq,hk,D", WIDE + PAST_128)
def test_infinities_that_every_row_sees(held, hq, hk, D):
    """Rows of q = 0 have weights of 1, of which bf16 holds all; other rows a token of weight 1 where the largest score's is."""
    g = _gen(hq + D)
    cache, table, lengths, q, starts = case(g, held, BF16, hq, hk, D, 16, [700, 640], rows=[130, 100])
    q[::3] = 0.0
    hold(cache, table, 200, 0, 5, math.inf)
    hold(cache, table, 350, 1, D - 3, -math.inf)
    hold(cache, table, 330, hk - 1, 9, math.nan)
    hold(cache, table, 223, 2, 1, math.inf, 1)
    hold(cache, table, 222, 2, 1, math.inf, 1)
    if held == BF16:
        # the largest score of a row of each kv head, x |q|^2 / sqrt(D), |q|^2 = 2.25 D or so: of 256 values 52 at x = 1 (104 at x = 2) times log 2, and the
        # infinities' weights 2^-52 of its own (2^-104, less than what reaches a row)
        cache.k[table[0, 350 // 16].long(), :, 350 % 16] = (2.0 if D <= 160 else 1.0) * q[1].view(hk, -1, D)[:, 0]
    for window, sinks in ((600, 0), (500, 40), (1 << 30, 0)):
        out, lse = check(cache, table, lengths, q, starts, window, sinks)
        G = hq // hk
        assert out[:130, :G, 5].eq(math.inf).all() and out[:130, G:2 * G, D - 3].eq(-math.inf).all() and out[130:, 2 * G:3 * G, 1].eq(math.inf).all()
        assert out[:130, -G:, 9].isnan().all() and lse.isfinite().all()


@pytest.mark.parametrize("held", [BF16, E2M1])
@pytest.mark.parametrize("hq,hk,D", [(16, 4, 128), (6, 2, 64), (5, 1, 256)])
def test_infinities_in_a_share_of_a_chunk(held, hq, hk, D):
    g = _gen(hq)
    cache, table, lengths, q, starts = case(g, held, BF16, hq, hk, D, 64, [9000, 5003], rows=[130, 77])
    q[::2] = 0.0
    hold(cache, table, 4000, 0, 5, math.inf)
    hold(cache, table, 2500, hk - 1, 6, -math.inf, 1)
    for window, sinks in ((8000, 4), (5000, 700), (1 << 30, 0)):
        out, _ = check(cache, table, lengths, q, starts, window, sinks)
        if window >= 8000:
            assert out[:130, :hq // hk, 5].eq(math.inf).all() and out[130:, -(hq // hk):, 6].eq(-math.inf).all()


@pytest.mark.parametrize("held", [BF16, E2M1])
@pytest.mark.parametrize("D", [64, 128, 256])
@pytest.mark.parametrize("rows", [2, 130])      # (few rows and chunks have a kernel each)
def test_infinities_of_small_weights(held, D, rows):
    """Weights that are powers of two, down to 2^-100 of the row's largest: scores are whole numbers times log 2."""
    g = _gen(D)
    hk = 96 if D <= 128 else 512
    cache, table, lengths, q, starts = case(g, held, BF16, hk, hk, D, 16, [700], rows=[rows])
    assert float(torch.tensor(math.log(2.0), dtype=torch.float32) * torch.tensor(1.4426950408889634, dtype=torch.float32)) == 1.0
    q.zero_()
    q[..., 0] = -1.0
    (cache.k.view(torch.uint8) if held == E2M1 else cache.k).zero_()
    exponents = torch.tensor([0, 1, 2, 23, 24, 60, 96], device="cuda")
    page, place = table[0, 200 // 16].long(), 200 % 16
    for head in range(hk):
        e = int(exponents[head % 7])
        if held == BF16:
            cache.k[page, head, place, 0] = float(e)
        elif e:      # 1, 2, 3 * 2^3, ...: a magnitude of the codes times a power of two
            e = {23: 24}.get(e, e)
            m = max(i for i, x in enumerate((0, 0.5, 1, 1.5, 2, 3, 4, 6)) if x and math.log2(e / x) % 1 == 0) if e != 60 else 0
            if e == 60:
                e, m = 64, 6
            size = (0, 0.5, 1, 1.5, 2, 3, 4, 6)[m]
            cache.k.view(torch.uint8)[page, head, place, 0] = m
            cache.k_scale[page, head, 0, place] = 127 + int(math.log2(e / size))
        hold(cache, table, 200, head, 7, math.inf)
    out, lse = check(cache, table, lengths, q, starts, 600, 0, scale=math.log(2.0))
    assert out[:, :, 7].eq(math.inf).all() and lse.isfinite().all()


@pytest.mark.parametrize("hq,hk,D", WIDE)
@pytest.mark.parametrize("rows", [2, 130])
def test_infinities_at_scores_of_minus_infinity_beside_a_window(hq, hk, D, rows):
    """Where a window begins or ends, a token of weight 0 is as one that is not seen: in a chunk as in few rows."""
    g = _gen(D)
    cache, table, lengths, q, starts = case(g, BF16, BF16, hq, hk, D, 16, [700], rows=[rows])
    q = q.abs()
    out = []
    for value in (math.inf, -math.inf, math.nan, 0.0):
        for token in (670, 690) if rows == 2 else (580, 600, 633, 690):
            page, place = table[0, token // 16].long(), token % 16
            cache.k[page, :, place] = -math.inf
            cache.v[page, :, place, token % 7] = value
        out.append(vt.paged_attention(q, cache, table, lengths, row_start=starts, max_rows=rows, window=40, return_lse=True))
    whole = q.ne(0).all(-1)      # (0 * -inf is NaN: a query with a zero in it, one of millions, has a score of NaN)
    for got in out[:-1]:
        assert torch.equal(got[0][whole], out[-1][0][whole]) and torch.equal(got[1][whole], out[-1][1][whole])
    assert out[-1][0][whole].isfinite().all() and out[-1][1][whole].isfinite().all() and whole.sum() > 0.99 * whole.numel()


@pytest.mark.parametrize("held", [BF16, E4M3, E2M1])
@pytest.mark.parametrize("D", [64, 128, 256])
@pytest.mark.parametrize("rows", [2, 130])
def test_bits_of_weights(held, D, rows):
    """A token of weight 1 and value -3/4 beside one of weight w, about 3/4, and value 1: (w - 3/4) / (1 + w) is small, and has w's error whole.  Chunks, and bf16
    rows over 4 bits, hold a weight as 8 bits that are cut off and a rest below 2^-7 of it that is rounded to 8: off by 2^-16 at most.  Others hold 24 bits.  fp32's part: z is
    a sum of two products, exp2 and the sums are off by some half steps of 2^-24: 2^-20 covers 16."""
    hk, length = 96 if D <= 128 else 512, 700
    cache, table, lengths, q, starts = case(_gen(D), held, BF16, hk, hk, D, 16, [length], rows=[rows])
    page_a, at_a = table[0, 300 // 16].long(), 300 % 16
    page_b, at_b = table[0, 411 // 16].long(), 411 % 16
    one, small = {BF16: (1.0, 0.75), E4M3: (0x38, 0x34), E2M1: (4, 3)}[held]      # (4 bits: of a scale of 1/2)
    if held == BF16:
        k, v = cache.k, cache.v
    else:
        k, v = torch.zeros(2, *cache.k.shape[:3], D, dtype=torch.uint8, device="cuda").unbind(0)
        for s in (cache.k_scale, cache.v_scale):
            s.fill_(127 if held == E4M3 else 126)
    k.zero_(), v.zero_()
    k[..., 0] = one      # all other tokens: far below
    k[page_a, :, at_a] = 0
    k[page_b, :, at_b] = 0
    k[page_b, :, at_b, 1] = k[page_b, :, at_b, 2] = one
    v[page_a, :, at_a] = -small if held == BF16 else small + (0x80 if held == E4M3 else 8)
    v[page_b, :, at_b] = one
    if held == E4M3:
        cache.k.view(torch.uint8).copy_(k), cache.v.view(torch.uint8).copy_(v)
    elif held == E2M1:
        for x, y in ((cache.k, k), (cache.v, v)):
            x.view(torch.uint8).copy_(y[..., ::2] + 16 * y[..., 1::2])
    q.zero_()
    q[..., 0] = -4000.0
    q[..., 1] = math.log2(0.75)
    q[..., 2] = (torch.rand(q.shape[:2], generator=_gen(D + 1), device="cuda") * 2 - 1) * 2.0 ** -7
    w = torch.exp2(q[..., 1].double() + q[..., 2].double())[..., None]
    want = (w - 0.75) / (1 + w)
    out, lse = vt.paged_attention(q, cache, table, lengths, row_start=starts, max_rows=rows, window=length, scale=math.log(2.0), return_lse=True)
    error = (2.0 ** -16 if rows > 2 or held == E2M1 else 0.0) + 2.0 ** -20
    half = torch.ldexp(torch.ones_like(want), torch.frexp(want).exponent - 9)      # of a step of bf16 at the value itself
    assert ((out.double() - want).abs() - half - error * w / (1 + w)).max().item() <= 0.0
    assert (lse.double() - torch.log1p(w[..., 0])).abs().max().item() <= 2.0 ** -20


@pytest.mark.parametrize("byte", [0, 1, 2, 3, 120, 246])
@pytest.mark.parametrize("hk,D,rows", [(256, 64, 130), (96, 128, 130), (512, 256, 300)])
def test_values_of_eight_bits_in_chunks_are_those_of_bf16(byte, hk, D, rows):
    """Each row sees its own token alone: what 8 bits hold of it, rounded to bf16 (below 2^-126 to multiples of 2^-133)."""
    cache, table, lengths, q, starts = case(_gen(D), E4M3, BF16, hk, hk, D, 16, [700], rows=[rows])
    codes = torch.arange(256, device="cuda", dtype=torch.uint8)
    codes = codes[(codes & 0x7F) != 0x7F][:254]
    cache.v.view(torch.uint8).copy_(codes[torch.randint(0, 254, cache.v.shape, generator=_gen(byte), device="cuda")])
    cache.v_scale.fill_(byte)
    out = vt.paged_attention(q, cache, table, lengths, row_start=starts, max_rows=rows, window=1)
    slots = cache.slots(table, torch.zeros(rows, dtype=torch.int64, device="cuda"), torch.arange(700 - rows, 700, device="cuda"))
    held = cache.v.view(torch.uint8).transpose(1, 2).reshape(-1, hk, D)[slots].view(E4M3).double() * 2.0 ** (byte - 127)
    assert torch.equal(out, held.float().to(BF16))
    assert torch.equal(out, vt.kv_cache_read(cache, slots)[1])


@pytest.mark.parametrize("held", [BF16, E4M3, E2M1])
@pytest.mark.parametrize("D", [64, 128, 256])
@pytest.mark.parametrize("rows", [2, 130])
@pytest.mark.parametrize("later", [0, 3, 7, 9, 40])
def test_the_largest_values(held, D, rows, later):
    """A token of values of 2^125, its score log 2 times `later` above all others': results of no more than that, whatever base the weights are counted from."""
    hk, length = 96 if D <= 128 else 512, 700
    cache, table, lengths, q, starts = case(_gen(D), held, BF16, hk, hk, D, 16, [length], rows=[rows])
    page, place = table[0, 411 // 16].long(), 411 % 16
    for x, s in ((cache.k, cache.k_scale), (cache.v, cache.v_scale)):
        (x if held == BF16 else x.view(torch.uint8)).zero_()
        if s is not None:
            s.fill_(127)
    if held == BF16:
        cache.k[page, :, place, 0] = 1.0
        cache.v[page, :, place] = 2.0 ** 125
    elif held == E4M3:
        cache.k.view(torch.uint8)[page, :, place, 0] = 0x38
        cache.v.view(torch.uint8)[page, :, place] = 0x38
        cache.v_scale[page, :, place] = 252
    else:
        cache.k.view(torch.uint8)[page, :, place, 0] = 2
        cache.v.view(torch.uint8)[page, :, place] = 0x22
        cache.v_scale[page, :, :, place] = 252
    q.zero_()
    q[..., 0] = later
    out, lse = check(cache, table, lengths, q, starts, length, 0, scale=math.log(2.0))
    assert out.isfinite().all() and out[0, 0, 0] >= 2.0 ** 115


@pytest.mark.parametrize("hq,hk,D", PAST_128)
@pytest.mark.parametrize("held", [E4M3, E2M1])
def test_chunks_of_heads_past_128_values(held, hq, hk, D):
    a = case(_gen(hq + D), held, BF16, hq, hk, D, 64, [400, 390, 700, 70, 65], rows=[200, 1, 97, 70, 100])
    for window, sinks in ((1, 0), (7, 2), (33, 0), (100, 20), (1 << 30, 0), (3, 1 << 30)):
        check(*a, window, sinks)
    for scale in (0.0, -0.2):
        check(*a, 100, 4, scale=scale)
    # ... some of which only some rows see
    cache, table = a[:2]
    hold(cache, table, 260, 0, 5, math.nan)
    hold(cache, table, 350, hk - 1, D - 3, math.nan)
    hold(cache, table, 630, 3, 9, math.nan, 2)
    for window, sinks in ((100, 20), (1 << 30, 0)):
        out, _ = check(*a, window, sinks)
        assert out[:30].isfinite().all() and out.isnan().any()


def test_a_long_chunk_of_heads_past_128_values_in_shares():
    for held in (E4M3, E2M1):
        a = case(_gen(8), held, BF16, 8, 2, 256, 64, [30000, 9000], rows=[200, 130])
        for window, sinks in ((29000, 4), (1 << 30, 0)):
            out, lse = check(*a, window, sinks)
            again = vt.paged_attention(a[3], *a[:3], row_start=a[4], max_rows=200, window=window, sinks=sinks, return_lse=True)
            assert torch.equal(out, again[0]) and torch.equal(lse, again[1])
