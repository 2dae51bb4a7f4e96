"""Attention of values where sums of bf16 terms, scales and masks can go wrong: infinities on either side, weights that bf16 does not hold, scale
bytes at the ends of their range.  Against the definitions in 64 bits, with the tolerances of test_gpu_attention.py."""
import math

import pytest
import torch

import paper_2506_22694_amd as vt
from test_gpu_attention import BF16, E4M3, F32, _case, _check_attention, _gen, _randn, _values, attend64

pytestmark = pytest.mark.gpu


def _place(table, page, token, b=0):
    return table[b, token // page].long(), token % page


# ---------------------------------------------------------------------------------------------- infinities that rows see
@pytest.mark.parametrize("D", [64, 96, 128, 256])
@pytest.mark.parametrize("dtype", [BF16, F32])
@pytest.mark.parametrize("length", [5, 300, 3000])      # (a request taken whole, and in shares)
def test_scores_of_minus_infinity(D, dtype, length):
    """Keys of -inf under positive queries: tokens as if not seen; all of them: nothing is seen."""
    g = _gen(D + length)
    hk, page = 2, 16
    cache, table, lengths, q, _ = _case(g, BF16, dtype, 4, hk, D, page, [length, length])
    q = q.abs()
    for token in {0, length // 2, length - 1} - {1}:
        page_id, at = _place(table, page, token)
        cache.k[page_id, :, at] = -math.inf
        cache.k[page_id, 0, at, 1:] = cache.k[page_id, 0, at, 1:].clamp(min=0.0)      # (of one head one value only)
    out, lse = _check_attention(cache, table, lengths, q, None)
    assert out.isfinite().all() and lse.isfinite().all()
    cache.k.fill_(-math.inf)
    out, lse = vt.paged_attention(q, cache, table, lengths, return_lse=True)
    assert out.eq(0).all() and lse.eq(-math.inf).all()


@pytest.mark.parametrize("D", [64, 128, 256])
@pytest.mark.parametrize("dtype", [BF16, F32])
@pytest.mark.parametrize("held", [BF16, E4M3])
def test_queries_of_infinity_and_the_largest_values(D, dtype, held):
    g = _gen(D)
    cache, table, lengths, q, _ = _case(g, held, dtype, 4, 2, D, 16, [200, 1000])
    k = cache.k.view(torch.uint8) if held == E4M3 else cache.k
    k[..., 3] = 0xB8 if held == E4M3 else -1.0      # -1 in e4m3
    q[0, 1, 3] = math.inf      # every score is -inf
    q[1, 2, 3] = -math.inf      # ... +inf, which has no weights
    out, lse = vt.paged_attention(q, cache, table, lengths, return_lse=True)
    assert out[0, 1].eq(0).all() and lse[0, 1] == -math.inf
    assert out[1, 2].isnan().all() and out[0, 0].isfinite().all() and out[1, 3].isfinite().all()
    # the largest finite values, on keys that bring them back to scores of some size
    if held == BF16:
        q[0, 1, 3] = q[1, 2, 3] = torch.finfo(dtype).max
        cache.k[..., 3] = (_randn(g, *cache.k.shape[:3]) * 2.0 ** -126).to(BF16)
        _check_attention(cache, table, lengths, q, None)


@pytest.mark.parametrize("D", [64, 80, 128, 256])
@pytest.mark.parametrize("dtype", [BF16, F32])
@pytest.mark.parametrize("rows", [None, [2, 9]])
def test_values_of_infinity_and_nan_that_all_rows_see(D, dtype, rows):
    """... reach their own column of the result and no other, before the last 64 tokens and among them, with a mask or without."""
    g = _gen(D)
    hk, page = 2, 32
    cache, table, lengths, q, starts = _case(g, BF16, dtype, 8, hk, D, page, [2100, 350], rows=rows)
    for b, token, head, d, value in ((0, 70, 0, 5, math.inf), (0, 71, 0, 5, math.inf), (0, 2099, 0, 6, -math.inf), (0, 1000, 1, 7, math.nan), (1, 3, 1, 11, -math.inf),
                                     (1, 9, 0, 2, math.inf), (1, 349, 0, 2, -math.inf), (1, 349, 0, 12, math.inf)):      # (of both signs: NaN)
        page_id, at = _place(table, page, token, b)
        cache.v[page_id, head, at, d] = value
    n = q.shape[0]
    for mask in (None, torch.full((n,), -1, device="cuda")):
        out, lse = _check_attention(cache, table, lengths, q, starts, mask=mask)
        assert lse.isfinite().all()
        assert out[-1, 4:, 11].eq(-math.inf).all() and out[-1, :4, 2].isnan().all() and out[0, :4, 5].eq(math.inf).all() and out[0, 4:, 7].isnan().all()
        assert out[0].isfinite().sum() == 8 * D - 12 and out[-1].isfinite().sum() == 8 * D - 12


# ---------------------------------------------------------------------------------------------- weights of 24 bits
def test_weights_that_bf16_does_not_hold():
    """One token of weight 1, all others just above 1/2 and off by the same part of it in bf16; values of 1: the result is 1."""
    cache, table, lengths, q, _ = _case(_gen(1), BF16, BF16, 4, 2, 64, 16, [40, 300, 3000])
    cache.k.zero_()
    cache.v.fill_(1.0)
    cache.k[..., 0] = 1.0
    for b in range(3):
        page_id, at = _place(table, 16, 7, b)
        cache.k[page_id, :, at] = 0.0
    q.zero_()
    q[..., 0] = 1.0
    out = vt.paged_attention(q, cache, table, lengths, scale=math.log(0.5 + 0.9 * 2.0 ** -9))
    assert out.eq(1.0).all()


@pytest.mark.parametrize("hq,hk,D", [(4, 2, 64), (32, 8, 128), (6, 3, 256), (40, 1, 64), (12, 2, 96)])
@pytest.mark.parametrize("held", [BF16, E4M3])
@pytest.mark.parametrize("rows", [None, [5, 2, 8]])
def test_results_of_bf16_rows_are_rounded_once(hq, hk, D, held, rows):
    g = _gen(hq + D)
    cache, table, lengths, q, starts = _case(g, held, BF16, hq, hk, D, 32, [333, 2222, 64], rows=rows)
    mask = None if rows is None else torch.randint(-(1 << 63), (1 << 63) - 1, (15,), generator=g, device="cuda") | 1
    out = vt.paged_attention(q, cache, table, lengths, row_start=starts, max_rows=1 if rows is None else 8, tail_mask=mask)
    first = [0, 1, 2, 3] if rows is None else starts.tolist()
    for b, length in enumerate(lengths.tolist()):
        at = slice(first[b], first[b + 1])
        k, v = _values(cache, table, b, length)
        see = torch.ones(first[b + 1] - first[b], length, dtype=torch.bool, device="cuda")
        if mask is not None:
            bit = torch.arange(length, device="cuda") - (length - 64)
            see &= (bit < 0) | (mask[at][:, None] >> bit.clamp(min=0) & 1).bool()
        want = attend64(q[at], k, v, see, D ** -0.5)[0]
        # half a step at the value itself, and fp32's part: scores off by (sqrt(D) / 2 + 8) half steps of the sum of their products' sizes, and 40 for
        # exp2 and the sums, as a part of every weight, above and below the line
        sizes = (q[at].double().abs()[:, None] * k.abs().repeat_interleave(hq // hk, 1)[None]).sum(-1).max().item() * D ** -0.5
        fp32 = (sizes * (math.sqrt(D) / 2 + 8) + 40) * 2.0 ** -24
        half = torch.ldexp(torch.ones_like(want), torch.frexp(want).exponent - 9)
        off = (out[at].double() - want).abs() - half - 2 * fp32 * attend64(q[at], k, v.abs(), see, D ** -0.5)[0]
        assert off.max().item() <= 0.0


# ---------------------------------------------------------------------------------------------- scale bytes at the ends of their range
@pytest.mark.parametrize("dtype", [BF16, F32])
@pytest.mark.parametrize("D", [64, 128, 256])
@pytest.mark.parametrize("rows", [2, 9])
def test_hidden_tokens_may_hold_any_scale(D, dtype, rows):
    """Tokens that a mask hides were never written: scales and codes of 255 there, beside tokens that are seen.  A row that sees one gets what
    comes of it, the others nothing."""
    g = _gen(D + rows)
    hk, page, length = 2, 16, 150
    cache, table, lengths, q, starts = _case(g, E4M3, dtype, 4, hk, D, page, [length, 70], rows=[rows, 2])
    hidden = (1 << 64) - 1
    for token, k_scale, v_scale, code in ((100, 255, 255, None), (101, 3, 255, 0x00), (117, 255, 3, 0x7F), (149, 255, 255, 0xFF), (140, 254, 255, 0x7E)):
        page_id, at = _place(table, page, token)
        cache.k_scale[page_id, :, at], cache.v_scale[page_id, :, at] = k_scale, v_scale
        if code is not None:
            cache.k.view(torch.uint8)[page_id, :, at] = code
            cache.v.view(torch.uint8)[page_id, :, at] = code
        hidden &= ~(1 << (token - length + 64))
    mask = torch.full((rows + 2,), hidden - (hidden >> 63 << 64), device="cuda")
    mask[rows:] = -1
    want, _ = _check_attention(cache, table, lengths, q, starts, mask=mask)
    assert want.isfinite().all()
    mask[0] |= 1 << (101 - length + 64)
    out = vt.paged_attention(q, cache, table, lengths, row_start=starts, max_rows=rows, tail_mask=mask)
    assert torch.equal(out[1:], want[1:])


def test_every_scale_byte_reads_back_as_its_power_of_two():
    page, D = 256, 16
    codes = torch.tensor([0x00, 0x01, 0x07, 0x08, 0x38, 0x39, 0x7E, 0x7F, 0x80, 0x81, 0x87, 0x88, 0xB8, 0xB9, 0xFE, 0xFF], dtype=torch.uint8, device="cuda")
    held = codes.expand(1, 1, page, D).contiguous()
    scale = torch.arange(256, dtype=torch.uint8, device="cuda").view(1, 1, page)
    cache = vt.KVCache.of(held.view(E4M3), held.clone().view(E4M3), scale, scale.clone())
    powers = torch.tensor([math.ldexp(1.0, i - 127) for i in range(256)], dtype=torch.float64, device="cuda")
    want = codes.view(E4M3).double()[None] * powers[:, None]
    for got in vt.kv_cache_read(cache, torch.arange(page, device="cuda"), dtype=F32):
        got = got[:, 0]
        assert torch.equal(got.isnan(), want.isnan())
        sure = (want == 0) | ((want.abs() >= 2.0 ** -126) & (want.abs() < 2.0 ** 128))
        assert torch.equal(got.double()[sure], want[sure])
        beyond = want.abs() >= 2.0 ** 128
        assert torch.equal(got.double()[beyond], want[beyond].sign() * math.inf)


@pytest.mark.parametrize("dtype", [BF16, F32])
@pytest.mark.parametrize("byte", [0, 1, 60, 200])
def test_attention_over_keys_of_any_scale(dtype, byte):
    """Scores of one scale byte, brought back to some size by the scale of the call or by queries."""
    g = _gen(byte)
    cache, table, lengths, q, _ = _case(g, E4M3, dtype, 4, 2, 64, 32, [300, 1000])
    cache.k_scale.fill_(byte)
    near = max(min(127 - byte, 100), -100)      # of the scale of the call; the rest in the queries, whose own values fp32 holds
    q = (q.double() * 2.0 ** (127 - byte - near)).to(dtype)
    _check_attention(cache, table, lengths, q, None, scale=2.0 ** (near - 10))
