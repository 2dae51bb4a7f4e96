"""Variants that the attention's calls choose by size alone: norm and rotation of several tokens to a workgroup (2048 tokens and more of few heads),
and the join by a wave of rows of up to 256 values.  Against the definitions in 64 bits, with the bounds of test_gpu_attention.py."""
import math

import pytest
import torch

import paper_2506_22694_amd as vt
from test_gpu_attention import (BF16, E4M3, F32, HALF, _case, _check_attention, _gen, _randn, _table64, close, held64, norm_rope64)

pytestmark = pytest.mark.gpu

# Tokens of a workgroup's at a time: the most of 2, 4 and 8 that leave 1024 workgroups and at most four heads to each group of lanes (256 / 8, 16 or 32
# lanes of a head).  n, q heads, k heads, values of a head, of them rotated
SEVERAL = [
    (2048, 8, 8, 128, 128),     # 2
    (2051, 5, 3, 256, 64),      # 2
    (4099, 6, 2, 96, 96),       # 4
    (8200, 4, 2, 128, 64),      # 8 (written with v: too)
    (9001, 7, 1, 16, 8),        # 8
    (2500, 17, 3, 64, 64),      # 2
]


def _inputs(n, hq, hk, D, rot, dtype, kv=1):
    g = _gen(n + D)
    rows = _randn(g, n, (hq + kv * hk) * D + 8).to(dtype)
    parts = [rows[:, :hq * D].unflatten(1, (hq, D))] + [rows[:, (hq + i * hk) * D:(hq + (i + 1) * hk) * D].unflatten(1, (hk, D)) for i in range(kv)]
    positions = torch.randint(0, 900, (n,), generator=g, device="cuda")
    w = [(_randn(g, D) * 0.3 + 1).to(dtype) for _ in range(2)]
    return g, parts, positions, _table64(900, rot), w


@pytest.mark.parametrize("n,hq,hk,D,rot", SEVERAL)
@pytest.mark.parametrize("dtype", [BF16, F32])
@pytest.mark.parametrize("interleaved", [False, True])
def test_norm_rope_of_several_tokens(n, hq, hk, D, rot, dtype, interleaved):
    _, (q, k), positions, table, w = _inputs(n, hq, hk, D, rot, dtype)
    got = vt.qk_norm_rope(q, k, positions, table, *w, eps=1e-5, interleaved=interleaved)
    for x, wx, y in ((q, w[0], got[0]), (k, w[1], got[1])):
        # fp32: a sum of D squares (D / 2 + 8 roundings at most, half of them to the root), two products and the rotation's three
        z = norm_rope64(x, None, None, wx, 1e-5, interleaved).abs()
        close(y, norm_rope64(x, positions, table, wx, 1e-5, interleaved), HALF[dtype], (D / 16 + 16) * 2.0 ** -24 * z.amax(-1, keepdim=True) * 2)


@pytest.mark.parametrize("n,hq,hk,D,rot", SEVERAL)
@pytest.mark.parametrize("dtype", [BF16, F32])
def test_gradients_of_several_tokens(n, hq, hk, D, rot, dtype):
    g, (q, k), positions, table, w = _inputs(n, hq, hk, D, rot, dtype)
    gq, gk = _randn(g, n, hq, D).to(dtype), _randn(g, n, hk, D).to(dtype)
    dq, dk, dwq, dwk = vt.qk_norm_rope_backward(gq, gk, q, k, positions, table, *w, eps=1e-5)
    for x, gy, wx, dx, dw in ((q, gq, w[0], dq, dwq), (k, gk, w[1], dk, dwk)):
        x64, w64 = x.double().requires_grad_(), wx.double().requires_grad_()
        norm_rope64(x64, positions, table, w64, 1e-5, False).backward(gy.double())
        r = 1 / (x.double().square().mean(-1, keepdim=True) + 1e-5).sqrt()
        size, unit = gy.double().abs().amax(-1, keepdim=True) * wx.double().abs().max() * r, x.double().abs().amax(-1, keepdim=True) * r
        # fp32: two sums of D terms and a dozen operations, on terms of up to `size` times the row's largest unit value squared
        close(dx, x64.grad, HALF[dtype], (D / 16 + 24) * 2.0 ** -24 * size * (1 + unit * unit))
        terms = (gy.double().abs().amax() * x.double().abs().mul(r).amax()).item()
        close(dw, w64.grad, 0.0, (math.sqrt(n * x.shape[1]) * 4 + 64) * 2.0 ** -24 * terms * 4)


@pytest.mark.parametrize("n,hq,hk,D,rot", SEVERAL)
@pytest.mark.parametrize("held", [BF16, E4M3])
def test_cache_writes_of_several_tokens(n, hq, hk, D, rot, held):
    g, (q, k, v), positions, table, w = _inputs(n, hq, hk, D, rot, BF16, kv=2)
    page = 64
    cache = vt.KVCache(-(-n // page) + 2, page, hk, D, dtype=held)
    slots = torch.randperm(cache.pages * page, generator=g, device="cuda")[:n]
    slots[::97] = -1
    kept = slots >= 0
    before = cache.k.view(torch.uint8).random_(generator=g).clone()
    y = vt.qkv_to_cache(q, k, v, cache, slots, positions, table, *w)
    z = norm_rope64(q, None, None, w[0], 1e-6, False).abs()
    close(y, norm_rope64(q, positions, table, w[0], 1e-6, False), HALF[BF16], (D / 16 + 16) * 2.0 ** -24 * z.amax(-1, keepdim=True) * 2)
    got = vt.kv_cache_read(cache, slots, dtype=F32)
    assert got[0][~kept].eq(0).all() and got[1][~kept].eq(0).all()
    assert torch.equal(got[1][kept].double(), held64(v.double(), held)[kept])
    # fp32's rounding may fall on the other side of a border of the held type's: one step of it, for few
    k64 = norm_rope64(k, positions, table, w[1], 1e-6, False)
    want = held64(k64, held)
    off = (got[0].double() - want)[kept].abs()
    step = 2.0 ** -7 if held == BF16 else 2.0 ** -3
    assert (off <= step * want[kept].abs() + 2.0 ** -9 * k64[kept].abs().amax(-1, keepdim=True) / 224).all()
    assert (off > 0).float().mean().item() < (0.02 if held == BF16 else 0.002)
    other = torch.ones(cache.pages * page, dtype=torch.bool, device="cuda")
    other[slots[kept]] = False
    assert torch.equal(cache.k.view(torch.uint8).transpose(1, 2)[other.view(-1, page)], before.transpose(1, 2)[other.view(-1, page)])


@pytest.mark.parametrize("dtype", [BF16, F32])
@pytest.mark.parametrize("hq,hk,D,requests,rows", [(8, 2, 256, 24, 8), (8, 2, 208, 24, 8), (16, 16, 256, 40, 3)])
def test_many_rows_of_large_heads_are_joined(hq, hk, D, requests, rows, dtype):
    """More than 1024 rows and heads, of requests in shares; the last has more requests than shares."""
    g = _gen(D + hk)
    lengths = [[2100, 0, 700, 129, 1, 1030, 90][i % 7] for i in range(requests)]
    counts = [rows if i % 5 else i % (rows + 1) for i in range(requests)]
    case = _case(g, E4M3, dtype, hq, hk, D, 32, lengths, rows=counts)
    _check_attention(*case, max_length=2112)
