"""Norm and rotation with gradients, the paged cache and the attention over it, against plain implementations in 64 bits.

Tolerances count roundings: half a step of a type is finfo.eps / 2 relative.  fp32 arithmetic gets a bound over its sums (named at each
test); a result in bf16 adds its one rounding.  Attention of bf16 rows rounds its weights p once to bf16 as well, which are at most all
2^-9 off in the same direction.
"""
import ctypes
import math

import pytest
import torch

import paper_2506_22694_amd as vt
from paper_2506_22694_amd import binding

pytestmark = pytest.mark.gpu

BF16, F32, E4M3 = torch.bfloat16, torch.float32, torch.float8_e4m3fn
HALF = {BF16: 2.0 ** -8, F32: 2.0 ** -24}      # half a step, relative (of the larger power of two)


def _gen(seed):
    return torch.Generator(device="cuda").manual_seed(seed)


def _randn(g, *shape):
    return torch.randn(shape, generator=g, device="cuda")


def _table64(positions, rot):
    return vt.rope_table(positions, rot, 10000.0, "cuda")


# ---------------------------------------------------------------------------------------------- 64-bit definitions
def norm_rope64(x, positions, table, weight, eps, interleaved):
    x = x.double()
    if weight is not None:
        x = x / (x.square().mean(-1, keepdim=True) + eps).sqrt() * weight.double()
    if table is None:
        return x
    rot = table.shape[1]
    ok = (positions >= 0) & (positions < table.shape[0])
    t = table.double()[positions.clamp(0, table.shape[0] - 1).long()]
    t[~ok] = math.nan
    c, s = t[:, None, :rot // 2], t[:, None, rot // 2:]
    if interleaved:
        a, b = x[..., 0:rot:2], x[..., 1:rot:2]
    else:
        a, b = x[..., :rot // 2], x[..., rot // 2:rot]
    ra, rb = a * c - b * s, b * c + a * s
    turned = torch.stack([ra, rb], -1).flatten(-2) if interleaved else torch.cat([ra, rb], -1)
    return torch.cat([turned, x[..., rot:]], -1)


def power_of_two(e):
    """2^e in float64 (2.0 ** e and torch.ldexp go through a power function, which is an ulp off for some e on the device)."""
    return torch.tensor([math.ldexp(1.0, i) for i in range(-150, 151)], dtype=torch.float64, device=e.device)[e.long() + 150]


def held64(x, dtype):
    """What a cache holds of rows x (float64)."""
    if dtype == BF16:
        return x.float().to(BF16).double()
    finite = torch.where(x.isfinite(), x, 0.0)
    half, e = torch.frexp(finite.abs().amax(-1, keepdim=True))
    scale = power_of_two((e - 9 + (half > 0.875).int()).clamp(min=-126))
    most = torch.where(scale == 2.0 ** 120, 240.0, 448.0).double()      # (256 * 2^120 would be infinite in fp32)
    y = torch.minimum(torch.maximum(x / scale, -most), most)      # (NaN stays)
    return y.float().to(E4M3).double() * scale


def attend64(q, k, v, see, scale):
    """q [rows, hq, D], k and v [tokens, hk, D], see [rows, tokens]: out, lse."""
    rows, hq, D = q.shape
    hk = k.shape[1]
    q, k, v = q.double(), k.double(), v.double()
    out, lse = torch.zeros(rows, hq, D, dtype=torch.float64, device=q.device), torch.full((rows, hq), -math.inf, dtype=torch.float64, device=q.device)
    for i in range(rows):
        at = see[i].nonzero().flatten()
        if at.numel() == 0:
            continue
        kk, vv = k[at].repeat_interleave(hq // hk, 1), v[at].repeat_interleave(hq // hk, 1)      # [t, hq, D]
        s = (q[i][None] * kk).sum(-1) * scale
        lse[i] = torch.logsumexp(s, 0)
        out[i] = (torch.softmax(s, 0)[..., None] * vv).sum(0)
    return out, lse


def close(got, want, rel, floor=0.0):
    """|got - want| <= rel * |want| + floor, NaN and infinities alike."""
    got = got.double()
    assert torch.equal(got.isnan(), want.isnan())
    odd = ~want.isfinite()
    assert torch.equal(got[odd & ~want.isnan()], want[odd & ~want.isnan()])
    far = ((got - want).abs() - rel * want.abs())[~odd]
    if torch.is_tensor(floor):
        far = far - floor.expand(want.shape)[~odd]
        floor = 0.0
    assert far.numel() == 0 or far.max().item() <= floor, far.max().item()


# ---------------------------------------------------------------------------------------------- norm and rotation
SHAPES = [      # n, hq, hk, D, rot
    (1, 1, 1, 8, 8), (3, 4, 2, 64, 64), (5, 6, 2, 96, 64), (7, 3, 1, 80, 40), (2, 32, 8, 128, 128), (17, 5, 5, 128, 32), (4, 2, 2, 256, 256), (6, 9, 3, 200, 8),
    (1030, 2, 1, 16, 16), (1, 33, 31, 72, 72), (3, 0, 2, 64, 32), (3, 2, 0, 64, 32)]


@pytest.mark.parametrize("n,hq,hk,D,rot", SHAPES)
@pytest.mark.parametrize("dtype", [BF16, F32])
@pytest.mark.parametrize("interleaved", [False, True])
@pytest.mark.parametrize("norm,rope", [(True, True), (True, False), (False, True)])
def test_norm_rope(n, hq, hk, D, rot, dtype, interleaved, norm, rope):
    g = _gen(n * 1000 + D)
    rows = _randn(g, n, (hq + hk) * D + 16).to(dtype)      # views of wider rows
    q, k = rows[:, :hq * D].unflatten(1, (hq, D)) if hq else rows.new_empty(n, 0, D), rows[:, hq * D:(hq + hk) * D].unflatten(1, (hk, D)) if hk else rows.new_empty(n, 0, D)
    positions = torch.randint(0, 500, (n,), generator=g, device="cuda", dtype=torch.int32 if interleaved else torch.int64) if rope else None
    table = _table64(500, rot) if rope else None
    wq, wk = ((_randn(g, D) * 0.3 + 1).to(dtype), (_randn(g, D) * 0.3 + 1).to(dtype)) if norm else (None, None)
    got = vt.qk_norm_rope(q, k, positions, table, wq, wk, eps=1e-5, interleaved=interleaved)
    for x, w, y in ((q, wq, got[0]), (k, wk, got[1])):
        want = norm_rope64(x, positions, table, w, 1e-5, interleaved)
        assert y.dtype == dtype and y.is_contiguous() and y.shape == x.shape
        # fp32: a sum of D squares (D / 2 + 8 roundings at most, half of them to the root), two products and the rotation's three
        z = norm_rope64(x, None, None, w, 1e-5, interleaved).abs()
        fp32 = (D / 16 + 16) * 2.0 ** -24 * z.amax(-1, keepdim=True) * 2 if x.numel() else 0.0
        close(y, want, HALF[dtype], fp32)


def test_norm_rope_in_place_and_out_of_the_table():
    g = _gen(1)
    n, hq, hk, D, rot = 9, 4, 2, 64, 32
    q, k = _randn(g, n, hq, D).to(BF16), _randn(g, n, hk, D).to(BF16)
    w = torch.ones(D, device="cuda", dtype=BF16)
    table = _table64(50, rot)
    positions = torch.tensor([0, 49, 50, -1, 7, 1 << 40, -(1 << 62), 3, 3], device="cuda")
    want = vt.qk_norm_rope(q, k, positions, table, w, w)
    bad = torch.tensor([0, 0, 1, 1, 0, 1, 1, 0, 0], device="cuda", dtype=torch.bool)
    for y in want:
        assert y[bad][..., :rot].isnan().all() and y[bad][..., rot:].isfinite().all() and y[~bad].isfinite().all()
    a, b = q.clone(), k.clone()
    got = vt.qk_norm_rope(a, b, positions, table, w, w, q_out=a, k_out=b)
    assert got[0] is a and got[1] is b
    for x, y in zip(want, got):
        assert torch.equal(x.nan_to_num(7.0), y.nan_to_num(7.0))


def test_norm_rope_values_at_the_edges():
    D = 64
    x = torch.zeros(6, 1, D, device="cuda")
    x[1] = math.inf
    x[2, 0, 5] = math.nan
    x[3] = 1e-30
    x[4] = 3e18
    x[5, 0, 0] = 1.0
    w = torch.ones(D, device="cuda")
    y, _ = vt.qk_norm_rope(x, x, None, None, w, w, eps=1e-6)
    want = norm_rope64(x, None, None, w, 1e-6, False)
    assert y[0].eq(0).all() and y[1].isnan().all() and y[2].isnan().all()
    close(y[3:], want[3:], 32 * 2.0 ** -24)


@pytest.mark.parametrize("n,hq,hk,D,rot", SHAPES)
@pytest.mark.parametrize("dtype", [BF16, F32])
@pytest.mark.parametrize("interleaved,norm,rope", [(False, True, True), (True, True, True), (False, False, True), (False, True, False)])
def test_norm_rope_gradients(n, hq, hk, D, rot, dtype, interleaved, norm, rope):
    g = _gen(n + D)
    q, k = _randn(g, n, hq, D).to(dtype), _randn(g, n, hk, D).to(dtype)
    gq, gk = _randn(g, n, hq, D).to(dtype), _randn(g, n, hk, D).to(dtype)
    positions = torch.randint(0, 90, (n,), generator=g, device="cuda") if rope else None
    table = _table64(90, rot) if rope else None
    wq, wk = ((_randn(g, D) * 0.3 + 1).to(dtype), (_randn(g, D) * 0.3 + 1).to(dtype)) if norm else (None, None)
    dq, dk, dwq, dwk = vt.qk_norm_rope_backward(gq, gk, q, k, positions, table, wq, wk, eps=1e-5, interleaved=interleaved)
    for x, gy, w, dx, dw in ((q, gq, wq, dq, dwq), (k, gk, wk, dk, dwk)):
        x64 = x.double().requires_grad_()
        w64 = w.double().requires_grad_() if norm else None
        norm_rope64(x64, positions, table, w64, 1e-5, interleaved).backward(gy.double())
        r = 1 / (x.double().square().mean(-1, keepdim=True) + 1e-5).sqrt() if norm else 1.0
        size = (gy.double().abs().amax(-1, keepdim=True) * (w.double().abs().max() if norm else 1) * r) if x.numel() else 0.0
        # fp32: two sums of D terms and a dozen operations, on terms of up to `size` times the row's largest unit value squared
        unit = (x.double().abs().amax(-1, keepdim=True) * r) if norm and x.numel() else 1.0
        close(dx, x64.grad, HALF[dtype], (D / 16 + 24) * 2.0 ** -24 * size * (1 + unit * unit) if x.numel() else 0.0)
        if norm:
            if x.numel() == 0:
                assert dw.eq(0).all()
                continue
            terms = (gy.double().abs().amax() * x.double().abs().mul(r).amax()).item()
            heads = x.shape[0] * x.shape[1]
            close(dw, w64.grad, 0.0, (math.sqrt(heads) * 4 + 64) * 2.0 ** -24 * terms * 4)
        else:
            assert dw is None


def test_gradients_agree_with_differences_and_through_autograd():
    g = _gen(5)
    n, hq, hk, D, rot = 5, 3, 1, 32, 16
    table, positions = _table64(40, rot), torch.randint(0, 40, (n,), generator=g, device="cuda")
    q, k = _randn(g, n, hq, D).requires_grad_(), _randn(g, n, hk, D).requires_grad_()
    wq, wk = (_randn(g, D) * 0.2 + 1).requires_grad_(), (_randn(g, D) * 0.2 + 1).requires_grad_()
    gq, gk = _randn(g, n, hq, D), _randn(g, n, hk, D)

    def loss(*a):
        y, z = vt.qk_norm_rope(a[0], a[1], positions, table, a[2], a[3])
        return (y.double() * gq).sum() + (z.double() * gk).sum()
    loss(q, k, wq, wk).backward()
    with torch.no_grad():
        for i, x in enumerate((q, k, wq, wk)):
            direction = _randn(g, *x.shape)
            step = 2.0 ** -7      # error of the difference: a step squared, and fp32 rounding over it
            moved = [[t + s * step * direction if j == i else t for j, t in enumerate((q, k, wq, wk))] for s in (1, -1)]
            slope = (loss(*moved[0]) - loss(*moved[1])).item() / (2 * step)
            want = (x.grad.double() * direction).sum().item()
            scale = x.grad.double().norm().item() * direction.double().norm().item()
            assert abs(slope - want) <= 0.01 * scale, i
    # a broadcast gradient (stride 0), parameters in bf16
    q16, w16 = q.detach().to(BF16).requires_grad_(), wq.detach().to(BF16).requires_grad_()
    k16 = k.detach().to(BF16)
    y, z = vt.qk_norm_rope(q16, k16, positions, table, w16, wk.detach().to(BF16))
    y.sum().backward()
    want = vt.qk_norm_rope_backward(torch.ones_like(y), torch.zeros_like(z), q16.detach(), k16, positions, table, w16.detach(), wk.detach().to(BF16))
    assert torch.equal(q16.grad, want[0]) and torch.equal(w16.grad, want[2].to(BF16)) and w16.grad.dtype == BF16
    with pytest.raises(ValueError):
        vt.qk_norm_rope(q16, k16, positions, table, w16, w16, q_out=torch.empty_like(q16))


def test_gradients_are_the_same_every_time_and_in_place():
    g = _gen(6)
    q, k, gq, gk = _randn(g, 3000, 8, 128).to(BF16), _randn(g, 3000, 2, 128).to(BF16), _randn(g, 3000, 8, 128).to(BF16), _randn(g, 3000, 2, 128).to(BF16)
    w = torch.ones(128, device="cuda", dtype=BF16)
    positions, table = torch.arange(3000, device="cuda"), _table64(3000, 128)
    first = vt.qk_norm_rope_backward(gq, gk, q, k, positions, table, w, w)
    for _ in range(3):
        for x, y in zip(first, vt.qk_norm_rope_backward(gq, gk, q, k, positions, table, w, w)):
            assert torch.equal(x, y)
    vt.qk_norm_rope_backward(gq, gk, q, k, positions, table, w, w, dq=gq, dk=gk)
    assert torch.equal(gq, first[0]) and torch.equal(gk, first[1])


# ---------------------------------------------------------------------------------------------- the cache
@pytest.mark.parametrize("n,hq,hk,D,page", [(1, 4, 2, 64, 16), (9, 3, 1, 80, 32), (33, 8, 8, 128, 64), (5, 2, 2, 256, 16), (70, 6, 3, 16, 128)])
@pytest.mark.parametrize("dtype", [BF16, F32])
@pytest.mark.parametrize("held", [BF16, E4M3])
@pytest.mark.parametrize("norm", [False, True])
def test_cache_write_and_read(n, hq, hk, D, page, dtype, held, norm):
    g = _gen(n + D)
    pages = n // page + 3
    cache = vt.KVCache(pages, page, hk, D, dtype=held)
    k0, v0 = cache.k.view(torch.uint8).random_(generator=g).clone(), cache.v.view(torch.uint8).random_(generator=g).clone()
    rows = (_randn(g, n, (hq + 2 * hk) * D) * 3).to(dtype)
    q, k, v = rows[:, :hq * D].unflatten(1, (hq, D)), rows[:, hq * D:(hq + hk) * D].unflatten(1, (hk, D)), rows[:, (hq + hk) * D:].unflatten(1, (hk, D))
    slots = torch.randperm(pages * page, generator=g, device="cuda")[:n]
    if n > 4:
        slots[1], slots[3] = -1, pages * page
    kept = (slots >= 0) & (slots < pages * page)
    if norm:
        w = (_randn(g, D) * 0.2 + 1).to(dtype)
        positions, table = torch.randint(0, 70, (n,), generator=g, device="cuda"), _table64(70, 16)
        q2 = vt.qkv_to_cache(q, k, v, cache, slots.int(), positions, table, w, w)
        plain = vt.qk_norm_rope(q, k, positions, table, w, w)
        assert torch.equal(q2, plain[0])
        k64 = norm_rope64(k, positions, table, w, 1e-6, False)
    else:
        vt.kv_cache_write(cache, k, v, slots)
        k64 = k.double()
    got = vt.kv_cache_read(cache, slots, dtype=F32)
    for x, y, exact in ((k64, got[0], not norm), (v.double(), got[1], True)):
        assert y[~kept].eq(0).all()
        want = held64(x, held)
        if exact:
            assert torch.equal(y[kept].double(), want[kept])
        else:      # fp32's rounding may fall on the other side of a border of the held type's: one step of it, for few
            off = (y.double() - want)[kept].abs()
            step = 2.0 ** -7 if held == BF16 else 2.0 ** -3
            assert (off <= step * want[kept].abs() + 2.0 ** -9 * x[kept].abs().amax(-1, keepdim=True) / 224).all()
            assert (off > 0).float().mean().item() < (0.02 if held == BF16 else 0.002) + 2 / off.numel()
    for x, y in zip(got, vt.kv_cache_read(cache, slots)):
        assert torch.equal(x, y.float())
    # nothing else is touched
    other = torch.ones(pages * page, dtype=torch.bool, device="cuda")
    other[slots[kept]] = False
    other = other.view(pages, page)
    for now, then in ((cache.k, k0), (cache.v, v0)):
        assert torch.equal(now.view(torch.uint8).transpose(1, 2)[other], then.transpose(1, 2)[other])


def test_every_code_of_eight_bits_reads_back_as_it_is_and_is_written_back():
    codes = torch.arange(256, device="cuda", dtype=torch.uint8).view(1, 1, 16, 16).contiguous()
    scale = torch.tensor([127, 1, 120, 130, 200, 247, 100, 127, 127, 127, 90, 127, 60, 127, 127, 127], device="cuda", dtype=torch.uint8).view(1, 1, 16)
    cache = vt.KVCache.of(codes.view(E4M3), codes.clone().view(E4M3), scale, scale.clone())
    k, v = vt.kv_cache_read(cache, torch.arange(16, device="cuda"), dtype=F32)
    want = codes.view(E4M3).double()[0, 0] * power_of_two(scale[0, 0].int() - 127)[:, None]
    normal = want.isnan() | (want == 0) | (want.abs() >= 2.0 ** -126)
    assert torch.equal(k[:, 0].isnan(), want.isnan())
    assert torch.equal(torch.where(normal, k[:, 0].double(), 0.0).nan_to_num(3.0), torch.where(normal, want, 0.0).nan_to_num(3.0))
    assert torch.equal(k.nan_to_num(3.0), v.nan_to_num(3.0))


def test_eight_bits_of_borders_zeros_infinities_and_nan():
    D = 16
    x = torch.zeros(10, 1, D, device="cuda")
    x[0, 0, :3] = torch.tensor([448.0, -448.0, 1.0])
    x[1, 0, :3] = torch.tensor([448.0 * (1 + 2 ** -23), 1.0, 17.0])            # the next scale
    x[2, 0, :4] = torch.tensor([math.inf, -math.inf, math.nan, 100.0])
    # (100 is halfway between 96 and 104)
    x[3, 0, :2] = torch.tensor([math.inf, math.nan])
    x[4, 0, :3] = torch.tensor([448.0, 17.0, 19.0])                            # ties between 16 and 18, 18 and 20
    x[5, 0, :3] = torch.tensor([3.4028234e38, 1.0, -3.4028234e38])
    x[6, 0, :2] = torch.tensor([2.0 ** -126, -2.0 ** -127])
    x[7, 0, :3] = torch.tensor([448.0, 2.0 ** -9, 2.0 ** -10])                 # the smallest code, and half of it
    x[8, 0, 0] = -0.0
    x[9] = math.inf
    cache = vt.KVCache(1, 16, 1, D, dtype=E4M3)
    slots = torch.arange(10, device="cuda")
    vt.kv_cache_write(cache, x, x, slots)
    k, v = vt.kv_cache_read(cache, slots, dtype=F32)
    assert torch.equal(k.nan_to_num(-5.0), v.nan_to_num(-5.0))
    assert cache.k_scale[0, 0, 0] == 127 and cache.k_scale[0, 0, 1] == 128
    assert k[0, 0, :3].tolist() == [448.0, -448.0, 1.0] and k[4, 0, 1:3].tolist() == [16.0, 20.0] and k[7, 0, 1:3].tolist() == [2.0 ** -9, 0.0]
    assert k[2, 0, 2].isnan() and k[2, 0, 3] == 96.0 and k[2, 0, 0] > 100 and k[2, 0, 0] == -k[2, 0, 1] == 448 * 2.0 ** (cache.k_scale[0, 0, 2].item() - 127)
    assert k[3, 0, 1].isnan() and k[3, 0, 2:].eq(0).all()
    finite = [0, 1, 4, 5, 7, 8]
    assert torch.equal(k[finite].double(), held64(x[finite].double(), E4M3))
    assert not k[9].isnan().any() and k[9].gt(0).all()


# ---------------------------------------------------------------------------------------------- attention
def _filled(g, held, pages, hk, page, D):
    cache = vt.KVCache(pages, page, hk, D, dtype=held)
    if held == BF16:
        cache.k.copy_(_randn(g, *cache.k.shape))
        cache.v.copy_(_randn(g, *cache.v.shape))
    else:
        for t, s in ((cache.k, cache.k_scale), (cache.v, cache.v_scale)):
            t.copy_((_randn(g, *t.shape) * 100).clamp(-448, 448).to(E4M3))
            s.copy_(torch.randint(118, 124, s.shape, generator=g, device="cuda"))
    return cache


def _case(g, held, dtype, hq, hk, D, page, lengths, rows=None, spare=2, gain=1.5):
    """cache, page_table, lengths, q, row_start, and each request's k and v in float64."""
    used = [-(-t // page) for t in lengths]
    cache = _filled(g, held, sum(used) + spare, hk, page, D)
    ids = torch.randperm(sum(used) + spare, generator=g, device="cuda").int()
    table = torch.full((len(lengths), max(max(used), 1)), -7, dtype=torch.int32, device="cuda")
    at = 0
    for b, u in enumerate(used):
        table[b, :u] = ids[at:at + u]
        at += u
    counts = rows or [1] * len(lengths)
    starts = torch.tensor([0] + counts, device="cuda").cumsum(0).int()
    q = (_randn(g, sum(counts), hq, D) * gain).to(dtype)
    return cache, table, torch.tensor(lengths, dtype=torch.int32, device="cuda"), q, starts if rows else None


def _values(cache, table, b, length):
    slots = cache.slots(table, torch.full((length,), b, device="cuda"), torch.arange(length, device="cuda"))
    k, v = vt.kv_cache_read(cache, slots, dtype=F32)
    return k.double(), v.double()


def _check_attention(cache, table, lengths, q, starts, mask=None, scale=None, seen_pages=None, **kw):
    n, hq, D = q.shape
    scale = D ** -0.5 if scale is None else scale
    max_rows = 1 if starts is None else int(starts.diff().max())
    out, lse = vt.paged_attention(q, cache, table, lengths, row_start=starts, max_rows=max_rows, tail_mask=mask, scale=scale, return_lse=True, **kw)
    assert out.dtype == q.dtype and lse.dtype == F32
    first = list(range(n + 1)) if starts is None else starts.tolist()
    for b, length in enumerate(lengths.tolist()):
        rows = slice(first[b], first[b + 1])
        if first[b] == first[b + 1]:
            continue
        k, v = _values(cache, table, b, length)
        see = torch.ones(first[b + 1] - first[b], length, dtype=torch.bool, device="cuda")
        if mask is not None:
            for i in range(see.shape[0]):
                bits = int(mask[rows][i]) & ((1 << 64) - 1)
                for t in range(max(0, length - 64), length):
                    see[i, t] = bool(bits >> (t - length + 64) & 1)
        if seen_pages is not None:
            see &= seen_pages[b][:length]
        want, want_lse = attend64(q[rows], k, v, see, scale)
        # A score is a sum of D products in fp32, off by up to sqrt(D) / 2 + 8 half steps of the sum of their sizes; p is off by that
        # much, absolute in the exponent, and by exp2's and the sums' few; bf16 rows: p is rounded to bf16.  out is a mean of values with
        # weights p, so off by p's relative error times the mean size of its values, then rounded once.
        g = hq // cache.heads
        sizes = (q[rows].double().abs()[:, None] * k.abs().repeat_interleave(g, 1)[None]).sum(-1) * abs(scale) if length else torch.zeros(1, device="cuda")
        fine = (sizes[sizes.isfinite()].max().item() if sizes.numel() and sizes.isfinite().any() else 0.0) * (math.sqrt(D) / 2 + 8) * 2.0 ** -24 + 40 * 2.0 ** -24
        weight = fine + (2.0 ** -8 if q.dtype == BF16 else 0.0)
        spread = attend64(q[rows], k, v.abs(), see, scale)[0]
        spread = torch.where(spread.isfinite(), spread, 0.0)
        close(out[rows], want, HALF[q.dtype], weight * 2 * spread)
        close(lse[rows], want_lse, 2.0 ** -23, fine * 2)
    return out, lse


LAYOUTS = [(1, 1, 64), (4, 2, 64), (8, 8, 128), (32, 8, 128), (7, 1, 128), (40, 2, 128), (6, 3, 256), (5, 1, 80), (9, 3, 16), (20, 1, 256), (72, 1, 64), (12, 2, 96)]


@pytest.mark.parametrize("hq,hk,D", LAYOUTS)
@pytest.mark.parametrize("held", [BF16, E4M3])
@pytest.mark.parametrize("dtype", [BF16, F32])
def test_attention_of_single_tokens(hq, hk, D, held, dtype):
    g = _gen(hq * D)
    for page, lengths in ((16, [1, 0, 17, 31, 32, 33, 63, 64, 65, 127, 128, 129, 300]), (64, [777, 1, 1500, 64]), (32, [4099])):
        case = _case(g, held, dtype, hq, hk, D, page, lengths)
        _check_attention(*case)


@pytest.mark.parametrize("hq,hk,D,rows", [(4, 2, 64, [3, 1, 0, 5]), (32, 8, 128, [8, 8, 1, 4]), (8, 8, 128, [16, 2, 7, 33]), (14, 2, 128, [5, 0, 3, 9]),
                                          (4, 1, 256, [8, 1, 2, 9]), (12, 3, 80, [6, 6, 6, 6]), (64, 1, 64, [2, 3, 1, 2])])
@pytest.mark.parametrize("held", [BF16, E4M3])
@pytest.mark.parametrize("dtype", [BF16, F32])
@pytest.mark.parametrize("masked", [False, True])
def test_attention_of_tree_levels(hq, hk, D, rows, held, dtype, masked):
    g = _gen(hq + D + masked)
    for lengths in ([40, 1, 64, 63], [200, 129, 65, 500], [700, 3, 1300, 90]):
        case = _case(g, held, dtype, hq, hk, D, 32, lengths, rows=rows)
        mask = None
        if masked:
            mask = torch.randint(-(1 << 63), (1 << 63) - 1, (sum(rows),), generator=g, device="cuda")
            mask[0] = 0              # a row that sees none of the last 64: nothing at all of 40 tokens
            mask[1] = -1
            mask[-1] = -(1 << 63)    # the newest token only
        _check_attention(*case, mask=mask)


@pytest.mark.parametrize("held", [BF16, E4M3])
@pytest.mark.parametrize("rows", [None, 3])
def test_attention_of_more_requests_than_shares(held, rows):
    """Requests begin and end anywhere in the shares; some have no rows, some no tokens."""
    g = _gen(30)
    n = 90
    lengths = [[1490, 0, 130, 128, 1, 700, 90, 260, 64][i * 7 % 9] for i in range(n)]
    counts = None if rows is None else [i * 5 % (rows + 1) for i in range(n)]
    case = _case(g, held, BF16, 8, 8, 64, 16, lengths, rows=counts)
    _check_attention(*case, max_length=1504)


def test_attention_of_hundreds_of_requests():
    """Shares that begin in any block of 64 requests, whole blocks without rows."""
    g = _gen(31)
    n = 333
    lengths = [(i * 37) % 400 if i % 11 else 0 for i in range(n)]
    lengths[200] = 2000
    counts = [0 if 64 <= i < 192 or i % 7 == 3 else 1 for i in range(n)]
    case = _case(g, BF16, BF16, 2, 1, 64, 16, lengths, rows=counts)
    _check_attention(*case, max_length=2048)


def test_attention_single_rows_with_a_mask():
    g = _gen(3)
    case = _case(g, BF16, BF16, 8, 2, 64, 16, [70, 5, 0, 64, 2000])
    _check_attention(*case, mask=torch.tensor([0, 0, 0, 1, 5], device="cuda"))


@pytest.mark.parametrize("held", [BF16, E4M3])
@pytest.mark.parametrize("D", [64, 128, 256, 48])
def test_attention_does_not_see_what_lies_past_the_end(held, D):
    """Places past a request's tokens, other pages and a page table's other entries hold NaN and infinities."""
    g = _gen(D)
    hk, page = 2, 32
    cache, table, lengths, q, starts = _case(g, held, BF16, 4, hk, D, page, [45, 1, 0, 128, 31, 600], rows=[2, 1, 1, 3, 1, 2])
    used = torch.zeros(cache.pages, page, dtype=torch.bool, device="cuda")
    for b, t in enumerate(lengths.tolist()):
        for i in range(-(-t // page)):
            used[table[b, i].long(), :min(page, t - i * page)] = True
    for x in (cache.k, cache.v):
        y = x.view(torch.uint8).view(cache.pages, hk, page, -1) if held == E4M3 else x
        bad = 0x7F if held == E4M3 else math.nan
        y.transpose(1, 2)[~used] = bad
    for s in (cache.k_scale, cache.v_scale):
        if s is not None:
            s.transpose(1, 2)[~used] = 255
    _check_attention(cache, table, lengths, q, starts)
    # one more page of the table, beyond what any request needs, and lengths that the caller bounds
    table2 = torch.cat([table, torch.full_like(table[:, :1], 1 << 30)], 1)
    a = vt.paged_attention(q, cache, table2, lengths, row_start=starts, max_rows=3, max_length=10000)
    b = vt.paged_attention(q, cache, table, lengths, row_start=starts, max_rows=3, max_length=10000)
    assert torch.equal(a, b)


@pytest.mark.parametrize("held", [BF16, E4M3])
@pytest.mark.parametrize("dtype", [BF16, F32])
@pytest.mark.parametrize("rows", [2, 9])
def test_masked_nan_and_infinities_reach_only_the_rows_that_see_them(held, dtype, rows):
    g = _gen(rows)
    hq, hk, D, page, length = 4, 2, 128, 16, 100
    cache, table, lengths, q, starts = _case(g, held, dtype, hq, hk, D, page, [length], rows=[rows])

    def put(x, token, head, d, value):
        x[table[0, token // page].long(), head, token % page, d] = value
    odd = [(80, math.nan)] if held == E4M3 else [(80, math.nan), (90, math.inf), (91, -math.inf), (92, math.inf), (95, math.inf)]
    for token, value in odd:
        put(cache.v.view(torch.uint8) if held == E4M3 else cache.v, token, 1, 7 + token % 3, 0x7F if held == E4M3 else value)
    put(cache.k.view(torch.uint8) if held == E4M3 else cache.k, 85, 0, 3, 0x7F if held == E4M3 else math.nan)
    every = (1 << 64) - 1
    hidden = every
    for token in (80, 85, 90, 91, 92, 95):
        hidden &= ~(1 << (token - length + 64))
    masks = [hidden] * rows
    masks[0] = hidden | 1 << (80 - length + 64)      # sees the NaN among the values
    if rows > 3:
        masks[2] = hidden | 1 << (90 - length + 64)       # infinity
        masks[3] = hidden | 1 << (91 - length + 64) | 1 << (90 - length + 64)
        masks[4] = hidden | 1 << (85 - length + 64)       # NaN among the keys
        masks[5] = hidden | 1 << (95 - length + 64) | 1 << (92 - length + 64)
    mask = torch.tensor([m - (1 << 64) if m >> 63 else m for m in masks], device="cuda")
    out, lse = _check_attention(cache, table, lengths, q, starts, mask=mask)
    assert out[1].isfinite().all() and lse[1].isfinite().all() and out[0].isnan().any()
    if rows > 3:
        assert out[-1].isfinite().all() and lse[4].isnan().any()


def test_pages_outside_the_cache_are_not_seen():
    g = _gen(8)
    cache, table, lengths, q, starts = _case(g, BF16, BF16, 4, 2, 64, 16, [100, 40, 20])
    seen = torch.ones(3, 112, dtype=torch.bool, device="cuda")
    for b, i, bad in ((0, 2, -1), (0, 5, cache.pages), (1, 0, 1 << 30), (2, 0, -(1 << 31)), (2, 1, cache.pages + 5)):
        table[b, i] = bad
        seen[b, 16 * i:16 * i + 16] = False
    readable = table.clone()
    readable[(table < 0) | (table >= cache.pages)] = 0
    out, lse = vt.paged_attention(q, cache, table, lengths, return_lse=True)
    for b, length in enumerate(lengths.tolist()):
        k, v = _values(cache, readable, b, length)
        want, want_lse = attend64(q[b:b + 1], k, v, seen[b:b + 1, :length], 0.125)
        spread = attend64(q[b:b + 1], k, v.abs(), seen[b:b + 1, :length], 0.125)[0]
        close(out[b:b + 1], want, 2.0 ** -8, spread * 2.0 ** -6)
        close(lse[b:b + 1], want_lse, 2.0 ** -23, 1e-5)
    assert out[2].eq(0).all() and lse[2].eq(-math.inf).all()


def test_lengths_and_rows_that_say_more_than_there_is():
    g = _gen(9)
    cache, table, lengths, q, _ = _case(g, BF16, BF16, 4, 2, 64, 16, [48, 48, 48, 48])
    want = vt.paged_attention(q, cache, table, lengths)
    wrong = torch.tensor([48, 1 << 30, (1 << 31) - 1, -5], dtype=torch.int32, device="cuda")
    got = vt.paged_attention(q, cache, table, wrong)
    assert torch.equal(got[:3], want[:3]) and got[3].eq(0).all()
    short = vt.paged_attention(q, cache, table, wrong, max_length=20)
    assert torch.equal(short[:3], vt.paged_attention(q, cache, table, torch.full_like(wrong, 20))[:3])
    out = torch.full_like(q, 7.0)
    starts = torch.tensor([0, 2, 1, 3, 90], dtype=torch.int32, device="cuda")      # out of order, past the rows; one row too many of max_rows
    vt.paged_attention(q, cache, table, lengths, row_start=starts, max_rows=1, out=out)
    assert out[0].ne(7.0).any() and out[1].ne(7.0).any() and out[3].ne(7.0).any() and out[2].eq(7.0).all()


def test_attention_scores_at_the_edges():
    """One token far above the others, scores of -inf, all equal, a scale of zero and a negative one."""
    g = _gen(10)
    cache, table, lengths, q, _ = _case(g, BF16, BF16, 4, 1, 64, 16, [500, 500])
    cache.k[table[0, 3].long(), 0, 5] = (q[0, 0] * 40).to(BF16)
    _check_attention(cache, table, lengths, q, None)
    for scale in (0.0, -0.3, 30.0):
        _check_attention(cache, table, lengths, q, None, scale=scale)
    cache.k.zero_()
    _check_attention(cache, table, lengths, q, None)
    # scores of -inf for some tokens, then for all: as if not seen
    q = q.abs()
    cache.k[table[0, 0].long()] = -math.inf
    out, lse = vt.paged_attention(q, cache, table, lengths, return_lse=True)
    k, v = _values(cache, table, 0, 500)
    see = torch.ones(1, 500, dtype=torch.bool, device="cuda")
    see[0, :16] = False
    want, want_lse = attend64(q[:1], k, v, see, 0.125)
    close(out[:1], want, 2.0 ** -8, 2.0 ** -7)
    close(lse[:1], want_lse, 0.0, 1e-5)
    cache.k.fill_(-math.inf)
    out, lse = vt.paged_attention(q, cache, table, lengths, return_lse=True)
    assert out.eq(0).all() and lse.eq(-math.inf).all()
    q[0, 2, 3] = math.nan
    out, lse = vt.paged_attention(q, cache, table, lengths, return_lse=True)
    assert out[0, 2].isnan().all() and lse[0, 2].isnan() and out[0, 1].eq(0).all() and out[1].eq(0).all()


@pytest.mark.parametrize("held,dtype", [(BF16, BF16), (E4M3, BF16), (BF16, F32)])
def test_attention_of_a_long_request_split_and_joined(held, dtype):
    g = _gen(11)
    case = _case(g, held, dtype, 8, 2, 128, 64, [30011, 0, 129], gain=2.0)
    out, lse = _check_attention(*case)
    # the split follows max_length: other pieces, the same to rounding
    for most in (30011, 32768, 1 << 30):
        o, l = vt.paged_attention(case[3], *case[:3], max_length=most, return_lse=True)
        close(o, out.double(), 2.0 ** -6 if dtype == BF16 else 2.0 ** -18, 2.0 ** -8 if dtype == BF16 else 2.0 ** -18)
        close(l, lse.double(), 2.0 ** -20)


def test_attention_rows_apart_in_place_and_on_another_stream():
    g = _gen(12)
    cache, table, lengths, q, starts = _case(g, BF16, BF16, 8, 2, 64, 16, [300, 4000], rows=[3, 2])
    want = vt.paged_attention(q, cache, table, lengths, row_start=starts, max_rows=3)
    wide = torch.zeros(5, 10 * 64, device="cuda", dtype=BF16)
    wide[:, 64:9 * 64] = q.flatten(1)
    apart = wide[:, 64:9 * 64].unflatten(1, (8, 64))
    stream = torch.cuda.Stream()
    stream.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(stream):
        got = vt.paged_attention(apart, cache, table, lengths, row_start=starts, max_rows=3, out=apart)
    torch.cuda.current_stream().wait_stream(stream)
    assert torch.equal(got, want) and wide[:, :64].eq(0).all() and wide[:, 9 * 64:].eq(0).all()


def test_a_cache_beyond_32_bits():
    """Pages whose rows lie past 2^32 bytes and past 2^31 values."""
    hk, D, page = 8, 128, 64
    pages = (5 << 30) // (hk * D * page * 2)
    cache = vt.KVCache(pages, page, hk, D)
    assert cache.k.numel() > 1 << 31
    g = _gen(13)
    ids = torch.tensor([pages - 1, pages - 2, 3], dtype=torch.int32, device="cuda")
    k, v = _randn(g, 150, hk, D).to(BF16), _randn(g, 150, hk, D).to(BF16)
    table = ids[None].contiguous()
    slots = cache.slots(table, torch.zeros(150, dtype=torch.int64, device="cuda"), torch.arange(150, device="cuda"))
    vt.kv_cache_write(cache, k, v, slots)
    for x, y in zip((k, v), vt.kv_cache_read(cache, slots)):
        assert torch.equal(x, y)
    assert torch.equal(cache.k[pages - 1, 2, 5], k[5, 2])
    q = _randn(g, 1, 8, D).to(BF16)
    _check_attention(cache, table, torch.tensor([150], dtype=torch.int32, device="cuda"), q, None)


def test_captured_in_a_graph():
    """The layer's calls in one graph, replayed among eager work on new inputs in the same tensors."""
    g = _gen(14)
    n, hq, hk, D, page = 6, 8, 2, 64, 16
    cache, table, lengths, _, starts = _case(g, E4M3, BF16, hq, hk, D, page, [500, 41], rows=[4, 2])
    rows = _randn(g, n, (hq + 2 * hk) * D).to(BF16)
    q, k, v = rows[:, :hq * D].unflatten(1, (hq, D)), rows[:, hq * D:(hq + hk) * D].unflatten(1, (hk, D)), rows[:, (hq + hk) * D:].unflatten(1, (hk, D))
    w, rope = torch.ones(D, device="cuda", dtype=BF16), _table64(600, D)
    tokens = torch.tensor([496, 497, 498, 499, 39, 40], device="cuda")
    slots = cache.slots(table, torch.tensor([0, 0, 0, 0, 1, 1], device="cuda"), tokens)
    ws = vt.AttentionWorkspace(n, hq, hk, D, 2, 4, 500, "cuda")
    out, q2 = torch.empty(n, hq, D, device="cuda", dtype=BF16), torch.empty(n, hq, D, device="cuda", dtype=BF16)
    kk, vv = torch.empty(n, hk, D, device="cuda", dtype=BF16), torch.empty(n, hk, D, device="cuda", dtype=BF16)

    def layer():
        vt.qkv_to_cache(q, k, v, cache, slots, tokens, rope, w, w, q_out=q2)
        vt.paged_attention(q2, cache, table, lengths, row_start=starts, max_rows=4, max_length=500, ws=ws, out=out)
        vt.kv_cache_read(cache, slots, k_out=kk, v_out=vv)
    layer()
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        layer()
    for _ in range(4):
        rows.copy_(_randn(g, *rows.shape))
        graph.replay()
        torch.cuda.synchronize()
        got = [x.clone() for x in (q2, out, kk, vv)]
        layer()
        for x, y in zip(got, (q2, out, kk, vv)):
            assert torch.equal(x, y)


def test_gradients_captured_in_a_graph():
    g = _gen(15)
    q, k, gq, gk = (_randn(g, 1500, h, 64).to(BF16) for h in (4, 2, 4, 2))
    w, rope, positions = torch.ones(64, device="cuda", dtype=BF16), _table64(1500, 64), torch.arange(1500, device="cuda")
    ws = torch.empty(vt.load_library().vt_qk_norm_rope_backward_ws_bytes(1500, 64), dtype=torch.uint8, device="cuda")
    call = lambda: vt.qk_norm_rope_backward(gq, gk, q, k, positions, rope, w, w, ws=ws)      # noqa: E731
    call()
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        got = call()
    for _ in range(3):
        gq.copy_(_randn(g, *gq.shape))
        graph.replay()
        torch.cuda.synchronize()
        for x, y in zip(got, call()):
            assert torch.equal(x, y)


def test_nothing_to_do():
    x = torch.empty(0, 4, 64, device="cuda", dtype=BF16)
    none = torch.empty(0, dtype=torch.int64, device="cuda")
    cache = vt.KVCache(1, 16, 4, 64)
    a, b = vt.qk_norm_rope(x, x, none, _table64(4, 64))
    assert a.shape == b.shape == (0, 4, 64)
    w = torch.ones(64, device="cuda", dtype=BF16)
    dq, dk, dwq, dwk = vt.qk_norm_rope_backward(x, x, x, x, none, _table64(4, 64), w, w)
    assert dq.shape == (0, 4, 64) and dwq.eq(0).all() and dwk.eq(0).all()
    vt.kv_cache_write(cache, x, x, none)
    assert vt.kv_cache_read(cache, none)[0].shape == (0, 4, 64)
    assert vt.paged_attention(x, cache, torch.empty(0, 3, dtype=torch.int32, device="cuda"), torch.empty(0, dtype=torch.int32, device="cuda")).shape == (0, 4, 64)
    q = torch.ones(2, 4, 64, device="cuda", dtype=BF16)
    out, lse = vt.paged_attention(q, cache, torch.zeros(2, 3, dtype=torch.int32, device="cuda"), torch.zeros(2, dtype=torch.int32, device="cuda"), return_lse=True)
    assert out.eq(0).all() and lse.eq(-math.inf).all()


def test_refusals_on_the_device():
    g = _gen(16)
    q, k = _randn(g, 3, 4, 64).to(BF16), _randn(g, 3, 2, 64).to(BF16)
    cache = vt.KVCache(2, 16, 2, 64)
    w = torch.ones(64, device="cuda", dtype=BF16)
    slots = torch.arange(3, device="cuda")
    table, lengths = torch.zeros(3, 1, dtype=torch.int32, device="cuda"), torch.ones(3, dtype=torch.int32, device="cuda")
    for call in (lambda: vt.qk_norm_rope(q, k, q_weight=w), lambda: vt.qk_norm_rope(q, k.float()), lambda: vt.qk_norm_rope(q, k, positions=slots),
                 lambda: vt.qk_norm_rope(q.transpose(1, 2).contiguous().transpose(1, 2), k), lambda: vt.qk_norm_rope(q, k, None, None, w.float(), w.float()),
                 lambda: vt.qk_norm_rope(q, k, slots[:2], _table64(4, 64)), lambda: vt.qkv_to_cache(q, k[:, :1], k[:, :1], cache, slots),
                 lambda: vt.kv_cache_write(cache, k, k[:2], slots), lambda: vt.kv_cache_write(cache, k, k, slots[:2]),
                 lambda: vt.paged_attention(q, cache, table, lengths[:2]), lambda: vt.paged_attention(q, cache, table.long(), lengths),
                 lambda: vt.paged_attention(q, cache, table, lengths, row_start=torch.arange(4, dtype=torch.int32, device="cuda")),
                 lambda: vt.paged_attention(q[..., :32], cache, table, lengths), lambda: vt.KVCache.of(cache.k, cache.v, slots, slots)):
        with pytest.raises(ValueError):
            call()
    for call in (lambda: vt.kv_cache_write(cache, k, k, slots.float()), lambda: vt.qk_norm_rope(q.half(), k.half())):
        with pytest.raises(TypeError):
            call()
    for call, status in ((lambda: vt.qk_norm_rope(q, k, None, None, w, w, eps=0.0), 2), (lambda: vt.qk_norm_rope(q, k, slots, _table64(4, 64)[:, :12].contiguous()), 4),
                         (lambda: vt.qk_norm_rope(q[:1].expand(3, 4, 64), k), 2), (lambda: vt.paged_attention(q[:, :3].contiguous(), cache, table, lengths), 2),
                         (lambda: vt.paged_attention(q, vt.KVCache(1, 24, 2, 64), table, lengths), 2)):
        with pytest.raises(vt.VocabTrimError) as e:
            call()
        assert e.value.status == status


# ---------------------------------------------------------------------------------------------- the native way through the binding
def _layer_calls():
    """name -> (call, arguments) of the attention's calls, plain ones."""
    g = _gen(20)
    n, hq, hk, D, page = 5, 4, 2, 64, 16
    q, k, v = (_randn(g, n, h, D).to(BF16) for h in (hq, hk, hk))
    w = torch.ones(D, device="cuda", dtype=BF16)
    rope, positions = _table64(40, 32), torch.arange(n, device="cuda")
    cache, table, lengths, rows, starts = _case(g, E4M3, BF16, hq, hk, D, page, [400, 30], rows=[3, 2])
    ws = vt.AttentionWorkspace(n, hq, hk, D, 2, 3, 512, "cuda")
    norm = dict(positions=positions, table=rope, q_weight=w, k_weight=w, eps=1e-5, interleaved=True)
    mask = torch.randint(-(1 << 62), 1 << 62, (n,), generator=g, device="cuda")
    return {
        "norm": (vt.qk_norm_rope, dict(q=q, k=k, **norm, q_out=torch.empty_like(q))),
        "norm alone": (vt.qk_norm_rope, dict(q=q, k=k, q_weight=w, k_weight=w)),
        "backward": (vt.qk_norm_rope_backward, dict(gq=q + 1, gk=k + 1, q=q, k=k, **norm)),
        "to cache": (vt.qkv_to_cache, dict(q=q, k=k, v=v, cache=cache, slots=torch.arange(n, device="cuda", dtype=torch.int32), **norm)),
        "read": (vt.kv_cache_read, dict(cache=cache, slots=torch.arange(9, device="cuda"))),
        "attend": (vt.paged_attention, dict(q=rows, cache=cache, page_table=table, lengths=lengths, row_start=starts, max_rows=3, tail_mask=mask,
                                            max_length=512, scale=0.2, ws=ws, return_lse=True)),
        "attend rows": (vt.paged_attention, dict(q=rows[:2], cache=cache, page_table=table, lengths=lengths, ws=ws, out_lse=torch.empty(2, hq, device="cuda"))),
    }


def _outcome(call, args):
    try:
        got = call(**args)
    except (RuntimeError, ValueError, TypeError, AttributeError, IndexError, OverflowError, ctypes.ArgumentError) as e:
        return type(e).__name__ if not isinstance(e, vt.VocabTrimError) else e.status
    torch.cuda.synchronize()
    return [x.clone() for x in (got if isinstance(got, tuple) else (got,)) if x is not None]      # (no q, no result; no weights, no gradients of them)


def test_the_native_way_and_pythons_give_the_same(monkeypatch):
    vt.load_library()
    native = binding._bind
    assert native is not None
    for name, (call, args) in _layer_calls().items():
        cases = [("plain", args)]
        for key, t in args.items():
            if isinstance(t, torch.Tensor):
                cases += [(key + " on the host", {**args, key: t.cpu()}), (key + " of another type", {**args, key: t.to(torch.float64)}),
                          (key + " no tensor", {**args, key: 3}), (key + " left out", {**args, key: None}), (key + " shorter", {**args, key: t[:-1].contiguous()})]
                if t.dim() == 3:
                    apart = torch.empty(t.shape[0], t.shape[1] + 2, t.shape[2], dtype=t.dtype, device="cuda")[:, 1:-1]
                    apart.copy_(t)
                    cases += [(key + " with rows apart", {**args, key: apart}), (key + " strided", {**args, key: t.repeat_interleave(2, -1)[..., ::2]}),
                              (key + " without rows", {**args, key: t[:0]}), (key + " transposed", {**args, key: t.transpose(0, 1)})]
            elif isinstance(t, (int, float)) and not isinstance(t, bool):
                cases += [(f"{key} = {v}", {**args, key: v}) for v in (0, -1, 1 << 40, 2.5, math.nan, "1")]
        for what, changed in cases:
            both = []
            for way in (native, None):
                monkeypatch.setattr(binding, "_bind", way)
                both.append(_outcome(call, changed))
            assert type(both[0]) is type(both[1]), (name, what, both)
            if isinstance(both[0], list):
                for x, y in zip(*both):
                    assert x.dtype == y.dtype and x.shape == y.shape and torch.equal(x.nan_to_num(9.0), y.nan_to_num(9.0)), (name, what)
            else:
                assert both[0] == both[1], (name, what, both)
            assert what != "plain" or isinstance(both[0], list), (name, both)


def test_plain_calls_take_the_native_way(monkeypatch):
    asked = []

    class Spy:
        def __getattr__(self, name):
            def call(*a):
                got = getattr(native, name)(*a)
                asked.append((name, got is not None))
                return got
            return call
    vt.load_library()
    native = binding._bind
    monkeypatch.setattr(binding, "_bind", Spy())
    for name, (call, args) in _layer_calls().items():
        call(**args)
        assert asked[-1][1], name
    q = torch.ones(2, 2, 64, device="cuda", requires_grad=True)
    y, _ = vt.qk_norm_rope(q, q.detach(), None, None, torch.nn.Parameter(torch.ones(64, device="cuda")), torch.ones(64, device="cuda"))
    assert asked[-1] == ("norm", False) and y.requires_grad
    torch.cuda.synchronize()
