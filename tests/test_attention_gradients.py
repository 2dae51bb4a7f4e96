"""What the attention's calls do where a gradient is asked for: qk_norm_rope has one, the cache and the attention over it refuse."""
import pytest
import torch
from torch.autograd import forward_ad

import paper_2506_22694_amd as vt

BF16 = torch.bfloat16


def _leaf(*shape, device="cpu"):
    return torch.ones(shape, device=device, dtype=BF16, requires_grad=True)


def test_calls_without_gradients_refuse_what_requires_one():
    x, leaf, w = torch.ones(2, 4, 64, dtype=BF16), _leaf(2, 4, 64), torch.ones(64, dtype=BF16)
    slots, table = torch.arange(2), torch.ones(8, 64)
    ints = torch.zeros(2, 1, dtype=torch.int32)
    for call in (lambda: vt.qkv_to_cache(leaf, x, x, None, slots), lambda: vt.qkv_to_cache(x, leaf, x, None, slots), lambda: vt.qkv_to_cache(x, x, leaf, None, slots),
                 lambda: vt.qkv_to_cache(x, x, x, None, slots, slots, table, _leaf(64), w), lambda: vt.qkv_to_cache(x, x, x, None, slots, slots, table, w, _leaf(64)),
                 lambda: vt.qkv_to_cache(x, x, x, None, slots, slots, table.clone().requires_grad_(), w, w), lambda: vt.kv_cache_write(None, x, leaf, slots),
                 lambda: vt.qkv_to_cache(x, x, x, None, slots, q_out=leaf), lambda: vt.qk_norm_rope(x, x, slots, table.clone().requires_grad_()),
                 lambda: vt.paged_attention(leaf, None, ints, ints[:, 0]), lambda: vt.paged_attention(x, None, ints, ints[:, 0], out=leaf),
                 lambda: vt.KVCache.of(_leaf(2, 2, 16, 64), _leaf(2, 2, 16, 64)), lambda: vt.kv_cache_read(None, slots, k_out=leaf)):
        with pytest.raises(ValueError, match="no gradient"):
            call()


@pytest.mark.gpu
def test_no_gradient_is_lost_on_the_device():
    x, leaf, w, param = (torch.ones(2, 2, 64, device="cuda", dtype=BF16), _leaf(2, 2, 64, device="cuda"), torch.ones(64, device="cuda", dtype=BF16),
                         torch.nn.Parameter(torch.ones(64, device="cuda", dtype=BF16)))
    cache = vt.KVCache(1, 16, 2, 64)
    slots, pages, lengths = torch.arange(2, device="cuda"), torch.zeros(2, 1, dtype=torch.int32, device="cuda"), torch.ones(2, dtype=torch.int32, device="cuda")
    ws = vt.AttentionWorkspace(2, 2, 2, 64, 2, 1, 16, "cuda")
    calls = [lambda: vt.qkv_to_cache(leaf, x, x, cache, slots), lambda: vt.qkv_to_cache(x, leaf, x, cache, slots), lambda: vt.qkv_to_cache(x, x, leaf, cache, slots),
             lambda: vt.qkv_to_cache(x, x, x, cache, slots, q_weight=param, k_weight=w), lambda: vt.qkv_to_cache(x, x, x, cache, slots, q_weight=w, k_weight=param),
             lambda: vt.qkv_to_cache(x, x, x, cache, slots, slots, torch.ones(8, 64, device="cuda", requires_grad=True)), lambda: vt.kv_cache_write(cache, leaf, x, slots),
             lambda: vt.paged_attention(leaf, cache, pages, lengths), lambda: vt.paged_attention(leaf, cache, pages, lengths, ws=ws),
             lambda: vt.paged_attention(x, cache, pages, lengths, ws=ws, out=_leaf(2, 2, 64, device="cuda")),
             lambda: vt.qk_norm_rope(x, x, slots, torch.ones(8, 64, device="cuda", requires_grad=True))]
    for call in calls:
        with pytest.raises(ValueError, match="no gradient"):
            call()
        with torch.no_grad():
            call()
    torch.cuda.synchronize()
    assert x.eq(1).all() and leaf.grad is None


@pytest.mark.parametrize("device", ["cpu", pytest.param("cuda", marks=pytest.mark.gpu)])
def test_dual_tensors_are_refused(device):
    x, w, table = torch.ones(2, 2, 64, device=device), torch.ones(64, device=device), torch.ones(8, 64, device=device)
    slots, pages, lengths = torch.arange(2, device=device), torch.zeros(2, 1, dtype=torch.int32, device=device), torch.ones(2, dtype=torch.int32, device=device)
    cache = ws = None
    if device == "cuda":
        cache, ws = vt.KVCache(1, 16, 2, 64), vt.AttentionWorkspace(2, 2, 2, 64, 2, 1, 16, device)
    with forward_ad.dual_level():
        dx, dw, dt = (forward_ad.make_dual(t, torch.ones_like(t)) for t in (x, w, table))
        calls = [lambda: vt.qk_norm_rope(dx, x), lambda: vt.qk_norm_rope(x, dx), lambda: vt.qk_norm_rope(x, x, None, None, dw, w), lambda: vt.qk_norm_rope(x, x, None, None, w, dw),
                 lambda: vt.qk_norm_rope(x, x, slots, dt), lambda: vt.qk_norm_rope_backward(dx, x, x, x, None, None, w, w),
                 lambda: vt.qk_norm_rope_backward(x, x, x, dx, None, None, w, w), lambda: vt.qkv_to_cache(dx, x, x, cache, slots), lambda: vt.qkv_to_cache(x, x, dx, cache, slots),
                 lambda: vt.kv_cache_write(cache, dx, x, slots), lambda: vt.paged_attention(dx, cache, pages, lengths, ws=ws)]
        for call in calls:
            for grad in (True, False):
                with torch.set_grad_enabled(grad), pytest.raises(ValueError, match="no tangent"):
                    call()
        if device == "cuda":      # others' tangents are nobody's business
            vt.paged_attention(x, cache, pages, lengths, ws=ws)


@pytest.mark.gpu
@pytest.mark.parametrize("dtype", [BF16, torch.float32])
@pytest.mark.parametrize("ahead", [1, 3, 8])
def test_gradients_that_begin_anywhere(dtype, ahead):
    """A piece of a concatenation's gradient is contiguous, and at no multiple of 16 bytes."""
    g = torch.Generator(device="cuda").manual_seed(ahead)

    def randn(*shape):
        return torch.randn(shape, generator=g, device="cuda").to(dtype)
    q, k, wq, wk = randn(5, 4, 64).requires_grad_(), randn(5, 2, 64).requires_grad_(), randn(64).requires_grad_(), randn(64).requires_grad_()
    y, z = vt.qk_norm_rope(q, k, None, None, wq, wk)
    given = randn(ahead + y.numel() + z.numel() + ahead)
    torch.cat([randn(ahead), y.flatten(), randn(ahead), z.flatten()]).backward(given)
    gy, gz = given[ahead:ahead + y.numel()].clone().view_as(y), given[2 * ahead + y.numel():].clone().view_as(z)
    want = vt.qk_norm_rope_backward(gy, gz, q.detach(), k.detach(), None, None, wq.detach(), wk.detach())
    for x, w in zip((q, k, wq, wk), want):
        assert torch.equal(x.grad, w.to(dtype))
