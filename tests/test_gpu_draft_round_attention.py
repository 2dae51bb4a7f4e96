"""examples/draft_round.py: the attention's share of every hidden row, against 64 bits over the keys and values that the cache holds, with a bound that
a row without attention and a row of another node's path are outside of."""
import pytest
import torch

import paper_2506_22694_amd as vt
from paper_2506_22694_amd import binding
from test_gpu_draft_round import _example

pytestmark = pytest.mark.gpu


def _rms(x):
    return x.square().mean().sqrt().item()


def _normed(drafter, y, weight, positions):
    """Rows y [n, heads, D], float64: norm and rotation."""
    c, s = drafter.rope[positions].double()[:, None].chunk(2, dim=-1)
    y = y / (y.square().mean(-1, keepdim=True) + 1e-6).sqrt() * weight.double()
    a, b = y.chunk(2, dim=-1)
    return torch.cat([a * c - b * s, b * c + a * s], -1)


def _projected(drafter, tokens):
    y = (drafter.embedding[tokens].double() @ drafter.qkv.double()).unflatten(1, (-1, drafter.head_dim))
    return torch.split(y, [drafter.q_heads, drafter.kv_heads, drafter.kv_heads], dim=1)


def _share64(drafter, token, position, k, v):
    """What the attention adds to the hidden row of a token that sees the cached rows k, v [tokens, heads, D]."""
    q = _normed(drafter, _projected(drafter, token[None])[0], drafter.q_norm, position[None])[0]
    group = drafter.q_heads // drafter.kv_heads
    k, v = k.repeat_interleave(group, 1), v.repeat_interleave(group, 1)
    p = torch.softmax((q[None] * k).sum(-1) * drafter.head_dim ** -0.5, dim=0)
    return (p[..., None] * v).sum(0).flatten() @ drafter.out.double()


@pytest.mark.parametrize("held", [torch.bfloat16, torch.float8_e4m3fn])
@pytest.mark.parametrize("n,page", [(1, 16), (9, 16), (20, 32), (517, 64)])
def test_the_attention_of_every_node(held, n, page):
    example, depth, width = _example(), 4, 6
    drafter = example.Drafter(d=512, q_heads=4, kv_heads=2, head_dim=64, vocabulary=4000, trimmed=1000, seed=n)
    pages = -(-(n + 64) // page) + 1
    cache = vt.KVCache(pages, page, 2, 64, held)
    table = torch.randperm(pages, generator=torch.Generator().manual_seed(1))[None].int().cuda()
    prompt = torch.randint(0, 4000, (n,), generator=torch.Generator().manual_seed(2)).cuda()
    tree = example.draft_round(drafter, prompt, cache, table, depth=depth, width=width, keep=10)

    # the prompt's rows, then the nodes' of all levels but the last, in the order they were drafted
    tokens = torch.cat([prompt, tree["token"][:-width].long()])
    positions = torch.cat([torch.arange(n, device="cuda"), n + tree["depth"][:-width].long()])
    count = tokens.numel()
    slots = cache.slots(table, torch.zeros(count, dtype=torch.int64, device="cuda"), torch.arange(count, device="cuda"))
    k, v = (x.double() for x in vt.kv_cache_read(cache, slots, dtype=torch.float32))
    _, k64, v64 = _projected(drafter, tokens)
    k64 = _normed(drafter, k64, drafter.k_norm, positions)
    # bf16: two roundings of half a step of 2^-8 (the projection's result, what is held; and fp32's); 8 bits: half a step of 2^-4 beside the first
    step = 2 * 2 ** -8 if held == torch.bfloat16 else 2 ** -4 + 2 ** -8
    for got, want in ((k, k64), (v, v64)):
        off = (got - want).square().mean((1, 2)).sqrt() - step * want.square().mean((1, 2)).sqrt()
        assert off.max().item() <= 0.0

    parent = tree["parent"].tolist()
    for i in range(depth * width):
        seen, at = [], parent[i]
        while at >= 0:
            seen.append(n + at)
            at = parent[at]
        row = n + parent[i] if parent[i] >= 0 else n - 1
        x = drafter.embedding[tokens[row]].double()

        def share(seen):
            rows = list(range(n)) + seen
            return _share64(drafter, tokens[row], positions[row], k[rows], v[rows])
        want, got = share(seen), tree["hidden"][i].double()
        # Half steps of 2^-8: the projection's q and q itself (their scores, and by those the share's parts, are off by that much: a score is a sum of
        # 64 products of unit size over the root of 64), the attention's result and its product of the share's size; the sum of the row's.
        bound = 2 ** -8 * (4 * _rms(want) + _rms(got))
        assert _rms(got - x - want) <= bound, i
        # (else the bound says nothing)
        assert _rms(got - x) > 4 * bound
        if n <= 20 and parent[i] >= 0:
            # another node of the parent's level in its place, or nothing
            first = parent[i] // width * width
            other = n + (parent[i] + 1 if parent[i] + 1 < first + width else first)
            assert _rms(got - x - share([other] + seen[1:])) > 2 * bound and _rms(got - x - share(seen[1:])) > 2 * bound, i


def test_a_round_takes_the_native_way_and_copies_nothing_from_the_host(monkeypatch):
    example = _example()
    drafter = example.Drafter(d=512, q_heads=4, kv_heads=2, head_dim=64, vocabulary=4000, trimmed=1000)
    cache, table = vt.KVCache(4, 64, 2, 64), torch.arange(4, dtype=torch.int32, device="cuda")[None].contiguous()
    prompt = torch.arange(100, device="cuda")
    memory = example.Memory(drafter, 200, 3, 8, 16)
    want = example.draft_round(drafter, prompt, cache, table, memory=memory)
    asked, native = [], binding._bind

    class Spy:
        def __getattr__(self, name):
            def call(*a):
                got = getattr(native, name)(*a)
                asked.append((name, got is not None and not (type(got) is int and got < 0)))
                return got
            return call
    monkeypatch.setattr(binding, "_bind", Spy())
    torch.cuda.set_sync_debug_mode("error")
    try:
        got = example.draft_round(drafter, prompt, cache, table, memory=memory)
    finally:
        torch.cuda.set_sync_debug_mode("default")
    names = [name for name, _ in asked]
    assert all(done for _, done in asked) and [names.count(x) for x in ("to_cache", "attend", "level", "rerank")] == [4, 3, 3, 1]
    for key in want:
        assert torch.equal(got[key], want[key]), key
