"""The 4-bit cache and the windowed attention together, as they are used: a draft round of examples/draft_round.py on a layer with a window, and a request's
life in a paged cache -- its prompt chunk by chunk, its tokens one at a time, a tree -- with the pages behind the window given to others."""
import math

import pytest
import torch

import paper_2506_22694_amd as vt
from test_gpu_attention import BF16, F32, _gen, _randn, _table64, norm_rope64
from test_gpu_draft_round import _example
from test_gpu_draft_round_attention import _projected, _rms, _share64
from test_gpu_four_bits import E2M1, held64
from test_gpu_window_attention import attend64, close, sees

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("held", [BF16, torch.float8_e4m3fn, E2M1])
@pytest.mark.parametrize("n,page,window,sinks", [(20, 32, 6, 2), (517, 64, 100, 4), (517, 16, 64, 0), (90, 16, 2, 1)])
def test_a_draft_round_on_a_layer_with_a_window(held, n, page, window, sinks):
    example, depth, width = _example(), 4, 6
    drafter = example.Drafter(d=512, q_heads=4, kv_heads=2, head_dim=64, vocabulary=4000, trimmed=1000, seed=n, window=window, sinks=sinks)
    pages = -(-(n + 64) // page) + 1
    cache = vt.KVCache(pages, page, 2, 64, held)
    table = torch.randperm(pages, generator=torch.Generator().manual_seed(1))[None].int().cuda()
    prompt = torch.randint(0, 4000, (n,), generator=torch.Generator().manual_seed(2)).cuda()
    tree = example.draft_round(drafter, prompt, cache, table, depth=depth, width=width, keep=10)

    tokens = torch.cat([prompt, tree["token"][:-width].long()])
    positions = torch.cat([torch.arange(n, device="cuda"), n + tree["depth"][:-width].long()])
    count = tokens.numel()
    slots = cache.slots(table, torch.zeros(count, dtype=torch.int64, device="cuda"), torch.arange(count, device="cuda"))
    k, v = (x.double() for x in vt.kv_cache_read(cache, slots, dtype=F32))
    # what is held of v is what the projection's rows are rounded to (bf16 rows are not compared: their rounding is the product's)
    if held == E2M1:
        rows = (drafter.embedding[prompt[:-1]] @ drafter.qkv).unflatten(1, (-1, 64))[:, 6:]
        assert torch.equal(v[:n - 1], held64(rows.double()))
    parent = tree["parent"].tolist()
    for i in range(depth * width):
        path, at = [], parent[i]
        while at >= 0:
            path.append(n + at)
            at = parent[at]
        row = n + parent[i] if parent[i] >= 0 else n - 1
        p = positions[row].item()
        x = drafter.embedding[tokens[row]].double()
        # (cached places count for the window: a node's own place is behind the prompt)
        rows = [t for t in list(range(n)) + path[::-1] if t > p - window or t < sinks]
        want, got = _share64(drafter, tokens[row], positions[row], k[rows], v[rows]), tree["hidden"][i].double()
        # Half steps of 2^-8: the projection's q and q itself, the attention's result and its product of the share's size; the sum of the row's.
        bound = 2 ** -8 * (4 * _rms(want) + _rms(got))
        assert _rms(got - x - want) <= bound, i
        assert _rms(got - x) > 4 * bound


def test_a_request_from_its_prompt_to_a_tree_while_pages_change_hands():
    g = _gen(50)
    hq, hk, D, page, window, sinks = 16, 4, 128, 16, 200, 4
    cache = vt.KVCache(80, page, hk, D, dtype=E2M1)
    for s in (cache.k_scale, cache.v_scale):
        s.fill_(255)      # NaN wherever nothing has been written
    w, rope = (_randn(g, D) * 0.2 + 1).to(BF16), _table64(1500, D)
    total, chunk = 1250, 300
    everything = _randn(g, total, hq + 2 * hk, D).to(BF16)
    q, k, v = everything.split([hq, hk, hk], dim=1)
    k64, v64 = held64(norm_rope64(k, torch.arange(total, device="cuda"), rope, w, 2.0 ** -20, False)), held64(v.double())
    table = torch.full((1, 100), -1, dtype=torch.int32, device="cuda")
    free, mine = list(range(80)), {}

    def own_pages(upto, lowest):
        """Pages for tokens up to `upto`; those of tokens before `lowest` that are no sinks go back, and hold NaN from then on."""
        for p in range(-(-upto // page)):
            if p not in mine and (p + 1) * page > lowest:
                mine[p] = free.pop(0)
        for p in [p for p in mine if sinks <= p * page and (p + 1) * page <= lowest]:
            for s in (cache.k_scale, cache.v_scale):
                s[mine[p]] = 255
            free.append(mine.pop(p))
        table.fill_(-1)
        for p, number in mine.items():
            table[0, p] = number

    def step(start, count, mask=None, positions=None, length=None):
        at = torch.arange(start, start + count, device="cuda")
        where = at if positions is None else positions
        slots = cache.slots(table, torch.zeros(count, dtype=torch.int64, device="cuda"), at)
        turned = vt.qkv_to_cache(q[start:start + count], k[start:start + count], v[start:start + count], cache, slots, where, rope, w, w, eps=2.0 ** -20)
        length = torch.tensor([start + count], dtype=torch.int32, device="cuda")
        starts = torch.tensor([0, count], dtype=torch.int32, device="cuda")
        out, lse = vt.paged_attention(turned, cache, table, length, row_start=starts, max_rows=count, tail_mask=mask, window=window, sinks=sinks,
                                      positions=None if mask is None else where, return_lse=True)
        kk, vv = k64[:start + count].clone(), v64[:start + count]
        if positions is not None:
            kk[start:] = held64(norm_rope64(k[start:start + count], positions, rope, w, 2.0 ** -20, False))
        see = sees(start + count, count, window, sinks, mask, positions)
        want, want_lse, spread = attend64(turned, kk, vv, see, D ** -0.5)
        sizes = (turned.double().abs().amax() * kk.abs().sum(-1).amax() * D ** -0.5).item()
        fine = sizes * (math.sqrt(D) / 2 + 8) * 2.0 ** -24 + 40 * 2.0 ** -24
        close(out, want, 2.0 ** -8, (fine + 2.0 ** -16) * 2 * spread)
        close(lse, want_lse, 2.0 ** -23, fine * 2)

    start = 0
    while start < 1200:      # the prompt
        own_pages(start + chunk, start - window + 1)
        step(start, chunk)
        start += chunk
    for _ in range(20):      # tokens
        own_pages(start + 1, start - window + 1)
        step(start, 1)
        start += 1
    # a tree's level of eight nodes behind the last token, each of its own
    own_pages(start + 8, start - window + 1 - 8)
    mask = torch.tensor([((1 << 56) - 1) | (1 << (56 + i)) for i in range(7)] + [((1 << 56) - 1) - (1 << 63)], device="cuda")
    step(start, 8, mask=mask, positions=torch.full((8,), start, device="cuda"))
    assert len(mine) < 2 * window // page + 2
