"""examples/draft_round.py: the attention's calls and the trimmed head's in one draft round, against a dense forward pass in 64 bits."""
import importlib.util
import os

import pytest
import torch

import paper_2506_22694_amd as vt

pytestmark = pytest.mark.gpu
ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))


def _example():
    spec = importlib.util.spec_from_file_location("draft_round", os.path.join(ROOT, "examples", "draft_round.py"))
    m = importlib.util.module_from_spec(spec)
    spec.loader.exec_module(m)
    return m


def _hidden64(drafter, tokens):
    """The hidden row of the last of `tokens`, whole sequence, in 64 bits."""
    n, D = len(tokens), drafter.head_dim
    x = drafter.embedding[torch.tensor(tokens, device="cuda")].double()
    qkv = (x @ drafter.qkv.double()).unflatten(1, (-1, D))
    q, k, v = torch.split(qkv, [drafter.q_heads, drafter.kv_heads, drafter.kv_heads], dim=1)
    c, s = drafter.rope[:n].double()[:, None].chunk(2, dim=-1)

    def turned(y, w):
        y = y / (y.square().mean(-1, keepdim=True) + 1e-6).sqrt() * w.double()
        a, b = y.chunk(2, dim=-1)
        return torch.cat([a * c - b * s, b * c + a * s], -1)
    q, k = turned(q, drafter.q_norm)[-1], turned(k, drafter.k_norm)
    group = drafter.q_heads // drafter.kv_heads
    k, v = k.repeat_interleave(group, 1), v.repeat_interleave(group, 1)
    p = torch.softmax((q[None] * k).sum(-1) * D ** -0.5, dim=0)
    return x[-1] + (p[..., None] * v).sum(0).flatten() @ drafter.out.double()


@pytest.mark.parametrize("held,prompt_length,page", [(torch.bfloat16, 1, 16), (torch.bfloat16, 517, 64), (torch.float8_e4m3fn, 130, 32)])
def test_every_node_is_drafted_from_its_own_path(held, prompt_length, page):
    example = _example()
    drafter = example.Drafter(d=512, q_heads=4, kv_heads=2, head_dim=64, vocabulary=4000, trimmed=1000, seed=prompt_length)
    pages = -(-(prompt_length + 64) // page) + 1
    cache = vt.KVCache(pages, page, 2, 64, held)
    table = torch.randperm(pages, generator=torch.Generator().manual_seed(1))[None].int().cuda()
    prompt = torch.randint(0, 4000, (prompt_length,), generator=torch.Generator().manual_seed(2)).cuda()
    tree = example.draft_round(drafter, prompt, cache, table, depth=4, width=6, keep=10)
    parent, token = tree["parent"].tolist(), tree["token"].tolist()
    # Seven roundings to bf16 lie between a path and its row (the projection, q, k, v, the attention's weights and result, the sum), half a
    # step of 2^-8 each, of values and of scores of size up to 4: 7 * 2^-8 * 4 of the attention's share, whose size is about 1 or less.  Eight
    # bits hold k and v to half a step of 2^-4 each, independent from value to value: sums of 64 of them are off by 2^-4 / 2 of a score's size.
    bound = 7 * 2 ** -8 * 4 if held == torch.bfloat16 else 7 * 2 ** -8 * 4 + 2 * 2 ** -4 * 4
    for i in range(len(token)):
        path, at = [], parent[i]
        while at >= 0:
            path.append(token[at])
            at = parent[at]
        want = _hidden64(drafter, prompt.tolist() + path[::-1])
        assert (tree["hidden"][i].double() - want).square().mean().sqrt() <= bound, i
        assert parent[i] < i and tree["depth"][i] == len(path)
        # the log-probability: the parent's and this token's on that row
        z = drafter.head.double() @ tree["hidden"][i].double()
        lp = torch.log_softmax(z, 0)[(drafter.map == token[i]).nonzero().item()] + (tree["cum"][parent[i]].double() if parent[i] >= 0 else 0.0)
        assert abs(tree["cum"][i].item() - lp.item()) <= 2e-3
    kept = tree["kept"].tolist()
    assert kept == sorted(kept) and len(kept) == 10 and all(parent[i] in kept or parent[i] < 0 for i in kept)
