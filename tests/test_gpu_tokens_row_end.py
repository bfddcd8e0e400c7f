"""Many tokens a sequence, with lengths past the end of the page-table row.  No caller may pass them; insertion stores the tokens
that the row has room for and nothing elsewhere, attention is over the row's tokens and reads nothing behind the row."""
import math

import numpy as np
import pytest
import torch

from paper_2406_10774_amd import binding as Q
from packed_util import D, Packed, Trees, attention64, check, left_alone

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("S,pages,over,new", [(16, 5, (1, 40), (30, 41)), (8, 9, (16, 3), (16, 75)), (64, 2, (200, 1), (150, 1)),
                                              (32, 3, (5, 1 << 20), (101, 7)), (16, 4, (0, 64), (64, 64))])
def test_insertion_past_the_row(S, pages, over, new):
    """Sequence b has over[b] tokens more than its row holds, the last new[b] of them all are inserted."""
    rng = np.random.default_rng(S)
    lens = [pages * S + n for n in over]
    p = Packed([S] * 2, new, heads=3, kv_heads=3, S=S, seed=S, cached=False)
    N = 2 * pages + 3
    table = torch.from_numpy(rng.permutation(N)[:2 * pages].reshape(2, pages).astype(np.int32)).to(p.dev)
    k_pool = torch.randn(N, 3, S, D, device=p.dev).half()
    v_pool, meta = torch.randn(N, 3, S, D, device=p.dev).half(), torch.zeros(3, N, 2, D, device=p.dev, dtype=torch.float16)
    cache = Q.Cache(k_pool, v_pool, meta, table, torch.full((2,), pages * S, dtype=torch.int32, device=p.dev))
    Q.quest_build_meta(cache)
    want = [x.clone() for x in (k_pool, v_pool, meta)]
    fits = [max(0, n - m) for n, m in zip(new, over)]           # new tokens that the row has room for: the first ones
    cache = Q.Cache(*want, table, torch.full((2,), pages * S, dtype=torch.int32, device=p.dev))
    cu = torch.tensor([0, fits[0], sum(fits)], dtype=torch.int32, device=p.dev)
    rows = torch.tensor([*range(fits[0]), *range(new[0], new[0] + fits[1])], dtype=torch.int32, device=p.dev)
    if sum(fits):
        Q.quest_append_tokens(cache, p.k_new, p.v_new, cu, rows=rows)
    cache = Q.Cache(k_pool, v_pool, meta, table, torch.tensor(lens, dtype=torch.int32, device=p.dev))
    Q.quest_append_tokens(cache, p.k_new, p.v_new, p.cu)
    torch.cuda.synchronize()
    for got, w, name in zip((k_pool, v_pool, meta), want, ("k", "v", "meta")):
        assert torch.equal(got.view(torch.int16), w.view(torch.int16)), name


@pytest.mark.parametrize("half", [True, False])
@pytest.mark.parametrize("S,pages,heads,kv_heads,over,new", [
    (16, 5, 4, 2, (1, 0, 1000), (1, 5, 40)),               # few rows, in one piece
    (8, 333, 8, 2, (3, 1 << 24, 0), (2, 1, 7)),            # few rows in splits
    (16, 37, 40, 40, (300, 7), (700, 650)),                # many rows, in one piece
    (32, 300, 8, 2, (90, 0), (300, 260)),                  # many rows in splits, paired row tiles
    (8, 1203, 16, 2, (250, 1 << 30), (300, 301)),          # queries before and behind the row's end
])
def test_attention_past_the_row(S, pages, heads, kv_heads, over, new, half):
    """Sequence b's length is over[b] more than its row holds; a query behind the row's end sees the whole row."""
    room = pages * S
    p = Packed([room] * len(over), [min(n, room) for n in new], heads=heads, kv_heads=kv_heads, S=S, seed=S)
    table = p.table[:, :pages].contiguous()                # the rows end with their pages
    list_pages = [[list(range(0, pages, 2)) + [pages, pages + 3, 1 << 28]] * kv_heads] * p.B
    t, listed = Trees(p), Trees(p, lists=list_pages)
    full = torch.full((p.B,), room, dtype=torch.int32, device=p.dev)
    past = torch.tensor([room + n for n in over], dtype=torch.int32, device=p.dev)
    scale = 1 / math.sqrt(D)

    def trees(lens, ws):
        cache = Q.Cache(p.k_pool, p.v_pool, p.meta, table, lens, num_heads=heads)
        results = []
        for x in (t, listed):
            out, lse = p.results(half)
            Q.quest_tree_attention(cache, p.q, p.k_new, p.v_new, p.cu, x.mask, scale, out, topk_idx=x.lists, lse=lse, workspace=ws)
            results += [out, lse]
        return results

    cache = Q.Cache(p.k_pool, p.v_pool, p.meta, table, past, num_heads=heads)
    for ws in (p.workspace(), None):
        for got, want in zip(trees(past, ws), trees(full, ws)):
            assert torch.equal(got, want)
        out, lse = p.results(half)
        Q.quest_prompt_attention(cache, p.q, p.cu, scale, out, lse=lse, workspace=ws)
        torch.cuda.synchronize()
        for b in range(p.B):
            at = p.rows(b)
            position = torch.arange(room + over[b] - p.new[b], room + over[b], device=p.dev)
            sees = torch.arange(room, device=p.dev) <= position[:, None]
            for h in range(heads):
                want = attention64(p.q[at, h].double(), *p.cached(b, h // p.G), sees, scale)
                check(out[at, h], lse[at, h], want, half, (b, h))
        left_alone(p, out, lse)


@pytest.mark.parametrize("half", [True, False])
@pytest.mark.parametrize("heads,kv_heads,lens,new,short", [
    (8, 2, (5000, 700, 3000), (300, 300, 200), 40),         # many rows in splits, paired row tiles
    (8, 2, (9000, 64, 9000), (20, 40, 3), 1),               # few rows in splits
    (40, 40, (700, 650), (700, 600), 0),                    # many rows, in one piece
])
def test_lengths_without_the_new_tokens(heads, kv_heads, lens, new, short, half):
    """Sequence 1's length is less than its new tokens (it does not count them yet, say).  No caller may pass that; the other sequences have
    their results, and queries at positions from 0 on theirs."""
    p = Packed(lens, new, heads=heads, kv_heads=kv_heads, seed=short, room=1 << 14 if kv_heads < 40 else 0)
    p.lens[1] = short
    p.seq_lens.copy_(torch.tensor(p.lens))
    scale = 1 / math.sqrt(D)
    for ws in (p.workspace(), None):
        out, lse = p.results(half)
        Q.quest_prompt_attention(p.cache, p.q, p.cu, scale, out, lse=lse, workspace=ws)
        torch.cuda.synchronize()
        for b in range(p.B):
            position = torch.arange(p.lens[b] - p.new[b], p.lens[b], device=p.dev)
            there = position >= 0
            at = torch.arange(int(p.cu_np[b]), int(p.cu_np[b + 1]), device=p.dev)[there]
            if not len(at):
                continue
            sees = torch.arange(p.lens[b], device=p.dev) <= position[there][:, None]
            for h in range(heads):
                want = attention64(p.q[at, h].double(), *p.cached(b, h // p.G), sees, scale)
                check(out[at, h], lse[at, h], want, half, (b, h))
        left_alone(p, out, lse)
