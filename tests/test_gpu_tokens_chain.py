"""Prompts, drafted tokens and decode steps together on one cache, as a serving loop calls them; captured graphs, streams,
repeated calls and pools beyond 32-bit offsets."""
import math

import numpy as np
import pytest
import torch

from paper_2406_10774_amd import binding as Q
from packed_util import D, Packed, Trees, check, attention64, check_prompt, check_tree, random_tree

pytestmark = pytest.mark.gpu
SCALE = 1 / math.sqrt(D)


def prompt(p, out, lse, ws):
    Q.quest_prompt_attention(p.cache, p.q, p.cu, SCALE, out, lse=lse, workspace=ws)


def tree(p, t, out, lse, ws):
    Q.quest_tree_attention(p.cache, p.q, p.k_new, p.v_new, p.cu, t.mask, SCALE, out, topk_idx=t.lists, lse=lse, workspace=ws)


@pytest.mark.parametrize("S,heads,kv_heads,half", [(16, 4, 4, False), (16, 16, 2, True), (8, 6, 2, False), (64, 8, 1, True)])
def test_serving_loop(S, heads, kv_heads, half):
    """Two prompts go into the cache in two parts each, then rounds of: pages chosen by the root's query, drafts checked over
    them, the accepted ones inserted, one decode step.  Every result against 64 bits on the cache as it then is."""
    rng = np.random.default_rng(S)
    parts = [[300, 517], [411, 90]]
    p = Packed([0, 0], [sum(x) for x in zip(*parts)], heads=heads, kv_heads=kv_heads, S=S, seed=S, cached=False, room=1200)
    pages = 1200 // S                                   # a row's worth of pages for each sequence
    N = 2 * pages + 1
    ids = rng.permutation(N)[:2 * pages].reshape(2, pages)
    table = torch.from_numpy(ids.astype(np.int32)).to(p.dev)
    k_pool = torch.full((N, kv_heads, S, D), math.nan, device=p.dev, dtype=torch.float16)
    v_pool, meta = k_pool.clone(), torch.zeros(kv_heads, N, 2, D, device=p.dev, dtype=torch.float16)
    lens = torch.zeros(2, device=p.dev, dtype=torch.int32)
    cache = Q.Cache(k_pool, v_pool, meta, table, lens, num_heads=heads)
    length = [0, 0]
    seed = [0]

    def step(new):
        """Packed data of the next `new` tokens over this cache."""
        seed[0] += 1
        x = Packed(length, new, heads=heads, kv_heads=kv_heads, S=S, seed=seed[0], cached=False)
        x.k_pool, x.v_pool, x.meta, x.table, x.seq_lens, x.cache = k_pool, v_pool, meta, table, lens, cache
        return x

    def grow(by):
        for b in range(2):
            length[b] += by[b]
        lens.copy_(torch.tensor(length))

    def metadata_is_right():
        fresh = torch.zeros_like(meta)
        Q.quest_build_meta(Q.Cache(k_pool, v_pool, fresh, table, lens, num_heads=heads))
        for b in range(2):
            used = table[b, :-(-length[b] // S)].long()
            assert torch.equal(fresh[:, used].view(torch.int16), meta[:, used].view(torch.int16))

    for new in parts:
        x = step(new)
        grow(new)
        x.lens = list(length)
        Q.quest_append_tokens(cache, x.k_new, x.v_new, x.cu)
        out, lse = x.results(half)
        prompt(x, out, lse, x.workspace())
        check_prompt(x, out, lse, half, SCALE, ("prompt", new))
        metadata_is_right()

    K = 256 // S
    scores = torch.zeros(2, kv_heads, pages, device=p.dev)
    idx = torch.zeros(2, kv_heads, K, device=p.dev, dtype=torch.int32)
    for new, kept in (([9, 4], [3, 4]), ([1, 30], [1, 2]), ([70, 12], [8, 1])):
        x = step(new)
        x.lens = list(length)
        roots = x.q[[0, new[0]]].contiguous()
        Q.quest_estimate(cache, roots, scores)
        Q.quest_topk(cache, scores, K, idx)
        t = Trees(x, seed=seed[0])
        t.lists = idx
        out, lse = x.results(half)
        tree(x, t, out, lse, x.workspace())
        check_tree(x, t, out, lse, half, SCALE, ("tree", new))
        # the first nodes of each sequence's drafts that make a path: here, any rows
        rows = torch.tensor([*rng.permutation(new[0])[:kept[0]], *(new[0] + rng.permutation(new[1])[:kept[1]])], dtype=torch.int32)
        grow(kept)
        cu = torch.tensor([0, kept[0], kept[0] + kept[1]], dtype=torch.int32, device=p.dev)
        Q.quest_append_tokens(cache, x.k_new, x.v_new, cu, rows=rows.to(p.dev))
        metadata_is_right()
        for b in range(2):
            for i in range(kept[b]):
                at = length[b] - kept[b] + i
                row = int(rows[(kept[0] if b else 0) + i])
                assert torch.equal(k_pool[table[b, at // S].long(), :, at % S], x.k_new[row])
        # a decode step of the next token, over everything
        x = step([1, 1])
        grow([1, 1])
        x.lens = list(length)
        ws = torch.zeros(Q.quest_step_workspace_bytes(cache, pages) // 4, device=p.dev)
        o, l = x.results(half)
        everything = torch.zeros(2, kv_heads, pages, device=p.dev, dtype=torch.int32)
        Q.quest_decode_step(cache, x.k_new[:2].contiguous(), x.v_new[:2].contiguous(), True, x.q[:2].contiguous(), pages, SCALE,
                            scores, everything, o, ws, lse=l)
        check_prompt(x, o, l, half, SCALE, "step")       # one query a sequence, the last position
        metadata_is_right()
        # and the same query as a prompt of one token
        o2, l2 = x.results(half)
        prompt(x, o2, l2, x.workspace())
        check_prompt(x, o2, l2, half, SCALE, "step as a prompt")


@pytest.mark.parametrize("heads,room", [(4, 0), (40, 8192)])
def test_captured_calls_serve_other_lengths(heads, room):
    """One graph of insertion, prompt and tree attention; replayed with other lengths, other rows and other data, eager calls
    and work in between; each replay as the eager calls.  The two attentions share a workspace."""
    shapes = [([400, 90, 1500], [37, 20, 11]), ([64, 0, 33], [1, 0, 33]), ([10, 700, 2000], [10, 5, 60]), ([5, 5, 5], [0, 0, 5])]
    total = 80
    most = Packed([2048] * 3, [total // 3] * 3, heads=heads, kv_heads=2, seed=1, room=room, spare_rows=total - 3 * (total // 3))
    ws = most.workspace()
    words = 1
    mask = torch.zeros(total, words, device=most.dev, dtype=torch.int64)
    kv = [torch.zeros(total, 2, D, device=most.dev, dtype=torch.float16) for _ in range(2)]
    outs = [most.results(True) for _ in range(2)]

    def calls(outs):
        Q.quest_append_tokens(most.cache, *kv, most.cu)
        Q.quest_prompt_attention(most.cache, most.q, most.cu, SCALE, outs[0][0], lse=outs[0][1], workspace=ws)
        Q.quest_tree_attention(most.cache, most.q, *kv, most.cu, mask, SCALE, outs[1][0], lse=outs[1][1], workspace=ws)

    calls(outs)
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        calls(outs)
    gen = torch.Generator(device=most.dev)
    for i, (lens, new) in enumerate(shapes + shapes[:2]):
        gen.manual_seed(i)
        rng = np.random.default_rng(i)
        most.cu.copy_(torch.from_numpy(np.concatenate([[0], np.cumsum(new)]).astype(np.int32)))
        most.seq_lens.copy_(torch.tensor(lens))
        for x in (most.k_pool, most.v_pool, most.q, *kv):
            x.copy_(torch.randn(x.shape, device=most.dev, dtype=torch.float16, generator=gen))
        mask.copy_(torch.from_numpy(rng.integers(-2 ** 63, 2 ** 63, (total, words), dtype=np.int64)))
        for o, l in outs:
            o.fill_(77)
            l.fill_(77)
        before = [x.clone() for x in (most.k_pool, most.v_pool, most.meta)]
        graph.replay()
        torch.cuda.synchronize()
        got = [x.clone() for x in (most.k_pool, most.v_pool, most.meta)]
        for x, y in zip((most.k_pool, most.v_pool, most.meta), before):
            x.copy_(y)
        eager = [most.results(True) for _ in range(2)]
        calls(eager)
        torch.cuda.synchronize()
        for x, y in zip((most.k_pool, most.v_pool, most.meta), got):
            assert torch.equal(x.view(torch.int16), y.view(torch.int16)), i
        for (o, l), (eo, el) in zip(outs, eager):
            assert torch.equal(o, eo) and torch.equal(l, el), i
            assert bool((o[sum(new):] == 77).all()) and bool((l[sum(new):] == 77).all())


def test_streams_and_repeats():
    """The same bits in every run; two streams at once, each with its workspace, as one after the other."""
    p = Packed([3000, 900, 50], [40, 3, 50], heads=16, kv_heads=4, seed=2)
    few = Packed([5000, 17], [2, 5], heads=4, kv_heads=1, seed=3)
    t, tf = Trees(p), Trees(few)
    want = [x.results(True) for x in (p, p, few, few)]

    def calls(res, ws):
        prompt(p, *res[0], ws)
        tree(p, t, *res[1], ws)
        prompt(few, *res[2], ws)
        tree(few, tf, *res[3], ws)

    size = max(p.workspace().numel(), few.workspace().numel())
    calls(want, torch.zeros(size, device=p.dev))
    torch.cuda.synchronize()
    streams = [torch.cuda.Stream() for _ in range(2)]
    work = [torch.zeros(size, device=p.dev) for _ in streams]
    got = [[[x.results(True) for x in (p, p, few, few)] for _ in range(6)] for _ in streams]
    torch.cuda.synchronize()
    for i in range(6):
        for s, stream in enumerate(streams):
            with torch.cuda.stream(stream):
                calls(got[s][i], work[s])
    torch.cuda.synchronize()
    for s in range(2):
        for res in got[s]:
            for (o, l), (wo, wl) in zip(res, want):
                assert torch.equal(o, wo) and torch.equal(l, wl)


def test_pools_beyond_32_bits():
    """Pages whose offsets pass 2^32 bytes, written by the insertion and read by both attentions."""
    Hkv, S, N = 32, 16, 36000                     # 4.7 GB a pool
    free, _ = torch.cuda.mem_get_info()
    if free < 14e9:
        pytest.skip("needs 14 GB of memory")
    p = Packed([600, 300], [600, 300], heads=Hkv, kv_heads=Hkv, S=S, seed=6, cached=False)
    k_pool = torch.empty(N, Hkv, S, D, device=p.dev, dtype=torch.float16)
    v_pool = torch.empty_like(k_pool)
    meta = torch.empty(Hkv, N, 2, D, device=p.dev, dtype=torch.float16)
    pages = 600 // S + 1
    table = torch.tensor([[N - 1 - i for i in range(pages)], [i if i % 2 else N // 2 + i for i in range(pages)]], dtype=torch.int32,
                         device=p.dev)
    p.k_pool, p.v_pool, p.meta, p.table = k_pool, v_pool, meta, table
    p.cache = Q.Cache(k_pool, v_pool, meta, table, p.seq_lens)
    Q.quest_append_tokens(p.cache, p.k_new, p.v_new, p.cu)
    for b in range(2):
        k, v = p.cached(b, Hkv - 1)
        assert torch.equal(k, p.k_new[p.rows(b), Hkv - 1].double()) and torch.equal(v, p.v_new[p.rows(b), Hkv - 1].double())
    built = torch.zeros_like(meta)
    Q.quest_build_meta(Q.Cache(k_pool, v_pool, built, table, p.seq_lens))
    for b in range(2):
        used = table[b, :-(-p.lens[b] // S)].long()
        assert torch.equal(built[:, used].view(torch.int16), meta[:, used].view(torch.int16))
    out, lse = p.results(True)
    prompt(p, out, lse, p.workspace())
    check_prompt(p, out, lse, True, SCALE)
    t = Trees(p, kind=lambda rng, n, words: np.eye(n, dtype=bool))
    out, lse = p.results(True)
    tree(p, t, out, lse, p.workspace())
    check_tree(p, t, out, lse, True, SCALE)
