"""Many tokens a sequence on the GPU: insertion against the one-token call, attention of prompts and of drafted
tokens against 64 bits, at the lengths, pages, groups, strides and masks where they can go wrong."""
import math

import numpy as np
import pytest
import torch

from paper_2406_10774_amd import binding as Q
from packed_util import D, Packed, Trees, check_prompt, check_tree

pytestmark = pytest.mark.gpu
SCALE = 1 / math.sqrt(D)
ROOMS = [0, 1 << 18]     # page-table rows that end with the sequence, and long ones: other kernels and splits


def run_prompt(p, half, scale=SCALE, workspace="full"):
    out, lse = p.results(half)
    ws = p.workspace() if workspace == "full" else None
    Q.quest_prompt_attention(p.cache, p.q, p.cu, scale, out, lse=lse, workspace=ws)
    torch.cuda.synchronize()
    return out, lse


def run_tree(p, t, half, scale=SCALE, workspace="full"):
    out, lse = p.results(half)
    ws = p.workspace() if workspace == "full" else None
    Q.quest_tree_attention(p.cache, p.q, p.k_new, p.v_new, p.cu, t.mask, scale, out, topk_idx=t.lists, lse=lse, workspace=ws)
    torch.cuda.synchronize()
    return out, lse


@pytest.mark.parametrize("half", [True, False])
@pytest.mark.parametrize("room", ROOMS)
@pytest.mark.parametrize("n", [1, 2, 31, 32, 33, 63, 64, 65, 127, 128, 129, 200, 255, 256, 257, 515, 1100])
def test_whole_prompts(n, room, half):
    p = Packed([n], [n], heads=3, kv_heads=3, seed=n, room=room)
    for ws in ("full", None):
        check_prompt(p, *run_prompt(p, half, workspace=ws), half, SCALE, (n, ws))


@pytest.mark.parametrize("room", ROOMS)
@pytest.mark.parametrize("heads,kv_heads", [(1, 1), (4, 4), (4, 1), (6, 2), (10, 2), (16, 2), (18, 1), (40, 1)])
def test_prompt_groups_ragged(heads, kv_heads, room):
    """Sequences of different lengths, one without new tokens, parts of prompts behind cached tokens."""
    p = Packed([150, 40, 333, 1, 70], [150, 0, 37, 1, 65], heads=heads, kv_heads=kv_heads, seed=heads, room=room)
    for half in (True, False):
        check_prompt(p, *run_prompt(p, half), half, SCALE, (heads, kv_heads, half))


@pytest.mark.parametrize("room", ROOMS)
@pytest.mark.parametrize("S", [8, 16, 32, 64])
def test_prompt_page_sizes_and_strides(S, room):
    for stride in (0, 8, 3 * D):
        p = Packed([301, 64, 7, 1210], [301, 20, 7, 100], heads=8, kv_heads=2, S=S, seed=S, stride=stride, room=room)
        check_prompt(p, *run_prompt(p, True), True, SCALE, (S, stride))


@pytest.mark.parametrize("new,past", [(1, 5000), (5, 3001), (64, 4100), (300, 2000)])
def test_prompt_parts_behind_long_contexts(new, past):
    """Few rows, many tokens: splits of the tokens, joined; without a workspace the same in one piece."""
    p = Packed([past + new, past // 3 + 1], [new, 1], heads=8, kv_heads=2, seed=new)
    for half in (True, False):
        for ws in ("full", None):
            check_prompt(p, *run_prompt(p, half, workspace=ws), half, SCALE, (new, past, half, ws))


@pytest.mark.parametrize("scale", [SCALE, -SCALE, 0.0, 1.0])
def test_prompt_scales(scale):
    for room in ROOMS:
        p = Packed([190], [190], heads=2, kv_heads=2, seed=5, spread=2.0, room=room)
        for half in (True, False):
            check_prompt(p, *run_prompt(p, half, scale), half, scale, scale)


@pytest.mark.parametrize("seed", range(24))
def test_prompts_in_splits(seed):
    """Ragged parts of prompts: odd and even numbers of row tiles, of both kernels, most of them in several splits."""
    rng = np.random.default_rng(seed)
    B, S = int(rng.integers(1, 5)), int(rng.choice([8, 16, 32, 64]))
    kv_heads = int(rng.integers(1, 4))
    heads = kv_heads * int(rng.choice([1, 2, 3, 4, 7]))
    new = [int(rng.integers(1, 700)) for _ in range(B)]
    lens = [n + int(rng.choice([0, rng.integers(0, 300), rng.integers(0, 5000)])) for n in new]
    p = Packed(lens, new, heads=heads, kv_heads=kv_heads, S=S, seed=seed, room=ROOMS[seed % 2])
    half = seed % 3 > 0
    whole = run_prompt(p, half)
    check_prompt(p, *whole, half, SCALE, seed)
    again = run_prompt(p, half)
    assert torch.equal(whole[0], again[0]) and torch.equal(whole[1], again[1])


@pytest.mark.parametrize("half", [True, False])
@pytest.mark.parametrize("kv_heads", [40, 8])
def test_prompts_that_fill_the_card(kv_heads, half):
    """Enough rows for the large kernel, in one piece."""
    p = Packed([700, 950, 40], [700, 333, 40], heads=40, kv_heads=kv_heads, seed=kv_heads)
    check_prompt(p, *run_prompt(p, half), half, SCALE)


@pytest.mark.parametrize("most,heads", [(40, 4), (60, 12)])
def test_prompt_of_more_sequences_than_lanes(most, heads):
    new = [int(x) for x in np.random.default_rng(0).integers(0, most, 150)]
    lens = [n + (7 * i) % 50 + 1 for i, n in enumerate(new)]
    lens[77] += 3000
    p = Packed(lens, new, heads=heads, kv_heads=1, seed=6)
    check_prompt(p, *run_prompt(p, True), True, SCALE)


@pytest.mark.parametrize("room", ROOMS)
def test_prompt_rising_logits(room):
    """The running maximum moves in every tile: logits grow along the sequence, then fall."""
    p = Packed([700], [700], heads=2, kv_heads=1, seed=7, room=room)
    t = torch.arange(700, device=p.dev)
    phys = p.table[0].long()[t // p.S]
    ramp = (torch.where(t < 400, t, 800 - t).float() * 0.25)[:, None, None].half()
    p.k_pool[phys, :, t % p.S] = ramp * torch.ones(1, 1, D, device=p.dev, dtype=torch.float16) / 16
    p.q[:700] = p.q[:700].abs()
    for half in (True, False):
        check_prompt(p, *run_prompt(p, half), half, SCALE, half)


@pytest.mark.parametrize("half", [True, False])
@pytest.mark.parametrize("room", ROOMS)
@pytest.mark.parametrize("n,ctx", [(1, 0), (1, 1), (1, 700), (5, 64), (8, 1000), (31, 65), (33, 129), (64, 300), (65, 300), (130, 77),
                                   (140, 3000), (3, 3000)])
def test_trees(n, ctx, room, half):
    p = Packed([ctx, ctx // 2], [n, max(1, n // 3)], heads=4, kv_heads=2, seed=n + ctx, stride=16, room=room)
    t = Trees(p, seed=n)
    for ws in ("full", None):
        check_tree(p, t, *run_tree(p, t, half, workspace=ws), half, SCALE, (n, ctx, ws))


@pytest.mark.parametrize("room", ROOMS)
@pytest.mark.parametrize("heads,kv_heads,S", [(1, 1, 16), (8, 1, 8), (6, 2, 32), (64, 2, 64), (20, 4, 16), (24, 1, 8), (32, 2, 32)])
def test_tree_groups_and_pages(heads, kv_heads, S, room):
    p = Packed([900, 0, 64, 1203], [12, 3, 0, 40], heads=heads, kv_heads=kv_heads, S=S, seed=S, room=room)
    t = Trees(p, seed=S, words=2)
    for half in (True, False):
        check_tree(p, t, *run_tree(p, t, half), half, SCALE, (heads, kv_heads, S, half))


def nothing(rng, n, words):
    return np.zeros((n, n), bool)


def everything(rng, n, words):
    return np.ones((n, n), bool)


def anything(rng, n, words):
    return rng.random((n, n)) < 0.3


@pytest.mark.parametrize("kind", [nothing, everything, anything])
def test_tree_masks(kind):
    """Also rows that see no drafted node, and, without a context, nothing at all: out 0, lse -inf."""
    for room in ROOMS:
        p = Packed([0, 50, 128], [20, 70, 64], heads=4, kv_heads=2, seed=3, room=room)
        t = Trees(p, kind=kind, words=3)
        for half in (True, False):
            for ws in ("full", None):
                out, lse = run_tree(p, t, half, workspace=ws)
                check_tree(p, t, out, lse, half, SCALE, (kind.__name__, half, room))
                if kind is nothing:
                    assert bool((out[:20] == 0).all()) and bool((lse[:20] == -math.inf).all())


@pytest.mark.parametrize("S", [8, 16, 32, 64])
@pytest.mark.parametrize("K", [1, 3, 17, 40])
def test_tree_listed_pages(S, K):
    """Lists as the selection leaves them, and with holes, ids of pages without tokens and a page twice."""
    rng = np.random.default_rng(S * K)
    p = Packed([1500, 30, 777], [9, 20, 1], heads=8, kv_heads=2, S=S, seed=K)   # (40 pages of 64: more than a row has)
    lists = np.full((3, 2, K), -1, np.int32)
    for b in range(3):
        pages = -(-p.lens[b] // S)
        for h in range(2):
            m = min(K, pages)
            lists[b, h, :m] = np.sort(rng.permutation(pages)[:m])
    rough = lists.copy()
    for b in range(3):
        for h in range(2):
            rng.shuffle(rough[b, h])
            if K >= 3:
                rough[b, h, K // 2] = -5 if h else 100000
                rough[b, h, 0] = rough[b, h, 1]
    for these in (lists, rough):
        t = Trees(p, lists=these, seed=K)
        for half in (True, False):
            for ws in ("full", None):
                check_tree(p, t, *run_tree(p, t, half, workspace=ws), half, SCALE, (S, K, half, ws))


@pytest.mark.parametrize("S", [8, 16, 32, 64])
def test_tree_many_rows_listed_pages(S):
    """Row tiles of 256 rows over lists that do not fit the small kernel, holes and missing pages among them."""
    rng = np.random.default_rng(S)
    p = Packed([5000, 70, 4100], [50, 33, 60], heads=16, kv_heads=2, S=S, seed=S)
    K = 2600 // S
    lists = rng.integers(-3, 5100 // S, (3, 2, K))
    t = Trees(p, lists=lists, seed=1)
    for half in (True, False):
        for ws in ("full", None):
            check_tree(p, t, *run_tree(p, t, half, workspace=ws), half, SCALE, (S, half, ws))


def test_tree_of_more_sequences_than_lanes():
    """Splits planned over three groups of 64 sequences, one of them long."""
    rng = np.random.default_rng(9)
    new = [int(x) for x in rng.integers(0, 9, 140)]
    lens = [int(x) for x in rng.integers(0, 200, 140)]
    lens[100] = 20000
    for room in ROOMS:
        p = Packed(lens, new, heads=2, kv_heads=1, seed=9, room=room)
        t = Trees(p)
        check_tree(p, t, *run_tree(p, t, True), True, SCALE, room)


def test_smaller_workspaces():
    """Any size is used as far as it goes; nothing is written behind it."""
    p = Packed([6000, 3500], [3, 2], heads=8, kv_heads=2, seed=4)
    t = Trees(p)
    many = Packed([6000, 3500], [60, 100], heads=8, kv_heads=2, seed=4)
    for x, call in ((p, "tree"), (p, "prompt"), (many, "prompt")):
        full = Q.quest_tokens_workspace_bytes(x.cache, x.total)
        for size in (16, 1 << 20, 5 << 20, full // 2, full):
            ws = torch.full((size // 4 + 64,), 5.0, device=x.dev)
            out, lse = x.results(False)
            if call == "tree":
                Q.quest_tree_attention(x.cache, x.q, x.k_new, x.v_new, x.cu, t.mask, SCALE, out, lse=lse, workspace=ws[:size // 4])
                check_tree(x, t, out, lse, False, SCALE, size)
            else:
                Q.quest_prompt_attention(x.cache, x.q, x.cu, SCALE, out, lse=lse, workspace=ws[:size // 4])
                check_prompt(x, out, lse, False, SCALE, size)
            assert bool((ws[size // 4:] == 5).all())


@pytest.mark.parametrize("scale", [-SCALE, 0.0, 1.0])
def test_tree_scales(scale):
    p = Packed([300], [17], heads=4, kv_heads=2, seed=8)
    t = Trees(p)
    for half in (True, False):
        check_tree(p, t, *run_tree(p, t, half, scale), half, scale, scale)


def test_without_lse():
    for new in (3, 80):
        p = Packed([2000, 9], [new, 9], heads=6, kv_heads=2, seed=new, room=4096)
        t = Trees(p)
        for ws in (p.workspace(), None):
            for with_lse in (True, False):
                out, lse = p.results(True)
                Q.quest_prompt_attention(p.cache, p.q, p.cu, SCALE, out, lse=lse if with_lse else None, workspace=ws)
                tree, tree_lse = p.results(True)
                Q.quest_tree_attention(p.cache, p.q, p.k_new, p.v_new, p.cu, t.mask, SCALE, tree, workspace=ws,
                                       lse=tree_lse if with_lse else None)
                if with_lse:
                    want = out, tree
                else:
                    assert torch.equal(out, want[0]) and torch.equal(tree, want[1])
                    assert bool((lse == 77).all()) and bool((tree_lse == 77).all())


@pytest.mark.parametrize("room", ROOMS)
def test_more_query_heads_than_a_row_tile(room):
    p = Packed([70, 900], [3, 2], heads=600, kv_heads=2, seed=1, room=room)
    t = Trees(p)
    check_prompt(p, *run_prompt(p, True), True, SCALE, room)
    check_tree(p, t, *run_tree(p, t, False), False, SCALE, room)


@pytest.mark.parametrize("room", ROOMS)
def test_largest_values(room):
    """Values at fp16's largest: their mean is that, whatever the weights' roundings, in one piece and in splits."""
    p = Packed([2500, 300], [20, 300], heads=8, kv_heads=2, seed=11, room=room)
    p.v_pool[...] = torch.where(p.v_pool.isnan(), p.v_pool, 65504.0)
    p.v_new[:320] = 65504.0
    t = Trees(p)
    for ws in ("full", None):
        for out, _ in (run_prompt(p, True, workspace=ws), run_tree(p, t, True, workspace=ws)):
            assert bool(((out[:320].float() - 65504).abs() <= 65504 * 2.0 ** -10).all())    # finite, within a step and a half
        for out, _ in (run_prompt(p, False, workspace=ws), run_tree(p, t, False, workspace=ws)):
            assert bool(((out[:320] - 65504).abs() <= 65504 * 2.0 ** -18).all())


@pytest.mark.parametrize("half", [True, False])
@pytest.mark.parametrize("n,ctx", [(7, 900), (300, 900)])
def test_largest_logits(n, ctx, half):
    """Queries and keys near fp16's largest: logits of 1e11 and gaps between them of 1e9, far beyond what the sums of
    128 channels round (2^-24 * 128 of 6e11, 5e6).  Each row's weight is on one key: the visible one of the largest factor."""
    p = Packed([ctx + n], [n], heads=4, kv_heads=2, seed=n)
    total = ctx + n
    sign = (torch.rand(2, D, device=p.dev) < 0.5).half() * 2 - 1
    order = torch.argsort(torch.rand(total, device=p.dev))
    factor = (30000 + 25 * order.float()).half()           # fp16 has steps of 16 and 32 there: runs of equal keys
    t = torch.arange(total, device=p.dev)
    phys = p.table[0].long()[t // p.S]
    p.k_pool[phys, :, t % p.S] = factor[:, None, None] * sign
    p.q[:n] = (60000 * sign.repeat_interleave(2, 0))[None].half()
    p.v_pool[phys, :, t % p.S] = factor[:, None, None] / 30000   # equal keys, equal values
    for row in run_prompt(p, half, scale=1.0), run_prompt(p, half, scale=1.0, workspace=None):
        out, lse = row
        visible = torch.cummax(factor.float(), 0).values[ctx:]
        assert bool((out[:n].float() == (visible.half() / 30000).float()[:, None, None]).all()), float(out[:n].max())
        want = visible.double() * 60000 * 128
        assert bool(((lse[:n].double() - want[:, None]).abs() <= 2.0 ** -16 * want[:, None]).all())
    p.k_new[:n] = factor[ctx:, None, None] * sign
    p.v_new[:n] = factor[ctx:, None, None] / 30000
    p.seq_lens.fill_(ctx)
    trees = Trees(p, kind=lambda rng, n, words: np.tril(np.ones((n, n), bool)))
    out, lse = run_tree(p, trees, half, scale=1.0)
    assert bool((out[:n].float() == (visible.half() / 30000).float()[:, None, None]).all())


@pytest.mark.parametrize("room", ROOMS)
def test_nan_queries(room):
    """A query that is not a number spoils its own row, sum and all, and no other."""
    p = Packed([2500, 300], [20, 300], heads=8, kv_heads=2, seed=12, room=room)
    t = Trees(p)
    runs = [lambda half=half, ws=ws, run=run: run(half, ws) for half in (True, False) for ws in ("full", None)
            for run in (lambda half, ws: run_prompt(p, half, workspace=ws), lambda half, ws: run_tree(p, t, half, workspace=ws))]
    before = [run() for run in runs]
    bad = torch.zeros(p.total, 8, dtype=torch.bool, device=p.dev)
    for row, h in ((3, 1), (19, 7), (20, 0), (250, 5)):
        bad[row, h] = True
    p.q[bad, 17] = math.nan
    for run, (out0, lse0) in zip(runs, before):
        out, lse = run()
        assert bool(out[bad].isnan().all()) and bool(lse[bad].isnan().all())
        assert torch.equal(out[~bad], out0[~bad]) and torch.equal(lse[~bad], lse0[~bad])


# ---- insertion

def one_by_one(p, past, rows):
    """What calls of quest_append_meta leave: the cache and the metadata, token after token."""
    k_pool, v_pool, meta, lens = p.k_pool.clone(), p.v_pool.clone(), p.meta.clone(), torch.zeros_like(p.seq_lens)
    for b in range(p.B):
        one = Q.Cache(k_pool, v_pool, meta, p.table[b:b + 1], lens[b:b + 1], num_heads=p.H)
        for i in range(p.new[b]):
            row = int(p.cu_np[b]) + i
            row = row if rows is None else int(rows[row])
            lens[b] = past[b] + i + 1
            Q.quest_append_meta(one, p.k_new[row].contiguous(), p.v_new[row].contiguous(), True)
    torch.cuda.synchronize()
    return k_pool, v_pool, meta


def same_bits(a, b):
    return torch.equal(a.view(torch.int16), b.view(torch.int16))


@pytest.mark.parametrize("S", [8, 16, 32, 64])
@pytest.mark.parametrize("stride", [0, 24])
def test_append_like_one_by_one(S, stride):
    new = [1, 0, 2 * S, 3 * S + 1, S - 1, 5, 1, 70]
    past = [0, 13, 0, S - 1, 1, S + S // 2, 2 * S, 3]
    p = Packed([n + m for n, m in zip(new, past)], new, heads=6, kv_heads=3, S=S, seed=S, stride=stride)
    p.k_new[::5, :, ::3] = 0.0
    p.k_new[1::5, :, ::3] = -0.0
    p.seq_lens.copy_(torch.tensor(past))
    p.seq_lens.clamp_(min=1)
    Q.quest_build_meta(p.cache)                    # entries of the tokens before (others are overwritten or not read)
    p.seq_lens.copy_(torch.tensor(p.lens))
    rng = np.random.default_rng(S)
    for rows in (None, rng.permutation(p.total - 3), rng.integers(0, p.total - 3, p.total - 3)):
        want = one_by_one(p, past, rows)
        keep = [x.clone() for x in (p.k_pool, p.v_pool, p.meta)]
        dev_rows = None if rows is None else torch.from_numpy(np.concatenate([rows, [-1] * 3]).astype(np.int32)).to(p.dev)
        Q.quest_append_tokens(p.cache, p.k_new, p.v_new, p.cu, rows=dev_rows)
        torch.cuda.synchronize()
        for got, w, name in zip((p.k_pool, p.v_pool, p.meta), want, ("k", "v", "meta")):
            assert same_bits(got, w), (S, name, rows is None)
        for x, y in zip((p.k_pool, p.v_pool, p.meta), keep):
            x.copy_(y)


def test_append_prompts_like_build():
    """A batch of more sequences than a wave has lanes; the metadata of whole prompts is what quest_build_meta gives."""
    new = [int(x) for x in np.random.default_rng(1).integers(1, 90, 100)]
    p = Packed(new, new, heads=2, kv_heads=2, seed=1, cached=False)
    Q.quest_append_tokens(p.cache, p.k_new, p.v_new, p.cu)
    got = p.meta.clone()
    p.meta.zero_()
    Q.quest_build_meta(p.cache)
    torch.cuda.synchronize()
    assert same_bits(got, p.meta)
    for b in range(p.B):
        k, v = p.cached(b, 1)
        assert torch.equal(k, p.k_new[p.rows(b), 1].double()) and torch.equal(v, p.v_new[p.rows(b), 1].double())
    used = torch.zeros(p.k_pool.shape[0], dtype=torch.bool, device=p.dev)
    for b in range(p.B):
        used[p.table[b, :-(-new[b] // p.S)].long()] = True
    assert bool(p.k_pool[~used].isnan().all()) and bool(p.v_pool[~used].isnan().all())
