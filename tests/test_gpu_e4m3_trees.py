"""Attention of drafted tokens over pages of 8 bits on the GPU, against 64 bits over the numbers that the pages stand for; the drafted
nodes' own keys and values are fp16."""
import math

import numpy as np
import pytest
import torch

from paper_2406_10774_amd import binding as Q
from e4m3_util import Packed8
from packed_util import Trees, check_tree
from test_gpu_tokens import anything, everything, nothing, run_tree

pytestmark = pytest.mark.gpu
SCALE = 1 / math.sqrt(128)
ROOMS = [0, 1 << 17]


@pytest.mark.parametrize("half", [True, False])
@pytest.mark.parametrize("room", ROOMS)
@pytest.mark.parametrize("n,ctx", [(1, 0), (1, 1), (1, 700), (5, 64), (8, 1000), (31, 65), (33, 129), (64, 300), (65, 300), (130, 77),
                                   (140, 3000), (3, 3000), (300, 200)])
def test_trees(n, ctx, room, half):
    p = Packed8([ctx, ctx // 2], [n, max(1, n // 3)], heads=4, kv_heads=2, seed=n + ctx, stride=16, room=room)
    t = Trees(p, seed=n)
    for ws in ("full", None):
        check_tree(p, t, *run_tree(p, t, half, workspace=ws), half, SCALE, (n, ctx, ws))


@pytest.mark.parametrize("room", ROOMS)
@pytest.mark.parametrize("heads,kv_heads,S", [(1, 1, 16), (8, 1, 8), (6, 2, 32), (64, 2, 64), (20, 4, 16), (24, 1, 8), (32, 2, 32)])
def test_groups_and_pages(heads, kv_heads, S, room):
    p = Packed8([900, 0, 64, 1203], [12, 3, 0, 40], heads=heads, kv_heads=kv_heads, S=S, seed=S, room=room)
    t = Trees(p, seed=S, words=2)
    for half in (True, False):
        check_tree(p, t, *run_tree(p, t, half), half, SCALE, (heads, kv_heads, S, half))


@pytest.mark.parametrize("kind", [nothing, everything, anything])
def test_masks(kind):
    """Also rows that see no drafted node, and, without a context, nothing at all: out 0, lse -inf."""
    for room in ROOMS:
        p = Packed8([0, 50, 128], [20, 70, 64], heads=4, kv_heads=2, seed=3, room=room)
        t = Trees(p, kind=kind, words=3)
        for half in (True, False):
            for ws in ("full", None):
                out, lse = run_tree(p, t, half, workspace=ws)
                check_tree(p, t, out, lse, half, SCALE, (kind.__name__, half, room))
                if kind is nothing:
                    assert bool((out[:20] == 0).all()) and bool((lse[:20] == -math.inf).all())


@pytest.mark.parametrize("S", [8, 16, 32, 64])
@pytest.mark.parametrize("K", [1, 3, 17, 40])
def test_listed_pages(S, K):
    rng = np.random.default_rng(S * K)
    p = Packed8([1500, 30, 777], [9, 20, 1], heads=8, kv_heads=2, S=S, seed=K)
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
def test_many_rows_listed_pages(S):
    """Row tiles of 256 rows over lists that do not fit the small kernel, holes and missing pages among them."""
    rng = np.random.default_rng(S)
    p = Packed8([5000, 70, 4100], [50, 33, 60], heads=16, kv_heads=2, S=S, seed=S)
    t = Trees(p, lists=rng.integers(-3, 5100 // S, (3, 2, 2600 // S)), seed=1)
    for half in (True, False):
        for ws in ("full", None):
            check_tree(p, t, *run_tree(p, t, half, workspace=ws), half, SCALE, (S, half, ws))


@pytest.mark.parametrize("seed", range(12))
def test_random_trees(seed):
    """Both kernels, in one piece and in splits that end among cached tokens or among nodes."""
    rng = np.random.default_rng(seed)
    B, S, kv_heads = int(rng.integers(1, 5)), int(rng.choice([8, 16, 32, 64])), int(rng.integers(1, 4))
    heads = kv_heads * int(rng.choice([1, 2, 4, 7]))
    new = [int(rng.integers(1, 260)) for _ in range(B)]
    lens = [int(rng.choice([0, rng.integers(0, 300), rng.integers(0, 6000)])) for _ in range(B)]
    p = Packed8(lens, new, heads=heads, kv_heads=kv_heads, S=S, seed=seed, room=ROOMS[seed % 2])
    t = Trees(p, seed=seed)
    half = seed % 3 > 0
    first = run_tree(p, t, half)
    check_tree(p, t, *first, half, SCALE, seed)
    again = run_tree(p, t, half)
    assert torch.equal(first[0], again[0]) and torch.equal(first[1], again[1])


def test_more_sequences_than_lanes():
    rng = np.random.default_rng(9)
    new = [int(x) for x in rng.integers(0, 9, 140)]
    lens = [int(x) for x in rng.integers(0, 200, 140)]
    lens[100] = 20000
    for room in ROOMS:
        p = Packed8(lens, new, heads=2, kv_heads=1, seed=9, room=room)
        t = Trees(p)
        check_tree(p, t, *run_tree(p, t, True), True, SCALE, room)


def test_rejected_nodes_leave_no_trace():
    """Drafts are checked, some are kept: what the cache held before the insertion is as it was."""
    p = Packed8([333, 1000], [6, 20], heads=8, kv_heads=2, seed=2, spare_rows=0)
    p.scales.nan_to_num_(1.0)
    t = Trees(p)
    before = [x.view(torch.uint8).clone() for x in (p.k_pool, p.v_pool, p.meta, p.scales)]
    out, lse = run_tree(p, t, True)
    check_tree(p, t, out, lse, True, SCALE)
    assert all(torch.equal(x, y.view(torch.uint8)) for x, y in zip(before, (p.k_pool, p.v_pool, p.meta, p.scales)))
