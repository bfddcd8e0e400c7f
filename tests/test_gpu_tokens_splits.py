"""Into how many splits the tokens of a long sequence are cut, whatever sequences it is batched with.  A split leaves 130 floats
for each of its rows in the workspace (the outputs, a reference and a sum), counted in one that was filled with NaN."""
import math

import numpy as np
import pytest
import torch

from paper_2406_10774_amd import binding as Q
from packed_util import D, Packed, Trees, check_prompt, check_tree

pytestmark = pytest.mark.gpu
SCALE = 1 / math.sqrt(D)
ROWS = [("alone", []), ("among short ones", [(40, 4)] * 9), ("among empty ones", [(300, 0)] * 9), ("more than lanes", [(20, 1)] * 70 + [(9, 0)] * 60)]


@pytest.mark.parametrize("others", [r[1] for r in ROWS], ids=[r[0] for r in ROWS])
@pytest.mark.parametrize("at", [0, -1])
@pytest.mark.parametrize("new", [4, 300])
def test_splits_of_a_long_sequence(others, at, new):
    """At most 95 (a quotient of at least 64 tiles, rounded down, is up to 1.5 times too small)."""
    past = 60000
    lens, news = [n for n, _ in others], [n for _, n in others]
    lens.insert(at % (len(lens) + 1), past)
    news.insert(at % (len(news) + 1), new)
    p = Packed([n + m for n, m in zip(lens, news)], news, heads=1, kv_heads=1, seed=new)
    d = Packed(lens, news, heads=1, kv_heads=1, seed=new)
    t = Trees(d)
    for x, call in ((p, "prompt"), (d, "tree")):
        out, lse = x.results(False)
        ws = x.workspace()
        if call == "prompt":
            Q.quest_prompt_attention(x.cache, x.q, x.cu, SCALE, out, lse=lse, workspace=ws)
            check_prompt(x, out, lse, False, SCALE, call)
        else:
            Q.quest_tree_attention(x.cache, x.q, x.k_new, x.v_new, x.cu, t.mask, SCALE, out, lse=lse, workspace=ws)
            check_tree(x, t, out, lse, False, SCALE, call)
        splits = int(torch.isfinite(ws).sum()) / (D + 2) / new
        assert 2 <= splits <= 95.5, (call, splits)


@pytest.mark.parametrize("seed", range(20))
def test_a_larger_workspace_changes_nothing(seed):
    """Calls use all they can in a workspace of the size that the library names for their tokens, or more."""
    rng = np.random.default_rng(seed)
    B, kv_heads = int(rng.integers(1, 12)), int(rng.choice([1, 2, 8, 40]))
    heads = kv_heads * int(rng.choice([1, 4]))
    most = int(rng.choice([3, 30, 300]))
    new = [int(x) for x in rng.integers(0, most + 1, B)]
    past = [int(rng.choice([0, 500, rng.integers(0, 6000)])) for _ in range(B)]
    room = int(rng.choice([0, 1 << 14]))
    shape = dict(heads=heads, kv_heads=kv_heads, seed=seed, room=room, spare_rows=int(rng.integers(0, 9)))
    p, d = Packed([n + m for n, m in zip(new, past)], new, **shape), Packed(past, new, **shape)
    t = Trees(d)
    for x, call in ((p, "prompt"), (d, "tree")):
        exact = Q.quest_tokens_workspace_bytes(x.cache, x.total)
        results = []
        for size in (exact, 200 << 20):
            out, lse = x.results(True)
            ws = torch.full((max(size, 16) // 4,), math.nan, device=x.dev)
            if call == "prompt":
                Q.quest_prompt_attention(x.cache, x.q, x.cu, SCALE, out, lse=lse, workspace=ws)
            else:
                Q.quest_tree_attention(x.cache, x.q, x.k_new, x.v_new, x.cu, t.mask, SCALE, out, lse=lse, workspace=ws)
            results.append((out, lse))
        torch.cuda.synchronize()
        assert torch.equal(results[0][0], results[1][0]) and torch.equal(results[0][1], results[1][1]), (call, B, heads, kv_heads, new, past)
