"""Into how many splits the tokens of a long sequence are cut, whatever sequences it is batched with.  A split leaves 130 floats
for each of its rows in the workspace (the outputs, a reference and a sum), counted in one that was filled with NaN."""
import math

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
