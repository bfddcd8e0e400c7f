"""Many tokens a sequence, with lengths past the end of the page-table row.  No caller may pass them; insertion stores the tokens
that the row has room for and nothing elsewhere."""
import numpy as np
import pytest
import torch

from paper_2406_10774_amd import binding as Q
from packed_util import D, Packed

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
