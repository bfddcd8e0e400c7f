"""One workspace for calls on an fp16 cache and on one of 8 bits of the same shape: where each keeps what."""
import ctypes
import math

import pytest
import torch

from paper_2406_10774_amd import binding as Q

P = 0x1000
D = 128
COUNTER = 256                                                      # bytes of an arrival counter's place


def sizes(batch, heads, kv_heads, pages, S=8):
    """Bytes of quest_workspace_bytes for pages of 8 bits, and the most that quest_topk takes for candidates."""
    lib, out = Q.load(), ctypes.c_size_t(0)
    c = Q.quest_cache(batch=batch, num_heads=heads, head_dim=D, page_size=S, max_pages_per_seq=pages, flags=Q.QUEST_FLAG_E4M3_PAGES,
                      num_phys_pages=pages, k_pool=P, v_pool=P, meta=P, page_table=P, seq_lens=P, num_kv_heads=kv_heads, scales=P)
    assert lib.quest_workspace_bytes(ctypes.byref(c), 1, ctypes.byref(out)) == 0
    whole, candidates = out.value, 0
    for k_pages in [1 << i for i in range(13)]:
        assert lib.quest_topk_workspace_bytes(ctypes.byref(c), k_pages, ctypes.byref(out)) == 0
        candidates = max(candidates, out.value)
    return whole, candidates


@pytest.mark.parametrize("batch,heads,kv_heads", [(1, 32, 32), (16, 32, 32), (16, 40, 40), (27, 19, 19), (65, 8, 8), (65, 32, 8),
                                                  (300, 18, 1)])
@pytest.mark.parametrize("pages", [16384, 20001, 40000])
def test_candidates_lie_behind_the_counters(batch, heads, kv_heads, pages):
    """Also where the attention over pages of 8 bits has no partial results: the counters there are the fp16 calls'."""
    whole, candidates = sizes(batch, heads, kv_heads, pages)
    assert candidates > 0 and whole >= candidates + batch * heads * COUNTER


@pytest.mark.gpu
@pytest.mark.parametrize("batch,heads,kv_heads", [(27, 19, 19), (16, 40, 40), (65, 16, 8), (2, 4, 2)])
def test_calls_take_turns(batch, heads, kv_heads):
    """Selection with candidates over pages of 8 bits, then a dense call over fp16 pages, on one buffer: each as on a buffer of its own."""
    dev, S, pages, N, K = "cuda:0", 8, 16384, 50, 300
    gen = torch.Generator(device=dev)
    gen.manual_seed(batch)

    def normal(*shape):
        return torch.randn(*shape, device=dev, generator=gen)

    table = torch.randint(N, (batch, pages), device=dev, dtype=torch.int32, generator=gen)
    lens = torch.randint(1, 5000, (batch,), device=dev, dtype=torch.int32, generator=gen)
    lens[1] = pages * S - 3
    meta = torch.zeros(kv_heads, N, 2, D, device=dev, dtype=torch.float16)
    halves = [normal(N, kv_heads, S, D).half() for _ in range(2)]
    eights = [normal(N, kv_heads, S, D).to(torch.float8_e4m3fn) for _ in range(2)]
    half = Q.Cache(*halves, meta, table, lens, num_heads=heads)
    eight = Q.Cache(*eights, meta, table, lens, num_heads=heads, scales=torch.ones(N, kv_heads, 2, device=dev))
    q, scores = normal(batch, heads, D).half(), normal(batch, kv_heads, pages)
    size = max(Q.quest_workspace_bytes(c, K) for c in (half, eight))
    assert Q.quest_topk_workspace_bytes(eight, K) > 0

    def fresh():
        return torch.zeros(size // 4, device=dev)

    def select(ws):
        idx = torch.full((batch, kv_heads, K), -7, device=dev, dtype=torch.int32)
        out, lse = torch.full((batch, heads, D), 77.0, device=dev), torch.full((batch, heads), 77.0, device=dev)
        Q.quest_select_decode(eight, q, scores, K, 1 / math.sqrt(D), idx, out, lse=lse, workspace=ws)
        return idx, out, lse

    def dense(cache, ws):
        out, lse = torch.full((batch, heads, D), 77.0, device=dev), torch.full((batch, heads), 77.0, device=dev)
        Q.quest_sparse_decode(cache, q, None, 0, 1 / math.sqrt(D), out, lse=lse, workspace=ws)
        return out, lse

    want = [select(fresh()), dense(half, fresh()), dense(eight, fresh())]
    lists = torch.full_like(want[0][0], -7)
    Q.quest_topk(eight, scores, K, lists)
    assert torch.equal(want[0][0], lists)
    ws = fresh()
    for _ in range(3):
        for got, alone in zip((select(ws), dense(half, ws), dense(eight, ws)), want):
            assert all(torch.equal(a, b) for a, b in zip(got, alone))
        assert not bool(ws.view(torch.int32)[:batch * heads * COUNTER // 4].any())
