"""Rotation, insertion and attention over pages of 8 bits together, as a serving loop calls them; captured graphs and streams."""
import math

import numpy as np
import pytest
import torch

from paper_2406_10774_amd import binding as Q
from e4m3_util import Packed8, table_of, turned
from packed_util import D, check_prompt
from test_gpu_e4m3_attention import check_decode
from test_gpu_e4m3_insert import Oracle, pool8

pytestmark = pytest.mark.gpu
SCALE = 1 / math.sqrt(D)


@pytest.mark.parametrize("S,heads,kv_heads,half", [(16, 4, 4, False), (16, 16, 2, True), (8, 6, 2, False), (64, 8, 1, True)])
def test_serving_loop(S, heads, kv_heads, half):
    """Two prompts go in in two parts each, turned by their position, then decode steps over selected pages and over all.  Codes and
    scales against the definition, attention against 64 bits on the cache as it then is, selection as on an fp16 cache."""
    rng = np.random.default_rng(S)
    pages = 1200 // S
    N = 2 * pages + 1
    ids = rng.permutation(N)[:2 * pages].reshape(2, pages).astype(np.int32)
    base = Packed8([0, 0], [0, 0], heads=heads, kv_heads=kv_heads, S=S, seed=S, cached=False)
    base.table_np, base.table = ids, torch.from_numpy(ids).to(base.dev)
    base.__dict__.update(pool8(N, kv_heads, S))
    base.describe()
    half_k, half_v = (torch.zeros(N, kv_heads, S, D, device=base.dev, dtype=torch.float16) for _ in range(2))
    half_meta = torch.zeros_like(base.meta)
    halves = Q.Cache(half_k, half_v, half_meta, base.table, base.seq_lens, num_heads=heads)
    rotation = Q.Rotation(table_of(pages * S, 128))
    length, seed = [0, 0], 0

    def step(new):
        nonlocal seed
        seed += 1
        x = Packed8([0, 0], new, heads=heads, kv_heads=kv_heads, S=S, seed=seed, cached=False, spare_rows=0)
        for b in range(2):
            length[b] += new[b]
        for name in ("k_pool", "v_pool", "meta", "scales", "table", "table_np", "seq_lens", "cache"):
            setattr(x, name, getattr(base, name))
        x.lens = list(length)
        base.seq_lens.copy_(torch.tensor(length))
        o = Oracle(base)
        raw_q, raw_k = x.q.clone(), x.k_new.clone()
        q = torch.empty_like(raw_q)
        Q.quest_rotate_append_tokens(base.cache, rotation, raw_q, raw_k, x.v_new, x.cu, q)
        Q.quest_rotate_append_tokens(halves, rotation, raw_q, raw_k, x.v_new, x.cu, torch.empty_like(q))
        where = torch.cat([torch.arange(l - n, l) for l, n in zip(length, new)])
        x.k_new = turned(raw_k, rotation.table, where, False).to(base.dev)
        assert torch.equal(q.cpu(), turned(raw_q, rotation.table, where, False))
        x.q = q
        o.check(base, o.insert(x))
        assert torch.equal(base.meta.view(torch.int16), half_meta.view(torch.int16))
        return x

    for new in ([300, 411], [517, 90]):
        x = step(new)
        out, lse = x.results(half)
        Q.quest_prompt_attention(base.cache, x.q, x.cu, SCALE, out, lse=lse, workspace=x.workspace())
        check_prompt(x, out, lse, half, SCALE, new)

    K = 256 // S
    scores, scores16 = (torch.zeros(2, kv_heads, pages, device=base.dev) for _ in range(2))
    idx, idx16 = (torch.zeros(2, kv_heads, K, device=base.dev, dtype=torch.int32) for _ in range(2))
    ws = torch.zeros(Q.quest_step_workspace_bytes(base.cache, K) // 4, device=base.dev)
    for _ in range(5):
        x = step([1, 1])
        out, lse = x.results(half)
        Q.quest_decode_step(base.cache, None, None, False, x.q, K, SCALE, scores, idx, out, ws, lse=lse)
        check_decode(x, out, lse, half, idx)
        Q.quest_estimate(halves, x.q, scores16)
        Q.quest_topk(halves, scores16, K, idx16)
        assert torch.equal(idx, idx16)
        Q.quest_sparse_decode(base.cache, x.q, None, 0, SCALE, out, lse=lse, workspace=ws)
        check_decode(x, out, lse, half)
        o2, l2 = x.results(half)                                    # the same query as a prompt of one token
        Q.quest_prompt_attention(base.cache, x.q, x.cu, SCALE, o2, lse=l2, workspace=x.workspace())
        check_prompt(x, o2, l2, half, SCALE)


@pytest.mark.parametrize("heads,kv_heads", [(4, 4), (8, 2)])
def test_captured_step(heads, kv_heads):
    """A decode step with rotation, captured once and replayed while lengths, tokens and pages change; every replay against the eager
    calls, with eager work and synchronisations between."""
    S, pages = 16, 300
    eager, captured = (Packed8([4000, 900], [1, 1], heads=heads, kv_heads=kv_heads, S=S, seed=1, spare_rows=0, room=pages * S) for _ in range(2))
    for p in (eager, captured):
        p.scales.nan_to_num_(1.0)
    spare = eager.table_np[0, -1]
    rotation = Q.Rotation(table_of(pages * S, 128))
    K = 40
    buffers = []
    for p in (eager, captured):
        width = p.table.shape[1]
        buffers.append(dict(q=p.q.contiguous(), k=p.k_new.contiguous(), v=p.v_new.contiguous(), out=p.results(False)[0], lse=p.results(False)[1],
                            turned=torch.zeros_like(p.q.contiguous()), scores=torch.zeros(2, kv_heads, width, device=p.dev),
                            idx=torch.zeros(2, kv_heads, K, device=p.dev, dtype=torch.int32),
                            all=p.results(False)[0], part=p.results(False)[0],
                            ws=torch.zeros(Q.quest_step_workspace_bytes(p.cache, K) // 4, device=p.dev), tw=p.workspace()))

    def step(p, b):
        Q.quest_rotate_append_tokens(p.cache, rotation, b["q"], b["k"], b["v"], p.cu, b["turned"])
        Q.quest_decode_step(p.cache, None, None, False, b["turned"], K, SCALE, b["scores"], b["idx"], b["out"], b["ws"], lse=b["lse"])
        Q.quest_sparse_decode(p.cache, b["turned"], None, 0, SCALE, b["all"], workspace=b["ws"])
        Q.quest_prompt_attention(p.cache, b["turned"], p.cu, SCALE, b["part"], workspace=b["tw"])

    stream = torch.cuda.Stream()
    torch.cuda.synchronize()
    with torch.cuda.stream(stream):
        step(captured, buffers[1])                                  # (lengths as they are: the same again later changes nothing)
    stream.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph, stream=stream):
        step(captured, buffers[1])
    step(eager, buffers[0])
    gen = torch.Generator(device="cuda:0")
    gen.manual_seed(5)
    for replay in range(6):
        for name in ("q", "k", "v"):
            x = torch.randn(buffers[0][name].shape, device="cuda:0", generator=gen).half() * (1 + replay)
            for b in buffers:
                b[name].copy_(x)
        if replay:
            for p in (eager, captured):
                p.lens = [n + 1 for n in p.lens]
                p.seq_lens.copy_(torch.tensor(p.lens))
                for b in range(2):                                  # (a page of its own for a sequence that grows into one)
                    if p.lens[b] % S == 1:
                        p.table[b, p.lens[b] // S] = int(spare) if b == 0 else int(p.table_np[1, 0])
        graph.replay()
        step(eager, buffers[0])
        torch.cuda.synchronize()
        for name in ("turned", "scores", "idx", "out", "lse", "all", "part"):
            a, b = (x[name] for x in buffers)
            if name == "scores":
                a, b = a[:, :, :50], b[:, :, :50]
            assert torch.equal(a, b), (replay, name)
        assert torch.equal(eager.k_pool.view(torch.uint8), captured.k_pool.view(torch.uint8)) and torch.equal(eager.scales, captured.scales)


def test_streams_and_two_workspaces():
    """Two calls at once on streams of their own, each with its workspace."""
    a, b = (Packed8([9000, 4000], [1, 1], heads=8, kv_heads=k, seed=k, spare_rows=0) for k in (8, 2))
    want = []
    for p in (a, b):
        out, lse = p.results(True)
        ws = torch.zeros(Q.quest_workspace_bytes(p.cache, 0) // 4, device=p.dev)
        Q.quest_sparse_decode(p.cache, p.q.contiguous(), None, 0, SCALE, out, lse=lse, workspace=ws)
        check_decode(p, out, lse, True)
        want.append((out, lse))
    streams = [torch.cuda.Stream(), torch.cuda.Stream()]
    results = [p.results(True) for p in (a, b)]
    spaces = [torch.zeros(Q.quest_workspace_bytes(p.cache, 0) // 4, device=p.dev) for p in (a, b)]
    queries = [p.q.contiguous() for p in (a, b)]
    torch.cuda.synchronize()
    for _ in range(10):
        for i, p in enumerate((a, b)):
            Q.quest_sparse_decode(p.cache, queries[i], None, 0, SCALE, results[i][0], lse=results[i][1], workspace=spaces[i],
                                  stream=streams[i].cuda_stream)
    torch.cuda.synchronize()
    for i in range(2):
        assert torch.equal(results[i][0], want[i][0]) and torch.equal(results[i][1], want[i][1])
