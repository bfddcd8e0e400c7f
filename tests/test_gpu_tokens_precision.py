"""How exact attention of prompts and of drafted tokens is: fp16 outputs of few rows are the fp32 result, rounded once."""
import math

import pytest
import torch

from paper_2406_10774_amd import binding as Q
from packed_util import D, Packed, Trees, attention64

pytestmark = pytest.mark.gpu
SCALE = 1 / math.sqrt(D)


def run(p, t, half, workspace=True):
    out, lse = p.results(half)
    ws = p.workspace() if workspace else None
    if t is None:
        Q.quest_prompt_attention(p.cache, p.q, p.cu, SCALE, out, lse=lse, workspace=ws)
    else:
        Q.quest_tree_attention(p.cache, p.q, p.k_new, p.v_new, p.cu, t.mask, SCALE, out, lse=lse, workspace=ws)
    torch.cuda.synchronize()
    return out, lse


def rounded_once(got, want, what):
    """The fp32 limit (eight times the square root of the number of 2^-24 roundings of 128-channel sums, exp2 and n tokens, of
    the sum of the weighted values' sizes), and half a step of fp16 at the result with that error: 2^-11 of it, 2^-25 at
    least."""
    o, _, weight, size, n = want
    limit = 8 * (math.sqrt(D) * 2.0 ** -24 * size + 2.0 ** -21 + n.double().sqrt() * 2.0 ** -24)
    bound = limit[:, None] * weight * (1 + 2.0 ** -11) + 2.0 ** -11 * o.abs() + 2.0 ** -25
    off = (got.double() - o).abs()
    assert bool((off <= bound).all()), (what, float((off / bound).max()), float(off.max()))


@pytest.mark.parametrize("room", [0, 1 << 16])
@pytest.mark.parametrize("new,past", [([1, 1], [900, 5000]), ([1], [0]), ([13], [0]), ([16, 3], [40, 2500]), ([5], [9000])])
def test_few_rows(new, past, room):
    """At most 64 rows (new tokens times query heads of a KV head) a sequence on average."""
    p = Packed([n + m for n, m in zip(new, past)], new, heads=8, kv_heads=2, seed=sum(new), room=room)
    trees = Packed(past, new, heads=8, kv_heads=2, seed=sum(new), room=room)
    t = Trees(trees)
    for ws in (True, False):
        out, lse = run(p, None, True, ws)
        single = run(p, None, False, ws)
        assert torch.equal(lse, single[1])
        drafts, _ = run(trees, t, True, ws)
        for b in range(p.B):
            at = p.rows(b)
            position = torch.arange(p.lens[b] - p.new[b], p.lens[b], device=p.dev)
            sees = torch.arange(p.lens[b], device=p.dev) <= position[:, None]
            seen = torch.cat([torch.ones(new[b], past[b], dtype=torch.bool, device=p.dev), torch.from_numpy(t.sees[b]).to(p.dev)], 1)
            for h in range(p.H):
                k, v = p.cached(b, h // p.G)
                rounded_once(out[at, h], attention64(p.q[at, h].double(), k, v, sees, SCALE), ("prompt", b, h, ws))
                k, v = trees.cached(b, h // p.G)
                k, v = torch.cat([k, trees.k_new[at, h // p.G].double()]), torch.cat([v, trees.v_new[at, h // p.G].double()])
                rounded_once(drafts[at, h], attention64(trees.q[at, h].double(), k, v, seen, SCALE), ("tree", b, h, ws))


def test_single_tokens_as_decode_steps():
    """One token a sequence, fp16 outputs: as exact as the decode call's over all pages."""
    p = Packed([700, 33, 4000], [1, 1, 1], heads=8, kv_heads=2, seed=3, spare_rows=0)
    out, _ = run(p, None, True)
    step = torch.empty_like(out)
    ws = torch.zeros(Q.quest_workspace_bytes(p.cache, 1) // 4, device=p.dev)
    Q.quest_sparse_decode(p.cache, p.q.contiguous(), None, 0, SCALE, step, workspace=ws)
    torch.cuda.synchronize()
    for b in range(p.B):
        sees = torch.ones(1, p.lens[b], dtype=torch.bool, device=p.dev)
        for h in range(p.H):
            want = attention64(p.q[p.rows(b), h].double(), *p.cached(b, h // p.G), sees, SCALE)
            rounded_once(step[p.rows(b), h], want, ("decode", b, h))
            rounded_once(out[p.rows(b), h], want, ("prompt", b, h))


@pytest.mark.parametrize("half", [True, False])
@pytest.mark.parametrize("new,past,heads,kv_heads,room", [([700], [0], 40, 40, 0), ([300], [1000], 8, 2, 1 << 16),
                                                          ([90, 400], [1300, 10], 8, 2, 1 << 16)])
def test_equal_values_come_back(new, past, heads, kv_heads, room, half):
    """Many rows, in one piece and in splits, over tokens that all have the same value: that value, whatever the roundings of the
    weights.  fp32: off by at most the roundings of two sums over n tokens (and a few more), 2.4 n 2^-24; below half a step of
    fp16, 2^-12 of the value at least, so that fp16 outputs are the value."""
    data = dict(heads=heads, kv_heads=kv_heads, seed=new[0], room=room, spread=2.0)
    p, drafts = Packed([n + m for n, m in zip(new, past)], new, **data), Packed(past, new, **data)
    value = torch.randn(D, device=p.dev).half()
    for x in (p, drafts):
        x.v_pool[...] = torch.where(x.v_pool.isnan(), x.v_pool, value)
        x.v_new[:sum(new)] = value
    t = Trees(drafts)
    limit = 2.4 * max(p.lens) * 2.0 ** -24
    assert limit < 2.0 ** -12
    for ws in (True, False):
        for x, tree in ((p, None), (drafts, t)):
            off = (run(x, tree, half, ws)[0][:sum(new)].double() - value.double()).abs() / value.double().abs()
            assert bool((off <= (0 if half else limit)).all()), float(off.max())


def test_equal_values_under_small_weights():
    """One key of weight 1 and 8000 of 2^-21.5, which are below fp16's normal numbers: left out of only one of the two sums they would be
    8000 * 2^-21.5 of the result, 2.7e-3.  The limit as above, and half a step."""
    n, past = 300, 8000
    p = Packed([past + n], [n], heads=8, kv_heads=2, seed=5, room=1 << 16)
    p.k_pool[...] = torch.where(p.k_pool.isnan(), p.k_pool, 0.0)
    p.k_pool[p.table[0, 0].long(), :, 0, 0] = 1.0
    p.q[:n] = 0.0
    p.q[:n, :, 0] = 21.5 * math.log(2)
    value = torch.randn(D, device=p.dev).half()
    p.v_pool[...] = torch.where(p.v_pool.isnan(), p.v_pool, value)
    limit = 2.4 * (past + n) * 2.0 ** -24 + 2.0 ** -11
    for ws in (p.workspace(), None):
        out, lse = p.results(True)
        Q.quest_prompt_attention(p.cache, p.q, p.cu, 1.0, out, lse=lse, workspace=ws)
        off = (out[:n].double() - value.double()).abs() / value.double().abs()
        assert bool((off <= limit).all()), float(off.max())
        want = [math.log(math.exp(float(p.q[0, 0, 0])) + past + i) for i in range(n)]
        off = (lse[:n].double() - torch.tensor(want, device=p.dev, dtype=torch.float64)[:, None]).abs()
        assert bool((off <= 2.4 * (past + n) * 2.0 ** -24 * want[0]).all()), float(off.max())


@pytest.mark.parametrize("n,room", [(3, 0), (300, 1 << 16)])
@pytest.mark.parametrize("bits", [14, 20, 25, 31, 36, 38, 41])
def test_small_weights(bits, n, room):
    """One key of weight 1 and value 0, 4000 of 2^-bits with values around 1: what they add up to.  With fp32 outputs a weight is off by
    2^-22 of itself or by 2^-39; with fp16 outputs of many rows by 2^-11 or 2^-32 (the base is put 2^-7 of the largest weight and
    fp16's smallest step, rounded to half of it, is 2^-24).  Beside that the fp32 limits."""
    past = 4000
    p = Packed([past + n], [n], heads=8, kv_heads=2, seed=bits, room=room)
    p.k_pool[...] = torch.where(p.k_pool.isnan(), p.k_pool, 0.0)
    p.k_pool[p.table[0, 0].long(), :, 0, 0] = 1.0
    p.q[:n] = 0.0
    p.q[:n, :, 0] = bits * math.log(2)
    p.v_pool[...] = torch.where(p.v_pool.isnan(), p.v_pool, p.v_pool.abs().clamp(max=3.0))
    p.v_pool[p.table[0, 0].long(), :, 0] = 0.0
    sees = torch.arange(past + n, device=p.dev) <= torch.arange(past, past + n, device=p.dev)[:, None]
    for ws in (p.workspace(), None):
        for half in (True, False):
            out, lse = p.results(half)
            Q.quest_prompt_attention(p.cache, p.q, p.cu, 1.0, out, lse=lse, workspace=ws)
            for h in (0, 7):
                k, v = p.cached(0, h // p.G)
                o, l, weight, size, seen = attention64(p.q[:n, h].double(), k, v, sees, 1.0)
                fp32 = 8 * (math.sqrt(D) * 2.0 ** -24 * size + 2.0 ** -21 + seen.double().sqrt() * 2.0 ** -24)
                few = not half or n < 64
                bound = (fp32[:, None] + (2.0 ** -22 if few else 2.0 ** -11)) * weight + seen[:, None] * 3.0 * 2.0 ** (-39 if few else -32)
                if half:
                    bound = bound + 2.0 ** -11 * o.abs() + 2.0 ** -25
                off = (out[:n, h].double() - o).abs()
                assert bool((off <= bound).all()), (half, float((off / bound).max()))
                assert bool(((lse[:n, h].double() - l).abs() <= fp32 * l.abs().clamp(min=1.0)).all())
