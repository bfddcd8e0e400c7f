"""Pages of 8 bits where calls leave the usual range: lengths that do not fit, unlike lengths in batches that are not shared out."""
import math

import numpy as np
import pytest
import torch

from paper_2406_10774_amd import binding as Q
from e4m3_util import Packed8, Pages, table_of
from packed_util import D, Packed, attention64, check

pytestmark = pytest.mark.gpu
SCALE = 1 / math.sqrt(D)


def bits(cache):
    """Everything a cache holds, as bytes."""
    held = [cache.k_pool, cache.v_pool, cache.meta] + ([] if cache.scales is None else [cache.scales])
    return [t.contiguous().view(torch.uint8).clone() for t in held]


def unfit(kind, S, kv_heads, heads):
    """Four sequences: one that fits; one shorter than its new tokens; one whose new tokens begin in the last page of its row, which
    holds tokens already, and go on behind it; one whose new tokens lie behind its row."""
    new, inside = [30, 20, S + 9, 9], S // 2
    p = kind([64, 20, 48, 48], new, heads=heads, kv_heads=kv_heads, S=S, seed=S)
    width = p.table.shape[1]
    spare = sorted(set(range(p.k_pool.shape[0])) - {int(x) for x in p.table_np.flatten()})
    p.table_np[2, -1] = spare[0]
    p.table.copy_(torch.from_numpy(p.table_np))
    x = torch.randn(kv_heads, S, D, device=p.dev).clamp(-3, 3)
    p.k_pool[spare[0]] = x.to(p.k_pool.dtype)
    p.v_pool[spare[0]] = (-x).to(p.v_pool.dtype)
    p.meta[:, spare[0], 0], p.meta[:, spare[0], 1] = -4.0, 0.25
    if kind is Packed8:
        p.scales[spare[0]] = 2.0 ** -9
    first = (width - 1) * S + inside                                # of sequence 2's new tokens
    p.seq_lens.copy_(torch.tensor([64, 19, first + new[2], (width + 2) * S], dtype=torch.int32))
    return p, spare[0], inside, first


@pytest.mark.parametrize("S", [8, 16, 32, 64])
@pytest.mark.parametrize("heads,kv_heads", [(2, 1), (96, 96)])
def test_insertion_of_lengths_that_do_not_fit(S, heads, kv_heads):
    """The tokens that have a place are inserted, with their page's scales and metadata; nothing else changes."""
    p, page, inside, _ = unfit(Packed8, S, kv_heads, heads)
    scales = p.scales.nan_to_num(1.0).cpu().numpy()
    pools = [Pages(pool.view(torch.uint8).cpu().numpy(), scales[..., i]) for i, pool in enumerate((p.k_pool, p.v_pool))]
    want_scales, meta = p.scales.clone(), p.meta.clone()
    places = [(int(p.table_np[0, t // S]), t % S, t - 34) for t in range(34, 64)]                     # page, slot, packed row
    places += [(page, inside + i, int(p.cu_np[2]) + i) for i in range(S - inside)]
    k, v = p.k_new.double().cpu().numpy(), p.v_new.double().cpu().numpy()
    for phys in sorted({at[0] for at in places}):
        slots = [at for at in places if at[0] == phys]
        rows = [at[2] for at in slots]
        for h in range(kv_heads):
            for pool, x, i in ((pools[0], k, 0), (pools[1], v, 1)):
                pool.insert(phys, h, slots[0][1], x[rows, h])
                want_scales[phys, h, i] = 2.0 ** int(pool.e[phys, h])
        keys = p.k_new[rows]
        lo, hi = keys.amin(0), keys.amax(0)
        opens = slots[0][1] == 0
        meta[:, phys, 0] = lo if opens else torch.minimum(meta[:, phys, 0], lo)
        meta[:, phys, 1] = hi if opens else torch.maximum(meta[:, phys, 1], hi)
    Q.quest_append_tokens(p.cache, p.k_new, p.v_new, p.cu)
    torch.cuda.synchronize()
    for pool, mine in zip((p.k_pool, p.v_pool), pools):
        assert np.array_equal(pool.view(torch.uint8).cpu().numpy(), mine.codes)
    assert torch.equal(p.scales.view(torch.int32), want_scales.view(torch.int32))
    assert torch.equal(p.meta.view(torch.int16), meta.view(torch.int16))


@pytest.mark.parametrize("S", [8, 16, 32, 64])
@pytest.mark.parametrize("kind", [Packed, Packed8])
def test_rotated_insertion_of_lengths_that_do_not_fit(S, kind):
    """As the rotation and then the insertion, bit for bit, whatever the lengths; and pages that none of them has a token for stay."""
    both, one = unfit(kind, S, 2, 4)[0], unfit(kind, S, 2, 4)[0]
    one.k_pool.copy_(both.k_pool), one.v_pool.copy_(both.v_pool)
    rotation = Q.Rotation(table_of(1000, 64), interleaved=S % 16 == 0)
    before, out, turned = bits(both.cache), torch.zeros(both.total, 4, D, device=both.dev, dtype=torch.float16), []
    Q.quest_rotate_append_tokens(both.cache, rotation, both.q.contiguous(), both.k_new.contiguous(), both.v_new.contiguous(), both.cu, out)
    for x in (one.q, one.k_new):
        turned.append(torch.zeros_like(x.contiguous()))
        Q.quest_rotate_tokens(one.cache, rotation, x.contiguous(), one.cu, turned[-1])
    Q.quest_append_tokens(one.cache, turned[1], one.v_new.contiguous(), one.cu)
    torch.cuda.synchronize()
    assert torch.equal(out.view(torch.int16), turned[0].view(torch.int16))
    after = bits(both.cache)
    for a, b in zip(after, bits(one.cache)):
        assert torch.equal(a, b)
    mine = {int(x) for x in both.table_np[0, 34 // S:-(-64 // S)]} | {int(both.table_np[2, -1])}
    others = [i for i in range(both.k_pool.shape[0]) if i not in mine]
    for i, (a, b) in enumerate(zip(after, before)):
        changed = (a != b).flatten(1).any(1) if i != 2 else (a != b).transpose(0, 1).flatten(1).any(1)
        assert not bool(changed[others].any()) and bool(changed[sorted(mine)].all() if i != 3 else True)


@pytest.mark.parametrize("batch,heads,kv_heads", [(18, 40, 40), (40, 40, 40), (65, 40, 40), (65, 8, 8), (100, 32, 8), (129, 18, 2)])
@pytest.mark.parametrize("longest,shortest,one", [(700, 650, None), (900, 1, 9000), (64, 64, None), (300, 0, 5000)])
def test_unlike_lengths_above_the_shares(batch, heads, kv_heads, longest, shortest, one):
    """More than 512 pairs of sequence and KV head (or eight query heads of one): each has a work-group, however long it is."""
    rng = np.random.default_rng(batch * heads + longest)
    lens = [int(rng.integers(shortest, longest + 1)) for _ in range(batch)]
    if one is not None:
        lens[batch // 2] = one
    p = Packed8(lens, [1] * batch, heads=heads, kv_heads=kv_heads, seed=longest, spare_rows=0)
    for half, ws in ((False, "full"), (True, None)):
        out, lse = p.results(half)
        workspace = torch.zeros(Q.quest_workspace_bytes(p.cache, 0) // 4, device=p.dev) if ws else None
        Q.quest_sparse_decode(p.cache, p.q.contiguous(), None, 0, SCALE, out, lse=lse, workspace=workspace)
        for b in sorted(set(range(0, batch, 9)) | {batch // 2, batch - 1}):
            for hk in range(kv_heads):
                k, v = p.cached(b, hk)
                at = slice(hk * p.G, (hk + 1) * p.G)
                sees = torch.ones(p.G, k.shape[0], dtype=torch.bool, device=p.dev)
                check(out[b, at], lse[b, at], attention64(p.q[b, at].double(), k, v, sees, SCALE), half, (b, hk))
        assert not bool((out == 77).any()) and not bool((lse == 77).any())
