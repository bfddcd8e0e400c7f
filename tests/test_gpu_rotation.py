"""Rotation of packed rows on the GPU, bit for bit against its definition, and together with insertion."""
import math

import numpy as np
import pytest
import torch

from paper_2406_10774_amd import binding as Q
from e4m3_util import Packed8, table_of, turned
from packed_util import D, Packed

pytestmark = pytest.mark.gpu


def bits(t):
    return t.contiguous().view(torch.int16)


def same(got, want):
    """Bit for bit, any NaN being as good as any other."""
    got, want = got.cpu(), want.cpu()
    return torch.equal(torch.isnan(got), torch.isnan(want)) and torch.equal(bits(got)[~torch.isnan(got)], bits(want)[~torch.isnan(want)])


def positions_of(p):
    return torch.cat([torch.arange(l - n, l) for l, n in zip(p.lens, p.new)]) if p.cu_np[-1] else torch.zeros(0, dtype=torch.long)


@pytest.mark.parametrize("interleaved", [False, True])
@pytest.mark.parametrize("rotary", [16, 32, 48, 64, 80, 96, 112, 128])
def test_rows(rotary, interleaved):
    """Ragged sequences, one of them empty; rows behind the last sequence stay as they are."""
    for stride, heads, lens, new in ((0, 5, [70, 1, 33, 5], [9, 1, 33, 0]), (24, 1, [1], [1]), (8 * D, 33, [200, 3], [130, 3])):
        p = Packed(lens, new, heads=heads, kv_heads=1, seed=rotary, stride=stride, cached=False)
        table = table_of(200, rotary)
        out = torch.full((p.total, heads, D), 77.0, device=p.dev, dtype=torch.float16)
        Q.quest_rotate_tokens(p.cache, Q.Rotation(table, interleaved=interleaved), p.q, p.cu, out)
        n = int(p.cu_np[-1])
        assert same(out[:n], turned(p.q[:n], table, positions_of(p), interleaved))
        assert bool((out[n:] == 77).all())


@pytest.mark.parametrize("interleaved", [False, True])
@pytest.mark.parametrize("rotary", [64, 128])
def test_rows_in_place_and_into_a_fused_projection(rotary, interleaved):
    p = Packed([40, 77], [40, 31], heads=8, kv_heads=2, seed=3, cached=False)
    table = table_of(100, rotary)
    r = Q.Rotation(table, interleaved=interleaved)
    n = int(p.cu_np[-1])
    want = turned(p.q[:n], table, positions_of(p), interleaved)
    fused = torch.full((p.total, 12, D), 3.0, device=p.dev, dtype=torch.float16)
    fused[:, :8] = p.q
    Q.quest_rotate_tokens(p.cache, r, fused[:, :8], p.cu, fused[:, :8])
    assert same(fused[:n, :8], want) and bool((fused[:, 8:] == 3).all()) and same(fused[n:, :8], p.q[n:])
    wide = torch.full((p.total, 12, D), 3.0, device=p.dev, dtype=torch.float16)
    Q.quest_rotate_tokens(p.cache, r, p.q, p.cu, wide[:, 2:10])
    assert same(wide[:n, 2:10], want) and bool((wide[:, :2] == 3).all()) and bool((wide[:, 10:] == 3).all()) and bool((wide[n:] == 3).all())


@pytest.mark.parametrize("interleaved", [False, True])
def test_given_positions(interleaved):
    """Any positions, the same ones twice; those outside the table make the rotated channels NaN and nothing else."""
    p = Packed([50, 9], [23, 6], heads=3, kv_heads=1, seed=5, cached=False)
    table = table_of(64, 96)
    given = torch.tensor(np.random.default_rng(0).integers(0, 64, p.total), dtype=torch.int32)
    given[[2, 7, 8, 20, 28]] = torch.tensor([-1, 64, 2 ** 31 - 1, -2 ** 31, 65], dtype=torch.int32)
    out = torch.empty(p.total, 3, D, device=p.dev, dtype=torch.float16)
    Q.quest_rotate_tokens(p.cache, Q.Rotation(table, interleaved=interleaved, positions=given.to(p.dev)), p.q, p.cu, out)
    n = int(p.cu_np[-1])
    want = turned(p.q[:n], table, given[:n], interleaved)
    assert bool(torch.isnan(want[2, :, :96]).all()) and same(out[:n], want)


def test_table_shorter_than_a_sequence():
    p = Packed([40], [40], heads=2, kv_heads=1, seed=6, cached=False)
    table = table_of(30, 128)
    out = torch.empty(p.total, 2, D, device=p.dev, dtype=torch.float16)
    Q.quest_rotate_tokens(p.cache, Q.Rotation(table), p.q, p.cu, out)
    assert same(out[:40], turned(p.q[:40], table, torch.arange(40), False)) and bool(torch.isnan(out[30:40]).all())


def test_more_sequences_than_lanes():
    rng = np.random.default_rng(1)
    new = [int(x) for x in rng.integers(0, 5, 200)]
    lens = [n + int(rng.integers(0, 90)) for n in new]
    p = Packed(lens, new, heads=2, kv_heads=1, seed=7, cached=False)
    table = table_of(100, 128)
    out = torch.empty(p.total, 2, D, device=p.dev, dtype=torch.float16)
    Q.quest_rotate_tokens(p.cache, Q.Rotation(table), p.q, p.cu, out)
    n = int(p.cu_np[-1])
    assert same(out[:n], turned(p.q[:n], table, positions_of(p), False))


def cache_of(p, dtype):
    return dict(k_pool=p.k_pool, v_pool=p.v_pool, meta=p.meta, **({"scales": p.scales} if dtype == 8 else {}))


def raw(t):
    return t.contiguous().view(torch.uint8).clone()


@pytest.mark.parametrize("bits_of_cache", [16, 8])
@pytest.mark.parametrize("S", [8, 16, 32, 64])
@pytest.mark.parametrize("rotary,interleaved", [(128, False), (64, False), (96, True), (128, True)])
def test_insertion_with_rotation_is_both_calls(bits_of_cache, S, rotary, interleaved):
    """Bit for bit what rotation of the rows, then insertion, leave behind; also of keys and values alone, and with given positions."""
    make = Packed8 if bits_of_cache == 8 else Packed
    for lens, new, heads, kv_heads, stride in (([100, 70, 5, 131], [1, 70, 0, 66], 6, 2, 0), ([9], [1], 1, 1, 8), ([3 * S], [2 * S + 1], 9, 3, 5 * D)):
        for given in (False, True):
            a, b = (make(lens, new, heads=heads, kv_heads=kv_heads, S=S, seed=S, stride=stride) for _ in range(2))
            c = make(lens, new, heads=heads, kv_heads=kv_heads, S=S, seed=S, stride=stride)
            table = table_of(150, rotary)
            positions = torch.randint(0, 150, (a.total,), dtype=torch.int32, device=a.dev) if given else None
            r = Q.Rotation(table, interleaved=interleaved, positions=positions)
            n = int(a.cu_np[-1])
            out = torch.full((a.total, heads, D), 77.0, device=a.dev, dtype=torch.float16)
            Q.quest_rotate_append_tokens(a.cache, r, a.q, a.k_new, a.v_new, a.cu, out)
            k = torch.zeros(b.total, kv_heads, D, device=b.dev, dtype=torch.float16)
            q = torch.full_like(out, 77.0)
            Q.quest_rotate_tokens(b.cache, r, b.q, b.cu, q)
            Q.quest_rotate_tokens(b.cache, r, b.k_new, b.cu, k)
            Q.quest_append_tokens(b.cache, k, b.v_new.contiguous(), b.cu)
            Q.quest_rotate_append_tokens(c.cache, r, None, c.k_new, c.v_new, c.cu)
            where = positions[:n] if given else positions_of(a)
            assert same(k[:n], turned(b.k_new[:n], table, where, interleaved))
            assert torch.equal(raw(out), raw(q))
            for name, t in cache_of(a, bits_of_cache).items():
                assert torch.equal(raw(t), raw(getattr(b, name))) and torch.equal(raw(t), raw(getattr(c, name))), name


@pytest.mark.parametrize("S", [32, 64])
@pytest.mark.parametrize("rotary,interleaved", [(128, False), (64, True)])
def test_insertion_of_many_heads_with_rotation_is_both_calls(S, rotary, interleaved):
    """More (page, head) pairs than large pages of 8 bits are shared out for."""
    a, b = (Packed8([100, 70, 5, 131, 90, 3, 20], [1, 70, 0, 66, 90, 3, 7], heads=80, kv_heads=80, S=S, seed=S) for _ in range(2))
    r = Q.Rotation(table_of(150, rotary), interleaved=interleaved)
    Q.quest_rotate_append_tokens(a.cache, r, None, a.k_new, a.v_new, a.cu)
    k = torch.zeros(b.total, 80, D, device=b.dev, dtype=torch.float16)
    Q.quest_rotate_tokens(b.cache, r, b.k_new, b.cu, k)
    Q.quest_append_tokens(b.cache, k, b.v_new.contiguous(), b.cu)
    for name, t in cache_of(a, 8).items():
        assert torch.equal(raw(t), raw(getattr(b, name))), name


def test_insertion_in_place_and_repeated():
    """Queries turned where they lie; a second call with the same tokens changes nothing but them."""
    p = Packed([90, 31], [40, 1], heads=4, kv_heads=2, seed=2)
    table = table_of(100, 128)
    r = Q.Rotation(table)
    n = int(p.cu_np[-1])
    want = turned(p.q[:n], table, positions_of(p), False)
    q = p.q.contiguous().clone()
    Q.quest_rotate_append_tokens(p.cache, r, q, p.k_new, p.v_new, p.cu, q)
    assert same(q[:n], want)
    before = [raw(t) for t in (p.k_pool, p.v_pool, p.meta)]
    Q.quest_rotate_append_tokens(p.cache, r, q, p.k_new, p.v_new, p.cu, q)
    assert all(torch.equal(x, raw(t)) for x, t in zip(before, (p.k_pool, p.v_pool, p.meta)))
    assert same(q[:n], turned(want, table, positions_of(p), False))
