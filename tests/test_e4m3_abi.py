"""Host-side checks of rotation and of pages of 8 bits, without a GPU: refusals before anything is enqueued."""
import ctypes

import numpy as np
import pytest
import torch

from paper_2406_10774_amd import binding
import e4m3_util as E

P = 0x1000
E8 = binding.QUEST_FLAG_E4M3_PAGES


def make_cache(**kw):
    base = dict(batch=2, num_heads=32, head_dim=128, page_size=16, max_pages_per_seq=2048, flags=0, num_phys_pages=2048,
                k_pool=P, v_pool=P, meta=P, page_table=P, seq_lens=P, num_kv_heads=8, scales=None)
    base.update(kw)
    return binding.quest_cache(**base)


def make_rotation(**kw):
    base = dict(table=P, positions=None, num_positions=100, rotary_dim=128, interleaved=0)
    base.update(kw)
    return binding.quest_rotation(**base)


ARGS = {
    "quest_rotate_tokens": dict(x=P, x_stride=4096, heads=32, cu=P, total=7, out=P, out_stride=4096, stream=None),
    "quest_rotate_append_tokens": dict(q=P, q_stride=4096, q_out=P, q_out_stride=4096, k_new=P, v_new=P, new_stride=1024, cu=P,
                                       total=7, stream=None),
}


def call(name, cache=None, rotation=None, **kw):
    args = dict(ARGS[name])
    assert set(kw) <= set(args)
    args.update(kw)
    c, r = make_cache(**(cache or {})), make_rotation(**(rotation or {}))
    return getattr(binding.load(), name)(ctypes.byref(c), ctypes.byref(r), *args.values())


@pytest.mark.parametrize("name", list(ARGS))
@pytest.mark.parametrize("rotation,status", [
    (dict(table=None), -1), (dict(table=P + 4), -2), (dict(num_positions=0), -2), (dict(rotary_dim=0), -3),
    (dict(rotary_dim=8), -3), (dict(rotary_dim=24), -3), (dict(rotary_dim=144), -3), (dict(rotary_dim=-16), -3)])
def test_bad_rotations(name, rotation, status):
    assert call(name, rotation=rotation) == status
    assert name.encode() in binding.load().quest_last_error()


@pytest.mark.parametrize("name", list(ARGS))
@pytest.mark.parametrize("cache,status", [
    (dict(head_dim=64), -3), (dict(page_size=24), -3), (dict(batch=0), -2), (dict(page_table=None), -1), (dict(seq_lens=None), -1),
    (dict(num_kv_heads=5), -2)])
def test_bad_caches(name, cache, status):
    assert call(name, cache=cache) == status
    assert name.encode() in binding.load().quest_last_error()


@pytest.mark.parametrize("name,kw,status", [
    ("quest_rotate_tokens", dict(x=None), -1), ("quest_rotate_tokens", dict(out=None), -1), ("quest_rotate_tokens", dict(cu=None), -1),
    ("quest_rotate_tokens", dict(heads=0), -2), ("quest_rotate_tokens", dict(heads=65536), -2), ("quest_rotate_tokens", dict(total=-1), -2),
    ("quest_rotate_tokens", dict(x_stride=4095), -2), ("quest_rotate_tokens", dict(out_stride=4088), -2),
    ("quest_rotate_tokens", dict(x=P + 8), -2), ("quest_rotate_tokens", dict(out=P + 2), -2),
    ("quest_rotate_append_tokens", dict(k_new=None), -1), ("quest_rotate_append_tokens", dict(v_new=None), -1),
    ("quest_rotate_append_tokens", dict(q_out=None), -1), ("quest_rotate_append_tokens", dict(cu=None), -1),
    ("quest_rotate_append_tokens", dict(total=-1), -2), ("quest_rotate_append_tokens", dict(new_stride=1016), -2),
    ("quest_rotate_append_tokens", dict(q_stride=4088), -2), ("quest_rotate_append_tokens", dict(q_out_stride=8), -2),
    ("quest_rotate_append_tokens", dict(q=P + 4), -2), ("quest_rotate_append_tokens", dict(v_new=P + 8), -2)])
def test_refused_arguments(name, kw, status):
    assert call(name, **kw) == status
    assert name.encode() in binding.load().quest_last_error()


def test_rotation_and_cache_missing():
    lib = binding.load()
    for name in ARGS:
        c, r = make_cache(), make_rotation()
        assert getattr(lib, name)(ctypes.byref(c), None, *ARGS[name].values()) == -1
        assert getattr(lib, name)(None, ctypes.byref(r), *ARGS[name].values()) == -1
    for pool in ("k_pool", "v_pool", "meta"):
        assert call("quest_rotate_append_tokens", cache={pool: None}) == -1


@pytest.mark.parametrize("name", list(ARGS))
def test_no_tokens_is_no_work(name):
    none = {k: None for k in ("x", "out", "q", "q_out", "k_new", "v_new") if k in ARGS[name]}
    assert call(name, total=0, **none) == 0


def every_call(c):
    """The calls of the library that touch the pools, with arguments that are right for an fp16 cache."""
    lib, cr, r = binding.load(), ctypes.byref(c), make_rotation()
    rr = ctypes.byref(r)
    return {
        "quest_build_meta": lambda: lib.quest_build_meta(cr, None),
        "quest_append_meta": lambda: lib.quest_append_meta(cr, P, P, 1, None),
        "quest_append_estimate": lambda: lib.quest_append_estimate(cr, P, P, 1, P, P, None),
        "quest_decode_step": lambda: lib.quest_decode_step(cr, P, P, 1, P, 8, 1.0, P, P, None, P, 0, None, P, 1 << 30, None),
        "quest_decode_step_static": lambda: lib.quest_decode_step_static(cr, P, P, 0, P, 8, 1.0, P, P, None, P, 0, None, None),
        "quest_tree_attention": lambda: lib.quest_tree_attention(cr, P, 4096, P, P, 1024, P, 7, P, 1, None, 0, 1.0, P, 0, None,
                                                                 None, 0, None),
        "quest_append_tokens": lambda: lib.quest_append_tokens(cr, P, P, 1024, None, P, 7, None),
        "quest_rotate_append_tokens": lambda: lib.quest_rotate_append_tokens(cr, rr, P, 4096, P, 4096, P, P, 1024, P, 7, None),
        "quest_prompt_attention": lambda: lib.quest_prompt_attention(cr, P, 4096, P, 7, 1.0, P, 0, None, None, 0, None),
        "quest_sparse_decode": lambda: lib.quest_sparse_decode(cr, P, None, 0, 1.0, P, 0, None, None, 0, None),
        "quest_select_decode": lambda: lib.quest_select_decode(cr, P, P, 8, 1.0, P, None, P, 0, None, None, 0, None),
    }


@pytest.mark.parametrize("name", ["quest_build_meta", "quest_append_meta", "quest_append_estimate", "quest_decode_step",
                                  "quest_decode_step_static"])
def test_calls_that_know_fp16_pages_only(name):
    assert every_call(make_cache(flags=E8, scales=P))[name]() == -3
    message = binding.load().quest_last_error()
    assert name.encode() in message and b"fp16 pages" in message


@pytest.mark.parametrize("name", ["quest_append_tokens", "quest_rotate_append_tokens", "quest_prompt_attention",
                                  "quest_tree_attention", "quest_sparse_decode", "quest_select_decode"])
@pytest.mark.parametrize("cache,status", [(dict(scales=None), -1), (dict(scales=P + 4), -2), (dict(scales=P, k_pool=P + 8), -2),
                                          (dict(scales=P, v_pool=P + 1), -2)])
def test_pools_of_8_bits(name, cache, status):
    assert every_call(make_cache(flags=E8, **cache))[name]() == status
    assert name.encode() in binding.load().quest_last_error()


def test_steps_of_8_bits_need_scales():
    c = make_cache(flags=E8)
    assert binding.load().quest_decode_step(ctypes.byref(c), None, None, 0, P, 8, 1.0, P, P, None, P, 0, None, None, 0, None) == -1


def test_workspaces_off_their_alignment():
    c, lib = make_cache(flags=E8, scales=P), binding.load()
    assert lib.quest_sparse_decode(ctypes.byref(c), P, None, 0, 1.0, P, 0, None, P + 8, 1 << 20, None) == -2
    assert lib.quest_select_decode(ctypes.byref(c), P, P, 8, 1.0, P, None, P, 0, None, P + 4, 1 << 20, None) == -2


def test_too_many_heads_and_sequences_for_a_launch():
    c = make_cache(flags=E8, scales=P, batch=65535, num_heads=4096, num_kv_heads=4096)
    assert every_call(c)["quest_sparse_decode"]() == -2


def test_workspace_bytes_have_one_size():
    lib, out = binding.load(), ctypes.c_size_t(0)
    for kw in (dict(), dict(num_kv_heads=32), dict(batch=300), dict(num_heads=1, num_kv_heads=1), dict(max_pages_per_seq=20000)):
        sizes = set()
        for k_pages in (0, 1, 128, 5000):
            c = make_cache(flags=E8, scales=P, **kw)
            assert lib.quest_workspace_bytes(ctypes.byref(c), k_pages, ctypes.byref(out)) == 0
            sizes.add(out.value)
        assert lib.quest_step_workspace_bytes(ctypes.byref(c), 7, ctypes.byref(out)) == 0
        sizes.add(out.value)
        assert len(sizes) == 1 and max(sizes) < 64 << 20


def test_binding_describes_pools_of_8_bits():
    pool, meta = torch.zeros(3, 8, 16, 128, dtype=torch.uint8), torch.zeros(8, 3, 2, 128, dtype=torch.float16)
    table, lens, scales = torch.zeros(2, 4, dtype=torch.int32), torch.zeros(2, dtype=torch.int32), torch.ones(3, 8, 2)
    for k in (pool, pool.view(torch.float8_e4m3fn)):
        assert binding.Cache(k, pool, meta, table, lens, scales=scales).c.flags == E8
    half = torch.zeros(3, 8, 16, 128, dtype=torch.float16)
    assert binding.Cache(half, half, meta, table, lens).c.flags == 0
    for k, v, s in ((pool, pool, None), (half, half, scales), (pool, half, scales), (pool, pool[:2], scales), (pool, None, scales),
                    (pool, pool, scales.double()), (pool, pool, scales[:2]), (pool, pool, torch.ones(3, 2, 8).transpose(1, 2)),
                    (pool.view(torch.float8_e5m2), pool, scales), (pool[:, ::2], pool[:, ::2], scales[:, ::2])):
        with pytest.raises(binding.QuestError):
            binding.Cache(k, v, meta, table, lens, scales=s)
    with pytest.raises(binding.QuestError):
        binding.Cache(half, half, meta, table, lens, flags=E8)


def test_binding_refuses_rotations_it_cannot_describe():
    table = torch.zeros(50, 64)
    binding.Rotation(table), binding.Rotation(table, positions=torch.zeros(9, dtype=torch.int32))
    for t in (table.half(), table.double(), table[:, ::2], table[0], table.t()):
        with pytest.raises(binding.QuestError):
            binding.Rotation(t)
    for p in (torch.zeros(9), torch.zeros(9, dtype=torch.int64), torch.zeros(18, dtype=torch.int32)[::2]):
        with pytest.raises(binding.QuestError):
            binding.Rotation(table, positions=p)

    pool, meta = torch.zeros(3, 8, 16, 128, dtype=torch.float16), torch.zeros(8, 3, 2, 128, dtype=torch.float16)
    cu, lens = torch.zeros(3, dtype=torch.int32), torch.zeros(2, dtype=torch.int32)
    cache = binding.Cache(pool, pool, meta, torch.zeros(2, 4, dtype=torch.int32), lens, num_heads=16)
    q, kv = torch.zeros(6, 16, 128, dtype=torch.float16), torch.zeros(6, 8, 128, dtype=torch.float16)
    rotation = binding.Rotation(table)
    few = binding.Rotation(table, positions=torch.zeros(5, dtype=torch.int32))

    def both(rotation=rotation, q=q, k=kv, v=kv, cu=cu, q_out=q):
        binding.quest_rotate_append_tokens(cache, rotation, q, k, v, cu, q_out, stream=0)

    def one(rotation=rotation, q=q, cu=cu, q_out=q):
        binding.quest_rotate_tokens(cache, rotation, q, cu, q_out, stream=0)

    for kw in (dict(rotation=few), dict(q=q[:, :8]), dict(q=q.float()), dict(q=None), dict(q_out=None), dict(q_out=q[:5]), dict(q=q[:5]),
               dict(k=kv[:, :4], v=kv[:, :4]), dict(v=kv[:5]), dict(cu=cu.long()), dict(cu=cu[:2])):
        with pytest.raises(binding.QuestError):
            both(**kw)
    for kw in (dict(rotation=few), dict(q=q.float()), dict(q_out=q[:5]), dict(q_out=q[:, :8]), dict(cu=cu[:2]), dict(q=q[0])):
        with pytest.raises(binding.QuestError):
            one(**kw)
    empty_q, empty = q[:0], kv[:0]                                 # no rows, no work: these return without a GPU
    both(q=empty_q, q_out=empty_q, k=empty, v=empty), both(q=None, q_out=None, k=empty, v=empty), one(q=empty_q, q_out=empty_q)


def test_definition_of_e4m3():
    """The tests' own numbers against torch's type, and rounding to the nearest, ties to even, against a search over all."""
    theirs = torch.arange(256, dtype=torch.uint8).view(torch.float8_e4m3fn).double().numpy()
    assert np.array_equal(E.VALUES, theirs, equal_nan=True)
    x = np.concatenate([E.MAGNITUDES, (E.MAGNITUDES[1:] + E.MAGNITUDES[:-1]) / 2, np.random.default_rng(0).uniform(0, 448, 2000),
                        2.0 ** np.random.default_rng(1).uniform(-12, 8.8, 2000)])
    x = np.concatenate([x, -x])
    codes = torch.from_numpy(x).float()
    exact = codes.double().numpy() == x                            # (float32 is what torch rounds)
    assert np.array_equal(E.nearest(x)[exact], codes.to(torch.float8_e4m3fn).view(torch.uint8).numpy()[exact])
    for e in range(-15, 9):
        assert E.exponent_for(np.ldexp(448.0, e)) == e
        assert e == 8 or E.exponent_for(np.ldexp(448.5, e)) == e + 1
    assert E.exponent_for(0.0) == -15 and E.exponent_for(61440.0) == 8
