"""Host-side checks of the calls on packed tokens, without a GPU: refusals before anything is enqueued."""
import ctypes

import pytest
import torch

from paper_2406_10774_amd import binding

P = 0x1000


def make_cache(**kw):
    base = dict(batch=2, num_heads=32, head_dim=128, page_size=16, max_pages_per_seq=2048, flags=0, num_phys_pages=2048,
                k_pool=P, v_pool=P, meta=P, page_table=P, seq_lens=P, num_kv_heads=8)
    base.update(kw)
    return binding.quest_cache(**base)


ARGS = {
    "quest_append_tokens": dict(k_new=P, v_new=P, new_stride=1024, rows=None, cu=P, total=7, stream=None),
    "quest_prompt_attention": dict(q=P, q_stride=4096, cu=P, total=7, scale=1.0, out=P, half=0, lse=None, ws=None,
                                   ws_bytes=0, stream=None),
    "quest_tree_attention": dict(q=P, q_stride=4096, k_new=P, v_new=P, new_stride=1024, cu=P, total=7, mask=P, words=1,
                                 topk=None, k_pages=0, scale=1.0, out=P, half=0, lse=None, ws=None, ws_bytes=0, stream=None),
}


def call(name, cache=None, **kw):
    args = dict(ARGS[name])
    assert set(kw) <= set(args)
    args.update(kw)
    c = make_cache(**(cache or {}))
    return getattr(binding.load(), name)(ctypes.byref(c), *args.values())


@pytest.mark.parametrize("name", list(ARGS))
@pytest.mark.parametrize("cache,status", [
    (dict(head_dim=64), -3), (dict(page_size=24), -3), (dict(batch=0), -2), (dict(num_heads=70000), -2),
    (dict(page_table=None), -1), (dict(seq_lens=None), -1), (dict(k_pool=None), -1), (dict(v_pool=None), -1),
    (dict(num_kv_heads=5), -2), (dict(max_pages_per_seq=0), -2)])
def test_bad_caches(name, cache, status):
    assert call(name, cache) == status
    assert name.encode() in binding.load().quest_last_error()


REFUSED = [
    ("quest_append_tokens", dict(cu=None), -1), ("quest_append_tokens", dict(total=-1), -2),
    ("quest_append_tokens", dict(total=2 ** 30), -2),
    ("quest_append_tokens", dict(k_new=None), -1), ("quest_append_tokens", dict(v_new=None), -1),
    ("quest_append_tokens", dict(k_new=P + 8), -2), ("quest_append_tokens", dict(v_new=P + 2), -2),
    ("quest_append_tokens", dict(new_stride=1028), -2), ("quest_append_tokens", dict(new_stride=1016), -2),
    ("quest_append_tokens", dict(new_stride=0), -2),
    ("quest_prompt_attention", dict(cu=None), -1), ("quest_prompt_attention", dict(total=-3), -2),
    ("quest_prompt_attention", dict(total=2 ** 30), -2),
    ("quest_prompt_attention", dict(q=None), -1), ("quest_prompt_attention", dict(out=None), -1),
    ("quest_prompt_attention", dict(q=P + 4), -2), ("quest_prompt_attention", dict(q_stride=4088), -2),
    ("quest_prompt_attention", dict(q_stride=-4096), -2), ("quest_prompt_attention", dict(q_stride=4100), -2),
    ("quest_prompt_attention", dict(out=P + 8), -2), ("quest_prompt_attention", dict(ws=P + 4, ws_bytes=1 << 20), -2),
    ("quest_tree_attention", dict(cu=None), -1), ("quest_tree_attention", dict(total=-1), -2),
    ("quest_tree_attention", dict(q=None), -1), ("quest_tree_attention", dict(k_new=None), -1),
    ("quest_tree_attention", dict(v_new=None), -1), ("quest_tree_attention", dict(out=None), -1),
    ("quest_tree_attention", dict(mask=None), -1), ("quest_tree_attention", dict(words=0), -2),
    ("quest_tree_attention", dict(topk=P, k_pages=0), -2), ("quest_tree_attention", dict(new_stride=1000), -2),
    ("quest_tree_attention", dict(q_stride=0), -2), ("quest_tree_attention", dict(out=P + 2), -2),
]


@pytest.mark.parametrize("name,kw,status", REFUSED)
def test_refused_arguments(name, kw, status):
    assert call(name, **kw) == status
    assert name.encode() in binding.load().quest_last_error()


@pytest.mark.parametrize("name", list(ARGS))
def test_missing_cache(name):
    assert getattr(binding.load(), name)(None, *ARGS[name].values()) == -1


def test_append_needs_metadata():
    assert call("quest_append_tokens", dict(meta=None)) == -1


@pytest.mark.parametrize("name", list(ARGS))
def test_no_tokens_is_no_work(name):
    """Nothing is enqueued, so this returns without a GPU; the tensors of no rows have no address."""
    none = {k: None for k in ("q", "k_new", "v_new", "out", "mask") if k in ARGS[name]}
    assert call(name, total=0, **none) == 0
    assert call(name, total=0, cu=None) == -1


def test_workspace_bytes():
    lib, out = binding.load(), ctypes.c_size_t(7)

    def need(total, **kw):
        c = make_cache(**kw)
        assert lib.quest_tokens_workspace_bytes(ctypes.byref(c), total, ctypes.byref(out)) == 0
        return out.value

    assert need(0) >= 0 and need(4) > 0
    c = make_cache()
    assert lib.quest_tokens_workspace_bytes(ctypes.byref(c), 4, None) == -1
    assert lib.quest_tokens_workspace_bytes(ctypes.byref(c), -1, ctypes.byref(out)) == -2
    assert lib.quest_tokens_workspace_bytes(None, 4, ctypes.byref(out)) == -1


def test_binding_refuses_rows_it_cannot_describe():
    """Heads apart, keys and values with different strides: before the library is asked."""
    x = torch.zeros(6, 16, 128, dtype=torch.float16)
    for k, v in ((x[:, ::2], x[:, ::2]), (x[:, :8], x[::2][:, :8]), (x[:, :8], torch.zeros(6, 8, 128, dtype=torch.float16)),
                 (x.transpose(1, 2)[:, :, :8], x.transpose(1, 2)[:, :, :8])):
        with pytest.raises(binding.QuestError):
            binding._row_stride(k, v)
    assert binding._row_stride(x[:, 4:12], x[:, :8]) == 16 * 128
    assert binding._row_stride(x[:1, :8]) == 8 * 128
