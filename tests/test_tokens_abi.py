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
    (dict(num_kv_heads=5), -2), (dict(max_pages_per_seq=0), -2), (dict(max_pages_per_seq=2 ** 27 - 1), -2),
    (dict(max_pages_per_seq=2 ** 27 - 1024), -2)])
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
    ("quest_tree_attention", dict(mask=P + 4), -2),
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


def test_workspace_bytes_do_not_fall():
    """Enough for every smaller number of tokens as well; nothing for rows of a page table that nothing is split in."""
    lib, out = binding.load(), ctypes.c_size_t(7)
    for kw in (dict(), dict(num_kv_heads=32), dict(batch=1, num_heads=1, num_kv_heads=1), dict(batch=500), dict(max_pages_per_seq=90)):
        c, last = make_cache(**kw), 0
        for total in (0, 1, 5, 33, 100, 1000, 30000, 1000000):
            assert lib.quest_tokens_workspace_bytes(ctypes.byref(c), total, ctypes.byref(out)) == 0
            assert last <= out.value <= 160 << 20
            last = out.value
    c = make_cache(max_pages_per_seq=20)
    assert lib.quest_tokens_workspace_bytes(ctypes.byref(c), 100, ctypes.byref(out)) == 0 and out.value == 0


class Caller:
    """Tensors of a valid call, on the CPU (refused, or of no rows: nothing is read)."""

    def __init__(self, rows=6):
        self.pool = torch.zeros(3, 8, 16, 128, dtype=torch.float16)
        self.meta = torch.zeros(8, 3, 2, 128, dtype=torch.float16)
        self.cu, lens = torch.zeros(3, dtype=torch.int32), torch.zeros(2, dtype=torch.int32)
        self.cache = binding.Cache(self.pool, self.pool, self.meta, torch.zeros(2, 4, dtype=torch.int32), lens, num_heads=16)
        self.q, self.kv = torch.zeros(rows, 16, 128, dtype=torch.float16), torch.zeros(rows, 8, 128, dtype=torch.float16)
        self.mask, self.out = torch.zeros(rows, 1, dtype=torch.int64), torch.zeros(rows, 16, 128)
        self.lse, self.lists = torch.zeros(rows, 16), torch.zeros(2, 8, 5, dtype=torch.int32)

    def append(self, **kw):
        a = dict(k_new=self.kv, v_new=self.kv, cu_tokens=self.cu, rows=None, stream=0) | kw
        binding.quest_append_tokens(self.cache, **a)

    def prompt(self, **kw):
        a = dict(q=self.q, cu_tokens=self.cu, sm_scale=1.0, out=self.out, lse=self.lse, stream=0) | kw
        binding.quest_prompt_attention(self.cache, **a)

    def tree(self, **kw):
        a = dict(q=self.q, k_new=self.kv, v_new=self.kv, cu_tokens=self.cu, tree_mask=self.mask, sm_scale=1.0, out=self.out,
                 topk_idx=self.lists, lse=self.lse, stream=0) | kw
        binding.quest_tree_attention(self.cache, **a)


def test_binding_refuses_what_it_cannot_describe():
    """Types, gaps, too few rows or heads: before the library is asked."""
    c = Caller()
    wide = torch.zeros(6, 16, 128, dtype=torch.float16)
    for k, v in ((wide[:, ::2], wide[:, ::2]), (wide[:, :8], c.kv), (wide, wide), (c.kv.float(), c.kv.float()),
                 (c.kv, c.kv[:5]), (c.kv, c.kv.bfloat16()), (c.kv[:, :4], c.kv[:, :4]),
                 (c.kv.transpose(1, 2).contiguous().transpose(1, 2), c.kv.transpose(1, 2).contiguous().transpose(1, 2))):
        for call in (c.append, c.tree):
            with pytest.raises(binding.QuestError):
                call(k_new=k, v_new=v)
    bad = [dict(cu_tokens=c.cu[:2]), dict(cu_tokens=c.cu.long())]
    for kw in bad + [dict(rows=c.cu.long()), dict(rows=torch.zeros(8, dtype=torch.int32)[::2])]:
        with pytest.raises(binding.QuestError):
            c.append(**kw)
    bad += [dict(q=c.q[:, :8]), dict(q=c.q.float()), dict(out=c.out[:5]), dict(out=c.out.bfloat16()), dict(out=c.out.double()),
            dict(out=torch.zeros(6, 17, 128)[:, :16]), dict(out=torch.zeros(16, 6, 128).transpose(0, 1)), dict(out=c.out[:, :8].contiguous()), dict(lse=c.lse[:4]), dict(lse=c.lse.half()),
            dict(lse=torch.zeros(6, 15))]
    for kw in bad:
        for call in (c.prompt, c.tree):
            with pytest.raises(binding.QuestError):
                call(**kw)
    for kw in (dict(tree_mask=c.mask.int()), dict(tree_mask=c.mask[:5]), dict(tree_mask=torch.zeros(6, 2, dtype=torch.int64)[:, :1]),
               dict(topk_idx=c.lists.long()), dict(topk_idx=c.lists[:1]), dict(topk_idx=c.lists[:, :, ::2]),
               dict(k_new=c.kv[:5], v_new=c.kv[:5])):
        with pytest.raises(binding.QuestError):
            c.tree(**kw)


def test_binding_takes_strided_rows():
    """Parts of a fused projection; no rows at all are no work, so these return without a GPU."""
    c = Caller(rows=0)
    c.append(), c.prompt(), c.tree(), c.tree(topk_idx=None, lse=None), c.prompt(lse=None)
    fused = torch.zeros(7, 32, 128, dtype=torch.float16)
    assert binding._rows_of(c.cache, (7, 16, 128), fused[:, :16], 16) == 32 * 128
    assert binding._rows_of(c.cache, (7, 8, 128), fused[:, 16:24], 8, fused[:, 24:]) == 32 * 128
    assert binding._rows_of(c.cache, (1, 16, 128), fused[3:4, :16], 16) == 16 * 128


def test_binding_refuses_other_devices_and_head_sizes(monkeypatch):
    """The caller's tensors lie on the CPU here: the cache says that it lies elsewhere, or that the current device is
    another."""
    c = Caller()
    narrow = torch.zeros(6, 8, 256, dtype=torch.float16)[:, :, :64]
    for call in (c.append, c.tree):
        with pytest.raises(binding.QuestError):
            call(k_new=narrow, v_new=narrow)
    one = binding.Cache(c.pool[:, :1], c.pool[:, :1], c.meta, c.cache.page_table, c.cache.seq_lens)
    with pytest.raises(binding.QuestError):   # 64 channels, 128 apart
        binding.quest_prompt_attention(one, c.q[:, :1, :64], c.cu, 1.0, torch.zeros(6, 1, 64), stream=0)
    with pytest.raises(binding.QuestError, match="workspace"):
        c.prompt(workspace=torch.zeros(64)[::2])
    c.cache.device = 0
    for call in (c.append, c.prompt, c.tree):
        with pytest.raises(binding.QuestError, match="on the cache's device"):
            call()
    monkeypatch.setattr(binding, "_current_device", lambda: 1)
    with pytest.raises(binding.QuestError, match="not the current one"):
        binding._stream_of(c.cache, 5)
    monkeypatch.setattr(binding, "_current_device", lambda: 0)
    assert binding._stream_of(c.cache, 5) == 5
