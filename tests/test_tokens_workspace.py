"""Sizes of the workspace for packed tokens: what calls can use, whatever the shape.  Host functions, no GPU."""
import ctypes

import pytest

from paper_2406_10774_amd import binding
from test_tokens_abi import make_cache


def workspace(total, **kw):
    out, c = ctypes.c_size_t(7), make_cache(**kw)
    assert binding.load().quest_tokens_workspace_bytes(ctypes.byref(c), total, ctypes.byref(out)) == 0
    return out.value


@pytest.mark.parametrize("heads", [1, 3, 8, 64, 100, 128, 129, 256, 512, 1024])
def test_workspace_is_no_larger_than_documented(heads):
    """At most 27 MB, or 140 MB with more than 64 rows a sequence, whatever the heads, batches and lengths; it does not fall."""
    for group in (1, 8):
        for batch in (1, 2, 3, 10, 63, 64, 200):
            for pages in (20, 90, 2048, 60000):
                kw = dict(batch=batch, num_heads=heads * group, num_kv_heads=heads, max_pages_per_seq=pages)
                last = 0
                for total in (0, 1, 2, 7, 8 * batch, 16 * batch, 64 * batch, 65 * batch, 300 * batch, 2000 * batch):
                    if total * heads * group > 2 ** 31 - 512 * batch * heads - 1:
                        continue
                    need = workspace(total, **kw)
                    assert last <= need <= (27e6 if total * group <= 64 * batch else 140e6), (kw, total, need)
                    last = need


def test_no_workspace_where_nothing_is_split():
    """As many sequences as the compute units take row tiles of at once leave none to split; from 129 KV heads on that holds for one
    row tile of 256 rows, from 257 on for one of 32."""
    assert workspace(64, batch=64, num_heads=8) == 0
    assert workspace(1, batch=1, num_heads=512, num_kv_heads=512) == 0
    assert workspace(5000, batch=1, num_heads=1024, num_kv_heads=1024) == 0
    assert workspace(5000, batch=1, num_heads=256, num_kv_heads=256) == workspace(64, batch=1, num_heads=256, num_kv_heads=256) > 0
    assert workspace(64, batch=32, num_heads=8) > 0
