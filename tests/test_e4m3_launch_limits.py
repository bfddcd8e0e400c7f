"""Rotation and insertion of more tokens than a launch has threads for: refused before anything is enqueued, without a GPU."""
import ctypes

import pytest

from paper_2406_10774_amd import binding as Q

P = 0x1000
MOST = 2 ** 32 - 1                                                 # threads of a launch


def cache(kv_heads, heads, flags):
    return Q.quest_cache(batch=1, num_heads=heads, head_dim=128, page_size=8, max_pages_per_seq=16, flags=flags, num_phys_pages=16,
                         k_pool=P, v_pool=P, meta=P, page_table=P, seq_lens=P, num_kv_heads=kv_heads, scales=P)


# A wave of 64 threads turns four tokens of four heads.
@pytest.mark.parametrize("heads,total", [(1, 2 ** 28 + 1), (1, 2 ** 31 - 2 ** 15), (2, 2 ** 29), (3, 2 ** 28 + 100), (7, 2 ** 27 + 100)])
def test_rotation(heads, total):
    assert (total // 4 + 1) * (-(-heads // 4)) * 64 > MOST
    c, r = cache(1, 1, 0), Q.quest_rotation(table=P, positions=None, num_positions=9, rotary_dim=128, interleaved=0)
    assert Q.load().quest_rotate_tokens(ctypes.byref(c), ctypes.byref(r), P, heads * 128, heads, P, total, P, heads * 128, None) == -2
    assert b"quest_rotate_tokens" in Q.load().quest_last_error()


@pytest.mark.parametrize("flags", [0, Q.QUEST_FLAG_E4M3_PAGES])
@pytest.mark.parametrize("heads,kv_heads,total,queries", [(1, 1, 2 ** 28, True), (2, 1, 2 ** 29, True), (1, 1, 2 ** 29 + 2 ** 15, False)])
def test_rotated_insertion(heads, kv_heads, total, queries, flags):
    c, r = cache(kv_heads, heads, flags), Q.quest_rotation(table=P, positions=None, num_positions=9, rotary_dim=128, interleaved=0)
    q = P if queries else None
    assert Q.load().quest_rotate_append_tokens(ctypes.byref(c), ctypes.byref(r), q, heads * 128, q, heads * 128, P, P, kv_heads * 128, P,
                                               total, None) == -2
    assert b"quest_rotate_append_tokens" in Q.load().quest_last_error()


def test_insertion_into_pages_of_8_bits():
    c = cache(1, 1, Q.QUEST_FLAG_E4M3_PAGES)
    assert Q.load().quest_append_tokens(ctypes.byref(c), P, P, 128, None, P, 2 ** 29 + 2 ** 15, None) == -2
    assert b"quest_append_tokens" in Q.load().quest_last_error()
