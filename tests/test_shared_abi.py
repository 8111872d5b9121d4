"""The entry points for shared prompts on a machine without a GPU: what they refuse on the
host, and the plain model of the page operations against hand-worked states."""
import ctypes

import numpy as np
import pytest

from paper_2607_06601_gb300 import build, trr


@pytest.fixture(scope="module")
def lib():
    build.build()
    return trr.load()


def test_without_a_cache_every_call_is_refused(lib):
    out = ctypes.c_uint64()
    assert lib.trr_workspace_bytes(None, ctypes.byref(out)) == 1
    assert lib.trr_fork(None, 0, None, None, None, None, 0, None) == 1
    assert lib.trr_evict(None, 0, None, None, 0, None) == 1
    assert lib.trr_free_seqs(None, 0, None, None) == 1
    assert lib.trr_compact(None, None, 0, None) == 1
    assert lib.trr_decode_attn_sinks(None, 0, 0, None, None, None, None, None, 0, 0, 0.0, None, None, 0, None) == 1
    assert lib.trr_decode_attn_shared(None, 0, 0, None, None, None, None, None, 0, 0, 0, None, 0.0, None, None, 0, None) == 1


class Shape:
    """What the model needs of a cache: one layer, pages of 2 tokens, positions alone."""
    L, S, Hkv, P, head_modes = 1, 4, 1, 2, 0


def state():
    """Sequence 0 holds positions 0, 2, 3, 7, 9 (class 0: pages 0, 2, 1) and 5 (class 2: page 0)."""
    m = {"last_pos": np.array([[9, -1, -1, -1]], np.int32), "ntok": np.zeros((1, 4, 4), np.int32),
         "presence": np.zeros((1, 4, 1), np.uint32), "next_page": np.array([3, 0, 1, 0], np.int32),
         "pools": [np.zeros((8, 16), np.uint8) for _ in range(4)]}
    for n in ("page_table", "page_first", "page_last"):
        m[n] = np.full((1, 4, 4, 5), -1, np.int32)
    m["ntok"][0, 0] = [5, 0, 1, 0]
    m["presence"][0, 0, 0] = sum(1 << p for p in (0, 2, 3, 5, 7, 9))
    m["page_table"][0, 0, 0, :3] = [0, 2, 1]
    m["page_first"][0, 0, 0, :3] = [0, 3, 9]
    m["page_last"][0, 0, 0, :3] = [2, 7, 9]
    m["page_table"][0, 0, 2, 0], m["page_first"][0, 0, 2, 0], m["page_last"][0, 0, 2, 0] = 0, 5, 5
    for page, pos in ((0, (0, 2)), (2, (3, 7)), (1, (9, 77))):
        m["pools"][0][page, :8] = np.array(pos, np.int32).view(np.uint8)
    m["pools"][2][0, :8] = np.array((5, 66), np.int32).view(np.uint8)
    return m


def test_model_of_a_fork_shares_full_pages_and_copies_the_cut_one():
    from _shared import model_fork
    m = state()
    model_fork(m, Shape, [0], [1], [6])  # 0, 2 | 3 and 5: page 2 is cut, page 1 left out
    assert m["page_table"][0, 1, 0].tolist() == [0, 3, -1, -1, -1] and m["page_table"][0, 1, 2, 0] == 1
    assert m["page_last"][0, 1, 0].tolist() == [2, 3, -1, -1, -1] and m["ntok"][0, 1].tolist() == [3, 0, 1, 0]
    assert m["next_page"].tolist() == [4, 0, 2, 0] and m["last_pos"][0].tolist() == [9, 5, -1, -1]
    assert m["presence"][0, 1, 0] == sum(1 << p for p in (0, 2, 3, 5))
    assert (m["pools"][0][3] == m["pools"][0][2]).all() and m["ntok"][0, 0].tolist() == [5, 0, 1, 0]


def test_model_of_eviction_release_and_compaction():
    from _shared import model_compact, model_evict, model_fork, model_free
    m = state()
    model_fork(m, Shape, [0], [1], [10])
    assert model_evict(m, Shape, [0], [8], 1) == {(0, 0): [3, 7]}  # page 0 holds the sink, page 1 is not full
    assert m["page_table"][0, 0, 0].tolist() == [0, 1, -1, -1, -1] and m["ntok"][0, 0].tolist() == [3, 0, 1, 0]
    assert m["presence"][0, 0, 0] == sum(1 << p for p in (0, 2, 5, 9)) and m["page_table"][0, 1, 0].tolist() == [0, 2, 3, -1, -1]
    model_free(m, [0])
    model_compact(m, Shape)  # pages 0, 2, 3 in use: 3 moves to the hole at 1
    assert m["page_table"][0, 1, 0].tolist() == [0, 2, 1, -1, -1] and m["next_page"].tolist() == [3, 0, 1, 0]
    assert m["pools"][0][1, :4].view(np.int32)[0] == 9 and m["page_table"][0, 1, 2, 0] == 0
