"""Prompts by chunks and reading back on a machine without a GPU: what the calls refuse on the host."""
import ctypes

import pytest
import torch

from paper_2607_06601_gb300 import build, trr


@pytest.fixture(scope="module")
def lib():
    build.build()
    return trr.load()


def test_without_a_cache_every_call_is_refused(lib):
    out = ctypes.c_uint64()
    assert lib.trr_chunk_workspace_bytes(None, 1, 1, 1, ctypes.byref(out)) == 1
    assert lib.trr_chunk_attn(None, 0, 0, None, None, None, 0, None, None, None, 0, 0, 0.0, None, None, None, 0, None) == 1
    assert lib.trr_kv_read(None, 0, 0, None, None, None, 0, 1, None, 0, None, 0, None, None) == 1


def test_the_binding_takes_tensors_of_the_gpu_only(lib):
    ids, offsets = torch.zeros(1, dtype=torch.int32), torch.zeros(2, dtype=torch.int32)
    rows = torch.zeros(4, 2, 64, dtype=torch.bfloat16)
    modes = torch.zeros(4, dtype=torch.uint8)
    space = torch.zeros(16, dtype=torch.uint8)
    with pytest.raises(ValueError):
        trr.trr_chunk_attn(None, 0, ids, ids, offsets, rows, modes, None, 1, 0, 0.0, rows, None, space)
    with pytest.raises(ValueError):
        trr.trr_kv_read(None, 0, ids, ids, offsets, rows, rows, None)


def test_the_binding_checks_lengths_and_types(lib):
    ids, offsets = torch.zeros(2, dtype=torch.int32), torch.zeros(2, dtype=torch.int32)
    rows = torch.zeros(4, 2, 64, dtype=torch.bfloat16)
    modes = torch.zeros(4, dtype=torch.uint8)
    with pytest.raises(ValueError, match="offsets"):
        trr.trr_chunk_attn(None, 0, ids, ids, offsets, rows, modes, None, 1, 0, 0.0, rows, None, modes)
    with pytest.raises(ValueError, match="starts"):
        trr.trr_kv_read(None, 0, ids, ids[:1], offsets, rows, rows, None)
    with pytest.raises(ValueError, match="one type"):
        trr.trr_kv_read(None, 0, ids[:1], ids[:1], offsets, rows, rows.float(), None)
