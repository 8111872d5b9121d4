"""Attention of chunks over keys that have something in common: an offset in all channels or in some, which adds the same to
all of a row's scores.  Rows are held to the library's bounds for attention, whatever the offset."""
import numpy as np
import pytest
import torch

from _shared import Holder
from paper_2607_06601_gb300 import workloads as wl
from test_gpu_chunk import LAYOUTS, check, holder

pytestmark = pytest.mark.gpu


@pytest.fixture(autouse=True)
def _gpu():
    if not torch.cuda.is_available():
        pytest.skip("needs a GPU")
    torch.cuda.set_device(0)


def keys(rng, h, n, kind):
    """Keys of standard deviation 1 (20 where the offset is 3000) and the widths that leave them so."""
    k = rng.standard_normal((n, h.Hkv, h.d))
    bits = rng.choice([2, 4, 8, 16], n)
    if kind == "all":
        k += 50.0
    elif kind == "one head":
        k[:, 0] -= 50.0
    elif kind == "channels":
        k += 40.0 * rng.standard_normal((h.Hkv, h.d))
        bits = rng.choice([8, 16], n)  # (a group's range is that of its channels: fewer bits leave steps of 10 and more)
    elif kind == "two channels":
        k[:, :, 3] += 100.0
        k[:, :, 10] -= 60.0
        bits = rng.choice([8, 16], n)
    elif kind == "large":
        k = 20.0 * k + 3000.0
    return wl.bf16_bits(k.astype(np.float32)), bits


@pytest.mark.parametrize("lay", LAYOUTS)
@pytest.mark.parametrize("kind", ["all", "one head", "channels", "two channels", "large"])
def test_keys_with_an_offset(lay, kind):
    rng = np.random.default_rng([1, len(kind), ord(kind[0])])
    h = holder(lay)
    n, new = 600, 150
    k, bits = keys(rng, h, n, kind)
    h.append(rng, 0, 1, np.arange(n), k=k, bits=bits)
    scale = 0.002 if kind == "large" else 0.0
    check(h, rng, [1, 1, 1], [n - new, 200, 0], [new, 30, 1], rng.choice(3, new + 31), rng.integers(1, 400, new + 31), 5, scale=scale)


def test_chunks_with_and_without_an_offset_in_one_call():
    rng = np.random.default_rng(2)
    h = holder(LAYOUTS[2], S=4)
    for s, kind in enumerate(["all", "none", "one head", "channels"]):
        k, bits = keys(rng, h, 400, kind)
        h.append(rng, 0, s, np.arange(400), k=k, bits=bits)
    lens = [100, 140, 3, 60]
    n = sum(lens)
    for _ in range(2):
        check(h, rng, [0, 1, 2, 3], [300, 200, 390, 340], lens, rng.choice(3, n), rng.integers(1, 300, n), 2)


def test_long_pasts_cut_between_runs():
    """Segments of 60 tiles, whose pieces are joined: the offset is added once."""
    rng = np.random.default_rng(3)
    n, new = 5000, 40
    h = Holder(1, 1, 8, 2, 64, 64, 32, n, [n // 32 + 2] * 4, archive=6)
    for at in range(0, n, 1000):
        k, bits = keys(rng, h, 1000, "all")
        h.append(rng, 0, 0, np.arange(at, at + 1000), k=k, bits=bits)
    check(h, rng, [0], [n - new], [new], [2] * new, [1] * new)


def test_a_key_far_from_the_offset():
    """Less the offset, one key is more than binary16 holds."""
    rng = np.random.default_rng(4)
    h = holder(LAYOUTS[0])
    n, new = 300, 90
    k = 20000.0 + 100.0 * rng.standard_normal((n, h.Hkv, h.d))
    k[137, 1, 7] = -60000.0
    h.append(rng, 0, 0, np.arange(n), k=wl.bf16_bits(k.astype(np.float32)), bits=np.full(n, 16), p_skip=0.0)
    check(h, rng, [0], [n - new], [new], rng.choice([1, 2], new), rng.integers(1, 200, new), 1, scale=2.0 ** -13)


def test_few_tokens():
    """One to nine of them, whose samples are the same tokens."""
    rng = np.random.default_rng(5)
    h = holder(LAYOUTS[1], S=9)
    for s in range(9):
        k, bits = keys(rng, h, s + 1, "all")
        h.append(rng, 0, s, np.arange(s + 1), k=k, bits=bits, p_skip=0.0)
    lens = [*range(1, 10)]
    check(h, rng, [*range(9)], [0] * 9, lens, [2] * 45, [1] * 45)


@pytest.mark.parametrize("lay", [dict(Hq=8, Hkv=8, d=128, G=64, P=16), dict(Hq=16, Hkv=8, d=64, G=32, P=32)])
def test_more_segments_than_shares(lay):
    """Segments that one CTA has whole beside others that are cut; keys with an offset, values with small channels, both and
    neither, sequence by sequence; with rows that see nothing."""
    rng = np.random.default_rng(6)
    S, n, new = 24, 260, 20
    h = holder(lay, S=S, maxctx=300, caps=S * 10, archive=S + 1)
    for s in range(S):
        k, bits = keys(rng, h, n, "all" if s % 2 else "none")
        v = rng.standard_normal((n, h.Hkv, h.d))
        if s % 4 > 1:
            v[:, :, ::3] *= 2.0 ** -22
            bits[:] = 16
        h.append(rng, 0, s, np.arange(20, 20 + n), k=k, v=wl.bf16_bits(v.astype(np.float32)), bits=bits)
    starts = [20 + n - new - (s % 5) * 50 for s in range(S)]
    starts[3], starts[7] = 5, 0
    check(h, rng, [*range(S)], starts, [new] * S, rng.choice(3, S * new, p=[.1, .4, .5]), rng.integers(1, 300, S * new), 0)
