"""Which rows the workgroups of rm_prompt_attention take, for offsets of any kind:
csrc/rm_slots.h, built for the host.  These need no GPU."""
import ctypes
import os
import random
import subprocess

import numpy as np
import pytest

from conftest import HERE, ROOT


@pytest.fixture(scope="module")
def slots(tmp_path_factory):
    to = str(tmp_path_factory.mktemp("slots") / "prompt_slots.so")
    subprocess.run(["g++", "-O2", "-std=c++17", "-shared", "-fPIC", "-Wall", "-Werror", "-I",
                    os.path.join(ROOT, "paper_2607_16784_amd", "csrc"), "-o", to,
                    os.path.join(HERE, "prompt_slots.cpp")], check=True)
    lib = ctypes.CDLL(to)
    lib.out_of_range.restype = ctypes.c_int64
    return lib


def pointer(a):
    return a.ctypes.data_as(ctypes.c_void_p)


def out_of_range(lib, offsets, tokens, most, window, group, kv=1):
    a = np.array(offsets, np.int32)
    return lib.out_of_range(pointer(a), len(offsets) - 1, tokens, most, window, group, kv)


@pytest.mark.parametrize("offsets,tokens,window,group", [
    ([0, 1000, 1200, 500, 600, 700, 1500], 1500, 64, 4),
    ([0, 900, 1000, 0, 0, 1000], 1000, 64, 4),
    ([0, 90000, 100000, 0, 0, 100000], 100000, 64, 1),
    ([0, 2 ** 31 - 1, -2 ** 31, 200], 200, 1, 2),
    ([900, 1000, 0, -7, 1001, 20], 1000, 0, 3),
])
def test_offsets_that_decrease(slots, offsets, tokens, window, group):
    for most in (tokens, tokens // 2, 0):
        assert out_of_range(slots, offsets, tokens, most, window, group) == 0


def test_any_offsets(slots):
    rng = random.Random(1)
    for turn in range(3000):
        tokens = rng.choice([1, 5, 64, 300, 1500, 4000])
        ends = [0, tokens, -1, tokens + 1, 2 ** 31 - 1, -2 ** 31]
        offsets = [rng.choice(ends) if rng.random() < 0.1 else rng.randint(0, tokens)
                   for _ in range(rng.randint(2, 9))]
        group, kv = rng.choice([(1, 1), (4, 2), (5, 1), (40, 1), (300, 1), (3, 3)])
        most = rng.choice([tokens, tokens, rng.randint(0, tokens), 2 * tokens])
        window = rng.choice([0, 1, 40, 64, 65, 1000, 2 ** 31 - 1])
        assert out_of_range(slots, offsets, tokens, most, window, group, kv) == 0, \
            (offsets, tokens, most, window, group, kv)


def test_pairs_beyond_31_bits(slots):
    # 2^31 pairs and more in all: slots far in front of a sequence's own
    offsets = [0, 2 ** 20 - 5, 2 ** 20]
    assert out_of_range(slots, offsets, 2 ** 20, 2 ** 16, 64, 2100) == 0


def test_every_pair_is_taken_once(slots):
    rng = random.Random(2)
    for turn in range(500):
        tokens = rng.choice([1, 63, 200, 1000])
        offsets = sorted(rng.randint(-3, tokens + 3) if rng.random() < 0.1 else
                         rng.randint(0, tokens) for _ in range(rng.randint(2, 12)))
        group, kv = rng.choice([(1, 1), (4, 2), (5, 1), (130, 1)])
        most = rng.choice([tokens, tokens, rng.randint(0, tokens)])
        window = rng.choice([0, 1, 64, 100])
        a = np.array(offsets, np.int32)
        taken = np.zeros((tokens, kv * group), np.int32)
        cleared = np.zeros(tokens, np.int32)
        slots.rows_taken(pointer(a), len(offsets) - 1, tokens, most, window, group, kv,
                         pointer(taken), pointer(cleared))
        good, bad = np.zeros(tokens, bool), np.zeros(tokens, bool)
        for lo, hi in zip(offsets, offsets[1:]):
            fits = lo >= 0 and hi <= tokens and hi - lo <= most
            (good if fits else bad)[max(lo, 0):min(hi, tokens)] = True
        assert np.all(taken[good] == 1) and np.all(taken[~good] == 0), offsets
        # a row may be cleared by two parts, which share it
        assert np.all(cleared[bad] >= 1) and np.all(cleared[~bad] == 0), offsets
