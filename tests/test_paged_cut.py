"""The cut of paged attention calls into work items (csrc/paged_cut.h, compiled for the host): never more items than are
launched, whatever the lengths, since rows of an item past the launch would not be attended."""
import ctypes
import os
import random
import shutil
import subprocess

import pytest

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
WAVES = [256, 512, 1024, 2048, 4096]  # items that the card holds, by type and width


@pytest.fixture(scope="module")
def lib(tmp_path_factory):
    cxx = shutil.which("g++") or shutil.which("c++")
    if cxx is None:
        pytest.skip("no C++ compiler")
    so = str(tmp_path_factory.mktemp("cut") / "paged_cut.so")
    r = subprocess.run([cxx, "-std=c++17", "-O1", "-Wall", "-Wextra", "-Werror", "-fPIC", "-shared", "-I",
                        os.path.join(ROOT, "paper_2511_03092_amd", "csrc"),
                        os.path.join(ROOT, "tests", "native", "paged_cut.cpp"), "-o", so], capture_output=True, text=True)
    assert r.returncode == 0, r.stderr
    L = ctypes.CDLL(so)
    L.paged_cut_of.argtypes = [ctypes.c_int, ctypes.c_int, ctypes.c_longlong, ctypes.c_void_p]
    return L


def _items(lib, waves, heads, nb, most):
    """Items of a call whose sequences have nb blocks, and the most that are launched for `most` blocks a sequence."""
    o = (ctypes.c_int * 2)()
    lib.paged_cut_of(len(nb) * heads, waves, len(nb) * heads * most, o)
    c = lib.paged_chunk_of(waves, o[0], len(nb), heads, (ctypes.c_int * len(nb))(*nb))
    assert c >= 1
    return heads * sum(-(-x // c) for x in nb), o[1]


@pytest.mark.parametrize("waves", WAVES)
def test_never_more_items_than_are_launched(lib, waves):
    rng = random.Random(waves)
    for i in range(4000):
        heads = rng.choice((1, 2, 4, 8))
        n = rng.choice((1, 2, 3, 7, 63, 64, 65, 100, rng.randint(1, 700)))
        most = rng.choice((1, 2, 33, 250, 4096))
        kind = rng.randrange(5)
        if kind == 0:
            nb = [rng.randint(0, most) for _ in range(n)]
        elif kind == 1:  # one more than a whole number of items each
            c = rng.randint(1, max(1, most - 1))
            nb = [min(most, c * rng.randint(0, max(0, (most - 1) // c)) + 1) for _ in range(n)]
        elif kind == 2:  # a long one among short ones
            nb = [min(most, rng.randint(0, 2)) for _ in range(n)]
            nb[rng.randrange(n)] = most
        elif kind == 3:
            nb = [most] * n
        else:
            nb = [0] * n
        got, launched = _items(lib, waves, heads, nb, most)
        assert got <= launched, (heads, nb, most, got, launched)


@pytest.mark.parametrize("waves", WAVES)
def test_lengths_one_past_every_item_length(lib, waves):
    """All sequences one block past k items of C, for every C that a call of that many comes to."""
    for heads in (1, 8):
        for n in (1, 5, 64, 65, 200):
            for c in list(range(1, 40)) + [77, 128]:
                for k in (1, 2, 3):
                    nb = [c * k + 1] * n
                    got, launched = _items(lib, waves, heads, nb, nb[0])
                    assert got <= launched, (heads, n, nb[0], got, launched)


def test_the_cards_items_are_filled(lib):
    """One long sequence is cut into about as many items as the card holds."""
    for waves in WAVES:
        got, launched = _items(lib, waves, 8, [100000], 100000)
        assert 0.9 * waves <= got <= waves <= launched


def test_sizes_past_32_bits(lib):
    """The most a call may hold: 65535 units of 2^28 rows."""
    n, most = 65535, 1 << 23
    got, launched = _items(lib, 2048, 1, [most] * n, most)
    assert got <= launched
