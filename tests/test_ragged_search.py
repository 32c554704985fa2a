"""The search that gives a block of the ragged attention its sequence, compiled for the host from the kernels' own header: every
interval has to come out with its own begin and length, for any number of sequences.  Runs without a GPU."""
import ctypes
import os
import random
import subprocess

import pytest

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))

SOURCE = r"""
#include "avion_ragged_search.h"

struct Lanes {  // an array in place of a wavefront
    const int* off;
    int S, T, border[64];
    void load(int lo, int step)
    {
        for (int l = 0; l < 64; ++l) border[l] = ragged_border(off, S, T, lo + l * step);
    }
    template <typename F>
    int count(F f) const
    {
        int n = 0;
        for (int l = 0; l < 64; ++l) n += f(l, border[l]);
        return n;
    }
    int at(int l) const { return border[l]; }
};

// The blocks of every `stride`th interval from `first` on: how many the search gives another interval, another begin, another length or
// another number to, or that lie past the end of a launch's slots
template <int SHIFT>
static int wrong(const int* off, int S, int T, int mul, int first, int stride)
{
    int bad = 0;
    const long slots = (((long)T * mul) >> SHIFT) + S + 2;
    for (int i = first; i < S + 2; i += stride) {
        const int begin = ragged_border(off, S, T, i), n = ragged_border(off, S, T, i + 1) - begin;
        const long rows = (long)n * mul, own = (rows + (1 << SHIFT) - 1) >> SHIFT, from = (((long)begin * mul) >> SHIFT) + i;
        for (long block = 0; block < own || block == 0; ++block) {
            Lanes lanes{off, S, T, {}};
            const RaggedPlace p = ragged_search<SHIFT>(lanes, S, mul, from + block);
            bad += from + block >= slots || p.i != i || p.begin != begin || p.n != n || p.block != block;
        }
    }
    return bad;
}
extern "C" int wrong_places(const int* off, int S, int T, int mul, int shift, int first, int stride)
{
    switch (shift) {
        case 0: return wrong<0>(off, S, T, mul, first, stride);
        case 5: return wrong<5>(off, S, T, mul, first, stride);
        case 6: return wrong<6>(off, S, T, mul, first, stride);
        case 7: return wrong<7>(off, S, T, mul, first, stride);
        case 8: return wrong<8>(off, S, T, mul, first, stride);
        default: return wrong<11>(off, S, T, mul, first, stride);
    }
}
// of sequences of one token each: the numbers of sequences lo .. hi - 1 (off holds 0 .. hi); the first that is wrong, or -1
extern "C" int first_wrong(const int* off, int lo, int hi, int stride)
{
    for (int S = lo; S < hi; ++S)
        if (wrong<0>(off, S, S, 1, S % stride, stride)) return S;
    return -1;
}
"""


@pytest.fixture(scope="module")
def search(tmp_path_factory):
    where = tmp_path_factory.mktemp("search")
    source, lib = where / "search.cpp", where / "search.so"
    source.write_text(SOURCE)
    subprocess.run(["g++", "-std=c++17", "-O2", "-Wall", "-Werror", "-shared", "-fPIC", "-I",
                    os.path.join(ROOT, "paper_2309_16669_amd", "csrc"), "-o", str(lib), str(source)], check=True)
    return ctypes.CDLL(str(lib))


def _array(numbers):
    return (ctypes.c_int * len(numbers))(*numbers)


def _ones(n):
    return _array(range(n + 1))


def test_every_interval_of_few_sequences(search):
    assert search.first_wrong(_ones(1500), 0, 1500, 1) == -1


@pytest.mark.parametrize("S", [3967, 3968, 3969, 4030, 4031, 4093, 4094, 4157, 4219, 4283, 4345, 5000, 6047, 6050, 6109, 16384])
def test_every_interval_of_many_sequences(search, S):
    assert search.first_wrong(_ones(S + 1), S, S + 1, 1) == -1


def test_every_number_of_sequences_up_to_20000(search):
    """All numbers, each with every 64th of its intervals from another one on; 64 in turn are all of them."""
    assert search.first_wrong(_ones(20001), 0, 20001, 64) == -1


@pytest.mark.parametrize("S", [1 << 16, 250047 - 2, 250048, 263000, 500009, (1 << 20) - 1, 1 << 20])
def test_the_most_sequences(search, S):
    """250047 = 63^3: three steps and four."""
    assert search.first_wrong(_ones(S + 1), S, S + 1, 37) == -1


@pytest.mark.parametrize("shift,mul", [(5, 1), (5, 4), (6, 8), (7, 1), (7, 8), (8, 1), (11, 1)])
@pytest.mark.parametrize("S", [0, 1, 61, 62, 63, 700, 4031, 4220, 6050])
def test_lengths_of_all_kinds(search, S, shift, mul):
    """Empty ones, one row, whole blocks and long ones, and rows before the first and behind the last."""
    rng = random.Random(S * 100 + shift)
    at, off = rng.choice((0, 5)), []
    for _ in range(S):
        off.append(at)
        at += rng.choice((0, 0, 1, 2, 31, 32, 33, 77, 128, rng.randint(0, 3000)))
    off.append(at)
    assert search.wrong_places(_array(off), S, at + rng.choice((0, 7)), mul, shift, 0, 1) == 0


def test_offsets_outside_the_tensor_are_held_inside(search):
    off = [-7] * 100 + [40, 300, 2 ** 31 - 1]
    assert search.wrong_places(_array(off), len(off) - 1, 500, 2, 5, 0, 1) == 0
