"""Arithmetic of the choice among a row's keys (a plain C++ header, compiled here): rows whose last chosen key is among those of pages
that score NaN, right below 2^32, and what the kernel does with them, step by step."""
import ctypes
import os
import subprocess

import numpy as np
import pytest

CSRC = os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "paper_2303_04670_amd", "csrc")
FEW = 256  # keys of a part that are ranked at once


@pytest.fixture(scope="module")
def header(tmp_path_factory):
    d = tmp_path_factory.mktemp("cache_choice")
    (d / "c.cpp").write_text(
        '#include "cache_choice.h"\n'
        'extern "C" int shift_of(unsigned lo, unsigned hi) { return evk::part_shift({lo, hi}); }\n'
        'extern "C" int parts_of(unsigned lo, unsigned hi, int shift) { return evk::part_count({lo, hi}, shift); }\n'
        'extern "C" void part_of(unsigned lo, unsigned hi, int shift, int part, unsigned* out) {\n'
        '  const evk::KeyRange r = evk::part_range({lo, hi}, shift, part);\n  out[0] = r.lo; out[1] = r.hi;\n}\n'
        'extern "C" unsigned forced() { return evk::kForced; }\nextern "C" unsigned not_a_number() { return evk::kNotANumber; }\n')
    so = d / "c.so"
    subprocess.run(["g++", "-std=c++17", "-O1", "-Wall", "-Werror", "-shared", "-fPIC", "-I", CSRC, "-o", str(so), str(d / "c.cpp")], check=True)
    lib = ctypes.CDLL(str(so))
    lib.forced.restype = lib.not_a_number.restype = ctypes.c_uint
    return lib


def part_of(header, lo, hi, shift, part):
    out = (ctypes.c_uint * 2)()
    header.part_of(ctypes.c_uint(lo), ctypes.c_uint(hi), shift, part, out)
    return out[0], out[1]


def key_of(header, score):
    """Keys in the order of the scores."""
    u = (np.asarray(score, np.float32) + np.float32(0)).view(np.uint32)
    return np.where(np.isnan(score), np.uint32(header.not_a_number()), np.where(u >> 31, ~u, u | np.uint32(1 << 31)))


def chosen(header, keys, count):
    """The pages that are chosen: the kernel's counting, in its order."""
    keys = keys.astype(np.uint64)
    if (keys != 0).sum() <= count:
        return np.flatnonzero(keys != 0).tolist()
    others = keys[(keys != 0) & (keys != header.forced())]
    need, lo, hi = count - int((keys == header.forced()).sum()), int(others.min()), int(others.max())
    edge, equal = header.forced(), count
    while need > 0:
        shift = header.shift_of(ctypes.c_uint(lo), ctypes.c_uint(hi))
        parts = header.parts_of(ctypes.c_uint(lo), ctypes.c_uint(hi), shift)
        assert 1 <= parts <= 2048
        inside = keys[(keys >= lo) & (keys <= hi)].astype(np.int64)
        number = np.bincount((inside - lo) >> shift, minlength=parts)
        assert len(number) == parts and number.sum() >= need
        above = np.concatenate([np.cumsum(number[::-1])[::-1][1:], [0]])
        part = int(np.flatnonzero((above < need) & (above + number >= need))[0])
        need, few = need - int(above[part]), int(number[part])
        old = lo, hi
        lo, hi = part_of(header, lo, hi, shift, part)
        assert old[0] <= lo <= hi <= old[1] and ((keys >= lo) & (keys <= hi)).sum() == few, "the part has lost its keys"
        if shift == 0:
            edge, equal = lo, need
            break
        if few <= FEW:
            ranked = np.sort(keys[(keys >= lo) & (keys <= hi)])[::-1]
            edge = int(ranked[need - 1])
            equal = need - int((ranked > edge).sum())
            break
    return sorted(np.flatnonzero(keys > edge).tolist() + np.flatnonzero(keys == edge).tolist()[:equal])


@pytest.mark.parametrize("n_pages,count,first,last", [(40, 3, 1, 1), (2000, 64, 1, 1), (2000, 600, 0, 3), (15626, 128, 2, 2), (5, 2, 0, 1)])
def test_rows_with_pages_that_are_no_numbers(header, n_pages, count, first, last):
    """0, need - 1, need, need + 1 and all pages NaN, among scores of either sign, far from them and close."""
    rng = np.random.default_rng(n_pages + count)
    need = count - first - last
    for bad in sorted({0, max(need - 1, 0), need, need + 1, n_pages}):
        for scores in (rng.standard_normal(n_pages), -2.0 ** rng.integers(8, 100, n_pages), np.full(n_pages, np.finfo(np.float32).max), np.zeros(n_pages)):
            scores = scores.astype(np.float32)
            scores[first + rng.permutation(n_pages - first - last)[:bad] if bad < n_pages else slice(None)] = np.nan
            keys = key_of(header, scores)
            keys[:first] = keys[n_pages - last:] = header.forced()
            order = np.lexsort((np.arange(n_pages), -keys.astype(np.int64)))
            assert chosen(header, keys, count) == sorted(order[:count].tolist()), (bad, scores[:4])


def test_parts_cover_their_range(header):
    """Ends next to 0 and 2^32, parts of every size: neighbouring parts touch, the last one ends where the range does."""
    ends = sorted({0, 1, 2, 2047, 2048, 2049, 1 << 20, 0x007fffff, 1 << 31, (1 << 31) + 5, 0xff800000, 0xfffff7ff, 0xfffffffd, 0xfffffffe, 0xffffffff})
    for lo in ends:
        for hi in (e for e in ends if e >= lo):
            shift = header.shift_of(ctypes.c_uint(lo), ctypes.c_uint(hi))
            parts = header.parts_of(ctypes.c_uint(lo), ctypes.c_uint(hi), shift)
            assert 1 <= parts <= 2048
            at = lo
            for part in range(parts):
                a, b = part_of(header, lo, hi, shift, part)
                assert a == at and a <= b
                at = b + 1
            assert at == hi + 1
