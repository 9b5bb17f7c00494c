"""How the embedding gradient's chunks share out the runs of the sorted ids (csrc/grad_runs.h, compiled for
the host): a walk through the sums, the fold and the join as the kernels make it, with token numbers in the
rows' place. Every row that an id points at is written once, with the sum of all of its tokens; no partial
sum is read that the same call has not written; nothing is written outside the table."""
from __future__ import annotations

import ctypes
import subprocess
import tempfile
from pathlib import Path

import numpy as np
import pytest

CSRC = Path(__file__).resolve().parent.parent / "paper_2609_22441_amd" / "csrc"

SHIM = r"""
#include <algorithm>
#include <vector>
#include "grad_runs.h"
using namespace ccj;
struct Part { int64_t sum = 0; bool set = false; };
struct Walk {
    const uint32_t *key; int64_t n, chunk, rows; int64_t *table; int *writes; int bad = 0;
    std::vector<Part> part, folded; std::vector<int64_t> list;
    int64_t leading(int64_t i, uint32_t k, int64_t most) const {
        int64_t c = 0;
        while (c < most && i + c < n && key[i + c] == k) ++c;
        return c;
    }
    bool goes_on(int64_t i1, uint32_t k) const {
        return i1 < n && key[i1] == k && key[std::min(n, i1 + chunk) - 1] == k;
    }
    void write(uint32_t k, int64_t sum) {
        if ((int64_t)k >= rows) { bad |= 1; return; }             // outside the table
        table[k] = sum; ++writes[k];
    }
    void put(std::vector<Part> &to, int64_t at, int64_t sum) { to[at].sum = sum; to[at].set = true; }
    int64_t get(const std::vector<Part> &from, int64_t at) {
        if (!from[at].set) bad |= 2;                              // not written by this call
        return from[at].sum;
    }
    void sums(int64_t c, bool listed) {
        const int64_t start = c * chunk, stop = std::min(n, start + chunk);
        const uint32_t low = key[start], high = key[stop - 1];
        const ChunkEnds e = chunk_ends(start, stop, n, chunk, start > 0 && key[start - 1] == low,
                                       leading(start, low, chunk),
                                       stop < n ? leading(stop, high, chunk) : 0, high, rows);
        uint32_t current = key[e.i0];
        bool first = true;
        int64_t sum = 0;
        auto finish = [&](bool open) {
            if (current < (uint64_t)rows) {
                if (open) put(part, c * 2 + (first && e.head ? 0 : 1), sum);
                else write(current, sum);
            }
        };
        auto add = [&](int64_t i) {
            if (key[i] != current) { finish(first && e.head); current = key[i]; first = false; sum = 0; }
            sum += i + 1;
        };
        const int64_t even = pipelined(e);
        for (int64_t i = e.i0; i < even && key[i] < (uint64_t)rows; i += 2 * kSumAhead)
            for (int j = 0; j < 2 * kSumAhead; ++j) add(i + j);
        if (even < e.i1 && key[even] < (uint64_t)rows)
            for (int64_t i = even; i < e.i1; ++i) add(i);
        finish((first && e.head) || e.tail);
        if (e.tail && !e.head && listed && current < (uint64_t)rows) list.push_back(c);
    }
    void fold(int64_t f, int64_t chunks) {
        struct Place { int64_t at; uint32_t key; };
        std::vector<Place> places;
        const int64_t c0 = f * kFold, c1 = std::min(chunks, c0 + kFold);
        bool last_open = false;
        for (int64_t c = c0; c < c1; ++c) {
            const int64_t i0 = c * chunk, i1 = std::min(n, i0 + chunk);
            const uint32_t low = key[i0], high = key[i1 - 1];
            const bool inside = i0 > 0 && key[i0 - 1] == low && low == high, on = goes_on(i1, high);
            if (inside && low < (uint64_t)rows) places.push_back({c * 2, low});
            if (on && !inside && high < (uint64_t)rows) places.push_back({c * 2 + 1, high});
            last_open = on && high < (uint64_t)rows;
        }
        bool open = !places.empty() && places[0].at == c0 * 2;
        int64_t sum = 0;
        for (size_t p = 0; p < places.size(); ++p) {
            sum += get(part, places[p].at);
            if (p + 1 < places.size() && places[p + 1].key == places[p].key) continue;
            const bool leaves = p + 1 == places.size() && last_open;
            if (leaves && !open) list.push_back(f);
            if (open || leaves) put(folded, f * 2 + (open ? 0 : 1), sum);
            else write(places[p].key, sum);
            open = false; sum = 0;
        }
    }
    void join(const std::vector<Part> &from, int64_t step, int64_t chunks) {
        for (int64_t c : list) {
            const uint32_t k = key[std::min(n, (c + 1) * step) - 1];
            int64_t end = c, sum = 0;
            while (end + 1 < chunks && goes_on((end + 1) * step, k)) ++end;
            for (int64_t d = c; d <= end; ++d) sum += get(from, d * 2 + (d == c ? 1 : 0));
            write(k, sum);
        }
    }
};
extern "C" int walk(const uint32_t *key, int64_t n, int64_t rows, int64_t chunk, int folds, int64_t *table,
                    int *writes) {
    Walk w{key, n, chunk, rows, table, writes};
    const int64_t chunks = (n + chunk - 1) / chunk, folded = (chunks + kFold - 1) / kFold;
    w.part.resize(chunks * 2); w.folded.resize(folded * 2);
    for (int64_t c = 0; c < chunks; ++c) w.sums(c, !folds);
    for (int64_t f = 0; folds && f < folded; ++f) w.fold(f, chunks);
    if (folds) w.join(w.folded, chunk * kFold, folded); else w.join(w.part, chunk, chunks);
    return w.bad;
}
"""


@pytest.fixture(scope="module")
def walk():
    with tempfile.TemporaryDirectory() as d:
        src, out = Path(d) / "walk.cpp", Path(d) / "walk.so"
        src.write_text(SHIM)
        subprocess.run(["g++", "-std=c++17", "-O1", "-Wall", "-Werror", "-shared", "-fPIC", f"-I{CSRC}",
                        str(src), "-o", str(out)], check=True)
        lib = ctypes.CDLL(str(out))

    def call(keys, rows, chunk, folds):
        keys = np.sort(keys).astype(np.uint32)
        table, writes = np.zeros(rows, np.int64), np.zeros(rows, np.int32)
        p = lambda a: a.ctypes.data_as(ctypes.c_void_p)
        bad = lib.walk(p(keys), ctypes.c_int64(len(keys)), ctypes.c_int64(rows), ctypes.c_int64(chunk),
                       int(folds), p(table), p(writes))
        want = np.bincount(keys, weights=np.arange(1, len(keys) + 1), minlength=rows + 1)[:rows]
        count = np.bincount(keys, minlength=rows + 1)[:rows]
        assert bad == 0, ("outside the table" if bad & 1 else "") + (" unwritten sums" if bad & 2 else "")
        assert (writes == (count > 0)).all() and (table == want).all()
    return call


@pytest.mark.parametrize("folds", [False, True])
@pytest.mark.parametrize("chunk", [8, 16, 32, 64])
@pytest.mark.parametrize("kind", ["distinct", "uniform", "runs"])
def test_ids_outside_the_table_end_anywhere_in_a_chunk(walk, kind, chunk, folds):
    """Valid ids end at every place of a chunk; after them chunks wholly of ids outside the table."""
    r = np.random.default_rng(chunk)
    for valid in range(40 * chunk - 1, 42 * chunk + 2):
        n = valid + 5 * chunk + 3
        rows = {"distinct": valid, "uniform": 3 * chunk, "runs": 7}[kind]
        keys = np.arange(valid) if kind == "distinct" else r.integers(0, rows, valid)
        walk(np.concatenate([keys, np.full(n - valid, rows)]), rows, chunk, folds)


@pytest.mark.parametrize("folds", [False, True])
@pytest.mark.parametrize("chunk", [8, 16, 32])
def test_any_ids(walk, chunk, folds):
    """Runs of every length around a chunk's and a fold's, with and without ids outside the table."""
    r = np.random.default_rng(chunk + folds)
    for _ in range(400):
        lengths = r.choice([1, 2, 3, chunk - 1, chunk, chunk + 1, 2 * chunk, 3 * chunk - 1, 16 * chunk,
                            17 * chunk + 1, int(r.integers(1, 40 * chunk))], int(r.integers(1, 30)))
        rows = len(lengths) + int(r.integers(0, 3))
        ids = np.repeat(np.sort(r.choice(rows, len(lengths), replace=False)), lengths)
        walk(np.concatenate([ids, np.full(int(r.choice([0, 1, chunk, 5 * chunk + 2])), rows)]), rows,
             chunk, folds)
