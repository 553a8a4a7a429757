"""CPU-only: where a position of a paged cache lies, by the library's own arithmetic compiled for the host: pages that are none,
positions outside of the table, page sizes of every kind; and the exponents of rows in 8 bits."""
import ctypes as C
import os
import subprocess

import numpy as np
import pytest

import attention_reference as A

CSRC = os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "paper_2407_01781_amd", "csrc")
SOURCE = r"""
#include "cache_rows.h"
extern "C" void rows_of(const int32_t* table, int64_t ld, int32_t cols, int32_t pages, int32_t page_rows, int32_t kv_heads, int32_t n, const int64_t* seq,
                        const int64_t* pos, const int32_t* head, int32_t* out) {
    const fx::PageTable t{table, ld, cols, pages, page_rows, kv_heads, fx::page_division(page_rows)};
    for (int i = 0; i < n; ++i) out[i] = fx::cache_row(t, seq[i], pos[i], head[i]);
}
extern "C" void columns(int32_t page_rows, int32_t n, const uint32_t* pos, uint32_t* out) {
    const fx::PageDivision d = fx::page_division(page_rows);
    for (int i = 0; i < n; ++i) out[i] = fx::page_column(pos[i], d);
}
extern "C" void exponents(int32_t n, const float* top, int32_t* out) { for (int i = 0; i < n; ++i) out[i] = fx::exponent_of(top[i]); }
"""


@pytest.fixture(scope="module")
def lib(tmp_path_factory):
    d = tmp_path_factory.mktemp("cache_rows")
    (d / "rows.cpp").write_text(SOURCE)
    subprocess.run(["g++", "-O1", "-std=c++17", "-fsanitize=undefined", "-fno-sanitize-recover", "-shared", "-fPIC", "-I", CSRC, str(d / "rows.cpp"), "-o", str(d / "rows.so")], check=True)
    return C.CDLL(str(d / "rows.so"))


def _p(a):
    return a.ctypes.data_as(C.c_void_p)


@pytest.mark.parametrize("page_rows", [1, 2, 3, 5, 7, 16, 24, 100, 255, 256, 257, 65535, 65536, (1 << 30) - 1, 1 << 30, (1 << 30) + 1, (1 << 31) - 1])
def test_columns(lib, page_rows):
    rng = np.random.default_rng(page_rows)
    edge = np.arange(-2, 3)[None, :] + page_rows * np.unique(np.concatenate([np.arange(4), rng.integers(0, (1 << 31) // page_rows + 1, 200), [(1 << 31) // page_rows]]))[:, None]
    pos = np.concatenate([edge.ravel(), rng.integers(0, 1 << 31, 5000), [0, (1 << 31) - 1]])
    pos = pos[(pos >= 0) & (pos < 1 << 31)].astype(np.uint32)
    out = np.zeros(len(pos), np.uint32)
    lib.columns(C.c_int32(page_rows), C.c_int32(len(pos)), _p(pos), _p(out))
    assert np.array_equal(out, pos // np.uint32(page_rows))


def test_rows(lib):
    """Against the definition, with pages below 0 and behind the last, and positions below 0, behind the table and beyond 31 bits."""
    rng = np.random.default_rng(1)
    seqs, cols, ld, pages, heads = 3, 4, 6, 9, 2
    for page_rows in (1, 5, 16):
        table = rng.integers(-3, pages + 3, size=(seqs, ld)).astype(np.int32)
        table[0, 0], table[1, 1], table[2, 3] = np.iinfo(np.int32).min, np.iinfo(np.int32).max, pages
        pos = np.concatenate([np.arange(-3, cols * page_rows + 3), [1 << 31, -(1 << 40), (1 << 62), (1 << 31) - 1]]).astype(np.int64)
        seq, head = np.repeat(np.arange(seqs), len(pos)), np.tile([0, 1], seqs * len(pos))[:seqs * len(pos)].astype(np.int32)
        at = np.tile(pos, seqs)
        out = np.zeros(len(at), np.int32)
        lib.rows_of(_p(table), C.c_int64(ld), C.c_int32(cols), C.c_int32(pages), C.c_int32(page_rows), C.c_int32(heads), C.c_int32(len(at)), _p(seq.astype(np.int64)), _p(at),
                    _p(head), _p(out))
        for s, p, h, got in zip(seq, at, head, out):
            there = 0 <= p < cols * page_rows
            page = int(table[s, p // page_rows]) if there else -1
            want = (page * heads + int(h)) * page_rows + int(p) % page_rows if 0 <= page < pages else -1
            assert got == want
            assert -1 <= got < pages * heads * page_rows            # never outside of the cache


def test_exponents(lib):
    rng = np.random.default_rng(2)
    top = np.concatenate([np.exp2(rng.uniform(-149, 128, 3000)), 448.0 * np.exp2(np.arange(-140, 119)), 448.0 * np.exp2(np.arange(-130, 119)) * (1 + 2.0 ** -20),
                          [0.0, 2.0 ** -149, 2.0 ** -126, 3.4028234e38]]).astype(np.float32)
    top = top[np.isfinite(top)]
    out = np.zeros(len(top), np.int32)
    lib.exponents(C.c_int32(len(top)), _p(top), _p(out))
    assert np.array_equal(out, A.exponents(top.astype(np.float64)[:, None]))
