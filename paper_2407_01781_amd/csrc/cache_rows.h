// Where a position of a paged cache lies, and the exponent of a row in 8 bits: plain arithmetic that the host's compiler takes
// too, so that what a wrong page or length would do is tested without a GPU.
#pragma once
#include <stdint.h>
#include <string.h>

#if defined(__HIPCC__)
#define FX_BOTH __host__ __device__ __forceinline__
#else
#define FX_BOTH inline
#endif

namespace fx {

// pos / page_rows = pos * magic >> shift for pos below 2^31: magic = floor(2^(31 + s) / d) + 1 with 2^s >= d is above the quotient
// by at most d / 2^(31 + s) of a unit for every unit of pos, less than 1 / d in all
struct PageDivision { uint32_t magic; int32_t shift; };
inline PageDivision page_division(int32_t page_rows) {
    int s = 0;
    while ((1ll << s) < page_rows) ++s;
    return PageDivision{(uint32_t)((1ull << (31 + s)) / (uint32_t)page_rows + 1), 31 + s};
}
FX_BOTH uint32_t page_column(uint32_t pos, const PageDivision& d) { return (uint32_t)(((uint64_t)pos * d.magic) >> d.shift); }

struct PageTable {
    const int32_t* table;       // [sequences, ld]
    int64_t ld;
    int32_t cols, pages, page_rows, kv_heads;
    PageDivision division;
};

// Row of the cache (over pages, heads, positions in a page) of a position whose page is known, or -1
FX_BOTH int32_t row_in_page(const PageTable& t, int32_t page, uint32_t pos, uint32_t col, int32_t head) {
    if (page < 0 || page >= t.pages) return -1;
    return (page * t.kv_heads + head) * t.page_rows + (int32_t)(pos - col * (uint32_t)t.page_rows);
}
// The same of any position of a sequence: -1 below 0, behind the table, and where the table has no page
FX_BOTH int32_t cache_row(const PageTable& t, int64_t seq, int64_t pos, int32_t head) {
    if (pos < 0 || pos > 0x7FFFFFFFll) return -1;
    const uint32_t col = page_column((uint32_t)pos, t.division);
    if (col >= (uint32_t)t.cols) return -1;
    return row_in_page(t, t.table[seq * t.ld + col], (uint32_t)pos, col, head);
}

// the least e + 127 in 0 .. 255 with top <= 448 2^e = 1.75 2^(e + 8)
FX_BOTH int exponent_of(float top) {
    uint32_t u;
    memcpy(&u, &top, 4);
    const int e = (int)(u >> 23) - 8 + ((u & 0x7FFFFF) > 0x600000u ? 1 : 0);
    return e < 0 ? 0 : e;
}

}  // namespace fx
