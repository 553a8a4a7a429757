// Shared by the attention kernels (attention.hip, attention_bwd.hip, attention_step.hip).
//
// All of them compute scores with the keys (or queries) that stream by as rows of the matrix instruction's result and the
// wave's own queries (or keys) as its columns.  A lane then owns one column: 32x32 result register r of lane l is row
// 8 (r / 4) + 4 (l / 32) + r % 4 of column l % 32, a softmax's statistics are a lane's own numbers but for one exchange between
// the halves, and registers 8t .. 8t+7 are, packed, the right operand of the next product as they stand: its contracted index
// runs over rows in the order in which the lanes hold them, and the left operand is fetched in that same order.
#pragma once
#include "conv_common.h"
#include "sequences.h"

namespace fx {

typedef __attribute__((address_space(3))) unsigned char lds_byte;
typedef __attribute__((ext_vector_type(4))) short s16x4;
typedef __attribute__((ext_vector_type(8))) short s16x8;

constexpr float kLog2e = 1.4426950408889634f, kLn2 = 0.6931471805599453f;
constexpr int kMostDim = 256, kMostParts = 4;

template <int DT> struct AttnType;
template <> struct AttnType<FX_F32> { typedef float T; static constexpr int ES = 4; };
template <> struct AttnType<FX_F16> { typedef _Float16 T; static constexpr int ES = 2; };
template <> struct AttnType<FX_BF16> { typedef __bf16 T; static constexpr int ES = 2; };

// waves of a SIMD at least, for which registers are allotted: rows of more than 256 bytes need more than 256
constexpr int least_waves(int row_bytes) { return row_bytes > 256 ? 1 : 2; }

// The same where rows of 256 bytes take all of 256 registers, and only where the loads are dealt out over four waves nothing spills
constexpr int least_waves_of(int row_bytes, bool dealt) { return row_bytes > 256 || (row_bytes == 256 && !dealt) ? 1 : 2; }

// whether two blocks of few rows share tiles of the others: rows of 16 bits from this many bytes on; of fp32, whose products take
// longer than their loads, only the widest
constexpr bool share_tiles(int dt, int row_bytes, bool gradients) { return dt == FX_F32 ? row_bytes > 256 : row_bytes > (gradients ? 128 : 64); }

// A tensor of heads on the device: bytes from row to row and head to head
struct HeadsView { unsigned char* p; int64_t ld, hs; };

struct AttnArgs {
    HeadsView q, k, v, out, gout, gq, gk, gv;
    const SeqTile* tiles;
    const int32_t *first_q, *first_k;       // NULL: keys have the queries' sequences
    float *lse, *stats;
    const float* glse;
    int64_t rows_q;
    int32_t n_tiles, tile_rows, few, heads, kv_heads, group, dim_bytes;
    int32_t causal, order, chunk, negative;
    int32_t shares;                         // 2: two workgroups share a key's queries, and their sums are joined
    float* sums;                            // [shares, kv_heads, rows_k, gk and gv, dim]
    int64_t rows_k;
    float c;            // |scale| log2(e)
    float scale;        // |scale|
};

// ------------------------------------------------------------------ tiles in LDS
// A tile has rows of RB bytes in pieces of 16, filled by loads that write LDS directly: a load writes 1024 bytes in the order of
// its lanes, R = 1024 / RB rows, so the order of the pieces is a matter of the addresses that the lanes load from.  Segments of four
// neighbouring pieces stay together (a quad of lanes loads 64 bytes of a row); segment by segment the R rows follow each other,
// and a row's four pieces are exchanged by x -> x ^ (row / 4).  Then the operands of a matrix instruction, whose
// lanes take one piece of 32 rows, or by transposing reads 32 bytes of four, meet each bank once, and a lane's addresses
// are one of two registers plus a constant.
template <int RB> struct LdsRows {
    static constexpr int R = 1024 / RB;
    static constexpr int kPad = R == 2 ? 128 : R == 1 ? 64 : 0;         // fewer than four rows a load: those that follow lie in other banks
    static constexpr int kLoad = 1024 + kPad;
    static constexpr int kSegment = R * 64;
    static_assert(R >= 1 && R * RB == 1024, "rows fill a load");
    // row part (additive over rows that have no bit in common) and the whole place of a piece
    static __host__ __device__ constexpr int row_at(int row) { return row / R * kLoad + row % R * 64; }
    static __device__ __forceinline__ int place(int row, int piece) { return row_at(row) + (piece >> 2) * kSegment + (((piece & 3) ^ (row >> 2 & 3)) << 4); }
    static constexpr int bytes(int rows) { return rows / R * kLoad; }
};

// The loads of a tile of ROWS rows by WAVES waves; a piece behind the row's end (dim_bytes) has an offset that no buffer holds
// and comes as zeros, and so do rows that do not exist.
constexpr uint32_t kNowhere = 0x80000000u;
template <int RB, int ROWS, int WAVES> struct TileLoad {
    typedef LdsRows<RB> L;
    static constexpr int kLoads = ROWS / L::R;
    static constexpr int N = kLoads / WAVES > 0 ? kLoads / WAVES : 1;
    static_assert(kLoads % WAVES == 0 || kLoads < WAVES, "the waves load equally");
    uint32_t off[N];
    __device__ __forceinline__ void init(int wave, int lane, int64_t ld, int dim_bytes) {
#pragma unroll
        for (int i = 0; i < N; ++i) {
            const int row = (wave * N + i) * L::R + (lane >> 2) % L::R, piece = (lane / (4 * L::R)) * 4 + ((lane & 3) ^ (row >> 2 & 3));
            off[i] = piece * 16 < dim_bytes ? (uint32_t)row * (uint32_t)ld + piece * 16 : kNowhere;
        }
    }
    // rows [row0, row0 + ROWS) of the n behind `base`
    __device__ __forceinline__ void load(lds_byte* lds, const unsigned char* base, int64_t ld, int row0, int n, int dim_bytes, int wave) const {
        if (kLoads < WAVES && wave >= kLoads) return;
        const int rows = min(n - row0, ROWS);
        const uint32_t bytes = rows > 0 ? (uint32_t)(rows - 1) * (uint32_t)ld + (uint32_t)dim_bytes : 0u;
        __amdgpu_buffer_rsrc_t r = __builtin_amdgcn_make_buffer_rsrc((void*)(base + row0 * ld), 0, (int)bytes, 0x27000);
#pragma unroll
        for (int i = 0; i < N; ++i)
            __builtin_amdgcn_raw_ptr_buffer_load_lds(r, (__attribute__((address_space(3))) void*)(lds + (wave * N + i) * L::kLoad), 16, off[i], 0, 0, 0);
    }
};

// Operand whose contracted index runs along a row: lane l takes pieces 2 step + l / 32 of row l % 32 of the 32 rows from row0 on
template <int DT, int RB> struct RowReader {
    typedef LdsRows<RB> L;
    typedef typename Elem<typename AttnType<DT>::T>::vec8 vec;
    int a[2];
    __device__ __forceinline__ void init(int lane) {
#pragma unroll
        for (int s = 0; s < 2; ++s) a[s] = L::place(lane & 31, 2 * s + (lane >> 5));
    }
    __device__ __forceinline__ vec operator()(const lds_byte* tile, int row0, int step) const {
        return *(const __attribute__((address_space(3))) vec*)(tile + a[step & 1] + (step >> 1) * L::kSegment + L::row_at(row0));
    }
};

// The same straight from global memory, for the rows that a wave keeps: zeros behind the sequence and behind the row
template <int DT, int STEPS> struct OwnRows {
    typedef typename Elem<typename AttnType<DT>::T>::vec8 vec;
    vec x[STEPS];
    __device__ __forceinline__ void load(const unsigned char* base, int64_t ld, int row0, int n, int dim_bytes, int lane, bool negative = false) {
        const int rows = min(n - row0, 32);
        const uint32_t bytes = rows > 0 ? (uint32_t)(rows - 1) * (uint32_t)ld + (uint32_t)dim_bytes : 0u;
        __amdgpu_buffer_rsrc_t r = __builtin_amdgcn_make_buffer_rsrc((void*)(base + row0 * ld), 0, (int)bytes, 0x27000);
#pragma unroll
        for (int s = 0; s < STEPS; ++s) {
            const int at = (2 * s + (lane >> 5)) * 16;
            u32x4 w = __builtin_amdgcn_raw_buffer_load_b128(r, at < dim_bytes ? (lane & 31) * (uint32_t)ld + at : kNowhere, 0, 0);
            if (negative) w ^= u32x4(DT == FX_F32 ? 0x80000000u : 0x80008000u);
            __builtin_memcpy(&x[s], &w, 16);
        }
    }
};

// Of one word of a tensor: the sign bits of the values that are not finite
template <int DT> __device__ __forceinline__ uint32_t not_finite(uint32_t w) {
    if (DT == FX_F32) return ((w & 0x7F800000u) + 0x00800000u) & 0x80000000u;
    if (DT == FX_F16) return ((w & 0x7C007C00u) + 0x04000400u) & 0x80008000u;
    return ((w & 0x7F807F80u) + 0x00800080u) & 0x80008000u;
}
// zeros in the place of values that are not finite
template <int DT> __device__ __forceinline__ uint32_t finite_only(uint32_t w) {
    const uint32_t bad = not_finite<DT>(w);
    return w & ~(DT == FX_F32 ? (uint32_t)((int)bad >> 31) : (bad >> 15) * 0xFFFFu);
}
// A 32x32 result in its registers as the right operand of a product over its rows
template <int DT> struct Weights;
template <> struct Weights<FX_F32> {
    f32x16 p;
    __device__ __forceinline__ void set(const f32x16& x) { p = x; }
    __device__ __forceinline__ f32x16 rest(const f32x16&) const { return f32x16(0.f); }
};
template <int DT> struct Weights16 {
    typedef typename Elem<typename AttnType<DT>::T>::vec8 vec;
    vec p[2];
    __device__ __forceinline__ void set(const f32x16& x) {
#pragma unroll
        for (int t = 0; t < 2; ++t) {
            u32x4 w;
#pragma unroll
            for (int e = 0; e < 4; ++e) w[e] = Elem<typename AttnType<DT>::T>::pack2(x[8 * t + 2 * e], x[8 * t + 2 * e + 1]);
            __builtin_memcpy(&p[t], &w, 16);
        }
    }
    // what the rounding of x left, of an infinity nothing
    __device__ __forceinline__ f32x16 rest(const f32x16& x) const {
        f32x16 y;
#pragma unroll
        for (int r = 0; r < 16; ++r) {
            const float rounded = (float)p[r >> 3][r & 7];
            y[r] = fabsf(rounded) < INFINITY ? x[r] - rounded : 0.f;
        }
        return y;
    }
};
template <> struct Weights<FX_F16> : Weights16<FX_F16> {};
template <> struct Weights<FX_BF16> : Weights16<FX_BF16> {};

// A sum over up to so many rows takes along what the rounding of its weights left: over more their errors cancel as good as ever, in
// a product with one or two they are the result's own, beside its rounding.  What is left of a weight may be 0 or negative and meets zeros
// in the place of infinities: those are in the product with the weight itself.  In the kernels of two waves alone, which calls of short sequences
// take: in the others it costs registers that they do not have.
constexpr int kTinyRows = 16;

// acc += (columns 32 col .. 32 col + 31 of the 32 rows from row0 on)^T w, the result's rows the tile's columns
template <int DT, int RB> struct ColumnProduct {
    typedef LdsRows<RB> L;
    int a[2];
    __device__ __forceinline__ void init(int lane) {
        const int half = lane >> 5, i = lane & 15;
#pragma unroll
        for (int e = 0; e < 2; ++e) {
            // fp32: the lane's column is a word of piece (l % 32) / 4, its rows 4 half + .. of every second group of eight.
            // 16 bits: a transposing read takes 8 bytes from each of 16 lanes, four rows of 16 columns, and gives each its column's four
            if (DT == FX_F32) a[e] = L::place(8 * e + 4 * half, (lane & 31) >> 2) + (lane & 3) * 4;
            else a[e] = L::place(8 * e + 4 * half + (i >> 2), (lane >> 4 & 1) * 2 + ((i & 3) >> 1)) + (i & 1) * 8;
        }
    }
    // FINITE: with zeros in the place of what is not
    template <bool FINITE = false> __device__ __forceinline__ void operator()(f32x16& acc, const lds_byte* tile, int row0, int col, const Weights<DT>& w) const {
        if constexpr (DT == FX_F32) {
#pragma unroll
            for (int r = 0; r < 16; ++r) {
                const float x = *(const __attribute__((address_space(3))) float*)(tile + a[r >> 2 & 1] + L::row_at(row0 + 16 * (r >> 3) + (r & 3)) + col * 2 * L::kSegment);
                acc = __builtin_amdgcn_mfma_f32_32x32x2f32(x, w.p[r], acc, 0, 0, 0);
            }
        } else {
#pragma unroll
            for (int t = 0; t < 2; ++t) {
                s16x4 h[2];
#pragma unroll
                for (int e = 0; e < 2; ++e)
                    h[e] = __builtin_amdgcn_ds_read_tr16_b64_v4i16((__attribute__((address_space(3))) s16x4*)(tile + a[e] + L::row_at(row0 + 16 * t) + col * L::kSegment));
                s16x8 x = __builtin_shufflevector(h[0], h[1], 0, 1, 2, 3, 4, 5, 6, 7);
                if (FINITE) {
                    u32x4 words;
                    __builtin_memcpy(&words, &x, 16);
#pragma unroll
                    for (int e = 0; e < 4; ++e) words[e] = finite_only<DT>(words[e]);
                    __builtin_memcpy(&x, &words, 16);
                }
                typename Elem<typename AttnType<DT>::T>::vec8 f;
                __builtin_memcpy(&f, &x, 16);
                acc = Elem<typename AttnType<DT>::T>::mma(f, w.p[t], acc);
            }
        }
    }
};

// Rows of a work item: its sequence's queries and keys
struct Pair { int q0, nq, k0, nk; };
__device__ __forceinline__ Pair pair_of(const AttnArgs& a, const SeqTile& t) {         // t: a tile of queries
    if (!a.first_k) return Pair{t.first, t.len, t.first, t.len};
    const int k0 = a.first_k[t.seq];
    return Pair{t.first, t.len, k0, a.first_k[t.seq + 1] - k0};
}
__device__ __forceinline__ Pair pair_of_keys(const AttnArgs& a, const SeqTile& t) {
    if (!a.first_q) return Pair{t.first, t.len, t.first, t.len};
    const int q0 = a.first_q[t.seq];
    return Pair{q0, a.first_q[t.seq + 1] - q0, t.first, t.len};
}

// ------------------------------------------------------------------ infinities and NaN in rows that are not seen
// A causal workgroup's diagonal tiles multiply weights of 0 with rows that are not seen, and 0 times an infinity is NaN.  Its waves
// look into those tiles before they multiply, put zeros in the place of what is not finite, and go over the rows that had it
// again behind the loop, for those alone that see them: at most the diagonal tiles' rows, whatever the length.  (16,384 x 4 x 64 f16 with
// two infinities among the values: 0.37 ms as without; 138 where what they had spoilt was summed anew over all keys.)
// As many wait states as any matrix instruction needs before its result is read.  Behind a loop, whose end and branches meet: the
// compiler has counted the states of one such path and not of a shorter one.
__device__ __forceinline__ void matrix_results_ready() {
#if defined(__HIP_DEVICE_COMPILE__)
    asm volatile("s_nop 15\n\ts_nop 2");
#endif
    __builtin_amdgcn_sched_barrier(0);
}
// The lane's number, made where it is used: what hangs on it is not kept in registers through the loop
__device__ __forceinline__ int lane_here() {
    int lane = threadIdx.x & 63;
#if defined(__HIP_DEVICE_COMPILE__)
    asm volatile("" : "+v"(lane));
#endif
    return lane;
}
constexpr int kFlags = 64;              // bytes of LDS behind a kernel's own, a word for every wave

// Puts zeros in the place of what is not finite in the wave's part of a tile's rows, ROWS / WAVES of them; which of them had
// such a value, a bit for each.
template <int DT, int RB, int ROWS, int WAVES> __device__ __forceinline__ uint32_t clean_rows(lds_byte* tile, int wave) {
    typedef LdsRows<RB> L;
    constexpr int R = ROWS / WAVES, LANES = 64 / R;
    static_assert(R >= 1 && R <= 32 && LANES <= RB / 16, "a lane has pieces of one row");
    const int lane = lane_here(), row = wave * R + lane % R;
    bool any = false;
#pragma unroll 1
    for (int piece = lane / R; piece < RB / 16; piece += LANES) {
        __attribute__((address_space(3))) u32x4* at = (__attribute__((address_space(3))) u32x4*)(tile + L::place(row, piece));
        u32x4 w = *at;
        if (!(not_finite<DT>(w[0]) | not_finite<DT>(w[1]) | not_finite<DT>(w[2]) | not_finite<DT>(w[3]))) continue;
        any = true;
#pragma unroll
        for (int i = 0; i < 4; ++i) w[i] = finite_only<DT>(w[i]);
        *at = w;
    }
    asm volatile("" ::: "memory");
    uint64_t b = __ballot(any);
#pragma unroll
    for (int o = R; o < 64; o *= 2) b |= b >> o;
    return (uint32_t)b & (uint32_t)((1ull << R) - 1);
}
// The waves' answers together, a bit for each of the tile's rows.  All waves of the workgroup are here.
template <int ROWS, int WAVES> __device__ __forceinline__ uint64_t cleaned_rows(lds_byte* flags, uint32_t mine, int wave) {
    __attribute__((address_space(3))) uint32_t* f = (__attribute__((address_space(3))) uint32_t*)flags;
    if (lane_here() == 0) f[wave] = mine;
    __syncthreads();
    uint64_t all = 0;
#pragma unroll
    for (int w = 0; w < WAVES; ++w) all |= (uint64_t)(uint32_t)uni((int)f[w]) << (w * (ROWS / WAVES));
    return all;
}
// Is one of a row's values not finite?  One answer for the wave
template <int DT> __device__ __forceinline__ bool row_not_finite(const unsigned char* row, int dim_bytes, int lane) {
    bool any = false;
    for (int at = lane * 4; at < dim_bytes; at += 256) any |= not_finite<DT>(*(const uint32_t*)(row + at)) != 0;
    return __any(any);
}
// The kernel's arguments, read again from where the launch left them: a path that is hardly ever taken would else keep them
// in scalar registers through the loop
__device__ __forceinline__ const AttnArgs& args_here() {
#if defined(__HIP_DEVICE_COMPILE__)
    uint64_t p = (uint64_t)__builtin_amdgcn_kernarg_segment_ptr();
    asm volatile("" : "+s"(p));
    return *(const AttnArgs*)p;
#else
    __builtin_unreachable();
#endif
}
__device__ __forceinline__ bool finite(float x) { return fabsf(x) < INFINITY; }

// The part of a row that a 32x32 result's registers belong to (store_columns): four elements of group g of columns 32 col ..
template <int DT> struct Four {
    float x[4];
    __device__ __forceinline__ void load(const unsigned char* row, int col, int g, int dim_bytes, int half) {
        typedef typename AttnType<DT>::T T;
        const int at = (col * 32 + 8 * g + 4 * half) * AttnType<DT>::ES;
        T y[4] = {T(0.f), T(0.f), T(0.f), T(0.f)};
        if (at < dim_bytes) __builtin_memcpy(y, __builtin_assume_aligned(row + at, 4 * sizeof(T)), sizeof(y));
#pragma unroll
        for (int e = 0; e < 4; ++e) x[e] = (float)y[e];
    }
};
// acc += w row where `sees`, columns from 32 col0 on
template <int DT, int N> __device__ __forceinline__ void add_row(f32x16 (&acc)[N], const unsigned char* row, float w, bool sees, int col0, int dim_bytes, int half) {
#pragma unroll
    for (int k = 0; k < N; ++k)
#pragma unroll
        for (int g = 0; g < 4; ++g) {
            Four<DT> f;
            f.load(row, col0 + k, g, dim_bytes, half);
#pragma unroll
            for (int e = 0; e < 4; ++e) acc[k][4 * g + e] = sees ? fmaf(w, f.x[e], acc[k][4 * g + e]) : acc[k][4 * g + e];
            __builtin_amdgcn_sched_barrier(0);          // a few registers at a time
        }
}
// The product of two rows, a half of the wave every second piece of 16 bytes
template <int DT> __device__ __forceinline__ float dot_rows(const unsigned char* a, const unsigned char* b, int dim_bytes, int half) {
    typedef typename AttnType<DT>::T T;
    constexpr int PER = 16 / AttnType<DT>::ES;
    float s = 0.f;
#pragma unroll 2
    for (int at = half * 16; at < dim_bytes; at += 32) {
        T x[PER], y[PER];
        __builtin_memcpy(x, __builtin_assume_aligned(a + at, 16), 16);
        __builtin_memcpy(y, __builtin_assume_aligned(b + at, 16), 16);
#pragma unroll
        for (int e = 0; e < PER; ++e) s = fmaf((float)x[e], (float)y[e], s);
    }
    return s + __shfl_xor(s, 32, 64);
}
__device__ __forceinline__ unsigned char* row_of_head(const HeadsView& v, int64_t row, int head) { return v.p + row * v.ld + head * v.hs; }

// Writes a 32x32 result whose rows are a row's elements 32 col .. and whose columns are rows, times f
template <int DT> __device__ __forceinline__ void store_columns(const f32x16& acc, float f, unsigned char* row, int col, int dim_bytes, int half) {
    constexpr int ES = AttnType<DT>::ES;
#pragma unroll
    for (int g = 0; g < 4; ++g) {
        const int at = (col * 32 + 8 * g + 4 * half) * ES;
        if (at >= dim_bytes) continue;
        if constexpr (DT == FX_F32) {
            *(f32x4*)(row + at) = f32x4{acc[4 * g] * f, acc[4 * g + 1] * f, acc[4 * g + 2] * f, acc[4 * g + 3] * f};
        } else {
            typedef Elem<typename AttnType<DT>::T> E;
            *(u32x2*)(row + at) = u32x2{E::pack2(acc[4 * g] * f, acc[4 * g + 1] * f), E::pack2(acc[4 * g + 2] * f, acc[4 * g + 3] * f)};
        }
    }
}

__device__ __forceinline__ float other_half(float x) { return __shfl_xor(x, 32, 64); }

// The piece of work of this workgroup.  Workgroups are dealt to the eight XCDs in turn, and tiles lie from long to short: every XCD
// takes `chunk` neighbouring tiles of each 8 chunk, all heads of a tile in a row where sequences are short (the heads' parts of
// a row share lines, the tiles of a sequence its keys, in one L2), head after head where they are long (the L2 then has
// one head's keys); or, with a multiple of eight heads, all tiles of its eighth of the heads.
enum Order { kTilesFirst = 0, kHeadsFirst = 1, kHeadsApart = 2 };
struct Work { int tile, head; };            // head < 0: none
__device__ __forceinline__ Work work_of(const AttnArgs& a, int heads) {
    const uint32_t xcd = blockIdx.x % 8, tiles = (uint32_t)a.n_tiles, chunk = (uint32_t)a.chunk, per_xcd = (tiles + 8 * chunk - 1) / (8 * chunk) * chunk;
    const uint32_t slot = blockIdx.x / 8;
    Work w;
    if (a.order == kHeadsApart) {
        const uint32_t h = slot / tiles;
        return Work{(int)(slot - h * tiles), (int)(xcd * (heads / 8) + h)};
    }
    const uint32_t by = a.order == kTilesFirst ? per_xcd : heads, high = slot / by, low = slot - high * by;
    const uint32_t t = a.order == kTilesFirst ? low : high, tile = t / chunk * (8 * chunk) + xcd * chunk + t % chunk;
    w.tile = (int)tile;
    w.head = tile >= tiles ? -1 : a.order == kTilesFirst ? (int)high : (int)low;
    return w;
}
static inline unsigned work_blocks(const AttnArgs& a, int64_t heads) {
    return (unsigned)((a.order == kHeadsApart ? heads / 8 * a.n_tiles : (a.n_tiles + 8 * a.chunk - 1) / (8 * a.chunk) * a.chunk * heads) * 8);
}

// The wave's result is put into LDS by those of the upper half of W waves and taken by the lower, until wave 0 has all
template <int N> __device__ __forceinline__ void put_result(float* to, const f32x16 (&x)[N], int lane) {
#pragma unroll
    for (int c = 0; c < N; ++c)
#pragma unroll
        for (int r = 0; r < 16; ++r) to[(c * 16 + r) * 64 + lane] = x[c][r];
}

// ------------------------------------------------------------------ host
static inline int dtype_size(fx_dtype dt) { return dt == FX_F32 ? 4 : 2; }

// A tensor of heads as an entry point got it
struct HeadsTensor {
    const char* name;
    const void* p;
    int64_t ld, hs, rows;
    int32_t heads;
    bool output, needed;
    HeadsView* view;
};
fx_status check_heads(const char* who, const HeadsTensor& t, int32_t dim, int es);

// workgroups that share the queries of a tile of keys
int key_shares(const AttnArgs& a, int32_t n_tiles, int32_t few, int64_t queries, int dim, fx_dtype dt);
// a: tiles of queries, b: those of keys
void attention_bwd_launch(const AttnArgs& a, const AttnArgs& b, fx_dtype dt, int dim, bool keys, hipStream_t st);

}  // namespace fx
