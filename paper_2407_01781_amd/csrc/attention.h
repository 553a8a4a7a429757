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
constexpr int kMostDim = 256;

template <int DT> struct AttnType;
template <> struct AttnType<FX_F32> { typedef float T; static constexpr int ES = 4; };
template <> struct AttnType<FX_F16> { typedef _Float16 T; static constexpr int ES = 2; };
template <> struct AttnType<FX_BF16> { typedef __bf16 T; static constexpr int ES = 2; };

// A tensor of heads on the device: bytes from row to row and head to head
struct HeadsView { unsigned char* p; int64_t ld, hs; };

struct AttnArgs {
    HeadsView q, k, v, out, gout, gq, gk, gv;
    const SeqTile* tiles;
    const int32_t *first_q, *first_k;
    float *lse, *delta;
    const float* glse;
    int64_t rows_q;
    int32_t n_tiles, heads, kv_heads, group, dim_bytes;
    int32_t causal, head_major, negative;
    float c;            // |scale| log2(e)
    float scale;        // |scale|
};

// ------------------------------------------------------------------ tiles in LDS
// ROWS rows of DP elements in pieces of 16 bytes, filled by loads that write LDS directly: lane l of a load writes 16 bytes
// at 16 l, so the pieces of a row are put in another order by the address that a lane loads from.  Piece c of row r stands
// at place c ^ mix(r): eight rows' pieces of one column, which a matrix operand's lanes fetch together, lie in different banks.
template <int RB> __device__ __forceinline__ int mix(int row) {
    constexpr int CR = RB / 16;
    if (CR >= 16) return (row & 7) << 1;
    if (CR == 8) return row & 7;
    return (row >> 1) & (CR - 1);
}
template <int RB> __device__ __forceinline__ int lds_piece(int row, int piece) { return row * RB + ((piece ^ mix<RB>(row)) << 4); }

// Offsets in the rows of global memory for the loads of a tile by WAVES waves; a piece behind the row's end (dim_bytes) has an
// offset that no buffer holds and loads as zeros.
constexpr uint32_t kNowhere = 0x80000000u;
template <int RB, int ROWS, int WAVES> struct TileLoad {
    static constexpr int N = ROWS * RB / 1024 / WAVES > 0 ? ROWS * RB / 1024 / WAVES : 1;
    static constexpr bool kAll = ROWS * RB / 1024 >= WAVES;         // every wave loads
    static_assert(ROWS * RB % 1024 == 0 && (!kAll || ROWS * RB / 1024 % WAVES == 0), "whole loads");
    uint32_t off[N];
    __device__ __forceinline__ void init(int wave, int lane, int64_t ld, int dim_bytes) {
#pragma unroll
        for (int i = 0; i < N; ++i) {
            const int at = (wave * N + i) * 1024 + lane * 16, row = at / RB, piece = ((at % RB) >> 4) ^ mix<RB>(row);
            off[i] = piece * 16 < dim_bytes ? (uint32_t)(row * (uint32_t)ld + piece * 16) : kNowhere;
        }
    }
    // rows [row0, row0 + ROWS) of `n` behind `base`; those from n on come as zeros
    __device__ __forceinline__ void load(lds_byte* lds, const unsigned char* base, int64_t ld, int row0, int n, int dim_bytes, int wave) const {
        if (!kAll && wave >= ROWS * RB / 1024) return;
        const int rows = min(n - row0, ROWS);
        const uint32_t bytes = rows > 0 ? (uint32_t)(rows - 1) * (uint32_t)ld + (uint32_t)dim_bytes : 0u;
        __amdgpu_buffer_rsrc_t r = __builtin_amdgcn_make_buffer_rsrc((void*)(base + row0 * ld), 0, (int)bytes, 0x27000);
#pragma unroll
        for (int i = 0; i < N; ++i)
            __builtin_amdgcn_raw_ptr_buffer_load_lds(r, (__attribute__((address_space(3))) void*)(lds + (wave * N + i) * 1024), 16, off[i], 0, 0, 0);
    }
};

// Left or right operand whose contracted index runs along a row: lane l takes pieces 2 step + l / 32 of row l % 32
template <int DT, int RB> __device__ __forceinline__ typename Elem<typename AttnType<DT>::T>::vec8 row_operand(const lds_byte* tile, int row, int step, int half) {
    typedef typename Elem<typename AttnType<DT>::T>::vec8 vec;
    return *(const __attribute__((address_space(3))) vec*)(tile + lds_piece<RB>(row, 2 * step + half));
}

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

// result += left^T right for 32 rows of a tile: left = columns 32 col .. 32 col + 31 of rows row0 .. row0 + 31, right = the 32x32
// result p in its registers (row as the contracted index), result row = column of left.
template <int DT> struct Weights;       // the right operand, packed
template <> struct Weights<FX_F32> {
    f32x16 p;
    __device__ __forceinline__ void set(const f32x16& x) { p = x; }
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
};
template <> struct Weights<FX_F16> : Weights16<FX_F16> {};
template <> struct Weights<FX_BF16> : Weights16<FX_BF16> {};

template <int DT, int RB> __device__ __forceinline__ void mma_columns(f32x16& acc, const lds_byte* tile, int row0, int col, const Weights<DT>& w, int lane) {
    const int half = lane >> 5;
    if constexpr (DT == FX_F32) {
        const int at = col * 128 + (lane & 31) * 4;
#pragma unroll
        for (int r = 0; r < 16; ++r) {
            const int row = row0 + 8 * (r >> 2) + 4 * half + (r & 3);
            const float a = *(const __attribute__((address_space(3))) float*)(tile + lds_piece<RB>(row, at >> 4) + (at & 15));
            acc = __builtin_amdgcn_mfma_f32_32x32x2f32(a, w.p[r], acc, 0, 0, 0);
        }
    } else {
        // a transposing read takes 8 bytes from each of 16 lanes, four rows of 16 columns, and gives lane i its column's four
        const int i = lane & 15, piece = col * 4 + ((lane >> 4) & 1) * 2 + ((i & 3) >> 1);
#pragma unroll
        for (int t = 0; t < 2; ++t) {
            s16x4 h[2];
#pragma unroll
            for (int e = 0; e < 2; ++e) {
                const int row = row0 + 16 * t + 8 * e + 4 * half + (i >> 2);
                h[e] = __builtin_amdgcn_ds_read_tr16_b64_v4i16((__attribute__((address_space(3))) s16x4*)(tile + lds_piece<RB>(row, piece) + (i & 1) * 8));
            }
            const s16x8 a = __builtin_shufflevector(h[0], h[1], 0, 1, 2, 3, 4, 5, 6, 7);
            typename Elem<typename AttnType<DT>::T>::vec8 f;
            __builtin_memcpy(&f, &a, 16);
            acc = Elem<typename AttnType<DT>::T>::mma(f, w.p[t], acc);
        }
    }
}

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

// The piece of work of this workgroup: workgroups are dealt to the eight XCDs in turn, and each XCD gets a range of neighbours
// -- the tiles of few heads, whose keys its L2 then holds, or, where sequences are short, all heads of neighbouring rows.
__device__ __forceinline__ bool work_of(const AttnArgs& a, int heads, int* tile, int* head) {
    const uint32_t total = (uint32_t)a.n_tiles * heads, per = gridDim.x / 8, item = (blockIdx.x % 8) * per + blockIdx.x / 8;
    if (item >= total) return false;
    if (a.head_major) { *head = item / a.n_tiles; *tile = item % a.n_tiles; }
    else { *tile = item / heads; *head = item % heads; }
    return true;
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

fx_status attention_bwd_launch(const AttnArgs& a, fx_dtype dt, int dim, int64_t longest_q, int64_t longest_k, const SeqTile* k_tiles, int32_t n_k_tiles, bool keys,
                               hipStream_t st);

}  // namespace fx
