// The paged cache of keys and values, and attention of one new row of each of many running sequences over it.
#include "attention.h"
#include "cache_rows.h"

#include <math.h>
#include <type_traits>

namespace fx {

typedef __attribute__((ext_vector_type(2))) float f32v2;

struct CacheArgs {
    unsigned char *k, *v;
    uint8_t *k_exp, *v_exp;
    const int32_t* start;               // of the rows written or read, or the lengths of a step
    PageTable t;
    int32_t dim, pitch;
};

// e4m3 code of x, which is at most 448 in size or NaN
__device__ __forceinline__ uint32_t to_e4m3(float a, float b) { return __builtin_amdgcn_cvt_pk_fp8_f32(a, b, 0, false) & 0xFFFF; }

// Eight elements of a row and head are a lane's; the lanes of a row (a power of two) find its largest value by shuffles.  Bound
// by HBM: sixteen bytes in and eight to sixteen out a lane, keys and values in one thread so that two loads are in flight.
struct CacheRows {
    const int32_t* first;           // sequences, or NULL: a row of each
    int32_t n_seqs, lanes_log2;
    int64_t rows;
    HeadsView k, v;
};

// Row r's place in the cache (row over pages, heads and positions), or -1
__device__ __forceinline__ int64_t place_of(const CacheArgs& c, const CacheRows& a, int64_t r, int head) {
    int64_t seq = r, in = 0;
    if (a.first) {
        int lo = 0, hi = a.n_seqs;              // the last sequence that begins at r or before: the one that has row r
        while (hi - lo > 1) { const int mid = (lo + hi) / 2; if (a.first[mid] <= r) lo = mid; else hi = mid; }
        seq = lo;
        in = r - a.first[lo];
    }
    return cache_row(c.t, seq, (int64_t)c.start[seq] + in, head);
}

// N elements of type T, at once where VEC, else those below n one by one and zeros
template <typename T, bool VEC> __device__ __forceinline__ void take8(T* x, const T* p, int n) {
    if (VEC) {
#pragma unroll
        for (int i = 0; i < (int)sizeof(T) / 2; ++i) ((u32x4*)x)[i] = n > 0 ? ((const u32x4*)p)[i] : u32x4(0u);
    } else {
#pragma unroll
        for (int e = 0; e < 8; ++e) x[e] = e < n ? p[e] : T(0.f);
    }
}
template <typename T, bool VEC> __device__ __forceinline__ void put8(T* p, const T* x, int n) {
    if (VEC) {
        if (n > 0)
#pragma unroll
            for (int i = 0; i < (int)sizeof(T) / 2; ++i) ((u32x4*)p)[i] = ((const u32x4*)x)[i];
    } else {
#pragma unroll
        for (int e = 0; e < 8; ++e)
            if (e < n) p[e] = x[e];
    }
}

template <int DT, bool E4M3, bool VEC>
__global__ __launch_bounds__(256) void k_cache_write(CacheArgs c, CacheRows a) {
    typedef typename AttnType<DT>::T T;
    const int lanes = 1 << a.lanes_log2, d = (threadIdx.x & (lanes - 1)) * 8;
    const int64_t unit = ((int64_t)blockIdx.x * 256 + threadIdx.x) >> a.lanes_log2, all = a.rows * c.t.kv_heads;
    const int64_t u = min(unit, all - 1), r = u / c.t.kv_heads;       // lanes without a row take part in the shuffles
    const int head = (int)(u - r * c.t.kv_heads);
    __attribute__((aligned(16))) T both[2][8];
    take8<T, VEC>(both[0], (const T*)(a.k.p + r * a.k.ld + head * a.k.hs) + d, c.dim - d);
    take8<T, VEC>(both[1], (const T*)(a.v.p + r * a.v.ld + head * a.v.hs) + d, c.dim - d);
    const int64_t at = place_of(c, a, r, head);
#pragma unroll
    for (int which = 0; which < 2; ++which) {
        const T* x = both[which];
        unsigned char* to = (which ? c.v : c.k) + (at * c.pitch + d) * (E4M3 ? 1 : AttnType<DT>::ES);
        const bool write = unit < all && at >= 0 && d < c.pitch;
        if (E4M3) {
            float f[8], top = 0.f;
#pragma unroll
            for (int e = 0; e < 8; ++e) {
                f[e] = (float)x[e];
                top = isfinite(f[e]) ? fmaxf(top, fabsf(f[e])) : top;
            }
            for (int o = 1; o < lanes; o *= 2) top = fmaxf(top, __shfl_xor(top, o, 64));
            const int ex = exponent_of(top);
#pragma unroll
            for (int e = 0; e < 8; ++e) f[e] = isfinite(f[e]) ? ldexpf(f[e], 127 - ex) : NAN;
            if (write) {
                *(u32x2*)to = u32x2{to_e4m3(f[0], f[1]) | to_e4m3(f[2], f[3]) << 16, to_e4m3(f[4], f[5]) | to_e4m3(f[6], f[7]) << 16};
                if (d == 0) (which ? c.v_exp : c.k_exp)[at] = (uint8_t)ex;
            }
        } else if (write) {
            put8<T, true>((T*)to, x, 8);
        }
    }
}

template <int DT, bool E4M3, bool VEC>
__global__ __launch_bounds__(256) void k_cache_read(CacheArgs c, CacheRows a) {
    typedef typename AttnType<DT>::T T;
    const int lanes = 1 << a.lanes_log2, d = (threadIdx.x & (lanes - 1)) * 8;
    const int64_t u = ((int64_t)blockIdx.x * 256 + threadIdx.x) >> a.lanes_log2, r = u / c.t.kv_heads;
    if (r >= a.rows || d >= c.dim) return;
    const int head = (int)(u - r * c.t.kv_heads);
    const int64_t at = place_of(c, a, r, head);
#pragma unroll
    for (int which = 0; which < 2; ++which) {
        const HeadsView s = which ? a.v : a.k;
        __attribute__((aligned(16))) T x[8];
        const unsigned char* from = (which ? c.v : c.k) + (at * c.pitch + d) * (E4M3 ? 1 : AttnType<DT>::ES);
        if (E4M3) {
            u32x2 w = u32x2(0u);
            int ex = 127;
            if (at >= 0) { w = *(const u32x2*)from; ex = (which ? c.v_exp : c.k_exp)[at]; }
#pragma unroll
            for (int e = 0; e < 4; ++e) {
                const f32v2 f = e & 1 ? __builtin_amdgcn_cvt_pk_f32_fp8((int)w[e >> 1], true) : __builtin_amdgcn_cvt_pk_f32_fp8((int)w[e >> 1], false);
                x[2 * e] = (T)ldexpf(f[0], ex - 127);
                x[2 * e + 1] = (T)ldexpf(f[1], ex - 127);
            }
        } else {
            take8<T, true>(x, (const T*)from, at >= 0 ? 8 : 0);
        }
        put8<T, VEC>((T*)(s.p + r * s.ld + head * s.hs) + d, x, c.dim - d);
    }
}

// ------------------------------------------------------------------ step
// One new row of every sequence over its pages.  A workgroup takes one key head of one sequence, up to 16 of its query heads,
// and a chunk of positions; each of its W waves takes every W-th tile of 32 positions and needs no other until the end.
//   scores     two 16x16 results, keys as rows and query heads as columns: lane l holds keys 4 (l / 16) + r of head l % 16.  A lane loads
//              16 bytes of the keys l % 16, the contracted dimensions in whatever order makes a load: the query's are in the same.
//   out        dimensions as rows, heads as columns, over the 32 keys in the order in which the lanes hold their weights.  A lane loads
//              VE neighbouring dimensions of each of its eight keys -- sixteen lanes a whole row -- and turns the 8 x VE block by byte
//              permutes into VE operands, dimension VE (l % 16) + j for the j-th.  Nothing of keys or values passes through LDS.
// Bound by HBM: 986,880 positions x 2 key heads x 64 bf16 in 93 us (5.4 TB/s), and 7 for the join; 64 sequences of up to 32,768 positions,
// 4 x 128 in 8 bits, in 237 us with the join (4.4 TB/s).
// Weights are split into a leading and a trailing part (three for fp32 queries over 8 bits), so that the product with 16-bit
// values loses nothing that the output would show.  fp16 ends at 2^-24: over values in it weights are taken times 2^15, and what both parts lose is 2^-40 of
// the largest.
constexpr int kStepTile = 32, kStepHeads = 16;

struct StepArgs {
    CacheArgs c;
    HeadsView q, out;
    float *lse, *part, *stats;          // part [row, head, split, pitch], stats [row, head, split, 2]: maximum (base 2), sum
    int64_t most;
    int32_t heads, group, groups, splits;
    int32_t whole;                      // queries may be loaded 16 bytes at a time
    float scale2;                       // scale log2(e)
};

// Workgroups of four waves that share a compute unit, a wave on each SIMD: registers are allotted for them
constexpr int step_resident(int dt, bool e4m3, int dp) {
    const bool wide = dt == FX_F32 && !e4m3;
    return dp > 128 ? (e4m3 && dt == FX_BF16 ? 2 : 1) : dp > 64 ? (dt == FX_F32 ? 2 : 3) : wide ? 3 : 4;
}

template <int DT, bool E4M3, int DP> struct StepShape {
    static constexpr bool kWide = DT == FX_F32 && !E4M3;           // fp32 keys and values
    static constexpr bool kF16 = DT == FX_F16 && !E4M3;            // products of fp16, of bf16 otherwise
    static constexpr int SB = E4M3 ? 1 : AttnType<DT>::ES;         // bytes of a stored element
    static constexpr int VE = DP / 16;                             // dimensions of a value's row that a lane loads
    static constexpr int KL = DP * SB / 64;                        // 16-byte loads of a key by a lane
    static constexpr int QP = !E4M3 || DT == FX_BF16 ? 1 : DT == FX_F16 ? 2 : 3;    // parts of a query
    static constexpr int PP = E4M3 && DT == FX_F32 ? 3 : 2;                        // parts of a weight
    static constexpr float kUp = kF16 ? 0x1p15f : 1.f;            // of a weight, whose own is at most 1
    static constexpr int kResident = step_resident(DT, E4M3, DP);
    // waves of a workgroup that has a sequence to itself: as many as the registers hold without spills
    static constexpr int kMany = DP > 128 ? 4 : DP > 64 || kWide || (E4M3 && DT != FX_BF16) ? 8 : 16;
};


template <bool F16> struct Mma16;
template <> struct Mma16<true> {
    typedef _Float16 T;
    typedef f16x8 vec;
    static __device__ __forceinline__ f32x4 mma(vec a, vec b, f32x4 c) { return __builtin_amdgcn_mfma_f32_16x16x32_f16(a, b, c, 0, 0, 0); }
};
template <> struct Mma16<false> {
    typedef __bf16 T;
    typedef bf16x8 vec;
    static __device__ __forceinline__ f32x4 mma(vec a, vec b, f32x4 c) { return __builtin_amdgcn_mfma_f32_16x16x32_bf16(a, b, c, 0, 0, 0); }
};

// pairs of codes, as bf16 times 2^(exponent of scale)
__device__ __forceinline__ uint32_t codes_to_bf16(uint32_t codes, float scale, bool high) {
    typedef __attribute__((ext_vector_type(2))) __bf16 bf16x2;
    const bf16x2 h = high ? __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(codes, scale, true) : __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(codes, scale, false);
    uint32_t u;
    __builtin_memcpy(&u, &h, 4);
    return u;
}

// Positions of a split: the sequence's own share, whole rounds of a workgroup's waves, and enough to be worth its beginning and end
constexpr int kLeastChunk = 256;
__device__ __forceinline__ int chunk_of(const StepArgs& a, int len) {
    return a.splits == 1 ? max(len, 1) : max(kLeastChunk, ((len - 1) / a.splits + 128) / 128 * 128);
}

template <int DT, bool E4M3, int DP, int W, int RESIDENT>
__global__ __launch_bounds__(64 * W, RESIDENT) void k_attention_step(StepArgs a) {
#if defined(__HIP_DEVICE_COMPILE__)
    typedef StepShape<DT, E4M3, DP> S;
    typedef typename AttnType<DT>::T T;
    typedef Mma16<S::kF16> M;
    constexpr int VE = S::VE, KL = S::KL, SB = S::SB, QP = S::QP, PP = S::PP;
    constexpr int VW = VE * SB >= 4 ? VE * SB / 4 : 1;             // words of a value's piece
    constexpr int KF = S::kWide ? KL : E4M3 ? 2 * KL : KL;         // operands of a key
    extern __shared__ __attribute__((aligned(16))) unsigned char smem[];
    const int wave = uni(threadIdx.x / 64), lane = threadIdx.x & 63, g = lane >> 4, m16 = lane & 15;
    uint32_t item = blockIdx.x;
    const int split = item % a.splits;
    item /= a.splits;
    const int part_of_group = item % a.groups;
    item /= a.groups;
    const int kv = item % a.c.t.kv_heads;
    const int64_t b = item / a.c.t.kv_heads;
    // row of the cache that position t + lane % 32 has, or -1; asked for one tile ahead
    const int32_t* table = a.c.t.table + b * a.c.t.ld;
    const int len = (int)max((int64_t)0, min((int64_t)a.c.start[b], a.most)), chunk = chunk_of(a, len);
    const int64_t from = (int64_t)split * chunk;
    if (a.splits > 1 && from >= len) return;           // the join knows as much
    const int end = (int)min((int64_t)len, from + chunk);
    const int first_head = kv * a.group + part_of_group * kStepHeads, n_heads = min(kStepHeads, a.group - part_of_group * kStepHeads);
    const int row_bytes = a.c.pitch * SB;

    // the queries, in the order of the keys' operands; zeros for heads and dimensions that are none
    u32x4 qw[QP][KF];
    {
        const T* qr = (const T*)(a.q.p + b * a.q.ld + (first_head + min(m16, n_heads - 1)) * a.q.hs);
        const bool some = m16 < n_heads;
#pragma unroll
        for (int f = 0; f < KF; ++f) {
            constexpr int PER = S::kWide ? 4 : 8;
            const int d0 = E4M3 ? (f >> 1) * 64 + g * 16 + (f & 1) * 8 : f * (4 * PER) + g * PER;
            float x[8];
            if (a.whole) {
                __attribute__((aligned(16))) T y[8];
                const bool there = some && d0 < a.c.dim;
#pragma unroll
                for (int i = 0; i < PER * (int)sizeof(T) / 16; ++i) ((u32x4*)y)[i] = there ? ((const u32x4*)(qr + d0))[i] : u32x4(0u);
#pragma unroll
                for (int e = 0; e < PER; ++e) x[e] = (float)y[e];
            } else {
#pragma unroll
                for (int e = 0; e < PER; ++e) x[e] = some && d0 + e < a.c.dim ? (float)qr[min(d0 + e, a.c.dim - 1)] : 0.f;
            }
            if constexpr (S::kWide) {
                qw[0][f] = u32x4{__float_as_uint(x[0]), __float_as_uint(x[1]), __float_as_uint(x[2]), __float_as_uint(x[3])};
            } else {
#pragma unroll
                for (int p = 0; p < QP; ++p) {
#pragma unroll
                    for (int e = 0; e < 4; ++e) {
                        qw[p][f][e] = Elem<typename M::T>::pack2(x[2 * e], x[2 * e + 1]);
                        if (p + 1 < QP) {
                            x[2 * e] -= Elem<typename M::T>::to_float((uint16_t)qw[p][f][e]);
                            x[2 * e + 1] -= Elem<typename M::T>::to_float((uint16_t)(qw[p][f][e] >> 16));
                        }
                    }
                }
            }
        }
    }
    f32x4 acc[VE];
#pragma unroll
    for (int j = 0; j < VE; ++j) acc[j] = f32x4(0.f);
    float top = -INFINITY, sum = 0.f;

    auto row_of = [&](int t) {
        const uint32_t pos = (uint32_t)t + (lane & 31), col = page_column(pos, a.c.t.division);
        const int page = col < (uint32_t)a.c.t.cols ? table[col] : -1;        // does not wait for the length
        return (int)pos < end ? row_in_page(a.c.t, page, pos, col, kv) : -1;
    };
    // Once; and again where the sums are not finite: an infinity among the values that are seen, times a weight's trailing part, which may
    // be 0 or negative, is not what it is times the weight.  `careful`: trailing parts meet zeros in such places.
    auto sum_up = [&](auto careful) {
    int t = (int)from + wave * kStepTile;
    int row = row_of(t);
    for (; t < end; t += W * kStepTile) {
        const uint64_t there = __ballot(row >= 0);          // both halves of the wave hold the same 32
        const int safe = max(row, 0);
        auto row_at = [&](int key) { return (int64_t)__shfl(safe, key, 64); };
        u32x4 kw[2][KL];
        float k_scale[2], v_scale[8];
        uint32_t vw[8][VW];
#pragma unroll
        for (int s = 0; s < 2; ++s) {
            const int64_t r = row_at(16 * s + m16);
            const unsigned char* p = a.c.k + r * row_bytes;
#pragma unroll
            for (int i = 0; i < KL; ++i) kw[s][i] = i * 64 + g * 16 < row_bytes ? *(const u32x4*)(p + i * 64 + g * 16) : u32x4(0u);
            if (E4M3) k_scale[s] = __uint_as_float((uint32_t)a.c.k_exp[r] << 23);
        }
#pragma unroll
        for (int i = 0; i < 8; ++i) {
            const int64_t r = row_at(16 * (i >> 2) + 4 * g + (i & 3));
            const unsigned char* p = a.c.v + r * row_bytes + m16 * VE * SB;
            if (E4M3) v_scale[i] = __uint_as_float((uint32_t)a.c.v_exp[r] << 23);
            if (m16 * VE < a.c.pitch) {
                if constexpr (VW >= 4) {
#pragma unroll
                    for (int w = 0; w < VW; w += 4) { const u32x4 x = *(const u32x4*)(p + 4 * w); vw[i][w] = x[0]; vw[i][w + 1] = x[1]; vw[i][w + 2] = x[2]; vw[i][w + 3] = x[3]; }
                } else if constexpr (VW == 2) {
                    const u32x2 x = *(const u32x2*)p;
                    vw[i][0] = x[0];
                    vw[i][1] = x[1];
                } else {
                    vw[i][0] = *(const uint32_t*)p;
                }
            } else {
#pragma unroll
                for (int w = 0; w < VW; ++w) vw[i][w] = 0;
            }
        }
        const int next = t + W * kStepTile;
        row = next < end ? row_of(next) : -1;

        float s[8];
#pragma unroll
        for (int h = 0; h < 2; ++h) {
            f32x4 r = f32x4(0.f);
            if constexpr (S::kWide) {
#pragma unroll
                for (int i = 0; i < KL; ++i)
#pragma unroll
                    for (int e = 0; e < 4; ++e) r = __builtin_amdgcn_mfma_f32_16x16x4f32(__uint_as_float(kw[h][i][e]), __uint_as_float(qw[0][i][e]), r, 0, 0, 0);
            } else {
#pragma unroll
                for (int f = 0; f < KF; ++f) {
                    u32x4 w;
                    if constexpr (E4M3) {
#pragma unroll
                        for (int e = 0; e < 4; ++e) w[e] = codes_to_bf16(kw[h][f >> 1][(f & 1) * 2 + (e >> 1)], k_scale[h], e & 1);
                    } else {
                        w = kw[h][f];
                    }
                    typename M::vec x, y;
                    __builtin_memcpy(&x, &w, 16);
#pragma unroll
                    for (int p = QP - 1; p >= 0; --p) { __builtin_memcpy(&y, &qw[p][f], 16); r = M::mma(x, y, r); }
                }
            }
#pragma unroll
            for (int e = 0; e < 4; ++e) s[4 * h + e] = r[e] * a.scale2;
        }
        if (there != ~0ull) {           // keys that are none: no score, and zeros in the place of what lies there
#pragma unroll
            for (int i = 0; i < 8; ++i)
                if (!(there >> (16 * (i >> 2) + 4 * g + (i & 3)) & 1)) {
                    s[i] = -INFINITY;
                    if (E4M3) v_scale[i] = 1.f;          // an exponent of 255 would make NaN of zeros
#pragma unroll
                    for (int w = 0; w < VW; ++w) vw[i][w] = 0;
                }
        }
        float best = fmaxf(fmaxf(fmaxf(s[0], s[1]), fmaxf(s[2], s[3])), fmaxf(fmaxf(s[4], s[5]), fmaxf(s[6], s[7])));
        best = fmaxf(best, __shfl_xor(best, 16, 64));
        best = fmaxf(best, __shfl_xor(best, 32, 64));
        if (__any(best > top)) {
            const float next_top = fmaxf(top, best), f = top == -INFINITY ? 0.f : __builtin_amdgcn_exp2f(top - next_top);
            top = next_top;
            sum *= f;
#pragma unroll
            for (int j = 0; j < VE; ++j) acc[j] *= f;
        }
        const float base = top == -INFINITY ? 0.f : top;
#pragma unroll
        for (int i = 0; i < 8; ++i) {
            s[i] = __builtin_amdgcn_exp2f(s[i] - base) * S::kUp;
            sum += s[i];
        }
        if constexpr (S::kWide) {
#pragma unroll
            for (int i = 0; i < 8; ++i)
#pragma unroll
                for (int j = 0; j < VE; ++j) acc[j] = __builtin_amdgcn_mfma_f32_16x16x4f32(__uint_as_float(vw[i][j]), s[i], acc[j], 0, 0, 0);
        } else {
            typename M::vec p[PP];
#pragma unroll
            for (int k = 0; k < PP; ++k) {
                u32x4 w;
#pragma unroll
                for (int e = 0; e < 4; ++e) {
                    w[e] = Elem<typename M::T>::pack2(s[2 * e], s[2 * e + 1]);
                    if (k + 1 < PP) {
                        s[2 * e] -= Elem<typename M::T>::to_float((uint16_t)w[e]);
                        s[2 * e + 1] -= Elem<typename M::T>::to_float((uint16_t)(w[e] >> 16));
                    }
                }
                __builtin_memcpy(&p[k], &w, 16);
            }
#pragma unroll
            for (int j = 0; j < VE; j += 2) {
                uint32_t x[8];          // dimensions j and j + 1 of the eight keys
#pragma unroll
                for (int i = 0; i < 8; ++i) x[i] = E4M3 ? codes_to_bf16(vw[i][j >> 2], v_scale[i], (j >> 1) & 1) : vw[i][j >> 1];
#pragma unroll
                for (int h = 0; h < 2; ++h) {
                    u32x4 w;
#pragma unroll
                    for (int e = 0; e < 4; ++e) w[e] = __builtin_amdgcn_perm(x[2 * e + 1], x[2 * e], h ? 0x07060302 : 0x05040100);
                    typename M::vec v, trailing;
                    __builtin_memcpy(&v, &w, 16);
                    if (decltype(careful)::value)
#pragma unroll
                        for (int e = 0; e < 4; ++e) w[e] = finite_only<S::kF16 ? FX_F16 : FX_BF16>(w[e]);
                    __builtin_memcpy(&trailing, &w, 16);
#pragma unroll
                    for (int k = PP - 1; k >= 0; --k) acc[j + h] = M::mma(k ? trailing : v, p[k], acc[j + h]);
                }
            }
        }
    }
    };
    sum_up(std::false_type{});
    if constexpr (!S::kWide) {
        bool odd = false;
#pragma unroll
        for (int j = 0; j < VE; ++j)
#pragma unroll
            for (int r = 0; r < 4; ++r) odd |= !finite(acc[j][r]);
        if (__any(odd)) {
#pragma unroll
            for (int j = 0; j < VE; ++j) acc[j] = f32x4(0.f);
            top = -INFINITY;
            sum = 0.f;
            sum_up(std::true_type{});
        }
    }
    sum += __shfl_xor(sum, 16, 64);
    sum += __shfl_xor(sum, 32, 64);
    if (S::kUp != 1.f) {
        sum *= 1.f / S::kUp;
#pragma unroll
        for (int j = 0; j < VE; ++j) acc[j] *= 1.f / S::kUp;
    }
    // the waves' results joined: three quarters of them put theirs into LDS, the others take three each
    float* shared = (float*)smem;
    constexpr int SLOT = DP * kStepHeads + 2 * kStepHeads;
#pragma unroll
    for (int left = W; left > 1;) {
        const int n = left >= 4 ? left / 4 : 1;
        if (wave >= n && wave < left) {
            float* to = shared + (wave - n) * SLOT;
#pragma unroll
            for (int j = 0; j < VE; ++j)
#pragma unroll
                for (int r = 0; r < 4; ++r) to[(j * 4 + r) * 64 + lane] = acc[j][r];
            if (g == 0) { to[DP * kStepHeads + m16] = top; to[DP * kStepHeads + kStepHeads + m16] = sum; }
        }
        __syncthreads();
        if (wave < n)
            for (int other = wave; other < left - n; other += n) {
                const float* in = shared + other * SLOT;
                const float top2 = in[DP * kStepHeads + m16], sum2 = in[DP * kStepHeads + kStepHeads + m16], both = fmaxf(top, top2);
                const float f = top == -INFINITY ? 0.f : __builtin_amdgcn_exp2f(top - both), f2 = top2 == -INFINITY ? 0.f : __builtin_amdgcn_exp2f(top2 - both);
                top = both;
                sum = sum * f + sum2 * f2;
#pragma unroll
                for (int j = 0; j < VE; ++j)
#pragma unroll
                    for (int r = 0; r < 4; ++r) acc[j][r] = acc[j][r] * f + in[(j * 4 + r) * 64 + lane] * f2;
            }
        left = n;
        if (left > 1) __syncthreads();
    }
    if (wave != 0 || m16 >= n_heads) return;
    const int head = first_head + m16;
    const float inv = sum == 0.f ? 0.f : 1.f / sum;
    T* out = (T*)(a.out.p + b * a.out.ld + head * a.out.hs);
    const int64_t slot = (b * a.heads + head) * a.splits + split;
#pragma unroll
    for (int r = 0; r < 4; ++r)
#pragma unroll
        for (int j = 0; j < VE; ++j) {
            const int d = (4 * g + r) * VE + j;
            if (d >= a.c.dim) continue;
            if (a.splits > 1) a.part[slot * a.c.pitch + d] = acc[j][r];
            else out[d] = (T)(acc[j][r] * inv);
        }
    if (g) return;
    if (a.splits > 1) { a.stats[2 * slot] = top; a.stats[2 * slot + 1] = sum; }
    else if (a.lse) a.lse[b * a.heads + head] = sum == 0.f ? -INFINITY : (top + __builtin_amdgcn_logf(sum)) * kLn2;
#endif
}

// The splits of a row and head joined: their factors in LDS, then the sums, a thread four dimensions of every n-th split
constexpr int kJoinThreads = 512, kMostSplits = 1024;
template <int DT>
__global__ __launch_bounds__(kJoinThreads) void k_attention_join(StepArgs a) {
    typedef typename AttnType<DT>::T T;
    __shared__ float f[kMostSplits], red[kJoinThreads / 64];
    __shared__ f32x4 sums[kJoinThreads];
    const int64_t item = blockIdx.x, b = item / a.heads;
    const int head = (int)(item % a.heads), tid = threadIdx.x;
    const int len = (int)max((int64_t)0, min((int64_t)a.c.start[b], a.most)), chunk = chunk_of(a, len), n = len ? (len - 1) / chunk + 1 : 0;
    const float* stats = a.stats + 2 * item * a.splits;
    float top = -INFINITY;
    for (int i = tid; i < n; i += kJoinThreads) top = fmaxf(top, stats[2 * i]);
    for (int o = 1; o < 64; o *= 2) top = fmaxf(top, __shfl_xor(top, o, 64));
    if ((tid & 63) == 0) red[tid / 64] = top;
    __syncthreads();
    for (int i = 0; i < kJoinThreads / 64; ++i) top = fmaxf(top, red[i]);
    __syncthreads();
    float sum = 0.f;
    for (int i = tid; i < n; i += kJoinThreads) {
        f[i] = stats[2 * i] == -INFINITY ? 0.f : __builtin_amdgcn_exp2f(stats[2 * i] - top);
        sum += f[i] * stats[2 * i + 1];
    }
    for (int o = 1; o < 64; o *= 2) sum += __shfl_xor(sum, o, 64);
    if ((tid & 63) == 0) red[tid / 64] = sum;
    __syncthreads();
    sum = 0.f;
    for (int i = 0; i < kJoinThreads / 64; ++i) sum += red[i];
    // as many splits side by side as there are threads for; their sums are added in order
    const int fours = a.c.pitch / 4, rows = kJoinThreads / fours, at = tid % fours, first = tid / fours;
    f32x4 acc = f32x4(0.f);
    if (first < rows) {
        const f32x4* part = (const f32x4*)(a.part + item * a.splits * a.c.pitch) + at;
#pragma unroll 8
        for (int i = first; i < n; i += rows) acc += f[i] * part[(int64_t)i * fours];
    }
    sums[tid] = acc;
    __syncthreads();
    if (tid >= fours) return;
    for (int r = 1; r < rows; ++r) acc += sums[r * fours + tid];
    T* out = (T*)(a.out.p + b * a.out.ld + head * a.out.hs) + 4 * tid;
#pragma unroll
    for (int e = 0; e < 4; ++e)
        if (4 * tid + e < a.c.dim) out[e] = (T)(sum == 0.f ? 0.f : acc[e] / sum);
    if (a.lse && tid == 0) a.lse[item] = sum == 0.f ? -INFINITY : (top + __builtin_amdgcn_logf(sum)) * kLn2;
}

template <int DT, bool E4M3, int DP> static void launch_step(const StepArgs& a, int64_t blocks, hipStream_t st) {
    constexpr int SLOT = (DP * kStepHeads + 2 * kStepHeads) * 4;
    typedef StepShape<DT, E4M3, DP> S;
    constexpr int MANY = S::kMany;
    static_assert((MANY - MANY / 4) * SLOT <= 160 * 1024, "a compute unit has 160 KiB");
    // One workgroup with many waves for each sequence only where every one of them has a compute unit to itself; more are better served by
    // four waves each, several workgroups on a unit (64 dimensions bf16, up to 300 positions, 1024 x 8 key heads: 218 -> 93 us, 256 x 4:
    // 29 -> 15; 64 x 4 of up to 1000 positions the other way: 14.2 with sixteen waves, 17.2 with four).
    if (MANY == 4 || a.splits > 1 || blocks > compute_units()) k_attention_step<DT, E4M3, DP, 4, S::kResident><<<(unsigned)blocks, 256, 3 * SLOT, st>>>(a);
    else k_attention_step<DT, E4M3, DP, MANY, 1><<<(unsigned)blocks, 64 * MANY, (MANY - MANY / 4) * SLOT, st>>>(a);
}

template <int DT, bool E4M3> static void launch_step_dim(const StepArgs& a, int64_t blocks, int64_t rows, hipStream_t st) {
    if (a.c.dim <= 64) launch_step<DT, E4M3, 64>(a, blocks, st);
    else if (a.c.dim <= 128) launch_step<DT, E4M3, 128>(a, blocks, st);
    else launch_step<DT, E4M3, 256>(a, blocks, st);
    if (a.splits > 1) k_attention_join<DT><<<(unsigned)(rows * a.heads), kJoinThreads, 0, st>>>(a);
}

// ------------------------------------------------------------------ host
static fx_status check_cache(const char* who, const fx_cache* c, fx_dtype dt, CacheArgs* a) {
    if (!c || (dt != FX_F32 && dt != FX_F16 && dt != FX_BF16) || c->kv_heads < 1 || c->dim < 1 || c->pages < 0 || c->page_rows < 1 || c->table_cols < 0 ||
        c->ld_table < c->table_cols) {
        set_error("%s: null cache, unknown dtype, or a size that is not positive", who);
        return FX_EINVAL;
    }
    if (c->store != FX_F32 && c->store != FX_F16 && c->store != FX_BF16 && c->store != FX_E4M3) { set_error("%s: unknown type of the cache", who); return FX_EINVAL; }
    if (c->store != FX_E4M3 && c->store != (int32_t)dt) { set_error("%s: rows of one type and a cache of another", who); return FX_EUNSUPPORTED; }
    if (c->dim > kMostDim) { set_error("%s: more than %d dimensions", who, kMostDim); return FX_ERANGE; }
    if (c->kv_heads > 65535) { set_error("%s: more than 65535 heads", who); return FX_ERANGE; }
    if ((int64_t)c->pages * c->page_rows > 0x7FFFFFFFll / c->kv_heads) { set_error("%s: more than 2^31-1 rows of pages and heads", who); return FX_ERANGE; }
    if (c->pages > 0 && (!c->d_k || !c->d_v || (uintptr_t)c->d_k % 16 || (uintptr_t)c->d_v % 16 || c->d_k == c->d_v)) {
        set_error("%s: d_k or d_v is null or not aligned to 16 bytes, or they are the same", who);
        return FX_EINVAL;
    }
    if (c->pages > 0 && (c->store == FX_E4M3 ? !c->d_k_exp || !c->d_v_exp || c->d_k_exp == c->d_v_exp : c->d_k_exp || c->d_v_exp)) {
        set_error("%s: exponents belong to a cache of 8 bits, one array for keys and one for values", who);
        return FX_EINVAL;
    }
    if ((c->table_cols > 0 && !c->d_table) || (uintptr_t)c->d_table % 4) { set_error("%s: d_table is null or not aligned to its elements", who); return FX_EINVAL; }
    *a = CacheArgs{(unsigned char*)c->d_k, (unsigned char*)c->d_v, c->d_k_exp, c->d_v_exp, nullptr,
                   PageTable{c->d_table, c->ld_table, c->table_cols, c->pages, c->page_rows, c->kv_heads, page_division(c->page_rows)}, c->dim,
                   (c->dim + 15) / 16 * 16};
    return FX_OK;
}

// Keys and values of a call: their views, whether they can be moved 16 bytes at a time, and the launch
static fx_status take_rows(const char* who, const HeadsTensor* t, const CacheArgs& c, fx_dtype dt, CacheRows* x, unsigned* blocks, bool* vec) {
    const int es = dtype_size(dt);
    HeadsView* view[2] = {&x->k, &x->v};
    *vec = c.dim % 8 == 0;
    for (int i = 0; i < 2; ++i) {
        *view[i] = HeadsView{(unsigned char*)t[i].p, t[i].ld * es, t[i].hs * es};
        *vec = *vec && (uintptr_t)t[i].p % 16 == 0 && view[i]->ld % 16 == 0 && (t[i].heads == 1 || view[i]->hs % 16 == 0);
    }
    while ((8 << x->lanes_log2) < c.pitch) ++x->lanes_log2;
    const int64_t threads = (x->rows * c.t.kv_heads) << x->lanes_log2;
    if (threads > (1ll << 32) - 256) { set_error("%s: too many rows for one launch", who); return FX_ERANGE; }
    *blocks = (unsigned)((threads + 255) / 256);
    return FX_OK;
}

}  // namespace fx

using namespace fx;

extern "C" fx_status fx_cache_write(const fx_cache* c, const fx_sequences* q, int64_t rows, const int32_t* d_start, fx_dtype dt, const void* d_k, int64_t ld_k,
                                    int64_t hs_k, const void* d_v, int64_t ld_v, int64_t hs_v, void* stream) {
    const char* who = "fx_cache_write";
    CacheArgs a;
    FX_TRY(check_cache(who, c, dt, &a));
    if (rows < 0 || (q && rows != q->rows)) { set_error("%s: %lld rows do not fit the sequences", who, (long long)rows); return FX_EINVAL; }
    const HeadsTensor t[] = {{"d_k", d_k, ld_k, hs_k, rows, c->kv_heads, false, true, nullptr}, {"d_v", d_v, ld_v, hs_v, rows, c->kv_heads, false, true, nullptr}};
    for (const HeadsTensor& x : t) FX_TRY(check_heads(who, x, c->dim, dtype_size(dt)));
    if (rows > 0 && (!d_start || (uintptr_t)d_start % 4)) { set_error("%s: d_start is null or not aligned to its elements", who); return FX_EINVAL; }
    if (rows > 0x7FFFFFFFll) { set_error("%s: more than 2^31-1 rows", who); return FX_ERANGE; }
    if (rows == 0 || a.t.pages == 0) return FX_OK;
    a.start = d_start;
    hipStream_t st = (hipStream_t)stream;
    ProfScope ps(kProfCache, st);
    CacheRows x{q ? q->d_first : nullptr, q ? q->B : 0, 0, rows, {}, {}};
    unsigned blocks;
    bool vec;
    FX_TRY(take_rows(who, t, a, dt, &x, &blocks, &vec));
#define FX_RUN(DT, E) do { if (vec) k_cache_write<DT, E, true><<<blocks, 256, 0, st>>>(a, x); else k_cache_write<DT, E, false><<<blocks, 256, 0, st>>>(a, x); } while (0)
#define FX_RUN_TYPES() do { const bool e = c->store == FX_E4M3; \
        if (dt == FX_F32) { if (e) FX_RUN(FX_F32, true); else FX_RUN(FX_F32, false); } \
        else if (dt == FX_F16) { if (e) FX_RUN(FX_F16, true); else FX_RUN(FX_F16, false); } \
        else { if (e) FX_RUN(FX_BF16, true); else FX_RUN(FX_BF16, false); } } while (0)
    FX_RUN_TYPES();
#undef FX_RUN
    FX_HIP_TRY(hipGetLastError());
    return FX_OK;
}

extern "C" fx_status fx_cache_read(const fx_cache* c, const fx_sequences* q, const int32_t* d_start, fx_dtype dt, void* d_k, int64_t ld_k, int64_t hs_k,
                                   void* d_v, int64_t ld_v, int64_t hs_v, void* stream) {
    const char* who = "fx_cache_read";
    CacheArgs a;
    FX_TRY(check_cache(who, c, dt, &a));
    if (!q) { set_error("%s: null sequences", who); return FX_EINVAL; }
    const int64_t rows = q->rows;
    const HeadsTensor t[] = {{"d_k", d_k, ld_k, hs_k, rows, c->kv_heads, true, true, nullptr}, {"d_v", d_v, ld_v, hs_v, rows, c->kv_heads, true, true, nullptr}};
    for (const HeadsTensor& x : t) FX_TRY(check_heads(who, x, c->dim, dtype_size(dt)));
    if (rows > 0 && d_k == d_v) { set_error("%s: d_k and d_v are the same", who); return FX_EINVAL; }
    if (rows > 0 && (!d_start || (uintptr_t)d_start % 4)) { set_error("%s: d_start is null or not aligned to its elements", who); return FX_EINVAL; }
    if (rows == 0) return FX_OK;
    a.start = d_start;
    hipStream_t st = (hipStream_t)stream;
    ProfScope ps(kProfCache, st);
    CacheRows x{q->d_first, q->B, 0, rows, {}, {}};
    unsigned blocks;
    bool vec;
    FX_TRY(take_rows(who, t, a, dt, &x, &blocks, &vec));
#define FX_RUN(DT, E) do { if (vec) k_cache_read<DT, E, true><<<blocks, 256, 0, st>>>(a, x); else k_cache_read<DT, E, false><<<blocks, 256, 0, st>>>(a, x); } while (0)
    FX_RUN_TYPES();
#undef FX_RUN
    FX_HIP_TRY(hipGetLastError());
    return FX_OK;
}

extern "C" fx_status fx_attention_step(const fx_cache* c, int64_t rows, const int32_t* d_len, int64_t most, fx_dtype dt, int32_t heads, float scale, const void* d_q,
                                       int64_t ld_q, int64_t hs_q, void* d_out, int64_t ld_out, int64_t hs_out, float* d_lse, void* stream) {
    const char* who = "fx_attention_step";
    CacheArgs a;
    FX_TRY(check_cache(who, c, dt, &a));
    if (rows < 0 || most < 0 || heads < 1 || heads % c->kv_heads || !std::isfinite(scale)) {
        set_error("%s: negative sizes, heads that are no multiple of the key heads, or a scale that is not finite", who);
        return FX_EINVAL;
    }
    if (heads > 65535) { set_error("%s: more than 65535 heads", who); return FX_ERANGE; }
    const HeadsTensor t[] = {{"d_q", d_q, ld_q, hs_q, rows, heads, false, true, nullptr}, {"d_out", d_out, ld_out, hs_out, rows, heads, true, true, nullptr}};
    for (const HeadsTensor& x : t) FX_TRY(check_heads(who, x, c->dim, dtype_size(dt)));
    if (rows > 0 && (!d_len || (uintptr_t)d_len % 4 || (uintptr_t)d_lse % 4)) { set_error("%s: d_len is null, or it or d_lse is not aligned to its elements", who); return FX_EINVAL; }
    if (rows > 0 && d_q == d_out) { set_error("%s: d_out is where d_q is", who); return FX_EINVAL; }
    if (rows > 0x7FFFFFFFll) { set_error("%s: more than 2^31-1 rows", who); return FX_ERANGE; }
    const int64_t all = (int64_t)a.t.cols * a.t.page_rows;
    if (all > 0x7FFFFFFFll - 8192) { set_error("%s: a table of more than 2^31-8193 positions", who); return FX_ERANGE; }
    if (rows == 0) return FX_OK;
    a.start = d_len;
    StepArgs s{};
    s.c = a;
    s.most = a.t.pages == 0 ? 0 : most == 0 ? all : std::min(most, all);
    hipStream_t st = (hipStream_t)stream;
    ProfScope ps(kProfAttnStep, st);
    const int es = dtype_size(dt);
    s.q = HeadsView{(unsigned char*)d_q, ld_q * es, hs_q * es};
    s.out = HeadsView{(unsigned char*)d_out, ld_out * es, hs_out * es};
    s.lse = d_lse;
    s.whole = a.dim % 8 == 0 && (uintptr_t)d_q % 16 == 0 && s.q.ld % 16 == 0 && s.q.hs % 16 == 0;
    s.heads = heads;
    s.group = heads / c->kv_heads;
    s.groups = (s.group + kStepHeads - 1) / kStepHeads;
    s.scale2 = scale * kLog2e;
    // Up to 1024 positions one workgroup takes them all and there is no second launch; beyond, every sequence is
    // split into as many parts, such that there are about eight workgroups for a compute unit -- of one sequence, as many as a
    // unit holds at a time -- where that leaves the longest 256 positions at least.  (Parts of equal length, more of them in longer sequences: 327 us for 64 sequences of up to 32,768
    // positions, 8 bits x 128, as most of two rounds of workgroups are there and the second is half empty; 32 of them for a unit 402.)  One sequence of
    // 986,880 positions x 2 x 64 bf16: 102 us with as many as are resident, 106 with eight.  A few of equal length would gain too (four of 100,000 x 4 x 128 in 8 bits 100 ->
    // 84, two of 400,000 x 2 x 64 bf16 85 -> 82), but their lengths are not known here, and of unequal ones the longest decides.
    const int64_t items = rows * c->kv_heads * s.groups;
    if (items >= (1ll << 32) / 256) { set_error("%s: too many rows for one launch", who); return FX_ERANGE; }       // threads of a launch are counted in 32 bits
    s.splits = 1;
    if (s.most > 1024)
        s.splits = (int32_t)std::max<int64_t>(1, std::min({(s.most + kLeastChunk - 1) / kLeastChunk, (int64_t)kMostSplits, (rows == 1 ? step_resident(dt, c->store == FX_E4M3, a.dim <= 64 ? 64 : a.dim <= 128 ? 128 : 256) : 8) * compute_units() / items}));
    void* part = nullptr;
    if (s.splits > 1) {
        FX_TRY(scratch_alloc(who, &part, ((size_t)rows * heads * s.splits) * (a.pitch + 2) * 4, st));
        s.part = (float*)part;
        s.stats = s.part + (size_t)rows * heads * s.splits * a.pitch;
    }
    if (c->store == FX_E4M3) {
        if (dt == FX_F32) launch_step_dim<FX_F32, true>(s, items * s.splits, rows, st);
        else if (dt == FX_F16) launch_step_dim<FX_F16, true>(s, items * s.splits, rows, st);
        else launch_step_dim<FX_BF16, true>(s, items * s.splits, rows, st);
    } else if (dt == FX_F32) launch_step_dim<FX_F32, false>(s, items * s.splits, rows, st);
    else if (dt == FX_F16) launch_step_dim<FX_F16, false>(s, items * s.splits, rows, st);
    else launch_step_dim<FX_BF16, false>(s, items * s.splits, rows, st);
    const hipError_t e = hipGetLastError();
    dev_free(part, st);
    if (e != hipSuccess) { set_error("%s: launch failed: %s", who, hipGetErrorString(e)); return FX_EDEVICE; }
    return FX_OK;
}
