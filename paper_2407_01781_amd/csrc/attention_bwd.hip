// Gradients of attention over packed sequences.
//
// Two kernels, each with its outputs in registers until they are whole, so that nothing is added in memory: the first goes
// over the keys for a workgroup's queries (gq) and leaves lse_i (base 2) and sum_j P_ij dP_ij - glse_i of every row for the second, which goes over
// the queries for a workgroup's keys (gk, gv).  Scores and dP are computed in both: seven products instead of five, for
// results that do not depend on an order of atomics and need no fp32 copy of gq in memory.
// P = exp(s - lse), dP = gout v^T, dS = P (dP - sum_j P dP + glse); gq = scale dS k, gk = scale dS^T q, gv = P^T gout.
// 16,384 x 16 x 128 bf16 causal: 1.46 ms for gq (1.1 PFLOP/s) and 2.13 for gk and gv with their join (1.0; LDS is read for as long as the matrix
// instructions run); 131,072 x 4 x 64 f16 in windows of 1,024: 0.29 and 0.34 ms.
#include "attention.h"

#include <limits.h>
#include <math.h>

namespace fx {

template <int DT, int DP> struct BwdShape {
    static constexpr int RB = DP * AttnType<DT>::ES;
    static constexpr int KT = RB > 128 ? 32 : 64;               // keys of a tile that streams by (two blocks' scores and dP are 64 registers)
    static constexpr int QT = RB > 128 ? 32 : 64;               // queries, a block of 32 after the other
    static constexpr int kKeys = LdsRows<RB>::bytes(KT), kQueries = LdsRows<RB>::bytes(QT), kStats = 2 * QT * 4;
    static constexpr int kFlagsKeys = 4 * kKeys, kFlagsQueries = 4 * kQueries + 2 * kStats;
    static constexpr int kLdsKeys = kFlagsKeys + kFlags, kLdsQueries = kFlagsQueries + kFlags;
    // Parts that the output's columns are dealt out in, as heads of their own: above 128 dimensions a lane's results, its own rows and
    // their products would not fit 512 registers without spills.
    static constexpr int kParts = DP > 128 ? (DT == FX_F32 ? 4 : 2) : 1;
    static constexpr int COLS = DP / 32 / kParts, STEPS = RB / 32;
    static constexpr int kPart = COLS * (DT == FX_F32 ? 2 : 1) * LdsRows<RB>::kSegment;         // from part to part in a tile
    // workgroups of RG blocks of rows, for each of which KS waves take the others' blocks in turn
    static constexpr int kBlock = LdsRows<RB>::bytes(32), kBlockStats = 32 * 8;
    static constexpr int kOwn = 2 * kBlock + kBlockStats;            // a wave's two tiles and what belongs to their rows
    template <int KS> static constexpr int buffers() { return 2 * kOwn * KS <= 128 * 1024 ? 2 : 1; }
    template <int RG, int KS> static constexpr int flags_few() { return std::max(buffers<KS>() * kOwn * KS, KS / 2 * RG * COLS * 4096); }
    template <int RG, int KS> static constexpr int lds_few() { return flags_few<RG, KS>() + kFlags; }
};

// a block's rows of 32 that do not exist: their queries are zeros, but zero times a key's infinity is none
__device__ __forceinline__ uint32_t rows_behind(int left) { return left < 32 ? ~0u << left : 0u; }
// zeros in the place of the rows of a 32x32 result that have a bit in `odd`
__device__ __forceinline__ void without(uint64_t odd, int half, f32x16& x, f32x16& y) {
    const uint32_t mine = (uint32_t)odd >> (4 * half);
#pragma unroll
    for (int r = 0; r < 16; ++r)
        if (mine >> (8 * (r >> 2) + (r & 3)) & 1) x[r] = y[r] = 0.f;
}

// ------------------------------------------------------------------ small gradients of scores in fp16
// A gradient of a score, P dP, is about the loss gradient's size over the number of keys: in fp16, whose least number is 2^-24, it
// would lose its digits or be 0 where gq and gk are far above that.  A row (of gq; a key of gk) takes its gradients of scores times a power of
// two, 2^lift, that follows the largest so far: at least 2^7 and at most 2^15, so that what is lost is 2^-32 of the largest; its sums are
// divided by it at their end.  The other types have fp32's exponents and no factor.  (131,072 x 4 x 64 in windows of 1,024: 612 us without, 631; 660 from 2^11 on,
// as it then has to come down in every other tile.)
constexpr float kMostLifted = 0x1p15f;
// A weight of gv is at most 1 and about 1 / keys: the statistics' lse is less by 15, so that weights and with them both gradients are
// 2^15 of themselves until they are stored, and what is lost of a weight is 2^-40
template <int DT> constexpr int weight_lift() { return DT == FX_F16 ? 15 : 0; }
template <int DT> constexpr int first_lift() { return DT == FX_F16 ? 60 : 0; }

// The gradients of scores of which one is too large for its lane's factor: by how much that comes down, as a power of two.  Infinities
// stay what they are and are not followed.
template <int NB> __device__ __forceinline__ int lower_by(const f32x16* x) {
    float big = 0.f;
#pragma unroll
    for (int t = 0; t < NB; ++t)
#pragma unroll
        for (int r = 0; r < 16; ++r) big = fmaxf(big, finite(x[t][r]) ? fabsf(x[t][r]) : 0.f);
    const auto halves = __builtin_amdgcn_permlane32_swap(__float_as_uint(big), __float_as_uint(big), false, false);
    big = fmaxf(__uint_as_float(halves[0]), __uint_as_float(halves[1]));
    return big > kMostLifted ? (int)(__float_as_uint(big) >> 23) - 127 - 7 : 0;
}
__device__ __forceinline__ float two_to(int e) { return __uint_as_float((uint32_t)(e + 127) << 23); }       // -126 .. 127

// ------------------------------------------------------------------ gradients of the queries
template <int DT, int DP, bool TINY = false> struct GqWave {
    typedef BwdShape<DT, DP> S;
    typedef typename AttnType<DT>::T T;
    static constexpr int RB = S::RB;
    RowReader<DT, RB> rows_of;
    ColumnProduct<DT, RB> columns;
    OwnRows<DT, S::STEPS> q, go;
    f32x16 acc[S::COLS];
    float lse2, glse, delta, c;
    int half, part, lift;
    bool one_key, one_tile, tiny;

    // A row that sees one key has dS = glse whatever it holds; the rounding of out would leave something.  Where a sequence's keys
    // are one tile, the sum over P dP is made of the tile's own numbers.
    __device__ __forceinline__ void init(const AttnArgs& a, const Pair& p, int head, int part_, int row0, int lane, int tile_keys) {
        half = lane >> 5;
        part = part_;
        c = a.c;
        const int row = row0 + (lane & 31);
        const int64_t at = head * a.rows_q + p.q0 + row;
        q.load(a.out.p + (int64_t)p.q0 * a.out.ld + head * a.out.hs, a.out.ld, row0, p.nq, a.dim_bytes, lane);
        go.load(a.gout.p + (int64_t)p.q0 * a.gout.ld + head * a.gout.hs, a.gout.ld, row0, p.nq, a.dim_bytes, lane);
        lse2 = row < p.nq ? a.lse[at] * kLog2e : INFINITY;
        glse = a.glse && row < p.nq ? a.glse[at] : 0.f;
        rows_of.init(lane);
        columns.init(lane);
        delta = 0.f;
#pragma unroll
        for (int i = 0; i < S::STEPS; ++i)
#pragma unroll
            for (int e = 0; e < 16 / AttnType<DT>::ES; ++e) delta = fmaf((float)q.x[i][e], (float)go.x[i][e], delta);
        delta += other_half(delta);
        one_key = p.nk == 1;
        one_tile = p.nk <= tile_keys;
        tiny = p.nk <= kTinyRows;
        lift = first_lift<DT>();
        if (one_key) delta = 0.f;
        if (lse2 == -INFINITY) {            // a row without a weight: whatever its gradients hold, they go nowhere
            lse2 = INFINITY;
            delta = glse = 0.f;
        }
        q.load(a.q.p + (int64_t)p.q0 * a.q.ld + head * a.q.hs, a.q.ld, row0, p.nq, a.dim_bytes, lane, a.negative);
#pragma unroll
        for (int k = 0; k < S::COLS; ++k) acc[k] = f32x16(0.f);
    }

    // odd: keys that are not finite, whose place in the tile has zeros (keys_again)
    template <int NB> __device__ __forceinline__ void blocks(const lds_byte* kt, const lds_byte* vt, int key0, bool masked, int last, uint64_t odd) {
        f32x16 p[NB], dp[NB];
        const float from = DT == FX_F16 ? (float)lift - lse2 : -lse2;         // the factor is the weights'
#pragma unroll
        for (int t = 0; t < NB; ++t) {
            p[t] = dp[t] = f32x16(0.f);
#pragma unroll
            for (int i = 0; i < S::STEPS; ++i) p[t] = Elem<T>::mma(rows_of(kt, t * 32, i), q.x[i], p[t]);
#pragma unroll
            for (int i = 0; i < S::STEPS; ++i) dp[t] = Elem<T>::mma(rows_of(vt, t * 32, i), go.x[i], dp[t]);
            if (one_key) dp[t] = f32x16(0.f);
#pragma unroll
            for (int r = 0; r < 16; ++r) p[t][r] = __builtin_amdgcn_exp2f(fmaf(p[t][r], c, from));
        }
        if (masked) {
            const int left = last - key0 - 4 * half;
#pragma unroll
            for (int t = 0; t < NB; ++t)
#pragma unroll
                for (int r = 0; r < 16; ++r)
                    if (32 * t + 8 * (r >> 2) + (r & 3) > left) p[t][r] = dp[t][r] = 0.f;
        }
        if (odd) {
#pragma unroll
            for (int t = 0; t < NB; ++t) without(odd >> (32 * t), half, p[t], dp[t]);
        }
        if (one_tile && !one_key) {
            delta = 0.f;
#pragma unroll
            for (int t = 0; t < NB; ++t)
#pragma unroll
                for (int r = 0; r < 16; ++r) delta = fmaf(p[t][r], dp[t][r], delta);
            delta += other_half(delta);
            if (DT == FX_F16) delta *= two_to(-lift);
        }
        const float off = delta - glse;
        if constexpr (DT == FX_F16) {
            float big = 0.f;
#pragma unroll
            for (int t = 0; t < NB; ++t)
#pragma unroll
                for (int r = 0; r < 16; ++r) {
                    p[t][r] *= dp[t][r] - off;
                    big = fmaxf(big, fabsf(p[t][r]));
                }
            if (__any(big > kMostLifted)) {
                const int by = lower_by<NB>(p);
                const float f = two_to(-by);
                lift -= by;
#pragma unroll
                for (int t = 0; t < NB; ++t) p[t] *= f;
#pragma unroll
                for (int k = 0; k < S::COLS; ++k) acc[k] *= f;
            }
        }
#pragma unroll
        for (int t = 0; t < NB; ++t) {
            Weights<DT> w;
            if constexpr (DT != FX_F16) {
#pragma unroll
                for (int r = 0; r < 16; ++r) p[t][r] *= dp[t][r] - off;
            }
            w.set(p[t]);
#pragma unroll
            for (int k = 0; k < S::COLS; ++k) columns(acc[k], kt + part * S::kPart, t * 32, k, w);
            if (TINY && DT != FX_F32 && tiny) {
                w.set(w.rest(p[t]));
#pragma unroll
                for (int k = 0; k < S::COLS; ++k) columns.template operator()<true>(acc[k], kt + part * S::kPart, t * 32, k, w);
            }
        }
    }

    // The keys from `from` on that are not finite, one by one: into the rows that see them (up to key `last`) alone
    __device__ __forceinline__ void keys_again(const AttnArgs& a, const Pair& p, int head, int row, int from, int end, int last) {
        const int lane = lane_here(), kv_head = head / a.group;
        const int64_t mine = p.q0 + min(row, p.nq - 1);
        for (int key = from; key < end; ++key) {
            const unsigned char* kr = row_of_head(a.k, p.k0 + key, kv_head);
            if (!row_not_finite<DT>(kr, a.dim_bytes, lane)) continue;
            const float s = dot_rows<DT>(row_of_head(a.q, mine, head), kr, a.dim_bytes, lane >> 5);
            const float dp = one_key ? 0.f : dot_rows<DT>(row_of_head(a.gout, mine, head), row_of_head(a.v, p.k0 + key, kv_head), a.dim_bytes, lane >> 5);
            const float w = __builtin_amdgcn_exp2f(fmaf(s, a.negative ? -a.c : a.c, -lse2));
            add_row<DT>(acc, kr, w * (dp - (delta - glse)), key <= last, part * S::COLS, a.dim_bytes, lane >> 5);
        }
    }

    // behind the last block
    __device__ __forceinline__ void end() {
        if constexpr (DT == FX_F16) {
#pragma unroll
            for (int k = 0; k < S::COLS; ++k) acc[k] *= two_to(-lift);
        }
    }

    __device__ __forceinline__ void store(const AttnArgs& a, const Pair& p, int head, int row) {
        if (row >= p.nq) return;
        if (half == 0 && part == 0) *(f32x2*)(a.stats + 2 * (head * a.rows_q + p.q0 + row)) = f32x2{lse2 - weight_lift<DT>(), delta - glse};
        if (!a.gq.p) return;
        unsigned char* out = a.gq.p + (int64_t)(p.q0 + row) * a.gq.ld + head * a.gq.hs;
        const float f = a.negative ? -a.scale : a.scale;
#pragma unroll
        for (int k = 0; k < S::COLS; ++k) store_columns<DT>(acc[k], f, out, part * S::COLS + k, a.dim_bytes, half);
    }
};

template <int DT, int DP, int W>
__global__ __launch_bounds__(64 * W, least_waves(DP * AttnType<DT>::ES)) void k_attention_gq(AttnArgs a) {
#if defined(__HIP_DEVICE_COMPILE__)         // the host pass has no buffer descriptors and drops stubs over them
    typedef BwdShape<DT, DP> S;
    constexpr int RB = S::RB, KT = S::KT;
    extern __shared__ __attribute__((aligned(1024))) unsigned char smem[];
    lds_byte* lds = (lds_byte*)smem;
    const Work work = work_of(a, a.heads * S::kParts);
    if (work.head < 0) return;
    const int head = work.head / S::kParts, kv_head = head / a.group;
    const int wave = uni(threadIdx.x / 64), lane = threadIdx.x & 63;
    const SeqTile st = a.tiles[work.tile];
    const Pair p = pair_of(a, st);
    const unsigned char* kb = a.k.p + (int64_t)p.k0 * a.k.ld + kv_head * a.k.hs;
    const unsigned char* vb = a.v.p + (int64_t)p.k0 * a.v.ld + kv_head * a.v.hs;
    TileLoad<RB, KT, W> lk, lv;
    lk.init(wave, lane, a.k.ld, a.dim_bytes);
    lv.init(wave, lane, a.v.ld, a.dim_bytes);
    const int row0 = st.row + wave * 32, row = row0 + (lane & 31), shift = p.nk - p.nq;
    const int seen = a.causal ? max(0, min(p.nk, min(st.row + 32 * W, p.nq) + shift)) : p.nk;
    const int seen_wave = row0 >= p.nq ? 0 : a.causal ? max(0, min(p.nk, min(row0 + 32, p.nq) + shift)) : p.nk;
    const int last = a.causal ? min(p.nk - 1, row + shift) : p.nk - 1, unmasked = a.causal ? min(p.nk - 1, row0 + shift) : p.nk - 1;
    const int n = a.gq.p || p.nk <= KT ? (seen + KT - 1) / KT : 0;          // without gq the sums alone, where they are made of the tile
    const int diagonal = a.causal ? max(0, st.row + 1 + shift) / KT : INT_MAX;      // the first tile that is not seen whole by some row of the workgroup
    if (n > 0) {
        lk.load(lds, kb, a.k.ld, 0, p.nk, a.dim_bytes, wave);
        lv.load(lds + 2 * S::kKeys, vb, a.v.ld, 0, p.nk, a.dim_bytes, wave);
    }
    GqWave<DT, DP, W == 2> w;
    w.init(a, p, head, work.head % S::kParts, row0, lane, KT);
    bool odd = false;
    for (int j = 0; j < n; ++j) {
        __builtin_amdgcn_s_waitcnt(0);
        __syncthreads();
        const int b = j & 1, key0 = j * KT;
        if (j + 1 < n) {
            lk.load(lds + (b ^ 1) * S::kKeys, kb, a.k.ld, key0 + KT, p.nk, a.dim_bytes, wave);
            lv.load(lds + (2 + (b ^ 1)) * S::kKeys, vb, a.v.ld, key0 + KT, p.nk, a.dim_bytes, wave);
        }
        uint64_t odd_keys = 0;
        if (j >= diagonal) {
            odd_keys = cleaned_rows<KT, W>(lds + S::kFlagsKeys, clean_rows<DT, RB, KT, W>(lds + b * S::kKeys, wave), wave);
            odd |= odd_keys != 0;
        }
        if (key0 >= seen_wave) continue;
        const lds_byte *kt = lds + b * S::kKeys, *vt = lds + (2 + b) * S::kKeys;
        const bool masked = key0 + KT - 1 > unmasked;
        if (KT == 64 && (W > 2 || key0 + 32 < seen_wave)) w.template blocks<2>(kt, vt, key0, masked, last, odd_keys);
        else w.template blocks<1>(kt, vt, key0, masked, last, odd_keys);
    }
    matrix_results_ready();
    w.end();
    if (odd) w.keys_again(args_here(), p, head, row, diagonal * KT, seen_wave, last);
    w.store(a, p, head, row);
#endif
}

// The results of a block's KS waves added, the upper half's by the lower until the first has all
template <int RG, int KS, int N> __device__ __forceinline__ void add_results(unsigned char* smem, f32x16 (&x)[N], int rg, int turn, int lane) {
#pragma unroll
    for (int h = KS / 2; h >= 1; h /= 2) {
        __syncthreads();
        if (turn >= h && turn < 2 * h) put_result<N>((float*)smem + ((turn - h) * RG + rg) * N * 1024, x, lane);
        __syncthreads();
        if (turn < h) {
            const float* in = (const float*)smem + (turn * RG + rg) * N * 1024;
#pragma unroll
            for (int k = 0; k < N; ++k)
#pragma unroll
                for (int r = 0; r < 16; ++r) x[k][r] += in[(k * 16 + r) * 64 + lane];
        }
    }
}

// For few queries: RG blocks of 32, for each of which KS waves take the blocks of 32 keys in turn
template <int DT, int DP, int RG, int KS>
__global__ __launch_bounds__(64 * RG * KS, least_waves(DP * AttnType<DT>::ES)) void k_attention_gq_few(AttnArgs a) {
#if defined(__HIP_DEVICE_COMPILE__)
    typedef BwdShape<DT, DP> S;
    constexpr int RB = S::RB, NB = S::template buffers<KS>();
    extern __shared__ __attribute__((aligned(1024))) unsigned char smem[];
    const Work work = work_of(a, a.heads * S::kParts);
    if (work.head < 0) return;
    const int head = work.head / S::kParts, kv_head = head / a.group;
    const int wave = uni(threadIdx.x / 64), lane = threadIdx.x & 63, rg = wave % RG, turn = wave / RG;
    lds_byte* lds = (lds_byte*)smem + turn * NB * S::kOwn;
    const SeqTile st = a.tiles[work.tile];
    const Pair p = pair_of(a, st);
    const unsigned char* kb = a.k.p + (int64_t)p.k0 * a.k.ld + kv_head * a.k.hs;
    const unsigned char* vb = a.v.p + (int64_t)p.k0 * a.v.ld + kv_head * a.v.hs;
    TileLoad<RB, 32, RG> lk, lv;
    lk.init(rg, lane, a.k.ld, a.dim_bytes);
    lv.init(rg, lane, a.v.ld, a.dim_bytes);
    const int row0 = st.row + rg * 32, row = row0 + (lane & 31), shift = p.nk - p.nq;
    const int seen = a.causal ? max(0, min(p.nk, min(st.row + 32 * RG, p.nq) + shift)) : p.nk;
    const int seen_wave = row0 >= p.nq ? 0 : a.causal ? max(0, min(p.nk, min(row0 + 32, p.nq) + shift)) : p.nk;
    const int last = a.causal ? min(p.nk - 1, row + shift) : p.nk - 1, unmasked = a.causal ? min(p.nk - 1, row0 + shift) : p.nk - 1;
    const int n = a.gq.p || p.nk <= 32 ? (seen + 31) / 32 : 0, rounds = (n + KS - 1) / KS;
    const int diagonal = a.causal ? max(0, st.row + 1 + shift) / 32 : INT_MAX;
    auto load = [&](int j, int b) {
        lk.load(lds + b * S::kOwn, kb, a.k.ld, j * 32, p.nk, a.dim_bytes, rg);
        lv.load(lds + b * S::kOwn + S::kBlock, vb, a.v.ld, j * 32, p.nk, a.dim_bytes, rg);
    };
    if (turn < n) load(turn, 0);
    GqWave<DT, DP> w;
    w.init(a, p, head, work.head % S::kParts, row0, lane, 32);
    bool odd = false;
    for (int i = 0; i < rounds; ++i) {
        const int j = i * KS + turn, b = NB == 2 ? i & 1 : 0;
        __builtin_amdgcn_s_waitcnt(0);
        if (RG > 1) __syncthreads();
        lds_byte* at = lds + b * S::kOwn;
        uint32_t odd_keys = 0;
        if (i * KS + KS > diagonal) {           // one of the turns' blocks
            odd_keys = j >= diagonal && j < n ? clean_rows<DT, RB, 32, RG>(at, rg) : 0;
            if (RG > 1) odd_keys = (uint32_t)cleaned_rows<32, RG>((lds_byte*)smem + S::template flags_few<RG, KS>() + turn * RG * 4, odd_keys, rg);
            odd |= odd_keys != 0;
        }
        if (NB == 2 && j + KS < n) load(j + KS, b ^ 1);
        if (j * 32 < seen_wave) w.template blocks<1>(at, at + S::kBlock, j * 32, j * 32 + 31 > unmasked, last, odd_keys);
        if (NB == 1) {
            __builtin_amdgcn_s_waitcnt(0);          // what is read there has been read
            if (RG > 1) __syncthreads();
            if (j + KS < n) load(j + KS, 0);
        }
    }
    matrix_results_ready();
    w.end();
    add_results<RG, KS>(smem, w.acc, rg, turn, lane);
    odd = __syncthreads_or(odd);
    if (turn == 0) {
        if (odd) w.keys_again(args_here(), p, head, row, diagonal * 32, seen_wave, last);
        w.store(a, p, head, row);
    }
#endif
}

// ------------------------------------------------------------------ gradients of keys and values
template <int DT, int DP, bool TINY = false> struct GkvWave {
    typedef BwdShape<DT, DP> S;
    typedef typename AttnType<DT>::T T;
    static constexpr int RB = S::RB;
    static constexpr float kDown = DT == FX_F16 ? 0x1p-15f : 1.f;
    static_assert(weight_lift<FX_F16>() == 15, "kDown undoes it");
    RowReader<DT, RB> rows_of;
    ColumnProduct<DT, RB> columns;
    OwnRows<DT, S::STEPS> k, v;
    f32x16 gk[S::COLS], gv[S::COLS];
    float c, lift;
    int half, part;
    bool one_key, tiny;

    __device__ __forceinline__ void init(const AttnArgs& a, const Pair& p, int kv_head, int part_, int key0, int lane) {
        half = lane >> 5;
        part = part_;
        c = a.c;
        one_key = p.nk == 1;
        tiny = p.nq * a.group <= kTinyRows;
        lift = two_to(first_lift<DT>());
        k.load(a.k.p + (int64_t)p.k0 * a.k.ld + kv_head * a.k.hs, a.k.ld, key0, p.nk, a.dim_bytes, lane, a.negative);
        v.load(a.v.p + (int64_t)p.k0 * a.v.ld + kv_head * a.v.hs, a.v.ld, key0, p.nk, a.dim_bytes, lane);
        rows_of.init(lane);
        columns.init(lane);
#pragma unroll
        for (int i = 0; i < S::COLS; ++i) gk[i] = gv[i] = f32x16(0.f);
    }

    // 32 queries whose first that sees the block's first key is `first`, counted from the block's first (all do where not masked)
    // odd: rows that are not finite, whose places in the tiles have zeros (rows_again), and those that do not exist
    __device__ __forceinline__ void block(const lds_byte* qt, const lds_byte* ot, const float* stats, bool masked, int first, uint32_t odd) {
        f32x16 p = f32x16(0.f), ds = f32x16(0.f);
#pragma unroll
        for (int i = 0; i < S::STEPS; ++i) p = Elem<T>::mma(rows_of(qt, 0, i), k.x[i], p);
#pragma unroll
        for (int i = 0; i < S::STEPS; ++i) ds = Elem<T>::mma(rows_of(ot, 0, i), v.x[i], ds);
        if (one_key) ds = f32x16(0.f);
        const float* stat = stats + 8 * half;
#pragma unroll
        for (int g = 0; g < 8; ++g) {           // lse and delta of two rows
            const f32x4 x = *(const f32x4*)(stat + 16 * (g >> 1) + 4 * (g & 1));
#pragma unroll
            for (int e = 0; e < 2; ++e) {
                const int r = 2 * g + e;
                p[r] = __builtin_amdgcn_exp2f(fmaf(p[r], c, -x[2 * e]));
                ds[r] = p[r] * (ds[r] - x[2 * e + 1]);
            }
        }
        if (masked) {
            const int lane = lane_here();
            first += (lane & 31) - 4 * (lane >> 5);
#pragma unroll
            for (int r = 0; r < 16; ++r)
                if (8 * (r >> 2) + (r & 3) < first) p[r] = ds[r] = 0.f;
        }
        if (odd) without(odd, half, p, ds);
        if constexpr (DT == FX_F16) {
            float big = 0.f;
#pragma unroll
            for (int r = 0; r < 16; ++r) {
                ds[r] *= lift;
                big = fmaxf(big, fabsf(ds[r]));
            }
            if (__any(big > kMostLifted)) {
                const float f = two_to(-lower_by<1>(&ds));
                lift *= f;
                ds *= f;
#pragma unroll
                for (int i = 0; i < S::COLS; ++i) gk[i] *= f;
            }
        }
        Weights<DT> wp, wd;
        wp.set(p);
        wd.set(ds);
#pragma unroll
        for (int i = 0; i < S::COLS; ++i) columns(gv[i], ot + part * S::kPart, 0, i, wp);
#pragma unroll
        for (int i = 0; i < S::COLS; ++i) columns(gk[i], qt + part * S::kPart, 0, i, wd);
        if (TINY && DT != FX_F32 && tiny) {
            wp.set(wp.rest(p));
            wd.set(wd.rest(ds));
#pragma unroll
            for (int i = 0; i < S::COLS; ++i) columns.template operator()<true>(gv[i], ot + part * S::kPart, 0, i, wp);
#pragma unroll
            for (int i = 0; i < S::COLS; ++i) columns.template operator()<true>(gk[i], qt + part * S::kPart, 0, i, wd);
        }
    }

    // Rows row0 .. end - 1 of a head that are not finite, one by one: into the keys that they see alone
    __device__ __forceinline__ void rows_again(const AttnArgs& a, const Pair& p, int head, int key, int row0, int end) {
        const int lane = lane_here(), kv_head = head / a.group;
        const int64_t mine = p.k0 + min(key, p.nk - 1);
        for (int row = row0; row < end; ++row) {
            const unsigned char *qr = row_of_head(a.q, p.q0 + row, head), *gr = row_of_head(a.gout, p.q0 + row, head);
            if (!row_not_finite<DT>(qr, a.dim_bytes, lane) && !row_not_finite<DT>(gr, a.dim_bytes, lane)) continue;
            const f32x2 stat = *(const f32x2*)(a.stats + 2 * (head * a.rows_q + p.q0 + row));
            const float s = dot_rows<DT>(row_of_head(a.k, mine, kv_head), qr, a.dim_bytes, lane >> 5);
            const float dp = one_key ? 0.f : dot_rows<DT>(row_of_head(a.v, mine, kv_head), gr, a.dim_bytes, lane >> 5);
            const float w = __builtin_amdgcn_exp2f(fmaf(s, a.negative ? -a.c : a.c, -stat[0]));
            const bool sees = row + p.nk - p.nq >= key;
            add_row<DT>(gk, qr, w * (dp - stat[1]), sees, part * S::COLS, a.dim_bytes, lane >> 5);
            add_row<DT>(gv, gr, w, sees, part * S::COLS, a.dim_bytes, lane >> 5);
        }
    }

    // behind the last block
    __device__ __forceinline__ void end() {
        if constexpr (DT == FX_F16) {
#pragma unroll
            for (int i = 0; i < S::COLS; ++i) gk[i] *= 1.f / lift;
        }
    }

    // the results of one share of the queries, in fp32
    __device__ __forceinline__ void store_sums(const AttnArgs& a, const Pair& p, int kv_head, int key, int share) {
        if (key >= p.nk) return;
        const int dim_bytes = a.dim_bytes / AttnType<DT>::ES * 4;
        unsigned char* to = (unsigned char*)a.sums + (((int64_t)share * a.kv_heads + kv_head) * a.rows_k + p.k0 + key) * 2 * dim_bytes;
        const float f = (a.negative ? -a.scale : a.scale) * kDown;
#pragma unroll
        for (int i = 0; i < S::COLS; ++i) {
            store_columns<FX_F32>(gk[i], f, to, part * S::COLS + i, dim_bytes, lane_here() >> 5);
            store_columns<FX_F32>(gv[i], kDown, to + dim_bytes, part * S::COLS + i, dim_bytes, lane_here() >> 5);
        }
    }
    __device__ __forceinline__ void store(const AttnArgs& a, const Pair& p, int kv_head, int key) {
        if (key >= p.nk) return;
        if (a.gk.p) {
            unsigned char* out = a.gk.p + (int64_t)(p.k0 + key) * a.gk.ld + kv_head * a.gk.hs;
            const float f = (a.negative ? -a.scale : a.scale) * kDown;
#pragma unroll
            for (int i = 0; i < S::COLS; ++i) store_columns<DT>(gk[i], f, out, part * S::COLS + i, a.dim_bytes, lane_here() >> 5);
        }
        if (a.gv.p) {
            unsigned char* out = a.gv.p + (int64_t)(p.k0 + key) * a.gv.ld + kv_head * a.gv.hs;
#pragma unroll
            for (int i = 0; i < S::COLS; ++i) store_columns<DT>(gv[i], kDown, out, part * S::COLS + i, a.dim_bytes, lane_here() >> 5);
        }
    }
};

// lse (base 2, less weight_lift) and delta of ROWS rows, as the first kernel left them, into LDS; zeros for a row that does not exist
template <int ROWS> __device__ __forceinline__ void load_stats(const AttnArgs& a, lds_byte* to, int head, int q0, int row0, int nq, int lane) {
#if defined(__HIP_DEVICE_COMPILE__)
    const uint64_t from = (uint64_t)(a.stats + 2 * (head * a.rows_q + q0 + row0));
    const uint64_t base = (uint32_t)uni((int)(uint32_t)from) | (uint64_t)(uint32_t)uni((int)(from >> 32)) << 32;        // one for the wave, the compiler does not see it
    __amdgpu_buffer_rsrc_t r = __builtin_amdgcn_make_buffer_rsrc((void*)base, 0, uni(max(0, min(nq - row0, ROWS)) * 8), 0x27000);
#pragma unroll
    for (int i = 0; i < ROWS / 32; ++i)
        __builtin_amdgcn_raw_ptr_buffer_load_lds(r, (__attribute__((address_space(3))) void*)(to + 256 * i), 4, lane * 4 + 256 * i, 0, 0, 0);
#endif
}

template <int DT, int DP, int W>
__global__ __launch_bounds__(64 * W, W == 4 && DP * AttnType<DT>::ES <= 128 ? 3 : least_waves_of(DP * AttnType<DT>::ES, W == 4)) void k_attention_gkv(AttnArgs a) {
#if defined(__HIP_DEVICE_COMPILE__)
    typedef BwdShape<DT, DP> S;
    constexpr int RB = S::RB, QT = S::QT;
    extern __shared__ __attribute__((aligned(1024))) unsigned char smem[];
    lds_byte* lds = (lds_byte*)smem;
    lds_byte* stats = lds + 4 * S::kQueries;
    const Work work = work_of(a, a.kv_heads * S::kParts * a.shares);
    if (work.head < 0) return;
    const int share = work.head & (a.shares - 1), head_part = work.head >> (a.shares - 1), kv_head = head_part / S::kParts;
    const int wave = uni(threadIdx.x / 64), lane = threadIdx.x & 63;
    const SeqTile st = a.tiles[work.tile];
    const Pair p = pair_of_keys(a, st);
    // the tile that most queries see is a causal sequence's first: it is begun first
    const int tile0 = a.causal ? (p.nk - 1) / (32 * W) * (32 * W) - st.row : st.row;
    const int key0 = tile0 + wave * 32, shift = p.nk - p.nq;
    TileLoad<RB, QT, W> lq, lo;
    lq.init(wave, lane, a.q.ld, a.dim_bytes);
    lo.init(wave, lane, a.gout.ld, a.dim_bytes);
    const int diagonal = a.causal ? tile0 + 32 * W - 1 - shift : 0;         // rows before this one do not see all of the workgroup's keys
    // all heads of the group in turn; of each the tiles from the first on in which a query sees the workgroup's first key
    const int begin = a.causal ? max(0, tile0 - shift) / QT * QT : 0, n = begin < p.nq ? (p.nq - begin + QT - 1) / QT * a.group : 0;
    const int j0 = share ? n / 2 : 0, j1 = share + 1 < a.shares ? n / 2 : n, per_head = max(1, n / a.group), items = j1 - j0;
    const int before = uni(j0 / per_head);
    int next_head = kv_head * a.group + before, next = begin + (j0 - before * per_head) * QT;
    int r0 = next - QT;
    auto load = [&](int b) {
        lq.load(lds + b * S::kQueries, a.q.p + (int64_t)p.q0 * a.q.ld + next_head * a.q.hs, a.q.ld, next, p.nq, a.dim_bytes, wave);
        lo.load(lds + (2 + b) * S::kQueries, a.gout.p + (int64_t)p.q0 * a.gout.ld + next_head * a.gout.hs, a.gout.ld, next, p.nq, a.dim_bytes, wave);
        if (wave == W - 1) load_stats<QT>(a, stats + b * S::kStats, next_head, p.q0, next, p.nq, lane);
        next += QT;
        if (next >= p.nq) { next = begin; ++next_head; }
    };
    if (items > 0) load(0);
    GkvWave<DT, DP, W == 2> w;
    w.init(a, p, kv_head, head_part % S::kParts, key0, lane);
    bool odd = false;
    for (int j = 0; j < items; ++j) {
        __builtin_amdgcn_s_waitcnt(0);
        __syncthreads();
        const int b = j & 1;
        r0 += QT;
        if (r0 >= p.nq) r0 = begin;
        if (j + 1 < items) load(b ^ 1);
        const lds_byte *qt = lds + b * S::kQueries, *ot = lds + (2 + b) * S::kQueries;
        uint64_t odd_rows = 0;
        if (r0 < diagonal) {
            const uint32_t mine = clean_rows<DT, RB, QT, W>(lds + b * S::kQueries, wave) | clean_rows<DT, RB, QT, W>(lds + (2 + b) * S::kQueries, wave);
            odd_rows = cleaned_rows<QT, W>(lds + S::kFlagsQueries, mine, wave);
            odd |= odd_rows != 0;
        }
        const float* st = (const float*)(smem + 4 * S::kQueries + b * S::kStats);
#pragma unroll
        for (int t = 0; t < QT; t += 32) {
            const int r = r0 + t;
            if (key0 >= p.nk || r >= p.nq || (a.causal && r + 31 + shift < key0)) continue;
            const bool masked = a.causal && r + shift < key0 + 31;
            w.block(qt + LdsRows<RB>::row_at(t), ot + LdsRows<RB>::row_at(t), st + 2 * t, masked, key0 - shift - r, (uint32_t)(odd_rows >> t) | rows_behind(p.nq - r));
        }
    }
    matrix_results_ready();
    w.end();
    if (odd)            // the same tiles of the workgroup's items
        for (int j = j0; j < j1; ++j) {
            const int of_head = j / per_head, row = begin + (j - of_head * per_head) * QT;
            if (row < diagonal) w.rows_again(args_here(), p, kv_head * a.group + of_head, key0 + (lane_here() & 31), row, min(row + QT, p.nq));
        }
    if (a.shares > 1) {
        w.store_sums(a, p, kv_head, key0 + (lane_here() & 31), share);
        return;
    }
    w.store(a, p, kv_head, key0 + (lane_here() & 31));
#endif
}

// The shares' sums of W blocks of 32 keys added, in their order
template <int DT, int W>
__global__ __launch_bounds__(64 * W) void k_attention_join_keys(AttnArgs a) {
#if defined(__HIP_DEVICE_COMPILE__)
    typedef typename AttnType<DT>::T T;
    const int tile = blockIdx.x % a.n_tiles, kv_head = blockIdx.x / a.n_tiles, wave = uni(threadIdx.x / 64), lane = threadIdx.x & 63;
    const Pair p = pair_of_keys(a, a.tiles[tile]);
    const int key0 = (a.causal ? (p.nk - 1) / (32 * W) * (32 * W) - a.tiles[tile].row : a.tiles[tile].row) + wave * 32, keys = min(32, p.nk - key0);
    const int dim = a.dim_bytes / AttnType<DT>::ES, fours = dim / 4;
    const int64_t share = a.rows_k * a.kv_heads * 2 * dim;
    const float* sums = a.sums + ((int64_t)kv_head * a.rows_k + p.k0 + key0) * 2 * dim;
    for (int i = lane; i < keys * 2 * fours; i += 64) {
        const int row = i / (2 * fours), at = i - row * 2 * fours, which = at >= fours, d = (at - which * fours) * 4;
        const HeadsView& out = which ? a.gv : a.gk;
        if (!out.p) continue;
        f32x4 x = *(const f32x4*)(sums + (int64_t)row * 2 * dim + at * 4);
        for (int s = 1; s < a.shares; ++s) x += *(const f32x4*)(sums + s * share + (int64_t)row * 2 * dim + at * 4);
        T* to = (T*)row_of_head(out, p.k0 + key0 + row, kv_head) + d;
#pragma unroll
        for (int e = 0; e < 4; ++e) to[e] = (T)x[e];
    }
#endif
}

// For few keys: RG blocks of 32, for each of which KS waves take the blocks of 32 queries of all heads in turn
template <int DT, int DP, int RG, int KS>
__global__ __launch_bounds__(64 * RG * KS, least_waves_of(DP * AttnType<DT>::ES, false)) void k_attention_gkv_few(AttnArgs a) {
#if defined(__HIP_DEVICE_COMPILE__)
    typedef BwdShape<DT, DP> S;
    constexpr int RB = S::RB, QT = 32, NB = S::template buffers<KS>();
    extern __shared__ __attribute__((aligned(1024))) unsigned char smem[];
    const Work work = work_of(a, a.kv_heads * S::kParts);
    if (work.head < 0) return;
    const int kv_head = work.head / S::kParts;
    const int wave = uni(threadIdx.x / 64), lane = threadIdx.x & 63, rg = wave % RG, turn = wave / RG;
    unsigned char* own = smem + turn * NB * S::kOwn;
    const SeqTile st = a.tiles[work.tile];
    const Pair p = pair_of_keys(a, st);
    const int tile0 = a.causal ? (p.nk - 1) / (32 * RG) * (32 * RG) - st.row : st.row;
    const int key0 = tile0 + rg * 32, shift = p.nk - p.nq;
    TileLoad<RB, QT, RG> lq, lo;
    lq.init(rg, lane, a.q.ld, a.dim_bytes);
    lo.init(rg, lane, a.gout.ld, a.dim_bytes);
    const int begin = a.causal ? max(0, tile0 - shift) / QT * QT : 0, per_head = begin < p.nq ? (p.nq - begin + QT - 1) / QT : 0;
    const int n = per_head * a.group, rounds = (n + KS - 1) / KS;
    const int diagonal = a.causal ? tile0 + 32 * RG - 1 - shift : 0;        // rows before this one do not see all of the workgroup's keys
    int head = kv_head * a.group, at = turn;            // the next block of the wave's turn: the at-th of the head
    auto load = [&](int b) {
        while (at >= per_head) { at -= per_head; ++head; }
        const int r0 = begin + at * QT;
        lds_byte* to = (lds_byte*)own + b * S::kOwn;
        lq.load(to, a.q.p + (int64_t)p.q0 * a.q.ld + head * a.q.hs, a.q.ld, r0, p.nq, a.dim_bytes, rg);
        lo.load(to + S::kBlock, a.gout.p + (int64_t)p.q0 * a.gout.ld + head * a.gout.hs, a.gout.ld, r0, p.nq, a.dim_bytes, rg);
        if (rg == RG - 1) load_stats<QT>(a, to + 2 * S::kBlock, head, p.q0, r0, p.nq, lane);
        at += KS;
        return r0;
    };
    int r0 = 0, next = 0;
    if (turn < n) next = load(0);
    GkvWave<DT, DP> w;
    w.init(a, p, kv_head, work.head % S::kParts, key0, lane);
    bool odd = false;
    for (int i = 0; i < rounds; ++i) {
        const int j = i * KS + turn, b = NB == 2 ? i & 1 : 0;
        __builtin_amdgcn_s_waitcnt(0);
        if (RG > 1) __syncthreads();
        r0 = next;
        uint32_t odd_rows = 0;
        if (begin < diagonal) {
            lds_byte* now = (lds_byte*)own + b * S::kOwn;
            if (j < n && r0 < diagonal) odd_rows = clean_rows<DT, RB, QT, RG>(now, rg) | clean_rows<DT, RB, QT, RG>(now + S::kBlock, rg);
            if (RG > 1) odd_rows = (uint32_t)cleaned_rows<QT, RG>((lds_byte*)smem + S::template flags_few<RG, KS>() + turn * RG * 4, odd_rows, rg);
            odd |= odd_rows != 0;
        }
        if (NB == 2 && j + KS < n) next = load(b ^ 1);
        if (j < n && key0 < p.nk && !(a.causal && r0 + 31 + shift < key0)) {
            const unsigned char* now = own + b * S::kOwn;
            const bool masked = a.causal && r0 + shift < key0 + 31;
            w.block((const lds_byte*)now, (const lds_byte*)now + S::kBlock, (const float*)(now + 2 * S::kBlock), masked, key0 - shift - r0, odd_rows | rows_behind(p.nq - r0));
        }
        if (NB == 1) {
            __builtin_amdgcn_s_waitcnt(0);          // what is read there has been read
            if (RG > 1) __syncthreads();
            if (j + KS < n) next = load(0);
        }
    }
    matrix_results_ready();
    w.end();
    add_results<RG, KS>(smem, w.gk, rg, turn, lane);
    add_results<RG, KS>(smem, w.gv, rg, turn, lane);
    odd = __syncthreads_or(odd);
    if (turn == 0) {
        if (odd)
            for (int h = 0; h < a.group; ++h)
                w.rows_again(args_here(), p, kv_head * a.group + h, key0 + (lane_here() & 31), begin, min((diagonal - begin + QT - 1) / QT * QT + begin, p.nq));
        w.store(a, p, kv_head, key0 + (lane_here() & 31));
    }
#endif
}

template <int DT, int DP> static void launch_bwd(const AttnArgs& a, const AttnArgs& b, bool keys, hipStream_t st) {
    typedef BwdShape<DT, DP> S;
    // as forward; eight waves have 256 registers each, which the gradients of wider rows do not do with
    constexpr int RG = share_tiles(DT, S::RB, true) ? 2 : 1, KS = RG == 1 ? (S::RB > 512 ? 2 : 4) : S::RB > 256 ? 2 : 4, KSK = RG == 1 ? KS : S::RB > 128 ? 2 : 4, KS1 = S::RB > 512 ? 2 : S::RB > 128 ? 4 : 8;
    constexpr int LDS = S::template lds_few<RG, KS>(), LDSK = S::template lds_few<RG, KSK>(), LDS1 = S::template lds_few<1, KS1>();
    static_assert(LDS + 1024 <= 160 * 1024 && LDSK + 1024 <= 160 * 1024 && LDS1 + 1024 <= 160 * 1024 && S::kLdsKeys <= 160 * 1024, "a compute unit has 160 KiB");
    static_assert(S::kParts <= kMostParts, "the launch is checked for them");
    const unsigned nq = work_blocks(a, a.heads * S::kParts), nk = work_blocks(b, b.kv_heads * S::kParts * b.shares);
    if (nq && a.few == 1) k_attention_gq_few<DT, DP, 1, KS1><<<nq, 64 * KS1, LDS1, st>>>(a);
    else if (nq && a.few) k_attention_gq_few<DT, DP, RG, KS><<<nq, 64 * RG * KS, LDS, st>>>(a);
    else if (nq && a.tile_rows == 64) k_attention_gq<DT, DP, 2><<<nq, 128, S::kLdsKeys, st>>>(a);
    else if (nq) k_attention_gq<DT, DP, 4><<<nq, 256, S::kLdsKeys, st>>>(a);
    if (!keys || !nk) return;
    if (b.few == 1) k_attention_gkv_few<DT, DP, 1, KS1><<<nk, 64 * KS1, LDS1, st>>>(b);
    else if (b.few) k_attention_gkv_few<DT, DP, RG, KSK><<<nk, 64 * RG * KSK, LDSK, st>>>(b);
    else if (b.tile_rows == 64) k_attention_gkv<DT, DP, 2><<<nk, 128, S::kLdsQueries, st>>>(b);
    else k_attention_gkv<DT, DP, 4><<<nk, 256, S::kLdsQueries, st>>>(b);
    if (b.shares > 1 && b.tile_rows == 64) k_attention_join_keys<DT, 2><<<b.n_tiles * b.kv_heads, 128, 0, st>>>(b);
    else if (b.shares > 1) k_attention_join_keys<DT, 4><<<b.n_tiles * b.kv_heads, 256, 0, st>>>(b);
}

template <int DT> static void launch_bwd_dim(const AttnArgs& a, const AttnArgs& b, int dim, bool keys, hipStream_t st) {
    if (dim <= 32) launch_bwd<DT, 32>(a, b, keys, st);
    else if (dim <= 64) launch_bwd<DT, 64>(a, b, keys, st);
    else if (dim <= 128) launch_bwd<DT, 128>(a, b, keys, st);
    else launch_bwd<DT, 256>(a, b, keys, st);
}

// A causal sequence's last keys have few queries.  Where all workgroups are resident at once those leave their compute unit half empty:
// a second workgroup for each tile, in an order from long to short, fills it.  bf16 causal, both gradients' kernels: 16,384 x 16 / 4 x 128 4996 ->
// 3626 us, 16,384 x 16 / 2 x 128 6325 -> 4348, 8,192 x 8 / 4 x 64 517 -> 363, 2,048 x 16 x 128 143 -> 137; with 1,024 queries for a key the join
// costs more than it gives (1,024 x 32 x 128: 92 -> 103).
int key_shares(const AttnArgs& a, int32_t n_tiles, int32_t few, int64_t queries, int dim, fx_dtype dt) {
    const int parts = dim <= 128 ? 1 : dt == FX_F32 ? 4 : 2;
    return a.causal && !few && queries >= 2048 && (a.gk.p || a.gv.p) && (int64_t)n_tiles * a.kv_heads * parts <= 2 * compute_units() ? 2 : 1;
}

void attention_bwd_launch(const AttnArgs& a, const AttnArgs& keys_tiles, fx_dtype dt, int dim, bool keys, hipStream_t st) {
    AttnArgs b = a;
    b.tiles = keys_tiles.tiles;
    b.n_tiles = keys_tiles.n_tiles;
    b.tile_rows = keys_tiles.tile_rows;
    b.few = keys_tiles.few;
    if (b.order != kHeadsFirst) b.order = b.kv_heads % 8 ? kTilesFirst : kHeadsApart;
    b.chunk = b.order == kHeadsFirst ? std::max(1, std::min(8, b.n_tiles / 64)) : 1;
    if (b.shares > 1) {         // the tiles with most queries first, over all heads and shares
        b.order = kHeadsFirst;
        b.chunk = 1;
    }
    if (dt == FX_F32) launch_bwd_dim<FX_F32>(a, b, dim, keys, st);
    else if (dt == FX_F16) launch_bwd_dim<FX_F16>(a, b, dim, keys, st);
    else launch_bwd_dim<FX_BF16>(a, b, dim, keys, st);
}

}  // namespace fx
