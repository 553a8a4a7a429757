// Attention over packed sequences: the forward kernel, and the entry points of both directions.
//
// out_i = sum_j exp(s_ij - lse_i) v_j, s = scale q k^T, lse_i = log sum_j exp(s_ij), in one pass over the keys with the running maximum and
// sum of each row.  Long sequences are bound by the matrix instructions and the exponentials between them: 32,768 x 16 x 128 bf16
// causal 4.2 ms, 1.04 PFLOP/s (a library product 1.38), 65,536 x 8 x 64 causal in four sequences 1.65 ms, 0.93.  Short ones are bound by
// a workgroup's chain of loads, two tiles and stores: 203,132 x 4 x 32 f16 in 3,400 sequences 65 us, 212 MB.
#include "attention.h"

#include <limits.h>
#include <math.h>

namespace fx {

// ------------------------------------------------------------------ forward
// What a wave keeps of its 32 queries, a column (lane % 32) each: the sums so far, the maximum that their weights are relative to,
// and the sum of the weights of the lane's half of the keys.
template <int DT, int DP, bool TINY = false> struct FwdWave {
    typedef typename AttnType<DT>::T T;
    static constexpr int RB = DP * AttnType<DT>::ES, STEPS = RB / 32, COLS = DP / 32;
    // By how many powers of two a weight may pass the reference's before that follows, and how many lie between the reference's own weight and 1.
    // fp16 ends at 2^-24: its largest weights are 2^11 to 2^15, and what a smaller one loses is 2^-36 of them.
    static constexpr float kLag = DT == FX_F16 ? 4.f : 8.f, kUp = DT == FX_F16 ? 11.f : 0.f;
    RowReader<DT, RB> rows_of;
    ColumnProduct<DT, RB> columns;
    OwnRows<DT, STEPS> q;
    f32x16 acc[COLS];
    float m, sum, c;
    int half;
    bool tiny = false;              // few keys in all

    __device__ __forceinline__ void init(const AttnArgs& a, int lane) {
        half = lane >> 5;
        rows_of.init(lane);
        columns.init(lane);
        c = a.c;
    }
    __device__ __forceinline__ void clear() {
#pragma unroll
        for (int k = 0; k < COLS; ++k) acc[k] = f32x16(0.f);
        m = -INFINITY;
        sum = 0.f;
    }

    // NB blocks of 32 keys from key0 on, of which the lane's query sees those up to `last` (all where not masked)
    template <int NB> __device__ __forceinline__ void blocks(const lds_byte* kt, const lds_byte* vt, int row0, int key0, bool masked, int last) {
        f32x16 s[NB];
#pragma unroll
        for (int t = 0; t < NB; ++t) {
            s[t] = f32x16(0.f);
#pragma unroll
            for (int i = 0; i < STEPS; ++i) s[t] = Elem<T>::mma(rows_of(kt, row0 + t * 32, i), q.x[i], s[t]);
        }
        if (masked) {
            const int left = last - key0 - 4 * half;
#pragma unroll
            for (int t = 0; t < NB; ++t)
#pragma unroll
                for (int r = 0; r < 16; ++r)
                    if (32 * t + 8 * (r >> 2) + (r & 3) > left) s[t][r] = -INFINITY;
        }
        float top = s[0][0];
#pragma unroll
        for (int t = 0; t < NB; ++t)
#pragma unroll
            for (int r = 0; r < 16; ++r) top = fmaxf(top, s[t][r]);
        top = fmaxf(top, other_half(top));
        // The maximum that weights are relative to follows the row's own only when that has grown by a factor of 2^kLag: acc and
        // sum are exact in whichever they are, a weight is at most 2^(kLag + kUp), and few tiles have to scale what is there.
        if (__any(top * c > m * c + kLag)) rescale(fmaxf(m, top));
        const float mc = m == -INFINITY ? 0.f : base(m);
        float part = 0.f;
#pragma unroll
        for (int t = 0; t < NB; ++t) {
#pragma unroll
            for (int r = 0; r < 16; ++r) {
                s[t][r] = __builtin_amdgcn_exp2f(fmaf(s[t][r], c, -mc));
                part += s[t][r];
            }
            Weights<DT> w;
            w.set(s[t]);
#pragma unroll
            for (int k = 0; k < COLS; ++k) columns(acc[k], vt, row0 + t * 32, k, w);
            if (TINY && DT != FX_F32 && tiny) {
                w.set(w.rest(s[t]));
#pragma unroll
                for (int k = 0; k < COLS; ++k) columns.template operator()<true>(acc[k], vt, row0 + t * 32, k, w);
            }
        }
        sum += part;
    }

    // the exponent of a weight of 1 (base 2), where the reference is x
    __device__ __forceinline__ float base(float x) const { return DT == FX_F16 ? fmaf(x, c, -kUp) : x * c; }
    __device__ __forceinline__ void rescale(float to) {
        const float f = m == -INFINITY ? 0.f : __builtin_amdgcn_exp2f((m - to) * c);
        m = to;
        sum *= f;
#pragma unroll
        for (int k = 0; k < COLS; ++k) acc[k] *= f;
    }

    __device__ __forceinline__ float lse() const { return DT == FX_F16 ? (base(m) + kUp) + __builtin_amdgcn_logf(sum * 0x1p-11f) : m * c + __builtin_amdgcn_logf(sum); }
    __device__ __forceinline__ void store(const AttnArgs& a, int row, int nq, int q0, int head) {
        if (row >= nq) return;
        const float f = sum == 0.f ? 0.f : 1.f / sum;
        unsigned char* out = a.out.p + (int64_t)(q0 + row) * a.out.ld + head * a.out.hs;
#pragma unroll
        for (int k = 0; k < COLS; ++k) store_columns<DT>(acc[k], f, out, k, a.dim_bytes, half);
        if (a.lse && half == 0) a.lse[head * a.rows_q + q0 + row] = sum == 0.f ? -INFINITY : lse() * kLn2;
    }
};

// The diagonal tiles' values that are not finite, from key `from` on, added for the rows that see them: a weight is positive, and such a
// value times it is what it is itself
template <int DT, int N> __device__ __forceinline__ void add_not_finite(f32x16 (&acc)[N], const unsigned char* vb, int64_t ld, int from, int end, int last, int dim_bytes, int lane) {
    for (int key = from; key < end; ++key) {
        const unsigned char* row = vb + key * ld;
        if (!row_not_finite<DT>(row, dim_bytes, lane)) continue;
#pragma unroll
        for (int k = 0; k < N; ++k)
#pragma unroll
            for (int g = 0; g < 4; ++g) {
                Four<DT> f;
                f.load(row, k, g, dim_bytes, lane >> 5);
#pragma unroll
                for (int e = 0; e < 4; ++e) acc[k][4 * g + e] += key <= last && !finite(f.x[e]) ? f.x[e] : 0.f;
                __builtin_amdgcn_sched_barrier(0);
            }
    }
}

// A workgroup has W waves of 32 queries of one head; keys and values come by in tiles of KT, two buffers of each.
template <int DT, int DP> struct FwdShape {
    static constexpr int RB = DP * AttnType<DT>::ES;
    static constexpr int KT = RB > 256 ? 32 : 64;
    static constexpr int kTile = LdsRows<RB>::bytes(KT);
    static constexpr int kFlagsAt = 4 * kTile, kLds = kFlagsAt + kFlags;
};

template <int DT, int DP, int W>
__global__ __launch_bounds__(64 * W, least_waves_of(DP * AttnType<DT>::ES, W == 4)) void k_attention(AttnArgs a) {
#if defined(__HIP_DEVICE_COMPILE__)         // the host pass has no buffer descriptors and drops stubs over them
    typedef FwdShape<DT, DP> S;
    constexpr int RB = S::RB, KT = S::KT;
    extern __shared__ __attribute__((aligned(1024))) unsigned char smem[];
    lds_byte* lds = (lds_byte*)smem;
    const Work work = work_of(a, a.heads);
    if (work.head < 0) return;
    const int wave = uni(threadIdx.x / 64), lane = threadIdx.x & 63;
    TileLoad<RB, KT, W> lk, lv;
    lk.init(wave, lane, a.k.ld, a.dim_bytes);
    lv.init(wave, lane, a.v.ld, a.dim_bytes);
    FwdWave<DT, DP, W == 2> w;
    w.init(a, lane);
    const int head = work.head, kv_head = head / a.group;
    const SeqTile st = a.tiles[work.tile];
    const Pair p = pair_of(a, st);
    const unsigned char* kb = a.k.p + (int64_t)p.k0 * a.k.ld + kv_head * a.k.hs;
    const unsigned char* vb = a.v.p + (int64_t)p.k0 * a.v.ld + kv_head * a.v.hs;
    // keys that some row of the workgroup, or of the wave, sees; and the last that this lane's row sees
    const int row0 = st.row + wave * 32, row = row0 + (lane & 31), shift = p.nk - p.nq;
    const int seen = a.causal ? max(0, min(p.nk, min(st.row + 32 * W, p.nq) + shift)) : p.nk;
    const int seen_wave = row0 >= p.nq ? 0 : a.causal ? max(0, min(p.nk, min(row0 + 32, p.nq) + shift)) : p.nk;
    const int last = a.causal ? min(p.nk - 1, row + shift) : p.nk - 1, unmasked = a.causal ? min(p.nk - 1, row0 + shift) : p.nk - 1;
    const int n = (seen + KT - 1) / KT;
    const int diagonal = a.causal ? max(0, st.row + 1 + shift) / KT : INT_MAX;           // the first tile that is not seen whole by some row of the workgroup
    if (n > 0) {
        lk.load(lds, kb, a.k.ld, 0, p.nk, a.dim_bytes, wave);
        lv.load(lds + 2 * S::kTile, vb, a.v.ld, 0, p.nk, a.dim_bytes, wave);
    }
    w.q.load(a.q.p + (int64_t)p.q0 * a.q.ld + head * a.q.hs, a.q.ld, row0, p.nq, a.dim_bytes, lane, a.negative);
    w.clear();
    w.tiny = p.nk <= kTinyRows;
    bool odd = false;
    for (int j = 0; j < n; ++j) {
        __builtin_amdgcn_s_waitcnt(0);
        __syncthreads();
        const int b = j & 1, key0 = j * KT;
        if (j + 1 < n) {
            lk.load(lds + (b ^ 1) * S::kTile, kb, a.k.ld, key0 + KT, p.nk, a.dim_bytes, wave);
            lv.load(lds + (2 + (b ^ 1)) * S::kTile, vb, a.v.ld, key0 + KT, p.nk, a.dim_bytes, wave);
        }
        const lds_byte *kt = lds + b * S::kTile, *vt = lds + (2 + b) * S::kTile;
        const bool masked = key0 + KT - 1 > unmasked;
        if (j >= diagonal) odd |= cleaned_rows<KT, W>(lds + S::kFlagsAt, clean_rows<DT, RB, KT, W>(lds + (2 + b) * S::kTile, wave), wave) != 0;
        if (key0 >= seen_wave) continue;
        // half a tile by itself only where sequences are short: a second form of the loop's body costs registers
        if (KT == 64 && (W > 2 || key0 + 32 < seen_wave)) w.template blocks<2>(kt, vt, 0, key0, masked, last);
        else w.template blocks<1>(kt, vt, 0, key0, masked, last);
    }
    matrix_results_ready();
    w.sum += other_half(w.sum);
    if (odd) add_not_finite<DT>(w.acc, vb, a.v.ld, diagonal * KT, seen_wave, last, a.dim_bytes, lane_here());
    w.store(a, row, p.nq, p.q0, head);
#endif
}

// The same for few queries: RG blocks of 32 queries, for each of which KS waves take the blocks of 32 keys in turn.  The RG waves of a
// turn share its tiles; at the end the KS results of a block of queries are joined.
template <int DT, int DP, int RG, int KS> struct FewShape {
    static constexpr int RB = DP * AttnType<DT>::ES;
    static constexpr int kTile = LdsRows<RB>::bytes(32);
    static constexpr int kBuffers = 4 * kTile * KS <= 128 * 1024 ? 2 : 1;
    static constexpr int kSlot = DP * 32 * 4 + 512;                 // a wave's result
    static constexpr int kFlagsAt = std::max(2 * kBuffers * kTile * KS, KS / 2 * RG * kSlot), kLds = kFlagsAt + kFlags;
};

template <int DT, int DP, int RG, int KS>
__global__ __launch_bounds__(64 * RG * KS, least_waves(DP * AttnType<DT>::ES)) void k_attention_few(AttnArgs a) {
#if defined(__HIP_DEVICE_COMPILE__)
    typedef FewShape<DT, DP, RG, KS> S;
    constexpr int RB = S::RB, COLS = DP / 32, NB = S::kBuffers;
    extern __shared__ __attribute__((aligned(1024))) unsigned char smem[];
    const Work work = work_of(a, a.heads);
    if (work.head < 0) return;
    const int head = work.head, kv_head = head / a.group;
    const int wave = uni(threadIdx.x / 64), lane = threadIdx.x & 63, rg = wave % RG, turn = wave / RG;
    lds_byte* lds = (lds_byte*)smem + turn * 2 * NB * S::kTile;
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
    const int n = (seen + 31) / 32, rounds = (n + KS - 1) / KS;         // a wave without a block in the last round waits with the others
    const int diagonal = a.causal ? max(0, st.row + 1 + shift) / 32 : INT_MAX;
    auto load = [&](int j, int b) {
        lk.load(lds + b * 2 * S::kTile, kb, a.k.ld, j * 32, p.nk, a.dim_bytes, rg);
        lv.load(lds + b * 2 * S::kTile + S::kTile, vb, a.v.ld, j * 32, p.nk, a.dim_bytes, rg);
    };
    if (turn < n) load(turn, 0);
    FwdWave<DT, DP> w;
    w.q.load(a.q.p + (int64_t)p.q0 * a.q.ld + head * a.q.hs, a.q.ld, row0, p.nq, a.dim_bytes, lane, a.negative);
    w.init(a, lane);
    w.clear();
    bool odd = false;
    for (int i = 0; i < rounds; ++i) {
        const int j = i * KS + turn, b = NB == 2 ? i & 1 : 0;
        __builtin_amdgcn_s_waitcnt(0);
        if (RG > 1) __syncthreads();
        lds_byte* at = lds + b * 2 * S::kTile;
        if (i * KS + KS > diagonal) {           // one of the turns' blocks
            uint32_t mine = j >= diagonal && j < n ? clean_rows<DT, RB, 32, RG>(at + S::kTile, rg) : 0;
            if (RG > 1) mine = (uint32_t)cleaned_rows<32, RG>((lds_byte*)smem + S::kFlagsAt + turn * RG * 4, mine, rg);
            odd |= mine != 0;
        }
        if (NB == 2 && j + KS < n) load(j + KS, b ^ 1);
        if (j * 32 < seen_wave) {
            const bool masked = j * 32 + 31 > unmasked;
            w.template blocks<1>(at, at + S::kTile, 0, j * 32, masked, last);
        }
        if (NB == 1) {
            __builtin_amdgcn_s_waitcnt(0);          // what is read there has been read
            if (RG > 1) __syncthreads();
            if (j + KS < n) load(j + KS, 0);
        }
    }
    matrix_results_ready();
    w.sum += other_half(w.sum);
#pragma unroll
    for (int h = KS / 2; h >= 1; h /= 2) {
        __syncthreads();
        if (turn >= h && turn < 2 * h) {
            float* to = (float*)(smem + ((turn - h) * RG + rg) * S::kSlot);
            put_result<COLS>(to, w.acc, lane);
            to[COLS * 1024 + lane] = w.m;
            to[COLS * 1024 + 64 + lane] = w.sum;
        }
        __syncthreads();
        if (turn < h) {
            const float* in = (const float*)(smem + (turn * RG + rg) * S::kSlot);
            const float m2 = in[COLS * 1024 + lane], sum2 = in[COLS * 1024 + 64 + lane], to = fmaxf(w.m, m2);
            w.rescale(to);
            const float f = m2 == -INFINITY ? 0.f : __builtin_amdgcn_exp2f((m2 - to) * a.c);
            w.sum = fmaf(sum2, f, w.sum);
#pragma unroll
            for (int k = 0; k < COLS; ++k)
#pragma unroll
                for (int r = 0; r < 16; ++r) w.acc[k][r] = fmaf(in[(k * 16 + r) * 64 + lane], f, w.acc[k][r]);
        }
    }
    odd = __syncthreads_or(odd);
    if (turn == 0) {
        if (odd) add_not_finite<DT>(w.acc, vb, a.v.ld, diagonal * 32, seen_wave, last, a.dim_bytes, lane_here());
        w.store(a, row, p.nq, p.q0, head);
    }
#endif
}

template <int DT, int DP> static void launch_fwd(const AttnArgs& a, hipStream_t st) {
    const unsigned blocks = work_blocks(a, a.heads);
    // one block of 32 and eight waves, where those have registers enough, or four; or two that share tiles, and four waves for each
    static_assert(FwdShape<DT, DP>::kLds <= 160 * 1024, "a compute unit has 160 KiB");
    constexpr int RB = DP * AttnType<DT>::ES, RG = share_tiles(DT, RB, false) ? 2 : 1, KS = RB > 512 ? 2 : 4, KS1 = RB > 128 ? KS : 8;
    static_assert(FewShape<DT, DP, 1, KS1>::kLds + 1024 <= 160 * 1024 && FewShape<DT, DP, RG, KS>::kLds + 1024 <= 160 * 1024, "a compute unit has 160 KiB");
    if (a.few == 1) k_attention_few<DT, DP, 1, KS1><<<blocks, 64 * KS1, FewShape<DT, DP, 1, KS1>::kLds, st>>>(a);
    else if (a.few) k_attention_few<DT, DP, RG, KS><<<blocks, 64 * RG * KS, FewShape<DT, DP, RG, KS>::kLds, st>>>(a);
    else if (a.tile_rows == 64) k_attention<DT, DP, 2><<<blocks, 128, FwdShape<DT, DP>::kLds, st>>>(a);
    else k_attention<DT, DP, 4><<<blocks, 256, FwdShape<DT, DP>::kLds, st>>>(a);
}

template <int DT> static void launch_fwd_dim(const AttnArgs& a, int dim, hipStream_t st) {
    if (dim <= 32) launch_fwd<DT, 32>(a, st);
    else if (dim <= 64) launch_fwd<DT, 64>(a, st);
    else if (dim <= 128) launch_fwd<DT, 128>(a, st);
    else launch_fwd<DT, 256>(a, st);
}

// ------------------------------------------------------------------ rows in an order that the kernels take
// Copies of a call, all in one launch: rows of dim_s elements a head, 16 bytes of the destination a thread (dim_d is whole pieces
// of 16 bytes, or dim_s where the destination is the caller's), zeros behind dim_s.
struct Copy { HeadsView src, dst; uint32_t heads, pieces, first_block; int64_t n; };
struct Copies { Copy c[8]; int32_t count, dim_s, dim_d; };

template <typename W>
__global__ __launch_bounds__(256) void k_heads_copy(Copies a) {
    constexpr int PER = 16 / sizeof(W);
    int which = 0;
    while (which + 1 < a.count && blockIdx.x >= a.c[which + 1].first_block) ++which;
    const Copy& c = a.c[which];
    const int64_t i = (int64_t)(blockIdx.x - c.first_block) * 256 + threadIdx.x;
    if (i >= c.n) return;
    const int64_t unit = i / c.pieces, r = unit / c.heads;
    const int e0 = (int)(i - unit * c.pieces) * PER;
    const int64_t h = unit - r * c.heads;
    const W* src = (const W*)(c.src.p + r * c.src.ld + h * c.src.hs) + e0;
    W* dst = (W*)(c.dst.p + r * c.dst.ld + h * c.dst.hs) + e0;
    W x[PER];
#pragma unroll
    for (int e = 0; e < PER; ++e) x[e] = e0 + e < a.dim_s ? src[e] : W(0);
#pragma unroll
    for (int e = 0; e < PER; ++e)
        if (e0 + e < a.dim_d) dst[e] = x[e];
}

struct CopyList {
    Copies a{};
    int64_t blocks = 0;
    void add(const HeadsView& src, const HeadsView& dst, int dim_d, int32_t heads, int64_t rows, int es) {
        const uint32_t pieces = (uint32_t)((dim_d * es + 15) / 16);
        const int64_t n = rows * heads * pieces;
        a.c[a.count++] = Copy{src, dst, (uint32_t)heads, pieces, (uint32_t)blocks, n};
        blocks += (n + 255) / 256;
    }
    fx_status run(const char* who, int dim_s, int dim_d, int es, hipStream_t st) {
        if (!a.count) return FX_OK;
        if (blocks > (1ll << 32) / 256 - 1) { set_error("%s: too many rows for one launch", who); return FX_ERANGE; }
        a.dim_s = dim_s;
        a.dim_d = dim_d;
        if (es == 4) k_heads_copy<uint32_t><<<(unsigned)blocks, 256, 0, st>>>(a);
        else k_heads_copy<uint16_t><<<(unsigned)blocks, 256, 0, st>>>(a);
        return FX_OK;
    }
};

// ------------------------------------------------------------------ checks
fx_status check_heads(const char* who, const HeadsTensor& t, int32_t dim, int es) {
    if (!t.p) {
        if (!t.needed || t.rows == 0) return FX_OK;
        set_error("%s: %s is null", who, t.name);
        return FX_EINVAL;
    }
    if ((uintptr_t)t.p % es || t.ld < dim || (t.heads > 1 && t.hs < dim)) {
        set_error("%s: %s is not aligned to its elements or has rows or heads closer than dim", who, t.name);
        return FX_EINVAL;
    }
    const int64_t most = 1ll << 46;
    if (t.ld > most || t.hs > most) { set_error("%s: %s has a stride of more than 2^46", who, t.name); return FX_ERANGE; }
    const bool rows_outside = t.heads == 1 || t.ld >= (t.heads - 1) * t.hs + dim;
    const bool heads_outside = t.rows <= 1 || (__int128)t.hs >= (__int128)(t.rows - 1) * t.ld + dim;
    if (t.output && !rows_outside && !heads_outside) { set_error("%s: rows and heads of %s overlap", who, t.name); return FX_EINVAL; }
    return FX_OK;
}

// What a call keeps until its launches are enqueued
struct Scratch {
    hipStream_t st;
    void* p[12];
    int n = 0;
    explicit Scratch(hipStream_t s) : st(s) {}
    ~Scratch() { while (n) dev_free(p[--n], st); }
    fx_status get(const char* who, void** out, size_t bytes) {
        FX_TRY(scratch_alloc(who, out, bytes, st));
        p[n++] = *out;
        return FX_OK;
    }
};

static fx_status check_attention(const char* who, const fx_attention* a) {
    if (!a || !a->q_seqs || (a->dt != FX_F32 && a->dt != FX_F16 && a->dt != FX_BF16) || a->heads < 1 || a->kv_heads < 1 || a->heads % a->kv_heads || a->dim < 1) {
        set_error("%s: null description or sequences, unknown dtype, no dimension, or heads that are no multiple of the key heads", who);
        return FX_EINVAL;
    }
    if (!std::isfinite(a->scale)) { set_error("%s: the scale is not finite", who); return FX_EINVAL; }
    if (a->kv_seqs && a->kv_seqs->B != a->q_seqs->B) { set_error("%s: %d sequences of queries and %d of keys", who, a->q_seqs->B, a->kv_seqs->B); return FX_EINVAL; }
    if (a->dim > kMostDim) { set_error("%s: more than %d dimensions", who, kMostDim); return FX_ERANGE; }
    if (a->heads > 65535) { set_error("%s: more than 65535 heads", who); return FX_ERANGE; }
    return FX_OK;
}

// Fills the views of the tensors; those whose order the kernels do not take are copied, and outputs get a place to be copied from
// (back).
static fx_status take_tensors(const char* who, HeadsTensor* t, int n, int32_t dim, fx_dtype dt, Scratch* scratch, CopyList* back, int* dim_in, hipStream_t st) {
    const int es = dtype_size(dt), per = 16 / es, padded = (dim + per - 1) / per * per;
    CopyList in;
    *dim_in = padded;
    for (int i = 0; i < n; ++i) {
        const HeadsView given{(unsigned char*)t[i].p, t[i].ld * es, t[i].hs * es};
        *t[i].view = given;
        if (!t[i].p || t[i].rows == 0) continue;
        const bool strides = given.ld % 16 == 0 && (t[i].heads == 1 || given.hs % 16 == 0) && given.ld <= (1ll << 24);
        if (dim % per == 0 && (uintptr_t)t[i].p % 16 == 0 && strides) continue;
        void* p = nullptr;
        FX_TRY(scratch->get(who, &p, (size_t)t[i].rows * t[i].heads * padded * es));
        *t[i].view = HeadsView{(unsigned char*)p, (int64_t)t[i].heads * padded * es, (int64_t)padded * es};
        if (t[i].output) back->add(*t[i].view, given, dim, t[i].heads, t[i].rows, es);
        else in.add(given, *t[i].view, padded, t[i].heads, t[i].rows, es);
    }
    return in.run(who, dim, padded, es, st);
}

static fx_status check_places(const char* who, const HeadsTensor* t, int n) {
    for (int i = 0; i < n; ++i)
        for (int j = 0; j < n; ++j)
            if (i != j && t[i].output && t[i].p && t[i].p == t[j].p && t[i].rows && t[j].rows) {
                set_error("%s: %s is where %s is", who, t[i].name, t[j].name);
                return FX_EINVAL;
            }
    return FX_OK;
}

// Tiles of 128 rows, four waves, or, where those would be less than 4/5 as full as tiles of 64, those, of two waves: keys are
// then loaded for half as many rows at a time, but no wave idles behind a sequence's end.  Where all blocks of 32 rows would
// not occupy every SIMD and there are other rows to share out, several waves take those in turn for one block (few = 1: fewer blocks
// than compute units; 2: more, and two blocks share tiles if rows are wide enough: 6,820 x 3 x 96 bf16 causal 111 -> 80 us, but
// gradients of 8,772 x 2 x 64 149 -> 168).
static void take_tiles(AttnArgs* a, const fx_sequences* q, int32_t heads, int64_t others, bool wide) {
    const int64_t waves = q->n_tiles[0] * heads;
    a->few = waves >= 4 * compute_units() || others <= 64 ? 0 : waves <= compute_units() || (wide && 64 * q->n_tiles[1] * 4 > 32 * q->n_tiles[0] * 5) ? 1 : 2;
    const int kind = a->few ? (a->few == 2 && wide ? 1 : 0) : 64 * q->n_tiles[1] * 5 <= 128 * q->n_tiles[2] * 4 ? 1 : 2;
    a->tiles = q->d_tiles[kind];
    a->n_tiles = (int32_t)q->n_tiles[kind];
    a->tile_rows = kSeqTileRows[kind];
}
// bytes of a row of a head in the kernel that takes it
static int kernel_row_bytes(int dim, fx_dtype dt) { return (dim <= 32 ? 32 : dim <= 64 ? 64 : dim <= 128 ? 128 : 256) * dtype_size(dt); }

static fx_status fill_args(const char* who, const fx_attention* d, AttnArgs* a, int64_t tiles, int32_t heads) {
    const fx_sequences *q = d->q_seqs, *k = d->kv_seqs ? d->kv_seqs : d->q_seqs;
    a->first_q = k == q ? nullptr : q->d_first;
    a->first_k = k == q ? nullptr : k->d_first;
    a->rows_q = q->rows;
    a->heads = d->heads;
    a->kv_heads = d->kv_heads;
    a->group = d->heads / d->kv_heads;
    a->causal = d->causal != 0;
    a->negative = d->scale < 0.f;
    a->scale = fabsf(d->scale);
    a->c = fmaxf(a->scale * kLog2e, 0x1p-149f);       // not 0: a masked score is -infinity and stays it
    a->order = k->longest <= 2048 ? kHeadsFirst : d->heads % 8 ? kTilesFirst : kHeadsApart;
    a->chunk = a->order == kHeadsFirst ? std::max(1, std::min(8, a->n_tiles / 64)) : 1;
    a->shares = 1;
    a->sums = nullptr;
    if (std::max(q->longest, k->longest) > 0x7FFFFFFFll - 1024) { set_error("%s: a sequence of more than 2^31-1025 rows", who); return FX_ERANGE; }
    if ((tiles + tiles / 8 + 8) * heads * (d->dim > 128 ? kMostParts : 1) > (1ll << 32) / 256 - 8) { set_error("%s: too many rows for one launch", who); return FX_ERANGE; }
    return FX_OK;
}

}  // namespace fx

using namespace fx;

extern "C" fx_status fx_attention_fwd(const fx_attention* d, void* d_out, int64_t ld_out, int64_t hs_out, float* d_lse, void* stream) {
    const char* who = "fx_attention_fwd";
    FX_TRY(check_attention(who, d));
    const int64_t nq = d->q_seqs->rows, nk = d->kv_seqs ? d->kv_seqs->rows : nq;
    AttnArgs a{};
    HeadsTensor t[] = {{"d_q", d->d_q, d->ld_q, d->hs_q, nq, d->heads, false, true, &a.q},
                  {"d_k", d->d_k, d->ld_k, d->hs_k, nk, d->kv_heads, false, true, &a.k},
                  {"d_v", d->d_v, d->ld_v, d->hs_v, nk, d->kv_heads, false, true, &a.v},
                  {"d_out", d_out, ld_out, hs_out, nq, d->heads, true, true, &a.out}};
    for (const HeadsTensor& x : t) FX_TRY(check_heads(who, x, d->dim, dtype_size(d->dt)));
    if ((uintptr_t)d_lse % 4) { set_error("%s: d_lse is not aligned to its elements", who); return FX_EINVAL; }
    FX_TRY(check_places(who, t, 4));
    take_tiles(&a, d->q_seqs, d->heads, (d->kv_seqs ? d->kv_seqs : d->q_seqs)->longest, share_tiles(d->dt, kernel_row_bytes(d->dim, d->dt), false));
    const int64_t tiles = a.n_tiles;
    FX_TRY(fill_args(who, d, &a, tiles, d->heads));
    if (nq == 0) return FX_OK;
    hipStream_t st = (hipStream_t)stream;
    ProfScope ps(kProfAttnFwd, st);
    Scratch scratch(st);
    CopyList back;
    int dim;
    FX_TRY(take_tensors(who, t, 4, d->dim, d->dt, &scratch, &back, &dim, st));
    a.dim_bytes = dim * dtype_size(d->dt);
    a.lse = d_lse;
    if (d->dt == FX_F32) launch_fwd_dim<FX_F32>(a, dim, st);
    else if (d->dt == FX_F16) launch_fwd_dim<FX_F16>(a, dim, st);
    else launch_fwd_dim<FX_BF16>(a, dim, st);
    FX_TRY(back.run(who, d->dim, d->dim, dtype_size(d->dt), st));
    FX_HIP_TRY(hipGetLastError());
    return FX_OK;
}

extern "C" fx_status fx_attention_bwd(const fx_attention* d, const void* d_out, int64_t ld_out, int64_t hs_out, const float* d_lse, const void* d_gout,
                                      int64_t ld_gout, int64_t hs_gout, const float* d_glse, void* d_gq, int64_t ld_gq, int64_t hs_gq, void* d_gk,
                                      int64_t ld_gk, int64_t hs_gk, void* d_gv, int64_t ld_gv, int64_t hs_gv, void* stream) {
    const char* who = "fx_attention_bwd";
    FX_TRY(check_attention(who, d));
    const fx_sequences* kq = d->kv_seqs ? d->kv_seqs : d->q_seqs;
    const int64_t nq = d->q_seqs->rows, nk = kq->rows;
    AttnArgs a{};
    const int n = 8;
    HeadsTensor t[n] = {{"d_q", d->d_q, d->ld_q, d->hs_q, nq, d->heads, false, true, &a.q},
                   {"d_k", d->d_k, d->ld_k, d->hs_k, nk, d->kv_heads, false, true, &a.k},
                   {"d_v", d->d_v, d->ld_v, d->hs_v, nk, d->kv_heads, false, true, &a.v},
                   {"d_out", d_out, ld_out, hs_out, nq, d->heads, false, true, &a.out},
                   {"d_gout", d_gout, ld_gout, hs_gout, nq, d->heads, false, true, &a.gout},
                   {"d_gq", d_gq, ld_gq, hs_gq, nq, d->heads, true, false, &a.gq},
                   {"d_gk", d_gk, ld_gk, hs_gk, nk, d->kv_heads, true, false, &a.gk},
                   {"d_gv", d_gv, ld_gv, hs_gv, nk, d->kv_heads, true, false, &a.gv}};
    for (const HeadsTensor& x : t) FX_TRY(check_heads(who, x, d->dim, dtype_size(d->dt)));
    if ((nq > 0 && !d_lse) || (uintptr_t)d_lse % 4 || (uintptr_t)d_glse % 4) { set_error("%s: d_lse is null, or it or d_glse is not aligned to its elements", who); return FX_EINVAL; }
    FX_TRY(check_places(who, t, n));
    AttnArgs b{};
    take_tiles(&b, kq, d->kv_heads, d->q_seqs->longest * (d->heads / d->kv_heads), share_tiles(d->dt, kernel_row_bytes(d->dim, d->dt), true));
    take_tiles(&a, d->q_seqs, d->heads, kq->longest, share_tiles(d->dt, kernel_row_bytes(d->dim, d->dt), true));
    FX_TRY(fill_args(who, d, &a, a.n_tiles, d->heads));
    FX_TRY(fill_args(who, d, &a, b.n_tiles, d->kv_heads));
    if (nq == 0 && nk == 0) return FX_OK;
    hipStream_t st = (hipStream_t)stream;
    ProfScope ps(kProfAttnBwd, st);
    Scratch scratch(st);
    CopyList back;
    int dim;
    FX_TRY(take_tensors(who, t, n, d->dim, d->dt, &scratch, &back, &dim, st));
    void* stats = nullptr;
    FX_TRY(scratch.get(who, &stats, (size_t)nq * d->heads * 8));
    a.dim_bytes = dim * dtype_size(d->dt);
    a.lse = const_cast<float*>(d_lse);
    a.glse = d_glse;
    a.stats = (float*)stats;
    a.rows_k = nk;
    a.shares = key_shares(a, b.n_tiles, b.few, d->q_seqs->longest * (d->heads / d->kv_heads), dim, d->dt);
    if (a.shares > 1) {
        void* p = nullptr;
        FX_TRY(scratch.get(who, &p, (size_t)a.shares * d->kv_heads * nk * 2 * dim * 4));
        a.sums = (float*)p;
    }
    attention_bwd_launch(a, b, d->dt, dim, d_gk || d_gv, st);
    FX_TRY(back.run(who, d->dim, d->dim, dtype_size(d->dt), st));
    FX_HIP_TRY(hipGetLastError());
    return FX_OK;
}
