// Gradients of attention over packed sequences.
//
// Two kernels, each with its outputs in registers until they are whole, so that nothing is added in memory: the first goes
// over the keys for a workgroup's queries (gq) and leaves sum_j P_ij dP_ij - glse_i of every row for the second, which goes over
// the queries for a workgroup's keys (gk, gv).  Scores and dP are computed in both: seven products instead of five, for
// results that do not depend on an order of atomics and need no fp32 copy of gq in memory.
#include "attention.h"

#include <math.h>

namespace fx {

template <int DT, int DP> struct BwdShape {
    static constexpr int RB = DP * AttnType<DT>::ES;
    static constexpr int T = 32;                // rows of a tile that streams by
    static constexpr int kTile = LdsRows<RB>::bytes(T);
    static constexpr int kLds = 4 * kTile + 4 * T * 4;
    // Parts that the output's columns are dealt out in, as heads of their own: above 128 dimensions a lane's results, its own rows and
    // their products would not fit 512 registers.
    static constexpr int kParts = DP > 128 ? 2 : 1;
    static constexpr int kCols = DP / 32 / kParts;
    static constexpr int kPart = kCols * (DT == FX_F32 ? 2 : 1) * LdsRows<RB>::kSegment;        // from part to part in a tile
};

// ------------------------------------------------------------------ gradients of the queries
template <int DT, int DP, int W>
__global__ __launch_bounds__(64 * W, DP * AttnType<DT>::ES > 256 ? 1 : 2) void k_attention_gq(AttnArgs a) {
#if defined(__HIP_DEVICE_COMPILE__)         // the host pass has no buffer descriptors and drops stubs over them
    typedef BwdShape<DT, DP> S;
    typedef typename AttnType<DT>::T T;
    constexpr int RB = S::RB, KT = S::T, STEPS = RB / 32, COLS = S::kCols;
    extern __shared__ __attribute__((aligned(1024))) unsigned char smem[];
    lds_byte* lds = (lds_byte*)smem;
    const Work work = work_of(a, a.heads * S::kParts);
    if (work.head < 0) return;
    const int head = work.head / S::kParts, part = work.head % S::kParts;
    const int wave = uni(threadIdx.x / 64), lane = threadIdx.x & 63, half = lane >> 5;
    const SeqTile st = a.tiles[work.tile];
    const int q0 = a.first_q[st.seq], nq = a.first_q[st.seq + 1] - q0, k0 = a.first_k[st.seq], nk = a.first_k[st.seq + 1] - k0;
    const int row0 = st.row + wave * 32, row = row0 + (lane & 31), shift = nk - nq;
    const int kv_head = head / a.group;
    const unsigned char* kb = a.k.p + (int64_t)k0 * a.k.ld + kv_head * a.k.hs;
    const unsigned char* vb = a.v.p + (int64_t)k0 * a.v.ld + kv_head * a.v.hs;
    const int seen = a.causal ? max(0, min(nk, min(st.row + 32 * W, nq) + shift)) : nk;
    const int seen_wave = row0 >= nq ? 0 : a.causal ? max(0, min(nk, min(row0 + 32, nq) + shift)) : nk;
    const int last = a.causal ? min(nk - 1, row + shift) : nk - 1;

    TileLoad<RB, KT, W> lk, lv;
    lk.init(wave, lane, a.k.ld, a.dim_bytes);
    lv.init(wave, lane, a.v.ld, a.dim_bytes);
    RowReader<DT, RB> rows_of;
    rows_of.init(lane);
    ColumnProduct<DT, RB> columns;
    columns.init(lane);
    OwnRows<DT, STEPS> q, go;
    go.load(a.gout.p + (int64_t)q0 * a.gout.ld + head * a.gout.hs, a.gout.ld, row0, nq, a.dim_bytes, lane);
    float delta = 0.f;
    {
        q.load(a.out.p + (int64_t)q0 * a.out.ld + head * a.out.hs, a.out.ld, row0, nq, a.dim_bytes, lane);
#pragma unroll
        for (int i = 0; i < STEPS; ++i)
#pragma unroll
            for (int e = 0; e < 16 / AttnType<DT>::ES; ++e) delta = fmaf((float)q.x[i][e], (float)go.x[i][e], delta);
        delta += other_half(delta);
    }
    q.load(a.q.p + (int64_t)q0 * a.q.ld + head * a.q.hs, a.q.ld, row0, nq, a.dim_bytes, lane, a.negative);
    const int64_t at = head * a.rows_q + q0 + row;
    const float lse2 = row < nq ? a.lse[at] * kLog2e : INFINITY;
    const float glse = a.glse && row < nq ? a.glse[at] : 0.f;
    // A row that sees one key has dS = glse whatever it holds; the rounding of out would leave something.  Where a sequence's keys
    // are one tile, the sum over P dP is made of the tile's own numbers below.
    const bool one_key = nk == 1, one_tile = nk <= KT;
    if (one_key) delta = 0.f;

    f32x16 acc[COLS];
#pragma unroll
    for (int c = 0; c < COLS; ++c) acc[c] = f32x16(0.f);
    const int n = a.gq.p || one_tile ? (seen + KT - 1) / KT : 0;
    if (n > 0) {
        lk.load(lds, kb, a.k.ld, 0, nk, a.dim_bytes, wave);
        lv.load(lds + 2 * S::kTile, vb, a.v.ld, 0, nk, a.dim_bytes, wave);
    }
    for (int j = 0; j < n; ++j) {
        __builtin_amdgcn_s_waitcnt(0);
        __syncthreads();
        const int b = j & 1, key0 = j * KT;
        if (j + 1 < n) {
            lk.load(lds + (b ^ 1) * S::kTile, kb, a.k.ld, key0 + KT, nk, a.dim_bytes, wave);
            lv.load(lds + (2 + (b ^ 1)) * S::kTile, vb, a.v.ld, key0 + KT, nk, a.dim_bytes, wave);
        }
        if (key0 >= seen_wave) continue;
        const lds_byte *kt = lds + b * S::kTile, *vt = lds + (2 + b) * S::kTile;
        f32x16 p = f32x16(0.f), dp = f32x16(0.f);
#pragma unroll
        for (int i = 0; i < STEPS; ++i) p = Elem<T>::mma(rows_of(kt, 0, i), q.x[i], p);
#pragma unroll
        for (int i = 0; i < STEPS; ++i) dp = Elem<T>::mma(rows_of(vt, 0, i), go.x[i], dp);
        if (one_key) dp = f32x16(0.f);
#pragma unroll
        for (int r = 0; r < 16; ++r) p[r] = __builtin_amdgcn_exp2f(fmaf(p[r], a.c, -lse2));
        const int unmasked = a.causal ? min(nk - 1, row0 + shift) : nk - 1;
        if (key0 + KT - 1 > unmasked) {
#pragma unroll
            for (int r = 0; r < 16; ++r)
                if (key0 + 8 * (r >> 2) + 4 * half + (r & 3) > last) { p[r] = 0.f; dp[r] = 0.f; }
        }
        if (one_tile && !one_key) {
            delta = 0.f;
#pragma unroll
            for (int r = 0; r < 16; ++r) delta = fmaf(p[r], dp[r], delta);
            delta += other_half(delta);
        }
        Weights<DT> w;
        f32x16 ds;
#pragma unroll
        for (int r = 0; r < 16; ++r) ds[r] = p[r] * (dp[r] - delta + glse);
        if (key0 + KT - 1 > unmasked) {
#pragma unroll
            for (int r = 0; r < 16; ++r)
                if (key0 + 8 * (r >> 2) + 4 * half + (r & 3) > last) ds[r] = 0.f;
        }
        w.set(ds);
#pragma unroll
        for (int c = 0; c < COLS; ++c) columns(acc[c], kt + part * S::kPart, 0, c, w);
    }
    if (row >= nq) return;
    if (half == 0 && part == 0) a.delta[at] = delta - glse;
    if (!a.gq.p) return;
    unsigned char* out = a.gq.p + (int64_t)(q0 + row) * a.gq.ld + head * a.gq.hs;
    const float f = a.negative ? -a.scale : a.scale;
#pragma unroll
    for (int c = 0; c < COLS; ++c) store_columns<DT>(acc[c], f, out, part * COLS + c, a.dim_bytes, half);
#endif
}

// ------------------------------------------------------------------ gradients of keys and values
template <int DT, int DP, int W>
__global__ __launch_bounds__(64 * W, DP * AttnType<DT>::ES > 256 ? 1 : 2) void k_attention_gkv(AttnArgs a) {
#if defined(__HIP_DEVICE_COMPILE__)         // the host pass has no buffer descriptors and drops stubs over them
    typedef BwdShape<DT, DP> S;
    typedef typename AttnType<DT>::T T;
    constexpr int RB = S::RB, QT = S::T, STEPS = RB / 32, COLS = S::kCols;
    extern __shared__ __attribute__((aligned(1024))) unsigned char smem[];
    lds_byte* lds = (lds_byte*)smem;
    float* stats = (float*)(smem + 4 * S::kTile);           // per buffer: lse, then delta
    const Work work = work_of(a, a.kv_heads * S::kParts);
    if (work.head < 0) return;
    const int kv_head = work.head / S::kParts, part = work.head % S::kParts;
    const int wave = uni(threadIdx.x / 64), lane = threadIdx.x & 63, half = lane >> 5;
    const SeqTile st = a.tiles[work.tile];
    const int q0 = a.first_q[st.seq], nq = a.first_q[st.seq + 1] - q0, k0 = a.first_k[st.seq], nk = a.first_k[st.seq + 1] - k0;
    // the tile that most queries see is a causal sequence's first: it is begun first
    const int tile0 = a.causal ? (nk - 1) / (32 * W) * (32 * W) - st.row : st.row;
    const int key0 = tile0 + wave * 32, key = key0 + (lane & 31), shift = nk - nq;
    const bool one_key = nk == 1;

    OwnRows<DT, STEPS> k, v;
    k.load(a.k.p + (int64_t)k0 * a.k.ld + kv_head * a.k.hs, a.k.ld, key0, nk, a.dim_bytes, lane, a.negative);
    v.load(a.v.p + (int64_t)k0 * a.v.ld + kv_head * a.v.hs, a.v.ld, key0, nk, a.dim_bytes, lane);
    TileLoad<RB, QT, W> lq, lo;
    lq.init(wave, lane, a.q.ld, a.dim_bytes);
    lo.init(wave, lane, a.gout.ld, a.dim_bytes);
    RowReader<DT, RB> rows_of;
    rows_of.init(lane);
    ColumnProduct<DT, RB> columns;
    columns.init(lane);
    f32x16 gk[COLS], gv[COLS];
#pragma unroll
    for (int c = 0; c < COLS; ++c) gk[c] = gv[c] = f32x16(0.f);
    // all heads of the group in turn; of each the tiles from the first on in which a query sees the workgroup's first key
    const int begin = a.causal ? max(0, tile0 - shift) / QT * QT : 0, n = begin < nq ? (nq - begin + QT - 1) / QT * a.group : 0;
    int next_head = kv_head * a.group, next = begin;
    auto load = [&](int b) {
        lq.load(lds + b * S::kTile, a.q.p + (int64_t)q0 * a.q.ld + next_head * a.q.hs, a.q.ld, next, nq, a.dim_bytes, wave);
        lo.load(lds + (2 + b) * S::kTile, a.gout.p + (int64_t)q0 * a.gout.ld + next_head * a.gout.hs, a.gout.ld, next, nq, a.dim_bytes, wave);
        if (threadIdx.x < 2 * QT) {
            const int r = next + threadIdx.x % QT;
            const int64_t at = next_head * a.rows_q + q0 + r;
            stats[b * 2 * QT + threadIdx.x] = threadIdx.x < QT ? (r < nq ? a.lse[at] * kLog2e : INFINITY) : r < nq ? a.delta[at] : 0.f;
        }
        next += QT;
        if (next >= nq) { next = begin; ++next_head; }
    };
    if (n > 0) load(0);
    int r0 = begin - QT;
    for (int j = 0; j < n; ++j) {
        __builtin_amdgcn_s_waitcnt(0);
        __syncthreads();
        const int b = j & 1;
        r0 += QT;
        if (r0 >= nq) r0 = begin;
        if (j + 1 < n) load(b ^ 1);
        if (key0 >= nk || (a.causal && r0 + QT - 1 + shift < key0)) continue;
        const lds_byte *qt = lds + b * S::kTile, *ot = lds + (2 + b) * S::kTile;
        f32x16 p = f32x16(0.f), dp = f32x16(0.f);
#pragma unroll
        for (int i = 0; i < STEPS; ++i) p = Elem<T>::mma(rows_of(qt, 0, i), k.x[i], p);
#pragma unroll
        for (int i = 0; i < STEPS; ++i) dp = Elem<T>::mma(rows_of(ot, 0, i), v.x[i], dp);
        if (one_key) dp = f32x16(0.f);
        f32x16 ds;
        const float* stat = stats + b * 2 * QT + 4 * half;
#pragma unroll
        for (int g = 0; g < 4; ++g) {
            const f32x4 lse = *(const f32x4*)(stat + 8 * g), delta = *(const f32x4*)(stat + QT + 8 * g);
#pragma unroll
            for (int e = 0; e < 4; ++e) {
                const int r = 4 * g + e;
                p[r] = __builtin_amdgcn_exp2f(fmaf(p[r], a.c, -lse[e]));
                ds[r] = p[r] * (dp[r] - delta[e]);
            }
        }
        if (a.causal && r0 + shift < key0 + 31) {
#pragma unroll
            for (int r = 0; r < 16; ++r)
                if (r0 + 8 * (r >> 2) + 4 * half + (r & 3) + shift < key) p[r] = ds[r] = 0.f;
        }
        Weights<DT> wp, wd;
        wp.set(p);
        wd.set(ds);
#pragma unroll
        for (int c = 0; c < COLS; ++c) columns(gv[c], ot + part * S::kPart, 0, c, wp);
#pragma unroll
        for (int c = 0; c < COLS; ++c) columns(gk[c], qt + part * S::kPart, 0, c, wd);
    }
    if (key >= nk) return;
    if (a.gk.p) {
        unsigned char* out = a.gk.p + (int64_t)(k0 + key) * a.gk.ld + kv_head * a.gk.hs;
        const float f = a.negative ? -a.scale : a.scale;
#pragma unroll
        for (int c = 0; c < COLS; ++c) store_columns<DT>(gk[c], f, out, part * COLS + c, a.dim_bytes, half);
    }
    if (a.gv.p) {
        unsigned char* out = a.gv.p + (int64_t)(k0 + key) * a.gv.ld + kv_head * a.gv.hs;
#pragma unroll
        for (int c = 0; c < COLS; ++c) store_columns<DT>(gv[c], 1.f, out, part * COLS + c, a.dim_bytes, half);
    }
#endif
}

template <int DT, int DP> static void launch_bwd(const AttnArgs& a, const AttnArgs& b, bool keys, hipStream_t st) {
    typedef BwdShape<DT, DP> S;
    const unsigned nq = (unsigned)(((int64_t)a.n_tiles * a.heads * S::kParts + 7) / 8 * 8), nk = (unsigned)(((int64_t)b.n_tiles * b.kv_heads * S::kParts + 7) / 8 * 8);
    if (nq) k_attention_gq<DT, DP, 4><<<nq, 256, S::kLds, st>>>(a);
    if (keys && nk) k_attention_gkv<DT, DP, 4><<<nk, 256, S::kLds, st>>>(b);
}

template <int DT> static void launch_bwd_dim(const AttnArgs& a, const AttnArgs& b, int dim, bool keys, hipStream_t st) {
    if (dim <= 32) launch_bwd<DT, 32>(a, b, keys, st);
    else if (dim <= 64) launch_bwd<DT, 64>(a, b, keys, st);
    else if (dim <= 128) launch_bwd<DT, 128>(a, b, keys, st);
    else launch_bwd<DT, 256>(a, b, keys, st);
}

fx_status attention_bwd_launch(const AttnArgs& a, fx_dtype dt, int dim, int64_t, int64_t longest_k, const SeqTile* k_tiles, int32_t n_k_tiles, bool keys, hipStream_t st) {
    AttnArgs b = a;
    b.tiles = k_tiles;
    b.n_tiles = n_k_tiles;
    (void)longest_k;
    if (dt == FX_F32) launch_bwd_dim<FX_F32>(a, b, dim, keys, st);
    else if (dt == FX_F16) launch_bwd_dim<FX_F16>(a, b, dim, keys, st);
    else launch_bwd_dim<FX_BF16>(a, b, dim, keys, st);
    return FX_OK;
}

}  // namespace fx
