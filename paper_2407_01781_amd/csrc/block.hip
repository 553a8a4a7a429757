// What stands around the body of a residual block: the norm before it, and behind it one pass that norms, gates, drops
// out and scales its output, adds it to the residual stream and norms the sum for the block that follows.  Dropout
// alone is the same pass without norms, gate and scale.
//
//   n(v; w)[c] = v[c] / sqrt(mean_c v^2 + eps) * w[c]
//   x'   = x + s * drop(r * act(gate)),  r = n(y; post) (y without post),   next = n(x'; next weight)
//
// All of it is bound by memory: every row is loaded once into registers, its sums are taken over the lanes that hold it
// (8 channels a lane, 8 lanes for a row of 64), and every result is written once.  Sums and all arithmetic are fp32; an
// output is rounded once, and the second norm works on x' as it is before that rounding.  Up to 512 channels rows share a
// wave and sum by lane moves; beyond, a row takes a workgroup and sums through LDS.
#include "rows.h"

namespace fx {

struct BlockArgs {
    int64_t rows;
    int32_t C;
    int32_t lanes_log2;             // lanes that share a row (256 threads where a row spans the workgroup)
    const unsigned char *x, *y, *gate;
    unsigned char *out, *norm;
    int64_t ld_x, ld_y, ld_gate, ld_out, ld_norm;       // bytes from row to row
    const void *post, *scale, *next;
    int32_t vec_f32;                // the three vectors are FX_F32 (else the rows' type)
    int32_t act;
    float eps, inv_C;
    DropArgs drop;
    // backward
    const unsigned char *gout, *gnorm;
    unsigned char *gx, *gy, *ggate;
    int64_t ld_gout, ld_gnorm, ld_gx, ld_gy, ld_ggate;
    float* partial;                 // [3][gridDim.x][C]: sums of the workgroup's rows for post, scale, next
    int32_t want;                   // bit 0 post, bit 1 scale, bit 2 next
};

enum { kModeNorm = 0, kModeJoin = 1, kModeDrop = 2 };

constexpr int kBlockThreads = 256;          // where several rows share a workgroup
constexpr int kWideThreads = 512;           // most threads of a row that takes a workgroup of its own

// sums over the lanes of a row, N of them at once
template <bool WIDE, int N>
__device__ __forceinline__ void group_sums(float (&v)[N], int lanes, float* lds) {
#pragma unroll
    for (int i = 0; i < N; ++i) v[i] = row_sum(v[i], WIDE ? 64 : lanes);
    if (!WIDE) return;
    const int waves = lanes >> 6;
    __syncthreads();                // the sums before these have been read
    if ((threadIdx.x & 63) == 0) {
#pragma unroll
        for (int i = 0; i < N; ++i) lds[i * (kWideThreads / 64) + (threadIdx.x >> 6)] = v[i];
    }
    __syncthreads();
#pragma unroll
    for (int i = 0; i < N; ++i) {
        v[i] = 0.f;
        for (int w = 0; w < waves; ++w) v[i] += lds[i * (kWideThreads / 64) + w];
    }
}

__device__ __forceinline__ float inv_rms(float sum_sq, float inv_C, float eps) { return 1.f / sqrtf(sum_sq * inv_C + eps); }

// act(z) and its derivative
__device__ __forceinline__ void gate_factors(int act, const float (&z)[kPiece], float (&f)[kPiece], float (&df)[kPiece]) {
    if (act == FX_GATE_SILU) {
#pragma unroll
        for (int e = 0; e < kPiece; ++e) {
            float up, down;
            sigmoids(z[e], up, down);
            f[e] = z[e] * up;
            df[e] = up * (1.f + z[e] * down);
        }
    } else {
#pragma unroll
        for (int e = 0; e < kPiece; ++e) {
            float down;
            sigmoids(z[e], f[e], down);
            df[e] = f[e] * down;
        }
    }
}

// The three forward passes.  A lane keeps its channels' weights while it takes row after row; the mask is drawn while the
// row's loads are on their way.  986,880 x 64 bf16: join with everything (632 MB) 116 us, 5.4 TB/s; dropout with a residual
// (379 MB) 68 us, 5.5 TB/s: a copy's rate.  128 waves a compute unit instead of the 32 it holds: 129 -> 117 us, as late
// workgroups fill the holes that others leave.
template <int DT, int KIND, bool WIDE, int MODE>
__global__ void __launch_bounds__(WIDE ? kWideThreads : kBlockThreads)
k_block_fwd(BlockArgs a) {
    __shared__ float lds[WIDE ? kWideThreads / 64 : 1];
    const int lanes = 1 << a.lanes_log2, lane = threadIdx.x & (lanes - 1), C = a.C, col = lane * kPiece;
    const int rows_here = WIDE ? 1 : kBlockThreads >> a.lanes_log2;
    const uint32_t mask = lane_mask(col, C);
    const uint64_t offset = a.drop.offset + (a.drop.d_more ? *a.drop.d_more : 0);
    float wp[kPiece], ws[kPiece], wn[kPiece];
    if (MODE == kModeJoin) load_vector<DT, KIND>(a.post, a.vec_f32, col, C, 1.f, wp);
    if (MODE == kModeJoin) load_vector<DT, KIND>(a.scale, a.vec_f32, col, C, 1.f, ws);
    if (MODE != kModeDrop) load_vector<DT, KIND>(a.next, a.vec_f32, col, C, 1.f, wn);
    for (int64_t r0 = (int64_t)blockIdx.x * rows_here; r0 < a.rows; r0 += (int64_t)gridDim.x * rows_here) {
        const int64_t mine = WIDE ? r0 : r0 + (threadIdx.x >> a.lanes_log2);
        const bool real = mine < a.rows;
        const int64_t row = real ? mine : a.rows - 1;
        Piece<DT> px, py, pg;
        if (MODE == kModeNorm || a.x) px = load_piece<DT, KIND>(a.x + row * a.ld_x, 0, col, C);
        if (MODE != kModeNorm) py = load_piece<DT, KIND>(a.y + row * a.ld_y, 0, col, C);
        if (MODE == kModeJoin && a.gate) pg = load_piece<DT, KIND>(a.gate + row * a.ld_gate, 0, col, C);
        float v[kPiece];
        unpack<DT>(masked(MODE == kModeNorm ? px : py, mask), v);
        if (MODE == kModeJoin && a.post) {
            float s[1] = {0.f};
#pragma unroll
            for (int e = 0; e < kPiece; ++e) s[0] += v[e] * v[e];
            group_sums<WIDE>(s, lanes, lds);
            const float rs = inv_rms(s[0], a.inv_C, a.eps);
#pragma unroll
            for (int e = 0; e < kPiece; ++e) v[e] *= rs * wp[e];
        }
        if (MODE == kModeJoin && a.gate) {
            float z[kPiece], f[kPiece], df[kPiece];
            unpack<DT>(pg, z);
            gate_factors(a.act, z, f, df);
#pragma unroll
            for (int e = 0; e < kPiece; ++e) v[e] *= f[e];
        }
        if (MODE != kModeNorm) {
            if (a.drop.below) {
                uint32_t w[4];
                philox8((uint32_t)lane, (uint32_t)row, offset, a.drop.seed, w);
#pragma unroll
                for (int e = 0; e < kPiece; ++e) v[e] = drop_value(w, e, a.drop, v[e]);
            }
            if (MODE == kModeJoin) {
                // A lane without channels holds the gate and weights of the row's last piece under a mask of its own: its
                // zeros times an infinite gate, which that piece may have dropped, must not enter the sum of the next norm.
#pragma unroll
                for (int e = 0; e < kPiece; ++e) v[e] = kept(v[e] * ws[e], mask);
            }
            if (a.x) {
                float x[kPiece];
                unpack<DT>(masked(px, mask), x);
#pragma unroll
                for (int e = 0; e < kPiece; ++e) v[e] += x[e];
            }
            if (WIDE) __syncthreads();      // an output may lie where an input lies: all waves have their pieces of the row
            if (real) store_piece<DT, KIND>(a.out + row * a.ld_out, 0, col, C, pack<DT>(v));
        }
        if (MODE == kModeNorm || (MODE == kModeJoin && a.next)) {
            float s[1] = {0.f};
#pragma unroll
            for (int e = 0; e < kPiece; ++e) s[0] += v[e] * v[e];
            group_sums<WIDE>(s, lanes, lds);
            const float rs = inv_rms(s[0], a.inv_C, a.eps);
#pragma unroll
            for (int e = 0; e < kPiece; ++e) v[e] *= rs * wn[e];
            if (real) store_piece<DT, KIND>(a.norm + row * a.ld_norm, 0, col, C, pack<DT>(v));
        }
    }
}

// The workgroup's sums of one vector's gradient to its row of the partial sums.
template <bool WIDE>
__device__ __forceinline__ void write_partial(float (&acc)[kPiece], int lanes, int C, float* out, float (*lds)[64 * kPiece]) {
    const int lane = threadIdx.x & (lanes - 1);
    if (WIDE) {
#pragma unroll
        for (int e = 0; e < kPiece; ++e)
            if (lane * kPiece + e < C) out[lane * kPiece + e] = acc[e];
        return;
    }
#pragma unroll
    for (int e = 0; e < kPiece; ++e)
        for (int o = lanes; o < 64; o <<= 1) acc[e] += __shfl_xor(acc[e], o);
    __syncthreads();
    if ((int)(threadIdx.x & 63) < lanes) {
#pragma unroll
        for (int e = 0; e < kPiece; ++e) lds[threadIdx.x >> 6][lane * kPiece + e] = acc[e];
    }
    __syncthreads();
    for (int i = threadIdx.x; i < min(C, lanes * kPiece); i += kBlockThreads) out[i] = (lds[0][i] + lds[1][i]) + (lds[2][i] + lds[3][i]);
}

// Gradients.  With D = gout + J^T gnorm (the gradient of x'), keep = 0 or drop's factor, yh = y / rms(y):
//   gx = D,  gscale = sum_rows D keep r a,  ggate = D keep s r a',  u = D keep s a  (a = act(gate), a' its derivative)
//   gpost = sum_rows u yh,  gy = J^T u,  gnext = sum_rows gnorm x'h
//   J^T of n(v; w) on g:  (g w - vh mean_c(g w vh)) / rms(v)
// The three sums over rows run in every lane's registers over the rows that its workgroup takes, are joined in the
// workgroup and added over the workgroups, in index order, by k_block_sums: the same bits from every call.
// 1,068,658 x 64 f16 with everything (1094 MB): 222 us, 4.9 TB/s, near a copy's rate, at 184 registers and so eight waves a
// compute unit, which is also how many workgroups are launched: 16 waves took 230 us where 8 took 217, the rows' sums of
// each being joined once.  Selecting what is dropped costs 3 of the 222 us and 8 registers (one word of bits a lane in place
// of eight masks: 7 us more); held to 168 or 128 registers the form without it spilled (221, 687 us).  The norm alone (77 registers) 194,497 x 256 bf16 54 us, best at 16
// waves (8: 95 us for 76 at 986,880 x 64).  A row that is small is bound by latency: 20,011 x 45 fp32 16 us for 22 MB.
template <int DT, int KIND, bool WIDE, int MODE>
__global__ void __launch_bounds__(WIDE ? kWideThreads : kBlockThreads)
k_block_bwd(BlockArgs a) {
    __shared__ float lds_sum[WIDE ? 3 * kWideThreads / 64 : 1];
    __shared__ float lds[WIDE ? 1 : 4][64 * kPiece];
    const int lanes = 1 << a.lanes_log2, lane = threadIdx.x & (lanes - 1), C = a.C, col = lane * kPiece;
    const int rows_here = WIDE ? 1 : kBlockThreads >> a.lanes_log2;
    const uint32_t mask = lane_mask(col, C);
    const uint64_t offset = a.drop.offset + (a.drop.d_more ? *a.drop.d_more : 0);
    float wp[kPiece], ws[kPiece], wn[kPiece], acc_post[kPiece], acc_scale[kPiece], acc_next[kPiece];
    if (MODE == kModeJoin) load_vector<DT, KIND>(a.post, a.vec_f32, col, C, 1.f, wp);
    if (MODE == kModeJoin) load_vector<DT, KIND>(a.scale, a.vec_f32, col, C, 1.f, ws);
    load_vector<DT, KIND>(a.next, a.vec_f32, col, C, 1.f, wn);
#pragma unroll
    for (int e = 0; e < kPiece; ++e) acc_post[e] = acc_scale[e] = acc_next[e] = 0.f;
    for (int64_t r0 = (int64_t)blockIdx.x * rows_here; r0 < a.rows; r0 += (int64_t)gridDim.x * rows_here) {
        const int64_t mine = WIDE ? r0 : r0 + (threadIdx.x >> a.lanes_log2);
        const bool real = mine < a.rows;
        const int64_t row = real ? mine : a.rows - 1;
        Piece<DT> px, py, pg, pgo, pgn;
        if (a.gnorm) {
            px = load_piece<DT, KIND>(a.x + row * a.ld_x, 0, col, C);
            pgn = load_piece<DT, KIND>(a.gnorm + row * a.ld_gnorm, 0, col, C);
        }
        if (a.gout) pgo = load_piece<DT, KIND>(a.gout + row * a.ld_gout, 0, col, C);
        if (MODE == kModeJoin) py = load_piece<DT, KIND>(a.y + row * a.ld_y, 0, col, C);
        if (MODE == kModeJoin && a.gate) pg = load_piece<DT, KIND>(a.gate + row * a.ld_gate, 0, col, C);
        // a row that does not exist counts as zeros, and as if its norms were 1
        const uint32_t m = real ? mask : 0;
        float sums[3] = {0.f, 0.f, 0.f};         // x'^2, gnorm w x', y^2
        float x[kPiece], g[kPiece], D[kPiece], y[kPiece];
        if (a.gnorm) {
            unpack<DT>(masked(px, m), x);
            unpack<DT>(masked(pgn, m), g);
#pragma unroll
            for (int e = 0; e < kPiece; ++e) { sums[0] += x[e] * x[e]; sums[1] += g[e] * wn[e] * x[e]; }
        }
        if (MODE == kModeJoin) {
            unpack<DT>(masked(py, m), y);
#pragma unroll
            for (int e = 0; e < kPiece; ++e) sums[2] += y[e] * y[e];
        }
        group_sums<WIDE>(sums, lanes, lds_sum);
        const float rx = real ? inv_rms(sums[0], a.inv_C, a.eps) : 1.f;
        const float ry = real && a.post ? inv_rms(sums[2], a.inv_C, a.eps) : 1.f;       // without post, r is y
        const float cx = sums[1] * a.inv_C * rx * rx;
#pragma unroll
        for (int e = 0; e < kPiece; ++e) D[e] = 0.f;
        if (a.gout) unpack<DT>(masked(pgo, m), D);
        if (a.gnorm) {
#pragma unroll
            for (int e = 0; e < kPiece; ++e) {
                D[e] += rx * (g[e] * wn[e] - x[e] * cx);
                acc_next[e] += g[e] * (x[e] * rx);
            }
        }
        if (real && a.gx) store_piece<DT, KIND>(a.gx + row * a.ld_gx, 0, col, C, pack<DT>(D));
        if (MODE == kModeJoin) {
            // What was dropped, and what a lane without channels or a row that does not exist holds, is selected out of the
            // products: its gate or its norm may be infinite or NaN, and zero times either is not zero.
            uint32_t keep[kPiece];
#pragma unroll
            for (int e = 0; e < kPiece; ++e) keep[e] = m;
            if (a.drop.below) {
                uint32_t w[4];
                philox8((uint32_t)lane, (uint32_t)row, offset, a.drop.seed, w);
#pragma unroll
                for (int e = 0; e < kPiece; ++e) {
                    D[e] = drop_value(w, e, a.drop, D[e]);
                    keep[e] = drop_keeps(w, e, a.drop.below) ? m : 0u;
                }
            }
            float f[kPiece], df[kPiece];
#pragma unroll
            for (int e = 0; e < kPiece; ++e) { f[e] = 1.f; df[e] = 0.f; }
            if (a.gate) {
                float z[kPiece];
                unpack<DT>(pg, z);
#pragma unroll
                for (int e = 0; e < kPiece; ++e) z[e] = kept(z[e], keep[e]);
                gate_factors(a.act, z, f, df);
            }
            float dot[1] = {0.f};                // u post yh
#pragma unroll
            for (int e = 0; e < kPiece; ++e) {
                y[e] *= ry;                      // yh
                const float yk = kept(y[e], keep[e]), r = yk * wp[e];
                acc_scale[e] += D[e] * (r * f[e]);
                const float t = D[e] * ws[e], u = t * f[e];
                df[e] *= t * r;
                acc_post[e] += u * yk;
                D[e] = u * wp[e];
                dot[0] += D[e] * yk;
            }
            if (real && a.ggate) store_piece<DT, KIND>(a.ggate + row * a.ld_ggate, 0, col, C, pack<DT>(df));
            if (a.post) {
                group_sums<WIDE>(dot, lanes, lds_sum);
                const float cy = dot[0] * a.inv_C;
#pragma unroll
                for (int e = 0; e < kPiece; ++e) D[e] = ry * (D[e] - y[e] * cy);
            }
            if (real && a.gy) store_piece<DT, KIND>(a.gy + row * a.ld_gy, 0, col, C, pack<DT>(D));
        }
    }
    const int64_t vec = (int64_t)gridDim.x * C;
    float* mine = a.partial + (int64_t)blockIdx.x * C;
    if (MODE == kModeJoin && (a.want & 1)) write_partial<WIDE>(acc_post, lanes, C, mine, lds);
    if (MODE == kModeJoin && (a.want & 2)) write_partial<WIDE>(acc_scale, lanes, C, mine + vec, lds);
    if (a.want & 4) write_partial<WIDE>(acc_next, lanes, C, mine + 2 * vec, lds);
}

// out[c] = sum over the workgroups' partial sums: 64 slices of them in index order, then the slices.  4 us for 512 x 192,
// bound by the latency of eight loads in a row and the launch (8 slices: 7 us).
template <int DT>
__global__ void __launch_bounds__(1024)
k_block_sums(const float* __restrict__ partial, int n, int C, void* out0, void* out1, void* out2) {
    __shared__ float lds[64][16];
    void* out = blockIdx.y == 0 ? out0 : blockIdx.y == 1 ? out1 : out2;
    if (!out) return;
    const int c = blockIdx.x * 16 + (threadIdx.x & 15), slice = threadIdx.x >> 4, per = (n + 63) / 64;
    float s = 0.f;
    if (c < C) {
        const float* in = partial + (int64_t)blockIdx.y * n * C + c;
        const int end = min(n, (slice + 1) * per);
#pragma unroll 16
        for (int i = slice * per; i < end; ++i) s += in[(int64_t)i * C];
    }
    lds[slice][threadIdx.x & 15] = s;
    __syncthreads();
    if (slice == 0 && c < C) {
        s = 0.f;
#pragma unroll 16
        for (int i = 0; i < 64; ++i) s += lds[i][threadIdx.x];
        if (DT == FX_F32) reinterpret_cast<float*>(out)[c] = s;
        else if (DT == FX_F16) reinterpret_cast<uint16_t*>(out)[c] = Elem<_Float16>::from_float(s);
        else reinterpret_cast<uint16_t*>(out)[c] = Elem<__bf16>::from_float(s);
    }
}

// ---------------------------------------------------------------------------------- host
static int esize(fx_dtype dt) { return dt == FX_F32 ? 4 : 2; }
static bool known(fx_dtype dt) { return dt == FX_F32 || dt == FX_F16 || dt == FX_BF16; }

// lanes that share a row; beyond a wave's 512 channels a row takes a workgroup of that many threads
struct RowShape {
    int lanes_log2;
    bool wide() const { return lanes_log2 > 6; }
    int threads() const { return wide() ? 1 << lanes_log2 : kBlockThreads; }
    int rows() const { return threads() >> lanes_log2; }
};

static RowShape row_shape(int32_t C) {
    RowShape s{0};
    while ((kPiece << s.lanes_log2) < C) ++s.lanes_log2;
    return s;
}

// Workgroups of a launch: all rows at once while they are few; from `most` waves a compute unit on, each takes several
// rows in turn.
static unsigned row_blocks(int64_t rows, const RowShape& s, int most) {
    return (unsigned)std::min<int64_t>((rows + s.rows() - 1) / s.rows(), (int64_t)compute_units() * std::max(1, most * 64 / s.threads()));
}

template <int DT, int KIND, int MODE>
static void launch_fwd(const BlockArgs& a, const RowShape& s, unsigned nb, hipStream_t st) {
    if (s.wide()) k_block_fwd<DT, KIND, true, MODE><<<nb, s.threads(), 0, st>>>(a);
    else k_block_fwd<DT, KIND, false, MODE><<<nb, s.threads(), 0, st>>>(a);
}

template <int DT, int KIND, int MODE>
static void launch_bwd(const BlockArgs& a, const RowShape& s, unsigned nb, hipStream_t st) {
    if (s.wide()) k_block_bwd<DT, KIND, true, MODE><<<nb, s.threads(), 0, st>>>(a);
    else k_block_bwd<DT, KIND, false, MODE><<<nb, s.threads(), 0, st>>>(a);
}

template <int DT, int MODE>
static void launch_block_kind(bool bwd, const BlockArgs& a, const RowShape& s, unsigned nb, hipStream_t st) {
    const int kind = a.C < kPiece ? kRowsNarrow : a.C % kPiece ? kRowsRagged : kRowsWhole;
#define FX_BLOCK(KIND) do { if (bwd) launch_bwd<DT, KIND, MODE == kModeDrop ? kModeJoin : MODE>(a, s, nb, st); \
                            else launch_fwd<DT, KIND, MODE>(a, s, nb, st); } while (0)
    if (kind == kRowsWhole) FX_BLOCK(kRowsWhole);
    else if (kind == kRowsRagged) FX_BLOCK(kRowsRagged);
    else FX_BLOCK(kRowsNarrow);
#undef FX_BLOCK
}

template <int MODE>
static void launch_block(bool bwd, fx_dtype dt, const BlockArgs& a, const RowShape& s, unsigned nb, hipStream_t st) {
    if (dt == FX_F32) launch_block_kind<FX_F32, MODE>(bwd, a, s, nb, st);
    else if (dt == FX_F16) launch_block_kind<FX_F16, MODE>(bwd, a, s, nb, st);
    else launch_block_kind<FX_BF16, MODE>(bwd, a, s, nb, st);
}

constexpr int kFwdWaves = 128, kBwdWaves = 8, kNormBwdWaves = 16;     // of a compute unit in one launch

static fx_status check_rows(const char* who, int64_t rows, int32_t C, fx_dtype dt) {
    if (rows < 0 || C < 1 || !known(dt)) { set_error("%s: negative rows, no channels or unknown dtype", who); return FX_EINVAL; }
    if (rows > 0x7FFFFFFFll || C > kMaxRowChannels) {
        set_error("%s: more than 2^31-1 rows or %d channels", who, kMaxRowChannels);
        return FX_ERANGE;
    }
    return FX_OK;
}

// a tensor of rows: there, aligned to its elements, rows that do not overlap
static fx_status check_tensor(const char* who, const char* name, const void* p, int64_t ld, int64_t rows, int32_t C, fx_dtype dt, bool needed) {
    if (!p) {
        if (!needed || rows == 0) return FX_OK;
        set_error("%s: %s is null", who, name);
        return FX_EINVAL;
    }
    if ((uintptr_t)p % esize(dt) || ld < C) {
        set_error("%s: %s is not aligned to its elements or has rows closer than C", who, name);
        return FX_EINVAL;
    }
    return FX_OK;
}

static fx_status check_vector(const char* who, const char* name, const void* p, fx_dtype dt) {
    if ((uintptr_t)p % esize(dt)) { set_error("%s: %s is not aligned to its elements", who, name); return FX_EINVAL; }
    return FX_OK;
}

static fx_status drop_args(const char* who, double p, uint64_t seed, uint64_t offset, const uint64_t* d_more, DropArgs* d) {
    if (!(p >= 0.0 && p <= 1.0) || (uintptr_t)d_more % 8) { set_error("%s: dropout's probability outside [0, 1] or its offset not aligned", who); return FX_EINVAL; }
    d->seed = seed;
    d->offset = offset;
    d->d_more = d_more;
    d->below = (uint32_t)(p * 65536.0 + 0.5);
    const double factor = d->below < 65536 ? 65536.0 / (65536.0 - d->below) : 0.0;
    d->factor = (float)factor;
    d->rest = (float)(factor - d->factor);
    return FX_OK;
}

// The last step of both backward calls: vectors over the workgroups' partial sums, zeros where there are no rows.
static fx_status finish_sums(fx_dtype vec_dt, const BlockArgs& a, unsigned nb, void* gpost, void* gscale, void* gnext, hipStream_t st) {
    ProfScope ps(kProfBlockSums, st);
    const dim3 grid((a.C + 15) / 16, 3);
    if (vec_dt == FX_F32) k_block_sums<FX_F32><<<grid, 1024, 0, st>>>(a.partial, (int)nb, a.C, gpost, gscale, gnext);
    else if (vec_dt == FX_F16) k_block_sums<FX_F16><<<grid, 1024, 0, st>>>(a.partial, (int)nb, a.C, gpost, gscale, gnext);
    else k_block_sums<FX_BF16><<<grid, 1024, 0, st>>>(a.partial, (int)nb, a.C, gpost, gscale, gnext);
    FX_HIP_TRY(hipGetLastError());
    return FX_OK;
}

template <int MODE>
static fx_status run_bwd(fx_dtype dt, fx_dtype vec_dt, BlockArgs& a, void* gpost, void* gscale, void* gnext, hipStream_t st) {
    const RowShape shape = row_shape(a.C);
    const unsigned nb = row_blocks(a.rows, shape, MODE == kModeNorm ? kNormBwdWaves : kBwdWaves);
    a.lanes_log2 = shape.lanes_log2;
    a.want = (gpost ? 1 : 0) | (gscale ? 2 : 0) | (gnext ? 4 : 0);
    void* partial = nullptr;
    if (a.want) FX_TRY(scratch_alloc(MODE == kModeNorm ? "fx_rms_norm_bwd" : "fx_block_join_bwd", &partial, (size_t)3 * std::max(nb, 1u) * a.C * sizeof(float), st));
    a.partial = (float*)partial;
    fx_status s = FX_OK;
    if (nb) {
        ProfScope ps(kProfBlockBwd, st);
        launch_block<MODE>(true, dt, a, shape, nb, st);
        const hipError_t e = hipGetLastError();
        if (e != hipSuccess) { set_error("launch of k_block_bwd failed: %s", hipGetErrorString(e)); s = FX_EDEVICE; }
    }
    if (s == FX_OK && a.want) s = finish_sums(vec_dt, a, nb, gpost, gscale, gnext, st);
    dev_free(partial, st);
    return s;
}

static void common_args(BlockArgs* a, int64_t rows, int32_t C, float eps) {
    *a = BlockArgs{};
    a->rows = rows;
    a->C = C;
    a->eps = eps;
    a->inv_C = 1.f / (float)C;
}

static bool good_eps(float eps) { return eps >= 0.f && eps < __builtin_inff(); }

}  // namespace fx

using namespace fx;

extern "C" fx_status fx_rms_norm_fwd(const void* d_x, int64_t ld_x, fx_dtype dt, int64_t rows, int32_t C, const void* d_weight,
                                     fx_dtype vec_dt, float eps, void* d_out, int64_t ld_out, void* stream) {
    const char* who = "fx_rms_norm_fwd";
    FX_TRY(check_rows(who, rows, C, dt));
    if ((vec_dt != dt && vec_dt != FX_F32) || !good_eps(eps)) { set_error("%s: the weight's dtype is neither the rows' nor FX_F32, or eps is negative or not finite", who); return FX_EINVAL; }
    FX_TRY(check_tensor(who, "d_x", d_x, ld_x, rows, C, dt, true));
    FX_TRY(check_tensor(who, "d_out", d_out, ld_out, rows, C, dt, true));
    FX_TRY(check_vector(who, "d_weight", d_weight, vec_dt));
    if (rows == 0) return FX_OK;
    BlockArgs a;
    common_args(&a, rows, C, eps);
    const int es = esize(dt);
    a.x = (const unsigned char*)d_x; a.ld_x = ld_x * es;
    a.norm = (unsigned char*)d_out; a.ld_norm = ld_out * es;
    a.next = d_weight; a.vec_f32 = vec_dt == FX_F32;
    const RowShape shape = row_shape(C);
    a.lanes_log2 = shape.lanes_log2;
    hipStream_t st = (hipStream_t)stream;
    ProfScope ps(kProfBlockFwd, st);
    launch_block<kModeNorm>(false, dt, a, shape, row_blocks(rows, shape, kFwdWaves), st);
    FX_HIP_TRY(hipGetLastError());
    return FX_OK;
}

extern "C" fx_status fx_rms_norm_bwd(const void* d_gout, int64_t ld_gout, const void* d_x, int64_t ld_x, fx_dtype dt, int64_t rows,
                                     int32_t C, const void* d_weight, fx_dtype vec_dt, float eps, void* d_gx, int64_t ld_gx,
                                     void* d_gweight, void* stream) {
    const char* who = "fx_rms_norm_bwd";
    FX_TRY(check_rows(who, rows, C, dt));
    if ((vec_dt != dt && vec_dt != FX_F32) || !good_eps(eps)) { set_error("%s: the weight's dtype is neither the rows' nor FX_F32, or eps is negative or not finite", who); return FX_EINVAL; }
    FX_TRY(check_tensor(who, "d_gout", d_gout, ld_gout, rows, C, dt, true));
    FX_TRY(check_tensor(who, "d_x", d_x, ld_x, rows, C, dt, true));
    FX_TRY(check_tensor(who, "d_gx", d_gx, ld_gx, rows, C, dt, false));
    FX_TRY(check_vector(who, "d_weight", d_weight, vec_dt));
    FX_TRY(check_vector(who, "d_gweight", d_gweight, vec_dt));
    BlockArgs a;
    common_args(&a, rows, C, eps);
    const int es = esize(dt);
    a.x = (const unsigned char*)d_x; a.ld_x = ld_x * es;
    a.gnorm = (const unsigned char*)d_gout; a.ld_gnorm = ld_gout * es;
    a.gx = (unsigned char*)d_gx; a.ld_gx = ld_gx * es;
    a.next = d_weight; a.vec_f32 = vec_dt == FX_F32;
    return run_bwd<kModeNorm>(dt, vec_dt, a, nullptr, nullptr, d_gweight, (hipStream_t)stream);
}

static fx_status check_join(const char* who, const fx_block_join* b, BlockArgs* a) {
    if (!b) { set_error("%s: null description", who); return FX_EINVAL; }
    FX_TRY(check_rows(who, b->rows, b->C, b->dt));
    if ((b->vec_dt != b->dt && b->vec_dt != FX_F32) || !good_eps(b->eps) || (b->act != FX_GATE_SIGMOID && b->act != FX_GATE_SILU)) {
        set_error("%s: the vectors' dtype is neither the rows' nor FX_F32, eps is negative or not finite, or the gate's function is unknown", who);
        return FX_EINVAL;
    }
    FX_TRY(check_tensor(who, "d_y", b->d_y, b->ld_y, b->rows, b->C, b->dt, true));
    FX_TRY(check_tensor(who, "d_gate", b->d_gate, b->ld_gate, b->rows, b->C, b->dt, false));
    FX_TRY(check_vector(who, "d_post", b->d_post, b->vec_dt));
    FX_TRY(check_vector(who, "d_scale", b->d_scale, b->vec_dt));
    FX_TRY(check_vector(who, "d_next", b->d_next, b->vec_dt));
    common_args(a, b->rows, b->C, b->eps);
    FX_TRY(drop_args(who, b->p, b->seed, b->offset, b->d_offset, &a->drop));
    const int es = esize(b->dt);
    a->y = (const unsigned char*)b->d_y; a->ld_y = b->ld_y * es;
    a->gate = (const unsigned char*)b->d_gate; a->ld_gate = b->ld_gate * es;
    a->post = b->d_post; a->scale = b->d_scale; a->next = b->d_next;
    a->vec_f32 = b->vec_dt == FX_F32;
    a->act = b->act;
    return FX_OK;
}

extern "C" fx_status fx_block_join_fwd(const fx_block_join* b, const void* d_x, int64_t ld_x, void* d_out, int64_t ld_out, void* d_norm,
                                       int64_t ld_norm, void* stream) {
    const char* who = "fx_block_join_fwd";
    BlockArgs a;
    FX_TRY(check_join(who, b, &a));
    FX_TRY(check_tensor(who, "d_x", d_x, ld_x, b->rows, b->C, b->dt, true));
    FX_TRY(check_tensor(who, "d_out", d_out, ld_out, b->rows, b->C, b->dt, true));
    FX_TRY(check_tensor(who, "d_norm", d_norm, ld_norm, b->rows, b->C, b->dt, b->d_next != nullptr));
    if (d_norm && !b->d_next) { set_error("%s: d_norm without d_next", who); return FX_EINVAL; }
    if (b->rows > 0 && d_norm == d_out) { set_error("%s: d_out and d_norm are the same", who); return FX_EINVAL; }
    if (b->rows == 0) return FX_OK;
    const int es = esize(b->dt);
    a.x = (const unsigned char*)d_x; a.ld_x = ld_x * es;
    a.out = (unsigned char*)d_out; a.ld_out = ld_out * es;
    a.norm = (unsigned char*)d_norm; a.ld_norm = ld_norm * es;
    const RowShape shape = row_shape(b->C);
    a.lanes_log2 = shape.lanes_log2;
    hipStream_t st = (hipStream_t)stream;
    ProfScope ps(kProfBlockFwd, st);
    launch_block<kModeJoin>(false, b->dt, a, shape, row_blocks(b->rows, shape, kFwdWaves), st);
    FX_HIP_TRY(hipGetLastError());
    return FX_OK;
}

extern "C" fx_status fx_block_join_bwd(const fx_block_join* b, const void* d_gout, int64_t ld_gout, const void* d_gnorm, int64_t ld_gnorm,
                                       const void* d_out, int64_t ld_out, void* d_gx, int64_t ld_gx, void* d_gy, int64_t ld_gy,
                                       void* d_ggate, int64_t ld_ggate, void* d_gpost, void* d_gscale, void* d_gnext, void* stream) {
    const char* who = "fx_block_join_bwd";
    BlockArgs a;
    FX_TRY(check_join(who, b, &a));
    const int64_t rows = b->rows;
    const int32_t C = b->C;
    if ((d_gnorm || d_gnext) && !b->d_next) { set_error("%s: the next norm's gradients without d_next", who); return FX_EINVAL; }
    if (rows > 0 && !d_gout && !d_gnorm) { set_error("%s: no gradient of either output", who); return FX_EINVAL; }
    if ((d_ggate && !b->d_gate) || (d_gpost && !b->d_post) || (d_gscale && !b->d_scale)) {
        set_error("%s: the gradient of an input that is absent", who);
        return FX_EINVAL;
    }
    FX_TRY(check_tensor(who, "d_gout", d_gout, ld_gout, rows, C, b->dt, false));
    FX_TRY(check_tensor(who, "d_gnorm", d_gnorm, ld_gnorm, rows, C, b->dt, false));
    FX_TRY(check_tensor(who, "d_out", d_out, ld_out, rows, C, b->dt, d_gnorm != nullptr));
    FX_TRY(check_tensor(who, "d_gx", d_gx, ld_gx, rows, C, b->dt, false));
    FX_TRY(check_tensor(who, "d_gy", d_gy, ld_gy, rows, C, b->dt, false));
    FX_TRY(check_tensor(who, "d_ggate", d_ggate, ld_ggate, rows, C, b->dt, false));
    if (rows > 0 && ((d_gx && (d_gx == d_gy || d_gx == d_ggate)) || (d_gy && d_gy == d_ggate))) {
        set_error("%s: two of d_gx, d_gy and d_ggate are the same", who);
        return FX_EINVAL;
    }
    FX_TRY(check_vector(who, "d_gpost", d_gpost, b->vec_dt));
    FX_TRY(check_vector(who, "d_gscale", d_gscale, b->vec_dt));
    FX_TRY(check_vector(who, "d_gnext", d_gnext, b->vec_dt));
    const int es = esize(b->dt);
    a.x = (const unsigned char*)d_out; a.ld_x = ld_out * es;
    a.gout = (const unsigned char*)d_gout; a.ld_gout = ld_gout * es;
    a.gnorm = (const unsigned char*)d_gnorm; a.ld_gnorm = ld_gnorm * es;
    a.gx = (unsigned char*)d_gx; a.ld_gx = ld_gx * es;
    a.gy = (unsigned char*)d_gy; a.ld_gy = ld_gy * es;
    a.ggate = (unsigned char*)d_ggate; a.ld_ggate = ld_ggate * es;
    return run_bwd<kModeJoin>(b->dt, b->vec_dt, a, d_gpost, d_gscale, d_gnext, (hipStream_t)stream);
}

extern "C" fx_status fx_dropout(const void* d_x, int64_t ld_x, fx_dtype dt, int64_t rows, int32_t C, double p, uint64_t seed, uint64_t offset,
                                const uint64_t* d_offset, const void* d_residual, int64_t ld_residual, void* d_out, int64_t ld_out,
                                void* stream) {
    const char* who = "fx_dropout";
    FX_TRY(check_rows(who, rows, C, dt));
    FX_TRY(check_tensor(who, "d_x", d_x, ld_x, rows, C, dt, true));
    FX_TRY(check_tensor(who, "d_residual", d_residual, ld_residual, rows, C, dt, false));
    FX_TRY(check_tensor(who, "d_out", d_out, ld_out, rows, C, dt, true));
    BlockArgs a;
    common_args(&a, rows, C, 0.f);
    FX_TRY(drop_args(who, p, seed, offset, d_offset, &a.drop));
    if (rows == 0) return FX_OK;
    const int es = esize(dt);
    a.y = (const unsigned char*)d_x; a.ld_y = ld_x * es;
    a.x = (const unsigned char*)d_residual; a.ld_x = ld_residual * es;
    a.out = (unsigned char*)d_out; a.ld_out = ld_out * es;
    const RowShape shape = row_shape(C);
    a.lanes_log2 = shape.lanes_log2;
    hipStream_t st = (hipStream_t)stream;
    ProfScope ps(kProfDropout, st);
    launch_block<kModeDrop>(false, dt, a, shape, row_blocks(rows, shape, kFwdWaves), st);
    FX_HIP_TRY(hipGetLastError());
    return FX_OK;
}
