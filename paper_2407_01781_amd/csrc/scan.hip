// Gated linear recurrence along the rows of a batch of sequences (the voxels of a grid in index order are one: leaf by
// leaf, so that neighbours in the sequence are neighbours in space), per channel:
//
//     h_t = f_t h_(t-1) + (1 - f_t) x_t,   f = sigmoid(gate),   h before the first row = h0
//
// and its gradients, with lambda_t the gradient of h_t and m_t = f_t lambda_t what reaches h_(t-1):
//
//     lambda_t = dh_t + m_(t+1),   m_t = f_t (dh_t + m_(t+1)),   m behind the last row = the gradient of the last state
//     dx_t = (1 - f_t) lambda_t,   dgate_t = lambda_t (h_(t-1) - x_t) f_t (1 - f_t),   dh0 = m of the first row
//
// so both ways are the same scan v <- f v + b, with b = (1 - f) x over the rows in order and b = f dh against it.  A
// run of rows acts on the value before it as v <- A v + H; runs compose as (A, H) then (A', H') = (A A', A' H + H').
// A run in which a sequence begins ignores the value before it: A = -1 marks that (a product of gates is never
// negative), and the composition selects, so that nothing of one sequence, an infinity or NaN neither, reaches the
// next.  All of it is fp32.
//
// One pass over the data.  A tile is some hundred rows of up to 64 channels: 8 lanes hold a row (8 channels each, 128
// bytes of a 16-bit type), and every lane takes a few rows that follow each other, in registers from the load to the
// store.  A workgroup scans its tile's runs in LDS, publishes the tile's (A, H), looks back over the tiles before it for
// the value that its first row starts from, and finishes its rows.  Tiles are taken in scan order by ticket, so whatever
// a workgroup waits for belongs to a workgroup that already runs, and that one waits for earlier tiles only.
#include "rows.h"

#include <mutex>
#include <new>
#include <vector>

struct fx_sequences {
    int64_t rows = 0;
    int32_t B = 0, n_empty = 0;
    void* buf = nullptr;
    hipStream_t stream = nullptr;
    // bit r: a sequence begins at row r; row `rows` counts as a beginning.  Words up to the one after that.
    const uint64_t* d_begin = nullptr;
    const int32_t* d_rank = nullptr;        // beginnings before each word
    const int32_t* d_id = nullptr;          // number of the k-th sequence that is not empty
    const int32_t* d_empty = nullptr;       // numbers of the empty ones
};

namespace fx {

constexpr int kScanThreads = 512;       // most threads of a workgroup
constexpr int kGroupTiles = 16;         // tiles whose joint (A, H) is published as one
constexpr int kLookWindow = 16;         // groups looked at together

// Rows of a lane: as many as leave a workgroup's registers (gate, input and, backward, state and x of all its rows) room
// for a second one on the compute unit.
template <int DT, bool BWD> struct ScanRows { static constexpr int n = BWD && DT == FX_F32 ? 2 : 4; };

struct ScanArgs {
    int64_t rows;
    int32_t C, lanes_log2;              // lanes of a row within the slab
    int32_t slabs, tiles, groups;       // 64 channels; tiles of a slab; groups of tiles
    const unsigned char *x, *gate, *h, *gh;
    unsigned char *out, *gx, *ggate;
    int64_t ld_x, ld_gate, ld_h, ld_gh, ld_out, ld_gx, ld_ggate;      // bytes from row to row
    const float *first;                 // [B, C] values before the first row in scan order (NULL: zeros)
    float* last;                        // [B, C] values behind the last
    const float* h0;                    // backward: the states before the sequences' first rows
    const uint64_t* begin;
    const int32_t *rank, *id;
    // what workgroups tell each other, where there is more than one tile: kNothing until it is written
    uint64_t* tile_runs;                // [slabs][tiles][64] (A, H) of every tile
    uint64_t* group_runs;               // [slabs][groups][64] (A, H) of every group, then the value behind it as (-1, H)
    uint32_t* ticket;
};

struct Run { float A, H; };
__device__ __forceinline__ Run then(const Run& l, const Run& r) {
    Run o;
    o.H = r.A < 0.f ? r.H : r.A * l.H + r.H;
    o.A = r.A < 0.f || l.A < 0.f ? -1.f : l.A * r.A;
    return o;
}
// the value behind a run
__device__ __forceinline__ float through(const Run& r, float v) { return r.A < 0.f ? r.H : r.A * v + r.H; }

// A lane's rows: u0 .. u0 + n - 1 in scan order, rows lo .. lo + n - 1 of the tensors (in turn or against it).
struct LaneRows {
    int64_t lo;
    uint32_t begin, stop;               // bit i: the sequence of row u0 + i begins / ends there, in scan order
    int n;                              // rows that exist
};

template <bool UP, int R>
__device__ __forceinline__ LaneRows lane_rows(const ScanArgs& a, int64_t u0) {
    LaneRows r;
    r.n = (int)max((int64_t)0, min((int64_t)R, a.rows - u0));
    r.begin = r.stop = 0;
    r.lo = 0;
    if (r.n == 0) return r;
    r.lo = UP ? u0 : a.rows - u0 - r.n;
    const uint64_t w0 = a.begin[r.lo >> 6], w1 = a.begin[(r.lo >> 6) + 1];
    const int sh = (int)(r.lo & 63);
    const uint32_t bits = (uint32_t)(sh ? (w0 >> sh) | (w1 << (64 - sh)) : w0) & ((2u << r.n) - 1);      // rows lo .. lo + n
    const uint32_t starts = bits & ((1u << r.n) - 1), ends = bits >> 1;
    if (UP) { r.begin = starts; r.stop = ends; }
    else {                              // bit i is row lo + n - 1 - i
        r.begin = __brev(ends) >> (32 - r.n);
        r.stop = __brev(starts) >> (32 - r.n);
    }
    return r;
}

// does a sequence begin, in scan order, at row u
template <bool UP>
__device__ __forceinline__ bool begins_at(const ScanArgs& a, int64_t u) {
    const int64_t r = UP ? u : a.rows - u;         // the row's own bit, or that of the row behind it
    return a.begin[r >> 6] >> (r & 63) & 1;
}

__device__ __forceinline__ int sequence_of(const ScanArgs& a, int64_t row) {
    const uint64_t w = a.begin[row >> 6] & ((2ull << (row & 63)) - 1);
    return a.id[a.rank[row >> 6] + __popcll(w) - 1];
}

// eight channels of a row of a [B, C] table, zeros without one
template <int KIND>
__device__ __forceinline__ void load_states(const float* t, int seq, int col, int C, float (&v)[kPiece]) {
#pragma unroll
    for (int e = 0; e < kPiece; ++e) v[e] = 0.f;
    if (t) unpack<FX_F32>(load_piece<FX_F32, KIND>(reinterpret_cast<const unsigned char*>(t + (int64_t)seq * C), col, C), v);
}
template <int KIND>
__device__ __forceinline__ void store_states(float* t, int seq, int col, int C, const float (&v)[kPiece]) {
    store_piece<FX_F32, KIND>(reinterpret_cast<unsigned char*>(t + (int64_t)seq * C), col, C, pack<FX_F32>(v));
}

// The scan over the lanes' runs within a workgroup.  Runs of all groups of lanes in LDS; a thread takes one channel of
// eight groups and leaves in their place what stands before each within the eight; the eights' own runs lie in seg.
struct ScanLds {
    float A[kScanThreads * kPiece], H[kScanThreads * kPiece];      // [group of lanes][channel of the slab]
    float seg_A[kScanThreads], seg_H[kScanThreads];                // [eight groups][channel]
    float before[kScanThreads];                                    // value before every eight groups
    uint64_t seen[kGroupTiles][64];                                // what a look back found, [tile or group][channel]
    int ticket;
};

__device__ __forceinline__ void put_run(ScanLds& s, int t, const float (&A)[kPiece], const float (&H)[kPiece]) {
#pragma unroll
    for (int i = 0; i < kPiece; i += 4) {
        *reinterpret_cast<f32x4*>(&s.A[t * kPiece + i]) = f32x4{A[i], A[i + 1], A[i + 2], A[i + 3]};
        *reinterpret_cast<f32x4*>(&s.H[t * kPiece + i]) = f32x4{H[i], H[i + 1], H[i + 2], H[i + 3]};
    }
}

__device__ __forceinline__ void scan_eights(ScanLds& s, int width_log2) {
    const int t = threadIdx.x, width = 1 << width_log2, c = t & (width - 1), seg = t >> width_log2;
    Run run{1.f, 0.f};
#pragma unroll
    for (int i = 0; i < 8; ++i) {
        const int at = ((seg * 8 + i) << width_log2) + c;
        const Run mine{s.A[at], s.H[at]};
        s.A[at] = run.A;
        s.H[at] = run.H;
        run = then(run, mine);
    }
    s.seg_A[t] = run.A;
    s.seg_H[t] = run.H;
}

// ---- what workgroups tell each other
// One 64-bit word a channel holds both numbers of a run, so a reader has all or nothing of it and nothing needs to be
// ordered around it.  No number has the bits of kNothing: a NaN is written with the same bits always.
constexpr uint32_t kNothing = 0xFFFFFFFFu;
constexpr int kMostPolls = 1 << 22;     // seconds; a wait ends long before, see the tickets

__device__ __forceinline__ uint32_t plain_bits(float v) { return v == v ? __float_as_uint(v) : 0x7FC00000u; }
__device__ __forceinline__ void publish(uint64_t* at, const Run& r) {
    __hip_atomic_store(at, (uint64_t)plain_bits(r.A) << 32 | plain_bits(r.H), __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
}
__device__ __forceinline__ uint64_t look(const uint64_t* at) { return __hip_atomic_load(at, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT); }
__device__ __forceinline__ bool is_there(uint64_t w) { return (uint32_t)(w >> 32) != kNothing; }
__device__ __forceinline__ Run run_in(uint64_t w) { return Run{__uint_as_float((uint32_t)(w >> 32)), __uint_as_float((uint32_t)w)}; }

// Words `from`, `from` + step, ... of `n` (64 words from one to the next) for this thread's channel into s.seen, waiting
// for those that are not there yet.  All threads of the workgroup take part; ends with a barrier.  A word that does not
// come within the bound counts as NaN.
__device__ __forceinline__ void gather_runs(ScanLds& s, const uint64_t* words, int64_t step, int n, int width_log2) {
    const int c = threadIdx.x & ((1 << width_log2) - 1), first = threadIdx.x >> width_log2, stride = blockDim.x >> width_log2;
    for (int i0 = first; i0 < n; i0 += 4 * stride) {
        uint64_t w[4];
#pragma unroll
        for (int k = 0; k < 4; ++k) {
            const int i = i0 + k * stride;
            w[k] = i < n ? look(words + step * i + c) : 0;
        }
        for (int polls = 0; polls < kMostPolls; ++polls) {
            bool all = true;
#pragma unroll
            for (int k = 0; k < 4; ++k) all = all && is_there(w[k]);
            if (all) break;
            __builtin_amdgcn_s_sleep(1);
#pragma unroll
            for (int k = 0; k < 4; ++k)
                if (!is_there(w[k])) w[k] = look(words + step * (i0 + k * stride) + c);
        }
#pragma unroll
        for (int k = 0; k < 4; ++k) {
            const int i = i0 + k * stride;
            if (i < n) s.seen[i][c] = is_there(w[k]) ? w[k] : (uint64_t)0xBF800000u << 32 | 0x7FC00000u;
        }
    }
    __syncthreads();
}

// The value before the tile for channel threadIdx.x (threads below `width`; others get 0), having published the tile's
// run and, from the last tile of a group, the group's.
__device__ __forceinline__ float look_back(const ScanArgs& a, ScanLds& s, int slab, int tile, bool begins, const Run& mine, int width_log2) {
    const int t = threadIdx.x, width = 1 << width_log2, group = tile / kGroupTiles, in_group = tile % kGroupTiles;
    const bool closes = in_group == kGroupTiles - 1;
    uint64_t* tiles = a.tile_runs + ((int64_t)slab * a.tiles + (tile - in_group)) * 64;
    uint64_t* groups = a.group_runs + (int64_t)slab * a.groups * 64;
    if (t < width && !closes) publish(tiles + in_group * 64 + t, mine);
    Run run{1.f, 0.f};                              // of the group's tiles before this one
    if (in_group && (!begins || closes)) {
        gather_runs(s, tiles, 64, in_group, width_log2);
        if (t < width)
#pragma unroll 2
            for (int i = 0; i < in_group; ++i) run = then(run, run_in(s.seen[i][t]));
    }
    if (closes && t < width) publish(groups + group * 64 + t, then(run, mine));
    float v = 0.f;
    if (!begins) {
        // backwards over the groups until the value behind one of them is known for every channel
        Run back{1.f, 0.f};
        for (int end = group; end > 0; end -= kLookWindow) {
            const int n = min(end, kLookWindow);
            __syncthreads();                        // the words of the turn before have been read
            gather_runs(s, groups + (int64_t)(end - 1) * 64, -64, n, width_log2);
            if (t < width)
#pragma unroll 2
                for (int i = 0; i < n && back.A >= 0.f; ++i) back = then(run_in(s.seen[i][t]), back);
            if (!__syncthreads_or(t < width && !(back.A < 0.f))) break;
        }
        if (t < width) v = through(run, back.H);
    }
    if (closes && t < width) publish(groups + group * 64 + t, Run{-1.f, through(mine, v)});
    return v;
}

__global__ void __launch_bounds__(256) k_scan_clear(uint64_t* words, int64_t n, uint32_t* ticket) {
    for (int64_t i = (int64_t)blockIdx.x * 256 + threadIdx.x; i < n; i += (int64_t)gridDim.x * 256) words[i] = ~0ull;
    if (blockIdx.x == 0 && threadIdx.x == 0) *ticket = 0;
}

// The smaller of a row's two sigmoids, its sign saying which: what a lane keeps of a gate between the two passes over
// its rows.
__device__ __forceinline__ float keep_gate(float z, float& f, float& g) {
    sigmoids(z, f, g);
    return z > 0.f ? g : -f;
}
__device__ __forceinline__ void kept_gate(float k, float& f, float& g) {
    const float small = fabsf(k), large = 1.f - small;
    const bool up = (int)__float_as_uint(k) >= 0;       // the sign of a zero counts too
    f = up ? large : small;
    g = up ? small : large;
}

template <int DT, int KIND, bool UP, bool BWD>
__global__ void __launch_bounds__(kScanThreads, BWD ? 2 : 4)
k_scan(ScanArgs a) {
    constexpr int R = ScanRows<DT, BWD>::n;
    __shared__ ScanLds s;
    const int t = threadIdx.x, lanes = 1 << a.lanes_log2, width_log2 = a.lanes_log2 + 3, width = 1 << width_log2;
    const int group = t >> a.lanes_log2;
    int turn = blockIdx.x;
    if (a.tile_runs) {
        if (t == 0) s.ticket = (int)atomicAdd(a.ticket, 1u);
        __syncthreads();
        turn = s.ticket;
    }
    const int slab = turn % a.slabs, tile = turn / a.slabs;
    const int col = slab * 64 + (t & (lanes - 1)) * kPiece;
    const int64_t tile0 = (int64_t)tile * (blockDim.x >> a.lanes_log2) * R, u0 = tile0 + group * R;
    const LaneRows lr = lane_rows<UP, R>(a, u0);
    constexpr int64_t step = UP ? 1 : -1;
    const int64_t r0 = UP ? lr.lo : lr.lo + max(lr.n, 1) - 1;        // the lane's first row in scan order
    Piece<DT> in[R], px[BWD ? R : 1], pp[BWD ? R : 1];
    float kept[R][kPiece];
    {
        const unsigned char *pg = a.gate + r0 * a.ld_gate, *pi = (BWD ? a.gh : a.x) + r0 * (BWD ? a.ld_gh : a.ld_x);
        Piece<DT> gate[R];
#pragma unroll
        for (int i = 0; i < R; ++i) {       // rows that do not exist: the last that does once more
            gate[i] = load_piece<DT, KIND>(pg, col, a.C);
            in[i] = load_piece<DT, KIND>(pi, col, a.C);
            if (i + 1 < lr.n) { pg += step * a.ld_gate; pi += step * (BWD ? a.ld_gh : a.ld_x); }
        }
#pragma unroll
        for (int i = 0; i < R; ++i) {
            float z[kPiece];
            unpack<DT>(gate[i], z);
#pragma unroll
            for (int e = 0; e < kPiece; ++e) kept[i][e] = z[e];
        }
    }
    {
        // the run of this lane's rows
        float A[kPiece], H[kPiece];
#pragma unroll
        for (int e = 0; e < kPiece; ++e) { A[e] = 1.f; H[e] = 0.f; }
#pragma unroll
        for (int i = 0; i < R; ++i) {
            if (lr.begin >> i & 1) load_states<KIND>(a.first, sequence_of(a, r0 + step * i), col, a.C, H);
            float v[kPiece];
            unpack<DT>(in[i], v);
#pragma unroll
            for (int e = 0; e < kPiece; ++e) {
                float f, g;
                kept[i][e] = keep_gate(kept[i][e], f, g);
                asm volatile("" : "+v"(kept[i][e]));        // one number is kept: f and g of all rows do not fit the registers
                H[e] = BWD ? f * (v[e] + H[e]) : f * H[e] + g * v[e];
                A[e] *= f;
            }
            __builtin_amdgcn_sched_barrier(0);      // a row after the other: the gates of all rows at once do not fit the registers
        }
        if (lr.begin) {
#pragma unroll
            for (int e = 0; e < kPiece; ++e) A[e] = -1.f;
        }
        put_run(s, t, A, H);
    }
    if (BWD) {
        // The rows run against the sequence: the state before a row lies at the row that comes next here.
        const unsigned char *p = a.x + r0 * a.ld_x, *q = a.h + r0 * a.ld_h;
        const bool more = UP ? r0 + lr.n < a.rows : r0 - lr.n >= 0;        // a row behind the lane's last
#pragma unroll
        for (int i = 0; i < R; ++i) {
            px[i] = load_piece<DT, KIND>(p, col, a.C);
            if (i + 1 < lr.n) p += step * a.ld_x;
            if (i + 1 < lr.n || (i + 1 == lr.n && more)) q += step * a.ld_h;
            pp[i] = load_piece<DT, KIND>(q, col, a.C);
        }
    }
    __syncthreads();
    scan_eights(s, width_log2);
    __syncthreads();
    {
        Run run{1.f, 0.f};
        if (t < width)
#pragma unroll 2
            for (int i = t; i < (int)blockDim.x; i += width) run = then(run, Run{s.seg_A[i], s.seg_H[i]});
        float v = a.tile_runs ? look_back(a, s, slab, tile, begins_at<UP>(a, tile0), run, width_log2) : 0.f;
        if (t < width)
#pragma unroll 2
            for (int i = t; i < (int)blockDim.x; i += width) { s.before[i] = v; v = through(Run{s.seg_A[i], s.seg_H[i]}, v); }
    }
    __syncthreads();
    float v[kPiece];
#pragma unroll
    for (int e = 0; e < kPiece; ++e)
        v[e] = through(Run{s.A[t * kPiece + e], s.H[t * kPiece + e]}, s.before[((group >> 3) << width_log2) + (t & (lanes - 1)) * kPiece + e]);
#pragma unroll
    for (int i = 0; i < R; ++i) {
        if (i >= lr.n) break;
        const int64_t row = r0 + step * i;
        const bool begins = lr.begin >> i & 1, ends = lr.stop >> i & 1;
        if (begins) load_states<KIND>(a.first, sequence_of(a, row), col, a.C, v);
        float w[kPiece];
        unpack<DT>(in[i], w);
        if (!BWD) {
#pragma unroll
            for (int e = 0; e < kPiece; ++e) {
                float f, g;
                kept_gate(kept[i][e], f, g);
                v[e] = f * v[e] + g * w[e];
            }
            store_piece<DT, KIND>(a.out + row * a.ld_out, col, a.C, pack<DT>(v));
        } else {
            float x[kPiece], p[kPiece], gx[kPiece], gz[kPiece];
            unpack<DT>(px[i], x);
            unpack<DT>(pp[i], p);
            if (ends) load_states<KIND>(a.h0, sequence_of(a, row), col, a.C, p);
#pragma unroll
            for (int e = 0; e < kPiece; ++e) {
                float f, g;
                kept_gate(kept[i][e], f, g);
                const float lam = w[e] + v[e];
                gx[e] = g * lam;
                gz[e] = lam * (p[e] - x[e]) * (f * g);
                v[e] = f * lam;
            }
            store_piece<DT, KIND>(a.gx + row * a.ld_gx, col, a.C, pack<DT>(gx));
            store_piece<DT, KIND>(a.ggate + row * a.ld_ggate, col, a.C, pack<DT>(gz));
        }
        if (ends && a.last) store_states<KIND>(a.last, sequence_of(a, row), col, a.C, v);
        __builtin_amdgcn_sched_barrier(0);
    }
}

// states of sequences without rows pass through
__global__ void k_scan_empty(const int32_t* __restrict__ empty, int n, int C, const float* __restrict__ first, float* __restrict__ last) {
    const int64_t i = (int64_t)blockIdx.x * blockDim.x + threadIdx.x;
    if (i >= (int64_t)n * C) return;
    const int64_t at = (int64_t)empty[i / C] * C + i % C;
    last[at] = first ? first[at] : 0.f;
}

// One row of each of many running sequences: h = f state + (1 - f) x, the state kept in fp32.
template <int DT, int KIND>
__global__ void __launch_bounds__(256)
k_scan_step(int64_t rows, int C, int pieces, const unsigned char* x, int64_t ld_x, const unsigned char* gate, int64_t ld_gate, const float* state,
            float* new_state, unsigned char* out, int64_t ld_out) {
    const int64_t i = (int64_t)blockIdx.x * blockDim.x + threadIdx.x, row = i / pieces;
    if (row >= rows) return;
    const int col = (int)(i - row * pieces) * kPiece;
    float z[kPiece], v[kPiece], h[kPiece];
    const Piece<DT> pz = load_piece<DT, KIND>(gate + row * ld_gate, col, C), pv = load_piece<DT, KIND>(x + row * ld_x, col, C);
#pragma unroll
    for (int e = 0; e < kPiece; ++e) h[e] = col + e < C ? state[row * C + col + e] : 0.f;
    unpack<DT>(pz, z);
    unpack<DT>(pv, v);
#pragma unroll
    for (int e = 0; e < kPiece; ++e) {
        float f, g;
        sigmoids(z[e], f, g);
        h[e] = f * h[e] + g * v[e];
        if (col + e < C) new_state[row * C + col + e] = h[e];
    }
    store_piece<DT, KIND>(out + row * ld_out, col, C, pack<DT>(h));
}

// ---------------------------------------------------------------------------------- host
static int esize(fx_dtype dt) { return dt == FX_F32 ? 4 : 2; }

static fx_status check_rows_of(const char* who, const char* name, const void* p, int64_t ld, int64_t rows, int32_t C, fx_dtype dt) {
    if (rows == 0) return FX_OK;
    if (!p || (uintptr_t)p % esize(dt) || ld < C) {
        set_error("%s: %s is null, not aligned to its elements or has rows closer than C", who, name);
        return FX_EINVAL;
    }
    return FX_OK;
}

static fx_status check_scan(const char* who, const fx_sequences* q, int32_t C, fx_dtype dt) {
    if (!q || C < 1 || (dt != FX_F32 && dt != FX_F16 && dt != FX_BF16)) {
        set_error("%s: null sequences, no channels or unknown dtype", who);
        return FX_EINVAL;
    }
    return FX_OK;
}

static void scan_args(ScanArgs* a, const fx_sequences* q, int32_t C) {
    *a = ScanArgs{};
    a->rows = q->rows;
    a->C = C;
    const int pieces = std::min(8, (C + kPiece - 1) / kPiece);
    while ((1 << a->lanes_log2) < pieces) ++a->lanes_log2;
    a->slabs = (C + 63) / 64;
    a->begin = q->d_begin;
    a->rank = q->d_rank;
    a->id = q->d_id;
}

template <int DT, int KIND, bool UP, bool BWD>
static fx_status launch_scan(ScanArgs& a, hipStream_t st) {
    // As many threads as leave every compute unit a tile, from a wave on.
    int threads = kScanThreads;
    int64_t rows_a_tile, tiles;
    for (;; threads /= 2) {
        rows_a_tile = (int64_t)(threads >> a.lanes_log2) * ScanRows<DT, BWD>::n;
        tiles = (a.rows + rows_a_tile - 1) / rows_a_tile;
        if (threads == 64 || tiles * a.slabs >= 2 * compute_units()) break;
    }
    if (tiles * a.slabs > 0x3FFFFFFF) { set_error("gated scan: too many tiles for one launch"); return FX_ERANGE; }
    a.tiles = (int)tiles;
    a.groups = (int)((tiles + kGroupTiles - 1) / kGroupTiles);
    void* work = nullptr;
    unsigned nb = (unsigned)a.slabs;
    if (tiles > 1) {
        const int64_t words = (int64_t)a.slabs * 64 * (a.tiles + a.groups);
        FX_TRY(dev_alloc(&work, (size_t)words * 8 + 256, st));
        a.tile_runs = (uint64_t*)work;
        a.group_runs = a.tile_runs + (int64_t)a.slabs * 64 * a.tiles;
        a.ticket = (uint32_t*)(a.tile_runs + words);
        k_scan_clear<<<(unsigned)std::min<int64_t>((words + 255) / 256, 1024), 256, 0, st>>>(a.tile_runs, words, a.ticket);
        nb = (unsigned)(tiles * a.slabs);
    }
    k_scan<DT, KIND, UP, BWD><<<nb, threads, 0, st>>>(a);
    const hipError_t e = hipGetLastError();
    dev_free(work, st);
    if (e != hipSuccess) { set_error("launch of the gated scan failed: %s", hipGetErrorString(e)); return FX_EDEVICE; }
    return FX_OK;
}

template <int DT, bool BWD>
static fx_status launch_scan_kind(ScanArgs& a, bool up, hipStream_t st) {
    const int kind = a.C < kPiece ? kRowsNarrow : a.C % kPiece ? kRowsRagged : kRowsWhole;
#define FX_SCAN(KIND) return up ? launch_scan<DT, KIND, true, BWD>(a, st) : launch_scan<DT, KIND, false, BWD>(a, st)
    if (kind == kRowsWhole) FX_SCAN(kRowsWhole);
    if (kind == kRowsRagged) FX_SCAN(kRowsRagged);
    FX_SCAN(kRowsNarrow);
#undef FX_SCAN
}

template <bool BWD>
static fx_status run_scan(const fx_sequences* q, ScanArgs& a, fx_dtype dt, bool up, hipStream_t st) {
    ProfScope ps(BWD ? kProfScanBwd : kProfScanFwd, st);
    if (a.last && q->n_empty) {
        k_scan_empty<<<(unsigned)(((int64_t)q->n_empty * a.C + 255) / 256), 256, 0, st>>>(q->d_empty, q->n_empty, a.C, a.first, a.last);
        FX_HIP_TRY(hipGetLastError());
    }
    if (a.rows == 0) return FX_OK;
    if (dt == FX_F32) return launch_scan_kind<FX_F32, BWD>(a, up, st);
    if (dt == FX_F16) return launch_scan_kind<FX_F16, BWD>(a, up, st);
    return launch_scan_kind<FX_BF16, BWD>(a, up, st);
}

}  // namespace fx

using namespace fx;

extern "C" fx_status fx_build_sequences(const int64_t* h_joffsets, int32_t B, int64_t rows, void* stream, fx_sequences** out) {
    const char* who = "fx_build_sequences";
    if (!out || B < 0 || rows < 0 || (B > 0 && !h_joffsets)) { set_error("%s: null pointer or negative size", who); return FX_EINVAL; }
    int64_t at = 0;
    for (int32_t b = 0; b < B; ++b) {
        if (h_joffsets[2 * b] != at || h_joffsets[2 * b + 1] < at) {
            set_error("%s: sequence %d does not begin where the one before it ends", who, b);
            return FX_EINVAL;
        }
        at = h_joffsets[2 * b + 1];
    }
    if (at != rows) { set_error("%s: the sequences do not end at the last row", who); return FX_EINVAL; }
    if (rows > 0x7FFFFFFFll) { set_error("%s: more than 2^31-1 rows", who); return FX_ERANGE; }
    hipStream_t st = (hipStream_t)stream;
    const int64_t words = rows / 64 + 2;
    const size_t bytes = (size_t)words * 12 + (size_t)B * 8;
    void* staging = nullptr;
    FX_HIP_TRY(hipStreamSynchronize(st));           // an upload before this one may still read the staging area
    FX_TRY(host_staging(&staging, bytes, 1));
    uint64_t* begin = (uint64_t*)staging;
    int32_t* rank = (int32_t*)(begin + words);
    int32_t* ids = rank + words;                    // the sequences with rows, then those without
    for (int64_t w = 0; w < words; ++w) begin[w] = 0;
    int32_t some = 0, empty = 0;
    for (int32_t b = 0; b < B; ++b) {
        const int64_t r = h_joffsets[2 * b];
        if (h_joffsets[2 * b + 1] == r) { ids[B - 1 - empty++] = b; continue; }
        begin[r >> 6] |= 1ull << (r & 63);
        ids[some++] = b;
    }
    begin[rows >> 6] |= 1ull << (rows & 63);
    for (int64_t w = 0, n = 0; w < words; ++w) { rank[w] = (int32_t)n; n += __builtin_popcountll(begin[w]); }
    fx_sequences* q = new (std::nothrow) fx_sequences;
    if (!q) { set_error("%s: out of host memory", who); return FX_ENOMEM; }
    const fx_status s = dev_alloc(&q->buf, bytes, st);
    if (s != FX_OK) { delete q; return s; }
    const hipError_t e = hipMemcpyAsync(q->buf, staging, bytes, hipMemcpyHostToDevice, st);
    if (e != hipSuccess || hipStreamSynchronize(st) != hipSuccess) {
        dev_free(q->buf, st);
        delete q;
        set_error("%s: upload failed: %s", who, hipGetErrorString(e));
        return FX_EDEVICE;
    }
    q->rows = rows;
    q->B = B;
    q->n_empty = empty;
    q->stream = st;
    q->d_begin = (const uint64_t*)q->buf;
    q->d_rank = (const int32_t*)(q->d_begin + words);
    q->d_id = q->d_rank + words;
    q->d_empty = q->d_id + some;
    *out = q;
    return FX_OK;
}

extern "C" void fx_sequences_destroy(fx_sequences* q) {
    if (!q) return;
    dev_free(q->buf, q->stream);
    delete q;
}

extern "C" fx_status fx_gated_scan_fwd(const fx_sequences* q, const void* d_x, int64_t ld_x, const void* d_gate, int64_t ld_gate, fx_dtype dt,
                                       int32_t C, int32_t reverse, const float* d_h0, void* d_h, int64_t ld_h, float* d_last, void* stream) {
    const char* who = "fx_gated_scan_fwd";
    FX_TRY(check_scan(who, q, C, dt));
    FX_TRY(check_rows_of(who, "d_x", d_x, ld_x, q->rows, C, dt));
    FX_TRY(check_rows_of(who, "d_gate", d_gate, ld_gate, q->rows, C, dt));
    FX_TRY(check_rows_of(who, "d_h", d_h, ld_h, q->rows, C, dt));
    if (q->rows > 0 && (d_h == d_x || d_h == d_gate)) { set_error("%s: d_h must not be an input", who); return FX_EINVAL; }
    ScanArgs a;
    scan_args(&a, q, C);
    const int es = esize(dt);
    a.x = (const unsigned char*)d_x; a.ld_x = ld_x * es;
    a.gate = (const unsigned char*)d_gate; a.ld_gate = ld_gate * es;
    a.out = (unsigned char*)d_h; a.ld_out = ld_h * es;
    a.first = d_h0;
    a.last = d_last;
    return run_scan<false>(q, a, dt, !reverse, (hipStream_t)stream);
}

extern "C" fx_status fx_gated_scan_bwd(const fx_sequences* q, const void* d_x, int64_t ld_x, const void* d_gate, int64_t ld_gate, const void* d_h,
                                       int64_t ld_h, const void* d_gh, int64_t ld_gh, fx_dtype dt, int32_t C, int32_t reverse, const float* d_h0,
                                       const float* d_glast, void* d_gx, int64_t ld_gx, void* d_ggate, int64_t ld_ggate, float* d_gh0,
                                       void* stream) {
    const char* who = "fx_gated_scan_bwd";
    FX_TRY(check_scan(who, q, C, dt));
    FX_TRY(check_rows_of(who, "d_x", d_x, ld_x, q->rows, C, dt));
    FX_TRY(check_rows_of(who, "d_gate", d_gate, ld_gate, q->rows, C, dt));
    FX_TRY(check_rows_of(who, "d_h", d_h, ld_h, q->rows, C, dt));
    FX_TRY(check_rows_of(who, "d_gh", d_gh, ld_gh, q->rows, C, dt));
    FX_TRY(check_rows_of(who, "d_gx", d_gx, ld_gx, q->rows, C, dt));
    FX_TRY(check_rows_of(who, "d_ggate", d_ggate, ld_ggate, q->rows, C, dt));
    const void* in[4] = {d_x, d_gate, d_h, d_gh};
    for (const void* p : in)
        if (q->rows > 0 && (p == d_gx || p == d_ggate)) { set_error("%s: a gradient must not lie where an input lies", who); return FX_EINVAL; }
    ScanArgs a;
    scan_args(&a, q, C);
    const int es = esize(dt);
    a.x = (const unsigned char*)d_x; a.ld_x = ld_x * es;
    a.gate = (const unsigned char*)d_gate; a.ld_gate = ld_gate * es;
    a.h = (const unsigned char*)d_h; a.ld_h = ld_h * es;
    a.gh = (const unsigned char*)d_gh; a.ld_gh = ld_gh * es;
    a.gx = (unsigned char*)d_gx; a.ld_gx = ld_gx * es;
    a.ggate = (unsigned char*)d_ggate; a.ld_ggate = ld_ggate * es;
    a.h0 = d_h0;
    a.first = d_glast;
    a.last = d_gh0;
    return run_scan<true>(q, a, dt, reverse != 0, (hipStream_t)stream);
}

extern "C" fx_status fx_gated_scan_step(const void* d_x, int64_t ld_x, const void* d_gate, int64_t ld_gate, fx_dtype dt, int64_t rows, int32_t C,
                                        const float* d_state, float* d_new_state, void* d_h, int64_t ld_h, void* stream) {
    const char* who = "fx_gated_scan_step";
    if (rows < 0 || C < 1 || (dt != FX_F32 && dt != FX_F16 && dt != FX_BF16) || (rows > 0 && (!d_state || !d_new_state))) {
        set_error("%s: negative rows, no channels, unknown dtype or null state", who);
        return FX_EINVAL;
    }
    FX_TRY(check_rows_of(who, "d_x", d_x, ld_x, rows, C, dt));
    FX_TRY(check_rows_of(who, "d_gate", d_gate, ld_gate, rows, C, dt));
    FX_TRY(check_rows_of(who, "d_h", d_h, ld_h, rows, C, dt));
    if (rows == 0) return FX_OK;
    const int pieces = (C + kPiece - 1) / kPiece, es = esize(dt);
    const int64_t blocks = (rows * pieces + 255) / 256;
    if (blocks > 0x7FFFFFFF) { set_error("%s: too many rows for one launch", who); return FX_ERANGE; }
    hipStream_t st = (hipStream_t)stream;
    ProfScope ps(kProfScanFwd, st);
    const int kind = C < kPiece ? kRowsNarrow : C % kPiece ? kRowsRagged : kRowsWhole;
#define FX_STEP(DT, KIND) k_scan_step<DT, KIND><<<(unsigned)blocks, 256, 0, st>>>(rows, C, pieces, (const unsigned char*)d_x, ld_x * es, \
        (const unsigned char*)d_gate, ld_gate * es, d_state, d_new_state, (unsigned char*)d_h, ld_h * es)
#define FX_STEP_KIND(DT) do { if (kind == kRowsWhole) FX_STEP(DT, kRowsWhole); else if (kind == kRowsRagged) FX_STEP(DT, kRowsRagged); \
                              else FX_STEP(DT, kRowsNarrow); } while (0)
    if (dt == FX_F32) FX_STEP_KIND(FX_F32);
    else if (dt == FX_F16) FX_STEP_KIND(FX_F16);
    else FX_STEP_KIND(FX_BF16);
#undef FX_STEP_KIND
#undef FX_STEP
    FX_HIP_TRY(hipGetLastError());
    return FX_OK;
}
