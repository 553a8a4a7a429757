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
// One pass over the data.  A tile is some hundred rows of up to 64 channels: 16 lanes hold a row (4 channels each), and
// every lane takes a few rows that follow each other, in registers from the load to the store.  A wave scans its lanes'
// runs by shuffles, the waves' runs meet in LDS; the workgroup publishes the tile's (A, H), looks back over the tiles
// before it for the value that its first row starts from, and finishes its rows: the decoupled look back of Merrill and
// Garland ("Single-pass parallel prefix scan with decoupled look-back", 2016), here over groups of tiles and in one
// order of additions.  Tiles are taken in scan order by ticket, so whatever a workgroup waits for belongs to a workgroup that already runs, and that one waits for earlier
// tiles only.
//
// Measured (986,880 x 64 bf16, one sequence: 379 MB, 74 us at a copy's rate): 127 us, 2.98 TB/s; in three launches (the
// tiles' runs, what stands before each, the rows: 632 MB) 168 us.  Where every tile begins a sequence of its own and
// nobody waits, 93 us (gradients 157): the look back costs the rest.  What bounds it are a workgroup's phases one after the other (ticket,
// rows, run, look back, store: 17 us a tile) with two workgroups a compute unit, all that its registers hold; vector
// instructions fill 40 % of the time, the tickets (11.6 ns each at one address) take 45 us of all in turn.  Gradients of
// 1,068,658 x 64 f16 in four sequences (821 MB, 161 us): 207 us, 4.0 TB/s.
#include "rows.h"

#include <new>

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
constexpr int kGroupTiles = 16;         // tiles whose joint (A, H) is published as one (8: 4 % slower at 986,880 x 64 bf16; 32, 64: +- 3 %)
constexpr int kLookWindow = 16;         // groups looked back over
constexpr int kQuad = 4;                // channels of a lane

// Rows of a lane, such that the kernel has 128 registers at most: two workgroups of 512 then share a compute unit.
// Forward, 8 rows of 4 channels hold 64 numbers between the passes (16 rows: 197 registers; the gates and inputs held as
// loaded and worked on twice, 16 rows: 136 us where 8 as they are take 133; 4 rows: twice the tiles to wait for).  Backward,
// gate and gradient of 8 rows of a 16-bit type hold 48; state and x are asked for behind the look back (asked for before
// it they hold 32 more: 158 registers, 212 us at 986,880 x 64 bf16 for 193).
template <int DT, bool BWD> struct ScanRows { static constexpr int n = 8 / (BWD && DT == FX_F32 ? 2 : 1); };

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
    const int32_t *rank, *id, *empty;
    int32_t n_empty;
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
    uint32_t starts;                    // bit j: a sequence begins at row lo + j, in the tensors' order
    int rank;                           // which of the sequences with rows row lo belongs to
    int n;                              // rows that exist
};

template <bool UP, int R>
__device__ __forceinline__ LaneRows lane_rows(const ScanArgs& a, int64_t u0) {
    LaneRows r;
    r.n = (int)max((int64_t)0, min((int64_t)R, a.rows - u0));
    r.lo = UP ? min(u0, a.rows - 1) : a.rows - min(u0, a.rows - 1) - max(r.n, 1);
    const int64_t word = r.lo >> 6;
    const uint64_t w0 = a.begin[word], w1 = a.begin[word + 1];
    const int sh = (int)(r.lo & 63);
    const uint32_t bits = (uint32_t)(sh ? (w0 >> sh) | (w1 << (64 - sh)) : w0) & ((2u << r.n) - 1);      // rows lo .. lo + n
    r.rank = a.rank[word] + __popcll(w0 & ((2ull << sh) - 1)) - 1;
    r.starts = bits & ((1u << r.n) - 1);
    const uint32_t ends = bits >> 1;
    if (UP || r.n == 0) { r.begin = r.starts; r.stop = ends; }
    else {                              // bit i is row lo + n - 1 - i
        r.begin = __brev(ends) >> (32 - r.n);
        r.stop = __brev(r.starts) >> (32 - r.n);
    }
    return r;
}

// number of the sequence that the lane's row i (in scan order) belongs to
template <bool UP>
__device__ __forceinline__ int sequence_of(const ScanArgs& a, const LaneRows& r, int i) {
    const int j = UP ? i : r.n - 1 - i;
    return a.id[r.rank + __popc(r.starts & ((2u << j) - 1) & ~1u)];
}

// The tile's rows: `count` rows from row `lowest` of the tensors on, the lane's own from the `lane`-th in scan order on.
// Addresses are a base that is the same in all lanes plus 32 bits of a lane; in a FULL tile the row's number moves the
// base.  A row that does not exist is read as the tile's last.
template <bool UP, int R, bool FULL>
struct TileRows {
    int64_t lowest;
    int count, lane;
    template <typename T>
    __device__ __forceinline__ T* base(T* tensor, int64_t ld, int i) const {
        return tensor + (lowest + (!FULL ? 0 : UP ? i : R - 1 - i)) * ld;
    }
    __device__ __forceinline__ uint32_t offset(int64_t ld, int i) const {
        if (FULL) return (uint32_t)(UP ? lane : count - R - lane) * (uint32_t)ld;
        const int k = min(lane + i, count - 1);
        return (uint32_t)(UP ? k : count - 1 - k) * (uint32_t)ld;
    }
};

// does a sequence begin, in scan order, at row u
template <bool UP>
__device__ __forceinline__ bool begins_at(const ScanArgs& a, int64_t u) {
    const int64_t r = UP ? u : a.rows - u;         // the row's own bit, or that of the row behind it
    return a.begin[r >> 6] >> (r & 63) & 1;
}

// four channels of a row of a [B, C] table, zeros without one
template <int KIND>
__device__ __forceinline__ void load_states(const float* t, int seq, int col, int C, float (&v)[kQuad]) {
#pragma unroll
    for (int e = 0; e < kQuad; ++e) v[e] = 0.f;
    if (t) unpack<FX_F32>(load_piece<FX_F32, KIND, kQuad>(reinterpret_cast<const unsigned char*>(t + (int64_t)seq * C), 0, col, C), v);
}
template <int KIND>
__device__ __forceinline__ void store_states(float* t, int seq, int col, int C, const float (&v)[kQuad]) {
    store_piece<FX_F32, KIND>(reinterpret_cast<unsigned char*>(t + (int64_t)seq * C), 0, col, C, pack<FX_F32>(v));
}

// four channels' runs
struct Runs { float A[kQuad], H[kQuad]; };
__device__ __forceinline__ Runs no_runs() {
    Runs r;
#pragma unroll
    for (int e = 0; e < kQuad; ++e) { r.A[e] = 1.f; r.H[e] = 0.f; }
    return r;
}
__device__ __forceinline__ void pass_through(const Runs& r, float (&v)[kQuad]) {
#pragma unroll
    for (int e = 0; e < kQuad; ++e) v[e] = through(Run{r.A[e], r.H[e]}, v[e]);
}
// Runs by channel in LDS.
struct RunTable {
    float A[64], H[64];
    __device__ __forceinline__ void put(int c, const Run& r) { A[c] = r.A; H[c] = r.H; }
    __device__ __forceinline__ void put4(int c, const Runs& r) {
        *reinterpret_cast<f32x4*>(&A[c]) = f32x4{r.A[0], r.A[1], r.A[2], r.A[3]};
        *reinterpret_cast<f32x4*>(&H[c]) = f32x4{r.H[0], r.H[1], r.H[2], r.H[3]};
    }
    __device__ __forceinline__ Run get(int c) const { return Run{A[c], H[c]}; }
};
struct ScanLds {
    RunTable wave[kScanThreads / 64];           // of every wave's rows
    RunTable tiles[kGroupTiles / 4];            // of four tiles each of the group, before this one
    RunTable groups[kLookWindow];               // of the groups before this one, backwards
    float before[kScanThreads / 64][64];        // value before every wave's rows
    f32x4 own_A[kScanThreads], own_H[kScanThreads];     // of the lanes before a lane in its wave: kept here while a tile waits, the registers are needed
    int ticket;
};

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

// Up to four words, 64 words from one to the next, waiting for those that are not there yet.  BACK: the words lie one
// before the other.  A word that does not come within the bound counts as NaN.
template <bool BACK>
__device__ __forceinline__ void gather_runs(const uint64_t* at, int n, Run (&r)[4]) {
    const int64_t step = BACK ? -64 : 64;
    uint64_t w[4];
#pragma unroll
    for (int k = 0; k < 4; ++k) w[k] = k < n ? look(at + step * k) : 0;
    for (int polls = 0; polls < kMostPolls; ++polls) {
        if (is_there(w[0]) && is_there(w[1]) && is_there(w[2]) && is_there(w[3])) break;
        __builtin_amdgcn_s_sleep(1);
#pragma unroll
        for (int k = 0; k < 4; ++k)
            if (!is_there(w[k])) w[k] = look(at + step * k);
    }
#pragma unroll
    for (int k = 0; k < 4; ++k) r[k] = is_there(w[k]) ? run_in(w[k]) : Run{-1.f, __uint_as_float(0x7FC00000u)};
}

// Publishes the tile's run and, from the last tile of a group, the group's, and leaves the value before every wave's rows
// in s.before; a lane is a channel here, and all but the waiting for others' words is done by the first wave.  All
// threads take part; ends with a barrier.
__device__ __forceinline__ void look_back(const ScanArgs& a, ScanLds& s, int slab, int tile, int begins) {
    const int wave = threadIdx.x >> 6, lane = threadIdx.x & 63, waves = blockDim.x >> 6;
    const int group = tile / kGroupTiles, in_group = tile % kGroupTiles;
    const bool here = lane < kQuad << a.lanes_log2, first = wave == 0 && here;
    const bool linked = a.tile_runs != nullptr, closes = linked && in_group == kGroupTiles - 1;
    // a tile that a sequence begins with asks nobody
    const bool asks = linked && !__builtin_amdgcn_readfirstlane(begins);
    uint64_t* tiles = a.tile_runs + ((int64_t)slab * a.tiles + (tile - in_group)) * 64 + lane;
    uint64_t* groups = a.group_runs + (int64_t)slab * a.groups * 64 + lane;
    Run mine{1.f, 0.f}, before{1.f, 0.f};           // of the tile; of the group's tiles before it
    if (first && linked) {
#pragma unroll 4
        for (int w = 0; w < waves; ++w) mine = then(mine, s.wave[w].get(lane));
        if (!closes) publish(tiles + in_group * 64, mine);
    }
    const int n_tiles = asks || closes ? in_group : 0, t_words = (n_tiles + 3) / 4;
#pragma unroll 1
    for (int k = wave; k < t_words; k += waves)
        if (here) {
            const int n = min(4, n_tiles - 4 * k);
            Run r[4], run{1.f, 0.f};
            gather_runs<false>(tiles + 4 * k * 64, n, r);
#pragma unroll
            for (int i = 0; i < 4; ++i)
                if (i < n) run = then(run, r[i]);
            s.tiles[k].put(lane, run);
        }
    if (closes) {
        __syncthreads();
        if (first) {
#pragma unroll 4
            for (int k = 0; k < t_words; ++k) before = then(before, s.tiles[k].get(lane));
            publish(groups + group * 64, then(before, mine));
        }
    }
    float v = 0.f, reach = 0.f;                     // before the tile, and before its group; of the first tile never used
    if (asks) {
        // The value behind the nearest group that knows it, through the groups after that one, one at a time: a group
        // that publishes what is behind it has come to the same bits, so it does not matter which one is found.
        const int n = min(group, kLookWindow), turn = closes ? 0 : t_words;     // waves that wait for a tile are not the first to wait for a group
#pragma unroll 1
        for (int polls = 0;; ++polls) {
#pragma unroll 1
            for (int k = (wave + waves - turn % waves) % waves; 4 * k < n; k += waves)
                if (here) {
                    Run r[4];
                    gather_runs<true>(groups + (int64_t)(group - 1 - 4 * k) * 64, min(4, n - 4 * k), r);
#pragma unroll
                    for (int i = 0; i < 4; ++i)
                        if (4 * k + i < n) s.groups[4 * k + i].put(lane, r[i]);
                }
            __syncthreads();
            bool known = n == 0 || !here || polls == kMostPolls;
#pragma unroll 4
            for (int k = 0; k < n; ++k) known = known || s.groups[k].A[lane] < 0.f;
            if (__all(known)) break;                // the same in every wave: each looks at all channels
            __syncthreads();
        }
        if (first) {
            if (n) reach = __uint_as_float(0x7FC00000u);        // from groups behind which nothing is known
#pragma unroll 4
            for (int k = n - 1; k >= 0; --k) reach = through(s.groups[k].get(lane), reach);
            if (!closes) {
#pragma unroll 4
                for (int k = 0; k < t_words; ++k) before = then(before, s.tiles[k].get(lane));
            }
            v = through(before, reach);
        }
    }
    if (closes && first) publish(groups + group * 64, Run{-1.f, through(then(before, mine), reach)});
    if (first) {
#pragma unroll 4
        for (int w = 0; w < waves; ++w) {
            s.before[w][lane] = v;
            v = through(s.wave[w].get(lane), v);
        }
    }
    __syncthreads();
}

// Before the tiles: nobody has said anything yet (2 MB of words for the 986,880 rows above, 3 us), and the states of
// sequences without rows pass through.
__global__ void __launch_bounds__(256)
k_scan_prepare(uint64_t* words, int64_t n, uint32_t* ticket, const int32_t* __restrict__ empty, int n_empty, int C, const float* __restrict__ first,
               float* __restrict__ last) {
    const int64_t t = (int64_t)blockIdx.x * 256 + threadIdx.x, step = (int64_t)gridDim.x * 256;
    for (int64_t i = t; i < n; i += step) words[i] = ~0ull;
    if (n && t == 0) *ticket = 0;
    for (int64_t i = t; i < (int64_t)n_empty * C; i += step) {
        const int64_t at = (int64_t)empty[i / C] * C + i % C;
        last[at] = first ? first[at] : 0.f;
    }
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

template <int DT, int KIND, bool UP, bool BWD, bool FULL>
__device__ __forceinline__ void scan_tile(const ScanArgs& a, ScanLds& s, int slab, int tile, int64_t tile0, int rows_a_tile) {
    constexpr int R = ScanRows<DT, BWD>::n;
    const int t = threadIdx.x, wave = t >> 6, lane = t & 63, lanes = 1 << a.lanes_log2;
    // The last lane of a row whose channels are not a multiple of four takes the last four: some of them a second time,
    // with the same bits, and so do the lanes that are left over, which store nothing.
    const int c4 = (lane & (lanes - 1)) * kQuad, col = KIND == kRowsNarrow ? c4 : min(slab * 64 + c4, a.C - kQuad);
    const bool stores = slab * 64 + c4 < a.C;
    TileRows<UP, R, FULL> tr;
    tr.count = FULL ? rows_a_tile : (int)min((int64_t)rows_a_tile, a.rows - tile0);
    tr.lowest = UP ? tile0 : a.rows - tile0 - tr.count;
    tr.lane = (t >> a.lanes_log2) * R;
    const LaneRows lr = lane_rows<UP, R>(a, tile0 + tr.lane);
    const int begins = begins_at<UP>(a, tile0);     // asked for here: in front of the tile's word to the others it would hold all of them up
    const unsigned char* in_rows = BWD ? a.gh : a.x;
    const int64_t ld_in = BWD ? a.ld_gh : a.ld_x;
    // One number or two of every value are held between the passes over the rows: forward, the state that the lane's own
    // rows make and the product of gates that a state before them enters it with; backward, the gate.
    Piece<DT, kQuad> in[R], px[BWD ? R : 1], pp[BWD ? R : 1];
    float held[R][kQuad], gates[BWD ? 1 : R][kQuad];
    Piece<DT, kQuad> gate[R];
#pragma unroll
    for (int i = 0; i < R; ++i) {
        gate[i] = load_piece<DT, KIND, kQuad>(tr.base(a.gate, a.ld_gate, i), tr.offset(a.ld_gate, i), col, a.C);
        in[i] = load_piece<DT, KIND, kQuad>(tr.base(in_rows, ld_in, i), tr.offset(ld_in, i), col, a.C);
        __builtin_amdgcn_sched_barrier(0);      // in turn: the first rows are worked on while the last are on their way
    }
    // of the first sequence that begins in the lane's rows and the first that ends, asked for along with the rows
    float start[kQuad], state0[kQuad];
    if (lr.begin) load_states<KIND>(a.first, sequence_of<UP>(a, lr, __ffs(lr.begin) - 1), col, a.C, start);
    int stopped = 0;
    if (lr.stop) {
        stopped = sequence_of<UP>(a, lr, __ffs(lr.stop) - 1);
        if (BWD) load_states<KIND>(a.h0, stopped, col, a.C, state0);
    }
    Runs mine = no_runs();                      // of this lane's rows
#pragma unroll
    for (int i = 0; i < R; ++i) {
        if (lr.begin >> i & 1) {
            if (lr.begin & ((1u << i) - 1)) load_states<KIND>(a.first, sequence_of<UP>(a, lr, i), col, a.C, start);
#pragma unroll
            for (int e = 0; e < kQuad; ++e) { mine.A[e] = 1.f; mine.H[e] = start[e]; }
        }
        float z[kQuad], v[kQuad];
        unpack<DT>(gate[i], z);
        unpack<DT>(in[i], v);
#pragma unroll
        for (int e = 0; e < kQuad; ++e) {
            float f, g;
            const float k = keep_gate(z[e], f, g);
            mine.H[e] = BWD ? f * (v[e] + mine.H[e]) : f * mine.H[e] + g * v[e];
            mine.A[e] *= f;
            held[i][e] = BWD ? k : mine.H[e];
            if (BWD) asm volatile("" : "+v"(held[i][e]));       // the number itself, not f and g that it stands for
            else gates[i][e] = mine.A[e];
        }
        if (BWD) {
#pragma unroll
            for (int k = 0; k < Piece<DT, kQuad>::kWords; ++k) asm volatile("" : "+v"(in[i].w[k]));     // as loaded, for the same reason
        }
        __builtin_amdgcn_sched_barrier(0);      // a row after the other: all rows' numbers at once do not fit the registers
    }
    // Runs of all lanes up to this one.  Where a sequence begins in a lane's rows, what stands before them is left out:
    // a bit a lane says so for all of its channels.
    uint64_t cut = __ballot(lr.begin != 0);
#pragma unroll 1
    for (int d = lanes; d < 64; d <<= 1) {
        const bool alone = (cut | ((1ull << d) - 1)) >> lane & 1;
#pragma unroll
        for (int e = 0; e < kQuad; ++e) {
            const float oA = __shfl_up(mine.A[e], d), oH = __shfl_up(mine.H[e], d);
            mine.H[e] = alone ? mine.H[e] : mine.A[e] * oH + mine.H[e];
            mine.A[e] = alone ? mine.A[e] : mine.A[e] * oA;
        }
        cut |= cut << d;
    }
    if (cut >> lane & 1) {
#pragma unroll
        for (int e = 0; e < kQuad; ++e) mine.A[e] = -1.f;
    }
    if (lane >= 64 - lanes) s.wave[wave].put4(c4, mine);
    // of the lanes before this one
#pragma unroll
    for (int e = 0; e < kQuad; ++e) {
        const float oA = __shfl_up(mine.A[e], lanes), oH = __shfl_up(mine.H[e], lanes);
        mine.A[e] = lane < lanes ? 1.f : oA;
        mine.H[e] = lane < lanes ? 0.f : oH;
    }
    s.own_A[t] = f32x4{mine.A[0], mine.A[1], mine.A[2], mine.A[3]};
    s.own_H[t] = f32x4{mine.H[0], mine.H[1], mine.H[2], mine.H[3]};
    __syncthreads();
    look_back(a, s, slab, tile, begins);
    if (BWD) {
        // The rows run against the sequence: the state before a row lies at the row that comes next here.  Behind the
        // last row of all there is none (and none is asked for): the row itself in its place.
        const int64_t more = tile0 + tr.count < a.rows ? a.ld_h : 0;
#pragma unroll
        for (int i = 0; i < R; ++i) {
            px[i] = load_piece<DT, KIND, kQuad>(tr.base(a.x, a.ld_x, i), tr.offset(a.ld_x, i), col, a.C);
            const bool last = tr.lane + i >= tr.count - 1;
            if (i + 1 < R && FULL) pp[i] = load_piece<DT, KIND, kQuad>(tr.base(a.h, a.ld_h, i + 1), tr.offset(a.ld_h, i + 1), col, a.C);
            else pp[i] = load_piece<DT, KIND, kQuad>(tr.base(a.h, a.ld_h, i) + (last ? (UP ? more : -more) : UP ? a.ld_h : -a.ld_h), tr.offset(a.ld_h, i), col, a.C);
        }
    }
    float v[kQuad];
    {
        const f32x4 b = *reinterpret_cast<const f32x4*>(&s.before[wave][c4]);
#pragma unroll
        for (int e = 0; e < kQuad; ++e) v[e] = b[e];
    }
    pass_through(Runs{{s.own_A[t][0], s.own_A[t][1], s.own_A[t][2], s.own_A[t][3]}, {s.own_H[t][0], s.own_H[t][1], s.own_H[t][2], s.own_H[t][3]}}, v);
#pragma unroll
    for (int i = 0; i < R; ++i) {
        if (!FULL && i >= lr.n) continue;
        const bool begins = lr.begin >> i & 1, ends = lr.stop >> i & 1;
        if (!BWD) {
            if (begins) {
#pragma unroll
                for (int e = 0; e < kQuad; ++e) v[e] = 0.f;     // what stands before the lane's rows ends here
            }
            float h[kQuad];
#pragma unroll
            for (int e = 0; e < kQuad; ++e) h[e] = gates[i][e] * v[e] + held[i][e];
            if (stores) store_piece<DT, KIND>(tr.base(a.out, a.ld_out, i), tr.offset(a.ld_out, i), col, a.C, pack<DT>(h));
            if (ends && a.last && stores) store_states<KIND>(a.last, lr.stop & ((1u << i) - 1) ? sequence_of<UP>(a, lr, i) : stopped, col, a.C, h);
        } else {
            if (begins) {
                if (lr.begin & (lr.begin - 1)) load_states<KIND>(a.first, sequence_of<UP>(a, lr, i), col, a.C, start);
#pragma unroll
                for (int e = 0; e < kQuad; ++e) v[e] = start[e];
            }
            float w[kQuad], x[kQuad], p[kQuad], gx[kQuad], gz[kQuad];
            unpack<DT>(in[i], w);
            unpack<DT>(px[i], x);
            unpack<DT>(pp[i], p);
            if (ends) {
                if (lr.stop & ((1u << i) - 1)) load_states<KIND>(a.h0, sequence_of<UP>(a, lr, i), col, a.C, state0);
#pragma unroll
                for (int e = 0; e < kQuad; ++e) p[e] = state0[e];
            }
#pragma unroll
            for (int e = 0; e < kQuad; ++e) {
                float f, g;
                kept_gate(held[i][e], f, g);
                const float lam = w[e] + v[e];
                gx[e] = g * lam;
                gz[e] = lam * (p[e] - x[e]) * (f * g);
                v[e] = f * lam;
            }
            if (stores) {
                store_piece<DT, KIND>(tr.base(a.gx, a.ld_gx, i), tr.offset(a.ld_gx, i), col, a.C, pack<DT>(gx));
                store_piece<DT, KIND>(tr.base(a.ggate, a.ld_ggate, i), tr.offset(a.ld_ggate, i), col, a.C, pack<DT>(gz));
            }
            if (ends && a.last && stores) store_states<KIND>(a.last, lr.stop & ((1u << i) - 1) ? sequence_of<UP>(a, lr, i) : stopped, col, a.C, v);
        }
        __builtin_amdgcn_sched_barrier(0);
    }
}

template <int DT, int KIND, bool UP, bool BWD>
// No register may be spilled here (the build refuses it): the compiler has stored one under the lanes of a branch that all
// lanes had taken it through.  Rows of fewer than four channels, whose pieces are loaded by tests, get more of them.
__global__ void __launch_bounds__(kScanThreads, KIND == kRowsNarrow && BWD ? 3 : 4)
k_scan(ScanArgs a) {
    __shared__ ScanLds s;
    int turn = blockIdx.x;
    if (a.tile_runs) {
        if (threadIdx.x == 0) s.ticket = (int)atomicAdd(a.ticket, 1u);
        __syncthreads();
        turn = __builtin_amdgcn_readfirstlane(s.ticket);
    }
    const int slab = turn % a.slabs, tile = turn / a.slabs, rows_a_tile = (blockDim.x >> a.lanes_log2) * ScanRows<DT, BWD>::n;
    const int64_t tile0 = (int64_t)tile * rows_a_tile;
    if (tile0 + rows_a_tile <= a.rows) scan_tile<DT, KIND, UP, BWD, true>(a, s, slab, tile, tile0, rows_a_tile);
    else scan_tile<DT, KIND, UP, BWD, false>(a, s, slab, tile, tile0, rows_a_tile);
}

// One row of each of many running sequences: h = f state + (1 - f) x, the state kept in fp32.  A thread is a piece of 8
// channels; bound by the launch at the sizes of a step (8 x 256: 3.2 us, of 10 us a call; 4,096 x 512 bf16, 29 MB: 12 us a
// call), short of a copy's rate beyond: 100,000 x 256 bf16 (358 MB) 104 us, 3.4 TB/s; the states move four bytes a lane at a
// time, 32 apart.
template <int DT, int KIND>
__global__ void __launch_bounds__(256)
k_scan_step(int64_t rows, int C, int pieces, const unsigned char* x, int64_t ld_x, const unsigned char* gate, int64_t ld_gate, const float* state,
            float* new_state, unsigned char* out, int64_t ld_out) {
    const int64_t i = (int64_t)blockIdx.x * blockDim.x + threadIdx.x, row = i / pieces;
    if (row >= rows) return;
    const int col = (int)(i - row * pieces) * kPiece;
    float z[kPiece], v[kPiece], h[kPiece];
    const Piece<DT> pz = load_piece<DT, KIND>(gate + row * ld_gate, 0, col, C), pv = load_piece<DT, KIND>(x + row * ld_x, 0, col, C);
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
    store_piece<DT, KIND>(out + row * ld_out, 0, col, C, pack<DT>(h));
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

constexpr int64_t kMostThreads = (1ll << 32) - 256;      // of a launch
constexpr int32_t kMostChannels = 1 << 24;      // a row's bytes and a tile's rows meet in 32 bits

static fx_status check_scan(const char* who, const fx_sequences* q, int32_t C, fx_dtype dt) {
    if (!q || C < 1 || (dt != FX_F32 && dt != FX_F16 && dt != FX_BF16)) {
        set_error("%s: null sequences, no channels or unknown dtype", who);
        return FX_EINVAL;
    }
    if (C > kMostChannels) { set_error("%s: more than %d channels", who, kMostChannels); return FX_ERANGE; }
    return FX_OK;
}

// Do two [rows, C] tables of fp32 share memory?  States are read by the workgroups of other channels (a slab of fewer than
// four takes the last of the slab before it along) and, backward, after others have written theirs: none may lie where one
// is written.
static bool share(const float* p, const float* q, int64_t rows, int32_t C) {
    const uintptr_t bytes = (uintptr_t)rows * C * sizeof(float), a = (uintptr_t)p, b = (uintptr_t)q;
    return p && q && (a < b ? b - a : a - b) < bytes;
}

static void scan_args(ScanArgs* a, const fx_sequences* q, int32_t C) {
    *a = ScanArgs{};
    a->rows = q->rows;
    a->C = C;
    const int quads = std::min(64 / kQuad, (C + kQuad - 1) / kQuad);
    while ((1 << a->lanes_log2) < quads) ++a->lanes_log2;
    a->slabs = (C + 63) / 64;
    a->begin = q->d_begin;
    a->rank = q->d_rank;
    a->id = q->d_id;
    a->empty = q->d_empty;
    a->n_empty = q->n_empty;
}

constexpr int64_t kMostOffset = 1ll << 31;      // bytes of a tile's rows: its last begins a row's distance before that

static int64_t most_ld(const ScanArgs& a) {
    return std::max({a.ld_x, a.ld_gate, a.ld_h, a.ld_gh, a.ld_out, a.ld_gx, a.ld_ggate});
}

static void launch_prepare(const ScanArgs& a, int64_t words, hipStream_t st) {
    const int64_t states = a.last ? (int64_t)a.n_empty * a.C : 0;
    k_scan_prepare<<<(unsigned)std::min<int64_t>((std::max(words, states) + 255) / 256, 1024), 256, 0, st>>>(
        a.tile_runs, words, a.ticket, a.empty, a.last ? a.n_empty : 0, a.C, a.first, a.last);
}

template <int DT, int KIND, bool UP, bool BWD>
static fx_status launch_scan(ScanArgs& a, hipStream_t st) {
    // Threads of a workgroup: one tile for everything if that can be, else at least 16 tiles if that can be, else as many
    // as there are.  Fewer and longer tiles have fewer others to wait for (986,880 x 64 bf16, 512 threads 133 us, 256 150 us;
    // 10,000 x 64 in 10 tiles a 1/16 of the compute units 12.7 us, in two a unit 17.1 us).
    int threads = kScanThreads;
    int64_t rows_a_tile, tiles;
    const int64_t ld = most_ld(a);
    for (;; threads /= 2) {
        rows_a_tile = (int64_t)(threads >> a.lanes_log2) * ScanRows<DT, BWD>::n;
        tiles = (a.rows + rows_a_tile - 1) / rows_a_tile;
        if (threads == 64) break;
        if (ld > kMostOffset / rows_a_tile) continue;
        if (tiles == 1 ? 2 * a.rows > rows_a_tile : tiles * a.slabs * 16 >= compute_units()) break;
    }
    if (ld > kMostOffset / rows_a_tile) { set_error("gated scan: rows lie more than %lld bytes apart", (long long)(kMostOffset / rows_a_tile)); return FX_ERANGE; }
    if (tiles * a.slabs > kMostThreads / threads) { set_error("gated scan: too many tiles for one launch"); return FX_ERANGE; }
    a.tiles = (int)tiles;
    a.groups = (int)((tiles + kGroupTiles - 1) / kGroupTiles);
    void* work = nullptr;
    unsigned nb = (unsigned)a.slabs;
    if (tiles <= 1 && a.last && a.n_empty) launch_prepare(a, 0, st);
    if (tiles > 1) {
        const int64_t words = (int64_t)a.slabs * 64 * (a.tiles + a.groups);
        FX_TRY(scratch_alloc("gated scan", &work, (size_t)words * 8 + 256, st));
        a.tile_runs = (uint64_t*)work;
        a.group_runs = a.tile_runs + (int64_t)a.slabs * 64 * a.tiles;
        a.ticket = (uint32_t*)(a.tile_runs + words);
        launch_prepare(a, words, st);
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
    if (a.C >= kQuad) return up ? launch_scan<DT, kRowsWhole, true, BWD>(a, st) : launch_scan<DT, kRowsWhole, false, BWD>(a, st);
    return up ? launch_scan<DT, kRowsNarrow, true, BWD>(a, st) : launch_scan<DT, kRowsNarrow, false, BWD>(a, st);
}

template <bool BWD>
static fx_status run_scan(ScanArgs& a, fx_dtype dt, bool up, hipStream_t st) {
    ProfScope ps(BWD ? kProfScanBwd : kProfScanFwd, st);
    if (a.rows == 0) {
        if (a.last && a.n_empty) launch_prepare(a, 0, st);
        FX_HIP_TRY(hipGetLastError());
        return FX_OK;
    }
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
    if (share(d_last, d_h0, q->B, C)) { set_error("%s: d_last must not lie where d_h0 lies", who); return FX_EINVAL; }
    ScanArgs a;
    scan_args(&a, q, C);
    const int es = esize(dt);
    a.x = (const unsigned char*)d_x; a.ld_x = ld_x * es;
    a.gate = (const unsigned char*)d_gate; a.ld_gate = ld_gate * es;
    a.out = (unsigned char*)d_h; a.ld_out = ld_h * es;
    a.first = d_h0;
    a.last = d_last;
    return run_scan<false>(a, dt, !reverse, (hipStream_t)stream);
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
    if (q->rows > 0 && d_gx == d_ggate) { set_error("%s: d_gx and d_ggate are the same", who); return FX_EINVAL; }
    if (share(d_gh0, d_glast, q->B, C) || share(d_gh0, d_h0, q->B, C)) { set_error("%s: d_gh0 must not lie where d_glast or d_h0 lies", who); return FX_EINVAL; }
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
    return run_scan<true>(a, dt, reverse != 0, (hipStream_t)stream);
}

extern "C" fx_status fx_gated_scan_step(const void* d_x, int64_t ld_x, const void* d_gate, int64_t ld_gate, fx_dtype dt, int64_t rows, int32_t C,
                                        const float* d_state, float* d_new_state, void* d_h, int64_t ld_h, void* stream) {
    const char* who = "fx_gated_scan_step";
    if (rows < 0 || C < 1 || (dt != FX_F32 && dt != FX_F16 && dt != FX_BF16) || (rows > 0 && (!d_state || !d_new_state))) {
        set_error("%s: negative rows, no channels, unknown dtype or null state", who);
        return FX_EINVAL;
    }
    if (C > kMostChannels) { set_error("%s: more than %d channels", who, kMostChannels); return FX_ERANGE; }
    FX_TRY(check_rows_of(who, "d_x", d_x, ld_x, rows, C, dt));
    FX_TRY(check_rows_of(who, "d_gate", d_gate, ld_gate, rows, C, dt));
    FX_TRY(check_rows_of(who, "d_h", d_h, ld_h, rows, C, dt));
    if (rows == 0) return FX_OK;
    // A row's last piece, where it is not whole, is read as the row's last eight channels: some are another thread's.
    if (d_h == d_x || d_h == d_gate) { set_error("%s: d_h must not be an input", who); return FX_EINVAL; }
    if (d_new_state != d_state && share(d_new_state, d_state, rows, C)) { set_error("%s: d_new_state overlaps d_state and is not d_state", who); return FX_EINVAL; }
    const int pieces = (C + kPiece - 1) / kPiece, es = esize(dt);
    if (rows > (0x7FFFFFFFll << 8) / pieces) { set_error("%s: too many rows", who); return FX_ERANGE; }
    hipStream_t st = (hipStream_t)stream;
    ProfScope ps(kProfScanFwd, st);
    const int kind = C < kPiece ? kRowsNarrow : C % kPiece ? kRowsRagged : kRowsWhole;
    // One launch, for all rows that there is memory for but of a few channels: a launch's threads are counted in 32 bits,
    // and more of them wrap without an error.
    const int64_t most = kMostThreads / pieces;
    for (int64_t r = 0; r < rows; r += most) {
        const int64_t n = std::min(most, rows - r);
        const unsigned blocks = (unsigned)((n * pieces + 255) / 256);
#define FX_STEP(DT, KIND) k_scan_step<DT, KIND><<<blocks, 256, 0, st>>>(n, C, pieces, (const unsigned char*)d_x + r * ld_x * es, ld_x * es, \
        (const unsigned char*)d_gate + r * ld_gate * es, ld_gate * es, d_state + r * C, d_new_state + r * C, (unsigned char*)d_h + r * ld_h * es, ld_h * es)
#define FX_STEP_KIND(DT) do { if (kind == kRowsWhole) FX_STEP(DT, kRowsWhole); else if (kind == kRowsRagged) FX_STEP(DT, kRowsRagged); \
                              else FX_STEP(DT, kRowsNarrow); } while (0)
        if (dt == FX_F32) FX_STEP_KIND(FX_F32);
        else if (dt == FX_F16) FX_STEP_KIND(FX_F16);
        else FX_STEP_KIND(FX_BF16);
#undef FX_STEP_KIND
#undef FX_STEP
    }
    FX_HIP_TRY(hipGetLastError());
    return FX_OK;
}
