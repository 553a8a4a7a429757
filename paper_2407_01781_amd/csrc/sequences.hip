// The tiles of the rows' division into sequences (fx_sequences::d_tiles).  Few are listed on the host and uploaded with the rest; many on the GPU: on
// the host 100,000 short sequences took ten times as long as all the rest of their division (1.46 ms with them, 0.29 so, 0.14 without any),
// and a program that only scans wants none of them.
#include "sequences.h"

#include <algorithm>

namespace fx {

constexpr int kSeqThreads = 1024, kSeqWaves = kSeqThreads / 64, kSeqClasses = 32, kSeqSums = 1 + kSeqTileKinds;       // of a class: its sequences, and their tiles of every kind
// Up to so many tiles of all kinds are listed on the host: 3,400 sequences of 203,132 rows, 17,085 tiles, 46 us so and 61 on the GPU; one of
// 986,880 rows, 53,970 tiles, 70 and 50
constexpr int64_t kTilesOnHost = 32768;

// Sequences are sorted by the power of two of their lengths; within one they keep their order
__host__ __device__ static inline int length_class(uint32_t len) { return len ? 31 - __builtin_clz(len) : -1; }
__host__ __device__ static inline uint32_t tiles_of(uint32_t len, int kind) { return (len + kSeqTileRows[kind] - 1) / kSeqTileRows[kind]; }

// A sequence in that order, and where its tiles of every kind begin
struct SeqPlace { uint32_t seq, at[kSeqTileKinds]; };
static_assert(kSeqSums == 4 && sizeof(SeqPlace) == 16, "counted and moved together");

__global__ __launch_bounds__(kSeqThreads) void k_seq_count(const int32_t* __restrict__ first, int32_t B, uint32_t* __restrict__ sums) {
    __shared__ uint32_t h[kSeqClasses * kSeqSums];
    for (int i = threadIdx.x; i < kSeqClasses * kSeqSums; i += kSeqThreads) h[i] = 0;
    __syncthreads();
    const int64_t b = (int64_t)blockIdx.x * kSeqThreads + threadIdx.x;
    const uint32_t len = b < B ? first[b + 1] - first[b] : 0;
    if (len) {
        uint32_t* mine = h + length_class(len) * kSeqSums;
        atomicAdd(mine, 1u);
        for (int t = 0; t < kSeqTileKinds; ++t) atomicAdd(mine + 1 + t, tiles_of(len, t));
    }
    __syncthreads();
    for (int i = threadIdx.x; i < kSeqClasses * kSeqSums; i += kSeqThreads) sums[(int64_t)blockIdx.x * kSeqClasses * kSeqSums + i] = h[i];
}

// Each block's sums become what stands before them: longer classes, and the class's earlier blocks
__global__ __launch_bounds__(kSeqClasses * kSeqSums) void k_seq_bases(uint32_t* __restrict__ sums, int blocks) {
    __shared__ uint32_t all[kSeqClasses * kSeqSums];
    uint32_t* mine = sums + threadIdx.x;
    uint32_t n = 0;
#pragma unroll 8
    for (int i = 0; i < blocks; ++i) n += mine[(int64_t)i * kSeqClasses * kSeqSums];
    all[threadIdx.x] = n;
    __syncthreads();
    uint32_t at = 0;
    for (int i = threadIdx.x + kSeqSums; i < kSeqClasses * kSeqSums; i += kSeqSums) at += all[i];
#pragma unroll 8
    for (int i = 0; i < blocks; ++i) {
        const uint32_t x = mine[(int64_t)i * kSeqClasses * kSeqSums];
        mine[(int64_t)i * kSeqClasses * kSeqSums] = at;
        at += x;
    }
}

__global__ __launch_bounds__(kSeqThreads) void k_seq_sort(const int32_t* __restrict__ first, int32_t B, const uint32_t* __restrict__ bases, SeqPlace* __restrict__ places) {
    __shared__ uint32_t of_wave[kSeqWaves][kSeqClasses][kSeqSums];
    for (int i = threadIdx.x; i < kSeqWaves * kSeqClasses * kSeqSums; i += kSeqThreads) (&of_wave[0][0][0])[i] = 0;
    __syncthreads();
    const int wave = threadIdx.x / 64, lane = threadIdx.x & 63;
    const int64_t b = (int64_t)blockIdx.x * kSeqThreads + threadIdx.x;
    const uint32_t len = b < B ? first[b + 1] - first[b] : 0;
    const int c = length_class(len);
    uint32_t n[kSeqSums] = {1, tiles_of(len, 0), tiles_of(len, 1), tiles_of(len, 2)}, before[kSeqSums] = {};
    for (uint64_t todo = __ballot(len != 0); todo;) {           // the classes that the wave has, one after the other
        const int now = __shfl(c, __ffsll((unsigned long long)todo) - 1, 64);
        const bool mine = c == now;
        todo &= ~__ballot(mine);
#pragma unroll
        for (int j = 0; j < kSeqSums; ++j) {
            uint32_t x = mine ? n[j] : 0;
            for (int d = 1; d < 64; d *= 2) { const uint32_t y = __shfl_up(x, d, 64); x += lane >= d ? y : 0; }
            if (mine) before[j] = x - n[j];
            if (lane == 63) of_wave[wave][now][j] = x;
        }
    }
    __syncthreads();
    if (!len) return;
    const uint32_t* base = bases + ((int64_t)blockIdx.x * kSeqClasses + c) * kSeqSums;
#pragma unroll
    for (int j = 0; j < kSeqSums; ++j) {
        before[j] += base[j];
        for (int w = 0; w < wave; ++w) before[j] += of_wave[w][c][j];
    }
    places[before[0]] = SeqPlace{(uint32_t)b, {before[1], before[2], before[3]}};
}

struct SeqTileLists { SeqTile* tiles[kSeqTileKinds]; int64_t n[kSeqTileKinds], all; };
__global__ __launch_bounds__(256) void k_seq_tiles(const int32_t* __restrict__ first, const SeqPlace* __restrict__ places, int32_t some, SeqTileLists l) {
    for (int64_t i = (int64_t)blockIdx.x * 256 + threadIdx.x; i < l.all; i += (int64_t)gridDim.x * 256) {
        int64_t at = i;
        int kind = 0;
        while (at >= l.n[kind]) at -= l.n[kind++];
        int32_t lo = 0, hi = some;              // the last that begins at this tile or before
        while (hi - lo > 1) { const int32_t mid = lo + (hi - lo) / 2; if (places[mid].at[kind] <= at) lo = mid; else hi = mid; }
        const int32_t b = (int32_t)places[lo].seq, r = first[b], len = first[b + 1] - r;
        const int32_t tile = (int32_t)tiles_of(len, kind) - 1 - (int32_t)(at - places[lo].at[kind]);
        l.tiles[kind][at] = SeqTile{b, tile * kSeqTileRows[kind], r, len};
    }
}

size_t tiles_on_host(const int64_t* n_tiles) {
    int64_t all = 0;
    for (int t = 0; t < kSeqTileKinds; ++t) all += n_tiles[t];
    return all <= kTilesOnHost ? (size_t)all : 0;
}

void list_tiles_on_host(const int64_t* h_joffsets, int32_t B, const int64_t* n_tiles, SeqTile* out) {
    uint32_t count[kSeqClasses][kSeqTileKinds] = {}, at[kSeqTileKinds] = {};
    const auto len_of = [&](int32_t b) { return (uint32_t)(h_joffsets[2 * b + 1] - h_joffsets[2 * b]); };
    for (int32_t b = 0; b < B; ++b)
        if (const uint32_t len = len_of(b))
            for (int t = 0; t < kSeqTileKinds; ++t) count[length_class(len)][t] += tiles_of(len, t);
    for (int c = kSeqClasses - 1; c >= 0; --c)
        for (int t = 0; t < kSeqTileKinds; ++t) { const uint32_t n = count[c][t]; count[c][t] = at[t]; at[t] += n; }
    SeqTile* const lists[kSeqTileKinds] = {out, out + n_tiles[0], out + n_tiles[0] + n_tiles[1]};
    for (int32_t b = 0; b < B; ++b)
        if (const uint32_t len = len_of(b))
            for (int t = 0; t < kSeqTileKinds; ++t) {
                uint32_t& place = count[length_class(len)][t];
                SeqTile* to = lists[t] + place;
                const uint32_t n = tiles_of(len, t);
                place += n;
                SeqTile tile{b, (int32_t)((n - 1) * kSeqTileRows[t]), (int32_t)h_joffsets[2 * b], (int32_t)len};
                for (uint32_t i = 0; i < n; ++i, tile.row -= kSeqTileRows[t]) to[i] = tile;
            }
}

fx_status list_tiles(const char* who, const fx_sequences* q, int32_t some, hipStream_t st) {
    SeqTileLists l{};
    for (int t = 0; t < kSeqTileKinds; ++t) {
        l.tiles[t] = const_cast<SeqTile*>(q->d_tiles[t]);
        l.all += l.n[t] = q->n_tiles[t];
    }
    const int blocks = (int)(((int64_t)q->B + kSeqThreads - 1) / kSeqThreads);
    const size_t of_places = (size_t)some * sizeof(SeqPlace);
    void* scratch = nullptr;
    FX_TRY(dev_alloc(&scratch, of_places + (size_t)blocks * kSeqClasses * kSeqSums * 4, st));
    uint32_t* sums = (uint32_t*)((char*)scratch + of_places);
    k_seq_count<<<blocks, kSeqThreads, 0, st>>>(q->d_first, q->B, sums);
    k_seq_bases<<<1, kSeqClasses * kSeqSums, 0, st>>>(sums, blocks);
    k_seq_sort<<<blocks, kSeqThreads, 0, st>>>(q->d_first, q->B, sums, (SeqPlace*)scratch);
    k_seq_tiles<<<(unsigned)std::min<int64_t>((l.all + 255) / 256, 1 << 16), 256, 0, st>>>(q->d_first, (const SeqPlace*)scratch, some, l);
    const hipError_t e = hipGetLastError();
    dev_free(scratch, st);
    if (e != hipSuccess) { set_error("%s: launch failed: %s", who, hipGetErrorString(e)); return FX_EDEVICE; }
    return FX_OK;
}

}  // namespace fx
