// Shared by the operators that work on rows of C channels (scan.hip, block.hip): pieces of eight channels as a lane's
// unit of work, the reduction over the lanes of a row, and dropout's generator.
#pragma once
#include "conv_common.h"

namespace fx {

constexpr int kPiece = 8;               // channels a lane loads, computes on and stores at a time
constexpr int kMaxRowChannels = 4096;   // widest row of the norms

// Kind of row: channels in whole pieces; a ragged last piece; fewer channels than a piece
enum RowKind { kRowsWhole = 0, kRowsRagged = 1, kRowsNarrow = 2 };

// N channels as they lie in memory
template <int DT, int N = kPiece> struct Piece {
    static constexpr int kBytes = DT == FX_F32 ? 4 : 2, kWords = N * kBytes / 4;
    uint32_t w[kWords];
};

// A few bytes at any address that is a multiple of the element's size: rows of an odd number of channels, and columns
// of a wider tensor, start anywhere.  One load or store instruction all the same.
template <int WORDS> struct __attribute__((packed, aligned(2))) Bytes { uint32_t w[WORDS]; };

// The piece that begins at channel `col` of the row `off` bytes behind `base` (apart from the base: where that is the same
// in all lanes, it stays in scalar registers).  Channels from C on come as zeros, but for a lane that has no channel at
// all: it gets some of the row's, for the caller to mask where they would count.  A ragged row's last
// piece is loaded as the row's last N channels and moved into place, so that no load passes the row's end and every
// lane, one without channels too, loads from inside the row.
template <int DT, int KIND, int N = kPiece>
__device__ __forceinline__ Piece<DT, N> load_piece(const unsigned char* base, uint32_t off, int col, int C) {
    Piece<DT, N> p;
    constexpr int ES = Piece<DT, N>::kBytes, NW = Piece<DT, N>::kWords, LW = NW < 4 ? NW : 4;
    if (KIND == kRowsNarrow) {
        const unsigned char* row = base + off;
#pragma unroll
        for (int i = 0; i < NW; ++i) p.w[i] = 0;
#pragma unroll
        for (int e = 0; e < N - 1; ++e)
            if (col + e < C) {
                if (DT == FX_F32) p.w[e % NW] = reinterpret_cast<const uint32_t*>(row)[col + e];
                else p.w[e >> 1] |= (uint32_t)reinterpret_cast<const uint16_t*>(row)[col + e] << (16 * (e & 1));
            }
        return p;
    }
    const int at = min(col, C - N);
    const unsigned char* src = base + (uint32_t)(off + at * ES);
#pragma unroll
    for (int i = 0; i < NW / LW; ++i) {
        const Bytes<LW> b = reinterpret_cast<const Bytes<LW>*>(src)[i];
#pragma unroll
        for (int j = 0; j < LW; ++j) p.w[LW * i + j] = b.w[j];
    }
    if (KIND == kRowsRagged) {      // move by col - at channels, 0 .. N - 1 and more where the lane has no channel at all
        const int bits = (col - at) * 8 * ES;
#pragma unroll
        for (int step = NW / 2; step >= 1; step >>= 1) {
            const bool on = bits & (32 * step);
#pragma unroll
            for (int i = 0; i < NW; ++i) {
                const uint32_t from = i + step < NW ? p.w[i + step] : 0u;
                p.w[i] = on ? from : p.w[i];
            }
        }
        if (ES == 2) {
#pragma unroll
            for (int i = 0; i < NW; ++i) p.w[i] = __builtin_amdgcn_alignbit(i + 1 < NW ? p.w[i + 1] : 0u, p.w[i], bits & 16);
        }
    }
    return p;
}

// All bits for a lane that has channels, none for one that has not.  Opaque: a test in its place becomes a branch behind
// every load, which waits for it.
__device__ __forceinline__ uint32_t lane_mask(int col, int C) {
    uint32_t m = col < C ? ~0u : 0u;
    asm volatile("" : "+v"(m));
    return m;
}
template <int DT, int N>
__device__ __forceinline__ Piece<DT, N> masked(Piece<DT, N> p, uint32_t mask) {
#pragma unroll
    for (int i = 0; i < Piece<DT, N>::kWords; ++i) p.w[i] &= mask;
    return p;
}

// v under a mask of all bits, zero under none, whatever v is: no product with a zero does that to an infinity or NaN
__device__ __forceinline__ float kept(float v, uint32_t mask) { return __uint_as_float(__float_as_uint(v) & mask); }

template <int DT, int N>
__device__ __forceinline__ void unpack(const Piece<DT, N>& p, float (&v)[N]) {
#pragma unroll
    for (int e = 0; e < N; ++e) {
        if (DT == FX_F32) v[e] = __uint_as_float(p.w[e % Piece<DT, N>::kWords]);
        else if (DT == FX_BF16) v[e] = __uint_as_float(e & 1 ? p.w[e >> 1] & 0xFFFF0000u : p.w[e >> 1] << 16);
        else v[e] = Elem<_Float16>::to_float((uint16_t)(p.w[e >> 1] >> (16 * (e & 1))));
    }
}

// one rounding to the storage type (round to nearest even)
template <int DT, int N>
__device__ __forceinline__ Piece<DT, N> pack(const float (&v)[N]) {
    Piece<DT, N> p;
    if (DT == FX_F32) {
#pragma unroll
        for (int e = 0; e < N; ++e) p.w[e % Piece<DT, N>::kWords] = __float_as_uint(v[e]);
    } else {
#pragma unroll
        for (int e = 0; e < N; e += 2)
            p.w[e >> 1] = DT == FX_F16 ? Elem<_Float16>::pack2(v[e], v[e + 1]) : Elem<__bf16>::pack2(v[e], v[e + 1]);
    }
    return p;
}

template <int DT, int KIND, int N>
__device__ __forceinline__ void store_piece(unsigned char* base, uint32_t off, int col, int C, const Piece<DT, N>& p) {
    constexpr int ES = Piece<DT, N>::kBytes, NW = Piece<DT, N>::kWords, LW = NW < 4 ? NW : 4;
    unsigned char* dst = base + (uint32_t)(off + col * ES);
    const int n = C - col;
    if (KIND != kRowsNarrow && n >= N) {
#pragma unroll
        for (int i = 0; i < NW / LW; ++i) {
            Bytes<LW> b;
#pragma unroll
            for (int j = 0; j < LW; ++j) b.w[j] = p.w[LW * i + j];
            reinterpret_cast<Bytes<LW>*>(dst)[i] = b;
        }
        return;
    }
    if (KIND == kRowsWhole || n <= 0) return;
    if (DT == FX_F32) {
#pragma unroll
        for (int e = 0; e < N - 1; ++e)
            if (e < n) reinterpret_cast<uint32_t*>(dst)[e] = p.w[e % NW];
    } else {                        // 4, 2 and 1 channels, the binary digits of what is left
        uint32_t a = p.w[0];
        int at = 0;
        if (N > 4 && (n & 4)) { reinterpret_cast<Bytes<2>*>(dst)[0] = Bytes<2>{{p.w[0], p.w[1 % NW]}}; a = p.w[2 % NW]; at = 4; }
        if (n & 2) { reinterpret_cast<Bytes<1>*>(dst + at * 2)[0] = Bytes<1>{{a}}; a = p.w[(at + 2) / 2 % NW]; at += 2; }
        if (n & 1) reinterpret_cast<uint16_t*>(dst)[at] = (uint16_t)a;
    }
}

// a vector of C values, FX_F32 or of the rows' type, by channel; `absent` where there is none
template <int DT, int KIND>
__device__ __forceinline__ void load_vector(const void* p, int is_f32, int col, int C, float absent, float (&v)[kPiece]) {
    const unsigned char* b = reinterpret_cast<const unsigned char*>(p);
#pragma unroll
    for (int e = 0; e < kPiece; ++e) v[e] = absent;
    if (p && is_f32) unpack<FX_F32>(load_piece<FX_F32, KIND>(b, 0, col, C), v);
    else if (p) unpack<DT>(load_piece<DT, KIND>(b, 0, col, C), v);
}

template <int CTRL>
__device__ __forceinline__ float dpp(float v) {
    return __uint_as_float((uint32_t)__builtin_amdgcn_update_dpp(0, (int)__float_as_uint(v), CTRL, 0xF, 0xF, true));
}

// Sum over the `lanes` (a power of two up to 64, the same in every lane) neighbours that share a row; every lane gets the
// same bits, as each step adds the same two numbers on both sides.  All 64 lanes must be active.
__device__ __forceinline__ float row_sum(float v, int lanes) {
    if (lanes > 1) v += dpp<0xB1>(v);           // lanes 1 0 3 2 of four
    if (lanes > 2) v += dpp<0x4E>(v);           // lanes 2 3 0 1
    if (lanes > 4) v += dpp<0x141>(v);          // eight lanes mirrored: the other four
    if (lanes > 8) v += dpp<0x140>(v);          // sixteen lanes mirrored: the other eight
    if (lanes > 16) v += __shfl_xor(v, 16);
    if (lanes > 32) v += __shfl_xor(v, 32);
    return v;
}

// sigmoid(z) and sigmoid(-z), each to its own last digits: the smaller is e / (1 + e) of e = exp(-|z|) <= 1, the larger
// what it leaves of 1, so neither overflows and neither is a difference of near numbers.  e is the square of exp(-|z| / 2):
// the instruction gives zero where its result is subnormal, a product does not, and gates that far out are all there is
// of a sum over rows with such gates.
__device__ __forceinline__ void sigmoids(float z, float& up, float& down) {
    const float root = __builtin_amdgcn_exp2f(-0.72134752044448f * fabsf(z)), e = root * root;
    const float small = e * __builtin_amdgcn_rcpf(1.f + e), large = 1.f - small;
    up = z > 0.f ? large : small;
    down = z > 0.f ? small : large;
}

// ---------------------------------------------------------------------------------- dropout
// Philox4x32 with seven rounds, the fewest that pass all of the tests of its authors (Salmon, Moraes, Dror and Shaw,
// "Parallel random numbers: as easy as 1, 2, 3", 2011): the four words of counter (piece, row, offset) under key `seed`
// are eight 16-bit numbers, one for each channel of the piece.  Nothing depends on how rows and channels are spread
// over lanes, so every kernel draws the same mask from the same (seed, offset).
struct DropArgs {
    uint64_t seed, offset;
    const uint64_t* d_more;     // added to the offset when the kernel runs (NULL: nothing)
    uint32_t below;             // kept from this number on: round(65536 p); 0: everything is kept
    float factor, rest;         // 65536 / (65536 - below) is the sum of the two
};

__device__ __forceinline__ void philox8(uint32_t piece, uint32_t row, uint64_t offset, uint64_t seed, uint32_t (&w)[4]) {
    uint32_t c0 = piece, c1 = row, c2 = (uint32_t)offset, c3 = (uint32_t)(offset >> 32);
    uint32_t k0 = (uint32_t)seed, k1 = (uint32_t)(seed >> 32);
#pragma unroll
    for (int r = 0; r < 7; ++r) {
        const uint64_t a = (uint64_t)c0 * 0xD2511F53u, b = (uint64_t)c2 * 0xCD9E8D57u;
        c0 = (uint32_t)(b >> 32) ^ c1 ^ k0;
        c1 = (uint32_t)b;
        c2 = (uint32_t)(a >> 32) ^ c3 ^ k1;
        c3 = (uint32_t)a;
        k0 += 0x9E3779B9u;
        k1 += 0xBB67AE85u;
    }
    w[0] = c0; w[1] = c1; w[2] = c2; w[3] = c3;
}

__device__ __forceinline__ bool drop_keeps(const uint32_t (&w)[4], int e, uint32_t below) {
    return ((w[e >> 1] >> (16 * (e & 1))) & 0xFFFFu) >= below;
}

// a kept value times 65536 / (65536 - below), rounded once: a factor of 24 bits would be off by a rounding of its own
// (the rest of an infinity is held finite: it must not meet the infinity with the other sign)
__device__ __forceinline__ float drop_value(const uint32_t (&w)[4], int e, const DropArgs& d, float v) {
    return drop_keeps(w, e, d.below) ? fmaf(v, d.factor, __builtin_amdgcn_fmed3f(v, -3.402823466e38f, 3.402823466e38f) * d.rest) : 0.f;
}

}  // namespace fx
