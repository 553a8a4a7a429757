// The rows' division into sequences (fx_build_sequences), as the recurrence and attention read it.
#pragma once
#include "common.h"

namespace fx {

// A tile of one sequence's rows: those from `row` (counted from the sequence's first) on, as many as its kind has; and
// the sequence itself, so that a workgroup's first load tells it all.
struct SeqTile { int32_t seq, row, first, len; };
constexpr int kSeqTileKinds = 3;
constexpr int kSeqTileRows[kSeqTileKinds] = {32, 64, 128};

}  // namespace fx

struct fx_sequences {
    int64_t rows = 0, longest = 0;
    int32_t B = 0, n_empty = 0;
    void* buf = nullptr;
    hipStream_t stream = nullptr;
    // bit r: a sequence begins at row r; row `rows` counts as a beginning.  Words up to the one after that.
    const uint64_t* d_begin = nullptr;
    const int32_t* d_rank = nullptr;        // beginnings before each word
    const int32_t* d_id = nullptr;          // number of the k-th sequence that is not empty
    const int32_t* d_empty = nullptr;       // numbers of the empty ones
    const int32_t* d_first = nullptr;       // [B + 1] first rows
    // Tiles of kSeqTileRows rows of all sequences, long sequences first and in each the last tile first: where a row sees
    // those before it, the tiles that take longest are begun first.
    const fx::SeqTile* d_tiles[fx::kSeqTileKinds] = {};
    int64_t n_tiles[fx::kSeqTileKinds] = {};
};

namespace fx {

// How many tiles the host lists: all, or none where they are many
size_t tiles_on_host(const int64_t* n_tiles);
void list_tiles_on_host(const int64_t* h_joffsets, int32_t B, const int64_t* n_tiles, SeqTile* out);
// Fills q's lists on the GPU; `some` sequences have rows
fx_status list_tiles(const char* who, const fx_sequences* q, int32_t some, hipStream_t st);

}  // namespace fx
