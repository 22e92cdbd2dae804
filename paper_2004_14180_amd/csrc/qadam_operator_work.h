// How the work of the operators beside the step is divided over launches, and the sizes of their scratch: arithmetic that the host
// and the kernels share.  Plain C++, so that it can be checked on the CPU at sizes no test allocates.
#pragma once

#include <stdint.h>

namespace qadam {

constexpr int64_t kMostItems = (int64_t)1 << 32;    // work-items of a launch: fewer

// ---- lists of tensors ---------------------------------------------------------------------------
constexpr int kListTile = 4096;         // elements of one tensor that a record of the list's table stands for
constexpr int kListGrads = 448;         // gradients' addresses of one launch: they travel as kernel arguments (4 KB in all)
constexpr int kTileBlocks = kListTile / 256;        // wavefronts of AdamW per record

// A launch takes the next tensors of the list, as many as their gradients' addresses and their wavefronts allow.
constexpr int64_t kMostLaunchTiles = kMostItems / (64 * kTileBlocks) - 1;
constexpr int64_t kMostListTiles = (int64_t)1 << 26;        // 2^38 elements, more than the memory holds in any type
constexpr bool list_launch_takes(int64_t tensors, int64_t tiles, int64_t next)
{
    return tensors < kListGrads && tiles + next <= kMostLaunchTiles;
}

// ---- embedding gradient -------------------------------------------------------------------------
constexpr int kSortTile = 4096;         // tokens of a workgroup of the sort in passes
constexpr int kSortBits = 9;            // of a digit, at most
constexpr int kRunPiece = 40;           // tokens of one row that a wavefront adds at most; longer runs are joined
constexpr int kChunk = 8;               // tokens whose pieces a wavefront takes

// a lane's columns: 4, or as few as leave no lane of a narrow matrix idle
inline int lane_columns(int dim) { return dim > 128 ? 4 : dim > 64 ? 2 : 1; }
inline int column_slices(int dim) { return (dim + 64 * lane_columns(dim) - 1) / (64 * lane_columns(dim)); }

// Lists that are not sorted: up to kDirectTokens tokens, and kDirectGroups workgroups of up to four slices of a token's columns.
constexpr int kDirectTokens = 2048;
constexpr int kDirectGroups = 2048;     // which all look through the list: us with more of them / sorted, added: 1500 tokens of 2048 bf16
                                        // 15.2 / 14.0, 1024 10.4 / 12.2; 2000 of 768 fp32 (below) 10.0 / 14.4
constexpr int kDirectWaves = 8;         // of a workgroup
constexpr int kDirectClear = 8;         // rows of a wavefront that clears, which reads the whole list for them
inline int log_group_slices(int dim)
{
    const int slices = column_slices(dim);
    return slices > 2 ? 2 : slices - 1;
}
inline int groups_per_token(int dim) { return (column_slices(dim) + (1 << log_group_slices(dim)) - 1) >> log_group_slices(dim); }
// the most tokens of a list that is not sorted: 2048 up to 1024 columns, 1024 up to 2048, 512 up to 4096
inline int64_t direct_tokens(int dim)
{
    const int64_t n = kDirectGroups / groups_per_token(dim);
    return n < kDirectTokens ? n : kDirectTokens;
}
inline int64_t direct_clear_groups(int64_t rows) { return (rows + kDirectWaves * kDirectClear - 1) / (kDirectWaves * kDirectClear); }

// Scratch: sorted lists have two pieces per block of kRunPiece tokens and one count of arrivals, others one of each per token.
inline int64_t sort_tiles(int64_t tokens) { return (tokens + kSortTile - 1) / kSortTile; }
inline int64_t places(int64_t tokens, int dim, int64_t per_block)
{
    const int64_t most = direct_tokens(dim), blocks = per_block * (tokens / kRunPiece + 1), direct = tokens < most ? tokens : most;
    return blocks > direct ? blocks : direct;
}
inline int64_t arrival_places(int64_t tokens, int dim) { return places(tokens, dim, 1); }
inline int64_t piece_places(int64_t tokens, int dim) { return places(tokens, dim, 2); }

// The sums of a sorted list: a wavefront per chunk of tokens and slice of columns (a handle's largest list has fewer than kMostSums), and
// those that look through rows to clear the ones without a token, kClearRows at a time; of more rows than kMostSums of them take at
// once, each takes several turns.
constexpr int kClearRows = 2;
constexpr int64_t kMostSums = (int64_t)1 << 25;
inline int64_t sum_groups(int64_t tokens, int dim) { return (tokens + kChunk - 1) / kChunk * column_slices(dim); }
inline int64_t clear_groups(int64_t rows)
{
    const int64_t n = (rows + kClearRows - 1) / kClearRows;
    return n < kMostSums ? n : kMostSums;
}

// How many boundaries between blocks lie within a run, counted from the nearest one: they are the first of all, so 64 are looked at
// together, and while all of a look belong to the run the next one is 64 times as wide, then narrower again.
struct RunSearch {
    int32_t count = 0, step = 1;
    bool widen = true;

    // the boundary that a lane looks at
    constexpr int32_t place(int lane) const { return count + (lane + 1) * step - 1; }

    // `matched` lanes, the first ones, found theirs within the run: whether there is another look
    constexpr bool next(int matched)
    {
        count += matched * step;
        if (widen && matched == 64) {
            step *= 64;
            return true;
        }
        widen = false;
        if (step == 1) return false;
        step /= 64;
        return true;
    }
};

}  // namespace qadam
