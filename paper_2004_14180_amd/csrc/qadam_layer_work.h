// How the work of layer norm, the product in 8-bit integers and sampling is divided over launches, and the sizes of their scratch:
// arithmetic that the host and the kernels share.  Plain C++, so that it can be checked on the CPU at sizes no test allocates.
#pragma once

#include <stdint.h>

namespace qadam {

// ---- layer norm ---------------------------------------------------------------------------------
constexpr int kNormRun = 8;             // elements of a lane that lie one behind the other
constexpr int kNormHeldDim = 8192;      // up to here a row stays in the registers of 1 to 16 wavefronts, beyond it is read several times

// Workgroups of the gradient whose sums over rows are kept apart until all are added, at most: scratch of 8 bytes each per column.
// 16384 rows of 2048 bf16, us per call: 256 57.0, 512 42.9, 768 41.3, 1024 47.1; 8191 rows of 1001 22.2, 17.6, 17.6, 20.9; 8192 rows of 4096,
// whose workgroups are larger, 42.0, 46.3.
constexpr int norm_partials(int dim)
{
    const int n = (1 << 21) / dim, most = dim <= 2048 ? 512 : 256;
    return n < 8 ? 8 : n > most ? most : n;
}

// ---- product in 8-bit integers ------------------------------------------------------------------
constexpr int linear8_padded(int inputs) { return (inputs + 127) / 128 * 128; }     // of a token's integers in scratch
constexpr int kMadeInputs = 8192;       // tokens * padded inputs up to which every workgroup makes the integers itself

constexpr int kRowsTokens = 16;         // up to here the rows' kernel
constexpr int kRowWaves = 4;            // of a workgroup of that kernel

// Workgroups share a tile's inputs where tiles are so few that most CUs have none: a CU takes a step of 128 inputs in 0.25 us however many of
// them are in LDS, 0.5 where weights pass through registers.  Adding the parts' sums takes 2 to 3 us, hence steps that a part has at least.
// us per call, one part / parts: 64 tokens of 8192 to 2048 22.5 / 14.4, of 4096 to 1024 14.3 / 12.6 (parts of 8 steps 15.2 and 12.0), of 65536 to
// 64 148 / 41 (8 parts at most 45.7); of 2048 to 8192 10.6 / 11.2, not taken.  Through registers: 64 tokens of 2047 to 2048 17.7 / 13.2 (parts of
// 8 steps 14.4), of 1023 12.9 / 12.1, all before two steps of weights were under way; since then 10.9 and 9.4.
constexpr int kPartTiles = 256;         // workgroups that may have a part
constexpr int kPartSum = 64 * 64;       // sums of a tile
constexpr int kMostParts = 16;
constexpr int part_steps(bool direct) { return direct ? 16 : 4; }

// Which kernel takes a product, by its sizes.  us per call on both sides of each line (2048 inputs, 8192 outputs, where nothing else is
// said): rows / tiles of 64: 9 tokens 9.1 / 9.9, 16 tokens 9.7 / 10.4, of 1023 to 2048 9.4 / 12.5; beyond 16, with rows in pairs of tiles, 17 tokens
// 10.3 / 10.2, 32 tokens 10.9 / 10.2, of 768 to 50257 18.9 / 13.6, of 768 to 2304 10.2 / 8.4.  Tiles of 64 / 128: 384 tokens 15.2 / 18.1, 512 tokens
// 17.1 / 18.4, 768 tokens 25.8 / 20.6; 1024 tokens of 768 to 2304 10.5 / 12.4, 2048 16.5 / 15.4.  Up to two tiles of 64 on a CU wait for their
// loads: steps of two / three of them in LDS: 64 tokens 14.0 / 11.2, 256 tokens 14.6 / 13.8, 512 tokens (four on a CU) 18.5 / 21.5; through
// registers, of 2047 to 2048, 512 tokens (one on a CU) 16.3 / 14.8, 1024 18.6 / 20.0.  Tiles of 256 run one to a CU and take 1.7 times what two
// tiles of 128 do: 128 / 256: 1024 tokens 23.4 / 28.7, 2048 tokens 43.5 / 38.4, 4096 83.7 / 72.7, 16384 337 / 280; 8192 tokens of 768 to
// 2304 36.4 / 40.1.
struct Linear8Plan {
    enum Kind { kRows, kTiles64Deep, kTiles64, kTiles128, kTiles256 } kind;
    bool made;              // the product's workgroups make the tokens' integers
    int split;              // of the rows' kernel: wavefronts that share the inputs
    int parts;              // of tiles of 64: workgroups that share them

    constexpr Linear8Plan(int64_t tokens, int64_t outputs, int inputs, bool floats, bool direct = true) : kind(kTiles128), made(false), split(1), parts(1)
    {
        const int64_t tiles128 = (tokens + 127) / 128 * ((outputs + 127) / 128), tiles256 = (tokens + 255) / 256 * ((outputs + 255) / 256);
        if (tokens <= kRowsTokens) {
            kind = kRows;
            made = floats && tokens * linear8_padded(inputs) <= kMadeInputs;
            const int64_t waves = (outputs + 15) / 16;
            while (split < kRowWaves && waves * split < 2048 && inputs > 256 * split) split *= 2;
        } else if (tiles128 <= 256) {
            const int64_t tiles64 = (tokens + 63) / 64 * ((outputs + 63) / 64);
            kind = tiles64 <= (direct ? 512 : 256) ? kTiles64Deep : kTiles64;
            while (parts < kMostParts && tiles64 * parts * 2 <= kPartTiles && linear8_padded(inputs) / 128 >= parts * 2 * part_steps(direct)) parts *= 2;
        } else if ((tiles256 + 255) / 256 * 17 < (tiles128 + 511) / 512 * 10) {
            kind = kTiles256;
        }
    }
};

// Whether a call of up to max_tokens tokens may let workgroups share tiles
constexpr bool linear8_may_share(int64_t outputs, int inputs, int64_t max_tokens)
{
    return max_tokens > kRowsTokens && Linear8Plan(kRowsTokens + 1, outputs, inputs, false, false).parts > 1;
}

// Place of a workgroup's tile.  Workgroups go to the 8 XCDs in turn: each XCD gets a run of tiles, columns of 4 tiles of tokens one after
// the other, so that the tiles that it works on together share rows of both operands in its L2.
constexpr int kTileColumn = 4;
constexpr void tile_place(int block, int across, int down, int* tm, int* tn)
{
    const int total = across * down, each = total / 8, more = total % 8, xcd = block % 8;
    const int at = xcd * each + (xcd < more ? xcd : more) + block / 8;
    const int per = kTileColumn * across, column = at / per, height = down - column * kTileColumn < kTileColumn ? down - column * kTileColumn : kTileColumn;
    *tm = column * kTileColumn + at % per % height;
    *tn = at % per / height;
}

}  // namespace qadam
