// How the work of layer norm, the product in 8-bit integers and sampling is divided over launches, and the sizes of their scratch:
// arithmetic that the host and the kernels share.  Plain C++, so that it can be checked on the CPU at sizes no test allocates.
#pragma once

#include <stdint.h>

namespace qadam {

// ---- layer norm ---------------------------------------------------------------------------------
constexpr int kNormRun = 8;             // elements of a lane that lie one behind the other
constexpr int kNormWaveDim = 2048;      // up to here a wavefront holds a row in registers,
constexpr int kNormGroupDim = 8192;     // up to here a workgroup of four does, beyond it rows are read several times

// Workgroups of the gradient whose sums over rows are kept apart until all are added, at most: scratch of 8 bytes each per column
constexpr int norm_partials(int dim)
{
    const int n = (1 << 21) / dim;
    return n < 8 ? 8 : n > 512 ? 512 : n;
}

// ---- product in 8-bit integers ------------------------------------------------------------------
constexpr int linear8_padded(int inputs) { return (inputs + 127) / 128 * 128; }     // of a token's integers in scratch
constexpr int kMadeInputs = 8192;       // tokens * padded inputs up to which every workgroup makes the integers itself

// Which kernel takes a product, by its sizes.
struct Linear8Plan {
    enum Kind { kRows16, kRows32, kRows64, kTiles128, kTiles256 } kind;
    bool made;              // the product's workgroups make the tokens' integers
    int split;              // of the rows' kernels: wavefronts that share the inputs

    constexpr Linear8Plan(int64_t tokens, int64_t outputs, int inputs, bool floats) : kind(kTiles128), made(false), split(1)
    {
        const int64_t tiles128 = (tokens + 127) / 128 * ((outputs + 127) / 128), tiles256 = (tokens + 255) / 256 * ((outputs + 255) / 256);
        if (tokens <= 64 || (tokens <= 512 && tiles128 < 192)) {
            kind = tokens <= 16 ? kRows16 : tokens <= 32 ? kRows32 : kRows64;
            made = floats && tokens <= 16 && tokens * linear8_padded(inputs) <= kMadeInputs;
            const int rows = kind == kRows16 ? 16 : 32, cols = kind == kRows16 ? 16 : kind == kRows32 ? 32 : 64;
            const int64_t waves = (outputs + rows - 1) / rows * ((tokens + cols - 1) / cols);
            while (split < 4 && waves * split < 2048 && inputs > 256 * split) split *= 2;
        } else if (tiles256 >= 384) {
            kind = kTiles256;
        }
    }
};

// Place of a workgroup's tile.  Workgroups go to the 8 XCDs in turn: each XCD gets a run of tiles, columns of 8 tiles of tokens one after
// the other, so that the tiles that it works on together share rows of both operands in its L2.
constexpr int kTileColumn = 8;
constexpr void tile_place(int block, int across, int down, int* tm, int* tn)
{
    const int total = across * down, each = total / 8, more = total % 8, xcd = block % 8;
    const int at = xcd * each + (xcd < more ? xcd : more) + block / 8;
    const int per = kTileColumn * across, column = at / per, height = down - column * kTileColumn < kTileColumn ? down - column * kTileColumn : kTileColumn;
    *tm = column * kTileColumn + at % per % height;
    *tn = at % per / height;
}

}  // namespace qadam
