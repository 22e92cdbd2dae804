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

}  // namespace qadam
