// Shared declarations between the host side of the operators beside the step (qadam_operators.cpp) and their gfx950 kernels
// (qadam_tensors.hip, qadam_embedding.hip).  Not part of the public interface.
#pragma once

#include <hip/hip_runtime_api.h>
#include <stdint.h>

#include "qadam_internal.h"
#include "qadam_operator_work.h"

namespace qadam {

// ---- lists of tensors ---------------------------------------------------------------------------
struct ListTile {
    int32_t tensor;         // of the list
    int32_t tile;           // of the tensor
    int32_t count;          // elements, of tensors that are not shifted
    int32_t grad_type;
};
static_assert(sizeof(ListTile) == 16, "records are read as scalar loads");

// One tensor as the kernels read it.
struct ListTensor {
    void*   param;
    void*   m;
    void*   v;
    float*  m_scales;
    float*  v_scales;
    void*   copy;
    int64_t numel;
    int32_t types;          // list_types(): what the kernels branch on; above kTypeBits the shift of the tensor's blocks
    float   weight_decay;
};
static_assert(sizeof(ListTensor) == 64, "records are read as scalar loads");

// weights fp32 without and with a copy, or in 16 bits; gradients in three types
constexpr int kNoCopy = 3;
constexpr int kTypeBits = 6;
constexpr int list_types(int param, int grad, int copy) { return param | grad << 2 | copy << 4; }

// With 32-bit states a tensor's blocks need not begin with it, and are laid so that they begin at lines of 128 bytes of the weights, by
// `shift` elements in front of the tensor: wavefronts that share lines cost a quarter of the step (124 M elements in slices at any
// offset, us per step: 690, and now 569; whole lines from the start 564).
inline int block_shift(const void* param, int size) { return (int)(reinterpret_cast<uintptr_t>(param) % 128 / size); }

struct GradTable {
    const void* grad[kListGrads];
};

struct AdamwScalars {
    float beta1, omb1, beta2, omb2;     // beta and 1 - beta
    float lr, lr1, inv_sbc2, eps;       // lr / (1 - beta1^t), 1 / sqrt(1 - beta2^t)
};

// tiles [first_tile, first_tile + num_tiles) of the list, whose tensors are at most kListGrads from first_tensor on
struct ListLaunch {
    const ListTile*   tiles;
    const ListTensor* tensors;
    int32_t first_tile, num_tiles, first_tensor;
    hipStream_t stream;
};

hipError_t launch_adamw(const ListLaunch& L, const AdamwScalars& S, const GradTable& G, const float* grad_factor, bool state8);

constexpr int kNormGroups = 1536;       // workgroups of a launch of the norm, at most
// arrivals of a launch: workgroups count in one of so many words, the last one of each in the first word, all in lines of their own
// (one word for all of 1024 workgroups costs 12 us, 12 ns each)
constexpr int kArrivalCounts = 32, kArrivalStride = 32, kArrivalWords = (kArrivalCounts + 1) * kArrivalStride;
inline int norm_groups(int num_tiles) { return num_tiles < 1 ? 1 : num_tiles < kNormGroups ? num_tiles : kNormGroups; }

// partial sums of a launch at sums + first_sum; the last launch (`total` > 0: sums of all launches) finishes
struct NormLaunch {
    double*   sums;
    uint32_t* arrived;      // zero between launches
    int32_t   first_sum, total;
    float     max_norm;
    float*    out;
};
hipError_t launch_grad_norm(const ListLaunch& L, const NormLaunch& N, const GradTable& G);

// ---- embedding ----------------------------------------------------------------------------------
struct TokenList {
    const void* tokens;
    int32_t bytes;          // 4 or 8
    int64_t num, padding, rows;
    uint32_t* status;
};

struct LookupLaunch {
    TokenList t;
    const void* weight;
    int32_t weight_type, out_type, dim;
    int64_t weight_stride, out_stride;
    float   scale;          // of a code j too
    void*   out;
    hipStream_t stream;
};
hipError_t launch_embedding_lookup(const LookupLaunch& L);

// Scratch of the gradient, for lists of up to max_tokens: the tokens' sorted order, and what joins long runs.
struct EmbeddingScratch {
    int32_t*  keys[2];      // [max_tokens] rows in ascending order, `rows` for tokens without one
    int32_t*  order[2];     // [max_tokens] their positions in the list
    uint32_t* counts;       // [tiles][1 << kSortBits]
    float*    pieces;       // [piece_places(max_tokens, dim)][dim]
    uint32_t* arrived;      // [arrival_places(max_tokens, dim)][slices of columns], zero between launches
};

struct EmbeddingGradLaunch {
    TokenList t;
    EmbeddingScratch w;
    const void* dout;
    void*   grad;
    int32_t dout_type, grad_type, dim, accumulate;
    int64_t dout_stride, grad_stride;
    float   scale;
    hipStream_t stream;
};
hipError_t launch_embedding_grad(const EmbeddingGradLaunch& L);

}  // namespace qadam
