// Shared declarations between the host side of layer norm, the product in 8-bit integers and sampling (qadam_layers.cpp) and their
// gfx950 kernels (qadam_layer_norm.hip, qadam_linear8.hip, qadam_sampler.hip).  Not part of the public interface.
#pragma once

#include <hip/hip_runtime_api.h>
#include <stdint.h>

#include "qadam_internal.h"
#include "qadam_layer_work.h"

namespace qadam {

// ---- layer norm ---------------------------------------------------------------------------------
struct NormForward {
    int64_t rows;
    const void* x;
    int64_t x_stride;
    const void *weight, *bias;
    void*   out;
    int64_t out_stride;
    float  *mean, *rstd;
    float   eps;
    int32_t dim, x_type, weight_type, out_type;
    hipStream_t stream;
};
hipError_t launch_layer_norm(const NormForward& L);

struct NormBackward {
    int64_t rows;
    const void *dout, *x;
    int64_t dout_stride, x_stride;
    const void* weight;
    const float *mean, *rstd;
    void*   dx;
    int64_t dx_stride;
    void   *dweight, *dbias;
    float*  partial;        // [norm_partials(dim)][2][dim]
    int32_t dim, dout_type, x_type, weight_type, dx_type, grad_type, accumulate;
    hipStream_t stream;
};
hipError_t launch_layer_norm_grad(const NormBackward& L);

// ---- product in 8-bit integers ------------------------------------------------------------------
// Tokens to integers, or a copy of integers; `padded` of each are written, zeros from `inputs` on.
struct TokensLaunch {
    int64_t tokens;
    const void* x;
    int64_t x_stride;
    int8_t* codes;
    int64_t codes_stride;
    float*  scales;         // not written for a copy
    int32_t inputs, padded, x_type;
    hipStream_t stream;
    uint32_t* arrived = nullptr;        // kPartTiles counters that become zeros, or null
};
hipError_t launch_tokens(const TokensLaunch& L);

struct ProductLaunch {
    int64_t tokens, outputs;
    const int8_t* codes;    // rows of linear8_padded(inputs) at addresses of 16 bytes
    int64_t codes_stride;
    const float* token_scales;
    const int8_t* weight;
    int64_t weight_stride;
    const float* weight_scales;
    const void* bias;
    void*   out;
    int64_t out_stride;
    float   code_scale;     // where there are no weight_scales
    int32_t inputs, bias_type, out_type;
    hipStream_t stream;
    int32_t* sums;          // kPartTiles * kPartSum, of workgroups that share a tile; null: none do
};
// X: how the tokens become L.codes, its own `codes` null where they need not.
hipError_t launch_product(const ProductLaunch& L, const TokensLaunch& X);

// ---- sampling -----------------------------------------------------------------------------------
struct SampleLaunch {
    int64_t rows, vocab;
    const void* logits;
    int64_t logits_stride;
    const float* u;
    void*   out;
    uint32_t* status;
    qadam_filters_t filters;
    int32_t logits_type, token_bytes;
    hipStream_t stream;
};
hipError_t launch_sample(const SampleLaunch& L);

}  // namespace qadam
