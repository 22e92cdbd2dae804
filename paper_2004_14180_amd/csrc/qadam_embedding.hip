// gfx950 kernels of the embedding: lookup with scaling, and the gradient by sorted tokens.
#include "qadam_elements.h"
#include "qadam_operators.h"

namespace qadam {
namespace {

constexpr int kThreads = 256;

// the row of token t, or -1 (padding, out of range)
__device__ __forceinline__ int64_t token_row(const TokenList& L, int64_t t, bool* out_of_range)
{
    const int64_t tok = L.bytes == 4 ? static_cast<const int32_t*>(L.tokens)[t] : static_cast<const int64_t*>(L.tokens)[t];
    *out_of_range = tok < 0 || tok >= L.rows;
    return *out_of_range || tok == L.padding ? -1 : tok;
}

__device__ __forceinline__ float element(const void* p, int type, int64_t i)
{
    if (type == QADAM_CODES8) return (float)static_cast<const int8_t*>(p)[i];
    if (type == QADAM_CODES16) return (float)static_cast<const int16_t*>(p)[i];
    return load_one(p, type, i);
}

__global__ void __launch_bounds__(kThreads) k_lookup(LookupLaunch L)
{
    for (int64_t t = blockIdx.x; t < L.t.num; t += gridDim.x) {
        bool outside;
        const int64_t row = token_row(L.t, t, &outside);
        if (outside && threadIdx.x == 0) atomicOr(L.t.status, QADAM_STATUS_TOKEN_RANGE);
        for (int k = threadIdx.x; k < L.dim; k += kThreads) {
            const float x = row < 0 ? 0.0f : element(L.weight, L.weight_type, row * L.weight_stride + k) * L.scale;
            store_one(L.out, L.out_type, t * L.out_stride + k, x);
        }
    }
}

// A workgroup per token: the first of its kind sums all of them.
__global__ void __launch_bounds__(kThreads) k_grad(EmbeddingGradLaunch L)
{
    for (int64_t t = blockIdx.x; t < L.t.num; t += gridDim.x) {
        bool outside, other;
        const int64_t row = token_row(L.t, t, &outside);
        if (outside && threadIdx.x == 0) atomicOr(L.t.status, QADAM_STATUS_TOKEN_RANGE);
        if (row < 0) continue;
        bool first = true;
        for (int64_t u = 0; first && u < t; ++u) first = token_row(L.t, u, &other) != row;
        if (!first) continue;
        for (int k = threadIdx.x; k < L.dim; k += kThreads) {
            float sum = 0.0f;
            for (int64_t u = t; u < L.t.num; ++u)
                if (token_row(L.t, u, &other) == row) sum += load_one(L.dout, L.dout_type, u * L.dout_stride + k);
            const int64_t at = row * L.grad_stride + k;
            const float x = sum * L.scale;
            store_one(L.grad, L.grad_type, at, L.accumulate ? load_one(L.grad, L.grad_type, at) + x : x);
        }
    }
}

__global__ void __launch_bounds__(kThreads) k_zero_rows(EmbeddingGradLaunch L)
{
    for (int64_t r = blockIdx.x; r < L.t.rows; r += gridDim.x)
        for (int k = threadIdx.x; k < L.dim; k += kThreads) store_one(L.grad, L.grad_type, r * L.grad_stride + k, 0.0f);
}

int groups(int64_t n) { return (int)(n < 65536 ? n : 65536); }

}  // namespace

hipError_t launch_embedding_lookup(const LookupLaunch& L)
{
    hipLaunchKernelGGL(k_lookup, dim3(groups(L.t.num)), dim3(kThreads), 0, L.stream, L);
    return hipGetLastError();
}

hipError_t launch_embedding_grad(const EmbeddingGradLaunch& L)
{
    if (!L.accumulate) {
        hipLaunchKernelGGL(k_zero_rows, dim3(groups(L.t.rows)), dim3(kThreads), 0, L.stream, L);
        if (const hipError_t e = hipGetLastError()) return e;
    }
    if (L.t.num > 0) hipLaunchKernelGGL(k_grad, dim3(groups(L.t.num)), dim3(kThreads), 0, L.stream, L);
    return hipGetLastError();
}

}  // namespace qadam
