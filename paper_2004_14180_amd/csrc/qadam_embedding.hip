// gfx950 kernels of the embedding: lookup with scaling, and the gradient by sorted tokens.
#include "qadam_elements.h"
#include "qadam_operators.h"

namespace qadam {
namespace {

constexpr int kThreads = 256;

// the row of token t, or -1 (padding, out of range)
__device__ __forceinline__ int64_t token_row(const TokenList& L, int64_t t, bool* out_of_range)
{
    const int64_t tok = L.bytes == 4 ? global(static_cast<const int32_t*>(L.tokens))[t] : global(static_cast<const int64_t*>(L.tokens))[t];
    *out_of_range = tok < 0 || tok >= L.rows;
    return *out_of_range || tok == L.padding ? -1 : tok;
}

// Lookup: 1 << log_lanes lanes per row take runs of 8 elements, a lane of ROWS rows at a time, whose loads are under way together.
constexpr int kRun = 8;

template <int WT, int OT, int ROWS>
__device__ __forceinline__ void lookup_rows(const LookupLaunch& L, int log_lanes)
{
    typedef typename Element<WT>::T W;
    typedef typename Element<OT>::T O;
    const int lanes = 1 << log_lanes, lane = threadIdx.x & (lanes - 1), groups = kThreads >> log_lanes;
    const int64_t t0 = (int64_t)blockIdx.x * (groups * ROWS) + (threadIdx.x >> log_lanes);
    int64_t row[ROWS];
#pragma unroll
    for (int r = 0; r < ROWS; ++r) {
        const int64_t t = t0 + r * groups;
        bool outside = false;
        row[r] = t < L.t.num ? token_row(L.t, t, &outside) : -1;
        if (outside && lane == 0) atomicOr(L.t.status, QADAM_STATUS_TOKEN_RANGE);
    }
    for (int at = lane * kRun; at < L.dim; at += lanes * kRun) {
        const bool whole = at + kRun <= L.dim;
        typename Run<WT, kRun>::V v[ROWS];
#pragma unroll
        for (int r = 0; r < ROWS; ++r) {
            const W* p = static_cast<const W*>(L.weight) + row[r] * L.weight_stride + at;
            if (row[r] < 0) v[r] = (W)0;
            else if (whole) v[r] = load_raw<WT, kRun, false>(p);
            else
                for (int k = 0; k < kRun; ++k) v[r][k] = at + k < L.dim ? global(p)[k] : (W)0;
        }
#pragma unroll
        for (int r = 0; r < ROWS; ++r) {
            const int64_t t = t0 + r * groups;
            if (t >= L.t.num) continue;
            // zero, whatever the scale
            const auto x = row[r] < 0 ? (typename Run<WT, kRun>::F)0.0f : to_float<WT, kRun>(v[r]) * L.scale;
            O* p = static_cast<O*>(L.out) + t * L.out_stride + at;
            if (whole) store_run<OT, kRun, false>(p, x);
            else
                for (int k = 0; k < kRun; ++k)
                    if (at + k < L.dim) global(p)[k] = (O)x[k];
        }
    }
}

template <int WT, int ROWS>
__global__ void __launch_bounds__(kThreads) k_lookup(LookupLaunch L, int log_lanes)
{
    if (L.out_type == QADAM_F32) lookup_rows<WT, QADAM_F32, ROWS>(L, log_lanes);
    else if (L.out_type == QADAM_BF16) lookup_rows<WT, QADAM_BF16, ROWS>(L, log_lanes);
    else lookup_rows<WT, QADAM_F16, ROWS>(L, log_lanes);
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

template <int WT>
static hipError_t lookup_of(const LookupLaunch& L)
{
    int log_lanes = 0;
    while ((1 << log_lanes) < kThreads && (1 << log_lanes) * kRun < L.dim) ++log_lanes;
    const int groups = kThreads >> log_lanes;
    // four rows per lane where that leaves every CU work
    constexpr int kMany = 4;
    const int64_t many = (L.t.num + groups * kMany - 1) / (groups * kMany), one = (L.t.num + groups - 1) / groups;
    if (many >= 1024) hipLaunchKernelGGL((k_lookup<WT, kMany>), dim3((unsigned)many), dim3(kThreads), 0, L.stream, L, log_lanes);
    else hipLaunchKernelGGL((k_lookup<WT, 1>), dim3((unsigned)one), dim3(kThreads), 0, L.stream, L, log_lanes);
    return hipGetLastError();
}

hipError_t launch_embedding_lookup(const LookupLaunch& all)
{
    // workgroups times threads of a launch stay below 2^32: parts of at most 2^24 tokens
    constexpr int64_t kPart = (int64_t)1 << 24;
    for (int64_t at = 0; at < all.t.num; at += kPart) {
        LookupLaunch L = all;
        L.t.tokens = static_cast<const char*>(all.t.tokens) + at * all.t.bytes;
        L.t.num = all.t.num - at < kPart ? all.t.num - at : kPart;
        L.out = static_cast<char*>(all.out) + at * all.out_stride * element_size(all.out_type);
        hipError_t e = hipErrorInvalidValue;
        switch (L.weight_type) {
        case QADAM_F32: e = lookup_of<QADAM_F32>(L); break;
        case QADAM_BF16: e = lookup_of<QADAM_BF16>(L); break;
        case QADAM_F16: e = lookup_of<QADAM_F16>(L); break;
        case QADAM_CODES8: e = lookup_of<QADAM_CODES8>(L); break;
        case QADAM_CODES16: e = lookup_of<QADAM_CODES16>(L); break;
        }
        if (e != hipSuccess) return e;
    }
    return hipSuccess;
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
