// gfx950 kernels on lists of tensors: AdamW with decoupled weight decay and states in 32 or 8 bits, and the norm of all gradients.
#include "qadam_elements.h"
#include "qadam_operators.h"

namespace qadam {
namespace {

constexpr int kWave = 64;
constexpr int kBlock = QADAM_STATE_BLOCK;       // a wavefront's 64 lanes of 4 elements
constexpr int kBlocks = 4;                      // blocks of a wavefront
constexpr int kWaveElems = kBlock * kBlocks;
constexpr int kWavesPerTile = kListTile / kWaveElems;
static_assert(kBlock == 4 * kWave, "");

constexpr float kFp8Max = 448.0f, kFp8Least = 0x1p-9f, kTinyBlock = 0x1p-116f;

// the largest of a wavefront's values, none of them negative, in every lane
__device__ __forceinline__ float wave_max(float x)
{
    for (int d = 1; d < kWave; d <<= 1) {
        const float y = __shfl_xor(x, d);
        x = __float_as_uint(y) > __float_as_uint(x) ? y : x;        // a NaN sorts above every number
    }
    return x;
}

// four values x (quotient of the block's scale) as four 8-bit floats
__device__ __forceinline__ uint32_t to_fp8(f4 x)
{
    int r = __builtin_amdgcn_cvt_pk_fp8_f32(x[0], x[1], 0, false);
    return (uint32_t)__builtin_amdgcn_cvt_pk_fp8_f32(x[2], x[3], r, true);
}

__device__ __forceinline__ f4 from_fp8(uint32_t c)
{
    const auto lo = __builtin_amdgcn_cvt_pk_f32_fp8((int)c, false), hi = __builtin_amdgcn_cvt_pk_f32_fp8((int)c, true);
    return f4{lo[0], lo[1], hi[0], hi[1]};
}

struct Moments {
    f4 m, v;
};

// x, m, v of four elements after the step; `r`: sqrt(v)
__device__ __forceinline__ void adamw(const AdamwScalars& S, float lr_decay, float factor, f4 grad, f4& x, f4& m, f4& v, f4& r)
{
#pragma unroll
    for (int k = 0; k < 4; ++k) {
        const float g = grad[k] * factor;
        m[k] = m[k] * S.beta1 + g * S.omb1;
        v[k] = v[k] * S.beta2 + (g * g) * S.omb2;
        r[k] = sqrtf(v[k]);
        x[k] = x[k] - x[k] * lr_decay;
        x[k] = x[k] - (m[k] * S.lr1) / (r[k] * S.inv_sbc2 + S.eps);
    }
}

// the scale of a block whose largest magnitude is `big`, and what its values are multiplied with
__device__ __forceinline__ float block_scale(float big, float* inv)
{
    if (big < kTinyBlock) big = 0.0f;
    *inv = big > 0.0f ? kFp8Max / big : 0.0f;
    return big / kFp8Max;
}

__device__ __forceinline__ float largest(f4 a)
{
    const float b = fmaxf(fabsf(a[0]), fabsf(a[1])), c = fmaxf(fabsf(a[2]), fabsf(a[3]));
    return fmaxf(b, c);
}

// One wavefront's block `block` of the tensor: elements that the lane does not have count as zeros.
template <bool STATE8>
__device__ void ragged_block(const AdamwScalars& S, const ListTensor& T, const void* grad, float lr_decay, float factor, int64_t block,
                             int lane)
{
    const int64_t first = block * kBlock + lane * 4;
    const int pt = T.types & 3, gt = T.types >> 2 & 3, ct = T.types >> 4;
    const int n = T.numel - first < 0 ? 0 : T.numel - first < 4 ? (int)(T.numel - first) : 4;
    f4 g = 0.0f, x = 0.0f, m = 0.0f, v = 0.0f, r;
    float sm = 0.0f, sv = 0.0f;
    if (STATE8) { sm = T.m_scales[block]; sv = T.v_scales[block]; }
    for (int k = 0; k < n; ++k) {
        g[k] = load_one(grad, gt, first + k);
        x[k] = load_one(T.param, pt, first + k);
        if (STATE8) {
            m[k] = __builtin_amdgcn_cvt_f32_fp8(static_cast<const uint8_t*>(T.m)[first + k], 0) * sm;
            v[k] = __builtin_amdgcn_cvt_f32_fp8(static_cast<const uint8_t*>(T.v)[first + k], 0) * sv;
        } else {
            m[k] = static_cast<const float*>(T.m)[first + k];
            v[k] = static_cast<const float*>(T.v)[first + k];
        }
    }
    if (STATE8) v = v * v;
    adamw(S, lr_decay, factor, g, x, m, v, r);
    uint32_t cm = 0, cv = 0;
    if (STATE8) {
        for (int k = n; k < 4; ++k) m[k] = r[k] = 0.0f;     // a factor that is zero times infinity
        float im, iv;
        const float nm = block_scale(wave_max(largest(m)), &im), nv = block_scale(wave_max(largest(r)), &iv);
        f4 qm = m * im, qv = r * iv;
        for (int k = 0; k < 4; ++k)
            if (r[k] > 0.0f && iv > 0.0f) qv[k] = fmaxf(qv[k], kFp8Least);
        cm = to_fp8(qm);
        cv = to_fp8(qv);
        if (lane == 0) { T.m_scales[block] = nm; T.v_scales[block] = nv; }
    }
    for (int k = 0; k < n; ++k) {
        store_one(T.param, pt, first + k, x[k]);
        if (ct != kNoCopy) store_one(T.copy, ct, first + k, x[k]);
        if (STATE8) {
            static_cast<uint8_t*>(T.m)[first + k] = (uint8_t)(cm >> 8 * k);
            static_cast<uint8_t*>(T.v)[first + k] = (uint8_t)(cv >> 8 * k);
        } else {
            static_cast<float*>(T.m)[first + k] = m[k];
            static_cast<float*>(T.v)[first + k] = v[k];
        }
    }
}

// A wavefront takes four blocks of one tensor, a workgroup a tile of four wavefronts.
template <bool STATE8>
__global__ void __launch_bounds__(kWave * kWavesPerTile)
k_adamw(const ListTile* __restrict__ tiles, const ListTensor* __restrict__ tensors, int first_tensor, AdamwScalars S,
        const float* __restrict__ grad_factor, GradTable G)
{
    const ListTile tile = tiles[blockIdx.x];
    const void* grad = G.grad[tile.tensor - first_tensor];
    if (!grad) return;
    const float factor = grad_factor ? *grad_factor : 1.0f;
    if (!(fabsf(factor) < INFINITY)) return;
    const ListTensor T = tensors[tile.tensor];
    const int lane = threadIdx.x % kWave, wave = __builtin_amdgcn_readfirstlane(threadIdx.x / kWave);
    const float lr_decay = S.lr * T.weight_decay;
    const int64_t block = (int64_t)tile.tile * (kListTile / kBlock) + wave * kBlocks;
    for (int b = 0; b < kBlocks; ++b)
        if ((block + b) * kBlock < T.numel) ragged_block<STATE8>(S, T, grad, lr_decay, factor, block + b, lane);
}

// Sum of the squares of the gradients: a workgroup takes every gridDim.x-th tile; the last one to arrive adds the sums of all.
constexpr int kNormThreads = 256;

__device__ __forceinline__ double group_sum(double x, double* shared)
{
    for (int d = 1; d < kWave; d <<= 1) x += __shfl_xor(x, d);
    if (threadIdx.x % kWave == 0) shared[threadIdx.x / kWave] = x;
    __syncthreads();
    x = 0.0;
    for (int w = 0; w < kNormThreads / kWave; ++w) x += shared[w];
    __syncthreads();
    return x;
}

__global__ void __launch_bounds__(kNormThreads)
k_grad_norm(const ListTile* __restrict__ tiles, const ListTensor* __restrict__ tensors, int num_tiles, int first_tensor, NormLaunch N,
            GradTable G)
{
    __shared__ double shared[kNormThreads / kWave];
    __shared__ bool last;
    double sum = 0.0;
    for (int i = blockIdx.x; i < num_tiles; i += gridDim.x) {
        const ListTile tile = tiles[i];
        const void* grad = G.grad[tile.tensor - first_tensor];
        if (!grad) continue;
        const int64_t first = (int64_t)tile.tile * kListTile, numel = tensors[tile.tensor].numel;
        const int type = tensors[tile.tensor].types >> 2 & 3;
        const int n = numel - first < kListTile ? (int)(numel - first) : kListTile;
        for (int k = threadIdx.x; k < n; k += kNormThreads) {
            const double g = load_one(grad, type, first + k);
            sum += g * g;
        }
    }
    sum = group_sum(sum, shared);
    if (threadIdx.x == 0)
        __hip_atomic_store(&N.sums[N.first_sum + blockIdx.x], sum, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
    if (N.total == 0) return;           // a later launch finishes
    if (threadIdx.x == 0)
        last = __hip_atomic_fetch_add(N.arrived, 1u, __ATOMIC_ACQ_REL, __HIP_MEMORY_SCOPE_AGENT) == gridDim.x - 1;
    __syncthreads();
    if (!last) return;
    sum = 0.0;
    for (int i = threadIdx.x; i < N.total; i += kNormThreads)
        sum += __hip_atomic_load(&N.sums[i], __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
    sum = group_sum(sum, shared);
    if (threadIdx.x == 0) {
        __hip_atomic_store(N.arrived, 0u, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
        const double norm = sqrt(sum);
        N.out[0] = (float)norm;
        N.out[1] = !(norm < (double)INFINITY) ? NAN : norm > (double)N.max_norm ? (float)((double)N.max_norm / norm) : 1.0f;
    }
}

}  // namespace

hipError_t launch_adamw(const ListLaunch& L, const AdamwScalars& S, const GradTable& G, const float* grad_factor, bool state8)
{
    const dim3 grid(L.num_tiles), block(kWave * kWavesPerTile);
    if (state8)
        hipLaunchKernelGGL(k_adamw<true>, grid, block, 0, L.stream, L.tiles + L.first_tile, L.tensors, L.first_tensor, S, grad_factor, G);
    else
        hipLaunchKernelGGL(k_adamw<false>, grid, block, 0, L.stream, L.tiles + L.first_tile, L.tensors, L.first_tensor, S, grad_factor, G);
    return hipGetLastError();
}

hipError_t launch_grad_norm(const ListLaunch& L, const NormLaunch& N, const GradTable& G)
{
    hipLaunchKernelGGL(k_grad_norm, dim3(norm_groups(L.num_tiles)), dim3(kNormThreads), 0, L.stream, L.tiles + L.first_tile, L.tensors,
                       L.num_tiles, L.first_tensor, N, G);
    return hipGetLastError();
}

}  // namespace qadam
