// gfx950 kernels of the product of tokens with a matrix of 8-bit integers.
#include "qadam_layers.h"
#include "qadam_row.h"

namespace qadam {
namespace {

typedef int i4 __attribute__((ext_vector_type(4)));
typedef int i16 __attribute__((ext_vector_type(16)));
typedef i4 i4u __attribute__((aligned(1)));

// ---- tokens to integers ---------------------------------------------------------------------------
constexpr int kThreads = 256;

// a = max |x|, as the bits of |x|: NaN is the largest of all
struct TokenScale {
    float inverse, scale;
    __device__ __forceinline__ explicit TokenScale(uint32_t bits)
    {
        const float a = __builtin_bit_cast(float, bits);
        const bool finite = bits < 0x7f800000u, zero = a < 0x1p-116f;
        inverse = !finite || zero ? 0.0f : (1.0f / a) * 127.0f;
        scale = !finite ? __builtin_nanf("") : zero ? 0.0f : a * (1.0f / 127.0f);
    }
    __device__ __forceinline__ int code(float x) const { return inverse == 0.0f ? 0 : (int)rintf(x * inverse); }
};

// One workgroup per token, which reads it twice; codes up to `padded` are written, zeros from `inputs` on.
__global__ void __launch_bounds__(kThreads) k_tokens(TokensLaunch L)
{
    __shared__ uint32_t most[kThreads / 64];
    for (int64_t t = blockIdx.x; t < L.tokens; t += gridDim.x) {
        int8_t* to = L.codes + t * L.codes_stride;
        if (L.x_type == QADAM_CODES8) {
            const int8_t* from = static_cast<const int8_t*>(L.x) + t * L.x_stride;
            for (int at = threadIdx.x; at < L.padded; at += kThreads) global(to)[at] = at < L.inputs ? global(from)[at] : 0;
            continue;
        }
        uint32_t m = 0;
        for (int at = threadIdx.x; at < L.inputs; at += kThreads) {
            const uint32_t bits = __builtin_bit_cast(uint32_t, load_one(L.x, L.x_type, t * L.x_stride + at)) & 0x7fffffffu;
            m = m > bits ? m : bits;
        }
        for (int k = 32; k > 0; k /= 2) {
            const uint32_t other = (uint32_t)__shfl_xor((int)m, k);
            m = m > other ? m : other;
        }
        __syncthreads();
        if (threadIdx.x % 64 == 0) most[threadIdx.x / 64] = m;
        __syncthreads();
        for (int w = 0; w < kThreads / 64; ++w) m = m > most[w] ? m : most[w];
        const TokenScale s(m);
        for (int at = threadIdx.x; at < L.padded; at += kThreads)
            global(to)[at] = at < L.inputs ? (int8_t)s.code(load_one(L.x, L.x_type, t * L.x_stride + at)) : 0;
        if (threadIdx.x == 0) global(L.scales)[t] = s.scale;
    }
}

// ---- the product ----------------------------------------------------------------------------------
constexpr int kTile = 128, kStep = 64, kPitch = kStep + 16;

// 16 integers of row n of the weights from k on, zeros from `inputs` on; nothing behind the matrix's last element is read
__device__ __forceinline__ i4 load_weights(const ProductLaunch& L, int64_t n, int k)
{
    if (n >= L.outputs || k >= L.inputs) return 0;
    const int8_t* p = L.weight + n * L.weight_stride + k;
    const int left = L.inputs - k;
    if (left >= 16) return *(const QADAM_GLOBAL i4u*)p;
    uint32_t w[4] = {};
#pragma unroll
    for (int i = 0; i < 15; ++i)
        if (i < left) w[i / 4] |= (uint32_t)(uint8_t)global(p)[i] << 8 * (i % 4);
    return {(int)w[0], (int)w[1], (int)w[2], (int)w[3]};
}

__device__ __forceinline__ void store_out(const ProductLaunch& L, int64_t t, int64_t n, int sum, float token_scale)
{
    float y = (float)sum * token_scale;
    y *= L.weight_scales ? global(L.weight_scales)[n] : L.code_scale;
    if (L.bias) y += load_one(L.bias, L.bias_type, n);
    const int64_t at = t * L.out_stride + n;
    if (L.out_type == QADAM_F32) global(static_cast<float*>(L.out))[at] = y;
    else if (L.out_type == QADAM_BF16) global(static_cast<__bf16*>(L.out))[at] = (__bf16)y;
    else global(static_cast<_Float16*>(L.out))[at] = (_Float16)y;
}

__global__ void __launch_bounds__(kThreads) k_product(ProductLaunch L, int64_t first)
{
    __shared__ __attribute__((aligned(16))) int8_t a_tile[kTile * kPitch], b_tile[kTile * kPitch];
    const int lane = threadIdx.x % 64, wave = threadIdx.x / 64;
    const int64_t across = (L.outputs + kTile - 1) / kTile, n0 = blockIdx.x % across * kTile, t0 = first + blockIdx.x / across * kTile;
    const int m0 = wave / 2 * 64, c0 = wave % 2 * 64;
    i16 acc[2][2];
    for (auto& r : acc)
        for (auto& c : r) c = 0;
    for (int k0 = 0; k0 < L.inputs; k0 += kStep) {
        __syncthreads();
        for (int i = threadIdx.x; i < kTile * (kStep / 16); i += kThreads) {
            const int row = i / (kStep / 16), k = i % (kStep / 16) * 16;
            i4 v = 0;
            if (t0 + row < L.tokens) v = *(const QADAM_GLOBAL i4*)(L.codes + (t0 + row) * L.codes_stride + k0 + k);
            *(i4*)(a_tile + row * kPitch + k) = v;
            *(i4*)(b_tile + row * kPitch + k) = load_weights(L, n0 + row, k0 + k);
        }
        __syncthreads();
#pragma unroll
        for (int k = 0; k < kStep; k += 32) {
            i4 a[2], b[2];
#pragma unroll
            for (int i = 0; i < 2; ++i) {
                a[i] = *(const i4*)(a_tile + (m0 + i * 32 + lane % 32) * kPitch + k + lane / 32 * 16);
                b[i] = *(const i4*)(b_tile + (c0 + i * 32 + lane % 32) * kPitch + k + lane / 32 * 16);
            }
#pragma unroll
            for (int i = 0; i < 2; ++i)
#pragma unroll
                for (int j = 0; j < 2; ++j) acc[i][j] = __builtin_amdgcn_mfma_i32_32x32x32_i8(a[i], b[j], acc[i][j], 0, 0, 0);
        }
    }
#pragma unroll
    for (int i = 0; i < 2; ++i)
#pragma unroll
        for (int j = 0; j < 2; ++j) {
            const int64_t n = n0 + c0 + j * 32 + lane % 32;
            if (n >= L.outputs) continue;
#pragma unroll
            for (int r = 0; r < 16; ++r) {
                const int64_t t = t0 + m0 + i * 32 + r % 4 + 8 * (r / 4) + 4 * (lane / 32);
                if (t < L.tokens) store_out(L, t, n, acc[i][j][r], global(L.token_scales)[t]);
            }
        }
}

}  // namespace

hipError_t launch_tokens(const TokensLaunch& L)
{
    k_tokens<<<dim3((int)(L.tokens < 4096 ? L.tokens : 4096)), dim3(kThreads), 0, L.stream>>>(L);
    return hipGetLastError();
}

hipError_t launch_product(const ProductLaunch& L)
{
    // tiles of a launch: fewer than 2^32 work-items
    const int64_t across = (L.outputs + kTile - 1) / kTile, most = ((int64_t)1 << 22) / across;
    for (int64_t t = 0; t < L.tokens; t += most * kTile) {
        const int64_t down = (L.tokens - t + kTile - 1) / kTile;
        k_product<<<dim3((int)(across * (down < most ? down : most))), dim3(kThreads), 0, L.stream>>>(L, t);
    }
    return hipGetLastError();
}

}  // namespace qadam
