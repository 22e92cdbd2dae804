// gfx950 kernels on lists of tensors: AdamW with decoupled weight decay and states in 32 or 8 bits, and the norm of all gradients.
//
// Both are one pass over memory and bound by it: AdamW moves 24 bytes per element with 32-bit states (weights, m and v read and written)
// or 12 + 16 / 256 with 8-bit ones, and the gradient; the norm reads the gradient.  The arithmetic, about 50 vector instructions per
// element with the division, the root and the 8-bit floats, takes half of the time that the bytes take.  What counts is that no access
// is ragged and that enough of them are under way:
//   * a workgroup is one wavefront and takes one block of 256 elements, 4 per lane: 16-byte accesses of fp32, 8 of 16 bits, 4 of 8.
//     The wavefronts drift apart and so mix their reads and writes.  us per step of 124 M elements with bf16 gradients / of 1.3 G with
//     8-bit states, with 1, 2, 4 blocks per wavefront: 567 / 580 / 574 and 3490 / 3640 / 3510;
//   * the list is a table of tiles on the device, so one launch serves 448 tensors, whose gradients' addresses are kernel arguments;
//   * element types are known at compile time behind one uniform branch; the last block of a tensor takes the same code with
//     neighbouring elements repeated, all loads still under way together (a loop over elements: 51 k elements 9.3 us, now 5.2);
//   * a block of the 8-bit states is a wavefront's block, so its two scales are maxima over lanes, by DPP, with no LDS.
// GPT-2 small's list (124 M, bf16 gradients and copy) 573 to 588 us by box, 5.9 to 6.1 TB/s; GPT-1.3B's with 8-bit states 3490 us, 6.05 TB/s;
// 124 M bf16 weights with states in 32 bits 429 us, in 8 bits 198 us, both 6.3 TB/s; the norm of 1.3 G bf16 390 us, 6.75 TB/s.  torch's
// addition in place reaches 5.9 TB/s here, this library's streams in place 6.0 to 6.3.
#include "qadam_elements.h"
#include "qadam_operators.h"

namespace qadam {
namespace {

constexpr int kWave = 64;
constexpr int kBlock = QADAM_STATE_BLOCK;       // a wavefront's 64 lanes of 4 elements
constexpr int kBlocksPerTile = kTileBlocks;
static_assert(kBlock == 4 * kWave && kBlocksPerTile * kBlock == kListTile, "");

constexpr float kFp8Max = 448.0f, kFp8Unit = 1.0f / 448.0f, kFp8Least = 0x1p-9f, kTinyBlock = 0x1p-116f;

// the largest of a wavefront's numbers, in every lane: within rows of 16 lanes, then from row to row, by DPP
template <int CTRL>
__device__ __forceinline__ uint32_t dpp_max(uint32_t x)
{
    const uint32_t y = (uint32_t)__builtin_amdgcn_update_dpp(0, (int)x, CTRL, 0xf, 0xf, false);     // 0 from where there is no lane
    return y > x ? y : x;
}

__device__ __forceinline__ float wave_max(uint32_t x)
{
    x = dpp_max<0x111>(x);      // one lane to the right, two, four, eight
    x = dpp_max<0x112>(x);
    x = dpp_max<0x114>(x);
    x = dpp_max<0x118>(x);
    x = dpp_max<0x142>(x);      // the row's last lane to the next row
    x = dpp_max<0x143>(x);      // lane 31 to the upper half
    return __uint_as_float((uint32_t)__builtin_amdgcn_readlane((int)x, kWave - 1));
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

typedef uint32_t word_u __attribute__((aligned(1)));
__device__ __forceinline__ uint32_t load_word(const uint8_t* p) { return __builtin_nontemporal_load((const QADAM_GLOBAL word_u*)p); }
__device__ __forceinline__ void store_word(uint8_t* p, uint32_t x) { __builtin_nontemporal_store(x, (QADAM_GLOBAL word_u*)p); }

// x, m, v of four elements after the step, `r` = sqrt(v): one rounding per operation in the order of the header, so that the step is
// the same bits as those operations one by one, whatever the layout.
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
    *inv = big > 0.0f ? kFp8Max * (1.0f / big) : 0.0f;
    return big * kFp8Unit;
}

// The largest magnitude, as bits: they order like the values, and a NaN is above every number, where a maximum of floats drops it.
__device__ __forceinline__ uint32_t largest(f4 a)
{
    uint32_t x = 0;
#pragma unroll
    for (int k = 0; k < 4; ++k) {
        const uint32_t y = __float_as_uint(fabsf(a[k]));
        x = y > x ? y : x;
    }
    return x;
}

// Of a ragged block a lane has the elements in [low, end); the others repeat the nearest one and are not stored.
__device__ __forceinline__ int nearest(int i, int low, int end) { return i < low ? low : i < end ? i : end - 1; }

// four elements at p + at
template <int TYPE, bool WHOLE>
__device__ __forceinline__ typename Run<TYPE, 4>::V load_four(const void* p, int at, int low, int end)
{
    const auto* q = static_cast<const typename Element<TYPE>::T*>(p);
    if constexpr (WHOLE) return load_raw<TYPE, 4>(q + at);
    typename Run<TYPE, 4>::V v;
#pragma unroll
    for (int k = 0; k < 4; ++k) v[k] = global(q)[nearest(at + k, low, end)];
    return v;
}

template <int TYPE, bool WHOLE>
__device__ __forceinline__ void store_four(void* p, int at, int low, int end, f4 x)
{
    auto* q = static_cast<typename Element<TYPE>::T*>(p);
    if constexpr (WHOLE) {
        store_run<TYPE, 4>(q + at, x);
    } else {
#pragma unroll
        for (int k = 0; k < 4; ++k)
            if (at + k >= low && at + k < end) global(q)[at + k] = (typename Element<TYPE>::T)x[k];
    }
}

// the same of bytes
template <bool WHOLE>
__device__ __forceinline__ uint32_t load_bytes(const void* p, int at, int end)
{
    const uint8_t* q = static_cast<const uint8_t*>(p);
    if constexpr (WHOLE) return load_word(q + at);
    uint32_t w = 0;
#pragma unroll
    for (int k = 0; k < 4; ++k) w |= (uint32_t)global(q)[at + k < end ? at + k : end - 1] << 8 * k;
    return w;
}

template <bool WHOLE>
__device__ __forceinline__ void store_bytes(void* p, int at, int end, uint32_t w)
{
    uint8_t* q = static_cast<uint8_t*>(p);
    if constexpr (WHOLE) {
        store_word(q + at, w);
    } else {
#pragma unroll
        for (int k = 0; k < 4; ++k)
            if (at + k < end) global(q)[at + k] = (uint8_t)(w >> 8 * k);
    }
}

// A block of a tensor, types known.  WHOLE: the tensor has all of it.
template <bool STATE8, int PT, int GT, int CT, bool WHOLE>
__device__ __forceinline__ void step_block(const AdamwScalars& S, const ListTensor& T, const void* grad, float lr_decay, float factor,
                                           int64_t first, int lane)
{
    const int64_t left = T.numel - first;
    const int at = lane * 4, low = first < 0 ? (int)-first : 0, end = left < kBlock ? (int)left : kBlock;
    const void* gp = static_cast<const typename Element<GT>::T*>(grad) + first;
    void* xp = static_cast<typename Element<PT>::T*>(T.param) + first;
    const auto grad4 = load_four<GT, WHOLE>(gp, at, low, end);
    const auto param4 = load_four<PT, WHOLE>(xp, at, low, end);
    f4 m, v, r;
    void *mp, *vp;
    int64_t block = 0;
    if constexpr (STATE8) {
        mp = static_cast<uint8_t*>(T.m) + first;
        vp = static_cast<uint8_t*>(T.v) + first;
        block = first / kBlock;
        const uint32_t cm = load_bytes<WHOLE>(mp, at, end), cv = load_bytes<WHOLE>(vp, at, end);
        const float sm = global(T.m_scales)[block], sv = global(T.v_scales)[block];
        m = from_fp8(cm) * sm;
        v = from_fp8(cv) * sv;
        v = v * v;
    } else {
        mp = static_cast<float*>(T.m) + first;
        vp = static_cast<float*>(T.v) + first;
        m = load_four<QADAM_F32, WHOLE>(mp, at, low, end);
        v = load_four<QADAM_F32, WHOLE>(vp, at, low, end);
    }
    f4 x = to_float<PT, 4>(param4);
    adamw(S, lr_decay, factor, to_float<GT, 4>(grad4), x, m, v, r);
    store_four<PT, WHOLE>(xp, at, low, end, x);
    if constexpr (CT != kNoCopy) store_four<CT, WHOLE>(static_cast<typename Element<CT>::T*>(T.copy) + first, at, low, end, x);
    if constexpr (STATE8) {
        if constexpr (!WHOLE)
#pragma unroll
            for (int k = 0; k < 4; ++k)
                if (at + k >= end) m[k] = r[k] = 0.0f;
        float im, iv;
        const float nm = block_scale(wave_max(largest(m)), &im), nv = block_scale(wave_max(largest(r)), &iv);
        f4 q = r * iv;
        const float least = nv > 0.0f ? kFp8Least : 0.0f;       // (not where the block is kept as zeros or holds a NaN; a NaN stays one)
#pragma unroll
        for (int k = 0; k < 4; ++k) q[k] = r[k] > 0.0f && q[k] < least ? least : q[k];
        store_bytes<WHOLE>(mp, at, end, to_fp8(m * im));
        store_bytes<WHOLE>(vp, at, end, to_fp8(q));
        if (lane == 0) {
            global(T.m_scales)[block] = nm;
            global(T.v_scales)[block] = nv;
        }
    } else {
        store_four<QADAM_F32, WHOLE>(mp, at, low, end, m);
        store_four<QADAM_F32, WHOLE>(vp, at, low, end, v);
    }
}

template <bool STATE8, bool WHOLE>
__device__ __forceinline__ void step_block(const AdamwScalars& S, const ListTensor& T, const void* grad, float lr_decay, float factor,
                                           int64_t first, int lane)
{
#define QADAM_CASE(P, G, CP) \
    case list_types(P, G, CP): step_block<STATE8, P, G, CP, WHOLE>(S, T, grad, lr_decay, factor, first, lane); break;
#define QADAM_CASES(P, CP) QADAM_CASE(P, QADAM_F32, CP) QADAM_CASE(P, QADAM_BF16, CP) QADAM_CASE(P, QADAM_F16, CP)
    switch (T.types & ((1 << kTypeBits) - 1)) {
        QADAM_CASES(QADAM_F32, kNoCopy)
        QADAM_CASES(QADAM_F32, QADAM_BF16)
        QADAM_CASES(QADAM_F32, QADAM_F16)
        QADAM_CASES(QADAM_BF16, kNoCopy)
        QADAM_CASES(QADAM_F16, kNoCopy)
    }
#undef QADAM_CASES
#undef QADAM_CASE
}

template <bool STATE8>
__global__ void __launch_bounds__(kWave)
k_adamw(const ListTile* __restrict__ tiles, const ListTensor* __restrict__ tensors, int first_tensor, AdamwScalars S,
        const float* __restrict__ grad_factor, GradTable G)
{
    const ListTile tile = tiles[blockIdx.x / kBlocksPerTile];
    const void* grad = G.grad[tile.tensor - first_tensor];
    if (!grad) return;
    const float factor = grad_factor ? *grad_factor : 1.0f;
    if (!(fabsf(factor) < INFINITY)) return;
    const ListTensor T = tensors[tile.tensor];
    const int lane = threadIdx.x;
    const float lr_decay = S.lr * T.weight_decay;
    const int64_t block = (int64_t)tile.tile * kBlocksPerTile + blockIdx.x % kBlocksPerTile;
    const int64_t first = block * kBlock - (STATE8 ? 0 : T.types >> kTypeBits);
    if (first >= 0 && first + kBlock <= T.numel) step_block<STATE8, true>(S, T, grad, lr_decay, factor, first, lane);
    else if (first < T.numel) step_block<STATE8, false>(S, T, grad, lr_decay, factor, first, lane);
}

// Sum of the squares of the gradients: a workgroup takes every gridDim.x-th tile; the last one to arrive adds the sums of all.  Squares
// and sums are fp64: exact squares, no overflow, and at the rate of this GPU they cost nothing beside the loads.
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

template <int TYPE, int N>
__device__ __forceinline__ double squares(typename Run<TYPE, N>::V v)
{
    double sum = 0.0;
#pragma unroll
    for (int k = 0; k < N; ++k) {
        const double g = (float)v[k];
        sum = fma(g, g, sum);
    }
    return sum;
}

// The squares of what a thread has of a tile: 16-byte runs from the first aligned address on, 256 runs apart, and of the up to 16 bytes
// in front of them and behind them an element per thread.
template <int TYPE>
__device__ __forceinline__ double tile_squares(const void* tile, int n)
{
    typedef typename Element<TYPE>::T T;
    constexpr int kRun = 16 / sizeof(T), kRuns = kListTile / (kRun * kNormThreads);
    const T* p = static_cast<const T*>(tile);
    const int thread = threadIdx.x, off = (int)(reinterpret_cast<uintptr_t>(p) % 16 / sizeof(T));
    const int head = off ? (kRun - off < n ? kRun - off : n) : 0;
    const T* q = p + head;
    const int runs = (n - head) / kRun, tail = n - head - runs * kRun;
    double sum = 0.0;
    if (off == 0 && n == kListTile) {
        typename Run<TYPE, kRun>::V v[kRuns];
#pragma unroll
        for (int j = 0; j < kRuns; ++j) v[j] = load_raw<TYPE, kRun>(q + (thread + j * kNormThreads) * kRun);
#pragma unroll
        for (int j = 0; j < kRuns; ++j) sum += squares<TYPE, kRun>(v[j]);
        return sum;
    }
    // (a run behind the last one is the last one again, and does not count)
    if (runs > 0) {
        typename Run<TYPE, kRun>::V v[kRuns];
#pragma unroll
        for (int j = 0; j < kRuns; ++j) {
            const int r = thread + j * kNormThreads;
            v[j] = load_raw<TYPE, kRun>(q + (r < runs ? r : runs - 1) * kRun);
        }
#pragma unroll
        for (int j = 0; j < kRuns; ++j)
            if (thread + j * kNormThreads < runs) sum += squares<TYPE, kRun>(v[j]);
    }
    if (thread < head + tail) {
        const double g = load_one(p, TYPE, thread < head ? thread : n - tail + thread - head);
        sum = fma(g, g, sum);
    }
    return sum;
}

// whether this is the last of `of` arrivals, which leaves zero
__device__ __forceinline__ bool arrive(uint32_t* count, uint32_t of)
{
    if (__hip_atomic_fetch_add(global(count), 1u, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT) != of - 1) return false;
    __hip_atomic_store(global(count), 0u, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
    return true;
}

__global__ void __launch_bounds__(kNormThreads)
k_grad_norm(const ListTile* __restrict__ tiles, int num_tiles, int first_tensor, NormLaunch N, GradTable G)
{
    __shared__ double shared[kNormThreads / kWave];
    __shared__ bool last;
    double sum = 0.0;
    ListTile next{};
    if ((int)blockIdx.x < num_tiles) next = tiles[blockIdx.x];
    for (int i = blockIdx.x; i < num_tiles; i += gridDim.x) {
        const ListTile tile = next;         // the next one's record is under way beside this one's elements
        if (i + (int)gridDim.x < num_tiles) next = tiles[i + gridDim.x];
        const void* grad = G.grad[tile.tensor - first_tensor];
        if (!grad) continue;
        const char* p = static_cast<const char*>(grad) + (int64_t)tile.tile * kListTile * element_size(tile.grad_type);
        if (tile.grad_type == QADAM_F32) sum += tile_squares<QADAM_F32>(p, tile.count);
        else if (tile.grad_type == QADAM_BF16) sum += tile_squares<QADAM_BF16>(p, tile.count);
        else sum += tile_squares<QADAM_F16>(p, tile.count);
    }
    sum = group_sum(sum, shared);
    if (threadIdx.x == 0)
        __hip_atomic_store(global(&N.sums[N.first_sum + blockIdx.x]), sum, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
    if (N.total == 0) return;           // a later launch finishes
    // The sums cross workgroups as agent-scope atomics: in memory before the arrival is counted, without a write-back of the caches
    // (12 M elements in 1024 workgroups: 42 us with one each, 21 without)
    if (threadIdx.x == 0) {
        asm volatile("s_waitcnt vmcnt(0)" ::: "memory");
        const uint32_t counts = gridDim.x < kArrivalCounts ? gridDim.x : kArrivalCounts, mine = blockIdx.x % counts;
        last = arrive(N.arrived + (mine + 1) * kArrivalStride, (gridDim.x - mine + counts - 1) / counts) && arrive(N.arrived, counts);
        asm volatile("" ::: "memory");
    }
    __syncthreads();
    if (!last) return;
    sum = 0.0;
    for (int i = threadIdx.x; i < N.total; i += kNormThreads)
        sum += __hip_atomic_load(global(&N.sums[i]), __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
    sum = group_sum(sum, shared);
    if (threadIdx.x == 0) {
        const double norm = sqrt(sum);
        N.out[0] = (float)norm;
        N.out[1] = !(norm < (double)INFINITY) ? NAN : norm > (double)N.max_norm ? (float)((double)N.max_norm / norm) : 1.0f;
    }
}

}  // namespace

hipError_t launch_adamw(const ListLaunch& L, const AdamwScalars& S, const GradTable& G, const float* grad_factor, bool state8)
{
    const dim3 grid(L.num_tiles * kBlocksPerTile), block(kWave);
    if (state8)
        hipLaunchKernelGGL(k_adamw<true>, grid, block, 0, L.stream, L.tiles + L.first_tile, L.tensors, L.first_tensor, S, grad_factor, G);
    else
        hipLaunchKernelGGL(k_adamw<false>, grid, block, 0, L.stream, L.tiles + L.first_tile, L.tensors, L.first_tensor, S, grad_factor, G);
    return hipGetLastError();
}

hipError_t launch_grad_norm(const ListLaunch& L, const NormLaunch& N, const GradTable& G)
{
    hipLaunchKernelGGL(k_grad_norm, dim3(norm_groups(L.num_tiles)), dim3(kNormThreads), 0, L.stream, L.tiles + L.first_tile,
                       L.num_tiles, L.first_tensor, N, G);
    return hipGetLastError();
}

}  // namespace qadam
