// gfx950 kernels of the product of tokens with a matrix of 8-bit integers.
//
// Sums of products of 8-bit integers are exact in 32 bits in whatever order they are taken, so that the work may be split over wavefronts
// in any way and the result stays the same bits.  Two ways, by sizes alone (Linear8Plan):
//   * few tokens (16 at most): bound by reading the weights.  They go from memory straight into the matrix instructions' registers, once, by as many
//     wavefronts as keep enough loads under way (k_product_rows);
//   * many tokens: bound by the matrix instructions and by what feeds them.  Tiles of both operands pass through LDS (k_product_tiles).
#include <type_traits>

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

__device__ __forceinline__ uint32_t larger(uint32_t a, uint32_t b) { return a > b ? a : b; }

template <int CTRL, int ROWS = 0xf>
__device__ __forceinline__ uint32_t moved_bits(uint32_t x)
{
    return (uint32_t)__builtin_amdgcn_update_dpp(0, (int)x, CTRL, ROWS, 0xf, false);
}

// Largest of a wavefront's values, the same in all lanes
__device__ __forceinline__ uint32_t wave_largest(uint32_t x)
{
    x = larger(x, moved_bits<0xb1>(x));
    x = larger(x, moved_bits<0x4e>(x));
    x = larger(x, moved_bits<0x141>(x));
    x = larger(x, moved_bits<0x140>(x));
    x = larger(x, moved_bits<0x142, 0xa>(x));
    x = larger(x, moved_bits<0x143, 0xc>(x));
    return (uint32_t)__builtin_amdgcn_readlane((int)x, 63);
}

__device__ __forceinline__ uint32_t largest_of(f8 x)
{
    typedef uint32_t u8 __attribute__((ext_vector_type(kRowRun)));
    const u8 bits = __builtin_bit_cast(u8, x) & 0x7fffffffu;       // of the whole vector: of an element it takes the first one's
    uint32_t m = 0;
#pragma unroll
    for (int i = 0; i < kRowRun; ++i) m = larger(m, bits[i]);
    return m;
}

__device__ __forceinline__ uint64_t codes_of(const TokenScale& s, f8 x)
{
    uint32_t w[2] = {};
#pragma unroll
    for (int i = 0; i < kRowRun; ++i) w[i / 4] |= (uint32_t)(s.code(x[i]) & 0xff) << 8 * (i % 4);
    return (uint64_t)w[1] << 32 | w[0];
}

// 8 integers at an address of any alignment, `n` of them
__device__ __forceinline__ void store_codes(int8_t* p, uint64_t v, int n)
{
    typedef uint64_t u8 __attribute__((aligned(1)));
    if (n >= kRowRun) {
        *(QADAM_GLOBAL u8*)p = v;
        return;
    }
#pragma unroll
    for (int i = 0; i < kRowRun - 1; ++i)
        if (i < n) global(p)[i] = (int8_t)(v >> 8 * i);
}

__device__ __forceinline__ void clear_arrived(const TokensLaunch& L)
{
    static_assert(kPartTiles == kThreads, "a counter per thread");
    if (L.arrived && blockIdx.x == 0) global(L.arrived)[threadIdx.x] = 0;
}

// A workgroup per token, and its next one under way; up to HELD * 2048 inputs stay in registers between the maximum and the integers, beyond
// that the row is read again.  Integers up to `padded` are written, zeros from `inputs` on.
template <int XT, int HELD>
__global__ void __launch_bounds__(kThreads) k_tokens(TokensLaunch L)
{
    __shared__ uint32_t most[2][kThreads / 64];
    constexpr int kAcross = kThreads * kRowRun;
    const int first = threadIdx.x * kRowRun;
    const auto* x = static_cast<const typename Element<XT>::T*>(L.x);
    typename Run<XT, kRowRun>::V next[HELD];
    auto load = [&](int64_t t) {
#pragma unroll
        for (int k = 0; k < HELD; ++k) {
            next[k] = 0;
            const int at = first + k * kAcross;
            if (at < L.inputs) next[k] = load_ahead<XT>(x + t * L.x_stride, at, L.inputs);
        }
    };
    load(blockIdx.x);
    clear_arrived(L);
    int turn = 0;
    for (int64_t t = blockIdx.x; t < L.tokens; t += gridDim.x, turn ^= 1) {
        int8_t* to = L.codes + t * L.codes_stride;
        const auto* from = x + t * L.x_stride;
        f8 held[HELD];
        uint32_t m = 0;
#pragma unroll
        for (int k = 0; k < HELD; ++k) {
            held[k] = loaded<XT>(next[k], first + k * kAcross, L.inputs);
            m = larger(m, largest_of(held[k]));
        }
        if (t + gridDim.x < L.tokens) load(t + gridDim.x);
        for (int at = first + HELD * kAcross; at < L.inputs; at += kAcross)
            m = larger(m, largest_of(loaded<XT>(load_ahead<XT>(from, at, L.inputs), at, L.inputs)));
        m = wave_largest(m);
        if (threadIdx.x % 64 == 0) most[turn][threadIdx.x / 64] = m;
        __syncthreads();
        for (int w = 0; w < kThreads / 64; ++w) m = larger(m, most[turn][w]);
        const TokenScale s(m);
#pragma unroll
        for (int k = 0; k < HELD; ++k) {
            const int at = first + k * kAcross;
            if (at < L.padded) store_codes(to + at, codes_of(s, held[k]), L.padded - at);
        }
        for (int at = first + HELD * kAcross; at < L.padded; at += kAcross) {
            f8 y = 0.0f;
            if (at < L.inputs) y = loaded<XT>(load_ahead<XT>(from, at, L.inputs), at, L.inputs);
            store_codes(to + at, codes_of(s, y), L.padded - at);
        }
        if (threadIdx.x == 0) global(L.scales)[t] = s.scale;
    }
}

// Tokens that are integers already, in rows of `padded`
__global__ void __launch_bounds__(kThreads) k_token_codes(TokensLaunch L)
{
    clear_arrived(L);
    for (int64_t t = blockIdx.x; t < L.tokens; t += gridDim.x) {
        const int8_t* from = static_cast<const int8_t*>(L.x) + t * L.x_stride;
        for (int at = threadIdx.x * kRowRun; at < L.padded; at += kThreads * kRowRun) {
            uint64_t v = 0;
            if (L.inputs - at >= kRowRun) v = __builtin_bit_cast(uint64_t, load_raw<QADAM_CODES8, kRowRun>(from + at));
            else
                for (int i = 0; i < L.inputs - at; ++i) v |= (uint64_t)(uint8_t)global(from)[at + i] << 8 * i;
            store_codes(L.codes + t * L.codes_stride + at, v, L.padded - at);
        }
    }
}

template <int XT>
void launch_tokens_of(const TokensLaunch& L, dim3 grid)
{
    if (L.inputs <= 2048) k_tokens<XT, 1><<<grid, dim3(kThreads), 0, L.stream>>>(L);
    else k_tokens<XT, 4><<<grid, dim3(kThreads), 0, L.stream>>>(L);
}

// ---- what both products share ---------------------------------------------------------------------
// 16 integers of a row of the weights from k on, zeros from `inputs` on; nothing behind the row's end is read
__device__ __forceinline__ i4 load_weights(const int8_t* row, int k, int inputs)
{
    const int left = inputs - k;
    if (left >= 16) return *(const QADAM_GLOBAL i4u*)(row + k);
    uint32_t w[4] = {};
    if (left > 0) {
#pragma unroll
        for (int i = 0; i < 15; ++i)
            if (i < left) w[i / 4] |= (uint32_t)(uint8_t)global(row)[k + i] << 8 * (i % 4);
    }
    return {(int)w[0], (int)w[1], (int)w[2], (int)w[3]};
}

__device__ __forceinline__ float output_scale(const ProductLaunch& L, int64_t n) { return L.weight_scales ? global(L.weight_scales)[n] : L.code_scale; }
__device__ __forceinline__ float output_bias(const ProductLaunch& L, int64_t n) { return L.bias ? load_one(L.bias, L.bias_type, n) : 0.0f; }

// Four outputs of a token, one rounding per operation
__device__ __forceinline__ f4 results(const ProductLaunch& L, i4 sum, float token, f4 scale, f4 bias)
{
    f4 y = __builtin_convertvector(sum, f4) * token * scale;
    if (L.bias) y += bias;          // -0 without one stays
    return y;
}

template <int OT, int N>
__device__ __forceinline__ void store_some(typename Element<OT>::T* p, typename Run<OT, N>::F y, int64_t n)
{
    if (n >= N) return store_run<OT, N, false>(p, y);
#pragma unroll
    for (int i = 0; i < N - 1; ++i)
        if (i < n) global(p)[i] = (typename Element<OT>::T)y[i];
}

// ... where a row has 16 of them: the 16 that end with the row's last one, loaded without a condition, if those from k on would pass it, which
// `in_place` moves to where they belong.  What it leaves behind the last one is any of the row's: tokens have zeros there.
__device__ __forceinline__ i4 load_window(const int8_t* row, int k, int inputs)
{
    return *(const QADAM_GLOBAL i4u*)(row + (k < inputs - 16 ? k : inputs - 16));
}

__device__ __forceinline__ i4 in_place(i4 v, int k, int inputs)
{
    const int by = k + 16 - inputs;
    if (inputs < 16 || by <= 0 || by >= 16) return v;       // shorter rows are not loaded like this
#pragma unroll
    for (int q = 2; q > 0; q /= 2)
        if (by & 4 * q) {
#pragma unroll
            for (int e = 0; e + q < 4; ++e) v[e] = v[e + q];
        }
    i4 w = v;
#pragma unroll
    for (int e = 0; e < 4; ++e) w[e] = (int)__builtin_amdgcn_alignbyte((uint32_t)v[e < 3 ? e + 1 : 3], (uint32_t)v[e], (uint32_t)(by & 3));
    return w;
}

// ---- few tokens -----------------------------------------------------------------------------------
// A wavefront takes 16 rows of the weights, all tokens (16 at most) and a part of the inputs; `split` of a workgroup's wavefronts share the
// rows and add their sums in LDS.  A lane's 16 integers of a matrix instruction are 16 bytes of one row, so the weights come from memory
// into their places, at any address.  AHEAD chunks of 64 inputs are under way at a time.
// MADE: the workgroup makes the tokens' integers itself, in LDS, which saves the launch that would, while its first weights are on the way.
// RAGGED: rows of 16 and more that are no multiple: one token of 1023 to 2048 6.3 us per call with loads under conditions, 5.4 without, of 2047
// 8.1 and 6.8; other widths take the same either way (2048 to 8192 5.5).
//
// One token of 768 to 50257 outputs, 38.6 MB of weights: 10.1 us per call, the kernel 9.6, of which 2.5 pass until the first product; the rest
// is 5.4 TB/s.  AHEAD 2, 6, 8, 12: 9.6, 10.2, 10.1, 11.4; with a launch for the integers in front 12.  Four wavefronts in a workgroup, where
// eight took 13.1: they hold the registers of a SIMD in larger lots.
// a barrier for what lies in LDS: loads from memory stay under way
__device__ __forceinline__ void lds_barrier()
{
    asm volatile("s_waitcnt lgkmcnt(0)" ::: "memory");
    __builtin_amdgcn_s_barrier();
    asm volatile("" ::: "memory");
}

template <int AHEAD, bool MADE, bool RAGGED>
__global__ void __launch_bounds__(64 * kRowWaves) k_product_rows(ProductLaunch L, TokensLaunch X, int split)
{
    extern __shared__ __attribute__((aligned(16))) int8_t lds[];
    __shared__ uint32_t most[kRowsTokens];
    const int lane = threadIdx.x % 64, wave = __builtin_amdgcn_readfirstlane(threadIdx.x / 64);
    const int padded = X.padded;
    const int part = wave % split, chunks = (L.inputs + 63) / 64, each = (chunks + split - 1) / split;
    const int begin = part * each, end = begin + each < chunks ? begin + each : chunks;
    const int64_t n0 = ((int64_t)blockIdx.x * (kRowWaves / split) + wave / split) * 16;
    const int k0 = lane / 16 * 16, t = lane % 16;

    // tokens that become integers here: runs of 8, a few per thread
    constexpr int kHeld = MADE ? kMadeInputs / (64 * kRowWaves * kRowRun) : 1;
    const int runs = padded / kRowRun;
    f8 held[kHeld];
    if constexpr (MADE) {
#pragma unroll
        for (int h = 0; h < kHeld; ++h) {
            const int q = h * 64 * kRowWaves + threadIdx.x, m = q / runs, at = q % runs * kRowRun;
            held[h] = 0.0f;
            if (m < (int)L.tokens && at < L.inputs) held[h] = load_part(X.x, X.x_type, m * X.x_stride + at, L.inputs - at);
        }
    }
    const int8_t* row = L.weight + (n0 + t < L.outputs ? n0 + t : L.outputs - 1) * L.weight_stride;
    const bool there = t < L.tokens;
    const int8_t* token = MADE ? lds + (there ? t : 0) * padded : L.codes + (there ? t : 0) * L.codes_stride;
    // chunks under way: chunk c of this wavefront's in place (c - begin) % AHEAD; zeros behind the last one
    i4 w[AHEAD], x[AHEAD];
    auto load_row = [&](int c, int u) {
        if constexpr (!RAGGED) w[u] = c < end ? load_weights(row, c * 64 + k0, L.inputs) : (i4)0;
        else w[u] = c < end ? load_window(row, c * 64 + k0, L.inputs) : (i4)0;
    };
    auto load_token = [&](int c, int u) {
        x[u] = 0;
        if (c < end && there) {
            if constexpr (MADE) x[u] = *(const i4*)(token + c * 64 + k0);
            else x[u] = *(const QADAM_GLOBAL i4*)(token + c * 64 + k0);
        }
    };
#pragma unroll
    for (int u = 0; u < AHEAD; ++u) {
        load_row(begin + u, u);
        if constexpr (!MADE) load_token(begin + u, u);
    }
    if constexpr (MADE) {
        if (threadIdx.x < kRowsTokens) most[threadIdx.x] = 0;
        lds_barrier();
#pragma unroll
        for (int h = 0; h < kHeld; ++h) {
            const int m = (h * 64 * kRowWaves + (int)threadIdx.x) / runs;
            if (m < (int)L.tokens) atomicMax(&most[m], largest_of(held[h]));
        }
        lds_barrier();
#pragma unroll
        for (int h = 0; h < kHeld; ++h) {
            const int q = h * 64 * kRowWaves + threadIdx.x, m = q / runs;
            if (m < (int)L.tokens) *(uint64_t*)(lds + q * kRowRun) = codes_of(TokenScale(most[m]), held[h]);
        }
        lds_barrier();
    }
    i4 acc = 0;
#pragma unroll 1
    for (int c = begin; c < end; c += AHEAD)
#pragma unroll
        for (int u = 0; u < AHEAD; ++u) {
            if (c + u >= end) break;
            if constexpr (MADE) load_token(c + u, u);
            if constexpr (RAGGED) w[u] = in_place(w[u], (c + u) * 64 + k0, L.inputs);
            acc = __builtin_amdgcn_mfma_i32_16x16x64_i8(w[u], x[u], acc, 0, 0, 0);
            load_row(c + AHEAD + u, u);
            if constexpr (!MADE) load_token(c + AHEAD + u, u);
        }
    if (split > 1) {
        __syncthreads();
        i4* sums = (i4*)lds;
        if (part > 0) sums[wave * 64 + lane] = acc;
        __syncthreads();
        if (part > 0) return;
        for (int p = 1; p < split; ++p) acc += sums[(wave + p) * 64 + lane];
    }
    const int64_t n = n0 + lane / 16 * 4;
    if (n >= L.outputs || !there) return;
    f4 scale, bias;
#pragma unroll
    for (int e = 0; e < 4; ++e) {
        const int64_t m = n + e < L.outputs ? n + e : L.outputs - 1;
        scale[e] = output_scale(L, m);
        bias[e] = output_bias(L, m);
    }
    const f4 y = results(L, acc, MADE ? TokenScale(most[t]).scale : global(L.token_scales)[t], scale, bias);
    const int64_t at = t * L.out_stride + n;
    if (L.out_type == QADAM_F32) store_some<QADAM_F32, 4>(static_cast<float*>(L.out) + at, y, L.outputs - n);
    else if (L.out_type == QADAM_BF16) store_some<QADAM_BF16, 4>(static_cast<__bf16*>(L.out) + at, y, L.outputs - n);
    else store_some<QADAM_F16, 4>(static_cast<_Float16*>(L.out) + at, y, L.outputs - n);
}

// ---- many tokens ----------------------------------------------------------------------------------
// A workgroup makes a tile of BM tokens and BN outputs, its wavefronts WM by WN parts of it, in steps of 128 inputs.  Both operands of a
// step pass through LDS, STAGES steps' worth of it: while one is multiplied, the next ones are loaded straight from memory into the
// others.  A row of 128 integers takes its 8 runs of 16 bytes in an order of its own, run ^ (row / 2 % 8), so that the 16 lanes that
// LDS serves together find theirs in different banks although rows are 128 bytes apart (by row % 8 two of them shared one: a quarter of
// the LDS's cycles, and 1 us of the call).
//
// A step's products are four blocks of 32 inputs.  Between the matrix instructions of one block the next block's operands are read from
// LDS and the next step's are loaded, one instruction after each, as the source has them (sched_barrier): in the compiler's order reads
// and products alternate with waits (the bare product of the sizes below, plain stores: 312 us, so 300).  The step changes in front of its
// last block, whose operands are in registers by then.
//
// 16384 tokens of 2048 to 8192 outputs: 260 us of a call's 280 to 285, 2.1 POPS; the tokens' integers take 18 (the calls of each alone, in a loop).
// The card's power sets it: the matrix units are busy 56 % of the time at 1.74 GHz, and the same product takes 199 us where all integers are
// zero; its matrix instructions alone, without loads and LDS, take 177.  Results (268 MB) are stored past the caches, since they would push the operands out: 333 us per
// call with ordinary stores, 291 so.  Taken back: steps of 64 inputs with three to five of them in LDS (306-313, 287), four wavefronts of
// 128 x 128 (without results 268, 256), columns of 8 and 16 tiles (291, 286), a higher priority of the products (the same).
// DIRECT: rows of the weights lie at addresses of 16 bytes and are loaded into LDS directly; else they pass through registers, STAGES - 1 steps
// of them on the way, all by loads of 16 bytes without a condition: 64 tokens of 2047 to 2048 10.9 us, 13.2 with conditions and a step less.
// parts: workgroups that share a tile of 64 by 64, each with a part of the steps.
constexpr int kStep = 128;

template <int BM, int BN, int WM, int WN, int STAGES>
struct Tiles {
    static constexpr int threads = 64 * WM * WN, mt = BM / WM / 32, nt = BN / WN / 32;
    static constexpr int a_bytes = BM * kStep, stage = (BM + BN) * kStep;
    static constexpr int a_loads = BM * 8 / threads, b_loads = BN * 8 / threads;
    static constexpr int pitch(int size) { return BN / WN * size + 16; }        // of a row of results in LDS
    // of the results: rows of each wavefront, then scale and bias of the tile's outputs
    static constexpr int columns(int size) { return WM * WN * 32 * pitch(size); }
    static constexpr int lds = STAGES * stage > columns(4) + 8 * BN ? STAGES * stage : columns(4) + 8 * BN;
};

template <int BM, int BN, int WM, int WN, int STAGES, bool DIRECT, int OT>
__global__ void __launch_bounds__(64 * WM * WN) k_product_tiles(ProductLaunch L, int64_t first, int across, int down, int parts, uint32_t* arrived)
{
    typedef Tiles<BM, BN, WM, WN, STAGES> S;
    extern __shared__ __attribute__((aligned(16))) int8_t lds[];
    const int lane = threadIdx.x % 64, wave = __builtin_amdgcn_readfirstlane(threadIdx.x / 64);
    constexpr bool kParts = BM * BN == kPartSum;
    const int tile = kParts ? blockIdx.x % (across * down) : blockIdx.x, part = kParts ? blockIdx.x / (across * down) : 0;
    int tm, tn;
    tile_place(tile, across, down, &tm, &tn);
    const int64_t t0 = first + (int64_t)tm * BM, n0 = (int64_t)tn * BN;
    const int steps = (L.inputs + kStep - 1) / kStep;
    const int begin = kParts ? steps * part / parts : 0, last = (kParts ? steps * (part + 1) / parts : steps) - begin - 1;

    // where this thread's runs of a step come from: rows behind the last one repeat it, inputs behind the last one repeat the row's first
    // ones (the tokens' integers are zeros there)
    const int8_t* a_base = L.codes + t0 * L.codes_stride;
    const int8_t* b_base = L.weight + n0 * L.weight_stride;
    const int a_rows = (int)(L.tokens - t0 < BM ? L.tokens - t0 : BM), b_rows = (int)(L.outputs - n0 < BN ? L.outputs - n0 : BN);
    uint32_t a_at[S::a_loads], b_at[S::b_loads];
    int b_run[S::b_loads];
#pragma unroll
    for (int i = 0; i < S::a_loads; ++i) {
        const int c = i * S::threads + threadIdx.x, row = c / 8, run = (c % 8 ^ (row >> 1 & 7)) * 16;
        a_at[i] = (uint32_t)(row < a_rows ? row : a_rows - 1) * (uint32_t)L.codes_stride + (uint32_t)run;
    }
    const int8_t* b_row[S::b_loads];
#pragma unroll
    for (int i = 0; i < S::b_loads; ++i) {
        const int c = i * S::threads + threadIdx.x, row = c / 8;
        b_run[i] = (c % 8 ^ (row >> 1 & 7)) * 16;
        if constexpr (DIRECT) b_at[i] = (uint32_t)(row < b_rows ? row : b_rows - 1) * (uint32_t)L.weight_stride;
        else b_row[i] = b_base + (int64_t)(row < b_rows ? row : b_rows - 1) * L.weight_stride;
    }
    i4 b_held[DIRECT ? 1 : STAGES - 1][DIRECT ? 1 : S::b_loads];        // of step s in s % (STAGES - 1)
    constexpr int kLoads = S::a_loads + S::b_loads;
    auto load = [&](int step, int buffer, int i, auto set) {
        int8_t* to = lds + buffer * S::stage;
        if (i < S::a_loads) {
            __builtin_amdgcn_global_load_lds((const QADAM_GLOBAL void*)(a_base + (a_at[i] + (uint32_t)(step * kStep))),
                                             (__attribute__((address_space(3))) void*)(to + (i * S::threads + wave * 64) * 16), 16, 0, 0);
        } else if constexpr (DIRECT) {
            const int b = i - S::a_loads, k = step * kStep + b_run[b];
            __builtin_amdgcn_global_load_lds((const QADAM_GLOBAL void*)(b_base + (b_at[b] + (uint32_t)(k < L.inputs ? k : 0))),
                                             (__attribute__((address_space(3))) void*)(to + S::a_bytes + (b * S::threads + wave * 64) * 16), 16, 0, 0);
        } else {
            const int b = i - S::a_loads;
            const int k = step * kStep + b_run[b];
            b_held[set.value][b] = L.inputs >= 16 ? load_window(b_row[b], k, L.inputs) : load_weights(b_row[b], k, L.inputs);
        }
    };
    // what was loaded into registers goes to LDS
    auto place = [&](int step, int buffer, auto set) {
        if constexpr (!DIRECT) {
#pragma unroll
            for (int b = 0; b < S::b_loads; ++b)
                *(i4*)(lds + buffer * S::stage + S::a_bytes + (b * S::threads + threadIdx.x) * 16) =
                    in_place(b_held[set.value][b], step * kStep + b_run[b], L.inputs);
        }
    };
    // This wavefront's loads into LDS have arrived but for the last `under_way`, and all wavefronts are here: the instructions that load
    // into LDS are not waited for by a barrier alone.
    auto meet = [](auto under_way) {
        asm volatile("s_waitcnt vmcnt(%0) lgkmcnt(0)" : : "n"(under_way.value) : "memory");
        __builtin_amdgcn_s_barrier();
        asm volatile("" ::: "memory");
    };
    constexpr std::integral_constant<int, (STAGES - 2) * kLoads> kAhead;        // the loads of the steps behind the next one

    i16 acc[S::mt][S::nt];
#pragma unroll
    for (int i = 0; i < S::mt; ++i)
#pragma unroll
        for (int j = 0; j < S::nt; ++j) acc[i][j] = 0;
    const int m0 = wave / WN * (BM / WM), c0 = wave % WN * (BN / WN);
    i4 a[2][S::mt], b[2][S::nt];
    constexpr int kOperands = S::mt + S::nt, kProducts = S::mt * S::nt;
    auto read = [&](int buffer, int block, int into, int i) {
        const int row = lane % 32, run = (block * 2 + lane / 32 ^ (row >> 1 & 7)) * 16;
        const int8_t* from = lds + buffer * S::stage + run;
        if (i < S::mt) a[into][i] = *(const i4*)(from + (m0 + i * 32 + row) * kStep);
        else b[into][i - S::mt] = *(const i4*)(from + S::a_bytes + (c0 + (i - S::mt) * 32 + row) * kStep);
    };
    // the products of the operands in a[from], b[from]; between them the reads of the next block's and the loads [begin, begin + count)
    auto block = [&](int from, bool reads, int buffer, int next, bool loads, int step, int into, int begin, int count, auto set) {
#pragma unroll
        for (int m = 0; m < kProducts; ++m) {
            const int i = m / S::nt, j = m % S::nt;
            acc[i][j] = __builtin_amdgcn_mfma_i32_32x32x32_i8(b[from][j], a[from][i], acc[i][j], 0, 0, 0);
            if (reads) {
#pragma unroll
                for (int q = 0; q < kOperands; ++q)
                    if (q * kProducts / kOperands == m) read(buffer, next, from ^ 1, q);
            }
            if (loads) {
#pragma unroll
                for (int q = 0; q < kLoads; ++q)
                    if (q < count && q * kProducts / count == m) load(step, into, begin + q, set);
            }
            __builtin_amdgcn_sched_barrier(0);
        }
    };
    static_assert(DIRECT || S::a_loads == S::b_loads, "the second half of the loads are the weights', which are placed before others take their registers");
    constexpr int kFirst = kLoads / 2;          // of a step's loads: the ones in front of the block in which the others are issued
    // steps behind the last one are the last one once more, unused
    auto step_of = [&](int s) { return begin + (s < last ? s : last); };
    constexpr int kSets = DIRECT ? 1 : STAGES - 1;
    constexpr std::integral_constant<int, 0> kSet0;
    constexpr std::integral_constant<int, kSets - 1> kSet1;
    static_assert(kSets <= 2, "sets of registers are named");
#pragma unroll
    for (int s = 0; s < STAGES - 1; ++s) {
#pragma unroll
        for (int i = 0; i < kLoads; ++i) {
            if (s % kSets == 0) load(step_of(s), s, i, kSet0);
            else load(step_of(s), s, i, kSet1);
        }
        __builtin_amdgcn_sched_barrier(0);      // `meet` counts them in this order
    }
    place(step_of(0), 0, kSet0);
    meet(kAhead);
#pragma unroll
    for (int i = 0; i < kFirst; ++i) load(step_of(STAGES - 1), STAGES - 1, i, kSet0);
#pragma unroll
    for (int q = 0; q < kOperands; ++q) read(0, 0, 0, q);
    int buffer = 0;                             // of step s
    // own: the set of registers that step s had and step s + STAGES - 1 gets; other: that of step s + 1
    auto multiply = [&](int s, auto own, auto other) {
        const int next = buffer + 1 < STAGES ? buffer + 1 : 0, before = buffer > 0 ? buffer - 1 : STAGES - 1;
        block(0, true, buffer, 1, true, step_of(s + STAGES - 1), before, kFirst, kLoads - kFirst, own);
        block(1, true, buffer, 2, false, 0, 0, 0, 0, own);
        block(0, true, buffer, 3, false, 0, 0, 0, 0, own);
        place(step_of(s + 1), next, other);
        meet(kAhead);
        block(1, true, next, 0, true, step_of(s + STAGES), buffer, 0, kFirst, own);
        buffer = next;
    };
    for (int s = 0; s < last; s += kSets) {
        multiply(s, kSet0, kSet1);
        if (kSets > 1 && s + 1 < last) multiply(s + 1, kSet1, kSet0);
    }
    block(0, true, buffer, 1, false, 0, 0, 0, 0, kSet0);
    block(1, true, buffer, 2, false, 0, 0, 0, 0, kSet0);
    block(0, true, buffer, 3, false, 0, 0, 0, 0, kSet0);
    block(1, false, 0, 0, false, 0, 0, 0, 0, kSet0);

    if constexpr (kParts)
        if (parts > 1) {
            // The workgroup that comes last adds the others' sums to its own.  Sums are stored and loaded past the caches that each XCD has of
            // its own (atomic at the scope of the GPU), so that it is enough to wait for the stores before the count: fences in their
            // place, which write back all of an L2, took 20 us.  Loads of four parts at a time save nothing.
            typedef uint64_t u8 __attribute__((ext_vector_type(8)));
            uint64_t* sums = (uint64_t*)L.sums + (int64_t)tile * parts * (kPartSum / 2) + threadIdx.x;
            const u8 own = __builtin_bit_cast(u8, acc[0][0]);
#pragma unroll
            for (int q = 0; q < 8; ++q) __hip_atomic_store(sums + part * (kPartSum / 2) + q * S::threads, own[q], __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
            meet(std::integral_constant<int, 0>());
            uint32_t* count = (uint32_t*)lds;
            if (threadIdx.x == 0) *count = atomicAdd(arrived + tile, 1u);
            __syncthreads();
            if (*count != (uint32_t)parts - 1) return;
            for (int p = 0; p < parts; ++p) {
                if (p == part) continue;
                u8 other;
#pragma unroll
                for (int q = 0; q < 8; ++q) other[q] = __hip_atomic_load(sums + p * (kPartSum / 2) + q * S::threads, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
                acc[0][0] += __builtin_bit_cast(i16, other);
            }
        }

    // Results through LDS, 32 tokens of a wavefront at a time, so that whole lines are stored: a lane holds 4 outputs of a token, and
    // 8 bytes each in 32 rows cost a quarter of the call.
    meet(std::integral_constant<int, 0>());
    typedef typename Element<OT>::T O;
    constexpr int kPitch = S::pitch(sizeof(O)), kRun = 16 / sizeof(O), kRuns = BN / WN / kRun;
    int8_t* own = lds + wave * 32 * kPitch;
    float* columns = (float*)(lds + S::columns(sizeof(O)));
    for (int i = threadIdx.x; i < BN; i += S::threads) {
        const int64_t n = n0 + i < L.outputs ? n0 + i : L.outputs - 1;
        columns[i] = output_scale(L, n);
        columns[BN + i] = output_bias(L, n);
    }
    __syncthreads();
#pragma unroll
    for (int i = 0; i < S::mt; ++i) {
        const int64_t t = t0 + m0 + i * 32;
        const float token = global(L.token_scales)[t + lane % 32 < L.tokens ? t + lane % 32 : L.tokens - 1];
#pragma unroll
        for (int j = 0; j < S::nt; ++j)
#pragma unroll
            for (int q = 0; q < 4; ++q) {
                const int at = j * 32 + 8 * q + lane / 32 * 4;
                const f4 scale = *(const f4*)(columns + c0 + at), bias = *(const f4*)(columns + BN + c0 + at);
                const i4 sum = {acc[i][j][q * 4], acc[i][j][q * 4 + 1], acc[i][j][q * 4 + 2], acc[i][j][q * 4 + 3]};
                typedef O o4 __attribute__((ext_vector_type(4)));
                *(o4*)(own + lane % 32 * kPitch + at * sizeof(O)) = __builtin_convertvector(results(L, sum, token, scale, bias), o4);
            }
#pragma unroll
        for (int q = 0; q < 32 * kRuns / 64; ++q) {
            const int c = q * 64 + lane, row = c / kRuns, at = c % kRuns * kRun;
            const int64_t n = n0 + c0 + at, left = L.outputs - n;
            typedef O on __attribute__((ext_vector_type(kRun)));
            typedef on onu __attribute__((aligned(sizeof(O))));
            const on v = *(const on*)(own + row * kPitch + at * sizeof(O));
            if (t + row >= L.tokens || left <= 0) continue;
            O* p = static_cast<O*>(L.out) + (t + row) * L.out_stride + n;
            if (left >= kRun) {
                __builtin_nontemporal_store(v, (QADAM_GLOBAL onu*)p);
            } else {
#pragma unroll
                for (int e = 0; e < kRun - 1; ++e)
                    if (e < left) global(p)[e] = v[e];
            }
        }
    }
}

template <int BM, int BN, int WM, int WN, int STAGES, bool DIRECT>
hipError_t tiles(const ProductLaunch& L, int parts = 1, uint32_t* arrived = nullptr)
{
    typedef Tiles<BM, BN, WM, WN, STAGES> S;
    // a launch takes as many rows of tiles as keep it below 2^22 workgroups
    const int across = (int)((L.outputs + BN - 1) / BN), most = (1 << 22) / across;
    for (int64_t t = 0; t < L.tokens; t += (int64_t)most * BM) {
        const int64_t rest = (L.tokens - t + BM - 1) / BM;
        const int down = (int)(rest < most ? rest : most);
        auto run = [&](auto kernel) {
            if constexpr (S::lds > 65536) {
                const hipError_t e = hipFuncSetAttribute(reinterpret_cast<const void*>(kernel), hipFuncAttributeMaxDynamicSharedMemorySize, S::lds);
                if (e != hipSuccess) return e;
            }
            kernel<<<dim3(across * down * parts), dim3(S::threads), S::lds, L.stream>>>(L, t, across, down, parts, arrived);
            return hipGetLastError();
        };
        const hipError_t e = L.out_type == QADAM_F32    ? run(k_product_tiles<BM, BN, WM, WN, STAGES, DIRECT, QADAM_F32>)
                             : L.out_type == QADAM_BF16 ? run(k_product_tiles<BM, BN, WM, WN, STAGES, DIRECT, QADAM_BF16>)
                                                        : run(k_product_tiles<BM, BN, WM, WN, STAGES, DIRECT, QADAM_F16>);
        if (e != hipSuccess) return e;
    }
    return hipSuccess;
}

template <int AHEAD, bool MADE>
hipError_t rows(const ProductLaunch& L, const TokensLaunch& X, int split)
{
    const bool ragged = L.inputs >= 16 && L.inputs % 16 != 0;
    const int of_a_group = 16 * (kRowWaves / split);
    int lds = split > 1 ? kRowWaves * 64 * 16 : 0;
    if (MADE && lds < (int)L.tokens * X.padded) lds = (int)L.tokens * X.padded;
    const dim3 grid((int)((L.outputs + of_a_group - 1) / of_a_group)), threads(64 * kRowWaves);
    if (ragged) k_product_rows<AHEAD, MADE, true><<<grid, threads, lds, L.stream>>>(L, X, split);
    else k_product_rows<AHEAD, MADE, false><<<grid, threads, lds, L.stream>>>(L, X, split);
    return hipGetLastError();
}

}  // namespace

hipError_t launch_tokens(const TokensLaunch& L)
{
    const dim3 grid((int)(L.tokens < 8192 ? L.tokens : 8192));
    if (L.x_type == QADAM_CODES8) k_token_codes<<<grid, dim3(kThreads), 0, L.stream>>>(L);
    else if (L.x_type == QADAM_F32) launch_tokens_of<QADAM_F32>(L, grid);
    else if (L.x_type == QADAM_BF16) launch_tokens_of<QADAM_BF16>(L, grid);
    else launch_tokens_of<QADAM_F16>(L, grid);
    return hipGetLastError();
}

hipError_t launch_product(const ProductLaunch& L, const TokensLaunch& X)
{
    // rows of the weights that can be loaded into LDS directly
    const bool direct = reinterpret_cast<uintptr_t>(L.weight) % 16 == 0 && L.weight_stride % 16 == 0 && L.inputs % 16 == 0 && L.weight_stride <= 1 << 22;
    const Linear8Plan p(L.tokens, L.outputs, L.inputs, X.x_type != QADAM_CODES8, direct);
    if (!p.made) {
        if (X.codes) {
            const hipError_t e = launch_tokens(X);
            if (e != hipSuccess) return e;
        }
    } else {
        return rows<4, true>(L, X, p.split);
    }
    const int parts = L.sums ? p.parts : 1;
    switch (p.kind) {
    case Linear8Plan::kRows: return rows<4, false>(L, X, p.split);
    case Linear8Plan::kTiles64Deep:
        return direct ? tiles<64, 64, 2, 2, 3, true>(L, parts, X.arrived) : tiles<64, 64, 2, 2, 3, false>(L, parts, X.arrived);
    case Linear8Plan::kTiles64: return direct ? tiles<64, 64, 2, 2, 2, true>(L) : tiles<64, 64, 2, 2, 2, false>(L);
    case Linear8Plan::kTiles256:
        if (direct) return tiles<256, 256, 4, 2, 2, true>(L);
        [[fallthrough]];
    default: return direct ? tiles<128, 128, 2, 2, 2, true>(L) : tiles<128, 128, 2, 2, 2, false>(L);
    }
}

}  // namespace qadam
