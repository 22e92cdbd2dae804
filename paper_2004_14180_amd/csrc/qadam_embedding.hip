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

// ------------------------------------------------------------------------------------------------
// Gradient.  The positions of the tokens are sorted by row, positions of one row ascending; a wavefront then adds the dout of a few
// runs of equal rows, a slice of the columns at a time, and writes each row of the gradient once.
// ------------------------------------------------------------------------------------------------

// the row of token t, or `rows`, which sorts behind all others
__device__ __forceinline__ uint32_t token_key(const TokenList& L, int64_t t, bool* outside)
{
    const int64_t row = token_row(L, t, outside);
    return row < 0 ? (uint32_t)L.rows : (uint32_t)row;
}

// Part `part` of `parts` of the matrix becomes zeros.
__device__ void fill_part(const EmbeddingGradLaunch& L, int part, int parts)
{
    const int size = element_size(L.grad_type);
    if (L.grad_stride == L.dim) {
        const int64_t bytes = L.t.rows * L.dim * size, each = ((bytes + parts - 1) / parts + 4095) / 4096 * 4096;
        const int64_t begin = part * each, end = begin + each < bytes ? begin + each : bytes;
        char* p = static_cast<char*>(L.grad);
        int64_t at = begin + threadIdx.x * 16;
        for (; at + 16 <= end; at += kThreads * 16) store_run<QADAM_F32, 4>(p + at, (f4)0.0f);
        if (at < end)
            for (; at < end; at += size) store_one(p + at, L.grad_type, 0, 0.0f);
        return;
    }
    for (int64_t r = part; r < L.t.rows; r += parts)
        for (int k = threadIdx.x; k < L.dim; k += kThreads) store_one(L.grad, L.grad_type, r * L.grad_stride + k, 0.0f);
}

// A token's place in the sorted list is the number of tokens before it: those of smaller rows, and of its row those in front.  Row and
// position are one number, `row << bits | position`; a workgroup counts the smaller ones for kTargets tokens.
constexpr int kTargets = 16;
constexpr int64_t kRankTokens = 16384;

__device__ __forceinline__ uint32_t wave_sum(uint32_t x)
{
#define QADAM_ADD(CTRL) x += (uint32_t)__builtin_amdgcn_update_dpp(0, (int)x, CTRL, 0xf, 0xf, false)
    QADAM_ADD(0x111); QADAM_ADD(0x112); QADAM_ADD(0x114); QADAM_ADD(0x118);     // within rows of 16 lanes, to their last one
#undef QADAM_ADD
    return (uint32_t)(__builtin_amdgcn_readlane((int)x, 15) + __builtin_amdgcn_readlane((int)x, 31) +
                      __builtin_amdgcn_readlane((int)x, 47) + __builtin_amdgcn_readlane((int)x, 63));
}

__global__ void __launch_bounds__(kThreads) k_rank(EmbeddingGradLaunch L, int bits, int rank_groups)
{
    if ((int)blockIdx.x >= rank_groups) {
        fill_part(L, blockIdx.x - rank_groups, gridDim.x - rank_groups);
        return;
    }
    __shared__ uint32_t target[kTargets], smaller[kTargets][kThreads / 64];
    const int num = (int)L.t.num, first = blockIdx.x * kTargets;
    bool outside = false;
    if (threadIdx.x < kTargets) {
        const int t = first + threadIdx.x;
        target[threadIdx.x] = t < num ? token_key(L.t, t, &outside) << bits | t : 0;
        if (outside) atomicOr(L.t.status, QADAM_STATUS_TOKEN_RANGE);
    }
    __syncthreads();
    uint32_t mine[kTargets], count[kTargets];
#pragma unroll
    for (int j = 0; j < kTargets; ++j) {
        mine[j] = __builtin_amdgcn_readfirstlane(target[j]);
        count[j] = 0;
    }
#pragma unroll 4
    for (int u = threadIdx.x; u < num; u += kThreads) {
        const uint32_t c = token_key(L.t, u, &outside) << bits | u;
#pragma unroll
        for (int j = 0; j < kTargets; ++j) count[j] += c < mine[j];
    }
#pragma unroll
    for (int j = 0; j < kTargets; ++j) {
        const uint32_t sum = wave_sum(count[j]);
        if (threadIdx.x % 64 == 0) smaller[j][threadIdx.x / 64] = sum;
    }
    __syncthreads();
    const int t = first + threadIdx.x;
    if (threadIdx.x < kTargets && t < num) {
        uint32_t rank = 0;
        for (int w = 0; w < kThreads / 64; ++w) rank += smaller[threadIdx.x][w];
        global(L.w.keys[0])[rank] = (int)(target[threadIdx.x] >> bits);
        global(L.w.order[0])[rank] = t;
    }
}

// Longer lists: a stable sort by digits of the row, low ones first.  Per pass the tiles' digits are counted, then each tile moves its
// tokens to where the counts of all digits and of the tiles in front put them.
struct SortPass {
    const int32_t *keys, *order;    // null: the tokens themselves
    int32_t *keys_out, *order_out;
    int32_t shift, bits, tiles;
};

__device__ __forceinline__ uint32_t sort_key(const EmbeddingGradLaunch& L, const SortPass& P, int i, bool* outside)
{
    *outside = false;
    return P.keys ? (uint32_t)global(P.keys)[i] : token_key(L.t, i, outside);
}

__global__ void __launch_bounds__(kThreads) k_count_digits(EmbeddingGradLaunch L, SortPass P)
{
    if ((int)blockIdx.x >= P.tiles) {
        fill_part(L, blockIdx.x - P.tiles, gridDim.x - P.tiles);
        return;
    }
    __shared__ uint32_t counts[1 << kSortBits];
    const int digits = 1 << P.bits, first = blockIdx.x * kSortTile;
    const int end = first + kSortTile < L.t.num ? first + kSortTile : (int)L.t.num;
    for (int d = threadIdx.x; d < digits; d += kThreads) counts[d] = 0;
    __syncthreads();
    bool any = false;
    for (int i = first + threadIdx.x; i < end; i += kThreads) {
        bool outside;
        atomicAdd(&counts[sort_key(L, P, i, &outside) >> P.shift & (digits - 1)], 1u);
        any |= outside;
    }
    if (any) atomicOr(L.t.status, QADAM_STATUS_TOKEN_RANGE);
    __syncthreads();
    for (int d = threadIdx.x; d < digits; d += kThreads) global(L.w.counts)[(int64_t)blockIdx.x * digits + d] = counts[d];
}

constexpr int kSortWaves = kThreads / 64, kWaveTokens = kSortTile / kSortWaves;

__global__ void __launch_bounds__(kThreads) k_move_digits(EmbeddingGradLaunch L, SortPass P)
{
    __shared__ uint32_t place[kSortWaves][1 << kSortBits], total[1 << kSortBits], before[kThreads];
    const int digits = 1 << P.bits, lane = threadIdx.x % 64, wave = threadIdx.x / 64;
    const int tile = blockIdx.x, num = (int)L.t.num;
    for (int d = threadIdx.x; d < kSortWaves << kSortBits; d += kThreads) place[0][d] = 0;
    __syncthreads();
    // this tile's digits, wavefront by wavefront
    const int first = tile * kSortTile + wave * kWaveTokens;
    const int end = first + kWaveTokens < num ? first + kWaveTokens : num;
    bool outside;
    for (int i = first + lane; i < end; i += 64) atomicAdd(&place[wave][sort_key(L, P, i, &outside) >> P.shift & (digits - 1)], 1u);
    // a thread's digits lie one behind the other: those of the tiles in front, and of all
    const int each = (digits + kThreads - 1) / kThreads, low = threadIdx.x * each;
    uint32_t sum = 0;
    for (int k = 0; k < each; ++k) {
        const int d = low + k;
        uint32_t front = 0, all = 0;
        if (d < digits)
#pragma unroll 8
            for (int u = 0; u < P.tiles; ++u) {
                const uint32_t n = global(L.w.counts)[(int64_t)u * digits + d];
                all += n;
                front += u < tile ? n : 0;
            }
        if (d < digits) total[d] = front + sum;
        sum += all;
    }
    before[threadIdx.x] = sum;
    __syncthreads();
    // tokens of smaller digits: the sums of the threads in front
    uint32_t ahead = 0;
    for (int u = 0; u < kThreads; u += 64) {
        const uint32_t n = u + lane < (int)threadIdx.x - lane ? before[u + lane] : 0;      // of the wavefronts in front
        ahead += wave_sum(n);
    }
    uint32_t within = sum;
    for (int s = 1; s < 64; s <<= 1) {
        const uint32_t n = __shfl_up(within, s);
        if (lane >= s) within += n;
    }
    ahead += within - sum;
    for (int k = 0; k < each; ++k) {
        const int d = low + k;
        if (d >= digits) break;
        uint32_t at = ahead + total[d];
        for (int w = 0; w < kSortWaves; ++w) {
            const uint32_t n = place[w][d];
            place[w][d] = at;
            at += n;
        }
    }
    __syncthreads();
    // 64 tokens at a time: those of one digit in the order of their lanes
    for (int i0 = first; i0 < end; i0 += 64) {
        const int i = i0 + lane;
        const bool valid = i < end;
        const uint32_t key = valid ? sort_key(L, P, i, &outside) : 0;
        const uint32_t d = key >> P.shift & (digits - 1);
        uint64_t same = __ballot(valid);
        for (int b = 0; b < P.bits; ++b) {
            const uint64_t set = __ballot(d >> b & 1);
            same &= d >> b & 1 ? set : ~set;
        }
        const int rank = __popcll(same & ((1ull << lane) - 1));
        if (valid) {
            const uint32_t at = place[wave][d] + rank;
            global(P.keys_out)[at] = (int)key;
            global(P.order_out)[at] = P.order ? global(P.order)[i] : i;
        }
        __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
        if (valid && rank == 0) place[wave][d] += __popcll(same);
        __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
    }
}

// Sums.  Positions of the sorted list are cut where a row begins and at multiples of kRunPiece; a wavefront takes the pieces that begin
// in its kChunk positions, in a slice of the columns.  A piece that is a whole run is finished here; the pieces of a longer run are put
// down, and the wavefront that arrives last adds them in order.
static_assert(kRunPiece % kChunk == 0 && kRunPiece < 64, "a piece ends at most kRunPiece behind the chunk's first position");
constexpr int kBatch = 8;

template <int TYPE, int N>
__device__ __forceinline__ typename Run<QADAM_F32, N>::F load_columns(const void* p, int n)
{
    if (n == N) return to_float<TYPE, N>(load_raw<TYPE, N, false>(p));
    typename Run<QADAM_F32, N>::F x = 0.0f;
    for (int k = 0; k < N; ++k)
        if (k < n) x[k] = load_one(p, TYPE, k);
    return x;
}

template <int N>
__device__ __forceinline__ typename Run<QADAM_F32, N>::F load_grad(const void* p, int type, int n)
{
    if (type == QADAM_F32) return load_columns<QADAM_F32, N>(p, n);
    if (type == QADAM_BF16) return load_columns<QADAM_BF16, N>(p, n);
    return load_columns<QADAM_F16, N>(p, n);
}

template <int N>
__device__ __forceinline__ void store_grad(void* p, int type, int n, typename Run<QADAM_F32, N>::F x)
{
    if (n == N) {
        if (type == QADAM_F32) store_run<QADAM_F32, N, false>(p, x);
        else if (type == QADAM_BF16) store_run<QADAM_BF16, N, false>(p, x);
        else store_run<QADAM_F16, N, false>(p, x);
        return;
    }
    for (int k = 0; k < N; ++k)
        if (k < n) store_one(p, type, k, x[k]);
}

template <int DT, int N>
__global__ void __launch_bounds__(64) k_sum_runs(EmbeddingGradLaunch L, int result, int slices)
{
    typedef typename Run<QADAM_F32, N>::F F;
    const int* keys = L.w.keys[result];
    const int lane = threadIdx.x, slice = blockIdx.x % slices, first = blockIdx.x / slices * kChunk, num = (int)L.t.num;
    const int rows = (int)L.t.rows;
    const int p = first + lane;
    const int key = p < num ? global(keys)[p] : rows, prev = p > 0 && p <= num ? global(keys)[p - 1] : -1;
    const int order = p < num ? global(L.w.order[result])[p] : 0;
    const uint64_t valid = __ballot(key < rows);
    const uint64_t runs = __ballot(key != prev) | ~valid;               // a run begins, or nothing more comes
    const uint64_t cuts = runs | __ballot(p % kRunPiece == 0);
    const uint64_t mine = cuts & valid & ((1ull << kChunk) - 1);
    if (!mine) return;
    const int begin = __builtin_ctzll(mine), last = 63 - __builtin_clzll(mine);
    const int end = last + 1 + __builtin_ctzll(cuts >> (last + 1));     // of the last piece: at most kRunPiece behind `first`
    const int col = (slice * 64 + lane) * N;
    const int n = L.dim - col < 0 ? 0 : L.dim - col < N ? L.dim - col : N;
    const int dsize = element_size(DT), gsize = element_size(L.grad_type);
    F sum = 0.0f;
    int piece = begin;
    for (int i = begin; i < end; i += kBatch) {
        F x[kBatch], old[kBatch];
#pragma unroll
        for (int j = 0; j < kBatch; ++j) {
            if (i + j >= end) break;
            const int64_t t = __builtin_amdgcn_readlane(order, i + j);
            x[j] = load_columns<DT, N>(static_cast<const char*>(L.dout) + (t * L.dout_stride + col) * dsize, n);
        }
#pragma unroll
        for (int j = 0; j < kBatch; ++j) {
            old[j] = 0.0f;
            if (i + j < end && L.accumulate && runs >> (i + j + 1) & 1) {
                const int64_t row = __builtin_amdgcn_readlane(key, i + j);
                old[j] = load_grad<N>(static_cast<const char*>(L.grad) + (row * L.grad_stride + col) * gsize, L.grad_type, n);
            }
        }
#pragma unroll
        for (int j = 0; j < kBatch; ++j) {
            if (i + j >= end) break;
            sum += x[j];
            if (!(cuts >> (i + j + 1) & 1)) continue;
            // the piece ends here
            const int row = __builtin_amdgcn_readlane(key, i + j);
            char* out = static_cast<char*>(L.grad) + ((int64_t)row * L.grad_stride + col) * gsize;
            if (runs >> piece & 1 && runs >> (i + j + 1) & 1) {
                F y = sum * L.scale;
                if (L.accumulate) y = old[j] + y;
                store_grad<N>(out, L.grad_type, n, y);
            } else {
                // blocks of kRunPiece positions that the run crosses: [head, tail]
                const int block = (first + piece) / kRunPiece;
                int head = block, tail = block;
                if (!(runs >> piece & 1))
                    for (;;) {
                        const int at = (head - lane) * kRunPiece - 1;
                        const uint64_t other = __ballot(at < 0 || global(keys)[at < 0 ? 0 : at] != row);
                        const int same = other ? __builtin_ctzll(other) : 64;
                        head -= same;
                        if (same < 64) break;
                    }
                for (;;) {
                    const int64_t at = (int64_t)(tail + 1 + lane) * kRunPiece;
                    const uint64_t other = __ballot(at >= num || global(keys)[at < num ? at : 0] != row);
                    const int same = other ? __builtin_ctzll(other) : 64;
                    tail += same;
                    if (same < 64) break;
                }
                float* put = L.w.pieces + (int64_t)(2 * block + (block == head)) * L.dim + col;
                for (int k = 0; k < N; ++k)
                    if (k < n) __hip_atomic_store(put + k, sum[k], __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
                __builtin_amdgcn_fence(__ATOMIC_RELEASE, "agent");
                uint32_t* arrived = L.w.arrived + (int64_t)head * slices + slice;
                int come = 0;
                if (lane == 0) come = (int)__hip_atomic_fetch_add(arrived, 1u, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
                come = __builtin_amdgcn_readfirstlane(come);
                if (come == tail - head) {
                    __builtin_amdgcn_fence(__ATOMIC_ACQUIRE, "agent");
                    if (lane == 0) __hip_atomic_store(arrived, 0u, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
                    F y = 0.0f;
#pragma unroll 4
                    for (int b = head; b <= tail; ++b) {
                        const float* get = L.w.pieces + (int64_t)(2 * b + (b == head)) * L.dim + col;
                        for (int k = 0; k < N; ++k)
                            if (k < n) y[k] += __hip_atomic_load(get + k, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
                    }
                    y = y * L.scale;
                    if (L.accumulate) y = load_grad<N>(out, L.grad_type, n) + y;
                    store_grad<N>(out, L.grad_type, n, y);
                }
            }
            sum = 0.0f;
            piece = i + j + 1;
        }
    }
}

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

static int bits_of(uint64_t n)
{
    int b = 0;
    while (n >> b) ++b;
    return b;
}

template <int DT>
static hipError_t sum_runs(const EmbeddingGradLaunch& L, int result)
{
    const int slices = column_slices(L.dim);
    const dim3 grid((unsigned)((L.t.num + kChunk - 1) / kChunk * slices)), block(64);
    switch (lane_columns(L.dim)) {
    case 4: hipLaunchKernelGGL((k_sum_runs<DT, 4>), grid, block, 0, L.stream, L, result, slices); break;
    case 2: hipLaunchKernelGGL((k_sum_runs<DT, 2>), grid, block, 0, L.stream, L, result, slices); break;
    default: hipLaunchKernelGGL((k_sum_runs<DT, 1>), grid, block, 0, L.stream, L, result, slices); break;
    }
    return hipGetLastError();
}

hipError_t launch_embedding_grad(const EmbeddingGradLaunch& L)
{
    // workgroups that fill the matrix with zeros, beside those that begin the sort
    const int64_t bytes = L.t.rows * L.dim * element_size(L.grad_type);
    const int fill = L.accumulate ? 0 : (int)(bytes / 65536 < 1 ? 1 : bytes / 65536 < 4096 ? bytes / 65536 : 4096);
    const int64_t num = L.t.num;
    const int row_bits = bits_of((uint64_t)L.t.rows), bits = bits_of((uint64_t)num);
    int result = 0;
    if (num <= kRankTokens && row_bits + bits <= 32) {
        const int groups = (int)((num + kTargets - 1) / kTargets);
        if (groups + fill > 0) hipLaunchKernelGGL(k_rank, dim3(groups + fill), dim3(kThreads), 0, L.stream, L, bits, groups);
        if (const hipError_t e = hipGetLastError()) return e;
    } else {
        const int passes = (row_bits + kSortBits - 1) / kSortBits, digit = (row_bits + passes - 1) / passes;
        const int tiles = (int)sort_tiles(num);
        for (int k = 0; k < passes; ++k) {
            const SortPass P{k ? L.w.keys[(k - 1) & 1] : nullptr, k ? L.w.order[(k - 1) & 1] : nullptr, L.w.keys[k & 1], L.w.order[k & 1],
                             k * digit, digit, tiles};
            hipLaunchKernelGGL(k_count_digits, dim3(tiles + (k == 0 ? fill : 0)), dim3(kThreads), 0, L.stream, L, P);
            if (const hipError_t e = hipGetLastError()) return e;
            hipLaunchKernelGGL(k_move_digits, dim3(tiles), dim3(kThreads), 0, L.stream, L, P);
            if (const hipError_t e = hipGetLastError()) return e;
            result = k & 1;
        }
    }
    if (num == 0) return hipSuccess;
    if (L.dout_type == QADAM_F32) return sum_runs<QADAM_F32>(L, result);
    if (L.dout_type == QADAM_BF16) return sum_runs<QADAM_BF16>(L, result);
    return sum_runs<QADAM_F16>(L, result);
}

}  // namespace qadam
