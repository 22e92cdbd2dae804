// gfx950 kernels of the embedding: lookup with scaling, and the gradient by sorted tokens.
//
// Both are bound by memory where they are long and by launches and chains of loads where they are short.  The gradient of a row is
// the sum of the dout of its tokens, so whoever adds must know them: atomics from every token would write each row as often as it
// occurs and in no fixed order, while a list of positions sorted by row lets every row be written once, from registers, and makes
// the result the same bits on every run.  Three ways, by sizes alone, us per call (second and third: in all of their launches):
//   * up to 2048 tokens, fewer beyond 1024 columns (direct_tokens), one launch that needs no sort: each token looks for its row in the
//     list (k_sum_direct).  1024 tokens of 768 fp32, added to the matrix: 5.6 (sorted: 12);
//   * up to 131072 tokens and 524 k rows, the sort is one launch (k_group) and the sums another (k_sum_runs).  16384 tokens of 2048
//     bf16 and a matrix of 50257 rows written whole, 479 MB: 90;
//   * beyond, the sort takes two launches per digit of up to 9 bits (140 k tokens: 54 for 17 bits of rows).
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

// Lookup: a lane takes a run of 8 elements of a row, the next lane the next run, and after a row's last run the next row's first.  Rows
// are read through the caches, since frequent tokens repeat; the output streams past them: 16384 tokens of 2048 bf16 23.0 us without,
// 16.8 now (93 MB; 5.6 TB/s).  Several rows per lane, under way together, only cost: 17.2 with two, 17.8 with four, 19.3 with eight.
constexpr int kRun = 8;

template <int WT, int OT>
__device__ __forceinline__ void lookup_run(const LookupLaunch& L, int64_t t, int64_t row, int at)
{
    typedef typename Element<WT>::T W;
    typedef typename Element<OT>::T O;
    const W* from = static_cast<const W*>(L.weight) + row * L.weight_stride;
    O* to = static_cast<O*>(L.out) + t * L.out_stride;
    if (at + kRun <= L.dim) {
        typename Run<WT, kRun>::F x = 0.0f;             // zero, whatever the scale
        if (row >= 0) x = to_float<WT, kRun>(load_raw<WT, kRun, false>(from + at)) * L.scale;
        store_run<OT, kRun>(to + at, x);
    } else {
        for (int k = at; k < L.dim; ++k) global(to)[k] = (O)(row < 0 ? 0.0f : (float)global(from)[k] * L.scale);
    }
}

template <int WT>
__global__ void __launch_bounds__(kThreads) k_lookup(LookupLaunch L, uint32_t runs)
{
    const uint32_t i = blockIdx.x * kThreads + threadIdx.x, t = i / runs, run = i - t * runs;
    if (t >= L.t.num) return;
    bool outside;
    const int64_t row = token_row(L.t, t, &outside);
    if (outside && run == 0) atomicOr(L.t.status, QADAM_STATUS_TOKEN_RANGE);
    const int at = (int)run * kRun;
    if (L.out_type == QADAM_F32) lookup_run<WT, QADAM_F32>(L, t, row, at);
    else if (L.out_type == QADAM_BF16) lookup_run<WT, QADAM_BF16>(L, t, row, at);
    else lookup_run<WT, QADAM_F16>(L, t, row, at);
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

// A row of the gradient becomes zeros, by one wavefront.
template <int GT>
__device__ __forceinline__ void clear_row(const EmbeddingGradLaunch& L, int64_t row, int lane)
{
    typedef typename Element<GT>::T G;
    constexpr int kWide = 16 / sizeof(G);
    G* p = static_cast<G*>(L.grad) + row * L.grad_stride;
    int at = lane * kWide;
    for (; at + kWide <= L.dim; at += 64 * kWide) store_run<GT, kWide>(p + at, (typename Run<GT, kWide>::F)0.0f);
    if (at < L.dim)
        for (; at < L.dim; ++at) global(p)[at] = (G)0.0f;
}

// Rows of this size that are cleared while lists are grouped, which leaves the memory idle: about 8 us and 0.6 per 1024 tokens, at 5 TB/s.
// 16384 tokens, 412 MB: none 99.6 us per call, a quarter of this 99.0, half 96.6, this 93.5 (then 88 with two rows per wavefront)
static int64_t early_rows(int64_t tokens, int64_t rows, int64_t row_bytes)
{
    const int64_t n = (40000000 + 3000 * tokens) / row_bytes;
    return n < rows ? n : rows;
}

// Lists of up to kGroupTokens tokens are sorted in one launch: workgroup b takes the rows with row % groups = b, so the order is by
// row % groups, then by row.  Every workgroup reads the whole list, a part per wavefront: it counts the tokens of smaller b, which
// gives the place of its own, and keeps those in LDS as `row / groups << bits | position`.  They are ordered by counting row / groups.
// One more workgroup writes `rows` behind the last one, for the tokens without a row.  256 groups, one per CU, as long as row / groups
// has no more than kSortBits bits; up to 1024 for more rows.
constexpr int kGroupBits = 8, kMostGroupBits = 10;
constexpr int kGroupThreads = 1024, kGroupWaves = kGroupThreads / 64;
constexpr int64_t kGroupTokens = 1 << 17;
constexpr int kKept = 752;              // tokens of a wavefront in LDS, so that two workgroups share a CU; a list of more than
                                        // 12032 tokens of which a wavefront finds more of its workgroup's is read again

template <bool WIDE>
struct TokenReader {
    const void* tokens;
    uint32_t rows, padding;

    __device__ __forceinline__ explicit TokenReader(const TokenList& L)
        : tokens(L.tokens), rows((uint32_t)L.rows), padding(L.padding >= 0 && L.padding < L.rows ? (uint32_t)L.padding : ~0u) {}

    // the row, or ~0
    __device__ __forceinline__ uint32_t operator()(int i, bool* outside) const
    {
        uint32_t low, high = 0;
        if constexpr (WIDE) {
            const uint64_t v = global(static_cast<const uint64_t*>(tokens))[i];
            low = (uint32_t)v;
            high = (uint32_t)(v >> 32);
        } else {
            low = global(static_cast<const uint32_t*>(tokens))[i];
        }
        *outside = high != 0 || low >= rows;
        return *outside || low == padding ? ~0u : low;
    }
};

__device__ __forceinline__ int lanes_below(uint64_t mask)
{
    return __builtin_amdgcn_mbcnt_hi((uint32_t)(mask >> 32), __builtin_amdgcn_mbcnt_lo((uint32_t)mask, 0));
}

template <bool WIDE, int GT>
__global__ void __launch_bounds__(kGroupThreads) k_group(EmbeddingGradLaunch L, int bits, int digit_bits, int group_bits, int64_t clear_from)
{
    __shared__ uint32_t kept[kGroupWaves][kKept];
    __shared__ uint32_t place[kGroupWaves][1 << kSortBits];
    __shared__ uint32_t wave_count[kGroupWaves], wave_smaller[kGroupWaves], wave_ahead[kGroupWaves];
    const int lane = threadIdx.x % 64, wave = __builtin_amdgcn_readfirstlane(threadIdx.x / 64), group = blockIdx.x;
    const int groups = 1 << group_bits;
    if (group > groups) {
        // the GPU's memory has little to do meanwhile: the last rows of the gradient, whether or not they have tokens
        const int64_t first = clear_from + ((int64_t)(group - groups - 1) * kGroupWaves + wave) * kClearRows;
        for (int64_t r = first; r < first + kClearRows && r < L.t.rows; ++r) clear_row<GT>(L, r, lane);
        return;
    }
    const TokenReader<WIDE> read(L.t);
    const int num = (int)L.t.num, part = ((num + kGroupWaves - 1) / kGroupWaves + 63) / 64 * 64;
    const int begin = wave * part, end = begin + part < num ? begin + part : num;
    int count = 0, smaller = 0;
    bool any_outside = false;
    constexpr int kLoads = 4;
    for (int i0 = begin; i0 < end; i0 += 64 * kLoads) {
        uint32_t row[kLoads];
        bool outside[kLoads];
#pragma unroll
        for (int k = 0; k < kLoads; ++k) {
            const int i = i0 + k * 64 + lane;
            row[k] = read(i < end ? i : end - 1, &outside[k]);
            if (i >= end) row[k] = ~0u;
        }
#pragma unroll
        for (int k = 0; k < kLoads; ++k) {
            any_outside |= outside[k];
            const uint64_t own = __ballot(row[k] != ~0u && (int)(row[k] & (groups - 1)) == group);
            smaller += __popcll(__ballot(row[k] != ~0u && (int)(row[k] & (groups - 1)) < group));
            if (!own) continue;
            const int at = count + lanes_below(own);
            if (own >> lane & 1 && at < kKept) kept[wave][at] = row[k] >> group_bits << bits | (uint32_t)(i0 + k * 64 + lane);
            count += __popcll(own);
        }
    }
    if (lane == 0) { wave_count[wave] = (uint32_t)count; wave_smaller[wave] = (uint32_t)smaller; }
    __syncthreads();
    int base = 0, total = 0;
    bool all_kept = true;
    for (int w = 0; w < kGroupWaves; ++w) {
        const int n = (int)wave_count[w];
        base += (int)wave_smaller[w];
        total += n;
        all_kept &= n <= kKept;
    }
    int32_t *keys = L.w.keys[0], *order = L.w.order[0];
    if (group == groups) {
        // every token with a row is smaller
        for (int i = base + threadIdx.x; i < num; i += kGroupThreads) global(keys)[i] = (int)L.t.rows;
        if (any_outside) atomicOr(L.t.status, QADAM_STATUS_TOKEN_RANGE);
        return;
    }
    if (total == 0) return;
    const uint32_t position = (1u << bits) - 1;
    // the wavefront's tokens, 64 at a time: body(whether the lane has one, row / groups << bits | position)
    auto each = [&](auto&& body) {
        if (all_kept) {
            for (int i = 0; i < count; i += 64) body(i + lane < count, kept[wave][i + lane < count ? i + lane : 0]);
        } else {
            for (int i = begin; i < end; i += 64) {
                bool outside;
                const uint32_t row = read(i + lane < end ? i + lane : end - 1, &outside);
                body(i + lane < end && row != ~0u && (int)(row & (groups - 1)) == group, row >> group_bits << bits | (uint32_t)(i + lane));
            }
        }
    };
    const int digits = 1 << digit_bits;
    for (int d = threadIdx.x; d < kGroupWaves << kSortBits; d += kGroupThreads) place[0][d] = 0;
    __syncthreads();
    each([&](bool valid, uint32_t c) {
        if (valid) atomicAdd(&place[wave][c >> bits], 1u);
    });
    __syncthreads();
    // thread d has digit d: its tokens in all wavefronts, then those of the digits in front
    const int d = threadIdx.x;
    uint32_t sum = 0;
    if (d < digits)
        for (int w = 0; w < kGroupWaves; ++w) sum += place[w][d];
    uint32_t ahead = sum;
    for (int s = 1; s < 64; s <<= 1) {
        const uint32_t n = __shfl_up(ahead, s);
        if (lane >= s) ahead += n;
    }
    if (lane == 63) wave_ahead[wave] = ahead;
    ahead -= sum;
    __syncthreads();
    for (int w = 0; w < wave; ++w) ahead += wave_ahead[w];
    if (d < digits) {
        uint32_t at = (uint32_t)base + ahead;
        for (int w = 0; w < kGroupWaves; ++w) {
            const uint32_t n = place[w][d];
            place[w][d] = at;
            at += n;
        }
    }
    __syncthreads();
    each([&](bool valid, uint32_t c) {
        const uint32_t digit = c >> bits;
        uint64_t same = __ballot(valid);
        for (int b = 0; b < digit_bits; ++b) {
            const uint64_t set = __ballot(digit >> b & 1);
            same &= digit >> b & 1 ? set : ~set;
        }
        const int rank = lanes_below(same);
        if (valid) {
            const uint32_t at = place[wave][digit] + rank;
            global(keys)[at] = (int)(digit << group_bits | (uint32_t)group);
            global(order)[at] = (int)(c & position);
        }
        __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
        if (valid && rank == 0) place[wave][digit] += __popcll(same);
        __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
    });
}

// the sum over the wavefront
__device__ __forceinline__ uint32_t wave_sum(uint32_t x)
{
#define QADAM_ADD(CTRL) x += (uint32_t)__builtin_amdgcn_update_dpp(0, (int)x, CTRL, 0xf, 0xf, false)
    QADAM_ADD(0x111); QADAM_ADD(0x112); QADAM_ADD(0x114); QADAM_ADD(0x118);     // within rows of 16 lanes, to their last one
#undef QADAM_ADD
    return (uint32_t)(__builtin_amdgcn_readlane((int)x, 15) + __builtin_amdgcn_readlane((int)x, 31) +
                      __builtin_amdgcn_readlane((int)x, 47) + __builtin_amdgcn_readlane((int)x, 63));
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
// in its kChunk positions, in a slice of the columns.  So the work is even whatever the tokens are: a frequent row is many wavefronts'.
// A piece that is a whole run is finished here; the pieces of a longer run are put down, and the wavefront that arrives last adds them
// in order.  Eight rows are under way at a time, when adding with the old values of theirs.
// Where a row is frequent the wavefronts with a whole piece are every (kRunPiece / kChunk)-th: an odd number, or they meet on a few CUs.
// us of the sums, 16384 tokens of 2048 bf16, matrix written / added to, 8191 of 1001 fp16 added, 131 k of 512 bf16 added; chunks of 8
// tokens with pieces of 24 75 / 50 / 14.9 / 83, 32 79 / 69 / - / 153, 40 73.6 / 48.6 / 14.4 / 74, 48 72 / 52 / 15.5 / 91, 56 72.8 /
// 45.6 / 17.6 / 71; of 6 with 30 74 / 51 / 14.7 / 83; of 4 with 36 75 / 56 / 14.5 / 87.
static_assert(kRunPiece % kChunk == 0 && kRunPiece < 64, "a piece ends at most kRunPiece behind the chunk's first position");
constexpr int kBatch = 8;

// the last `n` of the N columns
template <int TYPE, int N>
__device__ __forceinline__ void store_columns(typename Element<TYPE>::T* p, int n, typename Run<QADAM_F32, N>::F x)
{
    if (n == N) {
        store_run<TYPE, N>(p, x);
        return;
    }
    for (int k = 0; k < N; ++k)
        if (k >= N - n) global(p)[k] = (typename Element<TYPE>::T)x[k];
}

// Puts down the sum of a piece of a run that other wavefronts have pieces of too, one per block of kRunPiece positions; the last
// wavefront to arrive adds them in order.  What crosses from one wavefront to another are agent-scope atomics, which need no cache
// written back: a piece is in memory before its arrival is counted.  (With a release fence per piece, which writes back the L2, the sums of
// 16384 tokens of 2048 bf16 took 152 us instead of 35.)
template <int GT, int N, bool ACCUMULATE>
__device__ __forceinline__ void join_piece(const EmbeddingGradLaunch& L, const int32_t* keys, int row, int block, int32_t front, int32_t behind,
                                           bool is_head, typename Run<QADAM_F32, N>::F sum, int lane, int slice, int slices, int n, int col)
{
    typedef typename Run<QADAM_F32, N>::F F;
    typedef typename Element<GT>::T G;
    const int num = (int)L.t.num;
    // the run's blocks are [head, tail]; `key` holds the boundaries of the first look
    auto length = [&](int32_t key, auto&& boundary) {
        for (RunSearch search;;) {
            const uint64_t other = __ballot(key != row);
            if (!search.next(other ? __builtin_ctzll(other) : 64)) return search.count;
            key = boundary(search.place(lane));
        }
    };
    int head = block, tail = block;
    if (!is_head)
        head -= length(front, [&](int d) {
            const int at = (block - d) * kRunPiece - 1;
            return at < 0 ? -1 : global(keys)[at];
        });
    tail += length(behind, [&](int d) {
        const int64_t at = (int64_t)(block + 1 + d) * kRunPiece;
        return at < num ? global(keys)[at] : -1;
    });
    float* put = L.w.pieces + (int64_t)(2 * block + is_head) * L.dim + col;
#pragma unroll
    for (int k = 0; k < N; ++k)
        if (k >= N - n) __hip_atomic_store(global(put + k), sum[k], __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
    G* out = static_cast<G*>(L.grad) + col + (int64_t)row * L.grad_stride;
    typename Run<GT, N>::V old;
    if constexpr (ACCUMULATE) old = load_raw<GT, N, false>(out);
    asm volatile("s_waitcnt vmcnt(0)" ::: "memory");
    uint32_t* arrived = L.w.arrived + (int64_t)head * slices + slice;
    int come = 0;
    if (lane == 0) come = (int)__hip_atomic_fetch_add(global(arrived), 1u, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
    come = __builtin_amdgcn_readfirstlane(come);
    if (come != tail - head) return;
    asm volatile("" ::: "memory");
    if (lane == 0) __hip_atomic_store(global(arrived), 0u, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
    // in fp64: in fp32 each of a constant row's equal sums is rounded the same way, and 2^20 tokens of 0.51 were 2e-4 off
    typedef double D __attribute__((ext_vector_type(N)));
    D total = 0.0;
    for (int b = head; b <= tail; b += kBatch) {
        F x[kBatch];
#pragma unroll
        for (int j = 0; j < kBatch; ++j) {
            const int at = b + j <= tail ? b + j : tail;
            const float* get = L.w.pieces + (int64_t)(2 * at + (at == head)) * L.dim + col;
#pragma unroll
            for (int k = 0; k < N; ++k) x[j][k] = __hip_atomic_load(global(get + k), __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
        }
#pragma unroll
        for (int j = 0; j < kBatch; ++j)
            if (b + j <= tail) total += __builtin_convertvector(x[j], D);
    }
    F y = __builtin_convertvector(total, F) * L.scale;
    if constexpr (ACCUMULATE) y = to_float<GT, N>(old) + y;
    store_columns<GT, N>(out, n, y);
}

// what the sorted list is ordered by
__device__ __forceinline__ uint32_t sorted_by(uint32_t row, int group_bits)
{
    return group_bits ? row << (32 - group_bits) | row >> group_bits : row;
}

// Rows without a token become zeros: lane r looks for the wavefront's row r in the sorted list.
template <int GT>
__device__ __forceinline__ void clear_absent(const EmbeddingGradLaunch& L, const int* keys, int group_bits, int64_t first, int64_t end, int lane)
{
    const int64_t row = first + lane % kClearRows;
    const uint32_t want = sorted_by((uint32_t)row, group_bits);
    int low = 0, high = (int)L.t.num;       // the first one that is not smaller
    while (low < high) {
        const int mid = (low + high) / 2;
        const uint32_t k = (uint32_t)global(keys)[mid];
        const bool less = k < (uint32_t)L.t.rows && sorted_by(k, group_bits) < want;
        low = less ? mid + 1 : low;
        high = less ? high : mid;
    }
    const bool absent = low >= (int)L.t.num || global(keys)[low] != (int)row;
    const uint64_t clear = __ballot(absent);
    for (int r = 0; r < kClearRows; ++r)
        if (clear >> r & 1 && first + r < end) clear_row<GT>(L, first + r, lane);
}

template <int DT, int GT, int N, bool ACCUMULATE>
__global__ void __launch_bounds__(64) k_sum_runs(EmbeddingGradLaunch L, int result, int slices, int sum_groups, int group_bits, int64_t clear_rows)
{
    typedef typename Run<QADAM_F32, N>::F F;
    typedef typename Element<DT>::T D;
    typedef typename Element<GT>::T G;
    const int* keys = L.w.keys[result];
    const int lane = threadIdx.x;
    if (!ACCUMULATE && (int)blockIdx.x >= sum_groups) {
        const int64_t turn = (int64_t)((int)gridDim.x - sum_groups) * kClearRows;
        for (int64_t r = (int64_t)((int)blockIdx.x - sum_groups) * kClearRows; r < clear_rows; r += turn)
            clear_absent<GT>(L, keys, group_bits, r, clear_rows, lane);
        return;
    }
    const int slice = blockIdx.x % slices, first = blockIdx.x / slices * kChunk, num = (int)L.t.num;
    const int rows = (int)L.t.rows;
    const int p = first + lane;
    const int key = p < num ? global(keys)[p] : rows, prev = p > 0 && p <= num ? global(keys)[p - 1] : -1;
    const int order = p < num ? global(L.w.order[result])[p] : 0;
    // the rows at the boundaries of this block and those in front, and behind it: for join_piece
    const int block = first / kRunPiece, at_front = (block - lane) * kRunPiece - 1;
    const int64_t at_behind = (int64_t)(block + 1 + lane) * kRunPiece;
    const int32_t front = at_front < 0 ? -1 : global(keys)[at_front], behind = at_behind < num ? global(keys)[at_behind] : -1;
    const uint64_t valid = __ballot(key < rows);
    const uint64_t runs = __ballot(key != prev) | ~valid;               // a run begins, or nothing more comes
    const uint64_t cuts = runs | __ballot(p % kRunPiece == 0);
    const uint64_t mine = cuts & valid & ((1ull << kChunk) - 1);
    if (!mine) return;
    const int begin = __builtin_ctzll(mine), last = 63 - __builtin_clzll(mine);
    const int end = last + 1 + __builtin_ctzll(cuts >> (last + 1));     // of the last piece: at most kRunPiece behind `first`
    // a lane at the ragged end takes the last N columns, and writes those of them that no other lane has
    const int own = (slice * 64 + lane) * N;
    const int n = L.dim - own < 0 ? 0 : L.dim - own < N ? L.dim - own : N, col = n == N ? own : L.dim - N;
    const D* from = static_cast<const D*>(L.dout) + col;
    G* to = static_cast<G*>(L.grad) + col;
    F sum = 0.0f, earlier = 0.0f, later = 0.0f;
    int piece = begin, later_piece = -1;
    for (int i = begin; i < end; i += kBatch) {
        // all loads of a batch are under way together; behind the end they repeat the last one
        typename Run<DT, N>::V x[kBatch];
        typename Run<GT, N>::V old[kBatch];
#pragma unroll
        for (int j = 0; j < kBatch; ++j) {
            const int64_t t = __builtin_amdgcn_readlane(order, i + j < end ? i + j : end - 1);
            x[j] = load_raw<DT, N, false>(from + t * L.dout_stride);
        }
        if (ACCUMULATE && (runs >> (i + 1) & ((1ull << kBatch) - 1)))       // some row ends in this batch
#pragma unroll
            for (int j = 0; j < kBatch; ++j) {
                const int64_t row = __builtin_amdgcn_readlane(key, i + j < end ? i + j : end - 1);
                old[j] = load_raw<GT, N, false>(to + row * L.grad_stride);
            }
#pragma unroll
        for (int j = 0; j < kBatch; ++j) {
            if (i + j >= end) break;
            sum += to_float<DT, N>(x[j]);
            if (!(cuts >> (i + j + 1) & 1)) continue;
            // the piece ends here
            const int row = __builtin_amdgcn_readlane(key, i + j);
            G* out = to + (int64_t)row * L.grad_stride;
            if (runs >> piece & 1 && runs >> (i + j + 1) & 1) {
                F y = sum * L.scale;
                if constexpr (ACCUMULATE) y = to_float<GT, N>(old[j]) + y;
                store_columns<GT, N>(out, n, y);
            } else {
                // only the first piece can go on from a wavefront's in front, and only the last one into another's
                if (runs >> piece & 1) { later = sum; later_piece = piece; }
                else { earlier = sum; }
            }
            sum = 0.0f;
            piece = i + j + 1;
        }
    }
    if (!(runs >> begin & 1))
        join_piece<GT, N, ACCUMULATE>(L, keys, __builtin_amdgcn_readlane(key, begin), block, front, behind, false, earlier, lane, slice, slices,
                                      n, col);
    if (later_piece >= 0)
        join_piece<GT, N, ACCUMULATE>(L, keys, __builtin_amdgcn_readlane(key, later_piece), block, front, behind, true, later, lane, slice,
                                      slices, n, col);
}

// Short lists, in one launch without a sort: a workgroup per token and up to four slices of columns.  It looks through the list, and
// where its token is the first of its row adds the dout of all of them, a wavefront per slice; of more than kBatch tokens the
// wavefronts that a slice has take a part each.  A row of more than kDirectPiece tokens is added by the workgroups of every
// kDirectPiece-th of them, and the last one adds their sums.  Further workgroups clear the rows without a token.
constexpr int kDirectPart = kDirectTokens / kDirectWaves;
constexpr int kDirectPiece = 64;        // us, 2048 tokens of 768 bf16, half of them / all of one row: by one workgroup 63 / 121, now 16 / 24

template <bool WIDE, int GT>
__device__ __forceinline__ void clear_absent_direct(const EmbeddingGradLaunch& L, int64_t first, int lane)
{
    const TokenReader<WIDE> read(L.t);
    const int num = (int)L.t.num;
    uint32_t here = 0;
    for (int i = lane; i < num; i += 64) {
        bool outside;
        const uint32_t row = read(i, &outside), r = row - (uint32_t)first;
        if (row != ~0u && r < kDirectClear) here |= 1u << r;
    }
    for (int r = 0; r < kDirectClear; ++r)
        if (!__ballot(here >> r & 1) && first + r < L.t.rows) clear_row<GT>(L, first + r, lane);
}

template <bool WIDE, int DT, int GT, int N>
__global__ void __launch_bounds__(64 * kDirectWaves)
k_sum_direct(EmbeddingGradLaunch L, int slices, int log_group_slices, int groups_per_token, int sum_groups)
{
    typedef typename Run<QADAM_F32, N>::F F;
    typedef typename Element<DT>::T D;
    typedef typename Element<GT>::T G;
    __shared__ int list[kDirectWaves][kDirectPart], found[kDirectWaves], in_front[kDirectWaves];
    __shared__ F sums[kDirectWaves][64];
    const int lane = threadIdx.x % 64, wave = __builtin_amdgcn_readfirstlane(threadIdx.x / 64), num = (int)L.t.num;
    if ((int)blockIdx.x >= sum_groups) {
        clear_absent_direct<WIDE, GT>(L, ((int64_t)((int)blockIdx.x - sum_groups) * kDirectWaves + wave) * kDirectClear, lane);
        return;
    }
    const TokenReader<WIDE> read(L.t);
    const int group = blockIdx.x % groups_per_token, t = blockIdx.x / groups_per_token;
    // the wavefront's part of the list, with the workgroup's token under way beside it
    constexpr int kLoads = kDirectPart / 64;
    bool outside;
    const uint32_t own_row = read(t, &outside);
    uint32_t other[kLoads];
#pragma unroll
    for (int k = 0; k < kLoads; ++k) {
        const int i = wave * kDirectPart + k * 64 + lane;
        bool unused;
        other[k] = ~0u;
        if (i < num) other[k] = read(i, &unused);
    }
    const uint32_t row = __builtin_amdgcn_readfirstlane(own_row);
    if (row == ~0u) {
        if (outside && group == 0 && threadIdx.x == 0) atomicOr(L.t.status, QADAM_STATUS_TOKEN_RANGE);
        return;
    }
    int count = 0, front = 0;               // of the row's tokens, those in front of t
#pragma unroll
    for (int k = 0; k < kLoads; ++k) {
        const int i = wave * kDirectPart + k * 64 + lane;
        const uint64_t same = __ballot(other[k] == row);
        if (!same) continue;
        front += __popcll(__ballot(other[k] == row && i < t));
        if (same >> lane & 1) list[wave][count + lanes_below(same)] = i;
        count += __popcll(same);
    }
    if (lane == 0) { found[wave] = count; in_front[wave] = front; }
    __syncthreads();
    int total = 0, index = 0, before[kDirectWaves];
    for (int w = 0; w < kDirectWaves; ++w) {
        before[w] = total;
        total += found[w];
        index += in_front[w];
    }
    if (index % kDirectPiece != 0) return;
    // the position of the row's token m
    auto position = [&](int m) {
        int part = 0;
        for (int w = 1; w < kDirectWaves; ++w) part = m >= before[w] && found[w] > 0 ? w : part;
        return list[part][m - before[part]];
    };
    const int stop = index + kDirectPiece < total ? index + kDirectPiece : total;
    const int group_slices = 1 << log_group_slices, slice = group * group_slices + wave % group_slices, turn = wave >> log_group_slices;
    const int turns = stop - index > kBatch ? kDirectWaves >> log_group_slices : 1;
    if (turns == 1 && (turn > 0 || slice >= slices)) return;
    const int share = (stop - index + turns - 1) / turns;
    const int begin = index + turn * share, end = begin + share < stop ? begin + share : stop;
    const int own = (slice * 64 + lane) * N;
    const int n = L.dim - own < 0 ? 0 : L.dim - own < N ? L.dim - own : N, col = n == N ? own : L.dim - N;
    const D* from = static_cast<const D*>(L.dout) + col;
    G* out = static_cast<G*>(L.grad) + col + (int64_t)row * L.grad_stride;
    typename Run<GT, N>::V old;
    if (L.accumulate && turn == 0) old = load_raw<GT, N, false>(out);
    F sum = 0.0f;
    for (int i = begin; i < end; i += kBatch) {
        // lane j has the position of the batch's token j
        const int at = position(i + lane % kBatch < end ? i + lane % kBatch : end - 1);
        typename Run<DT, N>::V x[kBatch];
#pragma unroll
        for (int j = 0; j < kBatch; ++j) x[j] = load_raw<DT, N, false>(from + (int64_t)__builtin_amdgcn_readlane(at, j) * L.dout_stride);
#pragma unroll
        for (int j = 0; j < kBatch; ++j)
            if (i + j < end) sum += to_float<DT, N>(x[j]);
    }
    if (turns > 1) {
        sums[wave][lane] = sum;
        __syncthreads();
        if (turn > 0) return;
        for (int u = 1; u < turns; ++u) sum += sums[wave + u * group_slices][lane];
    }
    if (total > kDirectPiece) {
        // as in join_piece; a piece's place is its first token's, the row's count that of the row's first token
        if (slice >= slices) return;
        float* put = L.w.pieces + (int64_t)t * L.dim + col;
#pragma unroll
        for (int k = 0; k < N; ++k)
            if (k >= N - n) __hip_atomic_store(global(put + k), sum[k], __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
        asm volatile("s_waitcnt vmcnt(0)" ::: "memory");
        uint32_t* arrived = L.w.arrived + (int64_t)__builtin_amdgcn_readfirstlane(position(0)) * slices + slice;
        const int pieces = (total + kDirectPiece - 1) / kDirectPiece;
        int come = 0;
        if (lane == 0) come = (int)__hip_atomic_fetch_add(global(arrived), 1u, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
        if (__builtin_amdgcn_readfirstlane(come) != pieces - 1) return;
        asm volatile("" ::: "memory");
        if (lane == 0) __hip_atomic_store(global(arrived), 0u, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
        sum = 0.0f;
        for (int b = 0; b < pieces; b += kBatch) {
            const int at = position((b + lane % kBatch < pieces ? b + lane % kBatch : pieces - 1) * kDirectPiece);
            F x[kBatch];
#pragma unroll
            for (int j = 0; j < kBatch; ++j) {
                const float* get = L.w.pieces + (int64_t)__builtin_amdgcn_readlane(at, j) * L.dim + col;
#pragma unroll
                for (int k = 0; k < N; ++k) x[j][k] = __hip_atomic_load(global(get + k), __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
            }
#pragma unroll
            for (int j = 0; j < kBatch; ++j)
                if (b + j < pieces) sum += x[j];
        }
    }
    F y = sum * L.scale;
    if (L.accumulate) y = to_float<GT, N>(old) + y;
    store_columns<GT, N>(out, n, y);
}

}  // namespace

template <int WT>
static hipError_t lookup_of(const LookupLaunch& L, int64_t runs)
{
    hipLaunchKernelGGL(k_lookup<WT>, dim3((unsigned)((L.t.num * runs + kThreads - 1) / kThreads)), dim3(kThreads), 0, L.stream, L,
                       (uint32_t)runs);
    return hipGetLastError();
}

hipError_t launch_embedding_lookup(const LookupLaunch& all)
{
    // a launch's runs are counted in 32 bits
    const int64_t runs = (all.dim + kRun - 1) / kRun, part = ((int64_t)1 << 31) / runs;
    for (int64_t at = 0; at < all.t.num; at += part) {
        LookupLaunch L = all;
        L.t.tokens = static_cast<const char*>(all.t.tokens) + at * all.t.bytes;
        L.t.num = all.t.num - at < part ? all.t.num - at : part;
        L.out = static_cast<char*>(all.out) + at * all.out_stride * element_size(all.out_type);
        hipError_t e = hipErrorInvalidValue;
        switch (L.weight_type) {
        case QADAM_F32: e = lookup_of<QADAM_F32>(L, runs); break;
        case QADAM_BF16: e = lookup_of<QADAM_BF16>(L, runs); break;
        case QADAM_F16: e = lookup_of<QADAM_F16>(L, runs); break;
        case QADAM_CODES8: e = lookup_of<QADAM_CODES8>(L, runs); break;
        case QADAM_CODES16: e = lookup_of<QADAM_CODES16>(L, runs); break;
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

template <int DT, int GT, int N>
static hipError_t grad_of(const EmbeddingGradLaunch& L)
{
    const int64_t num = L.t.num;
    const int slices = column_slices(L.dim);
    int64_t clear_rows = L.accumulate ? 0 : L.t.rows;       // of the gradient, the first ones: if they have no token
    if (num <= direct_tokens(L.dim)) {
        const int log_slices = log_group_slices(L.dim), groups = groups_per_token(L.dim), sums = (int)num * groups;
        const dim3 grid((unsigned)(sums + direct_clear_groups(clear_rows))), block(64 * kDirectWaves);
        if (grid.x == 0) return hipSuccess;
        if (L.t.bytes == 8)
            hipLaunchKernelGGL((k_sum_direct<true, DT, GT, N>), grid, block, 0, L.stream, L, slices, log_slices, groups, sums);
        else
            hipLaunchKernelGGL((k_sum_direct<false, DT, GT, N>), grid, block, 0, L.stream, L, slices, log_slices, groups, sums);
        return hipGetLastError();
    }
    const int row_bits = bits_of((uint64_t)L.t.rows), bits = bits_of((uint64_t)num);
    int result = 0;
    int group_bits = 0;
    if (num <= kGroupTokens && row_bits <= kMostGroupBits + kSortBits) {
        group_bits = row_bits - kSortBits > kGroupBits ? row_bits - kSortBits : kGroupBits;
        const int digit = row_bits > group_bits ? row_bits - group_bits : 0;
        if (!L.accumulate) clear_rows -= early_rows(num, L.t.rows, (int64_t)L.dim * element_size(GT));
        const int64_t early = L.accumulate ? 0 : L.t.rows - clear_rows;
        constexpr int kEach = kGroupWaves * kClearRows;
        const dim3 grid((unsigned)((1 << group_bits) + 1 + (early + kEach - 1) / kEach)), block(kGroupThreads);
        if (L.t.bytes == 8) hipLaunchKernelGGL((k_group<true, GT>), grid, block, 0, L.stream, L, bits, digit, group_bits, clear_rows);
        else hipLaunchKernelGGL((k_group<false, GT>), grid, block, 0, L.stream, L, bits, digit, group_bits, clear_rows);
        if (const hipError_t e = hipGetLastError()) return e;
    } else {
        const int passes = (row_bits + kSortBits - 1) / kSortBits, digit = (row_bits + passes - 1) / passes;
        const int tiles = (int)sort_tiles(num);
        for (int k = 0; k < passes; ++k) {
            const SortPass P{k ? L.w.keys[(k - 1) & 1] : nullptr, k ? L.w.order[(k - 1) & 1] : nullptr, L.w.keys[k & 1], L.w.order[k & 1],
                             k * digit, digit, tiles};
            hipLaunchKernelGGL(k_count_digits, dim3(tiles), dim3(kThreads), 0, L.stream, L, P);
            if (const hipError_t e = hipGetLastError()) return e;
            hipLaunchKernelGGL(k_move_digits, dim3(tiles), dim3(kThreads), 0, L.stream, L, P);
            if (const hipError_t e = hipGetLastError()) return e;
            result = k & 1;
        }
    }
    const int sums = (int)qadam::sum_groups(num, L.dim);
    const dim3 grid((unsigned)(sums + clear_groups(clear_rows))), block(64);
    if (L.accumulate) hipLaunchKernelGGL((k_sum_runs<DT, GT, N, true>), grid, block, 0, L.stream, L, result, slices, sums, group_bits, clear_rows);
    else hipLaunchKernelGGL((k_sum_runs<DT, GT, N, false>), grid, block, 0, L.stream, L, result, slices, sums, group_bits, clear_rows);
    return hipGetLastError();
}

template <int DT, int GT>
static hipError_t grad_of(const EmbeddingGradLaunch& L)
{
    switch (lane_columns(L.dim)) {
    case 4: return grad_of<DT, GT, 4>(L);
    case 2: return grad_of<DT, GT, 2>(L);
    default: return grad_of<DT, GT, 1>(L);
    }
}

template <int DT>
static hipError_t grad_of(const EmbeddingGradLaunch& L)
{
    if (L.grad_type == QADAM_F32) return grad_of<DT, QADAM_F32>(L);
    if (L.grad_type == QADAM_BF16) return grad_of<DT, QADAM_BF16>(L);
    return grad_of<DT, QADAM_F16>(L);
}

hipError_t launch_embedding_grad(const EmbeddingGradLaunch& L)
{
    if (L.dout_type == QADAM_F32) return grad_of<QADAM_F32>(L);
    if (L.dout_type == QADAM_BF16) return grad_of<QADAM_BF16>(L);
    return grad_of<QADAM_F16>(L);
}

}  // namespace qadam
