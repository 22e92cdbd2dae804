// gfx950 kernel of sampling: a workgroup per row, which is read a few times, from the caches after the first.
//
// All filters keep the first tokens of one order, so none of them needs the tokens sorted: what a filter leaves is known by its sum of
// masses, and the token is where the sum in that order passes u times the smallest of them.  Masses are integers, whose sums are the
// same in any order: workgroups add them in LDS with atomics and the result is the same on every run.  The logits are sorted into
// kBins bins of equal width, from the largest on down to where masses vanish.  Bins are in the order of the logits, so that a sum is
// found by looking through the bins and then through one bin's tokens, which are few:
//   * top_k up to kMostTopK: the largest logit of each thread gives a bin that at least top_k tokens lie in or in front of; those (a few
//     more than top_k) are listed, and no mass of another token is taken.  The same where min_p is the only filter: it names the bin;
//   * else the masses of all tokens are added by bins, and each of the sums that are asked for takes one more pass, which lists a
//     bin's tokens;
//   * where the bin of a sum holds more than kList (2048) tokens: by digits of the logits, four passes with atomics for each sum.
// The last of these is slow, and not for many equal logits alone.  One row of 50257 fp32 of deviation 2, top_k 50 and top_p 0.95, takes 12.6 us
// at a temperature of 0.3, but 417 at 0.1, 468 at 0.3 with one token 14 above the others, and 840 where all but 40 tokens have the lowest
// finite fp32 (minus infinity: 13): fewer than top_k threads hold a logit within 29 temperatures of the largest, so that the last bin, whose tokens
// have no mass, is listed, found too long and searched by digits.  (Elementary torch operations take 290.)  One row of 128256 of deviation 0.3, top_p
// 0.9, takes 362 us with one temperature up to 1 for all rows, which leaves the bins 29 temperatures wide in all, and 65 with a temperature of its
// own, for which the smallest logit is looked for too.
//
// Bound by the instructions of one CU per row.  One row of 50257 fp32, top_k 50: 12.7 us, of which the list takes about 5, the threads' bins
// and sums 2 each.  256 rows of 50257 bf16 with filters of their own 49: of top_p's 92 thousand cycles the masses take 38 (31 operations per token,
// most of them in fp64) and the two lists 12 to 21 each.  33 rows of 32003 fp16 24.7; by digits throughout they took 300.  A run is looked at, and
// what another thread has of it masked, in its turn: masked as it is loaded, which waits for it, 14.6, 56.8 and 28.6; two runs under way
// 13.7, 51.7 and 25.3.  kBins of 2048, 4096 and 8192, bf16, top_p 0.9: 256 rows of 50257 37.8, 36.1 and 39.7 (behind top_k 2000 43.0, 44.4 and 49.0),
// 1000 rows of 5000 52.4, 56.5 and 70.8; 256 flat rows of 128256 501, 126 and 136.
#include "qadam_layers.h"
#include "qadam_row.h"

namespace qadam {
namespace {

constexpr int kThreads = 1024, kWaves = kThreads / 64;
constexpr int kDigitBits = 8, kDigits = 1 << kDigitBits;
constexpr int kBins = 2048, kThreadBins = kBins / kThreads;
constexpr int kList = 2048, kThreadList = kList / kThreads;
constexpr int kPairs = 512;             // tokens of a list that are ordered by comparing pairs
constexpr int kMostTopK = 512;          // top_k up to which the threads' largest logits name the candidates

// Order of logits as integers: the largest logit has the smallest key, equal logits (0 and -0 too) the same one.
__device__ __forceinline__ uint32_t key_of(float x)
{
    const uint32_t b = __builtin_bit_cast(uint32_t, x + 0.0f);
    return b >> 31 ? b : ~b & 0x7fffffffu;
}

__device__ __forceinline__ float logit_of(uint32_t key)
{
    return __builtin_bit_cast(float, key >> 31 ? key : ~key & 0x7fffffffu);
}

constexpr float kInf = __builtin_inff();

constexpr float kMost = 0x1.fffffep+127f;       // infinite logits count as this

// round(2^40 exp((x - largest) / temperature)): 2^y = 2^n 2^r with n = round(y) and r from -1/2 to 1/2, where the polynomial of degree 9 that
// meets 2^r at the ten Chebyshev nodes is within 2^-46 of it: 1/67 of a unit.  Beside 1.5 2^52 the last place of a number is 1, so
// that adding it rounds, and leaves n in the lower bits.
struct Mass {
    float largest;
    double per_unit;        // log2(e) / temperature

    __device__ __forceinline__ uint64_t operator()(float x) const
    {
        constexpr double kRound = 0x1.8p52;
        const double y = fmax(((double)x - (double)largest) * per_unit, -100.0);
        const double rounded = y + kRound, r = y - (rounded - kRound);
        const double r2 = r * r, r4 = r2 * r2;
        // by pairs, which do not wait for each other; 2^40 is in the coefficients
        const double e01 = __builtin_fma(0x1.62e42fefa39f7p+39, r, 0x1.000000000003dp+40);
        const double e23 = __builtin_fma(0x1.c6b08d704411ap+35, r, 0x1.ebfbdff8149f2p+37);
        const double e45 = __builtin_fma(0x1.5d87fe908f74fp+30, r, 0x1.3b2ab72b175efp+33);
        const double e67 = __builtin_fma(0x1.ffcb7678c7b33p+23, r, 0x1.43088e257ed10p+27);
        const double e89 = __builtin_fma(0x1.b6571dbf753eep+16, r, 0x1.63ef969af1055p+20);
        const double e = __builtin_fma(__builtin_fma(__builtin_fma(e89, r2, e67), r2, e45), r4, __builtin_fma(e23, r2, e01));
        // e is above 2^39 and below 2^41, n from -100 to 0: 2^n is an addition to the exponent, in the upper half
        const uint64_t bits = __builtin_bit_cast(uint64_t, e);
        const uint32_t high = (uint32_t)(bits >> 32) + ((uint32_t)__builtin_bit_cast(uint64_t, rounded) << 20);
        const double m = __builtin_bit_cast(double, (uint64_t)high << 32 | (uint32_t)bits) + 0x1p52;
        return __builtin_bit_cast(uint64_t, m) & 0xfffffffffffffull;
    }
};

// Bin of a logit, 0 for the largest: never falls where logits fall.
struct Bin {
    float largest, per_unit;

    __device__ __forceinline__ int operator()(float x) const { return (int)fminf((largest - x) * per_unit, (float)(kBins - 1)); }
};

struct Found {
    uint32_t key;           // of the element
    int64_t  nth;           // of those with this key, from 1 on, in the order of their indexes
    uint64_t sum;           // of the masses up to it and with it
};

// where a sum of masses passes `target` (beyond), or reaches it
struct Target {
    double value;
    bool   beyond;
    __device__ __forceinline__ bool operator()(uint64_t sum) const { return beyond ? (double)sum > value : (double)sum >= value; }
};

struct RowFilters {
    double temperature, top_p, min_p;
    int32_t top_k;
    float u;
};

struct Shared {
    RowFilters filters;
    uint64_t mass[kBins];
    uint32_t count[kBins];
    uint64_t list[kList];       // key << 32 | index: smaller in front
    uint64_t run[kList];        // sum of the masses of the list's up to this one and with it
    uint16_t rank[kList];       // its place in the order, from 1 on
    uint64_t wave_sum[2][kWaves];
    uint32_t wave_key[kWaves], wave_low[kWaves], wave_nan[kWaves], wave_equal[kWaves];
    uint64_t least;             // sum of the masses that reach min_p
    uint32_t listed, first;
    int      min_p_bin;
    // what a search leaves
    int64_t  place;
    uint64_t before, sum;
    Found    found;
};

template <int CTRL, int ROWS = 0xf>
__device__ __forceinline__ uint64_t moved_sum(uint64_t x)
{
    const uint32_t low = (uint32_t)__builtin_amdgcn_update_dpp(0, (int)(uint32_t)x, CTRL, ROWS, 0xf, false);
    const uint32_t high = (uint32_t)__builtin_amdgcn_update_dpp(0, (int)(uint32_t)(x >> 32), CTRL, ROWS, 0xf, false);
    return x + ((uint64_t)high << 32 | low);
}

// Sum of x over the threads in front of this one; `total`: of all.  `turn` alternates between uses.
__device__ __forceinline__ uint64_t sum_ahead(Shared& s, uint64_t x, int turn, uint64_t* total)
{
    const int lane = threadIdx.x % 64, wave = threadIdx.x / 64;
    uint64_t run = x;
    // the lane 1, 2, 4 and 8 places in front within rows of 16, then the last of the row in front, then lane 31
    run = moved_sum<0x111>(run);
    run = moved_sum<0x112>(run);
    run = moved_sum<0x114>(run);
    run = moved_sum<0x118>(run);
    run = moved_sum<0x142, 0xa>(run);
    run = moved_sum<0x143, 0xc>(run);
    if (lane == 63) s.wave_sum[turn][wave] = run;
    __syncthreads();
    // every row of 16 lanes adds the wavefronts' sums
    static_assert(kWaves == 16, "a row of lanes");
    uint64_t all = s.wave_sum[turn][lane % 16];
    all = moved_sum<0x111>(all);
    all = moved_sum<0x112>(all);
    all = moved_sum<0x114>(all);
    all = moved_sum<0x118>(all);
    auto of_lane = [&](int from) {
        return (uint64_t)(uint32_t)__builtin_amdgcn_readlane((int)(uint32_t)(all >> 32), from) << 32 |
               (uint32_t)__builtin_amdgcn_readlane((int)(uint32_t)all, from);
    };
    *total = of_lane(15);
    const uint64_t before = wave > 0 ? of_lane(__builtin_amdgcn_readfirstlane(wave - 1)) : 0;
    return before + run - x;
}

// SHORT: a vocabulary below kRowRun
template <int LT, bool SHORT>
struct Row {
    typedef typename Element<LT>::T T;
    Shared& s;
    const T* logits;
    int vocab;
    Mass mass;
    Bin bin;
    bool infinite;          // the largest logit is

    __device__ __forceinline__ float logit(int i) const { return fminf((float)global(logits)[i], kMost); }

    // kRowRun logits from `start` on, which is in front of `from` where the row ends before a whole run
    __device__ __forceinline__ typename Run<LT, kRowRun>::V load(int from, int* start) const
    {
        *start = SHORT || from + kRowRun <= vocab ? from : vocab - kRowRun;
        if constexpr (!SHORT) return load_raw<LT, kRowRun, false>(logits + *start);
        typename Run<LT, kRowRun>::V raw = (T)-kInf;
#pragma unroll
        for (int e = 0; e < kRowRun - 1; ++e)
            if (e < vocab) raw[e] = global(logits)[e];
        return raw;
    }

    // body(run of logits, index of the first): all of the row, minus infinity where another run has a logit too; a thread's next run is under
    // way meanwhile, so what was loaded is not looked at before its turn
    template <typename F>
    __device__ __forceinline__ void each(F&& body) const
    {
        constexpr int kAcross = kThreads * kRowRun;
        int at = threadIdx.x * kRowRun, next_start = 0;
        if (at >= vocab) return;
        typename Run<LT, kRowRun>::V next = load(at, &next_start);
#pragma unroll 1
        while (true) {
            f8 x = to_float<LT, kRowRun>(next);
            const int start = next_start;
            if (start < at) {
#pragma unroll
                for (int e = 0; e < kRowRun; ++e) x[e] = start + e < at ? -kInf : x[e];
            }
            if (infinite) {
#pragma unroll
                for (int e = 0; e < kRowRun; ++e) x[e] = fminf(x[e], kMost);
            }
            at += kAcross;
            if (at < vocab) next = load(at, &next_start);
            body(x, start);
            if (at >= vocab) return;
        }
    }

    // The tokens of the bins lo to hi (never those that are minus infinity) into the list, with their places in the order and the sums up
    // to them; their number, which may be beyond kList: then there is no list.
    __device__ __forceinline__ int collect(int lo, int hi) const
    {
        __syncthreads();
        if (threadIdx.x == 0) s.listed = 0;
        __syncthreads();
        // where these bins lie, and a little more; what is within is looked at closer
        const float width = 1.0f / bin.per_unit, slack = 0x1p-19f * (fabsf(bin.largest) + (float)(hi + 1) * width);
        const float least = hi < kBins - 1 ? fmaxf(bin.largest - (float)(hi + 1) * width - slack, -kMost) : -kMost;
        // differences that are not negative are in the order of their bits, in front of all that are negative
        const uint32_t within = __builtin_bit_cast(uint32_t, fmaxf(bin.largest - (float)lo * width + slack - least, 0.0f));
        each([&](f8 x, int at) {
            typedef uint32_t u8 __attribute__((ext_vector_type(kRowRun)));
            const u8 above = __builtin_bit_cast(u8, x - least);
            uint32_t nearest = above[0];
#pragma unroll
            for (int e = 1; e < kRowRun; ++e) nearest = above[e] < nearest ? above[e] : nearest;
            if (nearest > within) return;
            uint32_t take = 0;
#pragma unroll
            for (int e = 0; e < kRowRun; ++e) take |= (above[e] <= within ? 1u : 0u) << e;
            // few are taken: one place in the list after the other
            while (take) {
                const int e = __builtin_ctz(take);
                take &= take - 1;
                float v = x[0];
#pragma unroll
                for (int k = 1; k < kRowRun; ++k) v = e == k ? x[k] : v;
                const int b = bin(v);
                if (b < lo || b > hi) continue;
                const uint32_t to = atomicAdd(&s.listed, 1u);
                if (to < kList) s.list[to] = (uint64_t)key_of(v) << 32 | (uint32_t)(at + e);
            }
        });
        __syncthreads();
        const int n = (int)s.listed;
        if (n > kList) return n;
        if (n <= kPairs) {
            // `share` threads for a token, each of which looks at a part of the others
            if ((int)threadIdx.x < n) s.run[threadIdx.x] = listed_mass(threadIdx.x);
            __syncthreads();
            int share = 64;
            while (share > 1 && share * n > kThreads) share /= 2;
            const int i = threadIdx.x / share;
            uint64_t sum = 0;
            uint32_t rank = 0;
            if (i < n) {
                const uint64_t own = s.list[i];
                for (int j = threadIdx.x % share; j < n; j += share) {
                    const bool ahead = s.list[j] <= own;
                    sum += ahead ? s.run[j] : 0;
                    rank += ahead;
                }
            }
            for (int k = 1; k < share; k *= 2) {
                sum += (uint64_t)(uint32_t)__shfl_xor((int)(sum >> 32), k) << 32 | (uint32_t)__shfl_xor((int)(uint32_t)sum, k);
                rank += (uint32_t)__shfl_xor((int)rank, k);
            }
            __syncthreads();
            if (i < n && threadIdx.x % share == 0) { s.run[i] = sum; s.rank[i] = (uint16_t)rank; }
            __syncthreads();
            return n;
        }
        // sorted: by merging runs of which every other one is the other way round
        int size = 2 * kPairs;
        while (size < n) size *= 2;
        for (int i = n + threadIdx.x; i < size; i += kThreads) s.list[i] = ~0ull;
        for (int run = 2; run <= size; run *= 2)
            for (int step = run / 2; step > 0; step /= 2) {
                __syncthreads();
                for (int p = threadIdx.x; p < size / 2; p += kThreads) {
                    const int i = p / step * 2 * step + p % step;
                    const uint64_t a = s.list[i], b = s.list[i + step];
                    if ((a > b) == ((i & run) == 0)) { s.list[i] = b; s.list[i + step] = a; }
                }
            }
        __syncthreads();
        uint64_t m[kThreadList], own = 0, total;
#pragma unroll
        for (int k = 0; k < kThreadList; ++k) {
            const int i = threadIdx.x * kThreadList + k;
            own += m[k] = i < n ? listed_mass(i) : 0;
        }
        uint64_t sum = sum_ahead(s, own, 0, &total);
#pragma unroll
        for (int k = 0; k < kThreadList; ++k) {
            const int i = threadIdx.x * kThreadList + k;
            s.run[i] = sum += m[k];
            s.rank[i] = (uint16_t)(i + 1);
        }
        __syncthreads();
        return n;
    }

    __device__ __forceinline__ uint64_t listed_mass(int i) const { return mass(logit_of((uint32_t)(s.list[i] >> 32))); }

    // The token of the list at which the sum, from `before` on, satisfies `target`: s.place (of the list), s.sum
    __device__ __forceinline__ void search(int n, uint64_t before, Target target) const
    {
        for (int i = threadIdx.x; i < n; i += kThreads) {
            const uint64_t m = listed_mass(i), to = before + s.run[i];
            if (m > 0 && target(to) && !target(to - m)) { s.place = i; s.sum = to; }
        }
        __syncthreads();
    }

    // The bin in which the sum of s.mass (or s.count) satisfies `target`: s.place, and in s.before the sum in front of it.  Returns the sum
    // of all.
    __device__ __forceinline__ uint64_t search_bins(bool counts, Target target, int turn) const
    {
        uint64_t v[kThreadBins], own = 0, total;
        const int first = threadIdx.x * kThreadBins;
#pragma unroll
        for (int k = 0; k < kThreadBins; ++k) own += v[k] = counts ? s.count[first + k] : s.mass[first + k];
        uint64_t run = sum_ahead(s, own, turn, &total);
#pragma unroll
        for (int k = 0; k < kThreadBins; ++k) {
            if (target(run + v[k]) && !target(run)) { s.place = first + k; s.before = run; }
            run += v[k];
        }
        __syncthreads();
        return total;
    }

    // The first element in descending order at which the count of elements reaches `count` (> 0), or the sum of masses satisfies `target`:
    // by digits of the keys, of rows with many equal logits; leaves it in s.found
    __device__ __forceinline__ void by_digits(int64_t count, Target target) const
    {
        uint32_t prefix = 0;
        uint64_t sum_before = 0;
        int64_t count_before = 0;
        for (int shift = 32 - kDigitBits; shift >= 0; shift -= kDigitBits) {
            __syncthreads();
            for (int i = threadIdx.x; i < kDigits; i += kThreads) { s.mass[i] = 0; s.count[i] = 0; }
            __syncthreads();
            for (int i = threadIdx.x; i < vocab; i += kThreads) {
                const float x = logit(i);
                const uint32_t key = key_of(x);
                if (shift + kDigitBits < 32 && key >> (shift + kDigitBits) != prefix) continue;
                const int d = key >> shift & (kDigits - 1);
                atomicAdd(&s.count[d], 1u);
                atomicAdd((unsigned long long*)&s.mass[d], (unsigned long long)mass(x));
            }
            __syncthreads();
            if (threadIdx.x == 0) {
                int d = 0;
                uint64_t m = sum_before;
                int64_t c = count_before;
                for (; d < kDigits - 1; ++d) {
                    const uint64_t m2 = m + s.mass[d];
                    const int64_t c2 = c + s.count[d];
                    if (s.count[d] && (count > 0 ? c2 >= count : target(m2))) break;
                    m = m2; c = c2;
                }
                s.found.key = (uint32_t)d; s.found.nth = c; s.found.sum = m;
            }
            __syncthreads();
            prefix = prefix << kDigitBits | s.found.key;
            count_before = s.found.nth;
            sum_before = s.found.sum;
        }
        // equal elements have equal masses
        const uint64_t m = mass(logit_of(prefix));
        int64_t nth = 1;
        const int64_t equal = s.count[prefix & (kDigits - 1)];
        if (count > 0) {
            nth = count - count_before;
        } else if (m > 0) {
            nth = (int64_t)((target.value - (double)sum_before) / (double)m);
            nth = nth < 1 ? 1 : nth > equal ? equal : nth;
            while (nth > 1 && target(sum_before + (uint64_t)(nth - 1) * m)) --nth;
            while (nth < equal && !target(sum_before + (uint64_t)nth * m)) ++nth;
        }
        __syncthreads();
        if (threadIdx.x == 0) s.found = {prefix, nth, sum_before + (uint64_t)nth * m};
        __syncthreads();
    }

    // Index of the nth of the elements with a key, in s.place: wavefronts take parts of the row one behind the other.
    __device__ __forceinline__ void nth_of(uint32_t key, int64_t nth) const
    {
        const int lane = threadIdx.x % 64, wave = threadIdx.x / 64;
        const int part = (vocab + kThreads - 1) / kThreads * 64, begin = wave * part, end = begin + part < vocab ? begin + part : vocab;
        int64_t count = 0;
        for (int i = begin; i < end; i += 64) count += __popcll(__ballot(i + lane < end && key_of(logit(i + lane < end ? i + lane : begin)) == key));
        __syncthreads();
        if (lane == 0) s.wave_equal[wave] = (uint32_t)count;
        __syncthreads();
        int64_t before = 0;
        for (int w = 0; w < wave; ++w) before += s.wave_equal[w];
        if (before < nth && nth <= before + count)
            for (int i = begin; i < end; i += 64) {
                const bool equal = i + lane < end && key_of(logit(i + lane < end ? i + lane : begin)) == key;
                const uint64_t mask = __ballot(equal);
                const int ahead = __builtin_amdgcn_mbcnt_hi((uint32_t)(mask >> 32), __builtin_amdgcn_mbcnt_lo((uint32_t)mask, 0));
                if (equal && before + ahead + 1 == nth) s.place = i + lane;
                before += __popcll(mask);
            }
        __syncthreads();
    }
};

// what the filters keep by mass, and the draw
__device__ __forceinline__ uint64_t least_mass(const RowFilters& f) { return (uint64_t)ceil((f.min_p < 1.0 ? f.min_p : 1.0) * 0x1p40); }
__device__ __forceinline__ Target target_count(int64_t count) { return {(double)count, false}; }
__device__ __forceinline__ Target target_p(const RowFilters& f, uint64_t sum)
{
    const double v = (f.top_p > 0.0 ? f.top_p : 0.0) * (double)sum;
    return {v > 1.0 ? v : 1.0, false};          // at least one
}
__device__ __forceinline__ Target target_u(const RowFilters& f, uint64_t sum) { return {(double)f.u * (double)sum, true}; }

// The bin of the logits whose masses round to what min_p asks for, to one on either side; kBins - 1 beyond the bins.
__device__ __forceinline__ int min_p_bin(const Bin& bin, const RowFilters& f)
{
    const float below = (float)(-log(((double)least_mass(f) - 0.5) * 0x1p-40) * f.temperature);
    return (int)fminf(fmaxf(below, 0.0f) * bin.per_unit, (float)(kBins - 1));
}

// The token of a row whose largest logit is known.  `last` >= 0: all tokens that can be drawn lie in the bins 0 to last.
// Sums are asked for one after the other, each only where its filter is: 1 that of the first top_k, 2 that of those that top_p leaves, 3 that
// of those that reach min_p, 4 the token's.
template <int LT, bool SHORT>
__device__ __forceinline__ int64_t draw(const Row<LT, SHORT>& r, const RowFilters& f, int last)
{
    Shared& s = r.s;
    const bool counts = f.top_k > 0, by_min_p = f.min_p > 0.0;
    bool all_listed = false;        // the list holds all that can be drawn
    bool binned = true;             // s.mass, s.count hold the bins
    bool in_list = false;
    int n = 0;
    uint64_t sum = 0;
#pragma unroll 1
    for (int ask = last >= 0 ? 0 : 1; ask <= 4; ++ask) {
        int lo = 0, hi = last;
        uint64_t before = 0;
        int64_t rest = counts ? f.top_k : kList;        // tokens of the list whose sum is asked for
        Target target{};
        if (ask < 2) {
            if (all_listed) continue;
            __syncthreads();
            if (threadIdx.x == 0) s.least = 0;
        }
        if (ask == 1) {
            for (int i = threadIdx.x; i < kBins; i += kThreads) { s.mass[i] = 0; s.count[i] = 0; }
            __syncthreads();
            r.each([&](f8 x, int) {
#pragma unroll
                for (int e = 0; e < kRowRun; ++e) {
                    const uint64_t m = r.mass(x[e]);
                    if (m > 0) atomicAdd((unsigned long long*)&s.mass[r.bin(x[e])], (unsigned long long)m);
                }
            });
            if (counts)
                r.each([&](f8 x, int) {
#pragma unroll
                    for (int e = 0; e < kRowRun; ++e) atomicAdd(&s.count[r.bin(x[e])], 1u);
                });
            __syncthreads();
            // all of them: no bin is asked for
            sum = r.search_bins(false, {__builtin_inf(), false}, 0);
            if (!counts) continue;
            target = target_count(f.top_k);
        } else if (ask == 2) {
            if (!(f.top_p < 1.0)) continue;
            target = target_p(f, sum);
        } else if (ask == 3) {
            if (!by_min_p) continue;
            __syncthreads();
            if (all_listed) {
                if (s.least < sum) sum = s.least;
                continue;
            }
        } else if (ask == 4) {
            target = target_u(f, sum);
        }
        if (ask > 0 && binned && !all_listed) {
            if (ask == 3) {
                // the bin in which masses reach min_p, and one more on either side
                const int at = s.min_p_bin;
                lo = at > 0 ? at - 1 : 0;
                hi = at + 1 < kBins ? at + 1 : kBins - 1;
            } else {
                r.search_bins(ask == 1, target, 1);
                lo = hi = (int)s.place;
                before = s.before;
            }
            if (ask == 1 || ask == 3) {
                // the masses in front of the bins
                rest = ask == 1 ? f.top_k - (int64_t)before : kList;
                uint64_t own = 0;
#pragma unroll
                for (int k = 0; k < kThreadBins; ++k) own += (int)threadIdx.x * kThreadBins + k < lo ? s.mass[threadIdx.x * kThreadBins + k] : 0;
                sum_ahead(s, own, 0, &before);
            }
        }
        if (binned && !all_listed) n = r.collect(lo, hi);
        if (binned && n <= kList) {
            if (ask < 2 || ask == 3) {
                // the sum of the list's first ones, and of those of them that reach min_p; a list without one: no sum
                if (threadIdx.x == 0) s.sum = 0;
                __syncthreads();
                const int kept = rest < n ? (int)rest : n;
                for (int i = threadIdx.x; i < n; i += kThreads) {
                    if (s.rank[i] == kept) s.sum = s.run[i];
                    if (ask != 1 && by_min_p && s.rank[i] <= kept && r.listed_mass(i) >= least_mass(f))
                        atomicMax((unsigned long long*)&s.least, (unsigned long long)s.run[i]);
                }
                __syncthreads();
                if (ask == 3) sum = before + s.least < sum ? before + s.least : sum;
                else sum = before + s.sum;
                all_listed = ask == 0;
            } else {
                r.search(n, before, target);
                sum = s.sum;
                in_list = true;
            }
            __syncthreads();
        } else if (ask == 3) {
            const uint64_t least = least_mass(f);
            uint64_t own = 0;
            for (int i = threadIdx.x; i < r.vocab; i += kThreads) {
                const uint64_t m = r.mass(r.logit(i));
                own += m >= least ? m : 0;
            }
            atomicAdd((unsigned long long*)&s.least, (unsigned long long)own);
            __syncthreads();
            if (s.least < sum) sum = s.least;
            __syncthreads();
        } else if (ask > 0) {
            binned = in_list = false;
            r.by_digits(ask == 1 ? f.top_k : 0, target);
            sum = s.found.sum;
        }
    }
    if (in_list) return (int64_t)(uint32_t)s.list[s.place];
    r.nth_of(s.found.key, s.found.nth);
    return s.place;
}

// The largest or smallest of a wavefront's values, the same in all lanes; none is NaN where it counts
template <bool LARGEST, int CTRL, int ROWS = 0xf>
__device__ __forceinline__ float extreme(float x)
{
    const int own = __builtin_bit_cast(int, x);
    const float other = __builtin_bit_cast(float, __builtin_amdgcn_update_dpp(own, own, CTRL, ROWS, 0xf, false));
    return LARGEST ? fmaxf(x, other) : fminf(x, other);
}

template <bool LARGEST>
__device__ __forceinline__ float wave_extreme(float x)
{
    x = extreme<LARGEST, 0xb1>(x);
    x = extreme<LARGEST, 0x4e>(x);
    x = extreme<LARGEST, 0x141>(x);
    x = extreme<LARGEST, 0x140>(x);
    x = extreme<LARGEST, 0x142, 0xa>(x);
    x = extreme<LARGEST, 0x143, 0xc>(x);
    return __builtin_bit_cast(float, __builtin_amdgcn_readlane(__builtin_bit_cast(int, x), 63));
}

template <int LT, bool SHORT>
__global__ void __launch_bounds__(kThreads) k_sample(SampleLaunch L, int64_t first_row)
{
    __shared__ Shared s;
    const int lane = threadIdx.x % 64, wave = threadIdx.x / 64;
    const int64_t row = first_row + blockIdx.x;
    // in LDS: not all of it would fit the registers of 16 wavefronts
    const RowFilters& f = s.filters;
    if (threadIdx.x == 0) {
        RowFilters own;
        own.temperature = L.filters.temperatures ? (double)global(L.filters.temperatures)[row] : (double)L.filters.temperature;
        own.top_k = L.filters.top_ks ? global(L.filters.top_ks)[row] : L.filters.top_k;
        own.top_p = L.filters.top_ps ? (double)global(L.filters.top_ps)[row] : (double)L.filters.top_p;
        own.min_p = L.filters.min_ps ? (double)global(L.filters.min_ps)[row] : (double)L.filters.min_p;
        own.u = global(L.u)[row];
        own.u = !(own.u > 0.0f) ? 0.0f : own.u < 1.0f ? own.u : 0x1.fffffep-1f;
        if (!(own.top_k > 0 && own.top_k < L.vocab)) own.top_k = 0;
        s.filters = own;
    }
    Row<LT, SHORT> r{s, static_cast<const typename Element<LT>::T*>(L.logits) + row * L.logits_stride, (int)L.vocab, {}, {}, false};

    // Largest, NaN; the smallest that is no minus infinity where bins could be much wider than they need be.
    float high = -kInf, low = kInf;
    bool nan = false;
    const bool wide = L.filters.temperatures || L.filters.temperature > 1.0f;
    r.each([&](f8 x, int) {
#pragma unroll
        for (int e = 0; e < kRowRun; e += 2) {
            nan |= __builtin_isunordered(x[e], x[e + 1]);
            high = fmaxf(fmaxf(high, x[e]), x[e + 1]);
        }
        if (wide) {
#pragma unroll
            for (int e = 0; e < kRowRun; ++e) low = fminf(low, x[e] == -kInf ? kInf : x[e]);
        }
    });
    float all_high = wave_extreme<true>(high), all_low = wave_extreme<false>(low);
    const bool any_nan = __ballot(nan) != 0;
    __syncthreads();
    if (lane == 0) { s.wave_key[wave] = __builtin_bit_cast(uint32_t, all_high); s.wave_low[wave] = __builtin_bit_cast(uint32_t, all_low); s.wave_nan[wave] = any_nan; }
    __syncthreads();
    bool none = !(f.temperature >= 0.0 && f.temperature < (double)kInf);
    for (int w = 0; w < kWaves; ++w) {
        all_high = fmaxf(all_high, __builtin_bit_cast(float, s.wave_key[w]));
        all_low = fminf(all_low, __builtin_bit_cast(float, s.wave_low[w]));
        none |= s.wave_nan[w] != 0;
    }
    r.infinite = all_high == kInf;
    all_high = fminf(all_high, kMost) + 0.0f;
    all_low = wide ? fminf(all_low, kMost) : -kInf;
    none |= all_high == -kInf;
    int64_t token = -1;
    if (!none && f.temperature == 0.0) {
        // the lowest index of the largest
        if (threadIdx.x == 0) s.first = ~0u;
        __syncthreads();
        uint32_t first = ~0u;
        r.each([&](f8 x, int at) {
#pragma unroll
            for (int e = kRowRun - 1; e >= 0; --e)
                if (x[e] == all_high && (uint32_t)(at + e) < first) first = (uint32_t)(at + e);
        });
        if (first != ~0u) atomicMin(&s.first, first);
        __syncthreads();
        token = s.first;
    } else if (!none) {
        const double log2e = 0x1.71547652b82fep+0;
        r.mass = {all_high, log2e / f.temperature};
        // bins down to where masses vanish, 29 temperatures below the largest, or to the smallest logit; any scale is right.  At most 2^126, so that
        // kBins times the width of one, rounded, is finite.
        const float range = fminf(fminf(29.0f * (float)f.temperature, all_high - all_low), 0x1p126f);
        const float scale = (float)(kBins - 1) / range;
        r.bin = {all_high, scale < 1e30f ? scale : 1e30f};
        const bool by_k = f.top_k > 0 && f.top_k <= kMostTopK, by_min_p = !by_k && f.top_k == 0 && !(f.top_p < 1.0) && f.min_p > 0.0;
        if (f.min_p > 0.0 && threadIdx.x == 0) s.min_p_bin = min_p_bin(r.bin, f);
        __syncthreads();
        int last = -1;
        if (by_k) {
            for (int i = threadIdx.x; i < kBins; i += kThreads) { s.mass[i] = 0; s.count[i] = 0; }
            __syncthreads();
            atomicAdd(&s.count[r.bin(fminf(high, kMost))], 1u);
            __syncthreads();
            r.search_bins(true, target_count(f.top_k), 0);
            last = (int)s.place;
        } else if (by_min_p) {
            last = s.min_p_bin + 1;
        }
        token = draw(r, f, last);
    }
    if (threadIdx.x == 0) {
        if (L.token_bytes == 4) global(static_cast<int32_t*>(L.out))[row] = (int32_t)token;
        else global(static_cast<int64_t*>(L.out))[row] = token;
        if (token < 0) atomicOr(L.status, QADAM_STATUS_NO_TOKEN);
    }
}

}  // namespace

hipError_t launch_sample(const SampleLaunch& L)
{
    // rows of a launch: fewer than 2^32 work-items
    for (int64_t row = 0; row < L.rows; row += 1 << 21) {
        const dim3 grid((int)(L.rows - row < 1 << 21 ? L.rows - row : 1 << 21));
        auto run = [&](auto kernel) { kernel<<<grid, dim3(kThreads), 0, L.stream>>>(L, row); };
        if (L.logits_type == QADAM_F32) L.vocab < kRowRun ? run(k_sample<QADAM_F32, true>) : run(k_sample<QADAM_F32, false>);
        else if (L.logits_type == QADAM_BF16) L.vocab < kRowRun ? run(k_sample<QADAM_BF16, true>) : run(k_sample<QADAM_BF16, false>);
        else L.vocab < kRowRun ? run(k_sample<QADAM_F16, true>) : run(k_sample<QADAM_F16, false>);
    }
    return hipGetLastError();
}

}  // namespace qadam
