// gfx950 kernel of sampling.
#include "qadam_layers.h"
#include "qadam_row.h"

namespace qadam {
namespace {

constexpr int kThreads = 1024, kWaves = kThreads / 64;
constexpr int kDigitBits = 8, kDigits = 1 << kDigitBits;

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

// round(2^40 exp((x - largest) / temperature))
__device__ __forceinline__ uint64_t mass_of(float x, float largest, double temperature)
{
    if (x == largest) return (uint64_t)1 << 40;
    const double e = exp(((double)x - (double)largest) / temperature);
    return (uint64_t)rint(e * 0x1p40);
}

struct Found {
    uint32_t key;           // of the element
    int64_t  nth;           // of those with this key, from 1 on, in the order of their indexes
    uint64_t sum;           // of the masses up to it and with it
};

struct Row {
    const SampleLaunch& L;
    int64_t offset;
    float largest;
    double temperature;
    uint64_t* hist_mass;    // [kDigits], in LDS
    uint32_t* hist_count;
    Found* found;

    __device__ __forceinline__ float logit(int64_t i) const { return load_one(L.logits, L.logits_type, offset + i); }

    // The first element in descending order at which the count of elements reaches `count` (> 0), or, with count 0, the sum of masses
    // reaches `target` (`beyond`: is beyond it).
    __device__ Found find(int64_t count, double target, bool beyond) const
    {
        uint32_t prefix = 0;
        uint64_t sum_before = 0;
        int64_t count_before = 0;
        for (int shift = 32 - kDigitBits; shift >= 0; shift -= kDigitBits) {
            __syncthreads();
            for (int i = threadIdx.x; i < kDigits; i += kThreads) { hist_mass[i] = 0; hist_count[i] = 0; }
            __syncthreads();
            for (int64_t i = threadIdx.x; i < L.vocab; i += kThreads) {
                const float x = logit(i);
                const uint32_t key = key_of(x);
                if (shift + kDigitBits < 32 && key >> (shift + kDigitBits) != prefix) continue;
                const int d = key >> shift & (kDigits - 1);
                atomicAdd(&hist_count[d], 1u);
                atomicAdd((unsigned long long*)&hist_mass[d], (unsigned long long)mass_of(x, largest, temperature));
            }
            __syncthreads();
            if (threadIdx.x == 0) {
                int d = 0;
                uint64_t m = sum_before;
                int64_t c = count_before;
                for (; d < kDigits - 1; ++d) {
                    const uint64_t m2 = m + hist_mass[d];
                    const int64_t c2 = c + hist_count[d];
                    if (hist_count[d] && (count > 0 ? c2 >= count : beyond ? (double)m2 > target : (double)m2 >= target)) break;
                    m = m2; c = c2;
                }
                found->key = (uint32_t)d; found->nth = c; found->sum = m;
            }
            __syncthreads();
            prefix = prefix << kDigitBits | found->key;
            count_before = found->nth;
            sum_before = found->sum;
        }
        // equal elements have equal masses
        const uint64_t m = mass_of(logit_of(prefix), largest, temperature);
        int64_t nth = 1;
        const int64_t equal = hist_count[prefix & (kDigits - 1)];
        if (count > 0) {
            nth = count - count_before;
        } else if (m > 0) {
            const double before = (double)sum_before;
            nth = (int64_t)((target - before) / (double)m);
            nth = nth < 1 ? 1 : nth > equal ? equal : nth;
            auto enough = [&](int64_t n) {
                const double s = (double)(sum_before + (uint64_t)n * m);
                return beyond ? s > target : s >= target;
            };
            while (nth > 1 && enough(nth - 1)) --nth;
            while (nth < equal && !enough(nth)) ++nth;
        }
        return {prefix, nth, sum_before + (uint64_t)nth * m};
    }
};

__global__ void __launch_bounds__(kThreads) k_sample(SampleLaunch L)
{
    __shared__ uint64_t hist_mass[kDigits];
    __shared__ uint32_t hist_count[kDigits];
    __shared__ Found found;
    __shared__ uint32_t wave_key[kWaves], wave_equal[kWaves], wave_nan[kWaves];
    __shared__ uint64_t kept;
    const int lane = threadIdx.x % 64, wave = threadIdx.x / 64;
    for (int64_t row = blockIdx.x; row < L.rows; row += gridDim.x) {
        const double temperature = L.filters.temperatures ? (double)global(L.filters.temperatures)[row] : (double)L.filters.temperature;
        const int32_t top_k = L.filters.top_ks ? global(L.filters.top_ks)[row] : L.filters.top_k;
        const double top_p = L.filters.top_ps ? (double)global(L.filters.top_ps)[row] : (double)L.filters.top_p;
        const double min_p = L.filters.min_ps ? (double)global(L.filters.min_ps)[row] : (double)L.filters.min_p;
        Row r{L, row * L.logits_stride, 0.0f, temperature, hist_mass, hist_count, &found};
        uint32_t smallest = ~0u;
        bool nan = false;
        for (int64_t i = threadIdx.x; i < L.vocab; i += kThreads) {
            const float x = r.logit(i);
            nan |= x != x;
            const uint32_t k = key_of(x);
            smallest = smallest < k ? smallest : k;
        }
        for (int k = 32; k > 0; k /= 2) {
            const uint32_t other = (uint32_t)__shfl_xor((int)smallest, k);
            smallest = smallest < other ? smallest : other;
        }
        const bool any_nan = __ballot(nan) != 0;
        __syncthreads();
        if (lane == 0) { wave_key[wave] = smallest; wave_nan[wave] = any_nan; }
        if (threadIdx.x == 0) kept = 0;
        __syncthreads();
        bool none = !(temperature >= 0.0 && temperature < (double)__builtin_inff());
        for (int w = 0; w < kWaves; ++w) {
            smallest = smallest < wave_key[w] ? smallest : wave_key[w];
            none |= wave_nan[w] != 0;
        }
        r.largest = logit_of(smallest);
        none |= r.largest == -__builtin_inff();
        int64_t token = -1;
        if (!none) {
            Found at{smallest, 1, 0};
            if (temperature > 0.0) {
                uint64_t total = 0, least = 0;
                for (int64_t i = threadIdx.x; i < L.vocab; i += kThreads) {
                    const uint64_t m = mass_of(r.logit(i), r.largest, temperature);
                    total += m;
                    if (!(min_p > 0.0) || (double)m >= (min_p < 1.0 ? min_p : 1.0) * 0x1p40) least += m;
                }
                atomicAdd((unsigned long long*)&kept, (unsigned long long)total);
                __syncthreads();
                uint64_t sum = kept;
                __syncthreads();
                if (threadIdx.x == 0) kept = 0;
                __syncthreads();
                atomicAdd((unsigned long long*)&kept, (unsigned long long)least);
                __syncthreads();
                const uint64_t sum_least = kept;
                if (top_k > 0 && top_k < L.vocab) sum = r.find(top_k, 0.0, false).sum;
                if (top_p < 1.0) sum = r.find(0, (top_p > 0.0 ? top_p : 0.0) * (double)sum, false).sum;
                sum = sum < sum_least ? sum : sum_least;
                float u = global(L.u)[row];
                u = !(u > 0.0f) ? 0.0f : u < 1.0f ? u : 0x1.fffffep-1f;
                at = r.find(0, (double)u * (double)sum, true);
            }
            // the nth of the elements with this key: wavefronts take parts of the row one behind the other
            const int64_t part = (L.vocab + kThreads - 1) / kThreads * 64, begin = wave * part, end = begin + part < L.vocab ? begin + part : L.vocab;
            int64_t count = 0;
            for (int64_t i0 = begin; i0 < end; i0 += 64) count += __popcll(__ballot(i0 + lane < end && key_of(r.logit(i0 + lane < end ? i0 + lane : 0)) == at.key));
            if (lane == 0) wave_equal[wave] = (uint32_t)count;
            __syncthreads();
            int64_t before = 0;
            for (int w = 0; w < wave; ++w) before += wave_equal[w];
            if (before < at.nth && at.nth <= before + count) {
                for (int64_t i0 = begin; i0 < end; i0 += 64) {
                    const bool equal = i0 + lane < end && key_of(r.logit(i0 + lane < end ? i0 + lane : 0)) == at.key;
                    const uint64_t mask = __ballot(equal);
                    const int ahead = __builtin_amdgcn_mbcnt_hi((uint32_t)(mask >> 32), __builtin_amdgcn_mbcnt_lo((uint32_t)mask, 0));
                    if (equal && before + ahead + 1 == at.nth) {
                        if (L.token_bytes == 4) global(static_cast<int32_t*>(L.out))[row] = (int32_t)(i0 + lane);
                        else global(static_cast<int64_t*>(L.out))[row] = i0 + lane;
                    }
                    before += __popcll(mask);
                }
            }
        } else if (threadIdx.x == 0) {
            if (L.token_bytes == 4) global(static_cast<int32_t*>(L.out))[row] = (int32_t)token;
            else global(static_cast<int64_t*>(L.out))[row] = token;
            atomicOr(L.status, QADAM_STATUS_NO_TOKEN);
        }
    }
}

}  // namespace

hipError_t launch_sample(const SampleLaunch& L)
{
    k_sample<<<dim3((int)(L.rows < 65536 ? L.rows : 65536)), dim3(kThreads), 0, L.stream>>>(L);
    return hipGetLastError();
}

}  // namespace qadam
