// gfx950 kernels of layer norm and its gradient.
//
// Both are bound by memory: a row is read once and stays in registers over its sums, the next one is on the way meanwhile, and results
// stream past the caches.  16384 rows of 2048 bf16: forward 24 us (134 MB, 5.6 TB/s), backward 36 (201 MB, 5.6 TB/s) and 5 for the sums over
// rows; of 8192 fp32, per call, 246 us (4.4 TB/s) and 346 (4.7), bf16 109 and 157; 8191 rows of 1001 f16 at odd addresses 14.4 and 3.9; 1024 rows
// of 768 fp32 5.0 and 4.3, which are two chains of loads.
// Where a row ends within a lane's run, its last 8 elements are loaded as a whole run: backward of 8191 rows of 2047 bf16 27.8 us per call (of 2048
// 23.2), with loads of single elements 58.
// The variance is taken of differences from the mean, in a second pass over registers: sums of squares would cancel where rows lie far from 0.
#include <type_traits>

#include "qadam_layers.h"
#include "qadam_row.h"

namespace qadam {
namespace {

static_assert(kRowRun == kNormRun, "one run");
constexpr int kThreads = 256;                   // of a workgroup of the kernels without rows of their own
constexpr int group_threads(int lanes) { return lanes < kThreads ? kThreads : lanes; }      // of the others, `lanes` of them to a row

// Sums over the LANES lanes that share a row, 16 or whole wavefronts, the same in all of them.  `at`: places in LDS of this use alone.
template <int LANES>
__device__ __forceinline__ float lanes_sum(float x)
{
    if constexpr (LANES >= 64) return wave_sum(x);
    x += moved<0xb1>(x);
    x += moved<0x4e>(x);
    x += moved<0x141>(x);
    return x + moved<0x140>(x);
}

template <int LANES>
__device__ __forceinline__ float row_sum(float x, float* at)
{
    x = lanes_sum<LANES>(x);
    if constexpr (LANES > 64) {
        if (threadIdx.x % 64 == 0) at[threadIdx.x / 64] = x;
        __syncthreads();
        x = at[0];
#pragma unroll
        for (int w = 1; w < LANES / 64; ++w) x += at[w];
    }
    return x;
}

// ... of two at once
template <int LANES>
__device__ __forceinline__ void row_sums(float& x, float& y, float* at)
{
    x = lanes_sum<LANES>(x);
    y = lanes_sum<LANES>(y);
    if constexpr (LANES > 64) {
        constexpr int kWaves = LANES / 64;
        if (threadIdx.x % 64 == 0) { at[threadIdx.x / 64] = x; at[kWaves + threadIdx.x / 64] = y; }
        __syncthreads();
        x = at[0];
        y = at[kWaves];
#pragma unroll
        for (int w = 1; w < kWaves; ++w) { x += at[w]; y += at[kWaves + w]; }
    }
}

// a b + c, rounded once: the library is built without contraction
__device__ __forceinline__ f8 fused(f8 a, f8 b, f8 c)
{
    f8 y;
#pragma unroll
    for (int i = 0; i < kRowRun; ++i) y[i] = __builtin_fmaf(a[i], b[i], c[i]);
    return y;
}

// the first n elements, zeros behind them
__device__ __forceinline__ f8 first_of(f8 x, int n)
{
#pragma unroll
    for (int i = 0; i < kRowRun; ++i) x[i] = i < n ? x[i] : 0.0f;
    return x;
}

// What a lane holds of a row: RUNS runs of kRowRun elements, LANES lanes apart.
template <int LANES, int RUNS>
struct Lane {
    int lane, dim;
    __device__ __forceinline__ Lane(int d) : lane(threadIdx.x % LANES), dim(d) {}
    __device__ __forceinline__ int at(int k) const { return (k * LANES + lane) * kRowRun; }
    __device__ __forceinline__ int left(int k) const { return dim - at(k); }
    // of a workgroup's rows the one that this lane has a part of
    __device__ __forceinline__ int row() const
    {
        if constexpr (LANES < 64) return threadIdx.x / LANES;
        else return __builtin_amdgcn_readfirstlane(threadIdx.x / LANES);
    }
};

template <int LANES, int RUNS, int TYPE, bool REPEAT = false>
__device__ __forceinline__ void load_row(const Lane<LANES, RUNS>& l, const void* base, int64_t offset,
                                         typename Run<TYPE, kRowRun>::V (&out)[RUNS])
{
    const auto* p = static_cast<const typename Element<TYPE>::T*>(base) + offset;
#pragma unroll
    for (int k = 0; k < RUNS; ++k) {
        out[k] = 0;
        if (REPEAT || l.left(k) > 0) out[k] = load_ahead<TYPE, REPEAT>(p, l.at(k), l.dim);
    }
}

template <int LANES, int RUNS>
__device__ __forceinline__ void load_vector(const Lane<LANES, RUNS>& l, const void* base, int type, float missing, f8 (&out)[RUNS])
{
#pragma unroll
    for (int k = 0; k < RUNS; ++k) {
        out[k] = missing;
        if (base && l.left(k) > 0) out[k] = load_part(base, type, l.at(k), l.left(k));
    }
}

// Forward: LANES lanes hold a row in registers, take another one after it, which is on the way meanwhile, and keep the weights in registers.
template <int LANES, int RUNS, int XT>
__global__ void __launch_bounds__(group_threads(LANES)) k_layer_norm(NormForward L)
{
    __shared__ float sums[2][2][LANES / 64 + 1];
    constexpr int kRows = group_threads(LANES) / LANES;
    const Lane<LANES, RUNS> l(L.dim);
    const int64_t step = (int64_t)gridDim.x * kRows;
    int64_t row = (int64_t)blockIdx.x * kRows + l.row();
    if (row >= L.rows) return;
    typename Run<XT, kRowRun>::V raw[RUNS];
    load_row<LANES, RUNS, XT>(l, L.x, row * L.x_stride, raw);
    f8 w[RUNS], b[RUNS];
    load_vector(l, L.weight, L.weight_type, 1.0f, w);
    load_vector(l, L.bias, L.weight_type, 0.0f, b);
    const float inv = 1.0f / (float)L.dim;
    for (int turn = 0; row < L.rows; row += step, turn ^= 1) {
        f8 x[RUNS];
        float sum = 0.0f, squares = 0.0f;
#pragma unroll
        for (int k = 0; k < RUNS; ++k) {
            x[k] = loaded<XT>(raw[k], l.at(k), l.dim);
#pragma unroll
            for (int i = 0; i < kRowRun; ++i) sum += x[k][i];
        }
        if (row + step < L.rows) load_row<LANES, RUNS, XT>(l, L.x, (row + step) * L.x_stride, raw);
        const float mean = row_sum<LANES>(sum, sums[turn][0]) * inv;
#pragma unroll
        for (int k = 0; k < RUNS; ++k) {
            x[k] -= mean;
            if (l.left(k) < kRowRun) x[k] = first_of(x[k], l.left(k));
#pragma unroll
            for (int i = 0; i < kRowRun; ++i) squares = __builtin_fmaf(x[k][i], x[k][i], squares);
        }
        const float rstd = 1.0f / sqrtf(row_sum<LANES>(squares, sums[turn][1]) * inv + L.eps);
#pragma unroll
        for (int k = 0; k < RUNS; ++k)
            if (l.left(k) > 0) store_part(L.out, L.out_type, row * L.out_stride + l.at(k), fused(x[k] * rstd, w[k], b[k]), l.left(k));
        if (l.lane == 0) {
            if (L.mean) global(L.mean)[row] = mean;
            if (L.rstd) global(L.rstd)[row] = rstd;
        }
    }
}

// Rows that are too long for registers: a workgroup reads each three times, from the caches after the first; the gradient's kernels do so
// together.  us per call, forward and gradient: 16384 rows of 9001 fp32 455 and 897 (2.6 and 2.0 TB/s of what has to
// move), bf16 432 and 942; 2048 rows of 65536 fp32 320 and 687, bf16 170 and 577; 64 rows of 2^20 fp32 449 and 1162.
constexpr int kLongWaves = 16;

__global__ void __launch_bounds__(64 * kLongWaves) k_layer_norm_long(NormForward L)
{
    __shared__ float sums[2][2][kLongWaves];
    const float inv = 1.0f / (float)L.dim;
    int turn = 0;
    for (int64_t row = blockIdx.x; row < L.rows; row += gridDim.x, turn ^= 1) {
        float sum = 0.0f, squares = 0.0f;
        for (int at = threadIdx.x * kRowRun; at < L.dim; at += 64 * kLongWaves * kRowRun) {
            const f8 x = load_part(L.x, L.x_type, row * L.x_stride + at, L.dim - at);
#pragma unroll
            for (int i = 0; i < kRowRun; ++i) sum += x[i];
        }
        const float mean = row_sum<64 * kLongWaves>(sum, sums[turn][0]) * inv;
        for (int at = threadIdx.x * kRowRun; at < L.dim; at += 64 * kLongWaves * kRowRun) {
            const f8 x = load_part(L.x, L.x_type, row * L.x_stride + at, L.dim - at) - mean;
#pragma unroll
            for (int i = 0; i < kRowRun; ++i) squares += i < L.dim - at ? x[i] * x[i] : 0.0f;
        }
        const float rstd = 1.0f / sqrtf(row_sum<64 * kLongWaves>(squares, sums[turn][1]) * inv + L.eps);
        for (int at = threadIdx.x * kRowRun; at < L.dim; at += 64 * kLongWaves * kRowRun) {
            f8 y = (load_part(L.x, L.x_type, row * L.x_stride + at, L.dim - at) - mean) * rstd;
            if (L.weight) y *= load_part(L.weight, L.weight_type, at, L.dim - at);
            if (L.bias) y += load_part(L.bias, L.weight_type, at, L.dim - at);
            store_part(L.out, L.out_type, row * L.out_stride + at, y, L.dim - at);
        }
        if (threadIdx.x == 0) {
            if (L.mean) global(L.mean)[row] = mean;
            if (L.rstd) global(L.rstd)[row] = rstd;
        }
    }
}

// Backward: as forward, and every lane adds its columns of dweight and dbias over the rows that it takes; a workgroup's sums go to
// scratch and k_norm_sums adds those.
template <int LANES, int RUNS, int DT, int XT>
__global__ void __launch_bounds__(group_threads(LANES)) k_layer_norm_grad(NormBackward L)
{
    __shared__ float sums[2][2 * (LANES / 64) + 1];
    extern __shared__ __attribute__((aligned(16))) float columns[];          // of several rows at a time: dweight and dbias of each
    constexpr int kRows = group_threads(LANES) / LANES;
    const Lane<LANES, RUNS> l(L.dim);
    const int64_t step = (int64_t)gridDim.x * kRows;
    int64_t row = (int64_t)blockIdx.x * kRows + l.row();
    typename Run<DT, kRowRun>::V raw_dy[RUNS];
    typename Run<XT, kRowRun>::V raw_x[RUNS];
    float mean = 0.0f, rstd = 0.0f;
    auto load = [&](int64_t r) {
        load_row<LANES, RUNS, DT>(l, L.dout, r * L.dout_stride, raw_dy);
        load_row<LANES, RUNS, XT, true>(l, L.x, r * L.x_stride, raw_x);
        mean = global(L.mean)[r];
        rstd = global(L.rstd)[r];
    };
    if (row < L.rows) load(row);
    f8 w[RUNS], dw[RUNS], db[RUNS];
    load_vector(l, L.weight, L.weight_type, 1.0f, w);
#pragma unroll
    for (int k = 0; k < RUNS; ++k) dw[k] = db[k] = 0.0f;
    const float inv = 1.0f / (float)L.dim;
    for (int turn = 0; row < L.rows; row += step, turn ^= 1) {
        f8 g[RUNS], xh[RUNS];
        float sum = 0.0f, along = 0.0f;
        const float r = rstd;
#pragma unroll
        for (int k = 0; k < RUNS; ++k) {
            const f8 dy = loaded<DT>(raw_dy[k], l.at(k), l.dim);
            // Behind the row's end dout is 0, so that nothing there enters a sum while xh is finite, which (0 - mean) rstd need not be: x repeats
            // elements of the row there.
            xh[k] = (loaded<XT, true>(raw_x[k], l.at(k), l.dim) - mean) * r;
            db[k] += dy;
            dw[k] = fused(dy, xh[k], dw[k]);
            g[k] = dy * w[k];
#pragma unroll
            for (int i = 0; i < kRowRun; ++i) {
                sum += g[k][i];
                along = __builtin_fmaf(g[k][i], xh[k][i], along);
            }
        }
        if (row + step < L.rows) load(row + step);
        row_sums<LANES>(sum, along, sums[turn]);
        const float c1 = sum * inv, c2 = -(along * inv);
#pragma unroll
        for (int k = 0; k < RUNS; ++k)
            if (l.left(k) > 0) store_part(L.dx, L.dx_type, row * L.dx_stride + l.at(k), fused(xh[k], (f8)c2, g[k] - c1) * r, l.left(k));
    }
    if (!L.dweight && !L.dbias) return;
    float* out = L.partial + (int64_t)blockIdx.x * 2 * L.dim;
    if constexpr (kRows > 1) {
        constexpr int width = RUNS * LANES * kRowRun;
        float* own = columns + l.row() * 2 * width;
#pragma unroll
        for (int k = 0; k < RUNS; ++k) {
            *(f8*)(own + l.at(k)) = dw[k];
            *(f8*)(own + width + l.at(k)) = db[k];
        }
        __syncthreads();
        for (int i = threadIdx.x; i < L.dim; i += group_threads(LANES)) {
            float a = columns[i], b = columns[width + i];
#pragma unroll
            for (int v = 1; v < kRows; ++v) { a += columns[v * 2 * width + i]; b += columns[v * 2 * width + width + i]; }
            global(out)[i] = a;
            global(out)[L.dim + i] = b;
        }
    } else {
#pragma unroll
        for (int k = 0; k < RUNS; ++k)
            if (l.left(k) > 0) {
                store_part<QADAM_F32, false>(out + l.at(k), dw[k], l.left(k));
                store_part<QADAM_F32, false>(out + L.dim + l.at(k), db[k], l.left(k));
            }
    }
}

// ... of rows that are too long for registers: the sums over rows first, a lane per column and a slice of the rows per workgroup,
__global__ void __launch_bounds__(kThreads) k_norm_columns(NormBackward L)
{
    const int column = blockIdx.x * kThreads + threadIdx.x;
    if (column >= L.dim) return;
    float dw = 0.0f, db = 0.0f;
    for (int64_t row = blockIdx.y; row < L.rows; row += gridDim.y) {
        const float dy = load_one(L.dout, L.dout_type, row * L.dout_stride + column);
        dw += dy * ((load_one(L.x, L.x_type, row * L.x_stride + column) - global(L.mean)[row]) * global(L.rstd)[row]);
        db += dy;
    }
    float* out = L.partial + (int64_t)blockIdx.y * 2 * L.dim;
    global(out)[column] = dw;
    global(out)[L.dim + column] = db;
}

// ... then dx, which may replace what the sums read.
__global__ void __launch_bounds__(64 * kLongWaves) k_layer_norm_grad_long(NormBackward L)
{
    __shared__ float sums[2][2][kLongWaves];
    const float inv = 1.0f / (float)L.dim;
    int turn = 0;
    for (int64_t row = blockIdx.x; row < L.rows; row += gridDim.x, turn ^= 1) {
        const float mean = global(L.mean)[row], rstd = global(L.rstd)[row];
        auto run = [&](int at, f8& g, f8& xh) {
            const int n = L.dim - at;
            g = load_part(L.dout, L.dout_type, row * L.dout_stride + at, n);
            if (L.weight) g *= load_part(L.weight, L.weight_type, at, n);
            xh = first_of((load_part(L.x, L.x_type, row * L.x_stride + at, n) - mean) * rstd, n);
        };
        float sum = 0.0f, along = 0.0f;
        f8 g, xh;
        for (int at = threadIdx.x * kRowRun; at < L.dim; at += 64 * kLongWaves * kRowRun) {
            run(at, g, xh);
#pragma unroll
            for (int i = 0; i < kRowRun; ++i) {
                sum += g[i];
                along += g[i] * xh[i];
            }
        }
        const float c1 = row_sum<64 * kLongWaves>(sum, sums[turn][0]) * inv, c2 = row_sum<64 * kLongWaves>(along, sums[turn][1]) * inv;
        for (int at = threadIdx.x * kRowRun; at < L.dim; at += 64 * kLongWaves * kRowRun) {
            run(at, g, xh);
            store_part(L.dx, L.dx_type, row * L.dx_stride + at, (g - c1 - xh * c2) * rstd, L.dim - at);
        }
    }
}

// dweight and dbias: a workgroup per kSumColumns columns, whose threads take a slice of the workgroups' sums each, in fp64.  512 sums of 2048
// columns, 8 MB: 4.8 us; with 64 columns and 16 slices in a workgroup, so on a quarter of the CUs, 9.7.
constexpr int kSumThreads = 1024, kSumColumns = 16, kSumSlices = kSumThreads / kSumColumns;

__device__ __forceinline__ void store_one(void* p, int type, int64_t i, float x)
{
    if (type == QADAM_F32) global(static_cast<float*>(p))[i] = x;
    else if (type == QADAM_BF16) global(static_cast<__bf16*>(p))[i] = (__bf16)x;
    else global(static_cast<_Float16*>(p))[i] = (_Float16)x;
}

__global__ void __launch_bounds__(kSumThreads) k_norm_sums(NormBackward L, int groups)
{
    __shared__ double slices[kSumSlices][kSumColumns];
    const int c = threadIdx.x % kSumColumns, slice = threadIdx.x / kSumColumns, i = blockIdx.x * kSumColumns + c;
    double sum = 0.0;
    if (i < 2 * L.dim) {
#pragma unroll 8
        for (int k = slice; k < groups; k += kSumSlices) sum += (double)global(L.partial)[(int64_t)k * 2 * L.dim + i];
    }
    slices[slice][c] = sum;
#pragma unroll
    for (int half = kSumSlices / 2; half > 0; half /= 2) {
        __syncthreads();
        if (slice < half) slices[slice][c] += slices[slice + half][c];
    }
    if (slice != 0 || i >= 2 * L.dim) return;
    sum = slices[0][c];
    void* to = i < L.dim ? L.dweight : L.dbias;
    if (!to) return;
    const int column = i < L.dim ? i : i - L.dim;
    if (L.accumulate) sum += (double)load_one(to, L.grad_type, column);
    store_one(to, L.grad_type, column, (float)sum);
}

// workgroups of rows, `each` rows at a time, at most `most`
int groups_of(int64_t rows, int each, int most)
{
    const int64_t n = (rows + each - 1) / each;
    return (int)(n < most ? n : most);
}

// Lanes and runs per row, by its width.  us per call with rows in the registers of a wavefront / of as many as here: 16384 rows of 2048
// bf16 forward 25.7 / 25.8, backward 66 / 42.9; with a wavefront / 16 lanes: 40000 rows of 64 bf16 12.2 / 4.9 and 18.9 / 8.6.  Beyond 4096 columns
// a workgroup of 16 wavefronts has a CU to itself (the gradient's 102 and more registers), and nothing runs while it waits for a row's sums:
// 16384 rows of 8192 fp32 reach 4.4 and 4.7 TB/s where rows of 4096 reach 5.0; more runs on fewer lanes were not measured.
template <typename F>
void by_width(int dim, F&& body)
{
    if (dim <= 128) body(std::integral_constant<int, 16>(), std::integral_constant<int, 1>());
    else if (dim <= 512) body(std::integral_constant<int, 64>(), std::integral_constant<int, 1>());
    else if (dim <= 1024) body(std::integral_constant<int, 64>(), std::integral_constant<int, 2>());
    else if (dim <= 2048) body(std::integral_constant<int, 256>(), std::integral_constant<int, 1>());
    else if (dim <= 4096) body(std::integral_constant<int, 512>(), std::integral_constant<int, 1>());
    else body(std::integral_constant<int, 1024>(), std::integral_constant<int, 1>());
}

template <int XT>
void forward(const NormForward& L)
{
    by_width(L.dim, [&](auto lanes, auto runs) {
        constexpr int kGroup = group_threads(lanes.value);
        k_layer_norm<lanes.value, runs.value, XT><<<dim3(groups_of(L.rows, kGroup / lanes.value, 262144 / kGroup)), dim3(kGroup), 0, L.stream>>>(L);
    });
}

template <int DT, int XT>
void backward(const NormBackward& L, int* groups)
{
    by_width(L.dim, [&](auto lanes, auto runs) {
        constexpr int kGroup = group_threads(lanes.value), kRows = kGroup / lanes.value;
        *groups = groups_of(L.rows, kRows, norm_partials(L.dim));
        const int lds = kRows > 1 ? kRows * 2 * runs.value * lanes.value * kRowRun * (int)sizeof(float) : 0;
        k_layer_norm_grad<lanes.value, runs.value, DT, XT><<<dim3(*groups), dim3(kGroup), lds, L.stream>>>(L);
    });
}

template <int DT>
void backward(const NormBackward& L, int* groups)
{
    if (L.x_type == QADAM_F32) backward<DT, QADAM_F32>(L, groups);
    else if (L.x_type == QADAM_BF16) backward<DT, QADAM_BF16>(L, groups);
    else backward<DT, QADAM_F16>(L, groups);
}

}  // namespace

hipError_t launch_layer_norm(const NormForward& L)
{
    if (L.dim > kNormHeldDim) {
        k_layer_norm_long<<<dim3(groups_of(L.rows, 1, 512)), dim3(64 * kLongWaves), 0, L.stream>>>(L);
        return hipGetLastError();
    }
    if (L.x_type == QADAM_F32) forward<QADAM_F32>(L);
    else if (L.x_type == QADAM_BF16) forward<QADAM_BF16>(L);
    else forward<QADAM_F16>(L);
    return hipGetLastError();
}

hipError_t launch_layer_norm_grad(const NormBackward& L)
{
    int groups = 0;
    if (L.rows > 0 && L.dim > kNormHeldDim) {
        if (L.dweight || L.dbias) {
            groups = groups_of(L.rows, 1, norm_partials(L.dim));
            k_norm_columns<<<dim3((L.dim + kThreads - 1) / kThreads, groups), dim3(kThreads), 0, L.stream>>>(L);
        }
        k_layer_norm_grad_long<<<dim3(groups_of(L.rows, 1, 512)), dim3(64 * kLongWaves), 0, L.stream>>>(L);
    } else if (L.rows > 0) {
        if (L.dout_type == QADAM_F32) backward<QADAM_F32>(L, &groups);
        else if (L.dout_type == QADAM_BF16) backward<QADAM_BF16>(L, &groups);
        else backward<QADAM_F16>(L, &groups);
    }
    if ((L.dweight || L.dbias) && (L.rows > 0 || !L.accumulate))
        k_norm_sums<<<dim3((2 * L.dim + kSumColumns - 1) / kSumColumns), dim3(kSumThreads), 0, L.stream>>>(L, groups);
    return hipGetLastError();
}

}  // namespace qadam
