// gfx950 kernels of layer norm and its gradient.
#include "qadam_layers.h"
#include "qadam_row.h"

namespace qadam {
namespace {

constexpr int kWaves = 4, kThreads = 64 * kWaves;
static_assert(kRowRun == kNormRun, "one run");

// Sum over the WAVES wavefronts that share a row, the same in all lanes.  `at`: a place in LDS of this use alone.
template <int WAVES>
__device__ __forceinline__ float row_sum(float x, float* at)
{
    x = wave_sum(x);
    if constexpr (WAVES > 1) {
        if (threadIdx.x % 64 == 0) at[threadIdx.x / 64] = x;
        __syncthreads();
        x = at[0];
#pragma unroll
        for (int w = 1; w < WAVES; ++w) x += at[w];
    }
    return x;
}

// What a lane holds of a row: RUNS runs of kRowRun elements, WAVES * 64 lanes apart.
template <int WAVES, int RUNS>
struct Lane {
    int lane, dim;
    __device__ __forceinline__ Lane(int d) : lane(WAVES == 1 ? threadIdx.x % 64 : threadIdx.x), dim(d) {}
    __device__ __forceinline__ int at(int k) const { return (k * WAVES * 64 + lane) * kRowRun; }
    __device__ __forceinline__ int left(int k) const { return dim - at(k); }
};

template <int WAVES, int RUNS, int TYPE>
__device__ __forceinline__ void load_row(const Lane<WAVES, RUNS>& l, const void* base, int64_t offset,
                                         typename Run<TYPE, kRowRun>::V (&out)[RUNS])
{
    const auto* p = static_cast<const typename Element<TYPE>::T*>(base) + offset;
#pragma unroll
    for (int k = 0; k < RUNS; ++k) {
        out[k] = 0;
        if (l.left(k) > 0) out[k] = load_part<TYPE, false>(p + l.at(k), l.left(k));
    }
}

template <int WAVES, int RUNS>
__device__ __forceinline__ void load_vector(const Lane<WAVES, RUNS>& l, const void* base, int type, float missing, f8 (&out)[RUNS])
{
#pragma unroll
    for (int k = 0; k < RUNS; ++k) {
        out[k] = missing;
        if (base && l.left(k) > 0) out[k] = load_part(base, type, l.at(k), l.left(k));
    }
}

// Forward: WAVES wavefronts hold a row in registers and take the next one after it; the weights stay in registers.
template <int WAVES, int RUNS, int XT>
__global__ void __launch_bounds__(kThreads) k_layer_norm(NormForward L)
{
    __shared__ float sums[2][2][kWaves];
    const Lane<WAVES, RUNS> l(L.dim);
    const int64_t step = (int64_t)gridDim.x * (kWaves / WAVES);
    int64_t row = (int64_t)blockIdx.x * (kWaves / WAVES) + (WAVES == 1 ? __builtin_amdgcn_readfirstlane(threadIdx.x / 64) : 0);
    if (row >= L.rows) return;
    typename Run<XT, kRowRun>::V raw[RUNS];
    load_row<WAVES, RUNS, XT>(l, L.x, row * L.x_stride, raw);
    f8 w[RUNS], b[RUNS];
    load_vector(l, L.weight, L.weight_type, 1.0f, w);
    load_vector(l, L.bias, L.weight_type, 0.0f, b);
    const float inv = 1.0f / (float)L.dim;
    for (int turn = 0; row < L.rows; row += step, turn ^= 1) {
        f8 x[RUNS];
        float sum = 0.0f, squares = 0.0f;
#pragma unroll
        for (int k = 0; k < RUNS; ++k) {
            x[k] = to_float<XT, kRowRun>(raw[k]);
#pragma unroll
            for (int i = 0; i < kRowRun; ++i) sum += x[k][i];
        }
        if (row + step < L.rows) load_row<WAVES, RUNS, XT>(l, L.x, (row + step) * L.x_stride, raw);
        const float mean = row_sum<WAVES>(sum, sums[turn][0]) * inv;
#pragma unroll
        for (int k = 0; k < RUNS; ++k) {
            x[k] -= mean;
#pragma unroll
            for (int i = 0; i < kRowRun; ++i) squares += i < l.left(k) ? x[k][i] * x[k][i] : 0.0f;
        }
        const float rstd = 1.0f / sqrtf(row_sum<WAVES>(squares, sums[turn][1]) * inv + L.eps);
#pragma unroll
        for (int k = 0; k < RUNS; ++k)
            if (l.left(k) > 0) store_part(L.out, L.out_type, row * L.out_stride + l.at(k), x[k] * rstd * w[k] + b[k], l.left(k));
        if (l.lane == 0) {
            if (L.mean) global(L.mean)[row] = mean;
            if (L.rstd) global(L.rstd)[row] = rstd;
        }
    }
}

// Rows that are too long for registers: a workgroup reads each three times, from the caches after the first.
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
        const float mean = row_sum<kLongWaves>(sum, sums[turn][0]) * inv;
        for (int at = threadIdx.x * kRowRun; at < L.dim; at += 64 * kLongWaves * kRowRun) {
            const f8 x = load_part(L.x, L.x_type, row * L.x_stride + at, L.dim - at) - mean;
#pragma unroll
            for (int i = 0; i < kRowRun; ++i) squares += i < L.dim - at ? x[i] * x[i] : 0.0f;
        }
        const float rstd = 1.0f / sqrtf(row_sum<kLongWaves>(squares, sums[turn][1]) * inv + L.eps);
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
template <int WAVES, int RUNS, int DT, int XT>
__global__ void __launch_bounds__(kThreads) k_layer_norm_grad(NormBackward L)
{
    __shared__ float sums[2][2][kWaves];
    extern __shared__ float columns[];          // WAVES == 1: [2][dim]
    const Lane<WAVES, RUNS> l(L.dim);
    const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x / 64);
    const int64_t step = (int64_t)gridDim.x * (kWaves / WAVES);
    int64_t row = (int64_t)blockIdx.x * (kWaves / WAVES) + (WAVES == 1 ? wave : 0);
    f8 w[RUNS], dw[RUNS], db[RUNS];
    load_vector(l, L.weight, L.weight_type, 1.0f, w);
#pragma unroll
    for (int k = 0; k < RUNS; ++k) dw[k] = db[k] = 0.0f;
    const float inv = 1.0f / (float)L.dim;
    typename Run<DT, kRowRun>::V raw_dy[RUNS];
    typename Run<XT, kRowRun>::V raw_x[RUNS];
    float mean = 0.0f, rstd = 0.0f;
    if (row < L.rows) {
        load_row<WAVES, RUNS, DT>(l, L.dout, row * L.dout_stride, raw_dy);
        load_row<WAVES, RUNS, XT>(l, L.x, row * L.x_stride, raw_x);
        mean = global(L.mean)[row];
        rstd = global(L.rstd)[row];
    }
    for (int turn = 0; row < L.rows; row += step, turn ^= 1) {
        f8 g[RUNS], xh[RUNS];
        float sum = 0.0f, along = 0.0f;
        const float r = rstd;
#pragma unroll
        for (int k = 0; k < RUNS; ++k) {
            const f8 dy = to_float<DT, kRowRun>(raw_dy[k]);
            xh[k] = (to_float<XT, kRowRun>(raw_x[k]) - mean) * r;
            // no dout behind the row's end: nothing there enters a sum
            db[k] += dy;
            dw[k] += dy * xh[k];
            g[k] = dy * w[k];
#pragma unroll
            for (int i = 0; i < kRowRun; ++i) {
                sum += g[k][i];
                along += g[k][i] * xh[k][i];
            }
        }
        const int64_t next = row + step;
        if (next < L.rows) {
            load_row<WAVES, RUNS, DT>(l, L.dout, next * L.dout_stride, raw_dy);
            load_row<WAVES, RUNS, XT>(l, L.x, next * L.x_stride, raw_x);
            mean = global(L.mean)[next];
            rstd = global(L.rstd)[next];
        }
        const float c1 = row_sum<WAVES>(sum, sums[turn][0]) * inv, c2 = row_sum<WAVES>(along, sums[turn][1]) * inv;
#pragma unroll
        for (int k = 0; k < RUNS; ++k)
            if (l.left(k) > 0) store_part(L.dx, L.dx_type, row * L.dx_stride + l.at(k), (g[k] - c1 - xh[k] * c2) * r, l.left(k));
    }
    if (!L.dweight && !L.dbias) return;
    float* out = L.partial + (int64_t)blockIdx.x * 2 * L.dim;
    if constexpr (WAVES == 1) {
        // the workgroup's wavefronts one after the other, so that the order is always the same
        for (int turn = 0; turn < kWaves; ++turn) {
            if (wave == turn) {
#pragma unroll
                for (int k = 0; k < RUNS; ++k)
#pragma unroll
                    for (int i = 0; i < kRowRun; ++i)
                        if (i < l.left(k)) {
                            const int at = l.at(k) + i;
                            columns[at] = turn == 0 ? dw[k][i] : columns[at] + dw[k][i];
                            columns[L.dim + at] = turn == 0 ? db[k][i] : columns[L.dim + at] + db[k][i];
                        }
            }
            __syncthreads();
        }
        for (int i = threadIdx.x; i < 2 * L.dim; i += kThreads) global(out)[i] = columns[i];
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
            xh = (load_part(L.x, L.x_type, row * L.x_stride + at, n) - mean) * rstd;
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
        const float c1 = row_sum<kLongWaves>(sum, sums[turn][0]) * inv, c2 = row_sum<kLongWaves>(along, sums[turn][1]) * inv;
        for (int at = threadIdx.x * kRowRun; at < L.dim; at += 64 * kLongWaves * kRowRun) {
            run(at, g, xh);
            store_part(L.dx, L.dx_type, row * L.dx_stride + at, (g - c1 - xh * c2) * rstd, L.dim - at);
        }
    }
}

// dweight and dbias: a wavefront per 64 columns and slice of the workgroups' sums, in fp64.
constexpr int kSumWaves = 16;

__device__ __forceinline__ void store_one(void* p, int type, int64_t i, float x)
{
    if (type == QADAM_F32) global(static_cast<float*>(p))[i] = x;
    else if (type == QADAM_BF16) global(static_cast<__bf16*>(p))[i] = (__bf16)x;
    else global(static_cast<_Float16*>(p))[i] = (_Float16)x;
}

__global__ void __launch_bounds__(64 * kSumWaves) k_norm_sums(NormBackward L, int groups)
{
    __shared__ double slices[kSumWaves][64];
    const int lane = threadIdx.x % 64, wave = threadIdx.x / 64, i = blockIdx.x * 64 + lane;
    double sum = 0.0;
    if (i < 2 * L.dim)
        for (int k = wave; k < groups; k += kSumWaves) sum += (double)global(L.partial)[(int64_t)k * 2 * L.dim + i];
    slices[wave][lane] = sum;
    __syncthreads();
    if (wave != 0 || i >= 2 * L.dim) return;
    for (int w = 1; w < kSumWaves; ++w) sum += slices[w][lane];
    void* to = i < L.dim ? L.dweight : L.dbias;
    if (!to) return;
    const int column = i < L.dim ? i : i - L.dim;
    if (L.accumulate) sum += (double)load_one(to, L.grad_type, column);
    store_one(to, L.grad_type, column, (float)sum);
}

template <int XT>
void forward(const NormForward& L, int groups)
{
    const int d = L.dim;
    auto run = [&](auto kernel) { kernel<<<dim3(groups), dim3(kThreads), 0, L.stream>>>(L); };
    if (d <= 512) run(k_layer_norm<1, 1, XT>);
    else if (d <= 1024) run(k_layer_norm<1, 2, XT>);
    else if (d <= 2048) run(k_layer_norm<1, 4, XT>);
    else if (d <= 4096) run(k_layer_norm<4, 2, XT>);
    else run(k_layer_norm<4, 4, XT>);
}

template <int DT, int XT>
void backward(const NormBackward& L, int groups)
{
    const int d = L.dim;
    auto run = [&](auto kernel) { kernel<<<dim3(groups), dim3(kThreads), d <= kNormWaveDim ? 2 * d * sizeof(float) : 0, L.stream>>>(L); };
    if (d <= 512) run(k_layer_norm_grad<1, 1, DT, XT>);
    else if (d <= 1024) run(k_layer_norm_grad<1, 2, DT, XT>);
    else if (d <= 2048) run(k_layer_norm_grad<1, 4, DT, XT>);
    else if (d <= 4096) run(k_layer_norm_grad<4, 2, DT, XT>);
    else run(k_layer_norm_grad<4, 4, DT, XT>);
}

template <int DT>
void backward(const NormBackward& L, int groups)
{
    if (L.x_type == QADAM_F32) backward<DT, QADAM_F32>(L, groups);
    else if (L.x_type == QADAM_BF16) backward<DT, QADAM_BF16>(L, groups);
    else backward<DT, QADAM_F16>(L, groups);
}

// workgroups of rows, `each` rows at a time, at most `most`
int groups_of(int64_t rows, int each, int most)
{
    const int64_t n = (rows + each - 1) / each;
    return (int)(n < most ? n : most);
}

}  // namespace

hipError_t launch_layer_norm(const NormForward& L)
{
    if (L.dim > kNormGroupDim) {
        k_layer_norm_long<<<dim3(groups_of(L.rows, 1, 512)), dim3(64 * kLongWaves), 0, L.stream>>>(L);
        return hipGetLastError();
    }
    const int groups = groups_of(L.rows, L.dim <= kNormWaveDim ? kWaves : 1, 1024);
    if (L.x_type == QADAM_F32) forward<QADAM_F32>(L, groups);
    else if (L.x_type == QADAM_BF16) forward<QADAM_BF16>(L, groups);
    else forward<QADAM_F16>(L, groups);
    return hipGetLastError();
}

hipError_t launch_layer_norm_grad(const NormBackward& L)
{
    int groups = 0;
    if (L.rows > 0 && L.dim > kNormGroupDim) {
        if (L.dweight || L.dbias) {
            groups = groups_of(L.rows, 1, norm_partials(L.dim));
            k_norm_columns<<<dim3((L.dim + kThreads - 1) / kThreads, groups), dim3(kThreads), 0, L.stream>>>(L);
        }
        k_layer_norm_grad_long<<<dim3(groups_of(L.rows, 1, 512)), dim3(64 * kLongWaves), 0, L.stream>>>(L);
    } else if (L.rows > 0) {
        groups = groups_of(L.rows, L.dim <= kNormWaveDim ? kWaves : 1, norm_partials(L.dim));
        if (L.dout_type == QADAM_F32) backward<QADAM_F32>(L, groups);
        else if (L.dout_type == QADAM_BF16) backward<QADAM_BF16>(L, groups);
        else backward<QADAM_F16>(L, groups);
    }
    if ((L.dweight || L.dbias) && (L.rows > 0 || !L.accumulate))
        k_norm_sums<<<dim3((2 * L.dim + 63) / 64), dim3(64 * kSumWaves), 0, L.stream>>>(L, groups);
    return hipGetLastError();
}

}  // namespace qadam
