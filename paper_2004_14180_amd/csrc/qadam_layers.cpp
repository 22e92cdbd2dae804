// Host side of layer norm, the product in 8-bit integers and sampling: argument checks, the handles, the launches of each call.
#include <cmath>

#include "qadam_host.h"
#include "qadam_layers.h"

using namespace qadam;

namespace {

// Rows of `dim` elements that a call writes (least = dim) or only reads (least = 0: one row for all).  A stride that is neither 0 nor
// room for a row would make rows share elements.
int check_rows(const void* p, int type, int64_t rows, int64_t stride, int64_t dim, bool written, const char* name)
{
    if (written || stride != 0) return check_matrix(p, type, rows, stride, dim, name);
    return check_address(p, element_size(type), name);
}

int check_count(int64_t rows)
{
    if (rows < 0) return fail(QADAM_EINVAL, "a negative number of rows");
    if (rows > (int64_t)1 << 40) return fail(QADAM_ERANGE, "more than 2^40 rows");
    return QADAM_OK;
}

// optional
int check_vector(const void* p, int size, const char* name)
{
    return p ? check_address(p, size, name) : QADAM_OK;
}

}  // namespace

struct qadam_layer_norm_ctx {
    int device;
    int32_t dim;
    float eps;
    DeviceArray<float> partial;
};

struct qadam_linear8_ctx {
    int device;
    int32_t inputs;
    int64_t outputs, max_tokens;
    DeviceArray<int8_t> codes;
    DeviceArray<float> scales;
    DeviceArray<int32_t> sums;          // of workgroups that share a tile's inputs, and how many of them have left theirs
    DeviceArray<uint32_t> arrived;
};

struct qadam_sampler_ctx {
    int device;
    int64_t vocab, max_rows;
    DeviceArray<uint32_t> status;
};

extern "C" {

int qadam_layer_norm_init(qadam_layer_norm_t* out, int32_t dim, float eps)
{
    if (!out) return fail(QADAM_EINVAL, "null argument");
    *out = nullptr;
    if (dim < 1) return fail(QADAM_EINVAL, "dim < 1");
    if (dim > 1 << 20) return fail(QADAM_ERANGE, "more than 2^20 columns");
    if (!(eps >= 0.0f) || !std::isfinite(eps)) return fail(QADAM_EINVAL, "eps negative or not finite");
    return guarded([&]() -> int {
        std::unique_ptr<qadam_layer_norm_ctx> h(new qadam_layer_norm_ctx);
        h->dim = dim; h->eps = eps;
        QADAM_HIP(hipGetDevice(&h->device));
        QADAM_CHECK(allocate(h->partial, (size_t)norm_partials(dim) * 2 * (size_t)dim));
        *out = h.release();
        return QADAM_OK;
    });
}

int qadam_layer_norm_destroy(qadam_layer_norm_t h)
{
    delete h;
    return QADAM_OK;
}

int qadam_layer_norm(qadam_layer_norm_t h, int64_t rows, const void* x, int32_t x_type, int64_t x_stride, const void* weight,
                     const void* bias, int32_t weight_type, void* out, int32_t out_type, int64_t out_stride, float* mean, float* rstd,
                     void* stream)
{
    if (!h) return fail(QADAM_EINVAL, "null handle");
    QADAM_CHECK(check_count(rows));
    if (!float_type(x_type) || !float_type(out_type)) return fail(QADAM_EINVAL, "x_type, out_type");
    if ((weight || bias) && !float_type(weight_type)) return fail(QADAM_EINVAL, "weight_type");
    QADAM_CHECK(check_device(h->device));
    if (weight) QADAM_CHECK(check_address(weight, element_size(weight_type), "weight"));
    if (bias) QADAM_CHECK(check_address(bias, element_size(weight_type), "bias"));
    QADAM_CHECK(check_vector(mean, 4, "mean"));
    QADAM_CHECK(check_vector(rstd, 4, "rstd"));
    if (rows == 0) return QADAM_OK;
    QADAM_CHECK(check_rows(x, x_type, rows, x_stride, h->dim, false, "x"));
    QADAM_CHECK(check_rows(out, out_type, rows, out_stride, h->dim, true, "out"));
    QADAM_HIP(launch_layer_norm({rows, x, x_stride, weight, bias, out, out_stride, mean, rstd, h->eps, h->dim, x_type, weight_type, out_type,
                                 static_cast<hipStream_t>(stream)}));
    return QADAM_OK;
}

int qadam_layer_norm_grad(qadam_layer_norm_t h, int64_t rows, const void* dout, int32_t dout_type, int64_t dout_stride, const void* x,
                          int32_t x_type, int64_t x_stride, const void* weight, int32_t weight_type, const float* mean, const float* rstd,
                          void* dx, int32_t dx_type, int64_t dx_stride, void* dweight, void* dbias, int32_t grad_type, int32_t accumulate,
                          void* stream)
{
    if (!h) return fail(QADAM_EINVAL, "null handle");
    QADAM_CHECK(check_count(rows));
    if (!float_type(dout_type) || !float_type(x_type) || !float_type(dx_type)) return fail(QADAM_EINVAL, "dout_type, x_type, dx_type");
    if (weight && !float_type(weight_type)) return fail(QADAM_EINVAL, "weight_type");
    if ((dweight || dbias) && !float_type(grad_type)) return fail(QADAM_EINVAL, "grad_type");
    if ((accumulate | 1) != 1) return fail(QADAM_EINVAL, "accumulate is 0 or 1");
    QADAM_CHECK(check_device(h->device));
    if (weight) QADAM_CHECK(check_address(weight, element_size(weight_type), "weight"));
    if (dweight) QADAM_CHECK(check_address(dweight, element_size(grad_type), "dweight"));
    if (dbias) QADAM_CHECK(check_address(dbias, element_size(grad_type), "dbias"));
    if (rows > 0) {
        QADAM_CHECK(check_rows(dout, dout_type, rows, dout_stride, h->dim, false, "dout"));
        QADAM_CHECK(check_rows(x, x_type, rows, x_stride, h->dim, false, "x"));
        QADAM_CHECK(check_rows(dx, dx_type, rows, dx_stride, h->dim, true, "dx"));
        QADAM_CHECK(check_address(mean, 4, "mean"));
        QADAM_CHECK(check_address(rstd, 4, "rstd"));
    }
    QADAM_HIP(launch_layer_norm_grad({rows, dout, x, dout_stride, x_stride, weight, mean, rstd, dx, dx_stride, dweight, dbias, h->partial.get(),
                                      h->dim, dout_type, x_type, weight_type, dx_type, grad_type, accumulate, static_cast<hipStream_t>(stream)}));
    return QADAM_OK;
}

int qadam_linear8_init(qadam_linear8_t* out, int64_t outputs, int32_t inputs, int64_t max_tokens)
{
    if (!out) return fail(QADAM_EINVAL, "null argument");
    *out = nullptr;
    if (outputs < 1 || inputs < 1 || max_tokens < 0) return fail(QADAM_EINVAL, "outputs < 1, inputs < 1 or max_tokens < 0");
    if (outputs > 1 << 24) return fail(QADAM_ERANGE, "more than 2^24 outputs");
    if (inputs >= 1 << 17) return fail(QADAM_ERANGE, "2^17 inputs or more: a sum may not fit 32 bits");
    if (max_tokens > 1 << 24 || max_tokens * inputs > (int64_t)1 << 36) return fail(QADAM_ERANGE, "max_tokens beyond 2^24, or max_tokens * inputs beyond 2^36");
    return guarded([&]() -> int {
        std::unique_ptr<qadam_linear8_ctx> h(new qadam_linear8_ctx);
        h->outputs = outputs; h->inputs = inputs; h->max_tokens = max_tokens;
        QADAM_HIP(hipGetDevice(&h->device));
        QADAM_CHECK(allocate(h->codes, (size_t)max_tokens * (size_t)linear8_padded(inputs)));
        QADAM_CHECK(allocate(h->scales, (size_t)max_tokens));
        if (linear8_may_share(outputs, inputs, max_tokens)) {
            QADAM_CHECK(allocate(h->sums, (size_t)kPartTiles * kPartSum));
            QADAM_CHECK(allocate(h->arrived, kPartTiles));
        }
        *out = h.release();
        return QADAM_OK;
    });
}

int qadam_linear8_destroy(qadam_linear8_t h)
{
    delete h;
    return QADAM_OK;
}

int qadam_linear8_quantize(qadam_linear8_t h, int64_t num_tokens, const void* x, int32_t x_type, int64_t x_stride, int8_t* codes,
                           int64_t codes_stride, float* scales, void* stream)
{
    if (!h) return fail(QADAM_EINVAL, "null handle");
    QADAM_CHECK(check_count(num_tokens));
    if (!float_type(x_type)) return fail(QADAM_EINVAL, "x_type");
    QADAM_CHECK(check_device(h->device));
    if (num_tokens == 0) return QADAM_OK;
    QADAM_CHECK(check_rows(x, x_type, num_tokens, x_stride, h->inputs, false, "x"));
    QADAM_CHECK(check_rows(codes, QADAM_CODES8, num_tokens, codes_stride, h->inputs, true, "codes"));
    QADAM_CHECK(check_address(scales, 4, "scales"));
    QADAM_HIP(launch_tokens({num_tokens, x, x_stride, codes, codes_stride, scales, h->inputs, h->inputs, x_type, static_cast<hipStream_t>(stream)}));
    return QADAM_OK;
}

int qadam_linear8_forward(qadam_linear8_t h, int64_t num_tokens, const void* x, int32_t x_type, int64_t x_stride, const float* x_scales,
                          const int8_t* weight, int64_t weight_stride, const float* weight_scales, int32_t k_x, const void* bias,
                          int32_t bias_type, void* out, int32_t out_type, int64_t out_stride, void* stream)
{
    if (!h) return fail(QADAM_EINVAL, "null handle");
    QADAM_CHECK(check_count(num_tokens));
    if (num_tokens > h->max_tokens) return fail(QADAM_ERANGE, "num_tokens > max_tokens of the handle");
    if (x_type != QADAM_CODES8 && !float_type(x_type)) return fail(QADAM_EINVAL, "x_type");
    // an empty array of scales may have no address
    if (x_type == QADAM_CODES8 ? num_tokens > 0 && !x_scales : x_scales != nullptr) return fail(QADAM_EINVAL, "x_scales belong to x in QADAM_CODES8");
    if (!weight_scales && (k_x < 0 || k_x > 6)) return fail(QADAM_EINVAL, "k_x outside 0..6, and no weight_scales");
    if (bias && !float_type(bias_type)) return fail(QADAM_EINVAL, "bias_type");
    if (!float_type(out_type)) return fail(QADAM_EINVAL, "out_type");
    QADAM_CHECK(check_device(h->device));
    if (num_tokens == 0) return QADAM_OK;
    const int32_t K = h->inputs, padded = linear8_padded(K);
    QADAM_CHECK(check_rows(x, x_type, num_tokens, x_stride, K, false, "x"));
    QADAM_CHECK(check_vector(x_scales, 4, "x_scales"));
    QADAM_CHECK(check_rows(weight, QADAM_CODES8, h->outputs, weight_stride, K, true, "weight"));
    QADAM_CHECK(check_vector(weight_scales, 4, "weight_scales"));
    if (bias) QADAM_CHECK(check_address(bias, element_size(bias_type), "bias"));
    QADAM_CHECK(check_rows(out, out_type, num_tokens, out_stride, h->outputs, true, "out"));
    const hipStream_t s = static_cast<hipStream_t>(stream);
    // integers that lie as the kernels want them are taken where they are
    const bool there = x_type == QADAM_CODES8 && K == padded && x_stride % 16 == 0 && x_stride <= 1 << 22 && reinterpret_cast<uintptr_t>(x) % 16 == 0;
    const TokensLaunch X{num_tokens, x, x_stride, there ? nullptr : h->codes.get(), padded, h->scales.get(), K, padded, x_type, s,
                         h->arrived.get()};
    QADAM_HIP(launch_product({num_tokens, h->outputs, there ? static_cast<const int8_t*>(x) : h->codes.get(), there ? x_stride : padded,
                              x_scales ? x_scales : h->scales.get(), weight, weight_stride, weight_scales, bias, out, out_stride,
                              weight_scales ? 1.0f : std::ldexp(1.0f, -(k_x + 1)), K, bias_type, out_type, s, there ? nullptr : h->sums.get()}, X));
    return QADAM_OK;
}

int qadam_sampler_init(qadam_sampler_t* out, int64_t vocab, int64_t max_rows)
{
    if (!out) return fail(QADAM_EINVAL, "null argument");
    *out = nullptr;
    if (vocab < 1 || max_rows < 0) return fail(QADAM_EINVAL, "vocab < 1 or max_rows < 0");
    if (vocab > 1 << 22) return fail(QADAM_ERANGE, "a vocabulary of more than 2^22: its masses' sum may not fit 64 bits");
    if (max_rows > 1 << 24) return fail(QADAM_ERANGE, "more than 2^24 rows");
    return guarded([&]() -> int {
        std::unique_ptr<qadam_sampler_ctx> h(new qadam_sampler_ctx);
        h->vocab = vocab; h->max_rows = max_rows;
        QADAM_HIP(hipGetDevice(&h->device));
        QADAM_CHECK(allocate(h->status, 1));
        QADAM_HIP(hipMemset(h->status.get(), 0, sizeof(uint32_t)));
        QADAM_HIP(hipStreamSynchronize(nullptr));
        *out = h.release();
        return QADAM_OK;
    });
}

int qadam_sampler_destroy(qadam_sampler_t h)
{
    delete h;
    return QADAM_OK;
}

int qadam_sampler_sample(qadam_sampler_t h, int64_t rows, const void* logits, int32_t logits_type, int64_t logits_stride, const float* u,
                         const qadam_filters_t* filters, void* out, int32_t token_bytes, void* stream)
{
    if (!h || !filters) return fail(QADAM_EINVAL, "null argument");
    QADAM_CHECK(check_count(rows));
    if (rows > h->max_rows) return fail(QADAM_ERANGE, "rows > max_rows of the handle");
    if (!float_type(logits_type)) return fail(QADAM_EINVAL, "logits_type");
    if (token_bytes != 4 && token_bytes != 8) return fail(QADAM_EINVAL, "token_bytes is 4 or 8");
    if (!filters->temperatures && !(filters->temperature >= 0.0f && std::isfinite(filters->temperature)))
        return fail(QADAM_EINVAL, "temperature negative or not finite");
    QADAM_CHECK(check_device(h->device));
    QADAM_CHECK(check_vector(filters->temperatures, 4, "temperatures"));
    QADAM_CHECK(check_vector(filters->top_ks, 4, "top_ks"));
    QADAM_CHECK(check_vector(filters->top_ps, 4, "top_ps"));
    QADAM_CHECK(check_vector(filters->min_ps, 4, "min_ps"));
    if (rows == 0) return QADAM_OK;
    QADAM_CHECK(check_rows(logits, logits_type, rows, logits_stride, h->vocab, false, "logits"));
    QADAM_CHECK(check_address(u, 4, "u"));
    QADAM_CHECK(check_address(out, token_bytes, "out"));
    QADAM_HIP(launch_sample({rows, h->vocab, logits, logits_stride, u, out, h->status.get(), *filters, logits_type, token_bytes,
                             static_cast<hipStream_t>(stream)}));
    return QADAM_OK;
}

int qadam_sampler_get_status(qadam_sampler_t h, qadam_status_t* out, int32_t clear, void* stream)
{
    if (!h || !out) return fail(QADAM_EINVAL, "null argument");
    QADAM_CHECK(check_device(h->device));
    return read_status(h->status.get(), out, clear, static_cast<hipStream_t>(stream));
}

}  // extern "C"
