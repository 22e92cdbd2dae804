// Host side of the operators beside the step (lists of tensors, embedding): argument checks, the handles, the launches of each call.
#include <cmath>
#include <cstring>
#include <new>

#include "qadam_elements.h"
#include "qadam_host.h"
#include "qadam_operators.h"

using namespace qadam;

namespace {

// A list's tensors and tiles on the device, and its launches.
struct List {
    struct Part {
        int32_t first_tensor, num_tensors, first_tile, num_tiles;
    };
    int device = -1;
    std::vector<int64_t> numels;
    std::vector<int32_t> grad_sizes;
    std::vector<Part> parts;
    DeviceArray<ListTile> tiles;
    DeviceArray<ListTensor> tensors;

    static int64_t tiles_of(const ListTensor& t)
    {
        return t.numel > 0 ? (t.numel + (t.types >> kTypeBits) + kListTile - 1) / kListTile : 0;
    }

    int build(const std::vector<ListTensor>& host)
    {
        int64_t count = 0;
        for (const ListTensor& t : host) {
            static_assert(kMostLaunchTiles == (1 << 22) - 1 && kMostListTiles == 1 << 26 && kListTile == 4096, "the texts below");
            if (tiles_of(t) > kMostLaunchTiles) return fail(QADAM_ERANGE, "a tensor too large for one launch (elements / 4096 must stay below 2^22)");
            count += tiles_of(t);
            if (count > kMostListTiles) return fail(QADAM_ERANGE, "more than 2^38 elements in all");
        }
        std::vector<ListTile> all;
        all.reserve((size_t)count);
        for (size_t i = 0; i < host.size(); ++i) {
            const int32_t n = (int32_t)tiles_of(host[i]);
            if (parts.empty() || !list_launch_takes(parts.back().num_tensors, parts.back().num_tiles, n))
                parts.push_back({(int32_t)i, 0, (int32_t)all.size(), 0});
            for (int32_t k = 0; k < n; ++k) {
                const int64_t left = host[i].numel - (int64_t)k * kListTile;
                all.push_back({(int32_t)i, k, (int32_t)(left < kListTile ? left : kListTile), host[i].types >> 2 & 3});
            }
            ++parts.back().num_tensors;
            parts.back().num_tiles += n;
            numels.push_back(host[i].numel);
            grad_sizes.push_back(element_size(host[i].types >> 2 & 3));
        }
        QADAM_HIP(hipGetDevice(&device));
        QADAM_CHECK(upload(tiles, all));
        return upload(tensors, host);
    }

    int check_grads(const void* const* grads) const
    {
        if (numels.empty()) return QADAM_OK;
        if (!grads) return fail(QADAM_EINVAL, "grads");
        for (size_t i = 0; i < numels.size(); ++i)
            if (grads[i]) QADAM_CHECK(check_address(grads[i], grad_sizes[i], "grads[i]"));
        return QADAM_OK;
    }

    ListLaunch launch(const Part& p, void* stream) const
    {
        return {tiles.get(), tensors.get(), p.first_tile, p.num_tiles, p.first_tensor, static_cast<hipStream_t>(stream)};
    }

    static void fill(GradTable& G, const Part& p, const void* const* grads)
    {
        for (int32_t i = 0; i < p.num_tensors; ++i) G.grad[i] = grads[p.first_tensor + i];
    }
};

}  // namespace

struct qadam_adamw_ctx {
    qadam_adamw_config_t cfg;
    List list;
};

struct qadam_grad_norm_ctx {
    List list;
    int32_t total;
    DeviceArray<double> sums;
    DeviceArray<uint32_t> arrived;
};

struct qadam_embedding_ctx {
    int device;
    int64_t rows, max_tokens;
    int32_t dim;
    DeviceArray<uint32_t> status, counts, arrived;
    DeviceArray<int32_t> sorted;        // keys and order, twice
    DeviceArray<float> pieces;
    EmbeddingScratch scratch;
};

extern "C" {

int qadam_adamw_init(qadam_adamw_t* out, const qadam_adamw_config_t* cfg, const qadam_adamw_tensor_t* tensors, int32_t num_tensors)
{
    if (!out || !cfg) return fail(QADAM_EINVAL, "null argument");
    *out = nullptr;
    if (cfg->struct_size != sizeof(qadam_adamw_config_t)) return fail(QADAM_EINVAL, "config struct_size mismatch");
    if (cfg->state_bits != 32 && cfg->state_bits != 8) return fail(QADAM_EINVAL, "state_bits is 32 or 8");
    if (!(cfg->beta1 >= 0.0 && cfg->beta1 < 1.0) || !(cfg->beta2 >= 0.0 && cfg->beta2 < 1.0)) return fail(QADAM_EINVAL, "beta outside [0,1)");
    if (!(cfg->eps >= 0.0) || !std::isfinite(cfg->eps)) return fail(QADAM_EINVAL, "eps negative or not finite");
    if (num_tensors < 0 || (num_tensors > 0 && !tensors)) return fail(QADAM_EINVAL, "tensors");
    return guarded([&]() -> int {
        std::vector<ListTensor> host;
        for (int32_t i = 0; i < num_tensors; ++i) {
            const qadam_adamw_tensor_t& t = tensors[i];
            if (t.numel < 0) return fail(QADAM_EINVAL, "numel < 0");
            if (t.numel > (int64_t)1 << 40) return fail(QADAM_ERANGE, "more than 2^40 elements");
            if (!float_type(t.param_type) || !float_type(t.grad_type)) return fail(QADAM_EINVAL, "param_type, grad_type");
            if (!(t.weight_decay >= 0.0f) || !std::isfinite(t.weight_decay)) return fail(QADAM_EINVAL, "weight_decay negative or not finite");
            if (t.copy && (t.param_type != QADAM_F32 || (t.copy_type != QADAM_BF16 && t.copy_type != QADAM_F16)))
                return fail(QADAM_EINVAL, "a copy is QADAM_BF16 or QADAM_F16, of QADAM_F32 weights");
            if (t.numel > 0) {
                const bool state8 = cfg->state_bits == 8;
                QADAM_CHECK(check_address(t.param, element_size(t.param_type), "param"));
                QADAM_CHECK(check_address(t.m, state8 ? 1 : 4, "m"));
                QADAM_CHECK(check_address(t.v, state8 ? 1 : 4, "v"));
                if (state8) {
                    QADAM_CHECK(check_address(t.m_scales, 4, "m_scales"));
                    QADAM_CHECK(check_address(t.v_scales, 4, "v_scales"));
                }
                if (t.copy) QADAM_CHECK(check_address(t.copy, 2, "copy"));
            }
            const int shift = cfg->state_bits == 8 ? 0 : block_shift(t.param, element_size(t.param_type));
            host.push_back({t.param, t.m, t.v, t.m_scales, t.v_scales, t.copy, t.numel,
                            list_types(t.param_type, t.grad_type, t.copy ? t.copy_type : kNoCopy) | shift << kTypeBits, t.weight_decay});
        }
        std::unique_ptr<qadam_adamw_ctx> h(new qadam_adamw_ctx);
        h->cfg = *cfg;
        QADAM_CHECK(h->list.build(host));
        *out = h.release();
        return QADAM_OK;
    });
}

int qadam_adamw_destroy(qadam_adamw_t h)
{
    delete h;
    return QADAM_OK;
}

int qadam_adamw_step(qadam_adamw_t h, int64_t step, float lr, const void* const* grads, const float* grad_factor_dev, void* stream)
{
    if (!h) return fail(QADAM_EINVAL, "null handle");
    if (step < 1) return fail(QADAM_EINVAL, "step < 1");
    if (!std::isfinite(lr)) return fail(QADAM_EINVAL, "lr is not finite");
    QADAM_CHECK(check_device(h->list.device));
    QADAM_CHECK(h->list.check_grads(grads));
    if (grad_factor_dev) QADAM_CHECK(check_address(grad_factor_dev, 4, "grad_factor_dev"));
    hipStreamCaptureStatus capture = hipStreamCaptureStatusNone;
    QADAM_HIP(hipStreamIsCapturing(static_cast<hipStream_t>(stream), &capture));
    if (capture != hipStreamCaptureStatusNone)
        return fail(QADAM_EINVAL, "stream is capturing a graph: a replay would reuse this step's bias corrections");
    const double b1 = h->cfg.beta1, b2 = h->cfg.beta2;
    AdamwScalars S;
    S.beta1 = (float)b1; S.omb1 = (float)(1.0 - b1);
    S.beta2 = (float)b2; S.omb2 = (float)(1.0 - b2);
    S.lr = lr;
    S.lr1 = (float)((double)lr / (1.0 - std::pow(b1, (double)step)));
    S.inv_sbc2 = (float)(1.0 / std::sqrt(1.0 - std::pow(b2, (double)step)));
    S.eps = (float)h->cfg.eps;
    GradTable G;
    for (const List::Part& p : h->list.parts) {
        if (p.num_tiles == 0) continue;
        List::fill(G, p, grads);
        QADAM_HIP(launch_adamw(h->list.launch(p, stream), S, G, grad_factor_dev, h->cfg.state_bits == 8));
    }
    return QADAM_OK;
}

int qadam_grad_norm_init(qadam_grad_norm_t* out, const int64_t* numels, const int32_t* grad_types, int32_t num_tensors)
{
    if (!out) return fail(QADAM_EINVAL, "null argument");
    *out = nullptr;
    if (num_tensors < 0 || (num_tensors > 0 && (!numels || !grad_types))) return fail(QADAM_EINVAL, "tensors");
    return guarded([&]() -> int {
        std::vector<ListTensor> host;
        for (int32_t i = 0; i < num_tensors; ++i) {
            if (numels[i] < 0) return fail(QADAM_EINVAL, "numel < 0");
            if (numels[i] > (int64_t)1 << 40) return fail(QADAM_ERANGE, "more than 2^40 elements");
            if (!float_type(grad_types[i])) return fail(QADAM_EINVAL, "grad_types");
            ListTensor t{};
            t.numel = numels[i];
            t.types = list_types(QADAM_F32, grad_types[i], kNoCopy);
            host.push_back(t);
        }
        std::unique_ptr<qadam_grad_norm_ctx> h(new qadam_grad_norm_ctx);
        QADAM_CHECK(h->list.build(host));
        if (h->list.parts.empty()) h->list.parts.push_back({0, 0, 0, 0});
        h->total = 0;
        for (const List::Part& p : h->list.parts) h->total += norm_groups(p.num_tiles);
        QADAM_CHECK(allocate(h->sums, (size_t)h->total));
        QADAM_CHECK(allocate(h->arrived, kArrivalWords));
        QADAM_HIP(hipMemset(h->arrived.get(), 0, kArrivalWords * sizeof(uint32_t)));
        QADAM_HIP(hipStreamSynchronize(nullptr));
        *out = h.release();
        return QADAM_OK;
    });
}

int qadam_grad_norm_destroy(qadam_grad_norm_t h)
{
    delete h;
    return QADAM_OK;
}

int qadam_grad_norm(qadam_grad_norm_t h, const void* const* grads, float max_norm, float* out_dev, void* stream)
{
    if (!h) return fail(QADAM_EINVAL, "null handle");
    if (!(max_norm >= 0.0f)) return fail(QADAM_EINVAL, "max_norm negative or NaN");
    QADAM_CHECK(check_device(h->list.device));
    QADAM_CHECK(h->list.check_grads(grads));
    QADAM_CHECK(check_address(out_dev, 4, "out_dev"));
    NormLaunch N{h->sums.get(), h->arrived.get(), 0, 0, max_norm, out_dev};
    GradTable G;
    for (size_t i = 0; i < h->list.parts.size(); ++i) {
        const List::Part& p = h->list.parts[i];
        List::fill(G, p, grads);
        if (i + 1 == h->list.parts.size()) N.total = h->total;
        QADAM_HIP(launch_grad_norm(h->list.launch(p, stream), N, G));
        N.first_sum += norm_groups(p.num_tiles);
    }
    return QADAM_OK;
}

int qadam_embedding_init(qadam_embedding_t* out, int64_t rows, int32_t dim, int64_t max_tokens)
{
    if (!out) return fail(QADAM_EINVAL, "null argument");
    *out = nullptr;
    if (rows < 1 || dim < 1 || max_tokens < 0) return fail(QADAM_EINVAL, "rows < 1, dim < 1 or max_tokens < 0");
    if (rows > (int64_t)1 << 28) return fail(QADAM_ERANGE, "more than 2^28 rows");
    if (max_tokens > (int64_t)1 << 24) return fail(QADAM_ERANGE, "more than 2^24 tokens");
    if (dim > 1 << 20) return fail(QADAM_ERANGE, "more than 2^20 columns");
    static_assert(kChunk == 8 && kMostSums == 1 << 25, "the text below");
    if (sum_groups(max_tokens, dim) >= kMostSums)
        return fail(QADAM_ERANGE, "too many wavefronts for one launch (max_tokens / 8 times the slices of 256 columns must stay below 2^25)");
    return guarded([&]() -> int {
        std::unique_ptr<qadam_embedding_ctx> h(new qadam_embedding_ctx);
        h->rows = rows; h->dim = dim; h->max_tokens = max_tokens;
        QADAM_HIP(hipGetDevice(&h->device));
        QADAM_CHECK(allocate(h->status, 1));
        QADAM_HIP(hipMemset(h->status.get(), 0, sizeof(uint32_t)));
        const size_t n = (size_t)max_tokens, arrivals = (size_t)arrival_places(max_tokens, dim) * (size_t)column_slices(dim);
        if (n > 0) {
            QADAM_CHECK(allocate(h->sorted, 4 * n));
            QADAM_CHECK(allocate(h->counts, (size_t)sort_tiles(max_tokens) << kSortBits));
            QADAM_CHECK(allocate(h->pieces, (size_t)piece_places(max_tokens, dim) * (size_t)dim));
            QADAM_CHECK(allocate(h->arrived, arrivals));
            QADAM_HIP(hipMemset(h->arrived.get(), 0, arrivals * sizeof(uint32_t)));
        }
        int32_t* s = h->sorted.get();
        h->scratch = {{s, s + n}, {s + 2 * n, s + 3 * n}, h->counts.get(), h->pieces.get(), h->arrived.get()};
        QADAM_HIP(hipStreamSynchronize(nullptr));
        *out = h.release();
        return QADAM_OK;
    });
}

int qadam_embedding_destroy(qadam_embedding_t h)
{
    delete h;
    return QADAM_OK;
}

static int check_tokens(const qadam_embedding_ctx* h, const void* tokens, int32_t token_bytes, int64_t num_tokens)
{
    if (!h) return fail(QADAM_EINVAL, "null handle");
    if (token_bytes != 4 && token_bytes != 8) return fail(QADAM_EINVAL, "token_bytes is 4 or 8");
    if (num_tokens < 0) return fail(QADAM_EINVAL, "num_tokens < 0");
    if (num_tokens > (int64_t)1 << 40) return fail(QADAM_ERANGE, "more than 2^40 tokens");
    QADAM_CHECK(check_device(h->device));
    return num_tokens > 0 ? check_address(tokens, token_bytes, "tokens") : QADAM_OK;
}

int qadam_embedding_lookup(qadam_embedding_t h, const void* weight, int32_t weight_type, int32_t k_x, int64_t weight_stride,
                           const void* tokens, int32_t token_bytes, int64_t num_tokens, int64_t padding, float scale,
                           void* out, int32_t out_type, int64_t out_stride, void* stream)
{
    QADAM_CHECK(check_tokens(h, tokens, token_bytes, num_tokens));
    const bool codes = weight_type == QADAM_CODES8 || weight_type == QADAM_CODES16;
    if (!codes && !float_type(weight_type)) return fail(QADAM_EINVAL, "weight_type");
    if (codes && (k_x < 0 || k_x > 14 || (k_x > 6) != (weight_type == QADAM_CODES16)))
        return fail(QADAM_EINVAL, "k_x outside 0..6 (QADAM_CODES8) or 7..14 (QADAM_CODES16)");
    if (!float_type(out_type)) return fail(QADAM_EINVAL, "out_type");
    if (num_tokens == 0) return QADAM_OK;
    QADAM_CHECK(check_matrix(weight, weight_type, h->rows, weight_stride, h->dim, "weight"));
    QADAM_CHECK(check_matrix(out, out_type, num_tokens, out_stride, h->dim, "out"));
    LookupLaunch L;
    L.t = {tokens, token_bytes, num_tokens, padding, h->rows, h->status.get()};
    L.weight = weight; L.weight_type = weight_type; L.out_type = out_type; L.dim = h->dim;
    L.weight_stride = weight_stride; L.out_stride = out_stride;
    L.scale = codes ? std::ldexp(scale, -(k_x + 1)) : scale;
    L.out = out; L.stream = static_cast<hipStream_t>(stream);
    QADAM_HIP(launch_embedding_lookup(L));
    return QADAM_OK;
}

int qadam_embedding_grad(qadam_embedding_t h, const void* tokens, int32_t token_bytes, int64_t num_tokens, int64_t padding,
                         float scale, const void* dout, int32_t dout_type, int64_t dout_stride,
                         void* grad, int32_t grad_type, int64_t grad_stride, int32_t accumulate, void* stream)
{
    QADAM_CHECK(check_tokens(h, tokens, token_bytes, num_tokens));
    if (num_tokens > h->max_tokens) return fail(QADAM_ERANGE, "num_tokens > max_tokens of the handle");
    if (!float_type(dout_type)) return fail(QADAM_EINVAL, "dout_type");
    if (!float_type(grad_type)) return fail(QADAM_EINVAL, "grad_type");
    if ((accumulate | 1) != 1) return fail(QADAM_EINVAL, "accumulate is 0 or 1");
    if (num_tokens > 0) QADAM_CHECK(check_matrix(dout, dout_type, num_tokens, dout_stride, 0, "dout"));
    QADAM_CHECK(check_matrix(grad, grad_type, h->rows, grad_stride, h->dim, "grad"));
    EmbeddingGradLaunch L;
    L.t = {tokens, token_bytes, num_tokens, padding, h->rows, h->status.get()};
    L.w = h->scratch;
    L.dout = dout; L.grad = grad; L.dout_type = dout_type; L.grad_type = grad_type; L.dim = h->dim; L.accumulate = accumulate;
    L.dout_stride = dout_stride; L.grad_stride = grad_stride;
    L.scale = scale; L.stream = static_cast<hipStream_t>(stream);
    QADAM_HIP(launch_embedding_grad(L));
    return QADAM_OK;
}

int qadam_embedding_get_status(qadam_embedding_t h, qadam_status_t* out, int32_t clear, void* stream)
{
    if (!h || !out) return fail(QADAM_EINVAL, "null argument");
    QADAM_CHECK(check_device(h->device));
    return read_status(h->status.get(), out, clear, static_cast<hipStream_t>(stream));
}

}  // extern "C"
