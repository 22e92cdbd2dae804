// The common form of the binding's calls without Python work per buffer: every tensor is checked here for type, device, layout and
// size, and the library is called with the addresses.  Any other form (another type of tensor or number, a wrong size, a missing
// buffer) makes the function return None before anything is called, and the binding's own path takes or refuses the call.
//
// A step of a short vector is bound by the host: 51 k parameters and 4 workers, 21 buffers, 13.0 us of its 20.0 us per step were the
// checks in Python.
#include <memory>
#include <vector>

#include <torch/csrc/autograd/python_variable.h>

#include "../../include/qadam.h"

namespace {

constexpr char kPlanName[] = "qadam plan", kListName[] = "qadam list of tensors", kEmbeddingName[] = "qadam embedding", kLayerName[] = "qadam layer";

struct Plan {
    qadam_handle_t h;
    Py_ssize_t workers;
    int64_t params, segments, code_bytes, wcode_bytes;
    bool weight_ef;
    decltype(&qadam_worker_quantize) worker_quantize;
    decltype(&qadam_server_step) server_step;
    decltype(&qadam_weight_quantize) weight_quantize;
    decltype(&qadam_step_fused) step_fused;
    decltype(&qadam_step_fused_w) step_fused_w;
};

enum class Kind { f32, integers };

// Arguments in order; ok becomes false with the first one that is not of the common form.
struct Args {
    PyObject* const* next;
    bool ok;

    int64_t integer()
    {
        PyObject* o = *next++;
        if (!ok || !PyLong_Check(o)) { ok = false; return 0; }
        const long long v = PyLong_AsLongLong(o);
        if (v == -1 && PyErr_Occurred()) { PyErr_Clear(); ok = false; }
        return v;
    }

    float number()
    {
        PyObject* o = *next++;
        if (!ok || !(PyFloat_Check(o) || PyLong_Check(o))) { ok = false; return 0.0f; }
        const double v = PyFloat_AsDouble(o);
        if (v == -1.0 && PyErr_Occurred()) { PyErr_Clear(); ok = false; }
        return (float)v;
    }

    void* address(PyObject* o, Kind kind, int64_t need, int64_t device, bool optional = false)
    {
        if (!ok || (optional && o == Py_None)) return nullptr;
        ok = false;
        if (!THPVariable_CheckExact(o)) return nullptr;
        const at::Tensor& t = THPVariable_Unpack(o);
        if (!t.has_storage() || !t.is_cuda() || t.get_device() != device || !t.is_contiguous()) return nullptr;
        if (kind == Kind::f32 ? t.scalar_type() != at::kFloat || t.numel() < need
                              : !at::isIntegralType(t.scalar_type(), true) || t.numel() * (int64_t)t.element_size() < need)
            return nullptr;
        void* p = t.data_ptr();
        ok = true;
        return p;
    }

    void* tensor(Kind kind, int64_t need, int64_t device, bool optional = false)
    {
        return address(*next++, kind, need, device, optional);
    }

    template <typename T>
    void tensors(T* (&out)[QADAM_MAX_WORKERS], Py_ssize_t count, Kind kind, int64_t need, int64_t device)
    {
        PyObject* o = *next++;
        if (!(PyList_Check(o) || PyTuple_Check(o)) || PySequence_Fast_GET_SIZE(o) != count) ok = false;
        for (Py_ssize_t i = 0; ok && i < count; ++i) out[i] = static_cast<T*>(address(PySequence_Fast_GET_ITEM(o, i), kind, need, device));
    }
};

template <typename F>
PyObject* call(const Args& a, F&& f)
{
    if (!a.ok) Py_RETURN_NONE;
    int rc;
    Py_BEGIN_ALLOW_THREADS
    rc = f();
    Py_END_ALLOW_THREADS
    return PyLong_FromLong(rc);
}

// body(args, plan, device, stream): the arguments behind the plan, the device and the stream
template <typename Plan, const char* kPlanName, typename F>
PyObject* planned(PyObject* const* argv, Py_ssize_t argc, Py_ssize_t expected, F&& body)
{
    if (argc != expected) {
        PyErr_SetString(PyExc_TypeError, "wrong number of arguments");
        return nullptr;
    }
    if (argv[0] == Py_None) Py_RETURN_NONE;
    const Plan* plan = static_cast<const Plan*>(PyCapsule_GetPointer(argv[0], kPlanName));
    if (!plan) return nullptr;
    try {
        Args a{argv + 1, true};
        const int64_t device = a.integer();
        void* stream = reinterpret_cast<void*>(a.integer());
        return body(a, *plan, device, stream);
    } catch (const std::exception&) {
        Py_RETURN_NONE;
    }
}

PyObject* worker_quantize(PyObject*, PyObject* const* argv, Py_ssize_t argc)
{
    return planned<Plan, kPlanName>(argv, argc, 9, [](Args& a, const Plan& p, int64_t device, void* stream) {
        const int64_t worker = a.integer(), step = a.integer();
        if (worker < 0 || worker >= p.workers) a.ok = false;
        const float* grad = static_cast<float*>(a.tensor(Kind::f32, p.params, device));
        float* err = static_cast<float*>(a.tensor(Kind::f32, p.params, device));
        void* codes = a.tensor(Kind::integers, p.code_bytes, device);
        float* scales = static_cast<float*>(a.tensor(Kind::f32, p.segments, device));
        return call(a, [&] { return p.worker_quantize(p.h, (int32_t)worker, step, grad, err, codes, scales, stream); });
    });
}

PyObject* server_step(PyObject*, PyObject* const* argv, Py_ssize_t argc)
{
    return planned<Plan, kPlanName>(argv, argc, 11, [](Args& a, const Plan& p, int64_t device, void* stream) {
        const int64_t step = a.integer();
        const float lr = a.number(), beta2 = a.number();
        void* codes[QADAM_MAX_WORKERS];
        float* scales[QADAM_MAX_WORKERS];
        a.tensors(codes, p.workers, Kind::integers, p.code_bytes, device);
        a.tensors(scales, p.workers, Kind::f32, p.segments, device);
        float* s[3];
        for (float*& t : s) t = static_cast<float*>(a.tensor(Kind::f32, p.params, device));
        return call(a, [&] { return p.server_step(p.h, step, lr, beta2, codes, scales, s[0], s[1], s[2], stream); });
    });
}

PyObject* weight_quantize(PyObject*, PyObject* const* argv, Py_ssize_t argc)
{
    return planned<Plan, kPlanName>(argv, argc, 7, [](Args& a, const Plan& p, int64_t device, void* stream) {
        const int64_t step = a.integer();
        const float* x = static_cast<float*>(a.tensor(Kind::f32, p.params, device));
        float* werr = static_cast<float*>(a.tensor(Kind::f32, p.params, device, !p.weight_ef));
        void* wcodes = a.tensor(Kind::integers, p.wcode_bytes, device);
        return call(a, [&] { return p.weight_quantize(p.h, step, x, werr, wcodes, stream); });
    });
}

PyObject* step_fused(PyObject*, PyObject* const* argv, Py_ssize_t argc)
{
    return planned<Plan, kPlanName>(argv, argc, 15, [](Args& a, const Plan& p, int64_t device, void* stream) {
        const int64_t step = a.integer();
        const float lr = a.number(), beta2 = a.number();
        float *grads[QADAM_MAX_WORKERS], *errs[QADAM_MAX_WORKERS], *scales[QADAM_MAX_WORKERS];
        void* codes[QADAM_MAX_WORKERS];
        a.tensors(grads, p.workers, Kind::f32, p.params, device);
        a.tensors(errs, p.workers, Kind::f32, p.params, device);
        a.tensors(codes, p.workers, Kind::integers, p.code_bytes, device);
        a.tensors(scales, p.workers, Kind::f32, p.segments, device);
        float* s[3];
        for (float*& t : s) t = static_cast<float*>(a.tensor(Kind::f32, p.params, device));
        float* werr = static_cast<float*>(a.tensor(Kind::f32, p.params, device, !p.weight_ef));
        void* wcodes = a.tensor(Kind::integers, p.wcode_bytes, device);
        return call(a, [&] {
            return p.step_fused(p.h, step, lr, beta2, grads, errs, codes, scales, s[0], s[1], s[2], werr, wcodes, stream);
        });
    });
}

PyObject* step_fused_w(PyObject*, PyObject* const* argv, Py_ssize_t argc)
{
    return planned<Plan, kPlanName>(argv, argc, 15, [](Args& a, const Plan& p, int64_t device, void* stream) {
        const int64_t step = a.integer();
        const float lr = a.number(), beta2 = a.number();
        float *grads[QADAM_MAX_WORKERS], *mw[QADAM_MAX_WORKERS], *vw[QADAM_MAX_WORKERS], *errs[QADAM_MAX_WORKERS],
            *scales[QADAM_MAX_WORKERS];
        void* codes[QADAM_MAX_WORKERS];
        a.tensors(grads, p.workers, Kind::f32, p.params, device);
        a.tensors(mw, p.workers, Kind::f32, p.params, device);
        a.tensors(vw, p.workers, Kind::f32, p.params, device);
        a.tensors(errs, p.workers, Kind::f32, p.params, device);
        a.tensors(codes, p.workers, Kind::integers, p.code_bytes, device);
        a.tensors(scales, p.workers, Kind::f32, p.segments, device);
        float* x = static_cast<float*>(a.tensor(Kind::f32, p.params, device));
        float* werr = static_cast<float*>(a.tensor(Kind::f32, p.params, device, !p.weight_ef));
        void* wcodes = a.tensor(Kind::integers, p.wcode_bytes, device);
        return call(a, [&] { return p.step_fused_w(p.h, step, lr, beta2, grads, mw, vw, errs, codes, scales, x, werr, wcodes, stream); });
    });
}

// (the address of qadam_quantize_segment_noalloc, device, stream, k_g, n, grad, err, codes, scale); the sizes of the buffers are the
// caller's word, as in the binding
PyObject* quantize_segment(PyObject*, PyObject* const* argv, Py_ssize_t argc)
{
    if (argc != 9) {
        PyErr_SetString(PyExc_TypeError, "wrong number of arguments");
        return nullptr;
    }
    try {
        Args a{argv, true};
        const auto fn = reinterpret_cast<decltype(&qadam_quantize_segment_noalloc)>(a.integer());
        (void)a.integer();
        void* stream = reinterpret_cast<void*>(a.integer());
        const int64_t k_g = a.integer(), n = a.integer();
        if (k_g < INT32_MIN || k_g > INT32_MAX) a.ok = false;
        void* t[4] = {};
        for (void*& p : t) {
            PyObject* o = *a.next++;
            if (!a.ok) break;
            a.ok = false;
            if (!THPVariable_CheckExact(o)) break;
            const at::Tensor& v = THPVariable_Unpack(o);
            if (!v.has_storage() || !v.is_cuda() || !v.is_contiguous()) break;
            p = v.data_ptr();
            a.ok = true;
        }
        return call(a, [&] {
            return fn((int32_t)k_g, n, static_cast<float*>(t[0]), static_cast<float*>(t[1]), t[2], static_cast<float*>(t[3]), stream);
        });
    } catch (const std::exception&) {
        Py_RETURN_NONE;
    }
}

// A list of tensors, for AdamW's step or the gradients' norm: what its gradients have to be.
struct ListPlan {
    void* h;
    void* entry;
    std::vector<int64_t> numels;
    std::vector<at::ScalarType> types;
};

at::ScalarType scalar_type(int64_t type)
{
    return type == QADAM_F32 ? at::kFloat : type == QADAM_BF16 ? at::kBFloat16 : at::kHalf;
}

// -1: another one
int element_type(const at::Tensor& t)
{
    switch (t.scalar_type()) {
    case at::kFloat: return QADAM_F32;
    case at::kBFloat16: return QADAM_BF16;
    case at::kHalf: return QADAM_F16;
    case at::kChar: return QADAM_CODES8;
    case at::kShort: return QADAM_CODES16;
    default: return -1;
    }
}

// the tensor `o` if it lies on this device
const at::Tensor* on_device(Args& a, PyObject* o, int64_t device)
{
    if (!a.ok || !THPVariable_CheckExact(o)) { a.ok = false; return nullptr; }
    const at::Tensor& t = THPVariable_Unpack(o);
    if (!t.has_storage() || !t.is_cuda() || t.get_device() != device) { a.ok = false; return nullptr; }
    return &t;
}

std::vector<const void*> gradients(Args& a, const ListPlan& p, int64_t device)
{
    PyObject* o = *a.next++;
    const Py_ssize_t count = (Py_ssize_t)p.numels.size();
    std::vector<const void*> out(count, nullptr);
    if (!(PyList_Check(o) || PyTuple_Check(o)) || PySequence_Fast_GET_SIZE(o) != count) a.ok = false;
    for (Py_ssize_t i = 0; a.ok && i < count; ++i) {
        PyObject* item = PySequence_Fast_GET_ITEM(o, i);
        if (item == Py_None) continue;
        const at::Tensor* t = on_device(a, item, device);
        if (t && t->scalar_type() == p.types[i] && t->numel() == p.numels[i] && t->is_contiguous()) out[i] = t->data_ptr();
        else a.ok = false;
    }
    return out;
}

// exactly `count` fp32 one behind the other
float* floats(Args& a, int64_t count, int64_t device, bool optional = false)
{
    PyObject* o = *a.next++;
    if (optional && o == Py_None) return nullptr;
    const at::Tensor* t = on_device(a, o, device);
    if (!t || t->scalar_type() != at::kFloat || t->numel() != count || !t->is_contiguous()) { a.ok = false; return nullptr; }
    return static_cast<float*>(t->data_ptr());
}

PyObject* adamw_step(PyObject*, PyObject* const* argv, Py_ssize_t argc)
{
    return planned<ListPlan, kListName>(argv, argc, 7, [](Args& a, const ListPlan& p, int64_t device, void* stream) {
        const int64_t step = a.integer();
        const float lr = a.number();
        const std::vector<const void*> grads = gradients(a, p, device);
        const float* factor = floats(a, 1, device, true);
        return call(a, [&] {
            return reinterpret_cast<decltype(&qadam_adamw_step)>(p.entry)(static_cast<qadam_adamw_t>(p.h), step, lr, grads.data(), factor, stream);
        });
    });
}

PyObject* grad_norm(PyObject*, PyObject* const* argv, Py_ssize_t argc)
{
    return planned<ListPlan, kListName>(argv, argc, 6, [](Args& a, const ListPlan& p, int64_t device, void* stream) {
        const std::vector<const void*> grads = gradients(a, p, device);
        const float max_norm = a.number();
        float* out = floats(a, 2, device);
        return call(a, [&] {
            return reinterpret_cast<decltype(&qadam_grad_norm)>(p.entry)(static_cast<qadam_grad_norm_t>(p.h), grads.data(), max_norm, out, stream);
        });
    });
}

struct EmbeddingPlan {
    qadam_embedding_t h;
    int64_t rows, dim;
    decltype(&qadam_embedding_lookup) lookup;
    decltype(&qadam_embedding_grad) grad;
};

struct Tokens {
    const void* at;
    int32_t bytes;
    int64_t num;
};

Tokens tokens(Args& a, int64_t device)
{
    const at::Tensor* t = on_device(a, *a.next++, device);
    if (!t || (t->scalar_type() != at::kInt && t->scalar_type() != at::kLong) || !t->is_contiguous()) { a.ok = false; return {}; }
    return {t->data_ptr(), (int32_t)t->element_size(), t->numel()};
}

// A matrix, or tokens' rows in any shape one behind the other; at least one row.
struct Rows {
    void* at;
    int32_t type;
    int64_t stride;
};

Rows rows(Args& a, int64_t num, int64_t dim, int64_t device)
{
    const at::Tensor* t = on_device(a, *a.next++, device);
    const int type = t ? element_type(*t) : -1;
    if (type < 0 || num < 1 || t->dim() < 2 || t->size(-1) != dim || t->numel() != num * dim) { a.ok = false; return {}; }
    if (t->is_contiguous()) return {t->data_ptr(), type, dim};
    if (t->dim() != 2 || t->stride(1) != 1 || num < 2) { a.ok = false; return {}; }
    return {t->data_ptr(), type, t->stride(0)};
}

int64_t padding(Args& a)
{
    if (*a.next == Py_None) { ++a.next; return -1; }
    return a.integer();
}

PyObject* embedding_lookup(PyObject*, PyObject* const* argv, Py_ssize_t argc)
{
    return planned<EmbeddingPlan, kEmbeddingName>(argv, argc, 9, [](Args& a, const EmbeddingPlan& p, int64_t device, void* stream) {
        const Rows w = rows(a, p.rows, p.dim, device);
        const Tokens t = tokens(a, device);
        const Rows out = rows(a, t.num, p.dim, device);
        const float scale = a.number();
        const bool codes = *a.next != Py_None;
        const int64_t k_x = padding(a), pad = padding(a);
        if (codes != (w.type > QADAM_F16) || out.type > QADAM_F16 || k_x < INT32_MIN || k_x > INT32_MAX) a.ok = false;
        return call(a, [&] {
            return p.lookup(p.h, w.at, w.type, (int32_t)k_x, w.stride, t.at, t.bytes, t.num, pad, scale, out.at, out.type, out.stride, stream);
        });
    });
}

PyObject* embedding_grad(PyObject*, PyObject* const* argv, Py_ssize_t argc)
{
    return planned<EmbeddingPlan, kEmbeddingName>(argv, argc, 9, [](Args& a, const EmbeddingPlan& p, int64_t device, void* stream) {
        const Tokens t = tokens(a, device);
        const Rows d = rows(a, t.num, p.dim, device), g = rows(a, p.rows, p.dim, device);
        const float scale = a.number();
        const int64_t pad = padding(a), accumulate = a.integer();
        if (d.type > QADAM_F16 || g.type > QADAM_F16) a.ok = false;
        return call(a, [&] {
            return p.grad(p.h, t.at, t.bytes, t.num, pad, scale, d.at, d.type, d.stride, g.at, g.type, g.stride, accumulate != 0, stream);
        });
    });
}

// Layer norm, the product in 8-bit integers, sampling: rows of `dim` elements, the product's results of `outputs`.
struct LayerPlan {
    void* h;
    int64_t dim, outputs;
    void *entry, *entry2;
};

#define QADAM_ENTRY(address, function) reinterpret_cast<decltype(&function)>(address)

// rows of `dim` elements whose number the tensor itself gives
Rows first_rows(Args& a, int64_t dim, int64_t device, int64_t& num)
{
    num = 0;
    if (a.ok && THPVariable_CheckExact(*a.next)) {
        const at::Tensor& t = THPVariable_Unpack(*a.next);
        if (t.dim() >= 2) num = t.numel() / dim;
    }
    return rows(a, num, dim, device);
}

struct Vector {
    void* at;
    int32_t type;
};

// an optional vector of a float type; `like` (>= 0): the type that it has to have
Vector vector(Args& a, int64_t count, int64_t device, int like = -1)
{
    PyObject* o = *a.next++;
    if (o == Py_None) return {nullptr, like < 0 ? 0 : like};
    const at::Tensor* t = on_device(a, o, device);
    const int type = t ? element_type(*t) : -1;
    if (type < 0 || type > QADAM_F16 || (like >= 0 && type != like) || t->numel() != count || !t->is_contiguous()) { a.ok = false; return {}; }
    return {t->data_ptr(), type};
}

PyObject* layer_norm(PyObject*, PyObject* const* argv, Py_ssize_t argc)
{
    return planned<LayerPlan, kLayerName>(argv, argc, 9, [](Args& a, const LayerPlan& p, int64_t device, void* stream) {
        int64_t num;
        const Rows x = first_rows(a, p.dim, device, num);
        const Vector w = vector(a, p.dim, device), b = vector(a, p.dim, device, w.at ? w.type : -1);
        const Rows out = rows(a, num, p.dim, device);
        float* mean = floats(a, num, device, true);
        float* rstd = floats(a, num, device, true);
        if (x.type > QADAM_F16 || out.type > QADAM_F16) a.ok = false;
        return call(a, [&] {
            return QADAM_ENTRY(p.entry, qadam_layer_norm)(static_cast<qadam_layer_norm_t>(p.h), num, x.at, x.type, x.stride, w.at, b.at, b.type,
                                                          out.at, out.type, out.stride, mean, rstd, stream);
        });
    });
}

PyObject* layer_norm_grad(PyObject*, PyObject* const* argv, Py_ssize_t argc)
{
    return planned<LayerPlan, kLayerName>(argv, argc, 12, [](Args& a, const LayerPlan& p, int64_t device, void* stream) {
        int64_t num;
        const Rows dout = first_rows(a, p.dim, device, num), x = rows(a, num, p.dim, device);
        const Vector w = vector(a, p.dim, device);
        const float* mean = floats(a, num, device);
        const float* rstd = floats(a, num, device);
        const Rows dx = rows(a, num, p.dim, device);
        const Vector dw = vector(a, p.dim, device), db = vector(a, p.dim, device, dw.at ? dw.type : -1);
        const int64_t accumulate = a.integer();
        if (dout.type > QADAM_F16 || x.type > QADAM_F16 || dx.type > QADAM_F16) a.ok = false;
        return call(a, [&] {
            return QADAM_ENTRY(p.entry2, qadam_layer_norm_grad)(
                static_cast<qadam_layer_norm_t>(p.h), num, dout.at, dout.type, dout.stride, x.at, x.type, x.stride, w.at, w.type, mean, rstd,
                dx.at, dx.type, dx.stride, dw.at, db.at, db.type, accumulate != 0, stream);
        });
    });
}

PyObject* linear8_quantize(PyObject*, PyObject* const* argv, Py_ssize_t argc)
{
    return planned<LayerPlan, kLayerName>(argv, argc, 6, [](Args& a, const LayerPlan& p, int64_t device, void* stream) {
        int64_t num;
        const Rows x = first_rows(a, p.dim, device, num), codes = rows(a, num, p.dim, device);
        float* scales = floats(a, num, device);
        if (x.type > QADAM_F16 || codes.type != QADAM_CODES8) a.ok = false;
        return call(a, [&] {
            return QADAM_ENTRY(p.entry2, qadam_linear8_quantize)(static_cast<qadam_linear8_t>(p.h), num, x.at, x.type, x.stride,
                                                                 static_cast<int8_t*>(codes.at), codes.stride, scales, stream);
        });
    });
}

PyObject* linear8_forward(PyObject*, PyObject* const* argv, Py_ssize_t argc)
{
    return planned<LayerPlan, kLayerName>(argv, argc, 10, [](Args& a, const LayerPlan& p, int64_t device, void* stream) {
        int64_t num;
        const Rows x = first_rows(a, p.dim, device, num), w = rows(a, p.outputs, p.dim, device), out = rows(a, num, p.outputs, device);
        const float* scales = floats(a, p.outputs, device, true);
        if ((*a.next == Py_None) == (scales == nullptr)) a.ok = false;
        const int64_t k_x = padding(a);
        const float* x_scales = floats(a, num, device, true);
        const Vector b = vector(a, p.outputs, device);
        if ((x_scales ? x.type != QADAM_CODES8 : x.type > QADAM_F16) || w.type != QADAM_CODES8 || out.type > QADAM_F16 || k_x < INT32_MIN || k_x > INT32_MAX)
            a.ok = false;
        return call(a, [&] {
            return QADAM_ENTRY(p.entry, qadam_linear8_forward)(
                static_cast<qadam_linear8_t>(p.h), num, x.at, x.type, x.stride, x_scales, static_cast<int8_t*>(w.at), w.stride, scales,
                (int32_t)k_x, b.at, b.type, out.at, out.type, out.stride, stream);
        });
    });
}

PyObject* sample(PyObject*, PyObject* const* argv, Py_ssize_t argc)
{
    return planned<LayerPlan, kLayerName>(argv, argc, 10, [](Args& a, const LayerPlan& p, int64_t device, void* stream) {
        int64_t num;
        const Rows logits = first_rows(a, p.dim, device, num);
        const float* u = floats(a, num, device);
        const at::Tensor* out = on_device(a, *a.next++, device);
        if (!out || (out->scalar_type() != at::kInt && out->scalar_type() != at::kLong) || out->numel() != num || !out->is_contiguous()) a.ok = false;
        qadam_filters_t f{};
        auto one = [&](const float*& each, float& all) {
            if (PyFloat_Check(*a.next) || PyLong_Check(*a.next)) all = a.number();
            else each = floats(a, num, device);
        };
        one(f.temperatures, f.temperature);
        if (PyLong_Check(*a.next)) {
            const int64_t k = a.integer();
            if (k < INT32_MIN || k > INT32_MAX) a.ok = false;
            f.top_k = (int32_t)k;
        } else {
            const at::Tensor* t = on_device(a, *a.next++, device);
            if (!t || t->scalar_type() != at::kInt || t->numel() != num || !t->is_contiguous()) a.ok = false;
            else f.top_ks = static_cast<const int32_t*>(t->data_ptr());
        }
        one(f.top_ps, f.top_p);
        one(f.min_ps, f.min_p);
        if (logits.type > QADAM_F16) a.ok = false;
        return call(a, [&] {
            return QADAM_ENTRY(p.entry, qadam_sampler_sample)(static_cast<qadam_sampler_t>(p.h), num, logits.at, logits.type, logits.stride, u, &f,
                                                              out->data_ptr(), (int32_t)out->element_size(), stream);
        });
    });
}

template <typename Plan, const char* kPlanName>
PyObject* capsule_of(Plan* p)
{
    PyObject* capsule = PyCapsule_New(p, kPlanName, [](PyObject* c) { delete static_cast<Plan*>(PyCapsule_GetPointer(c, kPlanName)); });
    if (!capsule) delete p;
    return capsule;
}

// (handle, address of the entry point, sizes, element types)
PyObject* list_plan(PyObject*, PyObject* const* argv, Py_ssize_t argc)
{
    Args a{argv, argc == 4};
    const int64_t h = a.ok ? a.integer() : 0, entry = a.ok ? a.integer() : 0;
    if (!a.ok || !PyList_Check(argv[2]) || !PyList_Check(argv[3]) || PyList_GET_SIZE(argv[2]) != PyList_GET_SIZE(argv[3])) {
        PyErr_SetString(PyExc_TypeError, "two integers and two lists of integers expected");
        return nullptr;
    }
    try {
        auto p = std::make_unique<ListPlan>();
        p->h = reinterpret_cast<void*>(h);
        p->entry = reinterpret_cast<void*>(entry);
        for (Py_ssize_t i = 0; i < PyList_GET_SIZE(argv[2]); ++i) {
            PyObject* pair[2] = {PyList_GET_ITEM(argv[2], i), PyList_GET_ITEM(argv[3], i)};
            Args v{pair, true};
            p->numels.push_back(v.integer());
            p->types.push_back(scalar_type(v.integer()));
            if (!v.ok) {
                PyErr_SetString(PyExc_TypeError, "two integers and two lists of integers expected");
                return nullptr;
            }
        }
        return capsule_of<ListPlan, kListName>(p.release());
    } catch (const std::exception& e) {
        PyErr_SetString(PyExc_MemoryError, e.what());
        return nullptr;
    }
}

// (handle, rows, dim, addresses of the two entry points)
PyObject* embedding_plan(PyObject*, PyObject* const* argv, Py_ssize_t argc)
{
    Args a{argv, argc == 5};
    int64_t v[5];
    for (int i = 0; i < 5 && a.ok; ++i) v[i] = a.integer();
    if (!a.ok) {
        PyErr_SetString(PyExc_TypeError, "five integers expected");
        return nullptr;
    }
    return capsule_of<EmbeddingPlan, kEmbeddingName>(new EmbeddingPlan{
        reinterpret_cast<qadam_embedding_t>(v[0]), v[1], v[2], reinterpret_cast<decltype(&qadam_embedding_lookup)>(v[3]),
        reinterpret_cast<decltype(&qadam_embedding_grad)>(v[4])});
}

// (handle, elements of a row, outputs, addresses of the two entry points)
PyObject* layer_plan(PyObject*, PyObject* const* argv, Py_ssize_t argc)
{
    Args a{argv, argc == 5};
    int64_t v[5];
    for (int i = 0; i < 5 && a.ok; ++i) v[i] = a.integer();
    if (!a.ok || v[1] < 1) {
        PyErr_SetString(PyExc_TypeError, "five integers expected, the second one above 0");
        return nullptr;
    }
    return capsule_of<LayerPlan, kLayerName>(new LayerPlan{reinterpret_cast<void*>(v[0]), v[1], v[2], reinterpret_cast<void*>(v[3]),
                                                           reinterpret_cast<void*>(v[4])});
}

void free_plan(PyObject* capsule) { delete static_cast<Plan*>(PyCapsule_GetPointer(capsule, kPlanName)); }

// (handle, workers, params, segments, code bytes, weight code bytes, weight_ef, addresses of the five entry points)
PyObject* plan(PyObject*, PyObject* const* argv, Py_ssize_t argc)
{
    Args a{argv, argc == 12};
    int64_t v[12];
    for (Py_ssize_t i = 0; i < 12 && a.ok; ++i) v[i] = a.integer();
    if (!a.ok || v[1] < 1 || v[1] > QADAM_MAX_WORKERS) {
        PyErr_SetString(PyExc_TypeError, "twelve integers expected");
        return nullptr;
    }
    Plan* p = new Plan{reinterpret_cast<qadam_handle_t>(v[0]), (Py_ssize_t)v[1], v[2], v[3], v[4], v[5], v[6] != 0,
                       reinterpret_cast<decltype(&qadam_worker_quantize)>(v[7]), reinterpret_cast<decltype(&qadam_server_step)>(v[8]),
                       reinterpret_cast<decltype(&qadam_weight_quantize)>(v[9]), reinterpret_cast<decltype(&qadam_step_fused)>(v[10]),
                       reinterpret_cast<decltype(&qadam_step_fused_w)>(v[11])};
    PyObject* capsule = PyCapsule_New(p, kPlanName, free_plan);
    if (!capsule) delete p;
    return capsule;
}

#define QADAM_FUNCTION(name) {#name, reinterpret_cast<PyCFunction>(reinterpret_cast<void (*)()>(name)), METH_FASTCALL, nullptr}

PyMethodDef kFunctions[] = {QADAM_FUNCTION(plan), QADAM_FUNCTION(worker_quantize), QADAM_FUNCTION(server_step),
                            QADAM_FUNCTION(weight_quantize), QADAM_FUNCTION(step_fused), QADAM_FUNCTION(step_fused_w),
                            QADAM_FUNCTION(quantize_segment), QADAM_FUNCTION(list_plan), QADAM_FUNCTION(adamw_step),
                            QADAM_FUNCTION(grad_norm), QADAM_FUNCTION(embedding_plan), QADAM_FUNCTION(embedding_lookup),
                            QADAM_FUNCTION(embedding_grad), QADAM_FUNCTION(layer_plan), QADAM_FUNCTION(layer_norm),
                            QADAM_FUNCTION(layer_norm_grad), QADAM_FUNCTION(linear8_quantize), QADAM_FUNCTION(linear8_forward),
                            QADAM_FUNCTION(sample), {nullptr, nullptr, 0, nullptr}};

PyModuleDef kModule = {PyModuleDef_HEAD_INIT, "_args", "Calls of the library with tensors of the common form.", -1, kFunctions,
                       nullptr, nullptr, nullptr, nullptr};

}  // namespace

PyMODINIT_FUNC PyInit__args(void)
{
    PyObject* m = PyModule_Create(&kModule);
    // tensors are read through inlined code of this version
    if (m && PyModule_AddStringConstant(m, "torch_version", QADAM_TORCH_VERSION) < 0) { Py_DECREF(m); return nullptr; }
    return m;
}
