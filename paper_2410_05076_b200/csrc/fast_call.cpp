// Calls of the C-ABI whose device work takes a few microseconds, with their tensors checked and marshalled in C++: the same
// in Python costs more than the kernels take. Addresses of the C functions come from the binding (init), so
// that both use one loaded library.
#include <Python.h>

#include <ATen/core/Tensor.h>
#include <c10/cuda/CUDAStream.h>
#include <torch/csrc/autograd/python_variable.h>

#include <cstring>
#include <string>

#include "../../include/tidal.h"

namespace {

decltype(&tidal_page_map) f_page_map;
decltype(&tidal_kv_write) f_kv_write;
decltype(&tidal_block_bounds) f_block_bounds;
decltype(&tidal_block_select) f_block_select;
decltype(&tidal_block_attn) f_block_attn;
decltype(&tidal_rope) f_rope;
decltype(&tidal_rope_write) f_rope_write;
decltype(&tidal_chunk_attn) f_chunk_attn;
decltype(&tidal_chunk_weights) f_chunk_weights;
decltype(&tidal_evict_select) f_evict_select;
decltype(&tidal_kv_gather) f_kv_gather;

struct Refused {};                           // a Python exception is set

[[noreturn]] void refuse(const std::string& text) {
    PyErr_SetString(PyExc_ValueError, text.c_str());
    throw Refused{};
}

std::string shape_text(const int64_t* s, size_t n) {
    std::string t = "(";
    for (size_t i = 0; i < n; ++i) t += (i ? ", " : "") + std::to_string(s[i]);
    return t + (n == 1 ? ",)" : ")");
}

// The tensor behind an argument, null for None.
const at::Tensor* tensor(PyObject* o, const char* name, at::ScalarType type, int device) {
    if (o == Py_None) return nullptr;
    if (!THPVariable_Check(o)) refuse(std::string(name) + ": a tensor is wanted");
    const at::Tensor& t = THPVariable_Unpack(o);
    if (t.scalar_type() != type) refuse(std::string(name) + ": " + c10::toString(type) + " is wanted, got " + c10::toString(t.scalar_type()));
    if (!t.is_cuda() || t.get_device() != device)
        refuse(std::string(name) + ": a tensor on cuda:" + std::to_string(device) + " is wanted, got one on " + t.device().str());
    return &t;
}

const at::Tensor& required(PyObject* o, const char* name, at::ScalarType type, int device) {
    const at::Tensor* t = tensor(o, name, type, device);
    if (!t) refuse(std::string(name) + ": a tensor is wanted");
    return *t;
}

void contiguous(const at::Tensor& t, const char* name) {
    if (!t.is_contiguous()) refuse(std::string(name) + ": a contiguous tensor is wanted");
}

void shaped(const at::Tensor& t, const char* name, std::initializer_list<int64_t> want) {
    const auto s = t.sizes();
    if (s.size() != want.size() || !std::equal(want.begin(), want.end(), s.begin()))
        refuse(std::string(name) + ": shape " + shape_text(want.begin(), want.size()) + " is wanted, got " + shape_text(s.data(), s.size()));
}

void* contiguous_data(PyObject* o, const char* name, at::ScalarType type, int device, std::initializer_list<int64_t> want) {
    const at::Tensor* t = tensor(o, name, type, device);
    if (!t) return nullptr;
    contiguous(*t, name);
    shaped(*t, name, want);
    return t->data_ptr();
}

long as_long(PyObject* o) {
    const long v = PyLong_AsLong(o);
    if (v == -1 && PyErr_Occurred()) throw Refused{};
    return v;
}
int as_int(PyObject* o, const char* name) {
    const long v = as_long(o);
    if (v < INT32_MIN || v > INT32_MAX) refuse(std::string(name) + ": does not fit 32 bits");
    return (int)v;
}
int32_t count_of(const at::Tensor& t, const char* name) {
    if (t.numel() > INT32_MAX) refuse(std::string(name) + ": too many elements");
    return (int32_t)t.numel();
}

// The bytes of a ctypes tidal_kv_t.
struct Descriptor {
    Py_buffer view{};
    const tidal_kv_t* kv = nullptr;
    explicit Descriptor(PyObject* o) {
        if (PyObject_GetBuffer(o, &view, PyBUF_SIMPLE) != 0) throw Refused{};
        if (view.len != (Py_ssize_t)sizeof(tidal_kv_t)) { PyBuffer_Release(&view); refuse("layer: not a cache descriptor"); }
        kv = static_cast<const tidal_kv_t*>(view.buf);
    }
    ~Descriptor() { PyBuffer_Release(&view); }
    Descriptor(const Descriptor&) = delete;
};

// The bytes of a ctypes tidal_rope_t.
struct Plan {
    Py_buffer view{};
    const tidal_rope_t* rope = nullptr;
    explicit Plan(PyObject* o) {
        if (PyObject_GetBuffer(o, &view, PyBUF_SIMPLE) != 0) throw Refused{};
        if (view.len != (Py_ssize_t)sizeof(tidal_rope_t)) { PyBuffer_Release(&view); refuse("plan: not a rope_plan"); }
        rope = static_cast<const tidal_rope_t*>(view.buf);
    }
    ~Plan() { PyBuffer_Release(&view); }
    Plan(const Plan&) = delete;
};

// Rows [tokens, heads, head_dim] of bf16, those of a token contiguous; nothing for None.
struct Rows {
    void* data = nullptr;
    int64_t tokens = 0, heads = 0, stride = 0;
    Rows(PyObject* o, const char* name, int device) {
        const at::Tensor* t = tensor(o, name, at::kBFloat16, device);
        if (!t) return;
        if (t->dim() != 3 || t->size(2) != 128 || t->size(0) > INT32_MAX || t->size(1) > INT32_MAX)
            refuse(std::string(name) + ": [tokens, heads, 128] is wanted, got " + shape_text(t->sizes().data(), t->dim()));
        data = t->data_ptr();
        tokens = t->size(0);
        heads = t->size(1);
        if (tokens && heads && (t->stride(2) != 1 || (heads > 1 && t->stride(1) != 128))) refuse(std::string(name) + ": the rows of a token have to be contiguous");
        stride = tokens > 1 ? t->stride(0) : heads * 128;   // (a single token's stride says nothing: torch may give any)
    }
    void like(const Rows& other, const char* name) const {
        if (!data != !other.data || tokens != other.tokens || heads != other.heads) refuse(std::string(name) + ": the shape of its input is wanted");
    }
};

double as_double(PyObject* o) {
    const double v = PyFloat_AsDouble(o);
    if (v == -1.0 && PyErr_Occurred()) throw Refused{};
    return v;
}

tidal_ctx_t* context(PyObject* o) { return static_cast<tidal_ctx_t*>(PyLong_AsVoidPtr(o)); }
void* stream_of(int device) { return c10::cuda::getCurrentCUDAStream((c10::DeviceIndex)device).stream(); }

template <typename F>
PyObject* guarded(Py_ssize_t have, Py_ssize_t want, F&& body) {
    if (have != want) { PyErr_SetString(PyExc_TypeError, "wrong number of arguments"); return nullptr; }
    try {
        return PyLong_FromLong(body());
    } catch (const Refused&) {
        return nullptr;
    } catch (const std::exception& e) {
        PyErr_SetString(PyExc_RuntimeError, e.what());
        return nullptr;
    }
}

// page_map(ctx, device, old_lens, new_lens, page_table, free_pages, num_free, slots, num_free_out, positions, token_offsets)
PyObject* page_map(PyObject*, PyObject* const* a, Py_ssize_t n) {
    return guarded(n, 11, [&]() -> long {
        const int dev = as_int(a[1], "device");
        const at::Tensor& old_lens = required(a[2], "old_lens", at::kInt, dev);
        const at::Tensor& table = required(a[4], "page_table", at::kInt, dev);
        const at::Tensor& free_pages = required(a[5], "free_pages", at::kInt, dev);
        const at::Tensor& num_free = required(a[6], "num_free", at::kInt, dev);
        const at::Tensor& slots = required(a[7], "slots", at::kLong, dev);
        const at::Tensor& out = a[8] == Py_None ? num_free : required(a[8], "num_free_out", at::kInt, dev);
        contiguous(old_lens, "old_lens"); contiguous(table, "page_table"); contiguous(free_pages, "free_pages"); contiguous(slots, "slots");
        const int32_t batch = count_of(old_lens, "old_lens"), cap = count_of(slots, "slots"), pages = count_of(free_pages, "free_pages");
        if (table.dim() != 2 || table.size(0) != batch || table.size(1) > INT32_MAX)
            refuse("page_table: [" + std::to_string(batch) + ", pages] is wanted, got " + shape_text(table.sizes().data(), table.dim()));
        if (num_free.numel() != 1 || out.numel() != 1) refuse("num_free, num_free_out: one element is wanted");
        if (a[3] == Py_None) refuse("new_lens: a tensor is wanted");
        return f_page_map(context(a[0]), batch, static_cast<const int32_t*>(old_lens.data_ptr()),
                          static_cast<const int32_t*>(contiguous_data(a[3], "new_lens", at::kInt, dev, {batch})),
                          static_cast<int32_t*>(table.data_ptr()), (int32_t)table.size(1), pages, static_cast<int32_t*>(free_pages.data_ptr()),
                          static_cast<const int32_t*>(num_free.data_ptr()), static_cast<int32_t*>(out.data_ptr()), cap,
                          static_cast<int64_t*>(slots.data_ptr()), static_cast<int32_t*>(contiguous_data(a[9], "positions", at::kInt, dev, {cap})),
                          static_cast<int32_t*>(contiguous_data(a[10], "token_offsets", at::kInt, dev, {(int64_t)batch + 1})), stream_of(dev));
    });
}

// kv_write(ctx, device, descriptor, k_new, v_new, slots)
PyObject* kv_write(PyObject*, PyObject* const* a, Py_ssize_t n) {
    return guarded(n, 6, [&]() -> long {
        const int dev = as_int(a[1], "device");
        const Descriptor d(a[2]);
        const at::Tensor& slots = required(a[5], "slots", at::kLong, dev);
        contiguous(slots, "slots");
        const int32_t tokens = count_of(slots, "slots");
        const at::Tensor* row[2];
        for (int i = 0; i < 2; ++i) {
            const char* name = i ? "v_new" : "k_new";
            row[i] = &required(a[3 + i], name, at::kBFloat16, dev);
            shaped(*row[i], name, {tokens, d.kv->num_kv_heads, d.kv->head_dim});
            if (tokens && (row[i]->stride(2) != 1 || (d.kv->num_kv_heads > 1 && row[i]->stride(1) != d.kv->head_dim)))
                refuse(std::string(name) + ": the rows of a token have to be contiguous");
        }
        // (a single token's stride says nothing: torch may give any)
        const int64_t one = (int64_t)d.kv->num_kv_heads * d.kv->head_dim;
        return f_kv_write(context(a[0]), d.kv, tokens, row[0]->data_ptr(), row[1]->data_ptr(), tokens > 1 ? row[0]->stride(0) : one,
                          tokens > 1 ? row[1]->stride(0) : one, static_cast<const int64_t*>(slots.data_ptr()), stream_of(dev));
    });
}

int32_t bound_blocks(const tidal_kv_t* kv, const at::Tensor& t) {
    const bool paged = kv->kv_layout == TIDAL_KV_PAGED;
    const int64_t blocks = t.dim() == (paged ? 4 : 5) ? t.size(paged ? 0 : 2) : -1;
    if (paged) shaped(t, "bounds", {blocks, kv->num_kv_heads, 2, kv->head_dim});
    else shaped(t, "bounds", {kv->batch, kv->num_kv_heads, blocks, 2, kv->head_dim});
    if (blocks > INT32_MAX) refuse("bounds: too many blocks");
    contiguous(t, "bounds");
    return (int32_t)blocks;
}

// block_bounds(ctx, device, descriptor, bounds, start_lens, max_new)
PyObject* block_bounds(PyObject*, PyObject* const* a, Py_ssize_t n) {
    return guarded(n, 6, [&]() -> long {
        const int dev = as_int(a[1], "device");
        const Descriptor d(a[2]);
        const at::Tensor& bounds = required(a[3], "bounds", at::kBFloat16, dev);
        return f_block_bounds(context(a[0]), d.kv, static_cast<const int32_t*>(contiguous_data(a[4], "start_lens", at::kInt, dev, {d.kv->batch})),
                              as_int(a[5], "max_new"), bounds.data_ptr(), bound_blocks(d.kv, bounds), stream_of(dev));
    });
}

// block_select(ctx, device, descriptor, bounds, q, m, granularity, keep_first, keep_last, idx, idx_count)
PyObject* block_select(PyObject*, PyObject* const* a, Py_ssize_t n) {
    return guarded(n, 11, [&]() -> long {
        const int dev = as_int(a[1], "device");
        const Descriptor d(a[2]);
        const tidal_kv_t* kv = d.kv;
        const at::Tensor& bounds = required(a[3], "bounds", at::kBFloat16, dev);
        const int m = as_int(a[5], "m"), gran = as_int(a[6], "granularity");
        const int64_t hi = gran == TIDAL_SEL_PER_QHEAD ? kv->num_q_heads : gran == TIDAL_SEL_PER_KVHEAD ? kv->num_kv_heads : 1;
        const void* q = contiguous_data(a[4], "q", at::kBFloat16, dev, {kv->batch, kv->num_q_heads, kv->head_dim});
        void* idx = contiguous_data(a[9], "idx", at::kInt, dev, {kv->batch, hi, m > 1 ? m : 1});
        void* count = contiguous_data(a[10], "idx_count", at::kInt, dev, {kv->batch});
        return f_block_select(context(a[0]), kv, q, bounds.data_ptr(), bound_blocks(kv, bounds), m, gran, as_int(a[7], "keep_first"),
                              as_int(a[8], "keep_last"), static_cast<int32_t*>(idx), static_cast<int32_t*>(count), stream_of(dev));
    });
}

// block_attn(ctx, device, descriptor, q, idx, idx_count, out, out is bf16)
PyObject* block_attn(PyObject*, PyObject* const* a, Py_ssize_t n) {
    return guarded(n, 8, [&]() -> long {
        const int dev = as_int(a[1], "device");
        const Descriptor d(a[2]);
        const tidal_kv_t* kv = d.kv;
        const at::Tensor& idx = required(a[4], "idx", at::kInt, dev);
        contiguous(idx, "idx");
        if (idx.dim() != 3 || idx.size(0) != kv->batch || idx.size(1) > INT32_MAX || idx.size(2) > INT32_MAX)
            refuse("idx: [" + std::to_string(kv->batch) + ", Hi, m] is wanted, got " + shape_text(idx.sizes().data(), idx.dim()));
        const void* q = contiguous_data(a[3], "q", at::kBFloat16, dev, {kv->batch, kv->num_q_heads, kv->head_dim});
        void* out = contiguous_data(a[6], "out", a[7] == Py_True ? at::kBFloat16 : at::kFloat, dev, {kv->batch, kv->num_q_heads, kv->head_dim});
        return f_block_attn(context(a[0]), kv, q, static_cast<const int32_t*>(idx.data_ptr()),
                            static_cast<const int32_t*>(contiguous_data(a[5], "idx_count", at::kInt, dev, {kv->batch})), (int32_t)idx.size(2),
                            (int32_t)idx.size(1), static_cast<float*>(out), stream_of(dev));
    });
}

// rope(ctx, device, plan, q, k, positions, q_weight, k_weight, eps, q_out, k_out)
PyObject* rope(PyObject*, PyObject* const* a, Py_ssize_t n) {
    return guarded(n, 11, [&]() -> long {
        const int dev = as_int(a[1], "device");
        const Plan plan(a[2]);
        const Rows q(a[3], "q", dev), k(a[4], "k", dev), qo(a[9], "q_out", dev), ko(a[10], "k_out", dev);
        if (!q.data && !k.data && !q.tokens && !k.tokens && a[3] == Py_None && a[4] == Py_None) refuse("q, k: a tensor is wanted");
        qo.like(q, "q_out");
        ko.like(k, "k_out");
        const int64_t tokens = a[3] != Py_None ? q.tokens : k.tokens;
        if (a[3] != Py_None && a[4] != Py_None && q.tokens != k.tokens) refuse("k: as many tokens as q's are wanted");
        return f_rope(context(a[0]), plan.rope, (int32_t)tokens, (int32_t)q.heads, (int32_t)k.heads, q.data, q.stride, k.data, k.stride,
                      static_cast<const int32_t*>(contiguous_data(a[5], "positions", at::kInt, dev, {tokens})),
                      contiguous_data(a[6], "q_weight", at::kBFloat16, dev, {128}), contiguous_data(a[7], "k_weight", at::kBFloat16, dev, {128}),
                      (float)as_double(a[8]), qo.data, qo.stride, ko.data, ko.stride, stream_of(dev));
    });
}

// rope_write(ctx, device, descriptor, plan, q, k_new, v_new, positions, slots, q_weight, k_weight, eps, q_out)
PyObject* rope_write(PyObject*, PyObject* const* a, Py_ssize_t n) {
    return guarded(n, 13, [&]() -> long {
        const int dev = as_int(a[1], "device");
        const Descriptor d(a[2]);
        const Plan plan(a[3]);
        const at::Tensor& slots = required(a[8], "slots", at::kLong, dev);
        contiguous(slots, "slots");
        const int64_t tokens = count_of(slots, "slots");
        const Rows q(a[4], "q", dev), k(a[5], "k_new", dev), v(a[6], "v_new", dev), qo(a[12], "q_out", dev);
        qo.like(q, "q_out");
        if (a[4] != Py_None && (q.tokens != tokens || q.heads != d.kv->num_q_heads)) refuse("q: [tokens, num_q_heads, 128] is wanted");
        for (const auto& r : {std::make_pair(&k, "k_new"), std::make_pair(&v, "v_new")})
            if (r.first->tokens != tokens || r.first->heads != d.kv->num_kv_heads) refuse(std::string(r.second) + ": [tokens, num_kv_heads, 128] is wanted");
        return f_rope_write(context(a[0]), plan.rope, d.kv, (int32_t)tokens, q.data, q.stride, k.data, k.stride, v.data, v.stride,
                            static_cast<const int32_t*>(contiguous_data(a[7], "positions", at::kInt, dev, {tokens})),
                            static_cast<const int64_t*>(slots.data_ptr()), contiguous_data(a[9], "q_weight", at::kBFloat16, dev, {128}),
                            contiguous_data(a[10], "k_weight", at::kBFloat16, dev, {128}), (float)as_double(a[11]), qo.data, qo.stride, stream_of(dev));
    });
}

// chunk_attn(ctx, device, descriptor, q, q_offsets, max_new, causal, window, out, out is bf16, lse)
PyObject* chunk_attn(PyObject*, PyObject* const* a, Py_ssize_t n) {
    return guarded(n, 11, [&]() -> long {
        const int dev = as_int(a[1], "device");
        const Descriptor d(a[2]);
        const tidal_kv_t* kv = d.kv;
        const Rows q(a[3], "q", dev);
        if (a[3] == Py_None || q.heads != kv->num_q_heads) refuse("q: [tokens, num_q_heads, 128] is wanted");
        void* out = contiguous_data(a[8], "out", a[9] == Py_True ? at::kBFloat16 : at::kFloat, dev, {q.tokens, q.heads, 128});
        void* lse = contiguous_data(a[10], "lse", at::kFloat, dev, {q.tokens, q.heads});
        return f_chunk_attn(context(a[0]), kv, (int32_t)q.tokens, q.data, q.stride,
                            static_cast<const int32_t*>(contiguous_data(a[4], "q_offsets", at::kInt, dev, {(int64_t)kv->batch + 1})), as_int(a[5], "max_new"),
                            as_int(a[6], "causal"), as_int(a[7], "window"), static_cast<float*>(out), static_cast<float*>(lse), stream_of(dev));
    });
}

// [batch, heads, stride] of fp32, contiguous; heads and stride come back.
float* weight_rows(PyObject* o, const char* name, int device, int64_t batch, int64_t& heads, int64_t& stride) {
    const at::Tensor* t = tensor(o, name, at::kFloat, device);
    heads = stride = 0;
    if (!t) return nullptr;
    contiguous(*t, name);
    if (t->dim() != 3 || t->size(0) != batch || t->size(1) > INT32_MAX)
        refuse(std::string(name) + ": [" + std::to_string(batch) + ", heads, positions] is wanted, got " + shape_text(t->sizes().data(), t->dim()));
    heads = t->size(1);
    stride = t->size(2);
    return static_cast<float*>(t->data_ptr());
}

// chunk_weights(ctx, device, descriptor, q, q_offsets, lse, weights, decay, max_new, causal, window, last)
PyObject* chunk_weights(PyObject*, PyObject* const* a, Py_ssize_t n) {
    return guarded(n, 12, [&]() -> long {
        const int dev = as_int(a[1], "device");
        const Descriptor d(a[2]);
        const tidal_kv_t* kv = d.kv;
        const Rows q(a[3], "q", dev);
        if (a[3] == Py_None || q.heads != kv->num_q_heads) refuse("q: [tokens, num_q_heads, 128] is wanted");
        int64_t heads, stride;
        float* w = weight_rows(a[6], "weights", dev, kv->batch, heads, stride);
        return f_chunk_weights(context(a[0]), kv, (int32_t)q.tokens, q.data, q.stride,
                               static_cast<const int32_t*>(contiguous_data(a[4], "q_offsets", at::kInt, dev, {(int64_t)kv->batch + 1})), as_int(a[8], "max_new"),
                               as_int(a[9], "causal"), as_int(a[10], "window"), as_int(a[11], "last"),
                               static_cast<const float*>(contiguous_data(a[5], "lse", at::kFloat, dev, {q.tokens, q.heads})), (float)as_double(a[7]), w, stride,
                               (int32_t)heads, stream_of(dev));
    });
}

// evict_select(ctx, device, descriptor, weights, m, keep_first, keep_last, kept, new_lens)
PyObject* evict_select(PyObject*, PyObject* const* a, Py_ssize_t n) {
    return guarded(n, 9, [&]() -> long {
        const int dev = as_int(a[1], "device");
        const Descriptor d(a[2]);
        int64_t heads, stride;
        const float* w = weight_rows(a[3], "weights", dev, d.kv->batch, heads, stride);
        const int m = as_int(a[4], "m");
        void* kept = contiguous_data(a[7], "kept", at::kInt, dev, {d.kv->batch, heads, m > 1 ? m : 1});
        void* lens = contiguous_data(a[8], "new_lens", at::kInt, dev, {d.kv->batch});
        return f_evict_select(context(a[0]), d.kv, w, stride, (int32_t)heads, m, as_int(a[5], "keep_first"), as_int(a[6], "keep_last"),
                              static_cast<int32_t*>(kept), static_cast<int32_t*>(lens), stream_of(dev));
    });
}

// kv_gather(ctx, device, descriptor, descriptor or None, kept, counts, weights, weights_out)
PyObject* kv_gather(PyObject*, PyObject* const* a, Py_ssize_t n) {
    return guarded(n, 8, [&]() -> long {
        const int dev = as_int(a[1], "device");
        const Descriptor d(a[2]);
        const Descriptor into(a[3] == Py_None ? a[2] : a[3]);
        const at::Tensor& kept = required(a[4], "kept", at::kInt, dev);
        contiguous(kept, "kept");
        if (kept.dim() != 3 || kept.size(0) != d.kv->batch || kept.size(1) > INT32_MAX || kept.size(2) > INT32_MAX)
            refuse("kept: [" + std::to_string(d.kv->batch) + ", heads, m] is wanted, got " + shape_text(kept.sizes().data(), kept.dim()));
        int64_t heads, stride, heads_out, stride_out;
        const float* w = weight_rows(a[6], "weights", dev, d.kv->batch, heads, stride);
        float* wo = weight_rows(a[7], "weights_out", dev, d.kv->batch, heads_out, stride_out);
        if ((w && heads != kept.size(1)) || (wo && heads_out != kept.size(1))) refuse("weights, weights_out: as many heads as kept's are wanted");
        return f_kv_gather(context(a[0]), d.kv, a[3] == Py_None ? nullptr : into.kv, static_cast<const int32_t*>(kept.data_ptr()),
                           static_cast<const int32_t*>(contiguous_data(a[5], "counts", at::kInt, dev, {d.kv->batch})), (int32_t)kept.size(2),
                           (int32_t)kept.size(1), w, stride, wo, stride_out, stream_of(dev));
    });
}

// init(sizes of the cache descriptor and the rope plan, addresses of tidal_page_map, kv_write, block_bounds, block_select, block_attn, rope,
// rope_write, chunk_attn, chunk_weights, evict_select, kv_gather)
PyObject* init(PyObject*, PyObject* const* a, Py_ssize_t n) {
    return guarded(n, 13, [&]() -> long {
        if (as_long(a[0]) != (long)sizeof(tidal_kv_t) || as_long(a[1]) != (long)sizeof(tidal_rope_t)) refuse("a descriptor's size differs from the library's");
        int i = 2;
        auto take = [&](auto& f) { f = reinterpret_cast<std::remove_reference_t<decltype(f)>>(PyLong_AsVoidPtr(a[i++])); };
        take(f_page_map); take(f_kv_write); take(f_block_bounds); take(f_block_select); take(f_block_attn);
        take(f_rope); take(f_rope_write); take(f_chunk_attn); take(f_chunk_weights); take(f_evict_select); take(f_kv_gather);
        return 0;
    });
}

#define ENTRY(f) {#f, reinterpret_cast<PyCFunction>(reinterpret_cast<void (*)()>(f)), METH_FASTCALL, nullptr}
PyMethodDef methods[] = {ENTRY(init), ENTRY(page_map), ENTRY(kv_write), ENTRY(block_bounds), ENTRY(block_select), ENTRY(block_attn),
                         ENTRY(rope), ENTRY(rope_write), ENTRY(chunk_attn), ENTRY(chunk_weights), ENTRY(evict_select), ENTRY(kv_gather),
                         {nullptr, nullptr, 0, nullptr}};
PyModuleDef module = {PyModuleDef_HEAD_INIT, "_fast_call", nullptr, -1, methods, nullptr, nullptr, nullptr, nullptr};

}  // namespace

PyMODINIT_FUNC PyInit__fast_call() { return PyModule_Create(&module); }
