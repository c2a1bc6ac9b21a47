// Single-tensor and cache calls of the Python binding: the checks of srs.py on the tensors and the call into libsrs.so in one step.  The
// functions return what the library returned, or None where any argument is not what the checks ask for (or is anything but
// a plain tensor or integer): srs.py then goes its general way, which raises the errors.  What bounds a call on a small
// tensor is the host: extract and apply of 4096 elements took 11.7 us from Python and ctypes; it takes
// 7.8 us this way (8.1 against 12.1 us per pair in a loop of their own).
#include "srs.h"

#include <torch/csrc/autograd/python_variable.h>

#include <ATen/TensorSubclassLikeUtils.h>
#include <ATen/ops/empty.h>

#include <cmath>
#include <cstdint>

namespace {

// A plain contiguous tensor on the GPU of `width` bytes per element; null otherwise.
const at::Tensor *on_gpu(PyObject *o, size_t width) {
    if (!THPVariable_CheckExact(o)) return nullptr;
    const at::Tensor &t = THPVariable_Unpack(o);
    if (!t.defined() || at::isTensorSubclassLike(t) || !t.is_cuda() || t.layout() != at::kStrided) return nullptr;
    if ((size_t)t.element_size() != width || !t.is_contiguous()) return nullptr;
    return &t;
}

bool number(PyObject *o, uint64_t &v) {
    if (!PyLong_CheckExact(o)) return false;
    v = PyLong_AsUnsignedLongLong(o);
    if (v == (uint64_t)-1 && PyErr_Occurred()) { PyErr_Clear(); return false; }
    return true;
}

struct Payload { void *I, *V, *counts; };

bool payload(PyObject *const *args, uint64_t n, uint64_t be, uint64_t cap, size_t width, Payload &p) {
    if (be == 0 || cap == 0 || be > 0x7fffffffull || cap > 0x7fffffffull) return false;
    const at::Tensor *I = on_gpu(args[0], 4), *V = on_gpu(args[1], width), *c = on_gpu(args[2], 4);
    if (!I || !V || !c || I->scalar_type() != at::kInt) return false;
    const uint64_t nb = (n + be - 1) / be;
    if ((uint64_t)I->numel() < nb * cap || (uint64_t)V->numel() < nb * cap || (uint64_t)c->numel() < nb) return false;
    p = Payload{I->data_ptr(), V->data_ptr(), c->data_ptr()};
    return true;
}

typedef int (*ExtractFn)(void *, void *, const void *, uint64_t, uint64_t, void *, void *, void *, uint64_t, void *);
typedef int (*ApplyFn)(void *, void *, uint64_t, uint64_t, const void *, const void *, const void *, uint64_t, void *);

// Nothing that torch throws leaves a function: the general way meets the same tensor and reports it.
// extract(function, context, old, new, bucket_elems, I, V, counts, cap, stream, width, new_width)
PyObject *extract(PyObject *, PyObject *const *args, Py_ssize_t n_args) {
    uint64_t fn, ctx, be, cap, stream, width, new_width;
    if (n_args != 12 || !number(args[0], fn) || !number(args[1], ctx) || !number(args[4], be) || !number(args[8], cap) ||
        !number(args[9], stream) || !number(args[10], width) || !number(args[11], new_width))
        Py_RETURN_NONE;
    uint64_t n;
    Payload p;
    void *old_p, *new_p;
    try {
        const at::Tensor *o = on_gpu(args[2], width), *w = on_gpu(args[3], new_width);
        if (!o || !w || o->numel() != w->numel() || (new_width != width && w->scalar_type() != at::kFloat)) Py_RETURN_NONE;
        n = (uint64_t)o->numel();
        if (n > 0x7fffffffull || !payload(args + 5, n, be, cap, width, p)) Py_RETURN_NONE;
        old_p = o->data_ptr(), new_p = w->data_ptr();
    } catch (...) {
        Py_RETURN_NONE;
    }
    int rc;
    Py_BEGIN_ALLOW_THREADS
    rc = ((ExtractFn)fn)((void *)ctx, old_p, new_p, n, be, p.I, p.V, p.counts, cap, (void *)stream);
    Py_END_ALLOW_THREADS
    return PyLong_FromLong(rc);
}

// apply(function, context, weights, bucket_elems, I, V, counts, cap, stream, width)
PyObject *apply(PyObject *, PyObject *const *args, Py_ssize_t n_args) {
    uint64_t fn, ctx, be, cap, stream, width;
    if (n_args != 10 || !number(args[0], fn) || !number(args[1], ctx) || !number(args[3], be) || !number(args[7], cap) ||
        !number(args[8], stream) || !number(args[9], width))
        Py_RETURN_NONE;
    uint64_t n;
    Payload p;
    void *weights;
    try {
        const at::Tensor *w = on_gpu(args[2], width);
        if (!w) Py_RETURN_NONE;
        n = (uint64_t)w->numel();
        if (n > 0x7fffffffull || !payload(args + 4, n, be, cap, width, p)) Py_RETURN_NONE;
        weights = w->data_ptr();
    } catch (...) {
        Py_RETURN_NONE;
    }
    int rc;
    Py_BEGIN_ALLOW_THREADS
    rc = ((ApplyFn)fn)((void *)ctx, weights, n, be, p.I, p.V, p.counts, cap, (void *)stream);
    Py_END_ALLOW_THREADS
    return PyLong_FromLong(rc);
}

// ---- the cache's calls: arguments as in srs.py, after the library function, the context and its device --------------------------------

const at::Tensor *plain(PyObject *o, int64_t device) {
    if (!THPVariable_CheckExact(o)) return nullptr;
    const at::Tensor &t = THPVariable_Unpack(o);
    if (!t.defined() || at::isTensorSubclassLike(t) || !t.is_cuda() || t.layout() != at::kStrided || t.get_device() != device) return nullptr;
    return &t;
}

// A contiguous tensor of the type, of at least so many elements.
const at::Tensor *dense(PyObject *o, int64_t device, at::ScalarType type, int64_t at_least) {
    const at::Tensor *t = plain(o, device);
    return t && t->scalar_type() == type && t->is_contiguous() && t->numel() >= at_least ? t : nullptr;
}

bool real(PyObject *o, double &v) {
    if (PyFloat_CheckExact(o)) v = PyFloat_AS_DOUBLE(o);
    else if (PyLong_CheckExact(o)) v = PyLong_AsDouble(o);
    else return false;
    if (v == -1.0 && PyErr_Occurred()) { PyErr_Clear(); return false; }
    return true;
}

int type_code(at::ScalarType t) { return t == at::kBFloat16 ? SRS_BF16 : t == at::kHalf ? SRS_FP16 : t == at::kFloat ? SRS_FP32 : -1; }

bool rows(PyObject *o, int64_t device, int64_t tokens, int64_t head_dim, at::ScalarType type, srs_rows &r) {
    const at::Tensor *t = plain(o, device);
    if (!t || t->scalar_type() != type || t->dim() != 3 || t->size(0) != tokens || t->size(2) != head_dim || t->size(1) > 65536 || (head_dim != 1 && t->stride(2) != 1))
        return false;
    r = srs_rows{t->data_ptr(), (uint32_t)t->size(1), t->stride(0), t->stride(1)};
    return true;
}

bool cache_of(PyObject *ko, PyObject *vo, int64_t device, srs_cache &c, at::ScalarType &type) {
    const at::Tensor *k = plain(ko, device), *v = plain(vo, device);
    if (!k || !v || k->dim() != 4 || k->sizes() != v->sizes() || k->scalar_type() != v->scalar_type() || type_code(k->scalar_type()) < 0) return false;
    for (int d = 0; d < 4; ++d)
        if (k->size(d) > 0x7fffffff) return false;
    if (k->size(3) != 1 && (k->stride(3) != 1 || v->stride(3) != 1)) return false;
    type = k->scalar_type();
    c = srs_cache{k->data_ptr(), v->data_ptr(), type_code(type), (uint32_t)k->size(0), (uint32_t)k->size(1), (uint32_t)k->size(2), (uint32_t)k->size(3),
                  k->stride(0), k->stride(1), k->stride(2), v->stride(0), v->stride(1), v->stride(2)};
    return true;
}

struct Callee { uint64_t fn, ctx, device; };
bool callee(PyObject *const *args, Callee &c) { return number(args[0], c.fn) && number(args[1], c.ctx) && number(args[2], c.device) && c.device < 128; }

#define SRS_CALL(expr)              \
    int rc;                         \
    Py_BEGIN_ALLOW_THREADS          \
    rc = (expr);                    \
    Py_END_ALLOW_THREADS            \
    return PyLong_FromLong(rc)

// cache_tables(function, context, device, start, count, page_tokens, held, table, free_pages, free_count, token_begin, slots, positions, stream)
PyObject *cache_tables(PyObject *, PyObject *const *args, Py_ssize_t n_args) {
    Callee c;
    uint64_t page, stream;
    const at::Tensor *start, *count, *held, *table, *pages, *left, *begin, *slots, *positions;
    if (n_args != 14 || !callee(args, c) || !number(args[5], page) || page > 0x7fffffff || !number(args[13], stream)) Py_RETURN_NONE;
    int64_t n, width, most;
    try {
        if (!(start = dense(args[3], c.device, at::kInt, 0))) Py_RETURN_NONE;
        n = start->numel();
        if (!(count = dense(args[4], c.device, at::kInt, n)) || !(held = dense(args[6], c.device, at::kInt, n)) || !(table = dense(args[7], c.device, at::kInt, 0)) ||
            !(pages = dense(args[8], c.device, at::kInt, 0)) || !(left = dense(args[9], c.device, at::kInt, 1)) || !(begin = dense(args[10], c.device, at::kInt, n + 1)) ||
            !(slots = dense(args[11], c.device, at::kLong, 0)) || !(positions = dense(args[12], c.device, at::kInt, slots->numel())))
            Py_RETURN_NONE;
        if (table->dim() != 2 || table->size(0) != n || n > 0x7fffffff || table->size(1) > 0x7fffffff || pages->numel() > 0x7fffffff) Py_RETURN_NONE;
        width = table->size(1); most = slots->numel();
    } catch (...) {
        Py_RETURN_NONE;
    }
    SRS_CALL(((decltype(&srs_cache_tables))c.fn)((srs_ctx *)c.ctx, (int32_t *)start->data_ptr(), (int32_t *)count->data_ptr(), (uint32_t)n, (uint32_t)page,
                                                 (int32_t *)held->data_ptr(), (int32_t *)table->data_ptr(), (uint32_t)width, (int32_t *)pages->data_ptr(),
                                                 (int32_t *)left->data_ptr(), (uint32_t)pages->numel(), (int32_t *)begin->data_ptr(), (int64_t *)slots->data_ptr(),
                                                 (int32_t *)positions->data_ptr(), (uint64_t)most, (void *)stream));
}

// cache_release(function, context, device, keep, held, table, free_pages, free_count, stream)
PyObject *cache_release(PyObject *, PyObject *const *args, Py_ssize_t n_args) {
    Callee c;
    uint64_t stream;
    const at::Tensor *keep, *held, *table, *pages, *left;
    if (n_args != 9 || !callee(args, c) || !number(args[8], stream)) Py_RETURN_NONE;
    int64_t n;
    try {
        if (!(keep = dense(args[3], c.device, at::kInt, 0))) Py_RETURN_NONE;
        n = keep->numel();
        if (!(held = dense(args[4], c.device, at::kInt, n)) || !(table = dense(args[5], c.device, at::kInt, 0)) || !(pages = dense(args[6], c.device, at::kInt, 0)) ||
            !(left = dense(args[7], c.device, at::kInt, 1)))
            Py_RETURN_NONE;
        if (table->dim() != 2 || table->size(0) != n || n > 0x7fffffff || table->size(1) > 0x7fffffff || pages->numel() > 0x7fffffff) Py_RETURN_NONE;
    } catch (...) {
        Py_RETURN_NONE;
    }
    SRS_CALL(((decltype(&srs_cache_release))c.fn)((srs_ctx *)c.ctx, (int32_t *)keep->data_ptr(), (uint32_t)n, (int32_t *)held->data_ptr(), (int32_t *)table->data_ptr(),
                                                  (uint32_t)table->size(1), (int32_t *)pages->data_ptr(), (int32_t *)left->data_ptr(), (uint32_t)pages->numel(), (void *)stream));
}

// rope(function, context, device, x, out, positions, inv_freq, flags, magnitude, stream)
PyObject *rope(PyObject *, PyObject *const *args, Py_ssize_t n_args) {
    Callee c;
    uint64_t flags, stream;
    double magnitude;
    if (n_args != 10 || !callee(args, c) || !number(args[7], flags) || !real(args[8], magnitude) || !number(args[9], stream)) Py_RETURN_NONE;
    srs_rows x, out;
    int64_t tokens, d;
    int type;
    const at::Tensor *positions, *freq;
    try {
        const at::Tensor *t = plain(args[3], c.device);
        if (!t || t->dim() != 3 || (type = type_code(t->scalar_type())) < 0) Py_RETURN_NONE;
        tokens = t->size(0); d = t->size(2);
        if (!rows(args[3], c.device, tokens, d, t->scalar_type(), x) || !rows(args[4], c.device, tokens, d, t->scalar_type(), out) || x.heads != out.heads || d > 65536) Py_RETURN_NONE;
        if (!(positions = dense(args[5], c.device, at::kInt, tokens)) || !(freq = dense(args[6], c.device, at::kDouble, 0)) || freq->numel() > 65536) Py_RETURN_NONE;
    } catch (...) {
        Py_RETURN_NONE;
    }
    SRS_CALL(((decltype(&srs_rope))c.fn)((srs_ctx *)c.ctx, type, &x, &out, (uint64_t)tokens, (uint32_t)d, (int32_t *)positions->data_ptr(), (double *)freq->data_ptr(),
                                         (uint32_t)(2 * freq->numel()), (uint32_t)flags, (float)magnitude, (void *)stream));
}

// cache_write(function, context, device, k, v, k_cache, v_cache, slots, q, q_out, positions, inv_freq, flags, magnitude, stream); q, q_out,
// positions and inv_freq may be None
PyObject *cache_write(PyObject *, PyObject *const *args, Py_ssize_t n_args) {
    Callee c;
    uint64_t flags, stream;
    double magnitude;
    if (n_args != 15 || !callee(args, c) || !number(args[12], flags) || !real(args[13], magnitude) || !number(args[14], stream)) Py_RETURN_NONE;
    srs_cache cache;
    srs_rows k, v, q, q_out;
    const at::Tensor *slots, *positions = nullptr, *freq = nullptr;
    const bool queries = args[8] != Py_None;
    int64_t tokens;
    try {
        at::ScalarType type;
        if (!cache_of(args[5], args[6], c.device, cache, type) || !(slots = dense(args[7], c.device, at::kLong, 0))) Py_RETURN_NONE;
        tokens = slots->numel();
        if (!rows(args[3], c.device, tokens, cache.head_dim, type, k) || !rows(args[4], c.device, tokens, cache.head_dim, type, v)) Py_RETURN_NONE;
        if (args[11] != Py_None) {
            if (!(freq = dense(args[11], c.device, at::kDouble, 0)) || freq->numel() > 65536) Py_RETURN_NONE;
            if (freq->numel() && !(positions = dense(args[10], c.device, at::kInt, tokens))) Py_RETURN_NONE;
        }
        if (queries && (!freq || !freq->numel() || !rows(args[8], c.device, tokens, cache.head_dim, type, q) || !rows(args[9], c.device, tokens, cache.head_dim, type, q_out)))
            Py_RETURN_NONE;
    } catch (...) {
        Py_RETURN_NONE;
    }
    SRS_CALL(((decltype(&srs_cache_write))c.fn)((srs_ctx *)c.ctx, &cache, &k, &v, (uint64_t)tokens, (int64_t *)slots->data_ptr(), queries ? &q : nullptr, queries ? &q_out : nullptr,
                                                positions ? (int32_t *)positions->data_ptr() : nullptr, freq ? (double *)freq->data_ptr() : nullptr,
                                                freq ? (uint32_t)(2 * freq->numel()) : 0u, (uint32_t)flags, (float)magnitude, (void *)stream));
}

// cache_attention(function, context, device, workspace function, q, out, k_cache, v_cache, table, token_begin, start, scale, flags, window,
// sinks, lse, most_tokens, most_keys, workspace, stream, whether the stream is the current one); scale, lse and workspace may be None
PyObject *cache_attention(PyObject *, PyObject *const *args, Py_ssize_t n_args) {
    Callee c;
    uint64_t need_fn, flags, window, sinks, most_tokens, most_keys, stream, current;
    double scale;
    if (n_args != 21 || !callee(args, c) || !number(args[3], need_fn) || !number(args[12], flags) || !number(args[13], window) || !number(args[14], sinks) ||
        !number(args[16], most_tokens) || !number(args[17], most_keys) || !number(args[19], stream) || !number(args[20], current) || window > 0x7fffffff || sinks > 0x7fffffff)
        Py_RETURN_NONE;
    srs_cache cache;
    srs_rows q, out;
    const at::Tensor *table, *begin, *start, *lse = nullptr;
    at::Tensor room;
    int64_t tokens, n;
    void *workspace = nullptr;
    uint64_t bytes = 0;
    try {
        at::ScalarType type;
        const at::Tensor *t = plain(args[4], c.device);
        if (!t || t->dim() != 3 || !cache_of(args[6], args[7], c.device, cache, type)) Py_RETURN_NONE;
        tokens = t->size(0);
        if (!rows(args[4], c.device, tokens, cache.head_dim, type, q) || !rows(args[5], c.device, tokens, cache.head_dim, type, out)) Py_RETURN_NONE;
        if (!(start = dense(args[10], c.device, at::kInt, 0))) Py_RETURN_NONE;
        n = start->numel();
        if (!(table = dense(args[8], c.device, at::kInt, 0)) || table->dim() != 2 || table->size(0) != n || table->size(1) > 0x7fffffff || n > 0x7fffffff) Py_RETURN_NONE;
        if (!(begin = dense(args[9], c.device, at::kInt, n + 1))) Py_RETURN_NONE;
        if (args[15] != Py_None && !(lse = dense(args[15], c.device, at::kFloat, tokens * q.heads))) Py_RETURN_NONE;
        if (args[11] == Py_None) scale = 1.0 / std::sqrt((double)cache.head_dim);
        else if (!real(args[11], scale)) Py_RETURN_NONE;
        if (args[18] != Py_None) {
            const at::Tensor *w = plain(args[18], c.device);
            if (!w || !w->is_contiguous()) Py_RETURN_NONE;
            workspace = w->data_ptr(); bytes = (uint64_t)w->numel() * w->element_size();
        } else {
            bytes = ((decltype(&srs_cache_attention_workspace))need_fn)((uint32_t)n, (uint64_t)tokens, q.heads, cache.heads, cache.head_dim, (uint32_t)table->size(1), cache.page_tokens,
                                                                        (uint32_t)window, (uint32_t)sinks, most_tokens, most_keys);
            if (bytes) {
                if (!current) Py_RETURN_NONE;                       // memory of another stream: torch's own way
                room = at::empty({(int64_t)bytes}, at::TensorOptions().dtype(at::kByte).device(at::kCUDA, (c10::DeviceIndex)c.device));
                workspace = room.data_ptr();
            }
        }
    } catch (...) {
        Py_RETURN_NONE;
    }
    SRS_CALL(((decltype(&srs_cache_attention))c.fn)((srs_ctx *)c.ctx, &cache, &q, &out, lse ? (float *)lse->data_ptr() : nullptr, (uint64_t)tokens, (int32_t *)begin->data_ptr(),
                                                    (int32_t *)start->data_ptr(), (int32_t *)table->data_ptr(), (uint32_t)table->size(1), (uint32_t)n, (float)scale,
                                                    (uint32_t)flags, (uint32_t)window, (uint32_t)sinks, most_tokens, most_keys, workspace, bytes, (void *)stream));
}

#define SRS_METHOD(name) {#name, (PyCFunction)(void (*)(void))name, METH_FASTCALL, nullptr}
PyMethodDef methods[] = {{"extract", (PyCFunction)(void (*)(void))extract, METH_FASTCALL, nullptr},
                         {"apply", (PyCFunction)(void (*)(void))apply, METH_FASTCALL, nullptr},
                         SRS_METHOD(cache_tables), SRS_METHOD(cache_release), SRS_METHOD(rope), SRS_METHOD(cache_write), SRS_METHOD(cache_attention),
                         {nullptr, nullptr, 0, nullptr}};
PyModuleDef module = {PyModuleDef_HEAD_INIT, "_call", nullptr, -1, methods, nullptr, nullptr, nullptr, nullptr};

}  // namespace

// The version of the torch whose headers this was built against: srs.py takes the module only where it is the running one's.
PyMODINIT_FUNC PyInit__call(void) {
    PyObject *m = PyModule_Create(&module);
    if (m && PyModule_AddStringConstant(m, "torch_version", SRS_TORCH_VERSION) < 0) { Py_DECREF(m); return nullptr; }
    return m;
}
