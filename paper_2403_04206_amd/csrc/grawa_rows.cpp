// Argument marshalling of the Python binding in native code: the checks that grawa.py makes on the tensors of a call and what it
// passes on, instead of a dozen attribute look-ups a tensor; and whole calls of those that small models make one after the other.
// Such calls were bound by them: LGRAWA of 4 workers, 270 k columns 9.8 -> 8.4 us, without allocation and 8 workers 12.0 -> 10.7; a round of
// four scored steps and the communication, 4 workers, 9 k columns, takes the host 32.4 us with the checks alone and 24.7 with the calls.  Anything that is not
// plainly in order gives None, and grawa.py looks again and raises.
#include <torch/csrc/autograd/python_variable.h>

namespace {

struct Rows {
    void *p;
    int64_t ld;
    int dt; // GRAWA_F32 or GRAWA_BF16
};

// A plain CUDA tensor: subclasses and proxies go by their own Python attributes.  May throw (tensors of torch's transforms do).
const at::Tensor *plain_tensor(PyObject *o)
{
    if (!THPVariable_CheckExact(o)) return nullptr;
    const at::Tensor &t = THPVariable_Unpack(o);
    if (!t.defined() || t.layout() != at::kStrided || !t.is_cuda() || !t.has_storage()) return nullptr;
    if (t.key_set().has(c10::DispatchKey::Python) || t.unsafeGetTensorImpl()->has_symbolic_sizes_strides()) return nullptr;
    return &t;
}

// [K, >= P] with unit column stride whose rows do not overlap and whose storage holds them; float32, or with `grads` bfloat16 too.
bool rows_of(PyObject *o, int64_t K, int64_t P, bool grads, Rows &r)
{
    const at::Tensor *t = plain_tensor(o);
    if (!t || t->dim() != 2) return false;
    const at::ScalarType type = t->scalar_type();
    if (type != at::kFloat && !(grads && type == at::kBFloat16)) return false;
    const int64_t size = type == at::kFloat ? 4 : 2, ld = t->stride(0);
    if (t->stride(1) != 1 || K < 1 || P < 1 || t->size(0) != K || t->size(1) < P || (K > 1 && ld < P)) return false;
    const int64_t have = (int64_t)(t->storage().nbytes() / (size_t)size) - t->storage_offset();
    if (have < P || (K > 1 && ld > (have - P) / (K - 1))) return false; // (K - 1) ld + P elements from the view's start
    r = Rows{t->data_ptr(), ld, type == at::kFloat ? 0 : 1};
    return true;
}

// None, or a float32 vector of at least n elements with unit stride.
bool vector_of(PyObject *o, int64_t n, float *&p)
{
    p = nullptr;
    if (o == Py_None) return true;
    const at::Tensor *t = plain_tensor(o);
    if (!t || t->scalar_type() != at::kFloat || t->dim() != 1 || t->stride(0) != 1 || n < 1 || t->size(0) < n) return false;
    if ((int64_t)(t->storage().nbytes() / 4) - t->storage_offset() < n) return false;
    p = static_cast<float *>(t->data_ptr());
    return true;
}

bool holds(const at::Tensor &t, int64_t elements, int64_t size) // from the view's start on
{
    return (int64_t)(t.storage().nbytes() / (size_t)size) - t.storage_offset() >= elements;
}

// None, or a contiguous float32 tensor [K, L], with L = 0 [K].
bool table_of(PyObject *o, int64_t K, int64_t L, float *&p)
{
    p = nullptr;
    if (o == Py_None) return true;
    const at::Tensor *t = plain_tensor(o);
    if (!t || t->scalar_type() != at::kFloat || !t->is_contiguous() || t->dim() != (L ? 2 : 1) || t->size(0) != K || (L && t->size(1) != L) || !holds(*t, t->numel(), 4))
        return false;
    p = static_cast<float *>(t->data_ptr());
    return true;
}

bool number_of(PyObject *o, float &f) // as ctypes makes a C float of float(o)
{
    if (!PyFloat_CheckExact(o)) return false;
    f = (float)PyFloat_AS_DOUBLE(o);
    return true;
}

bool integer_of(PyObject *o, long long &v)
{
    if (!PyLong_CheckExact(o)) return false;
    v = PyLong_AsLongLong(o);
    if (v == -1 && PyErr_Occurred()) {
        PyErr_Clear();
        return false;
    }
    return true;
}

bool pointer_of(PyObject *o, void *&p)
{
    p = nullptr;
    if (!PyLong_CheckExact(o)) return false;
    p = PyLong_AsVoidPtr(o);
    if (!p && PyErr_Occurred()) {
        PyErr_Clear();
        return false;
    }
    return true;
}

// The handle that `current`, a Python function, gives: asked for last, since it sets torch's CUDA state up.
template <typename Call> PyObject *status_of(PyObject *current, const Call &call)
{
    PyObject *handle = PyObject_CallNoArgs(current);
    if (!handle) return nullptr;
    void *stream;
    const bool ok = pointer_of(handle, stream);
    Py_DECREF(handle);
    if (!ok) Py_RETURN_NONE;
    int status;
    Py_BEGIN_ALLOW_THREADS
    status = call(stream);
    Py_END_ALLOW_THREADS
    return PyLong_FromLong(status);
}

// rows(t, K, P, grads): (data pointer, row stride, dtype code).
PyObject *rows(PyObject *, PyObject *const *args, Py_ssize_t n)
{
    if (n != 4) {
        PyErr_SetString(PyExc_TypeError, "rows(tensor, K, P, grads)");
        return nullptr;
    }
    const long long K = PyLong_AsLongLong(args[1]), P = PyLong_AsLongLong(args[2]);
    const int grads = PyObject_IsTrue(args[3]);
    if (PyErr_Occurred()) return nullptr;
    try { // no C++ exception may leave
        Rows r;
        if (!rows_of(args[0], K, P, grads, r)) Py_RETURN_NONE;
        return Py_BuildValue("KLi", (unsigned long long)reinterpret_cast<uintptr_t>(r.p), (long long)r.ld, r.dt);
    } catch (...) {
        Py_RETURN_NONE;
    }
}

// Whole calls: the status, or None where an argument is not plainly in order.  `function` is the address of the library's function of
// that name, `current` a function that gives the stream's handle; the GIL is released as ctypes does.

// scored(function, plan, x, g, K, P, lr, gamma, center, mu, tau, current): grawa_local_step_scored
PyObject *scored(PyObject *, PyObject *const *args, Py_ssize_t n)
{
    typedef int (*Function)(void *, float *, int64_t, const void *, int64_t, int, float, const float *, float, float, float, void *);
    void *function, *plan;
    long long K, P;
    float lr, gamma, mu, tau, *center;
    Rows x, g;
    try {
        if (n != 12 || !pointer_of(args[0], function) || !pointer_of(args[1], plan) || !integer_of(args[4], K) || !integer_of(args[5], P) ||
            !rows_of(args[2], K, P, false, x) || !rows_of(args[3], K, P, true, g) || !number_of(args[6], lr) || !number_of(args[7], gamma) ||
            !vector_of(args[8], P, center) || !number_of(args[9], mu) || !number_of(args[10], tau))
            Py_RETURN_NONE;
    } catch (...) {
        Py_RETURN_NONE;
    }
    return status_of(args[11], [&](void *stream) {
        return reinterpret_cast<Function>(function)(plan, static_cast<float *>(x.p), x.ld, g.p, g.ld, g.dt, lr, center, mu, tau, gamma, stream);
    });
}

// local(function, plan, x, K, P, L, per_layer, lam, center_out, weights_out, est_out, current): grawa_local_lgrawa_update, grawa_local_mgrawa_update
PyObject *local(PyObject *, PyObject *const *args, Py_ssize_t n)
{
    typedef int (*Function)(void *, float *, int64_t, float, float *, float *, float *, void *);
    void *function, *plan;
    long long K, P, L, per_layer;
    float lam, *center, *weights, *est;
    Rows x;
    try {
        if (n != 12 || !pointer_of(args[0], function) || !pointer_of(args[1], plan) || !integer_of(args[3], K) || !integer_of(args[4], P) ||
            !integer_of(args[5], L) || !integer_of(args[6], per_layer) || L < 1 || !rows_of(args[2], K, P, false, x) || !number_of(args[7], lam) ||
            !vector_of(args[8], P, center) || !table_of(args[9], K, per_layer ? L : 0, weights) || !table_of(args[10], K, L, est))
            Py_RETURN_NONE;
    } catch (...) {
        Py_RETURN_NONE;
    }
    return status_of(args[11], [&](void *stream) {
        return reinterpret_cast<Function>(function)(plan, static_cast<float *>(x.p), x.ld, lam, center, weights, est, stream);
    });
}

// lgrawa(function, plan, x, g, K, P, L, lam, center_out, weights_out, current): grawa_lgrawa_update
PyObject *lgrawa(PyObject *, PyObject *const *args, Py_ssize_t n)
{
    typedef int (*Function)(void *, float *, int64_t, const void *, int64_t, int, float, float *, float *, void *);
    void *function, *plan;
    long long K, P, L;
    float lam, *center, *weights;
    Rows x, g;
    try {
        if (n != 11 || !pointer_of(args[0], function) || !pointer_of(args[1], plan) || !integer_of(args[4], K) || !integer_of(args[5], P) ||
            !integer_of(args[6], L) || L < 1 || !rows_of(args[2], K, P, false, x) || !rows_of(args[3], K, P, true, g) || !number_of(args[7], lam) ||
            !vector_of(args[8], P, center) || !table_of(args[9], K, L, weights))
            Py_RETURN_NONE;
    } catch (...) {
        Py_RETURN_NONE;
    }
    return status_of(args[10], [&](void *stream) {
        return reinterpret_cast<Function>(function)(plan, static_cast<float *>(x.p), x.ld, g.p, g.ld, g.dt, lam, center, weights, stream);
    });
}

// The feed-forward sublayer's calls, whose small forms take the card 3 us: a dropout by Python's checks 8.5 us, by these 3.6.

struct RowsArg { // grawa_rows_t
    void *data;
    int64_t worker, row;
};

struct MatsArg { // grawa_mats_t
    void *data;
    int64_t worker;
};

at::ScalarType type_of(long long dt) { return dt ? at::kBFloat16 : at::kFloat; }

// [K, T, d] with unit stride in the last axis.  The strides of what passes fit the storage, so no product overflows.
bool tokens_of(PyObject *o, int64_t K, int64_t T, int64_t d, long long dt, RowsArg &r)
{
    const at::Tensor *t = plain_tensor(o);
    if (!t || t->dim() != 3 || t->scalar_type() != type_of(dt) || t->size(0) != K || t->size(1) != T || t->size(2) != d) return false;
    const int64_t worker = K > 1 ? t->stride(0) : 0, row = T > 1 ? t->stride(1) : d, size = dt ? 2 : 4;
    if ((d > 1 && t->stride(2) != 1) || worker < 0 || row < 0 || T < 1) return false;
    const __int128 need = (__int128)(K - 1) * worker + (__int128)(T - 1) * row + d;
    if (need > (__int128)1 << 60 || !holds(*t, (int64_t)need, size)) return false;
    r = RowsArg{t->data_ptr(), worker, row};
    return true;
}

// [K, n] or [K, n1, n2], each worker's elements without gaps.
bool mats_of(PyObject *o, int64_t K, int64_t n1, int64_t n2, long long dt, MatsArg &m)
{
    const at::Tensor *t = plain_tensor(o);
    const int dims = n2 ? 3 : 2;
    if (!t || t->dim() != dims || t->scalar_type() != type_of(dt) || t->size(0) != K || t->size(1) != n1 || (n2 && t->size(2) != n2)) return false;
    if (n2 ? (n2 > 1 && t->stride(2) != 1) || (n1 > 1 && t->stride(1) != n2) : n1 > 1 && t->stride(1) != 1) return false;
    const int64_t worker = K > 1 ? t->stride(0) : 0, n = n2 ? n1 * n2 : n1;
    const __int128 need = (__int128)(K - 1) * worker + n;
    if (worker < 0 || need > (__int128)1 << 60 || !holds(*t, (int64_t)need, dt ? 2 : 4)) return false;
    m = MatsArg{t->data_ptr(), worker};
    return true;
}

// None, or a contiguous float32 tensor [K, T, 2].
bool stats_of(PyObject *o, int64_t K, int64_t T, float *&p)
{
    p = nullptr;
    if (o == Py_None) return true;
    const at::Tensor *t = plain_tensor(o);
    if (!t || t->scalar_type() != at::kFloat || !t->is_contiguous() || t->dim() != 3 || t->size(0) != K || t->size(1) != T || t->size(2) != 2 || !holds(*t, t->numel(), 4))
        return false;
    p = static_cast<float *>(t->data_ptr());
    return true;
}

// A contiguous int64 tensor of two or more; None where nothing is dropped.
bool rng_of(PyObject *o, float p, int64_t *&rng)
{
    rng = nullptr;
    if (o == Py_None) return p == 0.f;
    const at::Tensor *t = plain_tensor(o);
    if (!t || t->scalar_type() != at::kLong || t->dim() != 1 || t->size(0) < 2 || t->stride(0) != 1 || !holds(*t, 2, 8)) return false;
    rng = static_cast<int64_t *>(t->data_ptr());
    return true;
}

bool site_of(PyObject *o, uint32_t &site)
{
    long long v;
    if (!integer_of(o, v) || v < 0 || v >> 32) return false;
    site = (uint32_t)v;
    return true;
}

// The plan's K, T, d and dtype code from four numbers, and the tokens of `x`, at most the plan's.
bool plan_of(PyObject *const *args, long long &K, long long &T, long long &d, long long &dt, PyObject *x)
{
    long long most;
    if (!integer_of(args[0], K) || !integer_of(args[1], most) || !integer_of(args[2], d) || !integer_of(args[3], dt)) return false;
    const at::Tensor *t = plain_tensor(x);
    if (!t || t->dim() != 3 || t->size(1) > most) return false;
    T = t->size(1);
    return true;
}

// norm(function, plan, K, T, d, dtype, x, weight, bias, out, eps, stats, current): grawa_layer_norm
PyObject *norm(PyObject *, PyObject *const *args, Py_ssize_t n)
{
    typedef int (*Function)(void *, int64_t, const RowsArg *, const MatsArg *, const MatsArg *, float, const RowsArg *, float *, void *);
    void *function, *plan;
    long long K, T, d, dt;
    float eps, *stats;
    RowsArg x, out;
    MatsArg weight, bias{};
    try {
        if (n != 13 || !pointer_of(args[0], function) || !pointer_of(args[1], plan) || !plan_of(args + 2, K, T, d, dt, args[6]) ||
            !tokens_of(args[6], K, T, d, dt, x) || !mats_of(args[7], K, d, 0, dt, weight) || (args[8] != Py_None && !mats_of(args[8], K, d, 0, dt, bias)) ||
            !tokens_of(args[9], K, T, d, dt, out) || !number_of(args[10], eps) || !stats_of(args[11], K, T, stats))
            Py_RETURN_NONE;
    } catch (...) {
        Py_RETURN_NONE;
    }
    return status_of(args[12], [&](void *stream) { return reinterpret_cast<Function>(function)(plan, T, &x, &weight, args[8] == Py_None ? nullptr : &bias, eps, &out, stats, stream); });
}

// norm_back(function, plan, K, T, d, dtype, dy, x, weight, stats, dx, dweight, dbias, add, accumulate, current): grawa_layer_norm_backward
PyObject *norm_back(PyObject *, PyObject *const *args, Py_ssize_t n)
{
    typedef int (*Function)(void *, int64_t, const RowsArg *, const RowsArg *, const MatsArg *, const float *, const RowsArg *, const RowsArg *, const MatsArg *, const MatsArg *, int, void *);
    void *function, *plan;
    long long K, T, d, dt;
    float *stats;
    RowsArg dy, x, dx, add{};
    MatsArg weight, dweight, dbias{};
    try {
        if (n != 16 || !pointer_of(args[0], function) || !pointer_of(args[1], plan) || !plan_of(args + 2, K, T, d, dt, args[6]) ||
            !tokens_of(args[6], K, T, d, dt, dy) || !tokens_of(args[7], K, T, d, dt, x) || !mats_of(args[8], K, d, 0, dt, weight) ||
            args[9] == Py_None || !stats_of(args[9], K, T, stats) || !tokens_of(args[10], K, T, d, dt, dx) || !mats_of(args[11], K, d, 0, dt, dweight) ||
            (args[12] != Py_None && !mats_of(args[12], K, d, 0, dt, dbias)) || (args[13] != Py_None && !tokens_of(args[13], K, T, d, dt, add)) || !PyBool_Check(args[14]))
            Py_RETURN_NONE;
    } catch (...) {
        Py_RETURN_NONE;
    }
    return status_of(args[15], [&](void *stream) {
        return reinterpret_cast<Function>(function)(plan, T, &dy, &x, &weight, stats, args[13] == Py_None ? nullptr : &add, &dx, &dweight, args[12] == Py_None ? nullptr : &dbias,
                                                    args[14] == Py_True, stream);
    });
}

// None where it may be, or a contiguous uint8 tensor of at least what `size`, grawa_sublayer_save_bytes, says.
bool save_of(PyObject *o, void *size, void *plan, int64_t T, bool optional, void *&p)
{
    p = nullptr;
    if (o == Py_None) return optional;
    const at::Tensor *t = plain_tensor(o);
    int64_t need = 0;
    if (!t || t->scalar_type() != at::kByte || t->dim() != 1 || !t->is_contiguous() || reinterpret_cast<int (*)(const void *, int64_t, int64_t *)>(size)(plan, T, &need) != 0)
        return false;
    if (t->size(0) < need || !holds(*t, need, 1)) return false;
    p = t->data_ptr();
    return true;
}

// feed(function, size, plan, K, T, d, dtype, f, x, wg, wu, wd, out, save, residual, p, rng, site, current): grawa_ffn
PyObject *feed(PyObject *, PyObject *const *args, Py_ssize_t n)
{
    typedef int (*Function)(void *, int64_t, const RowsArg *, const MatsArg *, const MatsArg *, const MatsArg *, const RowsArg *, float, const int64_t *, uint32_t, const RowsArg *, void *, void *);
    void *function, *size, *plan, *save;
    long long K, T, d, dt, f;
    float p;
    int64_t *rng;
    uint32_t site;
    RowsArg x, out, residual{};
    MatsArg wg, wu, wd;
    try {
        if (n != 19 || !pointer_of(args[0], function) || !pointer_of(args[1], size) || !pointer_of(args[2], plan) || !plan_of(args + 3, K, T, d, dt, args[8]) ||
            !integer_of(args[7], f) || f < 1 || !tokens_of(args[8], K, T, d, dt, x) || !mats_of(args[9], K, f, d, dt, wg) || !mats_of(args[10], K, f, d, dt, wu) ||
            !mats_of(args[11], K, d, f, dt, wd) || !tokens_of(args[12], K, T, d, dt, out) || !save_of(args[13], size, plan, T, true, save) ||
            (args[14] != Py_None && !tokens_of(args[14], K, T, d, dt, residual)) || !number_of(args[15], p) || !rng_of(args[16], p, rng) || !site_of(args[17], site))
            Py_RETURN_NONE;
    } catch (...) {
        Py_RETURN_NONE;
    }
    return status_of(args[18], [&](void *stream) {
        return reinterpret_cast<Function>(function)(plan, T, &x, &wg, &wu, &wd, args[14] == Py_None ? nullptr : &residual, p, rng, site, &out, save, stream);
    });
}

// feed_back(function, size, plan, K, T, d, dtype, f, dy, x, wg, wu, wd, save, dx, dwg, dwu, dwd, accumulate, current): grawa_ffn_backward
PyObject *feed_back(PyObject *, PyObject *const *args, Py_ssize_t n)
{
    typedef int (*Function)(void *, int64_t, const RowsArg *, const RowsArg *, const MatsArg *, const MatsArg *, const MatsArg *, const void *, const RowsArg *, const MatsArg *, const MatsArg *,
                            const MatsArg *, int, void *);
    void *function, *size, *plan, *save;
    long long K, T, d, dt, f;
    RowsArg dy, x, dx;
    MatsArg m[6];
    try {
        if (n != 20 || !pointer_of(args[0], function) || !pointer_of(args[1], size) || !pointer_of(args[2], plan) || !plan_of(args + 3, K, T, d, dt, args[8]) ||
            !integer_of(args[7], f) || f < 1 || !tokens_of(args[8], K, T, d, dt, dy) || !tokens_of(args[9], K, T, d, dt, x) ||
            !save_of(args[13], size, plan, T, false, save) || !tokens_of(args[14], K, T, d, dt, dx) || !PyBool_Check(args[18]))
            Py_RETURN_NONE;
        for (int i = 0; i < 6; ++i) {
            const bool down = i % 3 == 2;
            if (!mats_of(args[i < 3 ? 10 + i : 12 + i], K, down ? d : f, down ? f : d, dt, m[i])) Py_RETURN_NONE;
        }
    } catch (...) {
        Py_RETURN_NONE;
    }
    return status_of(args[19], [&](void *stream) {
        return reinterpret_cast<Function>(function)(plan, T, &dy, &x, &m[0], &m[1], &m[2], save, &dx, &m[3], &m[4], &m[5], args[18] == Py_True, stream);
    });
}

// drop(function, x, out, p, rng, site, residual, current): grawa_dropout
PyObject *drop(PyObject *, PyObject *const *args, Py_ssize_t n)
{
    typedef int (*Function)(int, int64_t, int64_t, int, const RowsArg *, const RowsArg *, float, const int64_t *, uint32_t, const RowsArg *, void *);
    void *function;
    int64_t K, T, d;
    long long dt;
    float p;
    int64_t *rng;
    uint32_t site;
    RowsArg x, out, residual{};
    try {
        const at::Tensor *t = n == 8 ? plain_tensor(args[1]) : nullptr;
        if (!t || t->dim() != 3 || (t->scalar_type() != at::kFloat && t->scalar_type() != at::kBFloat16)) Py_RETURN_NONE;
        K = t->size(0), T = t->size(1), d = t->size(2), dt = t->scalar_type() == at::kBFloat16;
        if (K < 1 || K > 1 << 20 || d < 1 || !pointer_of(args[0], function) || !tokens_of(args[1], K, T, d, dt, x) || !tokens_of(args[2], K, T, d, dt, out) ||
            !number_of(args[3], p) || !rng_of(args[4], p, rng) || !site_of(args[5], site) || (args[6] != Py_None && !tokens_of(args[6], K, T, d, dt, residual)))
            Py_RETURN_NONE;
    } catch (...) {
        Py_RETURN_NONE;
    }
    return status_of(args[7], [&](void *stream) {
        return reinterpret_cast<Function>(function)((int)K, T, d, (int)dt, &x, args[6] == Py_None ? nullptr : &residual, p, rng, site, &out, stream);
    });
}

#define GRAWA_METHOD(f) {#f, reinterpret_cast<PyCFunction>(reinterpret_cast<void *>(f)), METH_FASTCALL, nullptr}
PyMethodDef methods[] = {GRAWA_METHOD(rows), GRAWA_METHOD(scored), GRAWA_METHOD(local), GRAWA_METHOD(lgrawa), GRAWA_METHOD(norm), GRAWA_METHOD(norm_back),
                         GRAWA_METHOD(feed), GRAWA_METHOD(feed_back), GRAWA_METHOD(drop), {nullptr, nullptr, 0, nullptr}};
PyModuleDef module = {PyModuleDef_HEAD_INIT, "_rows", nullptr, -1, methods, nullptr, nullptr, nullptr, nullptr};

} // namespace

// The functions above read torch's objects through the headers this file was compiled with, so the module names the torch
// and the Python that it is for, and grawa.py uses it with no other.
PyMODINIT_FUNC PyInit__rows()
{
    PyObject *m = PyModule_Create(&module);
    if (m && PyModule_AddStringConstant(m, "built_for", GRAWA_ROWS_BUILT_FOR) != 0) {
        Py_DECREF(m);
        return nullptr;
    }
    return m;
}
