// The sampling calls as Python functions (module _nd_call): they check tensors, collect their addresses and call the
// library.  A walk of 100 steps hands over 100 output arrays; checked and collected tensor by tensor through Python
// attributes and ctypes they cost the host 35 us for a sampling and a gathering call, more than the GPU works on 4,096
// walks, and a k-hop call 4 us.  The calls on rows of features are here for the same reason: a call that moves 64 rows
// took 15 us of the host and takes 5.  The library's entry points come as addresses (init), so the module is
// independent of which library binding.py has loaded.
#define PY_SSIZE_T_CLEAN
#include <Python.h>

#include <ATen/ops/empty.h>
#include <torch/csrc/autograd/python_variable.h>

#include <cstdint>
#include <cstring>
#include <exception>
#include <vector>

#include "../../include/nd.h"

namespace {

using SampleFn = int (*)(const void*, int, const void*, const int32_t*, int64_t, uint64_t, int32_t* const*, void*, size_t,
                         void*);
using StaticFn = int (*)(const void*, int, const void*, const int32_t*, int64_t, uint64_t, int32_t* const*, uint32_t*,
                         void*);
using PackFn = int (*)(const int32_t* const*, int32_t, const int64_t*, int64_t, int32_t*, void*);
SampleFn g_sample = nullptr;
StaticFn g_static = nullptr;
PackFn g_pack = nullptr;

// An address or handle given as an integer, None for null.
bool as_address(PyObject* o, void** out) {
    *out = nullptr;
    if (o == Py_None) return true;
    *out = PyLong_AsVoidPtr(o);
    return !(*out == nullptr && PyErr_Occurred());
}

const at::Tensor* as_tensor(PyObject* o, const char* what) {
    if (!THPVariable_Check(o)) {
        PyErr_SetString(PyExc_TypeError, what);
        return nullptr;
    }
    return &THPVariable_Unpack(o);
}

bool is_array(const at::Tensor& t) {
    return t.scalar_type() == at::kInt && t.is_cuda() && t.is_contiguous();
}

// Memory that a kernel reaches at the tensor's address: the GPU's, or pinned on the host.
bool is_reachable(const at::Tensor& t) { return t.is_cuda() || t.is_pinned(); }

// The tensors of a sequence: contiguous int32 arrays on a GPU.
struct Arrays {
    std::vector<int32_t*> ptr;
    std::vector<int64_t> len;
    bool take(PyObject* seq, const char* complaint, int64_t at_least = 0) {
        PyObject* fast = PySequence_Fast(seq, complaint);
        if (!fast) return false;
        const Py_ssize_t n = PySequence_Fast_GET_SIZE(fast);
        if (n < at_least) {
            PyErr_Format(PyExc_ValueError, "%zd arrays for %lld steps", n, (long long)at_least);
            Py_DECREF(fast);
            return false;
        }
        ptr.reserve((size_t)n);
        len.reserve((size_t)n);
        bool ok = true;
        for (Py_ssize_t i = 0; ok && i < n; ++i) {
            const at::Tensor* t = as_tensor(PySequence_Fast_GET_ITEM(fast, i), complaint);
            ok = t != nullptr;
            if (ok && !is_array(*t)) {
                PyErr_SetString(PyExc_TypeError, complaint);
                ok = false;
            }
            if (ok) {
                ptr.push_back((int32_t*)t->data_ptr());
                len.push_back(t->numel());
            }
        }
        Py_DECREF(fast);
        return ok;
    }
};

constexpr const char* kRoots = "roots must be a contiguous int32 CUDA tensor";
constexpr const char* kOutputs = "outputs must be contiguous int32 CUDA tensors";
constexpr const char* kSteps = "step arrays must be contiguous int32 CUDA tensors";

// What both sampling calls take: handle, app, params, roots, seed, outputs.
struct Call {
    void* handle = nullptr;
    int app = 0;
    Py_buffer params{};
    const int32_t* roots = nullptr;
    int64_t num_roots = 0;
    uint64_t seed = 0;
    Arrays out;
    ~Call() {
        if (params.obj) PyBuffer_Release(&params);
    }
    bool take(PyObject* const* a) {
        if (!as_address(a[0], &handle)) return false;
        app = (int)PyLong_AsUnsignedLongMask(a[1]);  // what has __index__ counts as an integer, NumPy's integers too
        if (PyErr_Occurred()) return false;
        seed = PyLong_AsUnsignedLongLongMask(a[4]);
        if (PyErr_Occurred()) return false;
        if (PyObject_GetBuffer(a[2], &params, PyBUF_SIMPLE) != 0) return false;  // the ctypes structure itself
        if (params.len != (Py_ssize_t)sizeof(nd_params)) {
            PyErr_SetString(PyExc_TypeError, "params must be an nd_params");
            return false;
        }
        const at::Tensor* r = as_tensor(a[3], kRoots);
        if (!r) return false;
        if (!is_array(*r)) {
            PyErr_SetString(PyExc_TypeError, kRoots);
            return false;
        }
        num_roots = r->numel();
        // the library reads an address per step and has no count of them
        nd_params p;
        std::memcpy(&p, params.buf, sizeof p);
        const int64_t steps = p.num_steps <= ND_MAX_WALK_STEPS ? p.num_steps : 0;  // more than that it refuses
        if (!out.take(a[5], kOutputs, num_roots > 0 ? steps : 0)) return false;
        if ((int64_t)out.ptr.size() < steps) out.ptr.resize((size_t)steps, nullptr);
        roots = (const int32_t*)r->data_ptr();
        return true;
    }
};

bool expects(Py_ssize_t got, Py_ssize_t want) {
    if (got == want) return true;
    PyErr_Format(PyExc_TypeError, "%zd arguments, expected %zd", got, want);
    return false;
}

PyObject* init(PyObject*, PyObject* const* a, Py_ssize_t n) {
    void *s, *t, *p;
    if (!expects(n, 4) || !as_address(a[0], &s) || !as_address(a[1], &t) || !as_address(a[2], &p)) return nullptr;
    const Py_ssize_t params_size = PyLong_AsSsize_t(a[3]);
    if (params_size < 0 && PyErr_Occurred()) return nullptr;
    if (params_size != (Py_ssize_t)sizeof(nd_params)) {
        PyErr_Format(PyExc_TypeError, "nd_params of %zd bytes, expected %zu", params_size, sizeof(nd_params));
        return nullptr;
    }
    g_sample = (SampleFn)s;
    g_static = (StaticFn)t;
    g_pack = (PackFn)p;
    Py_RETURN_NONE;
}

// sample(handle, app, params, roots, seed, outputs, workspace, stream) -> code
PyObject* sample(PyObject*, PyObject* const* a, Py_ssize_t n) try {
    Call c;
    void* stream;
    if (!expects(n, 8) || !c.take(a) || !as_address(a[7], &stream)) return nullptr;
    constexpr const char* kWorkspace = "workspace must be a CUDA tensor without gaps";
    const at::Tensor* w = as_tensor(a[6], kWorkspace);
    if (!w) return nullptr;
    if (!is_reachable(*w) || !w->is_non_overlapping_and_dense()) {
        PyErr_SetString(PyExc_TypeError, kWorkspace);
        return nullptr;
    }
    void* ws = w->data_ptr();
    const size_t bytes = (size_t)w->numel() * (size_t)w->element_size();
    int rc;
    Py_BEGIN_ALLOW_THREADS
    rc = g_sample(c.handle, c.app, c.params.buf, c.roots, c.num_roots, c.seed, c.out.ptr.data(), ws, bytes, stream);
    Py_END_ALLOW_THREADS
    return PyLong_FromLong(rc);
} catch (const std::exception& e) {
    PyErr_SetString(PyExc_RuntimeError, e.what());
    return nullptr;
}

// sample_static(handle, app, params, roots, seed, outputs, status or None, stream) -> code
PyObject* sample_static(PyObject*, PyObject* const* a, Py_ssize_t n) try {
    Call c;
    void* stream;
    if (!expects(n, 8) || !c.take(a) || !as_address(a[7], &stream)) return nullptr;
    uint32_t* status = nullptr;
    if (a[6] != Py_None) {
        constexpr const char* kStatus = "status must be a CUDA tensor of one 32-bit element";
        const at::Tensor* s = as_tensor(a[6], kStatus);
        if (!s) return nullptr;
        const bool holds = s->numel() > 0 && (size_t)s->numel() * (size_t)s->element_size() >= sizeof(uint32_t);
        if (!holds || !is_reachable(*s) || !s->is_non_overlapping_and_dense()) {
            PyErr_SetString(PyExc_TypeError, kStatus);
            return nullptr;
        }
        status = (uint32_t*)s->data_ptr();
    }
    int rc;
    Py_BEGIN_ALLOW_THREADS
    rc = g_static(c.handle, c.app, c.params.buf, c.roots, c.num_roots, c.seed, c.out.ptr.data(), status, stream);
    Py_END_ALLOW_THREADS
    return PyLong_FromLong(rc);
} catch (const std::exception& e) {
    PyErr_SetString(PyExc_RuntimeError, e.what());
    return nullptr;
}

// Entries of one record.
int64_t record_of(const Arrays& steps, int64_t num_samples) {
    int64_t length = 0;
    if (num_samples > 0)
        for (int64_t len : steps.len) length += len / num_samples;
    return length;
}

// pack(step arrays, samples, records, stream) -> code
PyObject* pack(PyObject*, PyObject* const* a, Py_ssize_t n) try {
    Arrays steps;
    void* stream;
    if (!expects(n, 4) || !steps.take(a[0], kSteps)) return nullptr;
    const int64_t num_samples = PyLong_AsLongLong(a[1]);
    if (PyErr_Occurred()) return nullptr;
    constexpr const char* kRecords = "samples must be a contiguous int32 CUDA tensor of num_samples * record entries";
    const at::Tensor* r = as_tensor(a[2], kRecords);
    if (!r || !as_address(a[3], &stream)) return nullptr;
    if (r->scalar_type() != at::kInt || r->numel() < num_samples * record_of(steps, num_samples) || !r->is_contiguous() ||
        (r->numel() > 0 && !is_reachable(*r))) {
        PyErr_SetString(PyExc_TypeError, kRecords);
        return nullptr;
    }
    int32_t* records = r->numel() > 0 ? (int32_t*)r->data_ptr() : nullptr;
    int rc;
    Py_BEGIN_ALLOW_THREADS
    rc = g_pack(steps.ptr.data(), (int32_t)steps.ptr.size(), steps.len.data(), num_samples, records, stream);
    Py_END_ALLOW_THREADS
    return PyLong_FromLong(rc);
} catch (const std::exception& e) {
    PyErr_SetString(PyExc_RuntimeError, e.what());
    return nullptr;
}

// record_length(step arrays, samples): entries of one record, after the same check of the arrays
PyObject* record_length(PyObject*, PyObject* const* a, Py_ssize_t n) try {
    Arrays steps;
    if (!expects(n, 2) || !steps.take(a[0], kSteps)) return nullptr;
    const int64_t num_samples = PyLong_AsLongLong(a[1]);
    if (PyErr_Occurred()) return nullptr;
    return PyLong_FromLongLong(record_of(steps, num_samples));
} catch (const std::exception& e) {
    PyErr_SetString(PyExc_RuntimeError, e.what());
    return nullptr;
}

// ------------------------------------------------------------------------------------------------- rows of features
using LossFn = int (*)(const void*, int64_t, const void*, int64_t, int, int64_t, int64_t, int32_t, const int32_t*, int32_t, float*,
                       float*, void*, size_t, void*);
using GradFn = int (*)(const void*, int64_t, const void*, int64_t, int, int64_t, int64_t, int32_t, const int32_t*, int32_t,
                       const float*, float*, float*, void*, int64_t, void*, int64_t, void*, size_t, void*);
using PositionsFn = int (*)(const int32_t*, int64_t, const int64_t*, int64_t, int32_t*, void*);
using ByTransitFn = int (*)(const void*, int64_t, int, int64_t, int32_t, const int32_t*, int64_t, const int64_t*, int32_t,
                            const float*, void*, int64_t, void*);
using ToSamplesFn = int (*)(const void*, int64_t, int, int64_t, int32_t, const int32_t*, int64_t, int32_t, const float*, void*,
                            int64_t, void*);
using WeightGradFn = int (*)(const void*, int64_t, const void*, int64_t, int, int64_t, int32_t, const int32_t*, int64_t, int32_t,
                             float*, void*);
using SumBytesFn = size_t (*)(int64_t, int32_t);
using GroupSumFn = int (*)(const void*, int64_t, int, int64_t, int32_t, const int32_t*, int64_t, const int32_t*, int64_t,
                           const int64_t*, int32_t, const float*, const int32_t*, void*, int64_t, int64_t, void*, size_t, void*);
struct {
    LossFn loss;
    GradFn grad;
    PositionsFn positions;
    ByTransitFn by_transit;
    ToSamplesFn to_samples;
    WeightGradFn weight_grad;
    SumBytesFn sum_bytes;
    GroupSumFn group_sum;
} g_rows{};

// init_rows(addresses in that order)
PyObject* init_rows(PyObject*, PyObject* const* a, Py_ssize_t n) {
    void* f[8];
    if (!expects(n, 8)) return nullptr;
    for (int i = 0; i < 8; ++i)
        if (!as_address(a[i], &f[i])) return nullptr;
    g_rows = {(LossFn)f[0], (GradFn)f[1], (PositionsFn)f[2], (ByTransitFn)f[3], (ToSamplesFn)f[4], (WeightGradFn)f[5],
              (SumBytesFn)f[6], (GroupSumFn)f[7]};
    Py_RETURN_NONE;
}

int type_of(at::ScalarType t) { return t == at::kFloat ? ND_F32 : t == at::kBFloat16 ? ND_BF16 : t == at::kHalf ? ND_F16 : -1; }

// The current device and the stream of a call.
struct Place {
    int64_t device = 0;
    void* stream = nullptr;
    bool take(PyObject* dev, PyObject* str) {
        device = PyLong_AsLongLong(dev);
        return !PyErr_Occurred() && as_address(str, &stream);
    }
    bool holds(const at::Tensor& t, const char* what) const {
        if (t.get_device() == device) return true;
        PyErr_Format(PyExc_ValueError, "%s lies on device %lld but device %lld is current", what, (long long)t.get_device(),
                     (long long)device);
        return false;
    }
};

// Rows of d numbers next to each other; what is expected of them: -1, anything.
struct Rows {
    void* ptr = nullptr;
    int64_t stride = 0, n = 0;
    int32_t d = 0;
    int type = -1;
    const at::Tensor* tensor = nullptr;
    bool take(PyObject* o, const char* what, const Place& place, int want_type = -1, int64_t want_d = -1, int64_t want_n = -1) {
        if (!THPVariable_Check(o) || !(tensor = &THPVariable_Unpack(o))->is_cuda() || tensor->dim() != 2 ||
            (type = type_of(tensor->scalar_type())) < 0) {
            PyErr_Format(PyExc_TypeError, "%s must be a 2-D CUDA tensor of float32, bfloat16 or float16", what);
            return false;
        }
        if (!place.holds(*tensor, what)) return false;
        const int64_t cols = tensor->size(1);
        n = tensor->size(0);
        if ((want_type >= 0 && type != want_type) || (want_d >= 0 && cols != want_d) || (want_n >= 0 && n != want_n)) {
            PyErr_Format(PyExc_ValueError, "%s is %lld x %lld, expected %lld x %lld of the type of the other rows", what,
                         (long long)n, (long long)cols, (long long)(want_n < 0 ? n : want_n),
                         (long long)(want_d < 0 ? cols : want_d));
            return false;
        }
        if (cols > 1 && tensor->stride(1) != 1) {
            PyErr_Format(PyExc_ValueError, "%s: the numbers of a row must lie next to each other", what);
            return false;
        }
        if (n > 1 && tensor->stride(0) < cols) {
            PyErr_Format(PyExc_ValueError, "%s: rows must not overlap", what);
            return false;
        }
        if (cols > ND_MAX_ROW) {  // what the library refuses, before it is cut to 32 bits
            d = ND_MAX_ROW + 1;
        } else {
            d = (int32_t)cols;
        }
        stride = n > 1 ? tensor->stride(0) : d;
        ptr = tensor->data_ptr();
        return true;
    }
};

// A contiguous array with at least so many entries; None where it may be left out.
struct Flat {
    void* ptr = nullptr;
    int64_t n = 0;
    const at::Tensor* tensor = nullptr;
    bool take(PyObject* o, const char* what, const Place& place, at::ScalarType type, int64_t entries, bool or_none = false) {
        if (or_none && o == Py_None) return true;
        if (!THPVariable_Check(o) || !(tensor = &THPVariable_Unpack(o))->is_cuda() || !tensor->is_contiguous() ||
            (type != at::ScalarType::Undefined && tensor->scalar_type() != type)) {
            if (type == at::ScalarType::Undefined)
                PyErr_Format(PyExc_TypeError, "%s must be a contiguous CUDA tensor", what);
            else
                PyErr_Format(PyExc_TypeError, "%s must be a contiguous CUDA tensor of %s", what, c10::toString(type));
            return false;
        }
        if (!place.holds(*tensor, what)) return false;
        n = tensor->numel();
        if (n < entries) {
            PyErr_Format(PyExc_ValueError, "%s has %lld entries, %lld are needed", what, (long long)n, (long long)entries);
            return false;
        }
        ptr = tensor->data_ptr();
        return true;
    }
    size_t bytes() const { return (size_t)n * (size_t)tensor->element_size(); }
};

// Slots of a row; slots that no call takes are refused by the library.
bool as_slots(PyObject* o, int32_t* m) {
    const int64_t v = PyLong_AsLongLong(o);
    if (PyErr_Occurred()) return false;
    *m = v < 0 ? 0 : v > ND_MAX_ROW_SLOTS ? ND_MAX_ROW_SLOTS + 1 : (int32_t)v;
    return true;
}
int64_t product_of(int64_t n, int32_t m) { return m > 0 && n <= INT64_MAX / m ? n * m : 0; }

// What a call made: the tensor, or the library's code.
PyObject* made(int rc, PyObject* given, at::Tensor& created) {
    if (rc != ND_OK) return PyLong_FromLong(rc);
    if (given != Py_None) {
        Py_INCREF(given);
        return given;
    }
    return THPVariable_Wrap(created);
}

// The interpreter's lock is free while the library works.
template <typename F, typename... A>
int without_lock(F f, A... args) {
    int rc;
    Py_BEGIN_ALLOW_THREADS
    rc = f(args...);
    Py_END_ALLOW_THREADS
    return rc;
}

#define ND_CATCH                                     \
    catch (const std::exception& e) {                \
        PyErr_SetString(PyExc_RuntimeError, e.what()); \
        return nullptr;                              \
    }

// positions(sorted_slots, n_slots, counts, out or None, device, stream)
PyObject* positions(PyObject*, PyObject* const* a, Py_ssize_t n) try {
    Place place;
    Flat slots, counts, out;
    if (!expects(n, 6) || !place.take(a[4], a[5]) || !slots.take(a[0], "sorted_slots", place, at::kInt, 0)) return nullptr;
    const int64_t n_slots = PyLong_AsLongLong(a[1]);
    if (PyErr_Occurred() || !counts.take(a[2], "counts", place, at::kLong, 2, true)) return nullptr;
    at::Tensor made_here;
    if (a[3] == Py_None) {
        made_here = at::empty({n_slots > 0 ? n_slots : 0}, slots.tensor->options());
        out.ptr = made_here.data_ptr();
    } else if (!out.take(a[3], "out", place, at::kInt, n_slots)) {
        return nullptr;
    }
    const int rc = without_lock(g_rows.positions, (const int32_t*)slots.ptr, slots.n, (const int64_t*)counts.ptr, n_slots,
                                (int32_t*)out.ptr, place.stream);
    return made(rc, a[3], made_here);
}
ND_CATCH

// by_transit(x, sorted_slots, m, weights, counts, out or None, device, stream)
PyObject* by_transit(PyObject*, PyObject* const* a, Py_ssize_t n) try {
    Place place;
    Rows x, out;
    Flat slots, weights, counts;
    int32_t m;
    if (!expects(n, 8) || !place.take(a[6], a[7]) || !x.take(a[0], "x", place) || !as_slots(a[2], &m) ||
        !slots.take(a[1], "sorted_slots", place, at::kInt, 0) ||
        !weights.take(a[3], "weights", place, at::kFloat, product_of(x.n, m), true) ||
        !counts.take(a[4], "counts", place, at::kLong, 2, true))
        return nullptr;
    at::Tensor made_here;
    if (a[5] == Py_None) {
        made_here = at::empty({slots.n, x.tensor->size(1)}, x.tensor->options());
        out.ptr = made_here.data_ptr();
        out.stride = x.d;
    } else if (!out.take(a[5], "out", place, x.type, x.tensor->size(1), slots.n)) {
        return nullptr;
    }
    const int rc = without_lock(g_rows.by_transit, x.ptr, x.stride, x.type, x.n, x.d, (const int32_t*)slots.ptr, slots.n,
                                     (const int64_t*)counts.ptr, m, (const float*)weights.ptr, out.ptr, out.stride, place.stream);
    return made(rc, a[5], made_here);
}
ND_CATCH

// How many rows the slots belong to.
bool rows_of(const Flat& index, int32_t m, int64_t* rows) {
    if (m < 1 || index.n % m != 0) {
        PyErr_Format(PyExc_ValueError, "index must hold %d slots per row", m);
        return false;
    }
    *rows = index.n / m;
    return true;
}

// to_samples(z, index, m, weights, out or None, device, stream)
PyObject* to_samples(PyObject*, PyObject* const* a, Py_ssize_t n) try {
    Place place;
    Rows z, out;
    Flat index, weights;
    int32_t m;
    int64_t rows;
    if (!expects(n, 7) || !place.take(a[5], a[6]) || !z.take(a[0], "z", place) || !as_slots(a[2], &m) ||
        !index.take(a[1], "index", place, at::kInt, 0) || !rows_of(index, m, &rows) ||
        !weights.take(a[3], "weights", place, at::kFloat, index.n, true))
        return nullptr;
    at::Tensor made_here;
    if (a[4] == Py_None) {
        made_here = at::empty({rows, z.tensor->size(1)}, z.tensor->options());
        out.ptr = made_here.data_ptr();
        out.stride = z.d;
    } else if (!out.take(a[4], "out", place, z.type, z.tensor->size(1), rows)) {
        return nullptr;
    }
    const int rc = without_lock(g_rows.to_samples, z.ptr, z.stride, z.type, z.n, z.d, (const int32_t*)index.ptr, rows, m,
                                     (const float*)weights.ptr, out.ptr, out.stride, place.stream);
    return made(rc, a[4], made_here);
}
ND_CATCH

// weight_grad(dy, z, index, m, out or None, device, stream)
PyObject* weight_grad(PyObject*, PyObject* const* a, Py_ssize_t n) try {
    Place place;
    Rows dy, z;
    Flat index, out;
    int32_t m;
    int64_t rows;
    if (!expects(n, 7) || !place.take(a[5], a[6]) || !z.take(a[1], "z", place) || !as_slots(a[3], &m) ||
        !index.take(a[2], "index", place, at::kInt, 0) || !rows_of(index, m, &rows) ||
        !dy.take(a[0], "dy", place, z.type, z.tensor->size(1), rows))
        return nullptr;
    at::Tensor made_here;
    if (a[4] == Py_None) {
        made_here = at::empty({index.n}, z.tensor->options().dtype(at::kFloat));
        out.ptr = made_here.data_ptr();
    } else if (!out.take(a[4], "out", place, at::kFloat, index.n)) {
        return nullptr;
    }
    const int rc = without_lock(g_rows.weight_grad, dy.ptr, dy.stride, z.ptr, z.stride, z.type, z.n, z.d,
                                (const int32_t*)index.ptr, rows, m, (float*)out.ptr, place.stream);
    return made(rc, a[4], made_here);
}
ND_CATCH

// group_sum(x, sorted_slots, group_start, m, weights, group_rows, num_rows or None, counts, out or None, workspace or None,
//           device, stream)
PyObject* group_sum(PyObject*, PyObject* const* a, Py_ssize_t n) try {
    Place place;
    Rows x, out;
    Flat slots, start, weights, group_rows, counts, workspace;
    int32_t m;
    if (!expects(n, 12) || !place.take(a[10], a[11]) || !x.take(a[0], "x", place) || !as_slots(a[3], &m) ||
        !slots.take(a[1], "sorted_slots", place, at::kInt, 0) || !start.take(a[2], "group_start", place, at::kInt, 1))
        return nullptr;
    const int64_t groups = start.n - 1;
    if (!weights.take(a[4], "weights", place, at::kFloat, product_of(x.n, m), true) ||
        !group_rows.take(a[5], "group_rows", place, at::kInt, groups, true) ||
        !counts.take(a[7], "counts", place, at::kLong, 2, true))
        return nullptr;
    const bool table = a[5] != Py_None;
    int64_t rows = groups;
    if (table && a[6] != Py_None) {
        rows = PyLong_AsLongLong(a[6]);
        if (PyErr_Occurred()) return nullptr;
        if (rows < 0) {
            PyErr_SetString(PyExc_ValueError, "num_rows is negative");
            return nullptr;
        }
    } else if (a[8] != Py_None && THPVariable_Check(a[8]) && THPVariable_Unpack(a[8]).dim() == 2) {
        rows = THPVariable_Unpack(a[8]).size(0);
    } else if (table) {
        PyErr_SetString(PyExc_ValueError, "group_rows need num_rows or out");
        return nullptr;
    }
    at::Tensor made_here, scratch;
    if (a[8] == Py_None) {
        made_here = at::empty({rows, x.tensor->size(1)}, x.tensor->options());
        out.ptr = made_here.data_ptr();
        out.stride = x.d;
    } else if (!out.take(a[8], "out", place, x.type, x.tensor->size(1), rows)) {
        return nullptr;
    }
    size_t bytes;
    if (a[9] == Py_None) {
        bytes = g_rows.sum_bytes(slots.n, x.d);
        scratch = at::empty({(int64_t)bytes}, x.tensor->options().dtype(at::kByte));
        workspace.ptr = scratch.data_ptr();
    } else {
        if (!workspace.take(a[9], "workspace", place, at::ScalarType::Undefined, 0)) return nullptr;
        bytes = workspace.bytes();
    }
    // an empty tensor has no address; without groups it is not read
    const void* rows_ptr = table && groups == 0 ? out.ptr : group_rows.ptr;
    const int rc = without_lock(g_rows.group_sum, x.ptr, x.stride, x.type, x.n, x.d, (const int32_t*)slots.ptr, slots.n,
                                    (const int32_t*)start.ptr, groups, (const int64_t*)counts.ptr, m, (const float*)weights.ptr,
                                    (const int32_t*)rows_ptr, out.ptr, out.stride, rows, workspace.ptr, bytes, place.stream);
    return made(rc, a[8], made_here);
}
ND_CATCH

// x, w, labels, loss, lse, workspace of the softmax loss
struct LossArgs {
    Place place;
    Rows x, w;
    Flat labels, loss, lse, workspace;
    int32_t k = 1;
    bool take(PyObject* const* a, PyObject* dev, PyObject* str) {
        if (!place.take(dev, str) || !x.take(a[0], "x", place) || !w.take(a[1], "w", place, x.type, x.tensor->size(1)) ||
            !labels.take(a[2], "labels", place, at::kInt, 0))
            return false;
        const at::Tensor& l = *labels.tensor;
        if ((l.dim() != 1 && l.dim() != 2) || l.size(0) != x.n) {
            PyErr_SetString(PyExc_ValueError, "labels must hold one row of labels per row of x");
            return false;
        }
        const int64_t per = l.dim() == 2 ? l.size(1) : 1;
        k = per > ND_MAX_LABELS ? ND_MAX_LABELS + 1 : (int32_t)per;
        return loss.take(a[3], "loss", place, at::kFloat, x.n) && lse.take(a[4], "lse", place, at::kFloat, x.n) &&
               workspace.take(a[5], "workspace", place, at::ScalarType::Undefined, 0);
    }
};

// softmax_loss(x, w, labels, loss, lse, workspace, device, stream) -> code
PyObject* softmax_loss(PyObject*, PyObject* const* a, Py_ssize_t n) try {
    LossArgs c;
    if (!expects(n, 8) || !c.take(a, a[6], a[7])) return nullptr;
    return PyLong_FromLong(without_lock(g_rows.loss, c.x.ptr, c.x.stride, c.w.ptr, c.w.stride, c.x.type, c.x.n, c.w.n, c.x.d,
                                       (const int32_t*)c.labels.ptr, c.k, (float*)c.loss.ptr, (float*)c.lse.ptr, c.workspace.ptr,
                                       c.workspace.bytes(), c.place.stream));
}
ND_CATCH

// softmax_loss_grad(x, w, labels, loss, lse, workspace, row_weight, dx, dw, device, stream) -> code
PyObject* softmax_loss_grad(PyObject*, PyObject* const* a, Py_ssize_t n) try {
    LossArgs c;
    Flat row_weight;
    Rows dx, dw;
    if (!expects(n, 11) || !c.take(a, a[9], a[10]) || !row_weight.take(a[6], "row_weight", c.place, at::kFloat, c.x.n, true))
        return nullptr;
    dx.stride = dw.stride = c.x.d;
    if (a[7] != Py_None && !dx.take(a[7], "dx", c.place, c.x.type, c.x.tensor->size(1), c.x.n)) return nullptr;
    if (a[8] != Py_None && !dw.take(a[8], "dw", c.place, c.x.type, c.x.tensor->size(1), c.w.n)) return nullptr;
    return PyLong_FromLong(without_lock(g_rows.grad, c.x.ptr, c.x.stride, c.w.ptr, c.w.stride, c.x.type, c.x.n, c.w.n, c.x.d,
                                       (const int32_t*)c.labels.ptr, c.k, (const float*)row_weight.ptr, (float*)c.loss.ptr,
                                       (float*)c.lse.ptr, dx.ptr, dx.stride, dw.ptr, dw.stride, c.workspace.ptr,
                                       c.workspace.bytes(), c.place.stream));
}
ND_CATCH

PyMethodDef methods[] = {
    {"init", (PyCFunction)(void (*)())init, METH_FASTCALL, nullptr},
    {"sample", (PyCFunction)(void (*)())sample, METH_FASTCALL, nullptr},
    {"sample_static", (PyCFunction)(void (*)())sample_static, METH_FASTCALL, nullptr},
    {"pack", (PyCFunction)(void (*)())pack, METH_FASTCALL, nullptr},
    {"record_length", (PyCFunction)(void (*)())record_length, METH_FASTCALL, nullptr},
    {"init_rows", (PyCFunction)(void (*)())init_rows, METH_FASTCALL, nullptr},
    {"positions", (PyCFunction)(void (*)())positions, METH_FASTCALL, nullptr},
    {"by_transit", (PyCFunction)(void (*)())by_transit, METH_FASTCALL, nullptr},
    {"to_samples", (PyCFunction)(void (*)())to_samples, METH_FASTCALL, nullptr},
    {"weight_grad", (PyCFunction)(void (*)())weight_grad, METH_FASTCALL, nullptr},
    {"group_sum", (PyCFunction)(void (*)())group_sum, METH_FASTCALL, nullptr},
    {"softmax_loss", (PyCFunction)(void (*)())softmax_loss, METH_FASTCALL, nullptr},
    {"softmax_loss_grad", (PyCFunction)(void (*)())softmax_loss_grad, METH_FASTCALL, nullptr},
    {nullptr, nullptr, 0, nullptr},
};
PyModuleDef module = {PyModuleDef_HEAD_INIT, "_nd_call", nullptr, -1, methods, nullptr, nullptr, nullptr, nullptr};

}  // namespace

PyMODINIT_FUNC PyInit__nd_call(void) { return PyModule_Create(&module); }
