// Python marshalling of the calls a monitor makes every step: checks the tensors, takes their device pointers and the
// current stream, and calls the C ABI with the GIL released.  The same checks written in Python cost more than the
// kernels of a small fleet: ten output tensors, five attributes each, a stream object and a foreign call are some 15 us
// per evaluation, against under 2 us here.  The training-step operators allocate their outputs and workspaces here too
// (a lookup of a short prompt: 11.5 us from Python, its kernel 2).
#define PY_SSIZE_T_CLEAN
#include <Python.h>
#include <ATen/ops/empty.h>
#include <c10/cuda/CUDAFunctions.h>
#include <c10/cuda/CUDAGuard.h>
#include <c10/cuda/CUDAStream.h>
#include <torch/csrc/autograd/python_variable.h>

#include "../../include/guard_b200.h"

namespace {

// The device pointer of an optional tensor, or false with a Python error set.  `type`: the wanted scalar type.
bool device_ptr(PyObject *obj, c10::ScalarType type, int64_t numel, void **out) {
    *out = nullptr;
    if (!obj || obj == Py_None) return true;
    if (!THPVariable_Check(obj)) {
        PyErr_SetString(PyExc_ValueError, "expected a contiguous CUDA tensor");
        return false;
    }
    const at::Tensor &t = THPVariable_Unpack(obj);
    if (!t.is_cuda() || !t.is_contiguous()) {
        PyErr_SetString(PyExc_ValueError, "expected a contiguous CUDA tensor");
        return false;
    }
    if (t.scalar_type() != type) {
        PyErr_Format(PyExc_ValueError, "expected dtype %s, got %s", c10::toString(type), c10::toString(t.scalar_type()));
        return false;
    }
    if (t.numel() < numel) {
        PyErr_Format(PyExc_ValueError, "tensor too small: %lld < %lld elements", (long long)t.numel(), (long long)numel);
        return false;
    }
    *out = t.data_ptr();
    return true;
}

// out[name], or None (borrowed for a plain dict, else kept alive by the caller through `hold`).
PyObject *lookup(PyObject *out, PyObject *name, PyObject **hold) {
    if (PyDict_CheckExact(out)) {
        PyObject *v = PyDict_GetItemWithError(out, name);
        return v ? v : (PyErr_Occurred() ? nullptr : Py_None);
    }
    return *hold = PyObject_CallMethod(out, "get", "O", name);
}

struct Output {
    const char *name;
    c10::ScalarType type;
    PyObject *key;
};

// The device pointers of a mapping's outputs; numel[i] elements at least, a negative number skips the output.  keep: a new
// tuple of N, which receives references to them, or NULL.
template <int N>
bool output_ptrs(PyObject *out, Output (&spec)[N], const int64_t (&numel)[N], void *(&ptr)[N], PyObject *keep = nullptr) {
    for (int i = 0; i < N; ++i) {
        ptr[i] = nullptr;
        if (keep) {                // (no slot is ever empty)
            Py_INCREF(Py_None);
            PyTuple_SET_ITEM(keep, i, Py_None);
        }
        if (numel[i] < 0) continue;
        if (!spec[i].key) spec[i].key = PyUnicode_InternFromString(spec[i].name);
        PyObject *hold = nullptr, *v = lookup(out, spec[i].key, &hold);
        const bool ok = v && device_ptr(v, spec[i].type, numel[i], &ptr[i]);
        if (ok && keep) {
            Py_INCREF(v);
            PyTuple_SET_ITEM(keep, i, v);
            Py_DECREF(Py_None);
        }
        Py_XDECREF(hold);
        if (!ok) return false;
    }
    return true;
}

// Makes the device current where it is not, and hands out its current stream.
struct Here {
    c10::cuda::OptionalCUDAGuard guard;
    void *stream;
    explicit Here(int device) {
        if (c10::cuda::current_device() != device) guard.set_index((c10::DeviceIndex)device);
        stream = (void *)c10::cuda::getCurrentCUDAStream((c10::DeviceIndex)device).stream();
    }
};

// A reference that is dropped unless it is given away.
struct Ref {
    PyObject *o;
    ~Ref() { Py_XDECREF(o); }
    PyObject *give() {
        PyObject *r = o;
        o = nullptr;
        return r;
    }
};

bool to_ll(PyObject *o, long long *v) {
    *v = PyLong_AsLongLong(o);
    return !(*v == -1 && PyErr_Occurred());
}

bool want_args(Py_ssize_t n, Py_ssize_t want) {
    if (n == want) return true;
    PyErr_Format(PyExc_TypeError, "expected %zd arguments, got %zd", want, n);
    return false;
}

// current_stream(device) -> int
PyObject *py_current_stream(PyObject *, PyObject *const *args, Py_ssize_t n) {
    long long dev;
    if (!want_args(n, 1) || !to_ll(args[0], &dev)) return nullptr;
    try {
        return PyLong_FromVoidPtr((void *)c10::cuda::getCurrentCUDAStream((c10::DeviceIndex)dev).stream());
    } catch (const std::exception &e) {
        PyErr_SetString(PyExc_RuntimeError, e.what());
        return nullptr;
    }
}

// ingest(handle, device, R, M, block, step_med, step_mad) -> status
PyObject *py_ingest(PyObject *, PyObject *const *args, Py_ssize_t n) {
    long long h, dev, R, M;
    if (!want_args(n, 7) || !to_ll(args[0], &h) || !to_ll(args[1], &dev) || !to_ll(args[2], &R) || !to_ll(args[3], &M)) return nullptr;
    if (!THPVariable_Check(args[4])) {
        PyErr_SetString(PyExc_ValueError, "block must be a tensor");
        return nullptr;
    }
    try {
        const at::Tensor &b = THPVariable_Unpack(args[4]);
        if (b.dim() != 3 || b.size(1) != R || b.size(2) != M) {
            PyErr_Format(PyExc_ValueError, "block must be [B, %lld, %lld]", R, M);
            return nullptr;
        }
        const int64_t B = b.size(0);
        void *pb, *pm, *pd;
        if (!device_ptr(args[4], c10::kFloat, 0, &pb) || !device_ptr(args[5], c10::kFloat, B * M, &pm) ||
            !device_ptr(args[6], c10::kFloat, B * M, &pd))
            return nullptr;
        Here here((int)dev);
        int rc;
        Py_BEGIN_ALLOW_THREADS
        rc = guard_ingest((guard_ctx *)h, (const float *)pb, B > 0x7FFFFFFF ? -1 : (int)B, (float *)pm, (float *)pd, here.stream);
        Py_END_ALLOW_THREADS
        return PyLong_FromLong(rc);
    } catch (const std::exception &e) {
        PyErr_SetString(PyExc_RuntimeError, e.what());
        return nullptr;
    }
}

Output g_score_out[10] = {{"wmed", c10::kFloat, nullptr},      {"fleet_med", c10::kFloat, nullptr}, {"fleet_mad", c10::kFloat, nullptr},
                          {"scores", c10::kFloat, nullptr},    {"counts", c10::kUInt16, nullptr},   {"mask", c10::kUInt32, nullptr},
                          {"flags", c10::kByte, nullptr},      {"tier", c10::kByte, nullptr},       {"topk_idx", c10::kInt, nullptr},
                          {"topk_score", c10::kFloat, nullptr}};

// score(handle, device, R, M, K, out, hold) -> status; with hold, references to the outputs in the place of a zero
PyObject *py_score(PyObject *, PyObject *const *args, Py_ssize_t n) {
    long long h, dev, R, M, K;
    if (!want_args(n, 7) || !to_ll(args[0], &h) || !to_ll(args[1], &dev) || !to_ll(args[2], &R) || !to_ll(args[3], &M) || !to_ll(args[4], &K))
        return nullptr;
    try {
        const int64_t numel[10] = {R * M, M, M, R * M, R * M, R, R, R, K > 0 ? K : -1, K > 0 ? K : -1};
        void *p[10];
        Ref keep{args[6] == Py_True ? PyTuple_New(10) : nullptr};
        if (args[6] == Py_True && !keep.o) return nullptr;
        if (!output_ptrs(args[5], g_score_out, numel, p, keep.o)) return nullptr;
        Here here((int)dev);
        int rc;
        Py_BEGIN_ALLOW_THREADS
        rc = guard_score((guard_ctx *)h, (float *)p[0], (float *)p[1], (float *)p[2], (float *)p[3], (uint16_t *)p[4], (uint32_t *)p[5],
                         (uint8_t *)p[6], (uint8_t *)p[7], (int32_t *)p[8], (float *)p[9], here.stream);
        Py_END_ALLOW_THREADS
        return rc == GUARD_OK && keep.o ? keep.give() : PyLong_FromLong(rc);
    } catch (const std::exception &e) {
        PyErr_SetString(PyExc_RuntimeError, e.what());
        return nullptr;
    }
}

Output g_node_out[3] = {{"node_flag", c10::kByte, nullptr}, {"node_tier", c10::kByte, nullptr}, {"node_stall", c10::kUInt16, nullptr}};

// node_verdict(handle, device, nodes, out) -> status
PyObject *py_node_verdict(PyObject *, PyObject *const *args, Py_ssize_t n) {
    long long h, dev, N;
    if (!want_args(n, 4) || !to_ll(args[0], &h) || !to_ll(args[1], &dev) || !to_ll(args[2], &N)) return nullptr;
    try {
        const int64_t numel[3] = {N, N, N};
        void *p[3];
        if (!output_ptrs(args[3], g_node_out, numel, p)) return nullptr;
        Here here((int)dev);
        int rc;
        Py_BEGIN_ALLOW_THREADS
        rc = guard_node_verdict((guard_ctx *)h, (uint8_t *)p[0], (uint8_t *)p[1], (uint16_t *)p[2], here.stream);
        Py_END_ALLOW_THREADS
        return PyLong_FromLong(rc);
    } catch (const std::exception &e) {
        PyErr_SetString(PyExc_RuntimeError, e.what());
        return nullptr;
    }
}

// join(handle, device) -> status
PyObject *py_join(PyObject *, PyObject *const *args, Py_ssize_t n) {
    long long h, dev;
    if (!want_args(n, 2) || !to_ll(args[0], &h) || !to_ll(args[1], &dev)) return nullptr;
    try {
        Here here((int)dev);
        int rc;
        Py_BEGIN_ALLOW_THREADS
        rc = guard_join((guard_ctx *)h, here.stream);
        Py_END_ALLOW_THREADS
        return PyLong_FromLong(rc);
    } catch (const std::exception &e) {
        PyErr_SetString(PyExc_RuntimeError, e.what());
        return nullptr;
    }
}

// A per-metric parameter.  dir (whole): any iterable of M values that int() takes.  The others: anything with a length, of M
// numbers, or one number for all metrics.
template <typename T>
bool per_metric(PyObject *obj, int M, bool whole, T *out) {
    auto one = [&](PyObject *v, T *dst) {
        if (whole) {
            PyObject *i = PyNumber_Long(v);
            if (!i) return false;
            *dst = (T)PyLong_AsUnsignedLongLongMask(i);
            Py_DECREF(i);
            return !PyErr_Occurred();
        }
        const double x = PyFloat_AsDouble(v);
        if (x == -1.0 && PyErr_Occurred()) return false;
        *dst = (T)x;
        return true;
    };
    if (!whole && (PyFloat_Check(obj) || PyLong_Check(obj) || !PyObject_HasAttrString(obj, "__len__"))) {
        if (!one(obj, &out[0])) return false;
        for (int m = 1; m < M; ++m) out[m] = out[0];
        return true;
    }
    PyObject *seq = PySequence_Fast(obj, "expected an iterable of per-metric values");
    if (!seq) return false;
    const Py_ssize_t len = PySequence_Fast_GET_SIZE(seq);
    bool ok = len == M;
    if (!ok) PyErr_Format(PyExc_ValueError, "expected %d per-metric values, got %zd", M, len);
    for (int m = 0; ok && m < M; ++m) ok = one(PySequence_Fast_GET_ITEM(seq, m), &out[m]);
    Py_DECREF(seq);
    return ok;
}

Output g_sweep_out[8] = {{"gpu_med", c10::kFloat, nullptr},   {"fleet_med", c10::kFloat, nullptr}, {"fleet_mad", c10::kFloat, nullptr},
                         {"fleet_cut", c10::kFloat, nullptr}, {"fail_mask", c10::kUInt32, nullptr}, {"gpu_pass", c10::kByte, nullptr},
                         {"node_pass", c10::kByte, nullptr},  {"status", c10::kUInt32, nullptr}};

// sweep_qualify(device, S, nodes, gpus_per_node, dir, thr, floor_rel, floor_abs, pct_ppm, workspace, out) -> status
PyObject *py_sweep_qualify(PyObject *, PyObject *const *args, Py_ssize_t n) {
    long long dev, nodes, gpn, pct;
    if (!want_args(n, 11) || !to_ll(args[0], &dev) || !to_ll(args[2], &nodes) || !to_ll(args[3], &gpn) || !to_ll(args[8], &pct)) return nullptr;
    try {
        if (!THPVariable_Check(args[1]) || !THPVariable_Check(args[9])) {
            PyErr_SetString(PyExc_ValueError, "S and workspace must be tensors");
            return nullptr;
        }
        const at::Tensor &S = THPVariable_Unpack(args[1]);
        const int64_t G = S.size(0), reps = S.size(1), M = S.size(2);
        int8_t dir[GUARD_MAX_METRICS];
        float thr[GUARD_MAX_METRICS], frel[GUARD_MAX_METRICS], fabs_[GUARD_MAX_METRICS];
        if (M < 1 || M > GUARD_MAX_METRICS) {
            PyErr_SetString(PyExc_ValueError, "number of metrics out of range");
            return nullptr;
        }
        void *ps, *pw;
        const int64_t numel[8] = {G * M, M, M, M, G, G, nodes, 1};
        void *p[8];
        if (!per_metric(args[4], (int)M, true, dir) || !per_metric(args[5], (int)M, false, thr) || !per_metric(args[6], (int)M, false, frel) ||
            !per_metric(args[7], (int)M, false, fabs_) || !device_ptr(args[1], c10::kFloat, 0, &ps) || !device_ptr(args[9], c10::kByte, 0, &pw) ||
            !output_ptrs(args[10], g_sweep_out, numel, p))
            return nullptr;
        guard_thresholds th{0, 2, 1, 8, 0.10f, 0.20f, dir, thr, frel, fabs_};
        const size_t wbytes = (size_t)THPVariable_Unpack(args[9]).numel();
        Here here((int)dev);
        int rc;
        Py_BEGIN_ALLOW_THREADS
        rc = guard_sweep_qualify((const float *)ps, (int)nodes, (int)gpn, (int)reps, (int)M, &th, (int32_t)pct, pw, wbytes, (float *)p[0],
                                 (float *)p[1], (float *)p[2], (float *)p[3], (uint32_t *)p[4], (uint8_t *)p[5], (uint8_t *)p[6],
                                 (uint32_t *)p[7], here.stream);
        Py_END_ALLOW_THREADS
        return PyLong_FromLong(rc);
    } catch (const std::exception &e) {
        PyErr_SetString(PyExc_RuntimeError, e.what());
        return nullptr;
    }
}

// ---- training-step operators --------------------------------------------------------------------------------------

constexpr int kMaxDevices = 64;
uint32_t *g_status[kMaxDevices];       // the status word of each device, set from Python

// set_status(device, address)
PyObject *py_set_status(PyObject *, PyObject *const *args, Py_ssize_t n) {
    long long dev, p;
    if (!want_args(n, 2) || !to_ll(args[0], &dev) || !to_ll(args[1], &p)) return nullptr;
    if (dev < 0 || dev >= kMaxDevices) {
        PyErr_SetString(PyExc_ValueError, "device out of range");
        return nullptr;
    }
    g_status[dev] = (uint32_t *)p;
    Py_RETURN_NONE;
}

// A call's tensors: checks that set a Python error and return false, and outputs made or taken from the caller's mapping.
struct Call {
    int device = -1;
    at::Tensor kept[8];        // what the caller's mapping held, which other threads may change while the GIL is released
    int n_kept = 0;
    const at::Tensor *cuda(PyObject *o, const char *what) {
        if (!THPVariable_Check(o) || !THPVariable_Unpack(o).is_cuda()) {
            PyErr_Format(PyExc_ValueError, "%s must be a CUDA tensor", what);
            return nullptr;
        }
        const at::Tensor &t = THPVariable_Unpack(o);
        if (device < 0) device = t.get_device();
        if (t.get_device() != device) {
            PyErr_Format(PyExc_ValueError, "%s is on cuda:%d, the other tensors on cuda:%d", what, (int)t.get_device(), device);
            return nullptr;
        }
        return &t;
    }
    static int dtype(const at::Tensor &t, const char *what) {
        if (t.scalar_type() == c10::kFloat) return GUARD_F32;
        if (t.scalar_type() == c10::kBFloat16) return GUARD_BF16;
        if (t.scalar_type() == c10::kHalf) return GUARD_F16;
        PyErr_Format(PyExc_ValueError, "%s must be float32, bfloat16 or float16, got %s", what, c10::toString(t.scalar_type()));
        return -1;
    }
    // Distance of the rows of a matrix whose rows are contiguous, or -1.
    static int64_t rows(const at::Tensor &t, const char *what) {
        if (t.dim() != 2) {
            PyErr_Format(PyExc_ValueError, "%s must be a matrix", what);
            return -1;
        }
        const int64_t n = t.size(0), d = t.size(1);
        if ((d > 1 && t.stride(1) != 1) || (n > 1 && t.stride(0) < d)) {
            PyErr_Format(PyExc_ValueError, "%s must have contiguous rows that do not overlap", what);
            return -1;
        }
        return n > 1 ? t.stride(0) : d;
    }
    static int token_bits(const at::Tensor &t, const char *what) {
        const int bits = t.scalar_type() == c10::kLong ? 64 : t.scalar_type() == c10::kInt ? 32 : 0;
        if (!bits || !t.is_contiguous()) {
            PyErr_Format(PyExc_ValueError, "%s must be contiguous, int32 or int64", what);
            return 0;
        }
        return bits;
    }
    bool flat(PyObject *o, const char *what, c10::ScalarType type, int64_t numel, void **to) {
        const at::Tensor *t = cuda(o, what);
        if (!t) return false;
        if (t->scalar_type() != type || !t->is_contiguous() || t->numel() != numel) {
            PyErr_Format(PyExc_ValueError, "%s must be contiguous, of %s and of %lld elements", what, c10::toString(type), (long long)numel);
            return false;
        }
        kept[n_kept++] = *t;
        *to = t->data_ptr();
        return true;
    }
    at::Tensor make(at::IntArrayRef size, c10::ScalarType type) const {
        return at::empty(size, at::TensorOptions().dtype(type).device(c10::Device(c10::kCUDA, (c10::DeviceIndex)device)));
    }
    // An entry of the caller's mapping (NULL pointer: missing or None; allowed only where optional), or, without a mapping, a
    // new tensor that is put into `made`.
    bool output(PyObject *out, PyObject *made, const char *name, c10::ScalarType type, at::IntArrayRef size, bool optional, void **to) {
        int64_t numel = 1;
        for (int64_t d : size) numel *= d;
        *to = nullptr;
        if (out == Py_None) {
            at::Tensor t = make(size, type);
            *to = t.data_ptr();
            Ref w{THPVariable_Wrap(std::move(t))};
            return w.o && PyDict_SetItemString(made, name, w.o) == 0;
        }
        Ref v{PyObject_CallMethod(out, "get", "s", name)};
        if (!v.o) return false;
        if (v.o == Py_None) {
            if (optional) return true;
            PyErr_Format(PyExc_ValueError, "out['%s'] is missing", name);
            return false;
        }
        return flat(v.o, name, type, numel, to) && wrote(kept[n_kept - 1]);
    }
    // Tells autograd that a tensor's values change, as torch's own in-place operations do.
    static bool wrote(const at::Tensor &t) {
        if (!t.is_inference()) t.unsafeGetTensorImpl()->bump_version();
        return true;
    }
    bool workspace(PyObject *given, size_t need, at::Tensor &keep, void **p, size_t *bytes) {
        if (given == Py_None) {
            if (need) keep = make({(int64_t)need}, c10::kByte);
            *p = need ? keep.data_ptr() : nullptr;
            *bytes = need;
            return true;
        }
        const at::Tensor *t = cuda(given, "workspace");
        if (!t) return false;
        if (t->scalar_type() != c10::kByte || !t->is_contiguous()) {
            PyErr_SetString(PyExc_ValueError, "workspace must be contiguous, of torch.uint8");
            return false;
        }
        *p = t->data_ptr();
        *bytes = (size_t)t->numel();
        return true;
    }
    bool status(PyObject *out, uint32_t **p) {
        *p = device >= 0 && device < kMaxDevices ? g_status[device] : nullptr;
        if (out == Py_None) return true;
        Ref v{PyObject_CallMethod(out, "get", "s", "status")};
        if (!v.o) return false;
        void *q;
        if (v.o == Py_None) return true;
        if (!flat(v.o, "status", c10::kUInt32, 1, &q)) return false;
        *p = (uint32_t *)q;
        return true;
    }
};

// The mapping of outputs, or the error code of the C call.
PyObject *result(int rc, PyObject *out, Ref &made) {
    if (rc != GUARD_OK) return PyLong_FromLong(rc);
    if (out == Py_None) return made.give();
    Py_INCREF(out);
    return out;
}

// embed(tokens, table, scale, out) -> outputs or status
PyObject *py_embed(PyObject *, PyObject *const *args, Py_ssize_t n) {
    if (!want_args(n, 4)) return nullptr;
    const double scale = PyFloat_AsDouble(args[2]);
    if (scale == -1.0 && PyErr_Occurred()) return nullptr;
    try {
        Call c;
        const at::Tensor *table = c.cuda(args[1], "table"), *tokens = table ? c.cuda(args[0], "tokens") : nullptr;
        if (!tokens) return nullptr;
        const int bits = Call::token_bits(*tokens, "tokens"), code = bits ? Call::dtype(*table, "table") : -1;
        const int64_t stride = code >= 0 ? Call::rows(*table, "table") : -1;
        if (stride < 0) return nullptr;
        const int64_t width = table->size(1);
        Here here(c.device);
        Ref made{PyDict_New()};
        c10::SmallVector<int64_t, 6> size(tokens->sizes().begin(), tokens->sizes().end());
        size.push_back(width);
        void *to;
        uint32_t *status;
        if (!made.o || !c.output(args[3], made.o, "out", table->scalar_type(), size, false, &to) || !c.status(args[3], &status)) return nullptr;
        const void *ids = tokens->data_ptr(), *from = table->data_ptr();
        const int64_t count = tokens->numel(), rows = table->size(0);
        int rc;
        Py_BEGIN_ALLOW_THREADS
        rc = guard_embed(ids, bits, count, from, rows, width, stride, code, (float)scale, to, status, here.stream);
        Py_END_ALLOW_THREADS
        return result(rc, args[3], made);
    } catch (const std::exception &e) {
        PyErr_SetString(PyExc_RuntimeError, e.what());
        return nullptr;
    }
}

// embed_grad(grad, tokens, rows, scale, padding_idx, accumulate, workspace, out) -> outputs or status
PyObject *py_embed_grad(PyObject *, PyObject *const *args, Py_ssize_t n) {
    long long rows, padding;
    if (!want_args(n, 8) || !to_ll(args[2], &rows) || !to_ll(args[4], &padding)) return nullptr;
    const double scale = PyFloat_AsDouble(args[3]);
    if (scale == -1.0 && PyErr_Occurred()) return nullptr;
    const int accumulate = PyObject_IsTrue(args[5]);
    if (accumulate < 0) return nullptr;
    try {
        Call c;
        const at::Tensor *given = c.cuda(args[0], "grad"), *tokens = given ? c.cuda(args[1], "tokens") : nullptr;
        if (!tokens) return nullptr;
        at::Tensor grad = *given;
        if (grad.dim() != 2 && grad.dim() > 0 && grad.is_contiguous() && grad.size(-1) > 0) grad = grad.view({-1, grad.size(-1)});
        const int bits = Call::token_bits(*tokens, "tokens"), code = bits ? Call::dtype(grad, "grad") : -1;
        const int64_t stride = code >= 0 ? Call::rows(grad, "grad") : -1;
        if (stride < 0) return nullptr;
        const int64_t count = grad.size(0), width = grad.size(1);
        if (tokens->numel() != count) {
            PyErr_Format(PyExc_ValueError, "%lld gradient rows for %lld tokens", (long long)count, (long long)tokens->numel());
            return nullptr;
        }
        if (accumulate && args[7] == Py_None) {
            PyErr_SetString(PyExc_ValueError, "accumulate needs out['dtable']");
            return nullptr;
        }
        Here here(c.device);
        Ref made{PyDict_New()};
        void *to, *ws;
        uint32_t *status;
        size_t bytes;
        at::Tensor keep;
        const size_t need = guard_embed_grad_workspace_bytes(count, rows, width);
        if (need == 0) return PyLong_FromLong(guard_embed_grad(nullptr, stride, code, nullptr, bits, count, rows, width, 1.0f, -1, 0, nullptr, nullptr, 0, nullptr, nullptr));
        if (!made.o || !c.output(args[7], made.o, "dtable", grad.scalar_type(), {rows, width}, false, &to) || !c.workspace(args[6], need, keep, &ws, &bytes) ||
            !c.status(args[7], &status))
            return nullptr;
        const void *from = grad.data_ptr(), *ids = tokens->data_ptr();
        int rc;
        Py_BEGIN_ALLOW_THREADS
        rc = guard_embed_grad(from, stride, code, ids, bits, count, rows, width, (float)scale, padding, accumulate, to, ws, bytes, status, here.stream);
        Py_END_ALLOW_THREADS
        return result(rc, args[7], made);
    } catch (const std::exception &e) {
        PyErr_SetString(PyExc_RuntimeError, e.what());
        return nullptr;
    }
}

// The product's inputs, as both directions take them.
struct Product {
    const at::Tensor *x = nullptr, *w = nullptr, *targets = nullptr;
    int bits = 0, code = -1;
    const void *px = nullptr, *pw = nullptr, *pt = nullptr;
    int64_t xs = -1, ws = -1, rows = 0, width = 0, vocab = 0;
    bool read(Call &c, PyObject *const *args) {
        if (!(x = c.cuda(args[0], "x")) || !(w = c.cuda(args[1], "w")) || !(targets = c.cuda(args[2], "targets")) || !(bits = Call::token_bits(*targets, "targets")) ||
            (code = Call::dtype(*x, "x")) < 0)
            return false;
        if (w->scalar_type() != x->scalar_type() || code == GUARD_F32) {
            PyErr_Format(PyExc_ValueError, "x and w must both be bfloat16 or both float16, got %s and %s", c10::toString(x->scalar_type()), c10::toString(w->scalar_type()));
            return false;
        }
        if ((xs = Call::rows(*x, "x")) < 0 || (ws = Call::rows(*w, "w")) < 0) return false;
        rows = x->size(0), width = x->size(1), vocab = w->size(0);
        px = x->data_ptr(), pw = w->data_ptr(), pt = targets->data_ptr();
        if (w->size(1) != width || targets->numel() != rows) {
            PyErr_SetString(PyExc_ValueError, "need x [rows, width], w [vocab, width] and rows targets");
            return false;
        }
        return true;
    }
};

// linear_xent(x, w, targets, ignore_index, workspace, out) -> outputs or status
PyObject *py_linear_xent(PyObject *, PyObject *const *args, Py_ssize_t n) {
    long long ignore;
    if (!want_args(n, 6) || !to_ll(args[3], &ignore)) return nullptr;
    try {
        Call c;
        Product p;
        if (!p.read(c, args)) return nullptr;
        Here here(c.device);
        Ref made{PyDict_New()};
        void *loss, *lse, *ws;
        uint32_t *status;
        size_t bytes;
        at::Tensor keep;
        if (!made.o || !c.output(args[5], made.o, "loss", c10::kFloat, {p.rows}, false, &loss) || !c.output(args[5], made.o, "lse", c10::kFloat, {p.rows}, false, &lse) ||
            !c.workspace(args[4], guard_linear_xent_workspace_bytes(p.rows, p.width, p.vocab, 0), keep, &ws, &bytes) || !c.status(args[5], &status))
            return nullptr;
        int rc;
        Py_BEGIN_ALLOW_THREADS
        rc = guard_linear_xent(p.px, p.xs, p.pw, p.ws, p.rows, p.width, p.vocab, p.code, p.pt, p.bits, ignore, (float *)loss, (float *)lse, ws, bytes, status,
                               here.stream);
        Py_END_ALLOW_THREADS
        return result(rc, args[5], made);
    } catch (const std::exception &e) {
        PyErr_SetString(PyExc_RuntimeError, e.what());
        return nullptr;
    }
}

// linear_xent_grad(x, w, targets, lse, grad_loss, ignore_index, workspace, out) -> outputs or status
PyObject *py_linear_xent_grad(PyObject *, PyObject *const *args, Py_ssize_t n) {
    long long ignore;
    if (!want_args(n, 8) || !to_ll(args[5], &ignore)) return nullptr;
    try {
        Call c;
        Product p;
        if (!p.read(c, args)) return nullptr;
        Here here(c.device);
        Ref made{PyDict_New()};
        void *dx, *dw, *lse, *g, *ws;
        uint32_t *status;
        size_t bytes;
        at::Tensor keep;
        const at::Tensor *grad = c.cuda(args[4], "grad_loss");
        if (!grad) return nullptr;
        const bool one = grad->numel() == 1 && p.rows != 1;
        if (!made.o || !c.flat(args[3], "lse", c10::kFloat, p.rows, &lse) || !c.flat(args[4], "grad_loss", c10::kFloat, one ? 1 : p.rows, &g) ||
            !c.output(args[7], made.o, "dx", p.x->scalar_type(), {p.rows, p.width}, true, &dx) ||
            !c.output(args[7], made.o, "dw", p.w->scalar_type(), {p.vocab, p.width}, true, &dw) ||
            !c.workspace(args[6], guard_linear_xent_workspace_bytes(p.rows, p.width, p.vocab, 1), keep, &ws, &bytes) || !c.status(args[7], &status))
            return nullptr;
        int rc;
        Py_BEGIN_ALLOW_THREADS
        rc = guard_linear_xent_grad(p.px, p.xs, p.pw, p.ws, p.rows, p.width, p.vocab, p.code, p.pt, p.bits, ignore, (const float *)lse, (const float *)g,
                                    one ? 0 : 1, dx, dw, ws, bytes, status, here.stream);
        Py_END_ALLOW_THREADS
        return result(rc, args[7], made);
    } catch (const std::exception &e) {
        PyErr_SetString(PyExc_RuntimeError, e.what());
        return nullptr;
    }
}

// wrote(tuple of tensors): they have been written in place
PyObject *py_wrote(PyObject *, PyObject *const *args, Py_ssize_t n) {
    if (!want_args(n, 1)) return nullptr;
    if (!PyTuple_CheckExact(args[0])) {
        PyErr_SetString(PyExc_TypeError, "expected a tuple");
        return nullptr;
    }
    for (Py_ssize_t i = 0; i < PyTuple_GET_SIZE(args[0]); ++i) {
        PyObject *o = PyTuple_GET_ITEM(args[0], i);
        if (THPVariable_Check(o)) Call::wrote(THPVariable_Unpack(o));
    }
    Py_RETURN_NONE;
}

PyMethodDef g_methods[] = {{"current_stream", (PyCFunction)(void (*)(void))py_current_stream, METH_FASTCALL, nullptr},
                           {"ingest", (PyCFunction)(void (*)(void))py_ingest, METH_FASTCALL, nullptr},
                           {"score", (PyCFunction)(void (*)(void))py_score, METH_FASTCALL, nullptr},
                           {"node_verdict", (PyCFunction)(void (*)(void))py_node_verdict, METH_FASTCALL, nullptr},
                           {"join", (PyCFunction)(void (*)(void))py_join, METH_FASTCALL, nullptr},
                           {"sweep_qualify", (PyCFunction)(void (*)(void))py_sweep_qualify, METH_FASTCALL, nullptr},
                           {"set_status", (PyCFunction)(void (*)(void))py_set_status, METH_FASTCALL, nullptr},
                           {"embed", (PyCFunction)(void (*)(void))py_embed, METH_FASTCALL, nullptr},
                           {"embed_grad", (PyCFunction)(void (*)(void))py_embed_grad, METH_FASTCALL, nullptr},
                           {"linear_xent", (PyCFunction)(void (*)(void))py_linear_xent, METH_FASTCALL, nullptr},
                           {"linear_xent_grad", (PyCFunction)(void (*)(void))py_linear_xent_grad, METH_FASTCALL, nullptr},
                           {"wrote", (PyCFunction)(void (*)(void))py_wrote, METH_FASTCALL, nullptr},
                           {nullptr, nullptr, 0, nullptr}};
PyModuleDef g_module = {PyModuleDef_HEAD_INIT, "_guard_native", nullptr, -1, g_methods, nullptr, nullptr, nullptr, nullptr};

}  // namespace

PyMODINIT_FUNC PyInit__guard_native(void) { return PyModule_Create(&g_module); }
