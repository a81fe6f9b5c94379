// host.cpp -- the per-step calls of include/picasso.h for Python: a CPython module that checks tensors, allocates
// outputs (with torch's allocator, on the current stream) and calls the library.  Through ctypes a call took about 12
// microseconds of Python, several times what its kernel runs on a small mesh; through this module about 5.
#include <Python.h>

#include <ATen/ATen.h>
#include <c10/core/StreamGuard.h>
#include <c10/core/impl/VirtualGuardImpl.h>
#include <torch/csrc/Exceptions.h>
#include <torch/csrc/autograd/python_variable.h>

#include <cmath>
#include <optional>
#include <string>
#include <vector>

#include "../../include/picasso.h"

namespace {

PyObject* g_current_device = nullptr;  // () -> index of the current device
PyObject* g_current_stream = nullptr;  // (device index) -> its current stream as a number
PyObject* g_raise = nullptr;           // (context, status): raises the exception for a failed call

struct PyError {};  // a Python exception has been set

[[noreturn]] void fail(PyObject* type, const char* text) {
    PyErr_SetString(type, text);
    throw PyError{};
}

// The positional arguments of a call.
struct Args {
    PyObject* const* a;
    Py_ssize_t n, at = 0;
    PyObject* next() {
        if (at >= n) fail(PyExc_TypeError, "too few arguments");
        return a[at++];
    }
    long long integer() {
        PyObject* o = next();
        long long v;
        if (PyLong_Check(o)) {
            v = PyLong_AsLongLong(o);
        } else {
            PyObject* l = PyNumber_Long(o);
            if (!l) throw PyError{};
            v = PyLong_AsLongLong(l);
            Py_DECREF(l);
        }
        if (v == -1 && PyErr_Occurred()) throw PyError{};
        return v;
    }
    int i32() { return (int)integer(); }
    picasso_ctx* context() { return reinterpret_cast<picasso_ctx*>((intptr_t)integer()); }
    void* stream() {
        PyObject* o = next();
        PyObject* number;
        if (o == Py_None) {
            PyObject* device = PyObject_CallNoArgs(g_current_device);
            if (!device) throw PyError{};
            number = PyObject_CallOneArg(g_current_stream, device);
            Py_DECREF(device);
        } else {
            number = PyObject_GetAttrString(o, "cuda_stream");
        }
        if (!number) throw PyError{};
        void* s = PyLong_AsVoidPtr(number);
        Py_DECREF(number);
        if (PyErr_Occurred()) throw PyError{};
        return s;
    }
    // a contiguous CUDA tensor of the given type, or (unless its shape is needed) null for None
    const at::Tensor* tensor(at::ScalarType type, const char* what, bool required) {
        PyObject* o = next();
        if (o == Py_None && !required) return nullptr;
        if (THPVariable_Check(o)) {
            const at::Tensor& t = THPVariable_Unpack(o);
            if (t.is_cuda() && t.scalar_type() == type && t.is_contiguous()) return &t;
        }
        PyObject* shape = required ? PyObject_GetAttrString(o, "shape") : nullptr;
        if (required && !shape) throw PyError{};  // (not an array at all)
        Py_XDECREF(shape);
        PyErr_Format(PyExc_TypeError, "%s: expected a contiguous CUDA tensor of dtype %s", what,
                     type == at::kFloat ? "torch.float32" : "torch.int32");
        throw PyError{};
    }
    const at::Tensor& f32(const char* what) { return *tensor(at::kFloat, what, true); }
    const at::Tensor& ints(const char* what) { return *tensor(at::kInt, what, true); }
    const at::Tensor* maybe_f32(const char* what) { return tensor(at::kFloat, what, false); }
    const at::Tensor* maybe_ints(const char* what) { return tensor(at::kInt, what, false); }
};

int rows(const at::Tensor& t, int dim = 0) {
    if (t.dim() <= dim) fail(PyExc_IndexError, "tuple index out of range");
    return (int)t.size(dim);
}
at::Tensor out_f32(at::IntArrayRef shape, const at::Tensor& like) { return at::empty(shape, at::TensorOptions().dtype(at::kFloat).device(like.device())); }
at::Tensor out_i32(at::IntArrayRef shape, const at::Tensor& like) { return at::empty(shape, at::TensorOptions().dtype(at::kInt).device(like.device())); }
float* F(const at::Tensor& t) { return static_cast<float*>(t.data_ptr()); }
int32_t* I(const at::Tensor& t) { return static_cast<int32_t*>(t.data_ptr()); }
float* F(const at::Tensor* t) { return t ? F(*t) : nullptr; }
int32_t* I(const at::Tensor* t) { return t ? I(*t) : nullptr; }

// The library's call without the interpreter's lock.
template <class Call>
int unlocked(Call call) {
    PyThreadState* s = PyEval_SaveThread();
    const int st = call();
    PyEval_RestoreThread(s);
    return st;
}
template <class Call>
void checked(picasso_ctx* c, Call call) {
    const int st = unlocked(call);
    if (st == PICASSO_OK) return;
    PyObject* r = PyObject_CallFunction(g_raise, "Ki", (unsigned long long)(intptr_t)c, st);
    Py_XDECREF(r);
    if (!PyErr_Occurred()) PyErr_SetString(PyExc_RuntimeError, "a library call failed");
    throw PyError{};
}

PyObject* wrap(at::Tensor t) { return THPVariable_Wrap(std::move(t)); }
PyObject* pack(std::initializer_list<PyObject*> items) {
    PyObject* t = PyTuple_New((Py_ssize_t)items.size());
    Py_ssize_t i = 0;
    for (PyObject* o : items) PyTuple_SET_ITEM(t, i++, o);
    return t;
}
PyObject* none() { Py_RETURN_NONE; }

// Exceptions of C++ become Python's, torch's (an allocation that fails, say) the ones that torch raises for them.
template <PyObject* (*Body)(Args&)>
PyObject* entry(PyObject*, PyObject* const* a, Py_ssize_t n) {
    try {
        Args args{a, n};
        return Body(args);
    } catch (const PyError&) {
    } catch (...) {
        torch::translate_exception_to_python(std::current_exception());
    }
    return nullptr;
}

PyObject* decimate(Args& a) {
    picasso_ctx* c = a.context();
    void* s = a.stream();
    const at::Tensor &v = a.f32("verts"), &f = a.ints("facets");
    const int target = a.i32();
    const at::Tensor *vo_ = a.maybe_f32("verts_out"), *fo_ = a.maybe_ints("facets_out"), *cid_ = a.maybe_ints("cluster_id");
    picasso_stats* stats = reinterpret_cast<picasso_stats*>((intptr_t)a.integer());
    const int N = rows(v), nF = rows(f);
    const at::Tensor vo = vo_ ? *vo_ : out_f32({std::max(N, 1), 3}, v), fo = fo_ ? *fo_ : out_i32({std::max(nF, 1), 3}, v),
                     cid = cid_ ? *cid_ : out_i32({std::max(N, 1)}, v);
    int32_t nv = 0, nf = 0;
    const int st = unlocked([&] { return picasso_decimate(c, s, F(v), N, I(f), nF, target, F(vo), I(fo), I(cid), &nv, &nf, stats); });
    if (st < 0) return pack({PyLong_FromLong(st), none(), none(), none()});
    return pack({PyLong_FromLong(st), wrap(vo.narrow(0, 0, nv)), wrap(fo.narrow(0, 0, nf)), wrap(cid.narrow(0, 0, N))});
}

// n int32 values of an object with the buffer interface (a contiguous numpy array)
struct HostInts {
    Py_buffer b{};
    HostInts(PyObject* o, bool writable) {
        if (PyObject_GetBuffer(o, &b, writable ? PyBUF_CONTIG : PyBUF_CONTIG_RO) != 0) throw PyError{};
    }
    ~HostInts() { PyBuffer_Release(&b); }
    HostInts(const HostInts&) = delete;
    int n() const { return (int)(b.len / 4); }
    int32_t* p() const { return static_cast<int32_t*>(b.buf); }
};

PyObject* decimate_batch(Args& a) {
    picasso_ctx* c = a.context();
    void* s = a.stream();
    const at::Tensor &v = a.f32("verts"), &f = a.ints("facets");
    const HostInts nv_in(a.next(), false), nf_in(a.next(), false), target(a.next(), false);
    const at::Tensor *vo_ = a.maybe_f32("verts_out"), *fo_ = a.maybe_ints("facets_out"), *cid_ = a.maybe_ints("cluster_id");
    const HostInts nv_out(a.next(), true), nf_out(a.next(), true);
    picasso_stats* stats = reinterpret_cast<picasso_stats*>((intptr_t)a.integer());
    const int N = rows(v), nF = rows(f), B = nv_in.n();
    if (nf_in.n() < B || target.n() < B || nv_out.n() < B || nf_out.n() < B) fail(PyExc_ValueError, "nv_in, nf_in and target_nv differ in length");
    const at::Tensor vo = vo_ ? *vo_ : out_f32({std::max(N, 1), 3}, v), fo = fo_ ? *fo_ : out_i32({std::max(nF, 1), 3}, v),
                     cid = cid_ ? *cid_ : out_i32({std::max(N, 1)}, v);
    const int st = unlocked([&] {
        return picasso_decimate_batch(c, s, B, F(v), I(f), nv_in.p(), nf_in.p(), target.p(), F(vo), I(fo), I(cid), nv_out.p(),
                                      nf_out.p(), stats);
    });
    if (st < 0) return pack({PyLong_FromLong(st), none(), none(), none()});
    long long nv = 0, nf = 0;
    for (int b = 0; b < B; ++b) {
        nv += nv_out.p()[b];
        nf += nf_out.p()[b];
    }
    return pack({PyLong_FromLong(st), wrap(vo.narrow(0, 0, nv)), wrap(fo.narrow(0, 0, nf)), wrap(cid.narrow(0, 0, N))});
}

PyObject* cluster_csr(Args& a) {
    picasso_ctx* c = a.context();
    void* s = a.stream();
    const at::Tensor& cid = a.ints("cluster_id");
    const int n_in = rows(cid), n_out = a.i32();
    const at::Tensor off = out_i32({n_out + 1}, cid), mem = out_i32({n_in}, cid);
    checked(c, [&] { return picasso_cluster_csr(c, s, I(cid), n_in, n_out, I(off), I(mem)); });
    return pack({wrap(off), wrap(mem)});
}

PyObject* pool_forward(Args& a) {
    picasso_ctx* c = a.context();
    void* s = a.stream();
    const int mode = a.i32();
    const at::Tensor &x = a.f32("x"), &off = a.ints("offsets");
    const at::Tensor *mem = a.maybe_ints("members"), *weight = a.maybe_f32("weight");
    const bool want = a.i32() != 0;
    const int n_in = rows(x), C = rows(x, 1), n_out = rows(off) - 1;
    const at::Tensor y = out_f32({n_out, C}, x), arg = want ? out_i32({n_out, C}, x) : at::Tensor();
    checked(c, [&] { return picasso_pool_forward(c, s, mode, F(x), n_in, C, I(off), I(mem), n_out, F(weight), F(y), want ? I(arg) : nullptr); });
    return want ? pack({wrap(y), wrap(arg)}) : wrap(y);
}

PyObject* pool_backward(Args& a) {
    picasso_ctx* c = a.context();
    void* s = a.stream();
    const int mode = a.i32();
    const at::Tensor &gy = a.f32("gy"), &cid = a.ints("cluster_id"), &off = a.ints("offsets");
    const at::Tensor *mem = a.maybe_ints("members"), *weight = a.maybe_f32("weight"), *arg = a.maybe_ints("argmax");
    const int n_in = rows(cid), C = rows(gy, 1), n_out = rows(off) - 1;
    const at::Tensor gx = out_f32({n_in, C}, gy);
    checked(c, [&] { return picasso_pool_backward(c, s, mode, F(gy), n_in, C, I(cid), I(off), I(mem), n_out, F(weight), I(arg), F(gx)); });
    return wrap(gx);
}

PyObject* unpool_forward(Args& a) {
    picasso_ctx* c = a.context();
    void* s = a.stream();
    const at::Tensor &y = a.f32("y"), &cid = a.ints("cluster_id");
    const int n_in = rows(cid), C = rows(y, 1);
    const at::Tensor x = out_f32({n_in, C}, y);
    checked(c, [&] { return picasso_unpool_forward(c, s, F(y), n_in, C, I(cid), F(x)); });
    return wrap(x);
}

PyObject* unpool_backward(Args& a) {
    picasso_ctx* c = a.context();
    void* s = a.stream();
    const at::Tensor &gx = a.f32("gx"), &off = a.ints("offsets");
    const at::Tensor* mem = a.maybe_ints("members");
    const int n_in = rows(gx), C = rows(gx, 1), n_out = rows(off) - 1;
    const at::Tensor gy = out_f32({n_out, C}, gx);
    checked(c, [&] { return picasso_unpool_backward(c, s, F(gx), n_in, C, I(off), I(mem), n_out, F(gy)); });
    return wrap(gy);
}

PyObject* vertex_corner_csr(Args& a) {
    picasso_ctx* c = a.context();
    void* s = a.stream();
    const at::Tensor& f = a.ints("facets");
    const int nF = rows(f), N = a.i32();
    const at::Tensor off = out_i32({N + 1}, f), cor = out_i32({3 * (int64_t)nF}, f);
    checked(c, [&] { return picasso_vertex_corner_csr(c, s, I(f), nF, N, I(off), I(cor)); });
    return pack({wrap(off), wrap(cor)});
}

PyObject* facet_geometry(Args& a) {
    picasso_ctx* c = a.context();
    void* s = a.stream();
    const at::Tensor &v = a.f32("verts"), &f = a.ints("facets");
    PyObject* per_mesh = a.next();
    const int alpha = a.i32(), beta = a.i32(), N = rows(v), nF = rows(f);
    std::vector<int32_t> nf;
    if (per_mesh != Py_None) {
        PyObject* seq = PySequence_Fast(per_mesh, "nf: expected a sequence of integers");
        if (!seq) throw PyError{};
        Args items{PySequence_Fast_ITEMS(seq), PySequence_Fast_GET_SIZE(seq)};
        try {
            while (items.at < items.n) nf.push_back(items.i32());
        } catch (const PyError&) {
            Py_DECREF(seq);
            throw;
        }
        Py_DECREF(seq);
    }
    const at::Tensor nrm = out_f32({nF, 3}, v), area = out_f32({nF}, v), lev = out_i32({nF}, v);
    checked(c, [&] {
        return picasso_facet_geometry(c, s, F(v), N, I(f), nF, per_mesh == Py_None ? 1 : (int)nf.size(),
                                      per_mesh == Py_None ? nullptr : nf.data(), alpha, beta, F(nrm), F(area), I(lev));
    });
    return pack({wrap(nrm), wrap(area), wrap(lev)});
}

PyObject* fuzzy_coefficients(Args& a) {
    picasso_ctx* c = a.context();
    void* s = a.stream();
    const at::Tensor &nrm = a.f32("normals"), &mu = a.f32("mu");
    const at::Tensor* iv = a.maybe_f32("inv_var");
    const int nF = rows(nrm), T = rows(mu);
    const at::Tensor pi = out_f32({nF, T}, nrm);
    checked(c, [&] { return picasso_fuzzy_coefficients(c, s, F(nrm), nF, F(mu), F(iv), T, F(pi)); });
    return wrap(pi);
}

PyObject* v2f_forward(Args& a) {
    picasso_ctx* c = a.context();
    void* s = a.stream();
    const at::Tensor &x = a.f32("x"), &f = a.ints("facets");
    const at::Tensor *level = a.maybe_ints("level"), *w = a.maybe_f32("w"), *out = a.maybe_f32("y");
    const int N = rows(x), C = rows(x, 1), nF = rows(f);
    const at::Tensor y = out ? *out : out_f32({nF, C}, x);
    checked(c, [&] { return picasso_v2f_forward(c, s, F(x), N, C, I(f), nF, I(level), F(w), F(y)); });
    return wrap(y);
}

PyObject* v2f_backward(Args& a) {
    picasso_ctx* c = a.context();
    void* s = a.stream();
    const at::Tensor* gy = a.maybe_f32("gy");
    const at::Tensor &x = a.f32("x"), &f = a.ints("facets");
    const at::Tensor *level = a.maybe_ints("level"), *w = a.maybe_f32("w"), *off = a.maybe_ints("offsets"),
                     *cor = a.maybe_ints("corners");
    const int N = rows(x), C = rows(x, 1), nF = rows(f);
    const at::Tensor gx = out_f32({N, C}, x), gw = out_f32({3, C}, x);
    checked(c, [&] { return picasso_v2f_backward(c, s, F(gy), F(x), N, C, I(f), nF, I(level), F(w), I(off), I(cor), F(gx), F(gw)); });
    return pack({wrap(gx), wrap(gw)});
}

PyObject* f2f_forward(Args& a) {
    picasso_ctx* c = a.context();
    void* s = a.stream();
    const at::Tensor& tex = a.f32("tex");
    const at::Tensor* bary = a.maybe_f32("bary");
    const at::Tensor& poff = a.ints("poff");
    const at::Tensor* w = a.maybe_f32("w");
    const int P = rows(tex), C = rows(tex, 1), nF = rows(poff) - 1;
    const at::Tensor y = out_f32({nF, C}, tex);
    checked(c, [&] { return picasso_f2f_forward(c, s, F(tex), F(bary), I(poff), nF, P, C, F(w), F(y)); });
    return wrap(y);
}

PyObject* f2f_backward(Args& a) {
    picasso_ctx* c = a.context();
    void* s = a.stream();
    const at::Tensor* gy = a.maybe_f32("gy");
    const at::Tensor& tex = a.f32("tex");
    const at::Tensor* bary = a.maybe_f32("bary");
    const at::Tensor& poff = a.ints("poff");
    const at::Tensor* w = a.maybe_f32("w");
    const int P = rows(tex), C = rows(tex, 1), nF = rows(poff) - 1;
    const at::Tensor gtex = out_f32({P, C}, tex), gw = out_f32({3, C}, tex);
    // (rows of points that belong to no facet are zero; only they are written twice)
    checked(c, [&] {
        const int st = picasso_f2f_clear_unowned(c, s, I(poff), nF, P, C, F(gtex));
        return st != PICASSO_OK ? st : picasso_f2f_backward(c, s, F(gy), F(tex), F(bary), I(poff), nF, P, C, F(w), F(gtex), F(gw));
    });
    return pack({wrap(gtex), wrap(gw)});
}

PyObject* f2v_forward(Args& a) {
    picasso_ctx* c = a.context();
    void* s = a.stream();
    const at::Tensor &y = a.f32("y"), &pi = a.f32("pi");
    const at::Tensor *w = a.maybe_f32("w"), *off = a.maybe_ints("offsets"), *cor = a.maybe_ints("corners");
    const int N = a.i32();
    const at::Tensor* out = a.maybe_f32("x");
    const int nF = rows(y), C = rows(y, 1), T = rows(pi, 1);
    const at::Tensor x = out ? *out : out_f32({N, C}, y);
    checked(c, [&] { return picasso_f2v_forward(c, s, F(y), nF, C, F(pi), T, F(w), I(off), I(cor), N, F(x)); });
    return wrap(x);
}

PyObject* f2v_backward(Args& a) {
    picasso_ctx* c = a.context();
    void* s = a.stream();
    const at::Tensor &gx = a.f32("gx"), &y = a.f32("y"), &pi = a.f32("pi");
    const at::Tensor *w = a.maybe_f32("w"), *f = a.maybe_ints("facets"), *off = a.maybe_ints("offsets");
    const bool want = a.i32() != 0;
    const int nF = rows(y), C = rows(y, 1), T = rows(pi, 1), N = rows(gx);
    const at::Tensor gy = out_f32({nF, C}, y), gw = out_f32({T, C}, y), gpi = want ? out_f32({nF, T}, y) : at::Tensor();
    checked(c, [&] {
        return picasso_f2v_backward(c, s, F(gx), F(y), nF, C, F(pi), T, F(w), I(f), I(off), N, F(gy), F(gw), want ? F(gpi) : nullptr);
    });
    return pack({wrap(gy), wrap(gw), want ? wrap(gpi) : none()});
}

// ---- operators on rows of features: their tensors may be of three types, and lie on the context's device

// The call's context, device and stream (None: the device's current one).
struct Where {
    picasso_ctx* c;
    int device;
    PyObject* given;
    void* s;
    explicit Where(Args& a) : c(a.context()), device(a.i32()), given(a.next()) {
        if (given == Py_None) {
            PyObject* d = PyLong_FromLong(device);
            if (!d) throw PyError{};
            PyObject* number = PyObject_CallOneArg(g_current_stream, d);
            Py_DECREF(d);
            s = pointer(number);
            return;
        }
        // (a kernel on a stream of another device than the current one, the context's, does not run where its tensors are)
        if (attribute("device_index") != device) fail(PyExc_TypeError, "stream: expected a stream of the context's CUDA device");
        s = pointer(PyObject_GetAttrString(given, "cuda_stream"));
    }
    // A tensor that this call allocates and returns.  On a stream that the caller names it comes from that stream's memory (what the
    // current one has freed may still be in use there), and the allocator learns that the current one, the caller's, will use it.
    at::Tensor empty(at::IntArrayRef shape, at::ScalarType type) const { return allocate(shape, type, true); }
    // ... and one that only the call's kernels use.
    at::Tensor workspace(size_t bytes) const { return allocate({(int64_t)std::max<size_t>(bytes, 16)}, at::kByte, false); }

private:
    at::Tensor allocate(at::IntArrayRef shape, at::ScalarType type, bool returned) const {
        const c10::Device on(c10::DeviceType::CUDA, (c10::DeviceIndex)device);
        const auto options = at::TensorOptions().device(on).dtype(type);
        if (given == Py_None) return at::empty(shape, options);
        const c10::Stream callers = c10::impl::VirtualGuardImpl(on.type()).getStream(on);
        const c10::StreamGuard guard(c10::Stream::unpack3(attribute("stream_id"), on.index(), on.type()));
        const at::Tensor t = at::empty(shape, options);
        if (returned && callers != guard.current_stream() && t.numel()) t.record_stream(callers);
        return t;
    }
    static void* pointer(PyObject* number) {
        if (!number) throw PyError{};
        void* p = PyLong_AsVoidPtr(number);
        Py_DECREF(number);
        if (PyErr_Occurred()) throw PyError{};
        return p;
    }
    long long attribute(const char* name) const {
        PyObject* number = PyObject_GetAttrString(given, name);
        if (!number) throw PyError{};
        const long long v = PyLong_AsLongLong(number);
        Py_DECREF(number);
        if (v == -1 && PyErr_Occurred()) throw PyError{};
        return v;
    }
};

[[noreturn]] void wrong(const char* what, const char* expected) {
    PyErr_Format(PyExc_TypeError, "%s: expected %s", what, expected);
    throw PyError{};
}
int type_of(const at::Tensor& t, const char* what) {
    switch (t.scalar_type()) {
        case at::kFloat: return PICASSO_F32;
        case at::kBFloat16: return PICASSO_BF16;
        case at::kHalf: return PICASSO_F16;
        default: wrong(what, "a tensor of dtype torch.float32, torch.bfloat16 or torch.float16");
    }
}
// A tensor on the context's device, or null for None where that is allowed.
const at::Tensor* on_device(Args& a, const Where& w, const char* what, bool required) {
    PyObject* o = a.next();
    if (o == Py_None && !required) return nullptr;
    if (!THPVariable_Check(o)) wrong(what, "a CUDA tensor");
    const at::Tensor& t = THPVariable_Unpack(o);
    if (!t.is_cuda() || t.get_device() != w.device) wrong(what, "a tensor on the context's CUDA device");
    return &t;
}
// ... of this type and shape, contiguous
const at::Tensor* exactly(Args& a, const Where& w, const char* what, at::ScalarType type, at::IntArrayRef shape, bool required) {
    const at::Tensor* t = on_device(a, w, what, required);
    if (t && (t->scalar_type() != type || t->sizes() != shape || !t->is_contiguous())) {
        std::string s = "a contiguous tensor of dtype ";
        s += at::toString(type);
        s += " and shape (";
        for (int64_t n : shape) s += std::to_string(n) + ",";
        wrong(what, (s + ")").c_str());
    }
    return t;
}
// A caller's tensor that the call has written: its version is raised, as by torch's own operations in place, so that a backward pass
// that saved the old contents is refused rather than wrong.
void written(const at::Tensor& t) {
    if (!t.is_inference()) t.unsafeGetTensorImpl()->bump_version();
}
int as_i32(int64_t n, const char* what) {
    if (n > 0x7FFFFFFF) wrong(what, "less than 2^31 rows and columns");
    return (int)n;
}
double number(Args& a) {
    const double v = PyFloat_AsDouble(a.next());
    if (v == -1.0 && PyErr_Occurred()) throw PyError{};
    return v;
}

// Rows of features [N, C], contiguous.
struct Features {
    const at::Tensor& x;
    int type, N, C;
    Features(Args& a, const Where& w, const char* what) : x(*on_device(a, w, what, true)), type(type_of(x, what)) {
        if (x.dim() != 2 || !x.is_contiguous()) wrong(what, "a contiguous tensor [rows, channels]");
        N = as_i32(x.size(0), what);
        C = as_i32(x.size(1), what);
    }
};

PyObject* layer_norm_forward(Args& a) {
    const Where w(a);
    const Features f(a, w, "x");
    const at::Tensor *gamma = exactly(a, w, "gamma", at::kFloat, {f.C}, false), *beta = exactly(a, w, "beta", at::kFloat, {f.C}, false);
    const float eps = (float)number(a);
    const at::Tensor* out = exactly(a, w, "out", f.x.scalar_type(), {f.N, f.C}, false);
    const at::Tensor y = out ? *out : w.empty({f.N, f.C}, f.x.scalar_type()), mean = w.empty({f.N}, at::kFloat), rstd = w.empty({f.N}, at::kFloat);
    checked(w.c, [&] {
        return picasso_layer_norm_forward(w.c, w.s, f.type, f.x.data_ptr(), f.N, f.C, F(gamma), F(beta), eps, y.data_ptr(), F(mean), F(rstd));
    });
    if (out) written(*out);
    return pack({wrap(y), wrap(mean), wrap(rstd)});
}

PyObject* layer_norm_backward(Args& a) {
    const Where w(a);
    const at::Tensor* gy = on_device(a, w, "gy", true);
    const Features f(a, w, "x");
    if (gy->scalar_type() != f.x.scalar_type() || gy->sizes() != f.x.sizes() || !gy->is_contiguous()) wrong("gy", "a contiguous tensor of x's dtype and shape");
    const at::Tensor *gamma = exactly(a, w, "gamma", at::kFloat, {f.C}, false), *mean = exactly(a, w, "mean", at::kFloat, {f.N}, true),
                     *rstd = exactly(a, w, "rstd", at::kFloat, {f.N}, true);
    const size_t bytes = picasso_layer_norm_workspace_bytes(f.type, f.N, f.C);
    const at::Tensor gx = w.empty({f.N, f.C}, f.x.scalar_type()), gg = w.empty({f.C}, at::kFloat), gb = w.empty({f.C}, at::kFloat), ws = w.workspace(bytes);
    checked(w.c, [&] {
        return picasso_layer_norm_backward(w.c, w.s, f.type, gy->data_ptr(), f.x.data_ptr(), f.N, f.C, F(gamma), F(mean), F(rstd), gx.data_ptr(),
                                           F(gg), F(gb), ws.data_ptr(), bytes);
    });
    return pack({wrap(gx), wrap(gg), wrap(gb)});
}

// An array of heads [T, H, D], the features of a head next to each other.
struct HeadsArg {
    const at::Tensor* t;
    picasso_heads h{};
    HeadsArg(const at::Tensor* t_, const char* what) : t(t_) {
        if (!t) return;
        if (t->dim() != 3 || (t->size(2) > 1 && t->stride(2) != 1)) wrong(what, "a tensor [rows, heads, features] with its features next to each other");
        // (the strides of an axis of one are arbitrary: replaced by what fits)
        const int64_t head = t->size(1) > 1 ? t->stride(1) : t->size(2), row = t->size(0) > 1 ? t->stride(0) : std::max(t->size(1) * t->size(2), head);
        h = picasso_heads{t->data_ptr(), row, head};
    }
    HeadsArg(Args& a, const Where& w, const char* what, bool required) : HeadsArg(on_device(a, w, what, required), what) {}
};
void alike(const HeadsArg& x, const char* what, at::ScalarType type, int64_t rows, int64_t heads, int64_t width) {
    if (x.t->scalar_type() == type && x.t->size(0) == rows && x.t->size(1) == heads && x.t->size(2) == width) return;
    PyErr_Format(PyExc_TypeError, "%s: expected a tensor of dtype %s and shape (%lld, %lld, %lld)", what, at::toString(type), (long long)rows,
                 (long long)heads, (long long)width);
    throw PyError{};
}

// q, k, v, their offsets, causal and the scale, which both passes take.
struct AttentionArgs {
    HeadsArg q, k, v;
    at::ScalarType dtype;
    int type, B, Tq, Tk, Hq, Hkv, D;
    const at::Tensor *qo, *ko;
    bool causal;
    float scale;
    AttentionArgs(Args& a, const Where& w) : q(a, w, "q", true), k(a, w, "k", true), v(a, w, "v", true) {
        dtype = q.t->scalar_type();
        type = type_of(*q.t, "q");
        Tq = as_i32(q.t->size(0), "q"), Hq = as_i32(q.t->size(1), "q"), D = as_i32(q.t->size(2), "q");
        Tk = as_i32(k.t->size(0), "k"), Hkv = as_i32(k.t->size(1), "k");
        alike(k, "k", dtype, Tk, Hkv, D);
        alike(v, "v", dtype, Tk, Hkv, D);
        qo = on_device(a, w, "q_offsets", true);
        if (qo->dim() != 1 || qo->size(0) < 2) wrong("q_offsets", "a contiguous tensor [sequences + 1] of dtype torch.int32");
        B = as_i32(qo->size(0) - 1, "q_offsets");
        ko = on_device(a, w, "k_offsets", false);
        for (const at::Tensor* o : {qo, ko})
            if (o && (o->scalar_type() != at::kInt || !o->is_contiguous() || o->dim() != 1 || o->size(0) != B + 1))
                wrong(o == qo ? "q_offsets" : "k_offsets", "a contiguous tensor [sequences + 1] of dtype torch.int32");
        if (!ko) {
            if (Tq != Tk) wrong("k_offsets", "offsets of the keys, whose number is not the queries'");
            ko = qo;
        }
        causal = a.i32() != 0;
        PyObject* s = a.next();
        if (s == Py_None) {
            scale = D > 0 ? (float)(1.0 / std::sqrt((double)D)) : 0.0f;
        } else {
            scale = (float)PyFloat_AsDouble(s);
            if (PyErr_Occurred()) throw PyError{};
        }
    }
};

PyObject* attention_forward(Args& a) {
    const Where w(a);
    const AttentionArgs x(a, w);
    const HeadsArg given(a, w, "out", false);
    if (given.t) alike(given, "out", x.dtype, x.Tq, x.Hq, x.D);
    const at::Tensor o = given.t ? *given.t : w.empty({x.Tq, x.Hq, x.D}, x.dtype), lse = w.empty({x.Hq, x.Tq}, at::kFloat);
    const HeadsArg out(&o, "out");
    const size_t bytes = picasso_attention_workspace_bytes(x.type, x.B, x.Tq, x.Tk, x.Hq, x.Hkv, x.D, 0);
    const at::Tensor ws = bytes ? w.workspace(bytes) : at::Tensor();
    checked(w.c, [&] {
        // (what this call allocates has no rows to leave as they were: those of no sequence are cleared)
        return picasso_attention_forward(w.c, w.s, x.type, &x.q.h, &x.k.h, &x.v.h, I(x.qo), I(x.ko), x.B, x.Tq, x.Tk, x.Hq, x.Hkv, x.D, x.causal,
                                         x.scale, given.t == nullptr, &out.h, F(lse), bytes ? ws.data_ptr() : nullptr, bytes);
    });
    if (given.t) written(*given.t);
    return pack({wrap(o), wrap(lse)});
}

PyObject* attention_backward(Args& a) {
    const Where w(a);
    const HeadsArg gout(a, w, "gout", true);
    const AttentionArgs x(a, w);
    const HeadsArg out(a, w, "out", true);
    alike(gout, "gout", x.dtype, x.Tq, x.Hq, x.D);
    alike(out, "out", x.dtype, x.Tq, x.Hq, x.D);
    const at::Tensor* lse = exactly(a, w, "lse", at::kFloat, {x.Hq, x.Tq}, true);
    const HeadsArg to_q(a, w, "gq", false), to_k(a, w, "gk", false), to_v(a, w, "gv", false);
    const bool given = to_q.t || to_k.t || to_v.t;
    if (given && !(to_q.t && to_k.t && to_v.t)) wrong("out", "all three gradients' tensors or none");
    if (given) {
        alike(to_q, "gq", x.dtype, x.Tq, x.Hq, x.D);
        alike(to_k, "gk", x.dtype, x.Tk, x.Hkv, x.D);
        alike(to_v, "gv", x.dtype, x.Tk, x.Hkv, x.D);
    }
    const at::Tensor tq = given ? *to_q.t : w.empty({x.Tq, x.Hq, x.D}, x.dtype), tk = given ? *to_k.t : w.empty({x.Tk, x.Hkv, x.D}, x.dtype),
                     tv = given ? *to_v.t : w.empty({x.Tk, x.Hkv, x.D}, x.dtype);
    const HeadsArg gq(&tq, "gq"), gk(&tk, "gk"), gv(&tv, "gv");
    const size_t bytes = picasso_attention_workspace_bytes(x.type, x.B, x.Tq, x.Tk, x.Hq, x.Hkv, x.D, 1);
    const at::Tensor ws = w.workspace(bytes);
    checked(w.c, [&] {
        return picasso_attention_backward(w.c, w.s, x.type, &gout.h, &x.q.h, &x.k.h, &x.v.h, &out.h, F(lse), I(x.qo), I(x.ko), x.B, x.Tq, x.Tk, x.Hq,
                                          x.Hkv, x.D, x.causal, x.scale, !given, &gq.h, &gk.h, &gv.h, ws.data_ptr(), bytes);
    });
    if (given)
        for (const at::Tensor* t : {&tq, &tk, &tv}) written(*t);
    return pack({wrap(tq), wrap(tk), wrap(tv)});
}

// A sequence of contiguous tensors on the context's device, of any shapes.  They live as long as this does, until the kernels are
// queued, whatever becomes of the sequence: a generator's may have no other owner, and another thread may change a list.  (What
// is allocated meanwhile must not get their memory.)
struct Tensors {
    PyObject* held;  // a tuple: nothing changes it
    std::vector<const void*> data;
    std::vector<int64_t> sizes;
    std::vector<int32_t> types;
    Tensors(PyObject* o, const Where& w, const char* what) : held(PySequence_Tuple(o)) {
        if (!held) throw PyError{};
        try {
            const Py_ssize_t n = PyTuple_GET_SIZE(held);
            data.reserve(n), sizes.reserve(n), types.reserve(n);
            for (Py_ssize_t k = 0; k < n; ++k) {
                if (!THPVariable_Check(PyTuple_GET_ITEM(held, k))) wrong(what, "a sequence of tensors");
                const at::Tensor& t = (*this)[k];
                if (!t.is_cuda() || t.get_device() != w.device || !t.is_contiguous()) wrong(what, "contiguous tensors on the context's CUDA device");
                types.push_back(type_of(t, what));
                data.push_back(t.data_ptr());
                sizes.push_back(t.numel());
            }
        } catch (...) {
            Py_DECREF(held);
            throw;
        }
    }
    ~Tensors() { Py_DECREF(held); }
    Tensors(const Tensors&) = delete;
    const at::Tensor& operator[](Py_ssize_t k) const { return THPVariable_Unpack(PyTuple_GET_ITEM(held, k)); }
    int n() const { return (int)data.size(); }
};

PyObject* gradient_norm(Args& a) {
    const Where w(a);
    const Tensors g(a.next(), w, "grads");
    const size_t bytes = picasso_gradients_workspace_bytes(g.n(), g.sizes.data());
    const at::Tensor norm = w.empty({1}, at::kFloat), ws = w.workspace(bytes);
    checked(w.c, [&] {
        return picasso_gradient_norm(w.c, w.s, g.n(), g.data.data(), g.sizes.data(), g.types.data(), F(norm), ws.data_ptr(), bytes);
    });
    return wrap(norm);
}

PyObject* clip_gradients(Args& a) {
    const Where w(a);
    const Tensors g(a.next(), w, "grads");
    const double max_norm = number(a);
    PyObject* o = a.next();
    std::optional<Tensors> out;
    if (o != Py_None) out.emplace(o, w, "out");
    if (out && (out->sizes != g.sizes || out->types != g.types)) wrong("out", "tensors of the gradients' dtypes and sizes");
    std::vector<void*> to;
    to.reserve(g.n());
    for (const void* p : out ? out->data : g.data) to.push_back(const_cast<void*>(p));
    const size_t bytes = picasso_gradients_workspace_bytes(g.n(), g.sizes.data());
    const at::Tensor norm = w.empty({1}, at::kFloat), ws = w.workspace(bytes);
    checked(w.c, [&] {
        return picasso_clip_gradients(w.c, w.s, g.n(), g.data.data(), g.sizes.data(), g.types.data(), max_norm, to.data(), F(norm), ws.data_ptr(),
                                      bytes);
    });
    for (int k = 0; k < g.n(); ++k) written(out ? (*out)[k] : g[k]);
    return wrap(norm);
}

// (current_device, current_stream, raise): the callables above
PyObject* set_callbacks(Args& a) {
    for (PyObject** p : {&g_current_device, &g_current_stream, &g_raise}) {
        PyObject* o = a.next();
        Py_INCREF(o);
        Py_XDECREF(*p);
        *p = o;
    }
    return none();
}

#define PICASSO_ENTRY(name) {#name, (PyCFunction)(void (*)(void))(PyObject * (*)(PyObject*, PyObject* const*, Py_ssize_t)) & entry<name>, METH_FASTCALL, nullptr}
PyMethodDef methods[] = {
    PICASSO_ENTRY(decimate), PICASSO_ENTRY(decimate_batch), PICASSO_ENTRY(cluster_csr), PICASSO_ENTRY(pool_forward),
    PICASSO_ENTRY(pool_backward), PICASSO_ENTRY(unpool_forward), PICASSO_ENTRY(unpool_backward),
    PICASSO_ENTRY(vertex_corner_csr), PICASSO_ENTRY(facet_geometry), PICASSO_ENTRY(fuzzy_coefficients),
    PICASSO_ENTRY(v2f_forward), PICASSO_ENTRY(v2f_backward), PICASSO_ENTRY(f2f_forward), PICASSO_ENTRY(f2f_backward),
    PICASSO_ENTRY(f2v_forward), PICASSO_ENTRY(f2v_backward), PICASSO_ENTRY(layer_norm_forward), PICASSO_ENTRY(layer_norm_backward),
    PICASSO_ENTRY(attention_forward), PICASSO_ENTRY(attention_backward), PICASSO_ENTRY(gradient_norm), PICASSO_ENTRY(clip_gradients),
    PICASSO_ENTRY(set_callbacks), {nullptr, nullptr, 0, nullptr}};
PyModuleDef module = {PyModuleDef_HEAD_INIT, "_host", "calls of include/picasso.h on torch tensors", -1, methods, nullptr, nullptr, nullptr, nullptr};

}  // namespace

PyMODINIT_FUNC PyInit__host() { return PyModule_Create(&module); }
