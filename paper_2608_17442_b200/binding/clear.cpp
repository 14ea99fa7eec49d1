// Binding of the operators on cleartext activations (include/fesc.h): checks tensors, fills the descriptor, hands over pointers and the current stream.
// A token's step keeps the GPU busy for three microseconds; looking at its eight tensors from Python takes ten, from here one.  Nothing is computed.
#define PY_SSIZE_T_CLEAN
#include <ATen/ops/empty.h>
#include <Python.h>
#include <c10/cuda/CUDAGuard.h>
#include <c10/cuda/CUDAStream.h>
#include <torch/csrc/autograd/python_variable.h>

#include <initializer_list>
#include <string>

#include "fesc.h"

namespace {

// the library's entry points, handed over by init(): the library is the one that the package has loaded
struct Library {
    decltype(&fesc_clear_scan) scan;
    decltype(&fesc_clear_scan_backward) scan_backward;
    decltype(&fesc_clear_scan_step) scan_step;
    decltype(&fesc_clear_norm) norm;
    decltype(&fesc_clear_norm_backward) norm_backward;
    decltype(&fesc_clear_scan_work) scan_work;
    decltype(&fesc_clear_scan_backward_work) scan_backward_work;
    decltype(&fesc_clear_norm_backward_work) norm_backward_work;
    decltype(&fesc_clear_last_error) last_error;
    decltype(&fesc_debug_bounds_register) debug_register;      // of a debug build; otherwise null
} lib;
PyObject* error_class;      // FescError(code, text)

struct Refused {
    int code;
    std::string what;
};

std::string text(at::IntArrayRef v) {
    std::string s = "(";
    for (size_t i = 0; i < v.size(); i++) s += (i ? ", " : "") + std::to_string(v[i]);
    return s + ")";
}

// One call: its name, and the device and type of the tensor that decides where it runs.
struct Call {
    const char* name;
    int device = -1;
    at::ScalarType type = at::kFloat;
    uint32_t code = 0;

    [[noreturn]] void refuse(const std::string& what) const { throw Refused{FESC_EINVAL, std::string(name) + ": " + what}; }
    const at::Tensor& tensor(const char* what, PyObject* o) const {
        if (!THPVariable_Check(o)) refuse(std::string(what) + " is not a tensor");
        return THPVariable_Unpack(o);
    }
    const at::Tensor& first(const char* what, PyObject* o, int dims) {
        const at::Tensor& t = tensor(what, o);
        if (!t.is_cuda()) refuse(std::string(what) + " is not on a CUDA device");
        device = t.get_device(), type = t.scalar_type();
        if (type == at::kBFloat16) code = FESC_BF16;
        else if (type == at::kHalf) code = FESC_F16;
        else if (type == at::kFloat) code = FESC_F32;
        else refuse(std::string(what) + " has the type " + c10::toString(type) + ": bfloat16, float16 and float32 are supported");
        if (t.dim() != dims) refuse(std::string(what) + " has " + std::to_string(t.dim()) + " dimensions, not " + std::to_string(dims));
        return t;
    }
    // Pointer of a tensor (None: null), which has to have this shape and type and to lie on the call's device.
    enum Form { DENSE, ROWS, ANY };      // contiguous; contiguous innermost dimension; any strides
    void* at(const char* what, PyObject* o, at::IntArrayRef shape, at::ScalarType t, Form form) const {
        if (o == Py_None) return nullptr;
        const at::Tensor& v = tensor(what, o);
        if (v.sizes() != shape) refuse(std::string(what) + " has the shape " + text(v.sizes()) + ", not " + text(shape));
        if (v.scalar_type() != t) refuse(std::string(what) + " has the type " + c10::toString(v.scalar_type()) + ", not " + c10::toString(t));
        if (!v.is_cuda() || v.get_device() != device) refuse(std::string(what) + " is on another device than the first tensor");
        if (form == DENSE ? !v.is_contiguous() : form == ROWS && shape.back() > 1 && v.strides().back() != 1)
            refuse(std::string(what) + (form == DENSE ? " is not contiguous" : ": the innermost dimension is not contiguous"));
        void* p = v.data_ptr();
        if (lib.debug_register && v.numel()) {
            int64_t span = 1;
            for (int64_t i = 0; i < v.dim(); i++) span += (v.size(i) - 1) * v.stride(i);
            lib.debug_register(p, span * v.element_size());
        }
        return p;
    }
    void* rows(const char* what, PyObject* o, at::IntArrayRef shape) const { return at(what, o, shape, type, ROWS); }
    float* f32(const char* what, PyObject* o, at::IntArrayRef shape, Form form = DENSE) const { return (float*)at(what, o, shape, at::kFloat, form); }

    // a workspace: the caller's, or one of torch's allocator (on the stream that is current, where the call runs)
    struct Work {
        at::Tensor t;
        void* p = nullptr;
        size_t bytes = 0;
    };
    Work work(PyObject* o, size_t need) const {
        Work w;
        if (o != Py_None) {
            w.t = tensor("work", o);
            if (!w.t.is_cuda() || w.t.get_device() != device || !w.t.is_contiguous()) refuse("the workspace is not contiguous, or on another device");
        } else if (need) {
            w.t = at::empty({(int64_t)need}, at::TensorOptions(at::kByte).device(at::kCUDA, device));
        } else {
            return w;
        }
        w.p = w.t.data_ptr(), w.bytes = w.t.numel() * w.t.element_size();
        if (lib.debug_register && w.bytes) lib.debug_register(w.p, w.bytes);
        return w;
    }
    // what the call has written counts as changed in place: autograd refuses gradients that would need the values before
    void wrote(std::initializer_list<PyObject*> list) const {
        for (PyObject* o : list)
            if (o != Py_None) {
                const at::Tensor& t = THPVariable_Unpack(o);
                if (!t.is_inference()) t.unsafeGetTensorImpl()->bump_version();
            }
    }
    void* stream() const { return c10::cuda::getCurrentCUDAStream(device).stream(); }
    void done(int rc) const {
        if (rc != FESC_OK) throw Refused{rc, lib.last_error()};
    }
};

// strides of batch, token and head of a [batch, L, H, ...] tensor, or of batch and head of a [batch, H, ...] one; 0 where there is one of them
void steps(int64_t (&s)[3], PyObject* o, bool tokens) {
    if (o == Py_None) return;
    const at::Tensor& t = THPVariable_Unpack(o);
    auto of = [&](int i) { return t.size(i) > 1 ? t.stride(i) : 0; };
    s[0] = of(0), s[1] = tokens ? of(1) : 0, s[2] = of(tokens ? 2 : 1);
}

struct ScanSizes {
    int64_t b, L, H, P, G, N;
    fesc_clear_scan_desc d = {};
};
ScanSizes scan_sizes(Call& call, PyObject* ox, PyObject* oB, bool tokens) {
    const at::Tensor& x = call.first("x", ox, tokens ? 4 : 3);
    const at::Tensor& B = call.tensor("B", oB);
    if (B.dim() != x.dim()) call.refuse("B has " + std::to_string(B.dim()) + " dimensions, not " + std::to_string(x.dim()));
    const int h = tokens ? 2 : 1;
    ScanSizes s = {x.size(0), tokens ? x.size(1) : 1, x.size(h), x.size(h + 1), B.size(h), B.size(h + 1)};
    const int64_t most = UINT32_MAX;
    if (s.b > most || s.L > most || s.H > most || s.P > most || s.G > most || s.N > most) call.refuse("a dimension is beyond 32 bits");
    s.d.batch = s.b, s.d.L = s.L, s.d.H = s.H, s.d.P = s.P, s.d.G = s.G, s.d.N = s.N, s.d.type = call.code;
    return s;
}

// Runs a call's body with `count` positional arguments; what it throws becomes a Python exception.
template <class F>
PyObject* run(PyObject* const* args, Py_ssize_t n, Py_ssize_t count, F body) {
    if (n != count) {
        PyErr_Format(PyExc_TypeError, "%zd arguments, not %zd", n, count);
        return nullptr;
    }
    try {
        body(args);
        Py_RETURN_NONE;
    } catch (const Refused& r) {
        PyObject* e = PyObject_CallFunction(error_class, "is", r.code, r.what.c_str());
        if (e) PyErr_SetObject(error_class, e), Py_DECREF(e);
    } catch (const c10::OutOfMemoryError& e) {      // of the workspace
        PyObject* torch = PyImport_ImportModule("torch");
        PyObject* type = torch ? PyObject_GetAttrString(torch, "OutOfMemoryError") : nullptr;
        if (type) PyErr_SetString(type, e.what_without_backtrace());
        Py_XDECREF(type), Py_XDECREF(torch);
    } catch (const std::exception& e) {
        PyErr_SetString(PyExc_RuntimeError, e.what());
    }
    return nullptr;
}

PyObject* clear_scan(PyObject*, PyObject* const* args, Py_ssize_t n) {      // x g B C y skip h0 h_out lengths work
    return run(args, n, 10, [](PyObject* const* a) {
        Call c{"clear_scan"};
        ScanSizes s = scan_sizes(c, a[0], a[2], true);
        const int64_t rows[] = {s.b, s.L, s.H, s.P}, cols[] = {s.b, s.L, s.G, s.N}, st[] = {s.b, s.H, s.P, s.N}, heads[] = {s.H}, all[] = {s.b};
        const c10::cuda::OptionalCUDAGuard guard(c10::Device(c10::kCUDA, c.device));
        void *x = c.rows("x", a[0], rows), *B = c.rows("B", a[2], cols), *C = c.rows("C", a[3], cols), *y = c.rows("y", a[4], rows);
        float *g = c.f32("g", a[1], {rows, 3}, Call::ANY), *skip = c.f32("skip", a[5], heads), *h0 = c.f32("h0", a[6], st), *h = c.f32("h_out", a[7], st);
        auto* len = (const int32_t*)c.at("lengths", a[8], all, at::kInt, Call::DENSE);
        steps(s.d.x, a[0], true), steps(s.d.y, a[4], true), steps(s.d.g, a[1], true), steps(s.d.B, a[2], true), steps(s.d.C, a[3], true);
        const Call::Work w = c.work(a[9], lib.scan_work(&s.d));
        c.done(lib.scan(&s.d, x, g, B, C, skip, h0, len, y, h, w.p, w.bytes, c.stream()));
        c.wrote({a[4], a[7], a[9]});
    });
}

PyObject* clear_scan_backward(PyObject*, PyObject* const* args, Py_ssize_t n) {      // x g B C dy dx dg dB dC skip dskip h0 dh_out dh0 lengths work
    return run(args, n, 16, [](PyObject* const* a) {
        Call c{"clear_scan_backward"};
        ScanSizes s = scan_sizes(c, a[0], a[2], true);
        const int64_t rows[] = {s.b, s.L, s.H, s.P}, cols[] = {s.b, s.L, s.G, s.N}, st[] = {s.b, s.H, s.P, s.N}, heads[] = {s.H}, all[] = {s.b};
        const c10::cuda::OptionalCUDAGuard guard(c10::Device(c10::kCUDA, c.device));
        void *x = c.rows("x", a[0], rows), *B = c.rows("B", a[2], cols), *C = c.rows("C", a[3], cols), *dy = c.rows("dy", a[4], rows), *dx = c.rows("dx", a[5], rows),
             *dB = c.rows("dB", a[7], cols), *dC = c.rows("dC", a[8], cols);
        float *g = c.f32("g", a[1], {rows, 3}, Call::ANY), *dg = c.f32("dg", a[6], {rows, 3}, Call::ANY), *skip = c.f32("skip", a[9], heads),
              *dskip = c.f32("dskip", a[10], heads), *h0 = c.f32("h0", a[11], st), *dh = c.f32("dh_out", a[12], st), *dh0 = c.f32("dh0", a[13], st);
        auto* len = (const int32_t*)c.at("lengths", a[14], all, at::kInt, Call::DENSE);
        steps(s.d.x, a[0], true), steps(s.d.y, a[4], true), steps(s.d.g, a[1], true), steps(s.d.B, a[2], true), steps(s.d.C, a[3], true);
        steps(s.d.dx, a[5], true), steps(s.d.dg, a[6], true), steps(s.d.dB, a[7], true), steps(s.d.dC, a[8], true);
        const Call::Work w = c.work(a[15], lib.scan_backward_work(&s.d));
        c.done(lib.scan_backward(&s.d, x, g, B, C, skip, h0, len, dy, dh, dx, dg, dB, dC, dskip, dh0, w.p, w.bytes, c.stream()));
        c.wrote({a[5], a[6], a[7], a[8], a[10], a[13], a[15]});
    });
}

PyObject* clear_scan_step(PyObject*, PyObject* const* args, Py_ssize_t n) {      // x g B C state y skip state_out
    return run(args, n, 8, [](PyObject* const* a) {
        Call c{"clear_scan_step"};
        ScanSizes s = scan_sizes(c, a[0], a[2], false);
        const int64_t rows[] = {s.b, s.H, s.P}, cols[] = {s.b, s.G, s.N}, st[] = {s.b, s.H, s.P, s.N}, heads[] = {s.H};
        const c10::cuda::OptionalCUDAGuard guard(c10::Device(c10::kCUDA, c.device));
        void *x = c.rows("x", a[0], rows), *B = c.rows("B", a[2], cols), *C = c.rows("C", a[3], cols), *y = c.rows("y", a[5], rows);
        float *g = c.f32("g", a[1], {rows, 2}, Call::ANY), *h = c.f32("state", a[4], st), *skip = c.f32("skip", a[6], heads),
              *to = a[7] == Py_None ? h : c.f32("state_out", a[7], st);
        steps(s.d.x, a[0], false), steps(s.d.y, a[5], false), steps(s.d.g, a[1], false), steps(s.d.B, a[2], false), steps(s.d.C, a[3], false);
        c.done(lib.scan_step(&s.d, x, g, B, C, skip, h, to, y, c.stream()));
        c.wrote({a[5], a[7] == Py_None ? a[4] : a[7]});
    });
}

struct NormSizes {
    int64_t shape[2];
    fesc_clear_norm_desc d = {};
};
NormSizes norm_sizes(Call& call, PyObject* y, PyObject* eps, PyObject* groups) {
    const at::Tensor& t = call.first("y", y, 2);
    NormSizes s = {{t.size(0), t.size(1)}};
    const double e = PyFloat_AsDouble(eps);
    const long long g = PyLong_AsLongLong(groups);
    if (PyErr_Occurred()) {
        PyErr_Clear();
        call.refuse("eps is a number, groups a whole number");
    }
    if (s.shape[1] > (int64_t)UINT32_MAX || g < 0 || g > (long long)UINT32_MAX) call.refuse("a dimension is beyond 32 bits");
    s.d.rows = s.shape[0], s.d.d = s.shape[1], s.d.groups = g, s.d.type = call.code, s.d.eps = (float)e;
    return s;
}
int64_t step(PyObject* o) {      // between rows
    if (o == Py_None) return 0;
    const at::Tensor& t = THPVariable_Unpack(o);
    return t.size(0) > 1 ? t.stride(0) : 0;
}

PyObject* clear_norm(PyObject*, PyObject* const* args, Py_ssize_t n) {      // y gamma n eps gate residual scale h groups
    return run(args, n, 9, [](PyObject* const* a) {
        Call c{"clear_norm"};
        NormSizes s = norm_sizes(c, a[0], a[3], a[8]);
        const c10::cuda::OptionalCUDAGuard guard(c10::Device(c10::kCUDA, c.device));
        const at::IntArrayRef d(s.shape + 1, 1);
        void *y = c.rows("y", a[0], s.shape), *out = c.rows("n", a[2], s.shape), *z = c.rows("gate", a[4], s.shape), *r = c.rows("residual", a[5], s.shape),
             *h = c.rows("h", a[7], s.shape);
        float *gamma = c.f32("gamma", a[1], d), *scale = c.f32("scale", a[6], d);
        s.d.y_stride = step(a[0]), s.d.n_stride = step(a[2]), s.d.gate_stride = step(a[4]), s.d.residual_stride = step(a[5]), s.d.h_stride = step(a[7]);
        c.done(lib.norm(&s.d, y, gamma, z, r, scale, out, h, c.stream()));
        c.wrote({a[2], a[7]});
    });
}

PyObject* clear_norm_backward(PyObject*, PyObject* const* args, Py_ssize_t n) {      // y gamma dn dy dgamma eps gate dgate residual dresidual scale dscale dh groups work
    return run(args, n, 15, [](PyObject* const* a) {
        Call c{"clear_norm_backward"};
        NormSizes s = norm_sizes(c, a[0], a[5], a[13]);
        const c10::cuda::OptionalCUDAGuard guard(c10::Device(c10::kCUDA, c.device));
        const at::IntArrayRef d(s.shape + 1, 1);
        void *y = c.rows("y", a[0], s.shape), *dn = c.rows("dn", a[2], s.shape), *dy = c.rows("dy", a[3], s.shape), *z = c.rows("gate", a[6], s.shape),
             *dz = c.rows("dgate", a[7], s.shape), *r = c.rows("residual", a[8], s.shape), *dr = c.rows("dresidual", a[9], s.shape), *dh = c.rows("dh", a[12], s.shape);
        float *gamma = c.f32("gamma", a[1], d), *dgamma = c.f32("dgamma", a[4], d), *scale = c.f32("scale", a[10], d), *dscale = c.f32("dscale", a[11], d);
        s.d.y_stride = step(a[0]), s.d.dn_stride = step(a[2]), s.d.dy_stride = step(a[3]), s.d.gate_stride = step(a[6]), s.d.dgate_stride = step(a[7]);
        s.d.residual_stride = step(a[8]), s.d.dresidual_stride = step(a[9]), s.d.dh_stride = step(a[12]);
        const Call::Work w = c.work(a[14], lib.norm_backward_work(&s.d));
        c.done(lib.norm_backward(&s.d, y, gamma, z, r, scale, dn, dh, dy, dgamma, dz, dr, dscale, w.p, w.bytes, c.stream()));
        c.wrote({a[3], a[4], a[7], a[9], a[11], a[14]});
    });
}

// init(FescError, addresses of the entry points in the order of Library)
PyObject* init(PyObject*, PyObject* const* args, Py_ssize_t n) {
    if (n != 11) {
        PyErr_SetString(PyExc_TypeError, "FescError and ten addresses");
        return nullptr;
    }
    void* p[10];
    for (int i = 0; i < 10; i++) p[i] = PyLong_AsVoidPtr(args[i + 1]);
    if (PyErr_Occurred()) return nullptr;
    static_assert(sizeof(lib) == sizeof(p), "one address each");
    memcpy(&lib, p, sizeof(p));
    Py_INCREF(args[0]);
    Py_XDECREF(error_class);
    error_class = args[0];
    Py_RETURN_NONE;
}

#define FAST(f) {#f, (PyCFunction)(void (*)(void))f, METH_FASTCALL, nullptr}
PyMethodDef methods[] = {FAST(init), FAST(clear_scan), FAST(clear_scan_backward), FAST(clear_scan_step), FAST(clear_norm), FAST(clear_norm_backward), {}};
PyModuleDef module = {PyModuleDef_HEAD_INIT, "_clear", nullptr, -1, methods};

}  // namespace

PyMODINIT_FUNC PyInit__clear(void) { return PyModule_Create(&module); }
