// Python extension that marshals the arguments of the 8-bit path's entry points
// (include/cpdp_q8.h): sizes, row strides, storage types and addresses are read
// off torch tensors, checked, and passed on.  q8.py holds the public functions.
//
// A small call is bound by the host: reading eight tensors from Python and
// calling through ctypes took 14 us for a norm of one token, whose kernel takes
// under 4.
#define PY_SSIZE_T_CLEAN
#include <Python.h>

#include <ATen/core/TensorBase.h>
#include <ATen/ops/empty.h>
#include <c10/hip/HIPFunctions.h>
#include <c10/hip/HIPStream.h>
#include <torch/csrc/autograd/python_variable.h>

#include <exception>
#include <stdexcept>
#include <string>

#include "cpdp_q8.h"

namespace {

// A Python error that is already set.
struct Raised : std::exception {};

[[noreturn]] void refuse(const char* name, const std::string& what) {
    throw std::invalid_argument(std::string(name) + ": " + what);
}

std::string shape_of(const at::Tensor& t) {
    std::string s = "(";
    for (int64_t i = 0; i < t.dim(); ++i) s += (i ? ", " : "") + std::to_string(t.size(i));
    return s + ")";
}

const at::Tensor& tensor(PyObject* o, const char* name) {
    if (!THPVariable_Check(o)) {
        PyErr_Format(PyExc_TypeError, "%s: a tensor expected, got %s", name, Py_TYPE(o)->tp_name);
        throw Raised();
    }
    return THPVariable_Unpack(o);
}

int storage(const at::Tensor& t, const char* name) {
    if (t.scalar_type() == at::kFloat) return CPDP_F32;
    if (t.scalar_type() == at::kBFloat16) return CPDP_BF16;
    refuse(name, std::string("torch.float32 or torch.bfloat16 expected, the tensor is ") +
                     c10::toString(t.scalar_type()));
}

struct Mat {
    void* p = nullptr;
    int64_t ld = 0;
    int dt = CPDP_F32;
    int64_t rows = 0, cols = 0;
};

// The tensors of one call: all on the current GPU.
class Call {
  public:
    // a matrix of the storage type `type` (kByte: fp32 or bf16); rows, cols < 0: any
    Mat mat(PyObject* o, const char* name, at::ScalarType type, int64_t rows = -1,
            int64_t cols = -1) {
        const at::Tensor& t = tensor(o, name);
        Mat m;
        if (type == at::kByte) {
            m.dt = storage(t, name);
        } else if (t.scalar_type() != type) {
            refuse(name, std::string(c10::toString(type)) + " expected, the tensor is " +
                             c10::toString(t.scalar_type()));
        }
        if (t.dim() != 2 || (rows >= 0 && t.size(0) != rows) || (cols >= 0 && t.size(1) != cols)) {
            const auto want = [](int64_t n) { return n < 0 ? std::string("any") : std::to_string(n); };
            refuse(name, "shape (" + want(rows) + ", " + want(cols) + ") expected, the tensor is " +
                             shape_of(t));
        }
        m.rows = t.size(0);
        m.cols = t.size(1);
        if (t.stride(1) != 1 && m.cols > 1)
            refuse(name, "rows have to be dense, their elements are " +
                             std::to_string(t.stride(1)) + " apart");
        // without a second row any aligned stride does
        m.ld = m.rows > 1 ? t.stride(0) : (m.cols + 15) / 16 * 16;
        m.p = place(t, name);
        return m;
    }
    Mat maybe(PyObject* o, const char* name, at::ScalarType type, int64_t rows, int64_t cols) {
        return o == Py_None ? Mat{} : mat(o, name, type, rows, cols);
    }
    // a dense vector of n elements; dt: its storage type, null where only fp32 does
    void* vec(PyObject* o, const char* name, int64_t n, int* dt = nullptr) {
        const at::Tensor& t = tensor(o, name);
        const int code = storage(t, name);
        if (dt != nullptr) *dt = code;
        else if (code != CPDP_F32) refuse(name, "torch.float32 expected, the tensor is bfloat16");
        if (t.dim() != 1 || t.size(0) != n || (n > 1 && t.stride(0) != 1))
            refuse(name, "a dense vector of " + std::to_string(n) + " expected, the tensor is " +
                             shape_of(t));
        return place(t, name);
    }
    const int64_t* wholes(PyObject* o, const char* name, int64_t n) {
        const at::Tensor& t = tensor(o, name);
        if (t.scalar_type() != at::kLong)
            refuse(name, std::string("torch.int64 expected, the tensor is ") +
                             c10::toString(t.scalar_type()));
        if (t.dim() != 1 || t.size(0) != n || (n > 1 && t.stride(0) != 1))
            refuse(name, "a dense vector of " + std::to_string(n) + " expected, the tensor is " +
                             shape_of(t));
        return static_cast<const int64_t*>(place(t, name));
    }
    float* scales(PyObject* o, const char* name, int64_t n) {
        return static_cast<float*>(vec(o, name, n));
    }
    float* maybe_scales(PyObject* o, const char* name, int64_t n) {
        return o == Py_None ? nullptr : scales(o, name, n);
    }
    // The stream: the one given, else torch's current one.
    void* stream(PyObject* o) {
        given_ = o != Py_None;
        if (!given_) return c10::hip::getCurrentHIPStream(device_).stream();
        void* s = PyLong_AsVoidPtr(o);
        if (s == nullptr && PyErr_Occurred()) throw Raised();
        return s;
    }
    // The workspace: the tensor given, else one from torch's allocator, which ties
    // it to the current stream.  After stream().
    void* workspace(PyObject* o, int64_t need, int64_t* bytes) {
        *bytes = 0;
        if (o == Py_None) {
            if (need == 0) return nullptr;
            if (given_) refuse("workspace", "needed where a stream is given");
            scratch_ = at::empty({need}, at::TensorOptions().dtype(at::kByte).device(
                                             at::Device(at::kCUDA, device_)));
            *bytes = need;
            return scratch_.data_ptr();
        }
        const at::Tensor& t = tensor(o, "workspace");
        if (!t.is_contiguous()) refuse("workspace", "a contiguous tensor expected");
        *bytes = (int64_t)t.nbytes();
        return place(t, "workspace");
    }

  private:
    void* place(const at::Tensor& t, const char* name) {
        if (!t.is_cuda())
            refuse(name, "a tensor on the current GPU expected, this one is on " + t.device().str());
        if (device_ < 0) device_ = c10::hip::current_device();
        if (t.get_device() != device_)
            refuse(name, "a tensor on the current GPU expected, this one is on " + t.device().str());
        return t.data_ptr();
    }
    c10::DeviceIndex device_ = -1;
    bool given_ = false;
    at::Tensor scratch_;
};

constexpr at::ScalarType kEither = at::kByte;

// torch.OutOfMemoryError
PyObject* out_of_memory = nullptr;

// Runs f(arguments), with n arguments expected; no exception leaves it.
template <class F>
PyObject* entry(PyObject* const* a, Py_ssize_t got, Py_ssize_t n, F f) {
    if (got != n) {
        PyErr_Format(PyExc_TypeError, "%zd arguments expected, got %zd", n, got);
        return nullptr;
    }
    try {
        return PyLong_FromLong(f(a));
    } catch (const Raised&) {
    } catch (const std::invalid_argument& e) {
        PyErr_SetString(PyExc_ValueError, e.what());
    } catch (const c10::OutOfMemoryError& e) {
        PyErr_SetString(out_of_memory, e.what_without_backtrace());
    } catch (const std::exception& e) {
        PyErr_SetString(PyExc_RuntimeError, e.what());
    }
    return nullptr;
}

// x, q, scale, y, stream
PyObject* rows(PyObject*, PyObject* const* args, Py_ssize_t n) {
    return entry(args, n, 5, [](PyObject* const* a) {
        Call c;
        const Mat x = c.mat(a[0], "x", kEither);
        const Mat q = c.mat(a[1], "q", at::kChar, x.rows, x.cols);
        float* s = c.scales(a[2], "scale", x.rows);
        const Mat y = c.maybe(a[3], "y", kEither, x.rows, x.cols);
        return cpdp_q8_rows(x.p, x.ld, x.dt, x.rows, x.cols, static_cast<int8_t*>(q.p), q.ld, s,
                            y.p, y.ld, y.dt, c.stream(a[4]));
    });
}

// q, scale, y, stream
PyObject* values(PyObject*, PyObject* const* args, Py_ssize_t n) {
    return entry(args, n, 4, [](PyObject* const* a) {
        Call c;
        const Mat q = c.mat(a[0], "q", at::kChar);
        const float* s = c.scales(a[1], "scale", q.rows);
        const Mat y = c.mat(a[2], "y", kEither, q.rows, q.cols);
        return cpdp_q8_values(static_cast<int8_t*>(q.p), q.ld, s, q.rows, q.cols, y.p, y.ld, y.dt,
                              c.stream(a[3]));
    });
}

at::ScalarType type_of(const Mat& m) { return m.dt == CPDP_BF16 ? at::kBFloat16 : at::kFloat; }

// x, w, eps, q, scale, residual, h, rstd, y, stream
PyObject* norm(PyObject*, PyObject* const* args, Py_ssize_t n) {
    return entry(args, n, 10, [](PyObject* const* a) {
        Call c;
        const Mat x = c.mat(a[0], "x", kEither);
        const int64_t T = x.rows, D = x.cols;
        int w_dt = 0;
        const void* w = c.vec(a[1], "w", D, &w_dt);
        const double eps = PyFloat_AsDouble(a[2]);
        if (eps == -1.0 && PyErr_Occurred()) throw Raised();
        const Mat q = c.mat(a[3], "q", at::kChar, T, D);
        float* s = c.scales(a[4], "scale", T);
        const Mat r = c.maybe(a[5], "residual", type_of(x), T, D);
        const Mat h = c.maybe(a[6], "h", type_of(x), T, D);
        float* rstd = c.maybe_scales(a[7], "rstd", T);
        const Mat y = c.maybe(a[8], "y", kEither, T, D);
        return cpdp_q8_norm(x.p, x.ld, r.p, r.ld, x.dt, w, w_dt, (float)eps, T, D, h.p, h.ld,
                            static_cast<int8_t*>(q.p), q.ld, s, rstd, y.p, y.ld, y.dt,
                            c.stream(a[9]));
    });
}

// dy, h, w, rstd, dx, dw, dres, workspace, stream
PyObject* norm_bwd(PyObject*, PyObject* const* args, Py_ssize_t n) {
    return entry(args, n, 9, [](PyObject* const* a) {
        Call c;
        const Mat dy = c.mat(a[0], "dy", kEither);
        const int64_t T = dy.rows, D = dy.cols;
        const Mat h = c.mat(a[1], "h", type_of(dy), T, D);
        int w_dt = 0, dw_dt = 0;
        const void* w = c.vec(a[2], "w", D, &w_dt);
        const float* rstd = c.scales(a[3], "rstd", T);
        const Mat dx = c.mat(a[4], "dx", type_of(dy), T, D);
        void* dw = c.vec(a[5], "dw", D, &dw_dt);
        const Mat dres = c.maybe(a[6], "dres", type_of(dy), T, D);
        void* stream = c.stream(a[8]);
        int64_t bytes;
        void* ws = c.workspace(a[7], cpdp_q8_norm_bwd_workspace(T, D), &bytes);
        return cpdp_q8_norm_bwd(dy.p, dy.ld, h.p, h.ld, dres.p, dres.ld, dy.dt, w, w_dt, rstd, T, D,
                                dx.p, dx.ld, dw, dw_dt, ws, bytes, stream);
    });
}

// a, a_scale, b, b_scale, y, workspace, stream
PyObject* matmul(PyObject*, PyObject* const* args, Py_ssize_t n) {
    return entry(args, n, 7, [](PyObject* const* v) {
        Call c;
        const Mat a = c.mat(v[0], "a", at::kChar);
        const float* as = c.scales(v[1], "a_scale", a.rows);
        const Mat b = c.mat(v[2], "b", at::kChar, -1, a.cols);
        const float* bs = c.scales(v[3], "b_scale", b.rows);
        const Mat y = c.mat(v[4], "y", kEither, a.rows, b.rows);
        void* stream = c.stream(v[6]);
        int64_t bytes;
        void* ws = c.workspace(v[5], cpdp_q8_matmul_workspace(a.rows, b.rows, a.cols), &bytes);
        return cpdp_q8_matmul(static_cast<int8_t*>(a.p), a.ld, as, static_cast<int8_t*>(b.p), b.ld,
                              bs, a.rows, b.rows, a.cols, y.p, y.ld, y.dt, ws, bytes, stream);
    });
}

void same_stride(const Mat& m, const Mat& as, const char* name, const char* other) {
    if (m.p != nullptr && m.rows > 1 && m.ld != as.ld)
        refuse(name, std::string("the row stride of ") + other + ", " + std::to_string(as.ld) +
                         ", expected; it is " + std::to_string(m.ld));
}

int kind_of(PyObject* o) {
    int over = 0;
    const long k = PyLong_AsLongAndOverflow(o, &over);
    if (k == -1 && PyErr_Occurred()) throw Raised();
    if (over != 0 || k != (int)k) refuse("kind", "no activation has that number");
    return (int)k;
}

// kind, g, u, q, scale, y, cg, sg, cu, su, stream
PyObject* act(PyObject*, PyObject* const* args, Py_ssize_t n) {
    return entry(args, n, 11, [](PyObject* const* a) {
        Call c;
        const int kind = kind_of(a[0]);
        const Mat g = c.mat(a[1], "g", kEither);
        const int64_t T = g.rows, F = g.cols;
        const Mat u = c.maybe(a[2], "u", type_of(g), T, F);
        const Mat q = c.mat(a[3], "q", at::kChar, T, F);
        float* s = c.scales(a[4], "scale", T);
        const Mat y = c.maybe(a[5], "y", kEither, T, F);
        const Mat cg = c.maybe(a[6], "cg", at::kChar, T, F);
        float* sg = c.maybe_scales(a[7], "sg", T);
        const Mat cu = c.maybe(a[8], "cu", at::kChar, T, F);
        float* su = c.maybe_scales(a[9], "su", T);
        if (kind == CPDP_ACT_SWIGLU ? a[2] == Py_None
                                    : a[2] != Py_None || a[8] != Py_None || a[9] != Py_None)
            refuse("u", kind == CPDP_ACT_SWIGLU ? "swiglu takes two inputs" : "gelu takes one input");
        same_stride(u, g, "u", "g");
        same_stride(cu, cg, "cu", "cg");
        return cpdp_q8_act(kind, g.p, u.p, g.ld, g.dt, T, F, static_cast<int8_t*>(q.p), q.ld, s,
                           y.p, y.ld, y.dt, static_cast<int8_t*>(cg.p), sg,
                           static_cast<int8_t*>(cu.p), su, cg.ld, c.stream(a[10]));
    });
}

// kind, da, cg, sg, dg, cu, su, du, stream
PyObject* act_bwd(PyObject*, PyObject* const* args, Py_ssize_t n) {
    return entry(args, n, 9, [](PyObject* const* a) {
        Call c;
        const int kind = kind_of(a[0]);
        const Mat da = c.mat(a[1], "da", kEither);
        const int64_t T = da.rows, F = da.cols;
        const Mat cg = c.mat(a[2], "cg", at::kChar, T, F);
        const float* sg = c.scales(a[3], "sg", T);
        const Mat dg = c.mat(a[4], "dg", type_of(da), T, F);
        const Mat cu = c.maybe(a[5], "cu", at::kChar, T, F);
        const float* su = c.maybe_scales(a[6], "su", T);
        const Mat du = c.maybe(a[7], "du", type_of(da), T, F);
        const bool none = a[5] == Py_None && a[6] == Py_None && a[7] == Py_None;
        const bool all = a[5] != Py_None && a[6] != Py_None && a[7] != Py_None;
        if (kind == CPDP_ACT_SWIGLU ? !all : !none)
            refuse("cu", kind == CPDP_ACT_SWIGLU ? "swiglu takes cu, su and du"
                                                 : "gelu takes one input");
        same_stride(cu, cg, "cu", "cg");
        same_stride(du, dg, "du", "dg");
        return cpdp_q8_act_bwd(kind, da.p, da.ld, da.dt, static_cast<int8_t*>(cg.p), sg,
                               static_cast<int8_t*>(cu.p), su, cg.ld, T, F, dg.p, du.p, dg.ld,
                               c.stream(a[8]));
    });
}

// dy, b, b_scale, dx, workspace, stream
PyObject* grad_input(PyObject*, PyObject* const* args, Py_ssize_t n) {
    return entry(args, n, 6, [](PyObject* const* a) {
        Call c;
        const Mat dy = c.mat(a[0], "dy", kEither);
        const int64_t T = dy.rows, N = dy.cols;
        const Mat b = c.mat(a[1], "b", at::kChar, N, -1);
        const float* s = c.scales(a[2], "b_scale", N);
        const Mat dx = c.mat(a[3], "dx", kEither, T, b.cols);
        void* stream = c.stream(a[5]);
        int64_t bytes;
        void* ws = c.workspace(
            a[4], cpdp_q8_grad_input_workspace(T, N, b.cols, dy.dt, dx.dt), &bytes);
        return cpdp_q8_grad_input(dy.p, dy.ld, dy.dt, static_cast<int8_t*>(b.p), b.ld, s, T, N,
                                  b.cols, dx.p, dx.ld, dx.dt, ws, bytes, stream);
    });
}

// dy, a, a_scale, dw, workspace, stream
PyObject* grad_weight(PyObject*, PyObject* const* args, Py_ssize_t n) {
    return entry(args, n, 6, [](PyObject* const* v) {
        Call c;
        const Mat dy = c.mat(v[0], "dy", kEither);
        const int64_t T = dy.rows, N = dy.cols;
        const Mat a = c.mat(v[1], "a", at::kChar, T, -1);
        const float* s = c.scales(v[2], "a_scale", T);
        const Mat dw = c.mat(v[3], "dw", kEither, N, a.cols);
        void* stream = c.stream(v[5]);
        int64_t bytes;
        void* ws = c.workspace(
            v[4], cpdp_q8_grad_weight_workspace(T, N, a.cols, dy.dt, dw.dt), &bytes);
        return cpdp_q8_grad_weight(dy.p, dy.ld, dy.dt, static_cast<int8_t*>(a.p), a.ld, s, T, N,
                                   a.cols, dw.p, dw.ld, dw.dt, ws, bytes, stream);
    });
}

// x, x_scale, w, w_scale, target, loss, lse, miss, workspace, stream
PyObject* xent(PyObject*, PyObject* const* args, Py_ssize_t n) {
    return entry(args, n, 10, [](PyObject* const* a) {
        Call c;
        const Mat x = c.mat(a[0], "x", at::kChar);
        const int64_t T = x.rows, K = x.cols;
        const float* xs = c.scales(a[1], "x_scale", T);
        const Mat w = c.mat(a[2], "w", at::kChar, -1, K);
        const float* ws = c.scales(a[3], "w_scale", w.rows);
        const int64_t* target = c.wholes(a[4], "target", T);
        float* loss = c.scales(a[5], "loss", T);
        float* lse = c.scales(a[6], "lse", T);
        float* miss = c.maybe_scales(a[7], "miss", T);
        void* stream = c.stream(a[9]);
        int64_t bytes;
        void* room = c.workspace(a[8], cpdp_q8_xent_workspace(T, w.rows, K), &bytes);
        const auto* xq = static_cast<int8_t*>(x.p);
        const auto* wq = static_cast<int8_t*>(w.p);
        return a[7] == Py_None
                   ? cpdp_q8_xent(xq, x.ld, xs, wq, w.ld, ws, target, T, w.rows, K, loss, lse,
                                  room, bytes, stream)
                   : cpdp_q8_xent_miss(xq, x.ld, xs, wq, w.ld, ws, target, T, w.rows, K, loss, lse,
                                       miss, room, bytes, stream);
    });
}

// x, x_scale, w, w_scale, target, lse, miss, g, dx, dw, workspace, stream
PyObject* xent_bwd(PyObject*, PyObject* const* args, Py_ssize_t n) {
    return entry(args, n, 12, [](PyObject* const* a) {
        Call c;
        const Mat x = c.mat(a[0], "x", at::kChar);
        const int64_t T = x.rows, K = x.cols;
        const float* xs = c.scales(a[1], "x_scale", T);
        const Mat w = c.mat(a[2], "w", at::kChar, -1, K);
        const float* ws = c.scales(a[3], "w_scale", w.rows);
        const int64_t* target = c.wholes(a[4], "target", T);
        const float* lse = c.scales(a[5], "lse", T);
        const float* miss = c.maybe_scales(a[6], "miss", T);
        const float* g = c.scales(a[7], "g", T);
        Mat dx = c.maybe(a[8], "dx", kEither, T, K);
        Mat dw = c.maybe(a[9], "dw", kEither, w.rows, K);
        if (a[8] == Py_None && a[9] == Py_None) refuse("dx", "neither dx nor dw is given");
        if (a[8] == Py_None) dx.dt = dw.dt;
        if (a[9] == Py_None) dw.dt = dx.dt;
        void* stream = c.stream(a[11]);
        int64_t bytes;
        void* room = c.workspace(
            a[10], cpdp_q8_xent_bwd_workspace(T, w.rows, K, dx.dt, dw.dt), &bytes);
        const auto* xq = static_cast<int8_t*>(x.p);
        const auto* wq = static_cast<int8_t*>(w.p);
        return a[6] == Py_None
                   ? cpdp_q8_xent_bwd(xq, x.ld, xs, wq, w.ld, ws, target, lse, g, T, w.rows, K,
                                      dx.p, dx.ld, dx.dt, dw.p, dw.ld, dw.dt, room, bytes, stream)
                   : cpdp_q8_xent_miss_bwd(xq, x.ld, xs, wq, w.ld, ws, target, lse, miss, g, T,
                                           w.rows, K, dx.p, dx.ld, dx.dt, dw.p, dw.ld, dw.dt,
                                           room, bytes, stream);
    });
}

#define ENTRY(name)                                                                          \
    {#name, reinterpret_cast<PyCFunction>(reinterpret_cast<void (*)()>(name)), METH_FASTCALL, \
     nullptr}
PyMethodDef methods[] = {ENTRY(rows),   ENTRY(values),  ENTRY(norm),       ENTRY(norm_bwd),
                         ENTRY(matmul), ENTRY(act),     ENTRY(act_bwd),    ENTRY(grad_input),
                         ENTRY(grad_weight), ENTRY(xent), ENTRY(xent_bwd), {nullptr, nullptr, 0, nullptr}};
PyModuleDef module = {PyModuleDef_HEAD_INIT, "_q8", nullptr, -1, methods,
                      nullptr,               nullptr, nullptr, nullptr};

}  // namespace

PyMODINIT_FUNC PyInit__q8() {
    PyObject* torch = PyImport_ImportModule("torch");
    if (torch == nullptr) return nullptr;
    out_of_memory = PyObject_GetAttrString(torch, "OutOfMemoryError");
    Py_DECREF(torch);
    return out_of_memory == nullptr ? nullptr : PyModule_Create(&module);
}
