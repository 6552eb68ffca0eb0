// The hot half of the operators' binding (ops.py): plain tensors on the current GPU, straight to the C calls.  A call that has
// anything else among its arguments returns None, and the other half, which raises every error of marshalling, makes it.
//
// On small tensors the host decides: layer norm of 197 x 768 takes 9.5 us a call through ctypes and 3.6 here, attention's forward pass over 16
// queries and keys 10.1 and 5.8.
#define PY_SSIZE_T_CLEAN
#include <Python.h>
#include <ATen/ATen.h>
#include <ATen/PythonTorchFunctionTLS.h>
#include <torch/csrc/autograd/python_variable.h>

#include <cmath>
#include <optional>

#include "kt_ops.h"

namespace {

PyObject *get_device, *get_stream, *cuda_stream;        // of kt_marshal.cpp

struct Entries {
    decltype(&kt_layernorm_fwd) layernorm_fwd;
    decltype(&kt_layernorm_bwd_workspace) layernorm_bwd_workspace;
    decltype(&kt_layernorm_bwd) layernorm_bwd;
    decltype(&kt_act8_save) act8_save;
    decltype(&kt_act8_restore) act8_restore;
    decltype(&kt_act8_weight_grad_workspace) weight_grad_workspace;
    decltype(&kt_act8_weight_grad) weight_grad;
    decltype(&kt_attention_fwd) attention_fwd;
    decltype(&kt_attention_bwd_workspace) attention_bwd_workspace;
    decltype(&kt_attention_bwd) attention_bwd;
};
constexpr int ENTRIES = sizeof(Entries) / sizeof(void *);

struct Ops {
    PyObject_HEAD
    Entries f;
};

// What one call has converted; `ok` turns false at the first form that is not taken here, and no Python error is left set.
struct Args {
    bool ok = true;
    long device = -1;
    void *stream = nullptr;
    bool own_stream = false;            // not torch's current one
    std::optional<at::Tensor> scratch;  // taken for the call

    explicit Args(PyObject *on)
    {
        PyObject *dev = PyObject_CallNoArgs(get_device);
        device = dev ? PyLong_AsLong(dev) : -1;
        PyObject *raw = nullptr;
        if (dev && on == Py_None) {
            raw = PyObject_CallOneArg(get_stream, dev);
        } else if (dev) {
            own_stream = true;
            raw = PyLong_Check(on) ? Py_NewRef(on) : PyObject_GetAttr(on, cuda_stream);
        }
        stream = raw && PyLong_Check(raw) ? PyLong_AsVoidPtr(raw) : (ok = false, nullptr);
        Py_XDECREF(raw);
        Py_XDECREF(dev);
        if (PyErr_Occurred() || at::impl::torch_function_mode_enabled()) fail();
    }
    bool fail()
    {
        PyErr_Clear();
        return ok = false;
    }
    // a tensor of torch's own class on the current GPU; only read while `ok`
    const at::Tensor &tensor(PyObject *x)
    {
        static const at::Tensor none;
        if (!ok || !THPVariable_CheckExact(x)) return fail(), none;
        const at::Tensor &t = THPVariable_Unpack(x);
        if (!t.defined() || !t.is_cuda() || t.layout() != at::kStrided || t.device().index() != device) return fail(), none;
        return t;
    }
    kt_dtype type(const at::Tensor &t)
    {
        if (!ok) return KT_F32;
        if (t.scalar_type() == at::kFloat) return KT_F32;
        if (t.scalar_type() == at::kBFloat16) return KT_BF16;
        return fail(), KT_F32;
    }
    // what has as many elements in memory, one after another; nullptr for None
    void *vector(PyObject *x, int64_t n, at::ScalarType type)
    {
        if (x == Py_None) return nullptr;
        const at::Tensor &t = tensor(x);
        if (!ok || t.scalar_type() != type || t.numel() != n || !t.is_contiguous()) return fail(), nullptr;
        return t.data_ptr();
    }
    double real(PyObject *x)
    {
        if (!ok) return 0;
        const double v = PyFloat_AsDouble(x);
        if (PyErr_Occurred()) fail();
        return v;
    }
    // address and size of the scratch memory that a call needs
    void *workspace(PyObject *given, int64_t need, int64_t *size)
    {
        *size = 0;
        if (!ok) return nullptr;
        if (given != Py_None) {
            const at::Tensor &t = tensor(given);
            if (!ok || !t.is_contiguous()) return fail(), nullptr;
            *size = t.numel() * (int64_t)t.element_size();
            return t.data_ptr();
        }
        if (need == 0) return nullptr;
        if (own_stream) return fail(), nullptr;         // memory of that stream: left to the other half
        scratch = at::empty({need}, at::TensorOptions().dtype(at::kByte).device(at::Device(at::kCUDA, (at::DeviceIndex)device)));
        *size = need;
        return scratch->data_ptr();
    }
};

struct Matrix {
    void *p = nullptr;
    int64_t rows = 0, cols = 0, ld = 0;
    kt_dtype type = KT_F32;
    at::ScalarType scalar = at::kFloat;
    Matrix(Args &x, PyObject *o)
    {
        const at::Tensor &t = x.tensor(o);
        if (!x.ok) return;
        type = x.type(t);
        scalar = t.scalar_type();
        const int64_t d = t.dim();
        if (d < 1) { x.fail(); return; }
        cols = t.size(d - 1);
        if (d == 2) {
            rows = t.size(0);
            if (cols > 1 && t.stride(1) != 1) { x.fail(); return; }
            ld = rows > 1 ? t.stride(0) : cols;
        } else {
            if (!t.is_contiguous() || cols < 1) { x.fail(); return; }
            rows = t.numel() / cols;
            ld = cols;
        }
        p = t.data_ptr();
    }
    void like(Args &x, const Matrix &m) const
    {
        if (x.ok && (rows != m.rows || cols != m.cols || scalar != m.scalar)) x.fail();
    }
};

// The two parts of a checkpoint of [rows, cols].
struct Act8 {
    int8_t *q = nullptr;
    uint8_t *e = nullptr;
    Act8(Args &x, PyObject *oq, PyObject *oe, int64_t rows, int64_t cols)
    {
        const int64_t groups = (cols + 31) / 32;
        if (!x.ok || oq == Py_None || oe == Py_None) { x.fail(); return; }
        q = static_cast<int8_t *>(x.vector(oq, rows * groups * 32, at::kChar));
        e = static_cast<uint8_t *>(x.vector(oe, rows * groups, at::kByte));
    }
};
// (q, e) as a tuple
bool is_pair(PyObject *o) { return PyTuple_CheckExact(o) && PyTuple_GET_SIZE(o) == 2; }

struct Heads : kt_heads {
    int64_t size[4] = {0, 0, 0, 0};
    at::ScalarType scalar = at::kFloat;
    Heads(Args &x, PyObject *o) : kt_heads{nullptr, 0, 0, 0}
    {
        const at::Tensor &t = x.tensor(o);
        if (!x.ok) return;
        if (t.dim() != 4 || (t.size(3) > 1 && t.stride(3) != 1)) { x.fail(); return; }
        data = t.data_ptr();
        batch = t.stride(0);
        token = t.stride(1);
        head = t.stride(2);
        scalar = t.scalar_type();
        for (int i = 0; i < 4; ++i) size[i] = t.size(i);
    }
    void like(Args &x, const Heads &h) const
    {
        for (int i = 0; i < 4; ++i)
            if (size[i] != h.size[i]) x.fail();
        if (scalar != h.scalar) x.fail();
    }
};

struct Attention : kt_attention {
    Attention(Args &x, const Heads &q, const Heads &k, PyObject *causal_, PyObject *scale_, PyObject *lens) : kt_attention{}
    {
        if (!x.ok) return;
        if (q.scalar != k.scalar || q.size[0] != k.size[0] || q.size[3] != k.size[3] || q.size[3] < 1) { x.fail(); return; }
        if (q.scalar == at::kFloat) dt = KT_F32;
        else if (q.scalar == at::kBFloat16) dt = KT_BF16;
        else { x.fail(); return; }
        batch = q.size[0];
        nq = q.size[1];
        nk = k.size[1];
        heads = q.size[2];
        kv_heads = k.size[2];
        dim = q.size[3];
        scale = scale_ == Py_None ? (float)std::pow((double)dim, -0.5) : (float)x.real(scale_);
        const int c = PyObject_IsTrue(causal_);
        if (c < 0) x.fail();
        causal = c > 0;
        k_lens = static_cast<const int32_t *>(x.vector(lens, batch, at::kInt));
    }
};

// The call itself without the interpreter lock, as ctypes makes it.
template <typename F> PyObject *finish(Args &x, F call)
{
    if (!x.ok) Py_RETURN_NONE;
    kt_status st;
    Py_BEGIN_ALLOW_THREADS
    st = call();
    Py_END_ALLOW_THREADS
    return PyLong_FromLong((long)st);
}

#define KT_OP(name, count)                                                                               \
    PyObject *name##_(const Entries &f, PyObject *const *a, Args &x);                                     \
    PyObject *name(PyObject *self, PyObject *const *a, Py_ssize_t n)                                     \
    {                                                                                                    \
        if (n != count) { PyErr_SetString(PyExc_TypeError, #name ": needs " #count " arguments"); return nullptr; } \
        try {                                                                                            \
            Args x(a[n - 1]);                                                                            \
            return name##_(reinterpret_cast<Ops *>(self)->f, a, x);                                      \
        } catch (...) { /* a tensor without memory, or none left: asked again through Python, which raises its own error */ \
            PyErr_Clear();                                                                               \
            Py_RETURN_NONE;                                                                              \
        }                                                                                                \
    }                                                                                                    \
    PyObject *name##_(const Entries &f, PyObject *const *a, Args &x)

// x, gamma, beta, eps, y, mean, rstd, y8, stream
KT_OP(layernorm_fwd, 9)
{
    const Matrix in(x, a[0]), out(x, a[4]);
    out.like(x, in);
    const at::Tensor &g = x.tensor(a[1]);
    const kt_dtype pdt = x.type(g);
    if (!x.ok) Py_RETURN_NONE;
    void *gamma = x.vector(a[1], in.cols, g.scalar_type()), *beta = x.vector(a[2], in.cols, g.scalar_type());
    const float eps = (float)x.real(a[3]);
    float *mean = static_cast<float *>(x.vector(a[5], in.rows, at::kFloat)), *rstd = static_cast<float *>(x.vector(a[6], in.rows, at::kFloat));
    int8_t *q = nullptr;
    uint8_t *e = nullptr;
    if (a[7] != Py_None) {
        if (!is_pair(a[7])) Py_RETURN_NONE;
        const Act8 c(x, PyTuple_GET_ITEM(a[7], 0), PyTuple_GET_ITEM(a[7], 1), in.rows, in.cols);
        q = c.q;
        e = c.e;
    }
    return finish(x, [&] { return f.layernorm_fwd(in.type, pdt, in.rows, in.cols, in.p, in.ld, gamma, beta, eps, out.p, out.ld, mean, rstd, q, e, x.stream); });
}

// dy, x, gamma, mean, rstd, dx, dgamma, dbeta, workspace, stream
KT_OP(layernorm_bwd, 10)
{
    const Matrix dy(x, a[0]), dx(x, a[5]);
    dx.like(x, dy);
    const at::Tensor &g = x.tensor(a[2]);
    const kt_dtype pdt = x.type(g);
    if (!x.ok) Py_RETURN_NONE;
    void *in = nullptr;
    int64_t ldx = 0, size;
    int8_t *q = nullptr;
    uint8_t *e = nullptr;
    if (is_pair(a[1])) {
        const Act8 c(x, PyTuple_GET_ITEM(a[1], 0), PyTuple_GET_ITEM(a[1], 1), dy.rows, dy.cols);
        q = c.q;
        e = c.e;
    } else {
        const Matrix m(x, a[1]);
        m.like(x, dy);
        in = m.p;
        ldx = m.ld;
    }
    void *gamma = x.vector(a[2], dy.cols, g.scalar_type());
    const float *mean = static_cast<float *>(x.vector(a[3], dy.rows, at::kFloat)), *rstd = static_cast<float *>(x.vector(a[4], dy.rows, at::kFloat));
    void *dgamma = x.vector(a[6], dy.cols, g.scalar_type()), *dbeta = x.vector(a[7], dy.cols, g.scalar_type());
    void *ws = x.workspace(a[8], f.layernorm_bwd_workspace(dy.rows, dy.cols), &size);
    return finish(x, [&] {
        return f.layernorm_bwd(dy.type, pdt, dy.rows, dy.cols, dy.p, dy.ld, in, ldx, q, e, gamma, mean, rstd, dx.p, dx.ld, dgamma, dbeta, ws, size, x.stream);
    });
}

// x, q, e, stream
KT_OP(act8_save, 4)
{
    const Matrix in(x, a[0]);
    const Act8 c(x, a[1], a[2], in.rows, in.cols);
    return finish(x, [&] { return f.act8_save(in.type, in.rows, in.cols, in.p, in.ld, c.q, c.e, x.stream); });
}

// q, e, y, stream
KT_OP(act8_restore, 4)
{
    const Matrix out(x, a[2]);
    const Act8 c(x, a[0], a[1], out.rows, out.cols);
    return finish(x, [&] { return f.act8_restore(out.type, out.rows, out.cols, c.q, c.e, out.p, out.ld, x.stream); });
}

// dy, q, e, dw, workspace, stream
KT_OP(act8_weight_grad, 6)
{
    const Matrix dy(x, a[0]), dw(x, a[3]);
    if (x.ok && dw.rows != dy.cols) x.fail();
    const Act8 c(x, a[1], a[2], dy.rows, dw.cols);
    int64_t size;
    if (!x.ok) Py_RETURN_NONE;
    void *ws = x.workspace(a[4], f.weight_grad_workspace(dy.type, dy.rows, dy.cols, dw.cols), &size);
    return finish(x, [&] { return f.weight_grad(dy.type, dw.type, dy.rows, dy.cols, dw.cols, dy.p, dy.ld, c.q, c.e, dw.p, dw.ld, ws, size, x.stream); });
}

// q, k, v, o, lse, causal, scale, k_lens, stream
KT_OP(attention_fwd, 9)
{
    const Heads q(x, a[0]), k(x, a[1]), v(x, a[2]), o(x, a[3]);
    v.like(x, k);
    o.like(x, q);
    const Attention s(x, q, k, a[5], a[6], a[7]);
    float *lse = static_cast<float *>(x.vector(a[4], q.size[0] * q.size[1] * q.size[2], at::kFloat));
    return finish(x, [&] { return f.attention_fwd(&s, &q, &k, &v, &o, lse, x.stream); });
}

// do, q, k, v, o, lse, dq, dk, dv, causal, scale, k_lens, workspace, stream
KT_OP(attention_bwd, 14)
{
    const Heads d(x, a[0]), q(x, a[1]), k(x, a[2]), v(x, a[3]), o(x, a[4]), dq(x, a[6]), dk(x, a[7]), dv(x, a[8]);
    for (const Heads *h : {&d, &o, &dq}) h->like(x, q);
    for (const Heads *h : {&v, &dk, &dv}) h->like(x, k);
    const Attention s(x, q, k, a[9], a[10], a[11]);
    const float *lse = static_cast<float *>(x.vector(a[5], q.size[0] * q.size[1] * q.size[2], at::kFloat));
    int64_t size;
    if (!x.ok) Py_RETURN_NONE;
    void *ws = x.workspace(a[12], f.attention_bwd_workspace(&s), &size);
    return finish(x, [&] { return f.attention_bwd(&s, &d, &q, &k, &v, &o, lse, &dq, &dk, &dv, ws, size, x.stream); });
}

#define KT_METHOD(name) {#name, reinterpret_cast<PyCFunction>(reinterpret_cast<void *>(name)), METH_FASTCALL, nullptr}
PyMethodDef methods[] = {KT_METHOD(layernorm_fwd), KT_METHOD(layernorm_bwd), KT_METHOD(act8_save), KT_METHOD(act8_restore),
                         KT_METHOD(act8_weight_grad), KT_METHOD(attention_fwd), KT_METHOD(attention_bwd), {nullptr, nullptr, 0, nullptr}};

// Ops(addresses of the entry points, in the order of Entries)
PyObject *ops_new(PyTypeObject *type, PyObject *args, PyObject *)
{
    if (PyTuple_GET_SIZE(args) != ENTRIES) { PyErr_SetString(PyExc_TypeError, "Ops: needs the address of every entry point"); return nullptr; }
    void *v[ENTRIES];
    for (int i = 0; i < ENTRIES; ++i) {
        v[i] = PyLong_AsVoidPtr(PyTuple_GET_ITEM(args, i));
        if (PyErr_Occurred()) return nullptr;
    }
    Ops *o = reinterpret_cast<Ops *>(type->tp_alloc(type, 0));
    if (o) memcpy(&o->f, v, sizeof v);
    return reinterpret_cast<PyObject *>(o);
}

PyTypeObject ops_type = {PyVarObject_HEAD_INIT(nullptr, 0)};

}  // namespace

// Adds the type Ops to the module.
bool kt_add_ops(PyObject *module, PyObject *device, PyObject *stream, PyObject *attribute)
{
    get_device = device;
    get_stream = stream;
    cuda_stream = attribute;
    ops_type.tp_name = "_kt_marshal.Ops";
    ops_type.tp_basicsize = sizeof(Ops);
    ops_type.tp_flags = Py_TPFLAGS_DEFAULT;
    ops_type.tp_new = ops_new;
    ops_type.tp_methods = methods;
    if (PyType_Ready(&ops_type) < 0) return false;
    Py_INCREF(&ops_type);
    if (PyModule_AddObject(module, "Ops", reinterpret_cast<PyObject *>(&ops_type)) == 0) return true;
    Py_DECREF(&ops_type);
    return false;
}
