// The calling side of pb.py in native code: argument checks, device pointers, the current stream and the call into
// libpbatch.so.  The kernels of a batch-1 layer take 3 to 5 us and a launch 3 us of host time; the same steps through
// ctypes and Python took 8 to 11 us per call (two thirds of it in the per-argument checks and the stream lookup), so
// that a program that calls layer by layer waited for the host.  1024 x 1024, one vector: 11.4 -> 4.8 us per
// PackedLinear call.
//
// A function here takes the call if every argument is what it expects (positional, CUDA tensor of the right type,
// contiguous, ...).  Anything else, wrong or merely unusual, goes to the Python function of the same name in pb.py, which
// raises the errors: one place for their texts.  pb.py does without this extension where it is not built or was built for
// another torch or Python.
#include <torch/csrc/autograd/python_variable.h>

#include <ATen/ATen.h>
#include <c10/hip/HIPFunctions.h>
#include <c10/hip/HIPGraphsC10Utils.h>
#include <c10/hip/HIPStream.h>

#include <tuple>
#include <type_traits>
#include <utility>

#include "pb.h"

namespace {

// what pb.py hands over once, when it has loaded the library
PyObject *g_desc_type = nullptr;    // the ctypes structures pb_desc
PyObject *g_adapters_type = nullptr;    // and pb_adapters
PyObject *g_error = nullptr;        // PbError(status, where)

enum Entry {
    kQuantizePack, kQuantizePackDesc, kQuantizePackMode, kUnpack, kMatmul, kMatmulStatic, kMatmulBiasAct, kMatmulAcc,
    kMatmulAccPairs, kActPrep, kMatmulPrepared, kFixedPoint, kLstmCell, kGatedLinear, kMatmulGrad,
    kGatedLinearGrad, kMatmulAdapters, kMatmulAdaptersGrad, kEntries
};
const char *const kNames[kEntries] = {
    "pb_quantize_pack", "pb_quantize_pack_desc", "pb_quantize_pack_mode", "pb_unpack", "pb_matmul", "pb_matmul_static",
    "pb_matmul_bias_act", "pb_matmul_acc", "pb_matmul_acc_pairs", "pb_act_prep", "pb_matmul_prepared", "pb_fixed_point",
    "pb_lstm_cell", "pb_gated_linear", "pb_matmul_grad", "pb_gated_linear_grad", "pb_matmul_adapters", "pb_matmul_adapters_grad"};
void *g_fn[kEntries];               // null until bound: every call then goes to `slow`
PyObject *g_slow[kEntries];
PyObject *g_slow_linear = nullptr;
// PackedLinear's operators, and the sizes of their workspaces
enum Method { kGated, kGatedGrad, kGrad, kAdapted, kAdaptedGrad, kOperators };
const char *const kMethodNames[kOperators] = {"gated", "gated_grad", "grad", "adapted", "adapted_grad"};
PyObject *g_slow_method[kOperators];
decltype(&pb_workspace_bytes) g_workspace_bytes;
decltype(&pb_grad_workspace_bytes) g_grad_workspace_bytes;
decltype(&pb_adapters_workspace_bytes) g_adapters_workspace_bytes;

// ---- arguments: `load` says whether the object is what the fast path expects ----
template <typename T, at::ScalarType DT, bool NULLABLE = false>
struct Ptr {
    T *v = nullptr;
    bool load(PyObject *o)
    {
        if (NULLABLE && o == Py_None) return true;
        if (!THPVariable_CheckExact(o)) return false;
        const at::Tensor &t = THPVariable_Unpack(o);
        if (!t.is_cuda() || t.scalar_type() != DT || !t.is_contiguous()) return false;
        v = static_cast<T *>(t.data_ptr());
        return true;
    }
    T *get() const { return v; }
};
using In = Ptr<const float, at::kFloat>;
using InOrNone = Ptr<const float, at::kFloat, true>;
using Out = Ptr<float, at::kFloat>;
using OutOrNone = Ptr<float, at::kFloat, true>;
using Bytes = Ptr<void, at::kByte>;
using Ints = Ptr<int32_t, at::kInt>;
using IntsOrNone = Ptr<const int32_t, at::kInt, true>;
using Longs = Ptr<int64_t, at::kLong>;

struct Int {
    int v = 0;
    bool load(PyObject *o)
    {
        if (!PyLong_CheckExact(o)) return false;
        const long x = PyLong_AsLong(o);
        if (x == -1 && PyErr_Occurred()) { PyErr_Clear(); return false; }
        v = static_cast<int>(x);
        return v == x;
    }
    int get() const { return v; }
};

struct Address {
    void *v = nullptr;
    bool load(PyObject *o)
    {
        if (!PyLong_CheckExact(o)) return false;
        v = PyLong_AsVoidPtr(o);
        if (!v && PyErr_Occurred()) { PyErr_Clear(); return false; }
        return true;
    }
};

template <typename S, PyObject **TYPE>
struct Struct {
    S v;
    bool load(PyObject *o)
    {
        if (reinterpret_cast<PyObject *>(Py_TYPE(o)) != *TYPE) return false;
        Py_buffer b;
        if (PyObject_GetBuffer(o, &b, PyBUF_SIMPLE) != 0) { PyErr_Clear(); return false; }
        const bool ok = b.len == (Py_ssize_t)sizeof(S);
        if (ok) v = *static_cast<const S *>(b.buf);
        PyBuffer_Release(&b);
        return ok;
    }
    const S *get() const { return &v; }
};
using Desc = Struct<pb_desc, &g_desc_type>;
using Adapters = Struct<pb_adapters, &g_adapters_type>;

void *current_stream() { return c10::hip::getCurrentHIPStream().stream(); }

bool capturing() { return c10::hip::currentStreamCaptureStatusMayInitCtx() != c10::hip::CaptureStatus::None; }

PyObject *status_result(int rc, const char *where)
{
    if (rc == PB_OK) Py_RETURN_NONE;
    PyObject *e = PyObject_CallFunction(g_error, "is", rc, where);
    if (e) {
        PyErr_SetObject(g_error, e);
        Py_DECREF(e);
    }
    return nullptr;
}

template <typename... A, size_t... I>
bool load_all(std::tuple<A...> &a, PyObject *const *args, std::index_sequence<I...>)
{
    return (std::get<I>(a).load(args[I]) && ...);
}

// fn(args..., stream) of libpbatch.so
template <int E, typename... A>
PyObject *call(PyObject *, PyObject *const *args, Py_ssize_t nargs, PyObject *kwnames)
{
    constexpr Py_ssize_t N = sizeof...(A);
    const bool plain = !kwnames && (nargs == N || (nargs == N + 1 && args[N] == Py_None));
    if (plain && g_fn[E]) {
        try {
            std::tuple<A...> a;
            if (load_all(a, args, std::make_index_sequence<N>())) {
                void *stream = current_stream();
                int rc;
                Py_BEGIN_ALLOW_THREADS
                rc = std::apply(
                    [&](const A &...x) {
                        return reinterpret_cast<int (*)(decltype(std::declval<A>().get())..., void *)>(g_fn[E])(x.get()..., stream);
                    },
                    a);
                Py_END_ALLOW_THREADS
                return status_result(rc, kNames[E]);
            }
        } catch (const std::exception &) {   // (a tensor without memory of its own, say)
        }
    }
    return PyObject_Vectorcall(g_slow[E], args, nargs, kwnames);
}

PyObject *s_rows, *s_cols, *s_bits, *s_max_batch, *s_desc, *s_packed, *s_scales, *s_workspace, *s_home_stream;
PyObject *s_count, *s_rank, *s_A, *s_B, *s_scale;

// The attributes of `self` that a call uses, held until it returns: one that is computed on access, or replaced by another
// thread meanwhile, must not give its memory back before the launch.
struct Held {
    PyObject *o[16];
    int n = 0;
    int workspace = 0;   // which of them
    ~Held() { while (n) Py_DECREF(o[--n]); }
    template <typename T>
    bool load(PyObject *self, PyObject *name, T &x)
    {
        PyObject *a = PyObject_GetAttr(self, name);
        if (!a) { PyErr_Clear(); return false; }
        o[n++] = a;
        return x.load(a);
    }
};

// linear(self, X, bits_used, out): PackedLinear.__call__
PyObject *linear(PyObject *, PyObject *const *args, Py_ssize_t nargs)
{
    if (nargs == 4 && g_fn[kMatmul] && THPVariable_CheckExact(args[1])) {
        try {
            Int rows, cols, max_batch, m;
            Desc d;
            Bytes packed, workspace;
            In scales, x;
            Out y;
            Address home;
            Held held;   // (nine attributes at most)
            PyObject *self = args[0];
            const at::Tensor &X = THPVariable_Unpack(args[1]);
            bool ok = x.load(args[1]) && held.load(self, s_rows, rows) && held.load(self, s_cols, cols) &&
                      held.load(self, s_max_batch, max_batch) && held.load(self, s_desc, d) &&
                      held.load(self, s_packed, packed) && held.load(self, s_scales, scales) &&
                      held.load(self, s_workspace, workspace) && (held.workspace = held.n - 1, held.load(self, s_home_stream, home)) &&
                      (args[2] == Py_None ? held.load(self, s_bits, m) : m.load(args[2]) && m.v != 0);
            const int64_t n = X.numel();
            ok = ok && cols.v > 0 && n > 0 && n % cols.v == 0 && n / cols.v <= max_batch.v;
            if (ok) {
                const int batch = static_cast<int>(n / cols.v);
                at::Tensor out;
                if (args[3] == Py_None) {
                    out = at::empty({batch, rows.v}, X.options().requires_grad(false));
                    y.v = static_cast<float *>(out.data_ptr());
                } else {
                    ok = y.load(args[3]);
                }
                if (ok) {
                    void *stream = current_stream();
                    const auto matmul = reinterpret_cast<decltype(&pb_matmul)>(g_fn[kMatmul]);
                    int rc;
                    // A batch goes through the workspace.  The holder's own serves the stream it was made on (the library keeps the
                    // launches of two threads apart); on another stream the call has one of its own, and under capture: a graph
                    // may be replayed on any stream (the memory is then the graph's, as that of the output).
                    at::Tensor own;
                    if ((batch > 1 || d.v.layout == PB_LAYOUT_ROWMAJOR_V1 || d.v.layout == PB_LAYOUT_TILE16_PAIRS_V1) &&
                        (stream != home.v || capturing()))
                        own = at::empty_like(THPVariable_Unpack(held.o[held.workspace]));
                    void *const work = own.defined() ? own.data_ptr() : workspace.v;
                    Py_BEGIN_ALLOW_THREADS
                    rc = matmul(packed.v, scales.v, &d.v, m.v, x.v, batch, y.v, work, stream);
                    Py_END_ALLOW_THREADS
                    if (rc != PB_OK) return status_result(rc, kNames[kMatmul]);
                    if (args[3] != Py_None) {
                        Py_INCREF(args[3]);
                        return args[3];
                    }
                    return THPVariable_Wrap(std::move(out));
                }
            }
        } catch (const std::exception &) {
        }
    }
    return PyObject_Vectorcall(g_slow_linear, args, nargs, nullptr);
}

// ---- PackedLinear's operators: f(self, every argument), with outputs and a workspace made here.  What is not as they expect it goes to the Python
// functions in pb.py, as above. ----
const at::Tensor *tensor(PyObject *o) { return THPVariable_CheckExact(o) ? &THPVariable_Unpack(o) : nullptr; }
bool plain(const at::Tensor *t, const at::Device &device, at::ScalarType type)
{
    return t && t->is_cuda() && t->scalar_type() == type && t->is_contiguous() && t->device() == device;
}

// What every operator uses of the layer
struct Layer {
    Held held;
    Int rows, cols, m;
    Desc d;
    Bytes packed;
    In scales;
    at::Device device = at::kCPU;
    bool load(PyObject *self, PyObject *bits_used)
    {
        if (!g_workspace_bytes || !held.load(self, s_packed, packed)) return false;
        device = THPVariable_Unpack(held.o[held.n - 1]).device();
        return device.index() == c10::hip::current_device() && held.load(self, s_rows, rows) && held.load(self, s_cols, cols) &&
               held.load(self, s_desc, d) && held.load(self, s_scales, scales) &&
               (bits_used == Py_None ? held.load(self, s_bits, m) : m.load(bits_used));
    }
    // n vectors of `length` values
    const float *vectors(PyObject *o, int length, int64_t *n) const
    {
        const at::Tensor *t = tensor(o);
        if (!plain(t, device, at::kFloat) || t->dim() != 2 || t->size(1) != length || t->size(0) < 1 || t->size(0) > PB_MAX_BATCH) return nullptr;
        if (*n && *n != t->size(0)) return nullptr;
        *n = t->size(0);
        return static_cast<const float *>(t->data_ptr());
    }
    // `length` values or None
    template <typename T>
    bool values(PyObject *o, at::ScalarType type, int64_t length, const T **p) const
    {
        *p = nullptr;
        if (o == Py_None) return true;
        const at::Tensor *t = tensor(o);
        if (!plain(t, device, type) || t->dim() != 1 || t->size(0) != length) return false;
        *p = static_cast<const T *>(t->data_ptr());
        return true;
    }
    at::Tensor floats(at::IntArrayRef shape) const { return at::empty(shape, at::TensorOptions().dtype(at::kFloat).device(device)); }
    at::Tensor work(size_t bytes) const
    {
        return at::empty({(int64_t)(bytes > 16 ? bytes : 16)}, at::TensorOptions().dtype(at::kByte).device(device));
    }
};
float *floats_of(const at::Tensor &t) { return static_cast<float *>(t.data_ptr()); }

// The tensors of an Adapters object as they are now, held until the call returns
struct AdapterSet {
    Held held;
    pb_adapters v{};
    at::Tensor A, B;
    bool load(PyObject *o, const Layer &l)
    {
        Int count, rank, rows, cols;
        PyObject *a = PyObject_GetAttr(o, s_A), *b = a ? PyObject_GetAttr(o, s_B) : nullptr, *s = b ? PyObject_GetAttr(o, s_scale) : nullptr;
        for (PyObject *x : {a, b, s})
            if (x) held.o[held.n++] = x;
        if (!s) { PyErr_Clear(); return false; }
        if (!held.load(o, s_count, count) || !held.load(o, s_rank, rank) || !held.load(o, s_rows, rows) || !held.load(o, s_cols, cols)) return false;
        const at::Tensor *ta = tensor(a), *tb = tensor(b);
        if (!ta || !tb || rows.v != l.rows.v || cols.v != l.cols.v) return false;
        const at::ScalarType type = ta->scalar_type();
        if (type != at::kFloat && type != at::kBFloat16 && type != at::kHalf) return false;
        if (!plain(ta, l.device, type) || !plain(tb, l.device, type)) return false;
        if (ta->sizes() != at::IntArrayRef({count.v, rank.v, cols.v}) || tb->sizes() != at::IntArrayRef({count.v, rows.v, rank.v})) return false;
        if (!l.values(s, at::kFloat, count.v, &v.scale)) return false;
        A = *ta;
        B = *tb;
        v.count = count.v;
        v.rank = rank.v;
        v.type = type == at::kFloat ? PB_TYPE_F32 : (type == at::kBFloat16 ? PB_TYPE_BF16 : PB_TYPE_F16);
        v.A = ta->data_ptr();
        v.B = tb->data_ptr();
        return true;
    }
};

template <typename F>
int without_gil(F f)
{
    int rc;
    Py_BEGIN_ALLOW_THREADS
    rc = f();
    Py_END_ALLOW_THREADS
    return rc;
}
template <typename... T>
PyObject *tuple_of(T... tensors)      // an undefined tensor is None
{
    PyObject *t = PyTuple_New(sizeof...(T));
    if (!t) return nullptr;
    Py_ssize_t i = 0;
    auto put = [&](at::Tensor &x) {
        PyObject *o = x.defined() ? THPVariable_Wrap(std::move(x)) : Py_NewRef(Py_None);
        if (!o) return false;
        PyTuple_SET_ITEM(t, i++, o);
        return true;
    };
    if (!(put(tensors) && ...)) {
        Py_DECREF(t);
        return nullptr;
    }
    return t;
}
// f(args) sets *result (or an error) where it takes the call
template <Method M, int N, typename F>
PyObject *method(PyObject *const *args, Py_ssize_t nargs, F f)
{
    if (nargs == N) {
        try {
            PyObject *result = nullptr;
            if (f(args, &result)) return result;
        } catch (const std::exception &) {
        }
        if (PyErr_Occurred()) PyErr_Clear();
    }
    return PyObject_Vectorcall(g_slow_method[M], args, nargs, nullptr);
}

// gated(self, X, gate, bits_used, bias, keep)
PyObject *gated(PyObject *, PyObject *const *args, Py_ssize_t nargs)
{
    return method<kGated, 6>(args, nargs, [](PyObject *const *a, PyObject **result) {
        Layer l;
        Int gate;
        int64_t n = 0;
        const float *x, *bias;
        if (!l.load(a[0], a[3]) || !(x = l.vectors(a[1], l.cols.v, &n)) || !gate.load(a[2]) || !l.values(a[4], at::kFloat, l.rows.v, &bias)) return false;
        if (a[5] != Py_True && a[5] != Py_False) return false;
        at::Tensor H = l.floats({n, l.rows.v / 2}), pre = a[5] == Py_True ? l.floats({n, l.rows.v}) : at::Tensor();
        const at::Tensor work = l.work(g_workspace_bytes(&l.d.v, (int)n));
        void *stream = current_stream();
        const int rc = without_gil([&] {
            return reinterpret_cast<decltype(&pb_gated_linear)>(g_fn[kGatedLinear])(l.packed.v, l.scales.v, &l.d.v, l.m.v, x, (int)n, bias, gate.v, floats_of(H),
                                                                                    pre.defined() ? floats_of(pre) : nullptr, work.data_ptr(), stream);
        });
        if (rc != PB_OK) *result = status_result(rc, kNames[kGatedLinear]);
        else *result = pre.defined() ? tuple_of(H, pre) : THPVariable_Wrap(std::move(H));
        return true;
    });
}

// gated_grad(self, pre, dH, gate, bits_used)
PyObject *gated_grad(PyObject *, PyObject *const *args, Py_ssize_t nargs)
{
    return method<kGatedGrad, 5>(args, nargs, [](PyObject *const *a, PyObject **result) {
        Layer l;
        Int gate;
        int64_t n = 0;
        const float *pre, *dH;
        if (!l.load(a[0], a[4]) || !(pre = l.vectors(a[1], l.rows.v, &n)) || !(dH = l.vectors(a[2], l.rows.v / 2, &n)) || !gate.load(a[3])) return false;
        at::Tensor dX = l.floats({n, l.cols.v}), dpre = l.floats({n, l.rows.v});
        const at::Tensor work = l.work(g_grad_workspace_bytes(&l.d.v, (int)n));
        void *stream = current_stream();
        const int rc = without_gil([&] {
            return reinterpret_cast<decltype(&pb_gated_linear_grad)>(g_fn[kGatedLinearGrad])(l.packed.v, l.scales.v, &l.d.v, l.m.v, pre, dH, (int)n, gate.v,
                                                                                             floats_of(dpre), floats_of(dX), work.data_ptr(), stream);
        });
        *result = rc != PB_OK ? status_result(rc, kNames[kGatedLinearGrad]) : tuple_of(dX, dpre);
        return true;
    });
}

// grad(self, dY, bits_used)
PyObject *grad(PyObject *, PyObject *const *args, Py_ssize_t nargs)
{
    return method<kGrad, 3>(args, nargs, [](PyObject *const *a, PyObject **result) {
        Layer l;
        int64_t n = 0;
        const float *dY;
        if (!l.load(a[0], a[2]) || !(dY = l.vectors(a[1], l.rows.v, &n))) return false;
        at::Tensor dX = l.floats({n, l.cols.v});
        const at::Tensor work = l.work(g_grad_workspace_bytes(&l.d.v, (int)n));
        void *stream = current_stream();
        const int rc = without_gil([&] {
            return reinterpret_cast<decltype(&pb_matmul_grad)>(g_fn[kMatmulGrad])(l.packed.v, l.scales.v, &l.d.v, l.m.v, dY, (int)n, floats_of(dX),
                                                                                  work.data_ptr(), stream);
        });
        *result = rc != PB_OK ? status_result(rc, kNames[kMatmulGrad]) : THPVariable_Wrap(std::move(dX));
        return true;
    });
}

// adapted(self, X, adapters, index, bits_used, bias)
PyObject *adapted(PyObject *, PyObject *const *args, Py_ssize_t nargs)
{
    return method<kAdapted, 6>(args, nargs, [](PyObject *const *a, PyObject **result) {
        Layer l;
        AdapterSet set;
        int64_t n = 0;
        const float *x, *bias;
        const int32_t *index;
        if (!l.load(a[0], a[4]) || !(x = l.vectors(a[1], l.cols.v, &n)) || !l.values(a[3], at::kInt, n, &index) ||
            !l.values(a[5], at::kFloat, l.rows.v, &bias) || !set.load(a[2], l)) return false;
        at::Tensor Y = l.floats({n, l.rows.v});
        const at::Tensor work = l.work(g_adapters_workspace_bytes(&l.d.v, &set.v, (int)n));
        void *stream = current_stream();
        const int rc = without_gil([&] {
            return reinterpret_cast<decltype(&pb_matmul_adapters)>(g_fn[kMatmulAdapters])(l.packed.v, l.scales.v, &l.d.v, l.m.v, x, (int)n, &set.v, index, bias,
                                                                                          floats_of(Y), work.data_ptr(), stream);
        });
        *result = rc != PB_OK ? status_result(rc, kNames[kMatmulAdapters]) : THPVariable_Wrap(std::move(Y));
        return true;
    });
}

// adapted_grad(self, X, dY, adapters, index, bits_used, inputs)
PyObject *adapted_grad(PyObject *, PyObject *const *args, Py_ssize_t nargs)
{
    return method<kAdaptedGrad, 7>(args, nargs, [](PyObject *const *a, PyObject **result) {
        Layer l;
        AdapterSet set;
        int64_t n = 0;
        const float *x, *dY;
        const int32_t *index;
        if (!l.load(a[0], a[5]) || !(x = l.vectors(a[1], l.cols.v, &n)) || !(dY = l.vectors(a[2], l.rows.v, &n)) ||
            !l.values(a[4], at::kInt, n, &index) || !set.load(a[3], l)) return false;
        if (a[6] != Py_True && a[6] != Py_False) return false;
        at::Tensor dX = a[6] == Py_True ? l.floats({n, l.cols.v}) : at::Tensor(), dA = l.floats(set.A.sizes()), dB = l.floats(set.B.sizes());
        const at::Tensor work = l.work(g_adapters_workspace_bytes(&l.d.v, &set.v, (int)n));
        void *stream = current_stream();
        const int rc = without_gil([&] {
            return reinterpret_cast<decltype(&pb_matmul_adapters_grad)>(g_fn[kMatmulAdaptersGrad])(
                l.packed.v, l.scales.v, &l.d.v, l.m.v, x, dY, (int)n, &set.v, index, dX.defined() ? floats_of(dX) : nullptr, floats_of(dA), floats_of(dB),
                work.data_ptr(), stream);
        });
        *result = rc != PB_OK ? status_result(rc, kNames[kMatmulAdaptersGrad]) : tuple_of(dX, dA, dB);
        return true;
    });
}

// bind(desc_type, adapters_type, error_type, {name: address})
PyObject *bind(PyObject *, PyObject *args)
{
    PyObject *desc, *adapters, *error, *fns;
    if (!PyArg_ParseTuple(args, "OOOO!", &desc, &adapters, &error, &PyDict_Type, &fns)) return nullptr;
    void *p[kEntries];
    for (int e = 0; e < kEntries; ++e) {
        PyObject *a = PyDict_GetItemString(fns, kNames[e]);
        if (!a) return PyErr_Format(PyExc_KeyError, "%s", kNames[e]);
        p[e] = PyLong_AsVoidPtr(a);
        if (!p[e]) return PyErr_Occurred() ? nullptr : PyErr_Format(PyExc_ValueError, "%s", kNames[e]);
    }
    void *sizes[3];
    const char *const size_names[3] = {"pb_workspace_bytes", "pb_grad_workspace_bytes", "pb_adapters_workspace_bytes"};
    for (int i = 0; i < 3; ++i) {
        PyObject *a = PyDict_GetItemString(fns, size_names[i]);
        if (!a) return PyErr_Format(PyExc_KeyError, "%s", size_names[i]);
        sizes[i] = PyLong_AsVoidPtr(a);
        if (!sizes[i]) return PyErr_Occurred() ? nullptr : PyErr_Format(PyExc_ValueError, "%s", size_names[i]);
    }
    Py_INCREF(desc);
    Py_INCREF(adapters);
    Py_INCREF(error);
    Py_XDECREF(g_desc_type);
    Py_XDECREF(g_adapters_type);
    Py_XDECREF(g_error);
    g_desc_type = desc;
    g_adapters_type = adapters;
    g_error = error;
    for (int e = 0; e < kEntries; ++e) g_fn[e] = p[e];
    g_grad_workspace_bytes = reinterpret_cast<decltype(&pb_grad_workspace_bytes)>(sizes[1]);
    g_adapters_workspace_bytes = reinterpret_cast<decltype(&pb_adapters_workspace_bytes)>(sizes[2]);
    g_workspace_bytes = reinterpret_cast<decltype(&pb_workspace_bytes)>(sizes[0]);
    Py_RETURN_NONE;
}

// set_slow({name: function}): the Python functions behind the fast ones ("linear" for PackedLinear.__call__, "gated" for PackedLinear.gated, ...)
PyObject *set_slow(PyObject *, PyObject *fns)
{
    if (!PyDict_Check(fns)) return PyErr_Format(PyExc_TypeError, "a dict of functions");
    for (int e = 0; e <= kEntries + kOperators; ++e) {
        const char *name = e < kEntries ? kNames[e] : (e == kEntries ? "linear" : kMethodNames[e - kEntries - 1]);
        PyObject *f = PyDict_GetItemString(fns, name);
        if (!f) return PyErr_Format(PyExc_KeyError, "%s", name);
        PyObject **slot = e < kEntries ? &g_slow[e] : (e == kEntries ? &g_slow_linear : &g_slow_method[e - kEntries - 1]);
        Py_INCREF(f);
        Py_XDECREF(*slot);
        *slot = f;
    }
    Py_RETURN_NONE;
}

// as many arguments as the C function has, each convertible to the parameter in its place, and the stream as the last
template <typename F>
struct Params;
template <typename... P>
struct Params<int (*)(P...)> {
    template <typename... A>
    static constexpr bool take()
    {
        if constexpr (sizeof...(P) == sizeof...(A) + 1)
            return std::is_invocable_v<int (*)(P...), decltype(std::declval<const A &>().get())..., void *>;
        else
            return false;
    }
};
template <auto F, int E, typename... A>
PyMethodDef fast()
{
    static_assert(Params<decltype(F)>::template take<A...>(), "not the arguments of the C function");
    return {kNames[E], reinterpret_cast<PyCFunction>(reinterpret_cast<void (*)()>(&call<E, A...>)), METH_FASTCALL | METH_KEYWORDS,
            nullptr};
}
PyMethodDef kMethods[] = {
    fast<&pb_quantize_pack, kQuantizePack, In, Int, Int, Int, Bytes, Out>(),
    fast<&pb_quantize_pack_desc, kQuantizePackDesc, In, Desc, Bytes, Out>(),
    fast<&pb_quantize_pack_mode, kQuantizePackMode, In, Desc, Int, Bytes, Out>(),
    fast<&pb_unpack, kUnpack, Bytes, Desc, Ints>(),
    fast<&pb_matmul, kMatmul, Bytes, In, Desc, Int, In, Int, Out, Bytes>(),
    fast<&pb_matmul_static, kMatmulStatic, Bytes, In, Desc, Int, In, Int, Out>(),
    fast<&pb_matmul_bias_act, kMatmulBiasAct, Bytes, In, Desc, Int, In, Int, InOrNone, Int, Out, Bytes>(),
    fast<&pb_matmul_acc, kMatmulAcc, Bytes, Desc, Int, In, Int, Longs, Bytes>(),
    fast<&pb_matmul_acc_pairs, kMatmulAccPairs, Bytes, Desc, Int, In, Int, Longs, Bytes>(),
    fast<&pb_act_prep, kActPrep, Desc, In, Int, Bytes>(),
    fast<&pb_matmul_prepared, kMatmulPrepared, Bytes, In, Desc, Int, Int, Out, Bytes>(),
    fast<&pb_fixed_point, kFixedPoint, Desc, In, Int, Ints, Bytes>(),
    fast<&pb_lstm_cell, kLstmCell, Bytes, In, Desc, Int, In, Int, In, In, InOrNone, Out, Out, Int, Bytes>(),
    fast<&pb_gated_linear, kGatedLinear, Bytes, In, Desc, Int, In, Int, InOrNone, Int, Out, OutOrNone, Bytes>(),
    fast<&pb_matmul_grad, kMatmulGrad, Bytes, In, Desc, Int, In, Int, Out, Bytes>(),
    fast<&pb_gated_linear_grad, kGatedLinearGrad, Bytes, In, Desc, Int, In, In, Int, Int, Out, Out, Bytes>(),
    fast<&pb_matmul_adapters, kMatmulAdapters, Bytes, In, Desc, Int, In, Int, Adapters, IntsOrNone, InOrNone, Out, Bytes>(),
    fast<&pb_matmul_adapters_grad, kMatmulAdaptersGrad, Bytes, In, Desc, Int, In, In, Int, Adapters, IntsOrNone, OutOrNone, OutOrNone,
         OutOrNone, Bytes>(),
    {"linear", reinterpret_cast<PyCFunction>(reinterpret_cast<void (*)()>(&linear)), METH_FASTCALL, nullptr},
    {"gated", reinterpret_cast<PyCFunction>(reinterpret_cast<void (*)()>(&gated)), METH_FASTCALL, nullptr},
    {"gated_grad", reinterpret_cast<PyCFunction>(reinterpret_cast<void (*)()>(&gated_grad)), METH_FASTCALL, nullptr},
    {"grad", reinterpret_cast<PyCFunction>(reinterpret_cast<void (*)()>(&grad)), METH_FASTCALL, nullptr},
    {"adapted", reinterpret_cast<PyCFunction>(reinterpret_cast<void (*)()>(&adapted)), METH_FASTCALL, nullptr},
    {"adapted_grad", reinterpret_cast<PyCFunction>(reinterpret_cast<void (*)()>(&adapted_grad)), METH_FASTCALL, nullptr},
    {"bind", bind, METH_VARARGS, nullptr},
    {"set_slow", set_slow, METH_O, nullptr},
    {nullptr, nullptr, 0, nullptr},
};

PyModuleDef kModule = {PyModuleDef_HEAD_INIT, "_binding", nullptr, -1, kMethods, nullptr, nullptr, nullptr, nullptr};

}  // namespace

PyMODINIT_FUNC PyInit__binding()
{
    s_rows = PyUnicode_InternFromString("rows");
    s_cols = PyUnicode_InternFromString("cols");
    s_bits = PyUnicode_InternFromString("bits");
    s_max_batch = PyUnicode_InternFromString("max_batch");
    s_desc = PyUnicode_InternFromString("desc");
    s_packed = PyUnicode_InternFromString("packed");
    s_scales = PyUnicode_InternFromString("scales");
    s_workspace = PyUnicode_InternFromString("workspace");
    s_home_stream = PyUnicode_InternFromString("home_stream");
    s_count = PyUnicode_InternFromString("count");
    s_rank = PyUnicode_InternFromString("rank");
    s_A = PyUnicode_InternFromString("A");
    s_B = PyUnicode_InternFromString("B");
    s_scale = PyUnicode_InternFromString("scale");
    PyObject *m = PyModule_Create(&kModule);
    if (m && PyModule_AddStringConstant(m, "BUILT_FOR", PB_BUILT_FOR) != 0) Py_CLEAR(m);   // (pb.py compares it)
    return m;
}
