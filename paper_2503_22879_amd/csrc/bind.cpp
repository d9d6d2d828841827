// Python argument marshalling of the device entry points of include/quamba_ssd.h, in native code.
//
// A generated token costs three library calls of 3 to 8 us of device work each at small batches, so what a call costs on
// the host is what a small model's token costs.  Marshalled in Python (about 50 attribute look-ups, tuple comparisons and
// ctypes conversions) a call took 8 to 11 us of host time; here the tensors' metadata are read from the tensor objects
// themselves.  Every check is made on every call; nothing is remembered from one call for the next but the
// addresses of the library's functions.
//
// The functions take positional arguments in the order of their Python signatures (binding.py) and return the library's
// status.  Tensors are torch tensors or None.
#include <Python.h>
#include <c10/hip/HIPStream.h>
#include <torch/csrc/autograd/python_variable.h>

#include <initializer_list>
#include <vector>

#include "quamba_ssd.h"

namespace {

// The library's entry points, by address: the library that binding.py has loaded.
struct Entry {
    decltype(&quamba_ssd_prefill_gated) prefill;
    decltype(&quamba_ssd_prefill_noalloc) prefill_noalloc;
    decltype(&quamba_ssd_decode_step_gated) decode;
    decltype(&quamba_ssd_decode_step_q8_gated) decode_q8;
    decltype(&quamba_ssd_quantize_state) quantize_state;
    decltype(&quamba_hadamard_quantize) hadamard;
    decltype(&quamba_mamba1_scan_gated) mamba1_scan;
    decltype(&quamba_mamba1_decode_step_gated) mamba1_decode;
    decltype(&quamba_conv1d_q8) conv1d;
    decltype(&quamba_fp8_quantize) fp8_quantize;
    decltype(&quamba_fp8_matmul) fp8_matmul;
    decltype(&quamba_beam_select) beam_select;
    decltype(&quamba_beam_reorder) beam_reorder;
} entry;

// The ctypes structures that carry the shape, the scale tables and the side inputs, and the classes that are read directly:
// types of binding.py.
PyObject *shape_type, *scales_type, *gate_struct_type, *device_scales_type, *gate_type;
PyObject *address_of;  // and its function from a ctypes pointer to its address or None

// Interned attribute names.
PyObject *s_tensors, *s_struct, *s_cuda_stream, *s_z, *s_z_scale, *s_dt_q, *s_dt_scale, *s_dt_bias;

struct Fail {};  // a Python exception is set

[[noreturn]] void fail(PyObject *type, const char *format, const char *name)
{
    PyErr_Format(type, format, name);
    throw Fail();
}

const at::Tensor *tensor_or_null(PyObject *o, const char *name)
{
    if (o == Py_None) return nullptr;
    if (!THPVariable_Check(o)) fail(PyExc_TypeError, "%s must be a torch tensor", name);
    return &THPVariable_Unpack(o);
}

void *device_pointer(const at::Tensor *t, const char *name)
{
    if (!t) return nullptr;
    if (!t->is_cuda() || !t->is_contiguous()) fail(PyExc_ValueError, "%s must be a contiguous device tensor", name);
    return t->data_ptr();
}

// Device pointer of a tensor argument (None: NULL), with the checks a C caller would have to make itself.
template <typename T>
T *pointer(PyObject *o, at::ScalarType type, std::initializer_list<int64_t> shape, const char *name)
{
    const at::Tensor *t = tensor_or_null(o, name);
    if (!t) return nullptr;
    void *p = device_pointer(t, name);
    if (t->scalar_type() != type) {
        PyErr_Format(PyExc_ValueError, "%s must have dtype %s, got %s", name, c10::toString(type),
                     c10::toString(t->scalar_type()));
        throw Fail();
    }
    if (t->sizes() != at::IntArrayRef(shape)) {
        std::string want, got;
        for (int64_t v : shape) want += std::to_string(v) + ", ";
        for (int64_t v : t->sizes()) got += std::to_string(v) + ", ";
        PyErr_Format(PyExc_ValueError, "%s must have shape (%s), got (%s)", name, want.c_str(), got.c_str());
        throw Fail();
    }
    return static_cast<T *>(p);
}

float number(PyObject *o)
{
    const double v = PyFloat_AsDouble(o);
    if (v == -1.0 && PyErr_Occurred()) throw Fail();
    return (float)v;
}

struct Ref {  // an owned reference
    PyObject *o;
    explicit Ref(PyObject *p) : o(p) { if (!o) throw Fail(); }
    ~Ref() { Py_DECREF(o); }
    Ref(const Ref &) = delete;
};

// The bytes of a ctypes structure, an instance of `type`: another object's bytes are not a structure, however many.
template <typename T>
T structure(PyObject *o, PyObject *type, const char *name)
{
    if (!PyObject_TypeCheck(o, reinterpret_cast<PyTypeObject *>(type))) {
        PyErr_Format(PyExc_TypeError, "%s must be a %s, not %s", name, reinterpret_cast<PyTypeObject *>(type)->tp_name,
                     Py_TYPE(o)->tp_name);
        throw Fail();
    }
    Py_buffer view;
    if (PyObject_GetBuffer(o, &view, PyBUF_SIMPLE) != 0) throw Fail();
    const bool fits = view.len >= (Py_ssize_t)sizeof(T);  // a subclass may have added fields
    T v;
    if (fits) memcpy(&v, view.buf, sizeof(T));
    PyBuffer_Release(&view);
    if (!fits) fail(PyExc_TypeError, "%s has the wrong size", name);
    return v;
}

quamba_ssd_shape_t shape_of(PyObject *o) { return structure<quamba_ssd_shape_t>(o, shape_type, "shape"); }

// The scale tables: a DeviceScales holds the five device tensors, in the struct's order; anything else (a subclass may say
// otherwise) is asked for its struct().
quamba_ssd_scales_t scales_of(PyObject *o)
{
    if (Py_TYPE(o) == reinterpret_cast<PyTypeObject *>(device_scales_type)) {
        Ref list(PyObject_GetAttr(o, s_tensors));
        if (PyList_Check(list.o) && PyList_GET_SIZE(list.o) == 5) {
            const void *p[5];
            int n = 0;
            for (; n < 5 && THPVariable_Check(PyList_GET_ITEM(list.o, n)); ++n)
                p[n] = THPVariable_Unpack(PyList_GET_ITEM(list.o, n)).data_ptr();
            if (n == 5)
                return {static_cast<const float *>(p[0]), static_cast<const int32_t *>(p[1]),
                        static_cast<const int32_t *>(p[2]), static_cast<const float *>(p[3]),
                        static_cast<const float *>(p[4])};
        }
    }
    Ref st(PyObject_CallMethodNoArgs(o, s_struct));
    return structure<quamba_ssd_scales_t>(st.o, scales_type, "scales.struct()");
}

PyObject *tuple_of(std::initializer_list<int64_t> v)
{
    PyObject *t = PyTuple_New((Py_ssize_t)v.size());
    Py_ssize_t i = 0;
    if (t)
        for (int64_t e : v) {
            PyObject *item = PyLong_FromLongLong(e);
            if (!item) {
                Py_DECREF(t);
                return nullptr;
            }
            PyTuple_SET_ITEM(t, i++, item);
        }
    return t;
}

// The optional side inputs (None: no struct): the fields of a Gate; anything else is asked for its struct().
struct GateArg {
    quamba_ssd_gate_t g;
    bool present = false;
    GateArg(PyObject *o, std::initializer_list<int64_t> z_shape, std::initializer_list<int64_t> dt_shape, int64_t nbias)
    {
        if (o == Py_None) return;
        present = true;
        if (Py_TYPE(o) != reinterpret_cast<PyTypeObject *>(gate_type)) {
            Ref zt(tuple_of(z_shape)), dtt(tuple_of(dt_shape)), nb(PyLong_FromLongLong(nbias));
            Ref st(PyObject_CallMethodObjArgs(o, s_struct, zt.o, dtt.o, nb.o, nullptr));
            g = structure<quamba_ssd_gate_t>(st.o, gate_struct_type, "gate.struct()");
            return;
        }
        Ref z(PyObject_GetAttr(o, s_z)), zs(PyObject_GetAttr(o, s_z_scale)), dq(PyObject_GetAttr(o, s_dt_q)),
            ds(PyObject_GetAttr(o, s_dt_scale)), db(PyObject_GetAttr(o, s_dt_bias));
        g.z = pointer<int8_t>(z.o, at::kChar, z_shape, "gate.z");
        g.z_scale = number(zs.o);
        g.dt_q = pointer<int8_t>(dq.o, at::kChar, dt_shape, "gate.dt_q");
        g.dt_scale = number(ds.o);
        g.dt_bias = pointer<float>(db.o, at::kFloat, {nbias}, "gate.dt_bias");
    }
    const quamba_ssd_gate_t *get() const { return present ? &g : nullptr; }
};

// The stream argument: None is torch's current stream, else an object with a cuda_stream attribute or the pointer itself, as
// a number or as anything that ctypes takes for a pointer (c_void_p, a pointer or array instance).
void *stream_of(PyObject *o)
{
    if (o == Py_None) return c10::hip::getCurrentHIPStream().stream();
    PyObject *a = PyObject_GetAttr(o, s_cuda_stream);
    if (!a) {
        PyErr_Clear();
        Py_INCREF(o);
        a = o;
    }
    Ref held(a);
    if (!PyLong_Check(a)) {
        Ref address(PyObject_CallFunctionObjArgs(address_of, a, nullptr));
        if (address.o == Py_None) return nullptr;
        void *p = PyLong_AsVoidPtr(address.o);
        if (PyErr_Occurred()) throw Fail();
        return p;
    }
    void *p = PyLong_AsVoidPtr(a);
    if (PyErr_Occurred()) throw Fail();
    return p;
}

void need(Py_ssize_t n, Py_ssize_t want)
{
    if (n != want) {
        PyErr_Format(PyExc_TypeError, "expected %zd arguments, got %zd", want, n);
        throw Fail();
    }
}

// Runs a library call without the interpreter lock and hands its status back.
template <typename F>
PyObject *call(F &&f)
{
    int rc;
    Py_BEGIN_ALLOW_THREADS
    rc = f();
    Py_END_ALLOW_THREADS
    return PyLong_FromLong(rc);
}

// Arguments of the SSD entry points that prefill and decode share.
struct Operands {
    const int8_t *x, *B, *C;
    const float *dt, *A, *D;
};

Operands prefill_operands(PyObject *const *a, const quamba_ssd_shape_t &s)
{
    Operands o;
    o.x = pointer<int8_t>(a[0], at::kChar, {s.batch, s.seqlen, s.nheads, s.headdim}, "x");
    o.B = pointer<int8_t>(a[1], at::kChar, {s.batch, s.seqlen, s.ngroups, s.d_state}, "B");
    o.C = pointer<int8_t>(a[2], at::kChar, {s.batch, s.seqlen, s.ngroups, s.d_state}, "C");
    o.dt = pointer<float>(a[3], at::kFloat, {s.batch, s.seqlen, s.nheads}, "dt");
    o.A = pointer<float>(a[4], at::kFloat, {s.nheads}, "A");
    o.D = pointer<float>(a[5], at::kFloat, {s.nheads}, "D");
    return o;
}

Operands decode_operands(PyObject *const *a, const quamba_ssd_shape_t &s)
{
    Operands o;
    o.x = pointer<int8_t>(a[0], at::kChar, {s.batch, s.nheads, s.headdim}, "x");
    o.B = pointer<int8_t>(a[1], at::kChar, {s.batch, s.ngroups, s.d_state}, "B");
    o.C = pointer<int8_t>(a[2], at::kChar, {s.batch, s.ngroups, s.d_state}, "C");
    o.dt = pointer<float>(a[3], at::kFloat, {s.batch, s.nheads}, "dt");
    o.A = pointer<float>(a[4], at::kFloat, {s.nheads}, "A");
    o.D = pointer<float>(a[5], at::kFloat, {s.nheads}, "D");
    return o;
}

// shape, scales, x, B, C, dt, A, D, init_state, y, final_state, workspace, stream, gate
PyObject *prefill(PyObject *const *a)
{
    const quamba_ssd_shape_t s = shape_of(a[0]);
    const quamba_ssd_scales_t sc = scales_of(a[1]);
    const at::Tensor *w = tensor_or_null(a[11], "workspace");
    void *ws = device_pointer(w, "workspace");
    const size_t ws_bytes = w ? (size_t)w->numel() * w->element_size() : 0;
    const GateArg gate(a[13], {s.batch, s.seqlen, s.nheads, s.headdim}, {s.batch, s.seqlen, s.nheads}, s.nheads);
    const Operands o = prefill_operands(a + 2, s);
    const float *init = pointer<float>(a[8], at::kFloat, {s.batch, s.nheads, s.headdim, s.d_state}, "init_state");
    uint16_t *y = pointer<uint16_t>(a[9], at::kHalf, {s.batch, s.seqlen, s.nheads, s.headdim}, "y");
    float *fin = pointer<float>(a[10], at::kFloat, {s.batch, s.nheads, s.headdim, s.d_state}, "final_state");
    void *stream = stream_of(a[12]);
    return call([&] {
        return entry.prefill(&s, &sc, gate.get(), o.x, o.B, o.C, o.dt, o.A, o.D, init, y, fin, ws, ws_bytes, stream);
    });
}

// shape, scales, x, B, C, dt, A, D, init_state, y, final_state, stream
PyObject *prefill_noalloc(PyObject *const *a)
{
    const quamba_ssd_shape_t s = shape_of(a[0]);
    const quamba_ssd_scales_t sc = scales_of(a[1]);
    const Operands o = prefill_operands(a + 2, s);
    const float *init = pointer<float>(a[8], at::kFloat, {s.batch, s.nheads, s.headdim, s.d_state}, "init_state");
    uint16_t *y = pointer<uint16_t>(a[9], at::kHalf, {s.batch, s.seqlen, s.nheads, s.headdim}, "y");
    float *fin = pointer<float>(a[10], at::kFloat, {s.batch, s.nheads, s.headdim, s.d_state}, "final_state");
    void *stream = stream_of(a[11]);
    return call([&] {
        return entry.prefill_noalloc(&s, &sc, o.x, o.B, o.C, o.dt, o.A, o.D, init, y, fin, stream);
    });
}

// shape, scales, x, B, C, dt, A, D, state, y, stream, gate
PyObject *decode(PyObject *const *a)
{
    const quamba_ssd_shape_t s = shape_of(a[0]);
    const quamba_ssd_scales_t sc = scales_of(a[1]);
    const GateArg gate(a[11], {s.batch, s.nheads, s.headdim}, {s.batch, s.nheads}, s.nheads);
    const Operands o = decode_operands(a + 2, s);
    float *state = pointer<float>(a[8], at::kFloat, {s.batch, s.nheads, s.headdim, s.d_state}, "state");
    uint16_t *y = pointer<uint16_t>(a[9], at::kHalf, {s.batch, s.nheads, s.headdim}, "y");
    void *stream = stream_of(a[10]);
    return call([&] { return entry.decode(&s, &sc, gate.get(), o.x, o.B, o.C, o.dt, o.A, o.D, state, y, stream); });
}

int64_t cells(const quamba_ssd_shape_t &s) { return (int64_t)s.ngroups * s.n_head_clusters * s.n_chan_clusters; }

// shape, scales, state_scales, x, B, C, dt, A, D, state_q, y, stream, gate
PyObject *decode_q8(PyObject *const *a)
{
    const quamba_ssd_shape_t s = shape_of(a[0]);
    const quamba_ssd_scales_t sc = scales_of(a[1]);
    const GateArg gate(a[12], {s.batch, s.nheads, s.headdim}, {s.batch, s.nheads}, s.nheads);
    const float *ss = pointer<float>(a[2], at::kFloat, {cells(s), s.d_state}, "state_scales");
    const Operands o = decode_operands(a + 3, s);
    int8_t *state = pointer<int8_t>(a[9], at::kChar, {s.batch, s.nheads, s.headdim, s.d_state}, "state_q");
    uint16_t *y = pointer<uint16_t>(a[10], at::kHalf, {s.batch, s.nheads, s.headdim}, "y");
    void *stream = stream_of(a[11]);
    return call([&] {
        return entry.decode_q8(&s, &sc, gate.get(), ss, o.x, o.B, o.C, o.dt, o.A, o.D, state, y, stream);
    });
}

// shape, scales, state_scales, state, state_q, stream
PyObject *quantize_state(PyObject *const *a)
{
    const quamba_ssd_shape_t s = shape_of(a[0]);
    const quamba_ssd_scales_t sc = scales_of(a[1]);
    const float *ss = pointer<float>(a[2], at::kFloat, {cells(s), s.d_state}, "state_scales");
    const float *state = pointer<float>(a[3], at::kFloat, {s.batch, s.nheads, s.headdim, s.d_state}, "state");
    int8_t *q = pointer<int8_t>(a[4], at::kChar, {s.batch, s.nheads, s.headdim, s.d_state}, "state_q");
    void *stream = stream_of(a[5]);
    return call([&] { return entry.quantize_state(&s, &sc, ss, state, q, stream); });
}

// y, s_y, out, stream
PyObject *hadamard(PyObject *const *a)
{
    const at::Tensor *y = tensor_or_null(a[0], "y");
    if (!y || y->dim() == 0) fail(PyExc_ValueError, "%s must be a tensor of rows", "y");
    const int64_t n = y->size(-1), rows = y->numel() / (n > 1 ? n : 1);
    if (rows == 0 && n > 0) return PyLong_FromLong(QUAMBA_OK);  // an empty tensor has no device pointer to pass
    const float s_y = number(a[1]);
    void *yp = device_pointer(y, "y");
    if (y->scalar_type() != at::kHalf) fail(PyExc_ValueError, "%s must have dtype torch.float16", "y");
    const at::Tensor *out = tensor_or_null(a[2], "out");
    void *op = device_pointer(out, "out");
    if (out && out->scalar_type() != at::kChar) fail(PyExc_ValueError, "%s must have dtype torch.int8", "out");
    if (out && out->sizes() != y->sizes()) fail(PyExc_ValueError, "%s must have the shape of y", "out");
    void *stream = stream_of(a[3]);
    return call([&] {
        return entry.hadamard(static_cast<const uint16_t *>(yp), rows, n > INT32_MAX ? 0 : (int32_t)n, s_y,
                              static_cast<int8_t *>(op), stream);
    });
}

// shape, scales, x, B, C, dt, A, D, y, init_state, final_state, stream, gate
PyObject *mamba1_scan(PyObject *const *a)
{
    const quamba_ssd_shape_t s = shape_of(a[0]);
    const quamba_ssd_scales_t sc = scales_of(a[1]);
    const int64_t b = s.batch, L = s.seqlen, D = s.headdim, N = s.d_state;
    const int8_t *x = pointer<int8_t>(a[2], at::kChar, {b, D, L}, "x");
    const int8_t *B = pointer<int8_t>(a[3], at::kChar, {b, N, L}, "B");
    const int8_t *C = pointer<int8_t>(a[4], at::kChar, {b, N, L}, "C");
    const float *dt = pointer<float>(a[5], at::kFloat, {b, D, L}, "dt");
    const float *A = pointer<float>(a[6], at::kFloat, {D, N}, "A");
    const float *Dk = pointer<float>(a[7], at::kFloat, {D}, "D");
    const float *init = pointer<float>(a[9], at::kFloat, {b, D, N}, "init_state");
    uint16_t *y = pointer<uint16_t>(a[8], at::kHalf, {b, D, L}, "y");
    float *fin = pointer<float>(a[10], at::kFloat, {b, D, N}, "final_state");
    void *stream = stream_of(a[11]);
    const GateArg gate(a[12], {b, D, L}, {b, D, L}, D);
    return call([&] { return entry.mamba1_scan(&s, &sc, gate.get(), x, B, C, dt, A, Dk, init, y, fin, stream); });
}

// shape, scales, x, B, C, dt, A, D, state, y, stream, gate
PyObject *mamba1_decode(PyObject *const *a)
{
    const quamba_ssd_shape_t s = shape_of(a[0]);
    const quamba_ssd_scales_t sc = scales_of(a[1]);
    const int64_t b = s.batch, D = s.headdim, N = s.d_state;
    const int8_t *x = pointer<int8_t>(a[2], at::kChar, {b, D}, "x");
    const int8_t *B = pointer<int8_t>(a[3], at::kChar, {b, N}, "B");
    const int8_t *C = pointer<int8_t>(a[4], at::kChar, {b, N}, "C");
    const float *dt = pointer<float>(a[5], at::kFloat, {b, D}, "dt");
    const float *A = pointer<float>(a[6], at::kFloat, {D, N}, "A");
    const float *Dk = pointer<float>(a[7], at::kFloat, {D}, "D");
    float *state = pointer<float>(a[8], at::kFloat, {b, D, N}, "state");
    uint16_t *y = pointer<uint16_t>(a[9], at::kHalf, {b, D}, "y");
    void *stream = stream_of(a[10]);
    const GateArg gate(a[11], {b, D}, {b, D}, D);
    return call([&] { return entry.mamba1_decode(&s, &sc, gate.get(), x, B, C, dt, A, Dk, state, y, stream); });
}

// shape, scales, xBC, weight, bias, in_w_scale, x_out, B_out, C_out, conv_state_in, conv_state_out, stream
PyObject *conv1d(PyObject *const *a)
{
    const quamba_ssd_shape_t s = shape_of(a[0]);
    const quamba_ssd_scales_t sc = scales_of(a[1]);
    const int64_t b = s.batch, L = s.seqlen, H = s.nheads, P = s.headdim, G = s.ngroups, N = s.d_state;
    const int64_t Ct = H * P + 2 * G * N;
    const int8_t *in = pointer<int8_t>(a[2], at::kChar, {b, L, Ct}, "xBC");
    const int8_t *weight = pointer<int8_t>(a[3], at::kChar, {Ct, 4}, "weight");
    const float *bias = pointer<float>(a[4], at::kFloat, {Ct}, "bias");
    const float scale = number(a[5]);
    const int8_t *st_in = pointer<int8_t>(a[9], at::kChar, {b, 3, Ct}, "conv_state_in");
    int8_t *x = pointer<int8_t>(a[6], at::kChar, {b, L, H, P}, "x_out");
    int8_t *B = pointer<int8_t>(a[7], at::kChar, {b, L, G, N}, "B_out");
    int8_t *C = pointer<int8_t>(a[8], at::kChar, {b, L, G, N}, "C_out");
    int8_t *st_out = pointer<int8_t>(a[10], at::kChar, {b, 3, Ct}, "conv_state_out");
    void *stream = stream_of(a[11]);
    return call([&] { return entry.conv1d(&s, &sc, in, weight, bias, scale, st_in, x, B, C, st_out, stream); });
}

// A device matrix whose rows lie any distance apart; values of a row lie side by side.
struct Matrix {
    void *p;
    int64_t rows, cols, stride;
    at::ScalarType type;
    Matrix(PyObject *o, const char *name)
    {
        const at::Tensor *t = tensor_or_null(o, name);
        if (!t || t->dim() != 2) fail(PyExc_ValueError, "%s must be a tensor of rows and columns", name);
        rows = t->size(0);
        cols = t->size(1);
        if (!t->is_cuda() || (cols > 1 && t->stride(1) != 1) || (rows > 1 && t->stride(0) < cols))
            fail(PyExc_ValueError, "%s must be a device tensor with rows of adjacent values that do not overlap", name);
        stride = rows > 1 ? t->stride(0) : cols;
        type = t->scalar_type();
        p = t->data_ptr();
    }
    // e4m3 codes, as such or as plain bytes
    uint8_t *codes(const char *name) const
    {
        if (type != at::kFloat8_e4m3fn && type != at::kByte)
            fail(PyExc_ValueError, "%s must have dtype torch.float8_e4m3fn or torch.uint8", name);
        return static_cast<uint8_t *>(p);
    }
    void expect(int64_t r, int64_t c, const char *name) const
    {
        if (rows != r || cols != c) {
            PyErr_Format(PyExc_ValueError, "%s must have shape (%lld, %lld), got (%lld, %lld)", name, (long long)r, (long long)c,
                         (long long)rows, (long long)cols);
            throw Fail();
        }
    }
};

int32_t dtype_of(at::ScalarType type, const char *name)
{
    switch (type) {
        case at::kFloat: return QUAMBA_F32;
        case at::kHalf: return QUAMBA_F16;
        case at::kBFloat16: return QUAMBA_BF16;
        default: fail(PyExc_ValueError, "%s must have dtype torch.float32, torch.float16 or torch.bfloat16", name);
    }
}

int64_t blocks(int64_t n, int64_t of) { return (n + of - 1) / of; }

int64_t integer(PyObject *o)
{
    const long long v = PyLong_AsLongLong(o);
    if (v == -1 && PyErr_Occurred()) throw Fail();
    return v;
}

int32_t small_integer(PyObject *o, const char *name)
{
    const int64_t v = integer(o);
    if (v < INT32_MIN || v > INT32_MAX) fail(PyExc_ValueError, "%s does not fit 32 bits", name);
    return (int32_t)v;
}

// x, q, scales, block_rows, stream
PyObject *fp8_quantize(PyObject *const *a)
{
    const Matrix x(a[0], "x"), q(a[1], "q");
    const int32_t block_rows = small_integer(a[3], "block_rows"), type = dtype_of(x.type, "x");
    uint8_t *codes = q.codes("q");
    q.expect(x.rows, x.cols, "q");
    float *scales = pointer<float>(a[2], at::kFloat, {blocks(x.rows, block_rows > 0 ? block_rows : 1), blocks(x.cols, 128)}, "scales");
    void *stream = stream_of(a[4]);
    return call([&] { return entry.fp8_quantize(x.rows, x.cols, block_rows, x.p, type, x.stride, codes, q.stride, scales, stream); });
}

// x, x_scales, w, w_scales, y, workspace, stream
PyObject *fp8_matmul(PyObject *const *a)
{
    const Matrix x(a[0], "x"), w(a[2], "w"), y(a[4], "y");
    const uint8_t *xc = x.codes("x"), *wc = w.codes("w");
    w.expect(w.rows, x.cols, "w");
    y.expect(x.rows, w.rows, "y");
    const int32_t type = dtype_of(y.type, "y");
    const float *xs = pointer<float>(a[1], at::kFloat, {x.rows, blocks(x.cols, 128)}, "x_scales");
    const float *ws = pointer<float>(a[3], at::kFloat, {blocks(w.rows, 128), blocks(x.cols, 128)}, "w_scales");
    const at::Tensor *space = tensor_or_null(a[5], "workspace");
    void *sp = device_pointer(space, "workspace");
    const size_t bytes = space ? (size_t)space->numel() * space->element_size() : 0;
    void *stream = stream_of(a[6]);
    return call([&] {
        return entry.fp8_matmul(x.rows, w.rows, x.cols, xc, x.stride, xs, wc, w.stride, ws, y.p, type, y.stride, sp, bytes, stream);
    });
}

// logits, scores, out_scores, out_parents, out_tokens, workspace, finished, pad_token, stream
PyObject *beam_select(PyObject *const *a)
{
    const at::Tensor *logits = tensor_or_null(a[0], "logits"), *best = tensor_or_null(a[2], "out_scores");
    if (!logits || logits->dim() != 3) fail(PyExc_ValueError, "%s must be a tensor [batch, beams, vocab]", "logits");
    if (!best || best->dim() != 2) fail(PyExc_ValueError, "%s must be a tensor [batch, count]", "out_scores");
    const int64_t b = logits->size(0), K = logits->size(1), V = logits->size(2), count = best->size(1);
    if (b > INT32_MAX || K > INT32_MAX || V > INT32_MAX || count > INT32_MAX) return PyLong_FromLong(QUAMBA_ESHAPE);
    const int64_t stride = K > 1 ? logits->stride(1) : b > 1 ? logits->stride(0) : V;
    if (!logits->is_cuda() || (V > 1 && logits->stride(2) != 1) || (K > 1 && b > 1 && logits->stride(0) != K * stride))
        fail(PyExc_ValueError, "%s must be a device tensor with rows of adjacent values, one distance apart", "logits");
    const int32_t type = dtype_of(logits->scalar_type(), "logits");
    const float *scores = pointer<float>(a[1], at::kFloat, {b, K}, "scores");
    float *out = pointer<float>(a[2], at::kFloat, {b, count}, "out_scores");
    int32_t *parents = pointer<int32_t>(a[3], at::kInt, {b, count}, "out_parents");
    int32_t *tokens = pointer<int32_t>(a[4], at::kInt, {b, count}, "out_tokens");
    const at::Tensor *space = tensor_or_null(a[5], "workspace");
    void *sp = device_pointer(space, "workspace");
    const size_t bytes = space ? (size_t)space->numel() * space->element_size() : 0;
    const at::Tensor *finished = tensor_or_null(a[6], "finished");
    const bool flags = finished && finished->scalar_type() == at::kBool;
    const uint8_t *done = pointer<uint8_t>(a[6], flags ? at::kBool : at::kByte, {b, K}, "finished");
    const int32_t pad = small_integer(a[7], "pad_token");
    void *stream = stream_of(a[8]);
    void *lp = logits->data_ptr();
    return call([&] {
        return entry.beam_select((int32_t)b, (int32_t)K, (int32_t)V, (int32_t)count, lp, type, stride, scores, done, pad, out, parents,
                                 tokens, sp, bytes, stream);
    });
}

// parents, caches (a sequence of tensors [batch, beams, ...]), stream
PyObject *beam_reorder(PyObject *const *a)
{
    const at::Tensor *t = tensor_or_null(a[0], "parents");
    if (!t || t->dim() != 2) fail(PyExc_ValueError, "%s must be a tensor [batch, beams]", "parents");
    const int64_t b = t->size(0), K = t->size(1);
    if (b > INT32_MAX || K > INT32_MAX) return PyLong_FromLong(QUAMBA_ESHAPE);
    const int32_t *parents = pointer<int32_t>(a[0], at::kInt, {b, K}, "parents");
    Ref list(PySequence_Fast(a[1], "caches must be a sequence of tensors"));
    const Py_ssize_t n = PySequence_Fast_GET_SIZE(list.o);
    if (n > INT32_MAX) return PyLong_FromLong(QUAMBA_ESHAPE);
    std::vector<quamba_beam_cache_t> caches((size_t)n);
    for (Py_ssize_t i = 0; i < n; ++i) {
        const at::Tensor *c = tensor_or_null(PySequence_Fast_GET_ITEM(list.o, i), "every cache");
        if (!c || c->dim() < 2 || c->size(0) != b || c->size(1) != K)
            fail(PyExc_ValueError, "%s must be a tensor [batch, beams, ...]", "every cache");
        caches[i].data = device_pointer(c, "every cache");
        caches[i].bytes = b && K ? (int64_t)(c->numel() / (b * K) * c->element_size()) : 0;
    }
    void *stream = stream_of(a[2]);
    return call([&] { return entry.beam_reorder((int32_t)b, (int32_t)K, parents, (int32_t)n, caches.data(), stream); });
}

template <PyObject *(*F)(PyObject *const *), int N>
PyObject *method(PyObject *, PyObject *const *a, Py_ssize_t n)
{
    try {
        need(n, N);
        return F(a);
    } catch (const Fail &) {
        return nullptr;
    } catch (const std::exception &e) {  // torch's own errors (a tensor without storage, a lost device)
        PyErr_SetString(PyExc_RuntimeError, e.what());
        return nullptr;
    }
}

// The addresses of the library's functions, in the order of Entry, and what binding.py has for the objects above.
PyObject *bind(PyObject *, PyObject *const *a, Py_ssize_t n)
{
    constexpr int kEntries = 13;
    PyObject **const objects[] = {&shape_type, &scales_type, &gate_struct_type, &device_scales_type, &gate_type, &address_of};
    constexpr int kObjects = sizeof(objects) / sizeof(objects[0]);
    void *p[kEntries];
    if (n != kEntries + kObjects) {
        PyErr_Format(PyExc_TypeError, "expected %d addresses and %d objects", kEntries, kObjects);
        return nullptr;
    }
    for (int i = 0; i < kEntries; ++i) {
        p[i] = PyLong_AsVoidPtr(a[i]);
        if (PyErr_Occurred()) return nullptr;
    }
    for (int i = 0; i < kObjects; ++i) {
        if (i + 1 < kObjects ? !PyType_Check(a[kEntries + i]) : !PyCallable_Check(a[kEntries + i])) {
            PyErr_SetString(PyExc_TypeError, "expected types and a function");
            return nullptr;
        }
        Py_INCREF(a[kEntries + i]);
        Py_XDECREF(*objects[i]);
        *objects[i] = a[kEntries + i];
    }
    static_assert(sizeof(Entry) == sizeof(p), "one address per entry point");
    memcpy(&entry, p, sizeof(entry));
    Py_RETURN_NONE;
}

#define QUAMBA_METHOD(name, nargs) \
    {#name, reinterpret_cast<PyCFunction>(reinterpret_cast<void (*)()>(&method<name, nargs>)), METH_FASTCALL, nullptr}

PyMethodDef methods[] = {
    {"bind", reinterpret_cast<PyCFunction>(reinterpret_cast<void (*)()>(&bind)), METH_FASTCALL, nullptr},
    QUAMBA_METHOD(prefill, 14),
    QUAMBA_METHOD(prefill_noalloc, 12),
    QUAMBA_METHOD(decode, 12),
    QUAMBA_METHOD(decode_q8, 13),
    QUAMBA_METHOD(quantize_state, 6),
    QUAMBA_METHOD(hadamard, 4),
    QUAMBA_METHOD(mamba1_scan, 13),
    QUAMBA_METHOD(mamba1_decode, 12),
    QUAMBA_METHOD(conv1d, 12),
    QUAMBA_METHOD(fp8_quantize, 5),
    QUAMBA_METHOD(fp8_matmul, 7),
    QUAMBA_METHOD(beam_select, 9),
    QUAMBA_METHOD(beam_reorder, 3),
    {nullptr, nullptr, 0, nullptr}};

PyModuleDef module = {PyModuleDef_HEAD_INIT, "_bind", nullptr, -1, methods, nullptr, nullptr, nullptr, nullptr};

}  // namespace

PyMODINIT_FUNC PyInit__bind(void)
{
    const struct { PyObject **to; const char *text; } names[] = {
        {&s_tensors, "tensors"}, {&s_struct, "struct"}, {&s_cuda_stream, "cuda_stream"}, {&s_z, "z"},
        {&s_z_scale, "z_scale"}, {&s_dt_q, "dt_q"}, {&s_dt_scale, "dt_scale"}, {&s_dt_bias, "dt_bias"}};
    for (const auto &e : names)
        if (!(*e.to = PyUnicode_InternFromString(e.text))) return nullptr;
    return PyModule_Create(&module);
}
