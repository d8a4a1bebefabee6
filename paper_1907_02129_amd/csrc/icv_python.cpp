// Argument marshalling of the operators on sequences and in 8-bit floating point: tensors checked against the problem's
// description (the library sees addresses only), and the call.  In C++ because a small call's time is these checks: five to
// ten tensors, each asked for its type, device, sizes, strides and address, took 2 us of a 6.6 us call from Python,
// where the kernel takes 4.  binding.py is the interface; nothing here launches or computes anything of its own.
#define PY_SSIZE_T_CLEAN
#include <Python.h>
#include <torch/csrc/autograd/python_variable.h>
#include "icv.h"

namespace {

struct Raised {};          // a Python exception is set

[[noreturn]] void refuse(const char* name, PyObject* t, const char* expected)
{
    PyObject* parts[4] = {PyObject_GetAttrString(t, "dtype"), PyObject_GetAttrString(t, "shape"), PyObject_CallMethod(t, "stride", nullptr),
                          PyObject_GetAttrString(t, "device")};
    if (parts[0] && parts[1] && parts[2] && parts[3])
        PyErr_Format(PyExc_ValueError, "%s: %s expected, got %S, %S, strides %S, on %S", name, expected, parts[0], parts[1], parts[2], parts[3]);
    for (PyObject* p : parts) Py_XDECREF(p);
    throw Raised{};
}

const at::Tensor& tensor(const char* name, PyObject* o)
{
    if (!THPVariable_Check(o)) {
        PyErr_Format(PyExc_TypeError, "%s: a tensor expected, got %R", name, (PyObject*)Py_TYPE(o));
        throw Raised{};
    }
    return THPVariable_Unpack(o);
}

bool on(const at::Tensor& t, int device) { return t.is_cuda() && t.get_device() == device; }

// Address of a [rows][cols] matrix whose rows lie `stride` elements apart; codes: bytes, as uint8 or float8_e4m3fn.
void* matrix(const char* name, PyObject* o, int64_t rows, int64_t cols, int64_t stride, at::ScalarType type, int device)
{
    const at::Tensor& t = tensor(name, o);
    const bool right = t.scalar_type() == type || (type == at::kByte && t.scalar_type() == at::kFloat8_e4m3fn);
    if (!right || !on(t, device) || t.dim() != 2 || t.size(0) < rows || t.size(1) < cols || (rows > 1 && t.stride(0) != stride) ||
        (cols > 1 && t.stride(1) != 1)) {
        char want[160];
        snprintf(want, sizeof(want), "a %s matrix of at least %lld x %lld, strides (%lld, 1), on GPU %d", at::toString(type), (long long)rows,
                 (long long)cols, (long long)stride, device);
        refuse(name, o, want);
    }
    return t.data_ptr();
}

// Address of a contiguous tensor of at least n elements; None for none.
void* vector(const char* name, PyObject* o, int64_t n, at::ScalarType type, int device)
{
    if (o == Py_None) return nullptr;
    const at::Tensor& t = tensor(name, o);
    if (t.scalar_type() != type || !on(t, device) || t.numel() < n || !t.is_contiguous()) {
        char want[160];
        snprintf(want, sizeof(want), "a contiguous %s tensor of at least %lld elements on GPU %d", at::toString(type), (long long)n, device);
        refuse(name, o, want);
    }
    return t.data_ptr();
}

// Address of at least `slots` state slots of per_slot elements, each contiguous, slot_stride apart; None for none.
void* state_slots(const char* name, PyObject* o, int64_t slots, int64_t per_slot, int64_t slot_stride, at::ScalarType type, int device)
{
    if (o == Py_None || per_slot == 0) return nullptr;
    const at::Tensor& t = tensor(name, o);
    bool right = t.scalar_type() == type && on(t, device) && t.dim() >= 2 && t.size(0) >= slots && t.numel() == t.size(0) * per_slot &&
                 (slots <= 1 || t.stride(0) == slot_stride);
    int64_t inner = 1;
    for (int64_t d = t.dim() - 1; right && d > 0; d--) {
        if (t.size(d) > 1 && t.stride(d) != inner) right = false;
        inner *= t.size(d);
    }
    if (!right) {
        char want[200];
        snprintf(want, sizeof(want), "%lld slots of %lld elements of %s, %lld apart, on GPU %d", (long long)slots, (long long)per_slot,
                 at::toString(type), (long long)slot_stride, device);
        refuse(name, o, want);
    }
    return t.data_ptr();
}

// The library's functions and binding.py's struct types, handed over once.
struct {
    decltype(&icv_causal_conv1d) conv;
    decltype(&icv_selective_scan_workspace_bytes) scan_bytes;
    decltype(&icv_selective_scan) scan;
    decltype(&icv_quantize_fp8) quantize;
    decltype(&icv_matmul_fp8) matmul;
} lib;
PyObject *kSequences, *kConv, *kScan, *kQuantize, *kMatmul;

// A copy of the struct behind a ctypes object of the given type.
template <typename T>
T params(PyObject* o, PyObject* type)
{
    const int is = PyObject_IsInstance(o, type);
    if (is < 0) throw Raised{};
    if (!is) {
        PyErr_Format(PyExc_TypeError, "%R expected, got %R", type, (PyObject*)Py_TYPE(o));
        throw Raised{};
    }
    Py_buffer view;
    if (PyObject_GetBuffer(o, &view, PyBUF_SIMPLE) < 0) throw Raised{};
    T p;
    const bool fits = view.len == (Py_ssize_t)sizeof(T);
    if (fits) memcpy(&p, view.buf, sizeof(T));
    PyBuffer_Release(&view);
    if (!fits) {
        PyErr_SetString(PyExc_TypeError, "struct of another size");
        throw Raised{};
    }
    return p;
}

icv_sequences sequences(PyObject* o, int device)
{
    const icv_sequences s = params<icv_sequences>(o, kSequences);
    static PyObject* const name = PyUnicode_InternFromString("device");
    PyObject* d = PyObject_GetAttr(o, name);
    if (!d) throw Raised{};
    const long its = PyLong_AsLong(d);
    Py_DECREF(d);
    if (its == -1 && PyErr_Occurred()) throw Raised{};
    if (its >= 0 && its != device) {
        PyErr_SetString(PyExc_ValueError, "icv takes tensors of one device");
        throw Raised{};
    }
    return s;
}

at::ScalarType row_type(int32_t dtype) { return dtype == ICV_F32 ? at::kFloat : at::kBFloat16; }       // others: refused by the library
int64_t or_dense(int64_t stride, int64_t dense) { return stride ? stride : dense; }

// Each takes the device and the raw stream, then binding.py's arguments in their order; returns the status.
long conv(int dev, void* stream, PyObject* const* a)
{
    const icv_causal_conv_params p = params<icv_causal_conv_params>(a[0], kConv);
    const icv_sequences s = sequences(a[1], dev);
    const at::ScalarType t = row_type(p.dtype);
    const int64_t D = p.channels, slot = ((int64_t)p.taps - 1) * D;
    void* x = matrix("input", a[2], s.tokens, D, or_dense(p.in_row_stride, D), t, dev);
    void* f = vector("filter", a[3], D * p.taps, t, dev);
    void* b = vector("bias", a[4], D, at::kFloat, dev);
    void* st = state_slots("state", a[5], p.state_slots, slot, or_dense(p.state_slot_stride, slot), t, dev);
    void* y = matrix("output", a[6], s.tokens, D, or_dense(p.out_row_stride, D), t, dev);
    return lib.conv(&p, &s, x, f, (const float*)b, st, y, stream);
}

long scan(int dev, void* stream, PyObject* const* a)
{
    const icv_scan_params p = params<icv_scan_params>(a[0], kScan);
    const icv_sequences s = sequences(a[1], dev);
    const at::ScalarType t = row_type(p.dtype);
    const int64_t n = s.tokens, D = p.channels, N = p.states, bc = (int64_t)p.groups * N;
    icv_scan_tensors q;
    q.x = matrix("x", a[2], n, D, or_dense(p.x_row_stride, D), t, dev);
    q.dt = matrix("dt", a[3], n, D, or_dense(p.dt_row_stride, D), t, dev);
    q.A = (const float*)vector("A", a[4], D * N, at::kFloat, dev);
    q.B = matrix("B", a[5], n, bc, or_dense(p.b_row_stride, bc), t, dev);
    q.C = matrix("C", a[6], n, bc, or_dense(p.c_row_stride, bc), t, dev);
    q.D = (const float*)vector("D", a[7], D, at::kFloat, dev);
    q.z = a[8] == Py_None ? nullptr : matrix("z", a[8], n, D, or_dense(p.z_row_stride, D), t, dev);
    q.dt_bias = (const float*)vector("dt_bias", a[9], D, at::kFloat, dev);
    q.state = (float*)state_slots("state", a[10], p.state_slots, D * N, or_dense(p.state_slot_stride, D * N), at::kFloat, dev);
    q.out = matrix("output", a[11], n, D, or_dense(p.out_row_stride, D), t, dev);
    void* workspace = nullptr;
    if (const size_t need = lib.scan_bytes(&p, &s)) {
        if (a[12] != Py_None) {
            const at::Tensor& w = tensor("workspace", a[12]);
            if (on(w, dev) && w.is_contiguous() && (size_t)w.nbytes() >= need) workspace = w.data_ptr();
        }
        if (!workspace) {
            PyErr_Format(PyExc_ValueError, "workspace: a contiguous tensor of at least %zu bytes on GPU %d expected", need, dev);
            throw Raised{};
        }
    }
    return lib.scan(&p, &s, &q, workspace, stream);
}

long quantize(int dev, void* stream, PyObject* const* a)
{
    const icv_quantize_params p = params<icv_quantize_params>(a[0], kQuantize);
    const int64_t kb = ((int64_t)p.depth + 127) / 128, br = p.block_rows > 0 ? p.block_rows : 1, M = p.rows;
    void* x = matrix("input", a[1], M, p.depth, or_dense(p.in_row_stride, p.depth), row_type(p.dtype), dev);
    void* codes = matrix("codes", a[2], M, 128 * kb, or_dense(p.code_row_stride, 128 * kb), at::kByte, dev);
    void* scales = vector("scales", a[3], kb * ((M + br - 1) / br), at::kFloat, dev);
    return lib.quantize(&p, x, codes, (float*)scales, stream);
}

long matmul(int dev, void* stream, PyObject* const* a)
{
    const icv_matmul_params p = params<icv_matmul_params>(a[0], kMatmul);
    const int64_t kb = ((int64_t)p.depth + 127) / 128, M = p.rows, N = p.cols;
    void* x = matrix("a", a[1], M, 128 * kb, or_dense(p.a_row_stride, 128 * kb), at::kByte, dev);
    void* xs = vector("a_scales", a[2], kb * M, at::kFloat, dev);
    void* w = matrix("b", a[3], N, 128 * kb, or_dense(p.b_row_stride, 128 * kb), at::kByte, dev);
    void* ws = vector("b_scales", a[4], kb * ((N + 127) / 128), at::kFloat, dev);
    void* b = vector("bias", a[5], N, at::kFloat, dev);
    void* y = matrix("output", a[6], M, N, or_dense(p.out_row_stride, N), (p.out_type & 255) == ICV_OUT_ACC ? at::kFloat : at::kBFloat16, dev);
    return lib.matmul(&p, x, (const float*)xs, w, (const float*)ws, (const float*)b, y, stream);
}

template <long (*F)(int, void*, PyObject* const*), int N>
PyObject* call(PyObject*, PyObject* const* args, Py_ssize_t n)
{
    if (n != N + 2) {
        PyErr_Format(PyExc_TypeError, "%d arguments expected, got %zd", N + 2, n);
        return nullptr;
    }
    const long device = PyLong_AsLong(args[0]);
    void* stream = PyLong_AsVoidPtr(args[1]);
    if (PyErr_Occurred()) return nullptr;
    try {
        return PyLong_FromLong(F((int)device, stream, args + 2));
    } catch (const Raised&) {
    } catch (const std::exception& e) {
        PyErr_SetString(PyExc_RuntimeError, e.what());
    }
    return nullptr;
}

// bind(addresses of the five functions in the order of `lib`, the five struct types)
PyObject* bind(PyObject*, PyObject* args)
{
    unsigned long long f[5];
    PyObject* t[5];
    if (!PyArg_ParseTuple(args, "KKKKKOOOOO", f, f + 1, f + 2, f + 3, f + 4, t, t + 1, t + 2, t + 3, t + 4)) return nullptr;
    lib.conv = (decltype(lib.conv))f[0];
    lib.scan_bytes = (decltype(lib.scan_bytes))f[1];
    lib.scan = (decltype(lib.scan))f[2];
    lib.quantize = (decltype(lib.quantize))f[3];
    lib.matmul = (decltype(lib.matmul))f[4];
    PyObject** types[5] = {&kSequences, &kConv, &kScan, &kQuantize, &kMatmul};
    for (int i = 0; i < 5; i++) {
        Py_INCREF(t[i]);
        Py_XSETREF(*types[i], t[i]);
    }
    Py_RETURN_NONE;
}

PyMethodDef kMethods[] = {
    {"bind", bind, METH_VARARGS, nullptr},
    {"causal_conv1d", (PyCFunction)(void (*)())call<conv, 7>, METH_FASTCALL, nullptr},
    {"selective_scan", (PyCFunction)(void (*)())call<scan, 13>, METH_FASTCALL, nullptr},
    {"quantize_fp8", (PyCFunction)(void (*)())call<quantize, 4>, METH_FASTCALL, nullptr},
    {"matmul_fp8", (PyCFunction)(void (*)())call<matmul, 7>, METH_FASTCALL, nullptr},
    {nullptr, nullptr, 0, nullptr}};
PyModuleDef kModule = {PyModuleDef_HEAD_INIT, "_icv_python", nullptr, -1, kMethods, nullptr, nullptr, nullptr, nullptr};

}  // namespace

PyMODINIT_FUNC PyInit__icv_python(void) { return PyModule_Create(&kModule); }
