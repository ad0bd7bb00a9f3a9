// Host side of the Python binding: the checks of the tensors of a call (on the GPU, contiguous, of the expected type and
// shape) and their addresses, and the current stream, without a Python call per property.  A pass over the input layer of 8
// shards of N=512 h=1024 hands over 28 tensors; their checks in Python took longer than its kernels: 30.3 us a pass with them,
// 15.5 us so.  N=98 h=128 V=2929 p=8 fp32 step: 85 -> 53 us.
//
// Every function returns None where a check fails or anything is unusual (a subclass of Tensor, a tensor without memory of its
// own): the caller then goes through the same checks in Python, which say what is wrong.  Nothing is kept between calls.
#define PY_SSIZE_T_CLEAN
#include <Python.h>

#include <c10/hip/HIPFunctions.h>
#include <c10/hip/HIPStream.h>
#include <torch/csrc/Dtype.h>
#include <torch/csrc/autograd/python_variable.h>
#include <torch/version.h>

#include <cstdint>
#include <cstring>
#include <initializer_list>

namespace {

bool type_ok(const at::Tensor& t, PyObject* dtypes) {
    if (dtypes == Py_None) return true;
    if (!PyTuple_Check(dtypes)) return false;
    for (Py_ssize_t i = 0; i < PyTuple_GET_SIZE(dtypes); ++i) {
        PyObject* d = PyTuple_GET_ITEM(dtypes, i);
        if (THPDtype_Check(d) && reinterpret_cast<THPDtype*>(d)->scalar_type == t.scalar_type()) return true;
    }
    return false;
}

bool shape_ok(const at::Tensor& t, PyObject* shape) {
    if (shape == Py_None) return true;
    if (!PyTuple_Check(shape) || PyTuple_GET_SIZE(shape) != t.dim()) return false;
    for (int64_t i = 0; i < t.dim(); ++i) {
        const long long n = PyLong_AsLongLong(PyTuple_GET_ITEM(shape, i));
        if (n != t.size(i)) {
            PyErr_Clear();
            return false;
        }
    }
    return true;
}

// bf16 data may come as bit patterns.
bool bf16_like(at::ScalarType t) { return t == at::kBFloat16 || t == at::kShort || t == at::kUInt16; }
int vp_dtype_of(at::ScalarType t) { return t == at::kFloat ? 0 : bf16_like(t) ? 1 : -1; }

// The address of the tensor's first element in `out`, if it passes all checks.
bool address(PyObject* o, PyObject* dtypes, PyObject* shape, uint64_t& out) {
    if (!THPVariable_CheckExact(o)) return false;
    try {
        const at::Tensor& t = THPVariable_Unpack(o);
        if (!t.defined() || !t.is_cuda() || !t.is_contiguous() || !type_ok(t, dtypes) || !shape_ok(t, shape)) return false;
        out = reinterpret_cast<uint64_t>(t.data_ptr());
        return true;
    } catch (...) {
        return false;
    }
}

// ptr(tensor, dtypes or None, shape or None) -> int
PyObject* ptr(PyObject*, PyObject* const* a, Py_ssize_t n) {
    uint64_t p;
    if (n != 3 || !address(a[0], a[1], a[2], p)) Py_RETURN_NONE;
    return PyLong_FromUnsignedLongLong(p);
}

// ptrs(list of tensors, dtypes or None, shape of each or list of their shapes) -> bytes: an array of pointers
PyObject* ptrs(PyObject*, PyObject* const* a, Py_ssize_t n) {
    if (n != 3 || !PyList_Check(a[0])) Py_RETURN_NONE;
    const Py_ssize_t k = PyList_GET_SIZE(a[0]);
    const bool each = PyList_Check(a[2]);
    if (each && PyList_GET_SIZE(a[2]) != k) Py_RETURN_NONE;
    PyObject* out = PyBytes_FromStringAndSize(nullptr, k * (Py_ssize_t)sizeof(uint64_t));
    if (!out) return nullptr;
    for (Py_ssize_t i = 0; i < k; ++i) {
        uint64_t p;
        if (!address(PyList_GET_ITEM(a[0], i), a[1], each ? PyList_GET_ITEM(a[2], i) : a[2], p)) {
            Py_DECREF(out);
            Py_RETURN_NONE;
        }
        std::memcpy(PyBytes_AS_STRING(out) + i * sizeof(uint64_t), &p, sizeof p);
    }
    return out;
}

// same_shapes(list of tensors) -> bool
PyObject* same_shapes(PyObject*, PyObject* list) {
    if (!PyList_Check(list)) Py_RETURN_NONE;
    try {
        for (Py_ssize_t i = 0; i < PyList_GET_SIZE(list); ++i) {
            if (!THPVariable_CheckExact(PyList_GET_ITEM(list, i))) Py_RETURN_NONE;
            if (THPVariable_Unpack(PyList_GET_ITEM(list, i)).sizes() != THPVariable_Unpack(PyList_GET_ITEM(list, 0)).sizes())
                Py_RETURN_FALSE;
        }
    } catch (...) {
        Py_RETURN_NONE;
    }
    Py_RETURN_TRUE;
}

// on_current_device(tuple of tensors or None) -> True, where all tensors are on the current device
PyObject* on_current_device(PyObject*, PyObject* ts) {
    if (!PyTuple_Check(ts)) Py_RETURN_NONE;
    try {
        const auto here = c10::hip::current_device();
        for (Py_ssize_t i = 0; i < PyTuple_GET_SIZE(ts); ++i) {
            PyObject* o = PyTuple_GET_ITEM(ts, i);
            if (o == Py_None) continue;
            if (!THPVariable_CheckExact(o)) Py_RETURN_NONE;
            const at::Tensor& t = THPVariable_Unpack(o);
            if (!t.defined() || !t.is_cuda() || t.get_device() != here) Py_RETURN_NONE;
        }
    } catch (...) {
        Py_RETURN_NONE;
    }
    Py_RETURN_TRUE;
}

// The memory of an object of the buffer protocol (a ctypes array).
struct Buffer {
    Py_buffer view{};
    explicit Buffer(PyObject* o) {
        if (PyObject_GetBuffer(o, &view, PyBUF_SIMPLE) != 0) PyErr_Clear();
    }
    ~Buffer() { PyBuffer_Release(&view); }
    template <typename T>
    const T* of(Py_ssize_t n) const { return view.buf && view.len == n * (Py_ssize_t)sizeof(T) ? static_cast<const T*>(view.buf) : nullptr; }
};

// unchanged(list of tensors, their addresses, numbers of elements and vp_dtypes as arrays) -> True, where they still are as the
// arrays say (13 ns a tensor)
PyObject* unchanged(PyObject*, PyObject* const* a, Py_ssize_t n) {
    if (n != 4 || !PyList_Check(a[0])) Py_RETURN_NONE;
    const Py_ssize_t k = PyList_GET_SIZE(a[0]);
    if (k == 0) Py_RETURN_NONE;
    const Buffer buffers[3] = {Buffer(a[1]), Buffer(a[2]), Buffer(a[3])};
    const uint64_t* ptrs = buffers[0].of<uint64_t>(k);
    const int64_t* counts = buffers[1].of<int64_t>(k);
    const int32_t* dts = buffers[2].of<int32_t>(k);
    if (!ptrs || !counts || !dts) Py_RETURN_NONE;
    try {
        for (Py_ssize_t i = 0; i < k; ++i) {
            PyObject* o = PyList_GET_ITEM(a[0], i);
            if (!THPVariable_CheckExact(o)) Py_RETURN_NONE;
            const at::Tensor& t = THPVariable_Unpack(o);
            if (!t.defined() || t.numel() != counts[i] || vp_dtype_of(t.scalar_type()) != dts[i] || !t.is_contiguous()) Py_RETURN_NONE;
            if (counts[i] && reinterpret_cast<uint64_t>(t.data_ptr()) != ptrs[i]) Py_RETURN_NONE;
        }
    } catch (...) {
        Py_RETURN_NONE;
    }
    Py_RETURN_TRUE;
}

// stream() -> int: the current stream of the current device
PyObject* stream(PyObject*, PyObject*) {
    try {
        return PyLong_FromVoidPtr(reinterpret_cast<void*>(c10::hip::getCurrentHIPStream().stream()));
    } catch (...) {
        Py_RETURN_NONE;
    }
}

// ---- whole calls: checks, addresses and the call itself, without a Python call per tensor (a single token through the norms
// around a block: 6.7 us of host time with them, 4.3 us so).

// Checks the tensors of one call and collects their addresses.
struct Call {
    at::DeviceIndex here = c10::hip::current_device();
    bool ok = true;

    // vp_dtype of a tensor
    int dtype(PyObject* o) {
        const int dt = THPVariable_CheckExact(o) ? vp_dtype_of(THPVariable_Unpack(o).scalar_type()) : -1;
        if (dt < 0) ok = false;
        return dt;
    }
    // the address of a tensor of the shape and type; None is null
    void* at(PyObject* o, int dtype, std::initializer_list<int64_t> shape) {
        if (o == Py_None || !ok) return nullptr;
        ok = false;
        if (!THPVariable_CheckExact(o)) return nullptr;
        const at::Tensor& t = THPVariable_Unpack(o);
        if (!t.defined() || !t.is_cuda() || t.get_device() != here || !t.is_contiguous()) return nullptr;
        if (dtype == 0 ? t.scalar_type() != at::kFloat : !bf16_like(t.scalar_type())) return nullptr;
        if (t.sizes() != at::IntArrayRef(shape.begin(), shape.size())) return nullptr;
        ok = true;
        return t.data_ptr();
    }
    // N and h of a matrix; a gate's rows (0 for None; a gate without rows has no address and would be taken for none)
    int64_t size(PyObject* o, int64_t d) {
        if (o == Py_None) return 0;
        if (!THPVariable_CheckExact(o) || !THPVariable_Unpack(o).defined() || THPVariable_Unpack(o).dim() != 2 ||
            THPVariable_Unpack(o).size(d) == 0) {
            ok = false;
            return 0;
        }
        return THPVariable_Unpack(o).size(d);
    }
    // the stream to launch on: the current one for None
    void* stream(PyObject* o) {
        if (o == Py_None) return c10::hip::getCurrentHIPStream().stream();
        if (!PyLong_CheckExact(o)) {
            ok = false;
            return nullptr;
        }
        return number(PyLong_AsVoidPtr(o));
    }
    double real(PyObject* o) { return number(PyFloat_AsDouble(o)); }
    long integer(PyObject* o) { return number(PyLong_AsLong(o)); }
    void* pointer(PyObject* o) { return number(PyLong_AsVoidPtr(o)); }

private:
    template <typename T>
    T number(T v) {
        if (PyErr_Occurred()) {
            PyErr_Clear();
            ok = false;
        }
        return v;
    }
};

using Forward = int (*)(const void*, const void*, const void*, int64_t, const void*, const void*, const void*, const void*, int64_t,
                        int64_t, int, uint32_t, float, float, void*, void*, float*, void*);
using Backward = int (*)(const void*, int, const void*, const void*, const void*, const void*, int64_t, const void*, const void*,
                         const void*, const float*, int64_t, int64_t, int, uint32_t, float, int, void*, void*, float*, float*,
                         float*, float*, float*, void*, size_t, void*);

// block_norm_fwd(function, x, y, H, r, stats, gate, w, b, w_post, b_post, scale, eps, flags, stream) -> status
PyObject* block_norm_fwd(PyObject*, PyObject* const* a, Py_ssize_t n) {
    if (n != 15) Py_RETURN_NONE;
    int status = 0;
    try {
        Call c;
        const auto f = reinterpret_cast<Forward>(c.pointer(a[0]));
        const int64_t N = c.size(a[1], 0), h = c.size(a[1], 1), rows = c.size(a[6], 0);
        if (!c.ok || a[1] == Py_None) Py_RETURN_NONE;
        const int dt = c.dtype(a[1]);
        void *x = c.at(a[1], dt, {N, h}), *y = c.at(a[2], dt, {N, h}), *H = c.at(a[3], dt, {N, h}), *r = c.at(a[4], dt, {N, h});
        void *stats = c.at(a[5], 0, {4, N}), *gate = c.at(a[6], dt, {rows, h}), *w = c.at(a[7], dt, {h}), *b = c.at(a[8], dt, {h});
        void *w_post = c.at(a[9], dt, {h}), *b_post = c.at(a[10], dt, {h});
        const float scale = (float)c.real(a[11]), eps = (float)c.real(a[12]);
        const uint32_t flags = (uint32_t)c.integer(a[13]);
        void* stream = c.stream(a[14]);
        if (!c.ok) Py_RETURN_NONE;
        Py_BEGIN_ALLOW_THREADS
        status = f(x, y, gate, rows, w_post, b_post, w, b, N, h, dt, flags, scale, eps, r, H, static_cast<float*>(stats), stream);
        Py_END_ALLOW_THREADS
    } catch (...) {
        Py_RETURN_NONE;
    }
    return PyLong_FromLong(status);
}

// block_norm_bwd(function, dH, r, y, stats, dx, dy, dr, gate, w, w_post, b_post, scale, flags, dgate, dw, db, dw_post, db_post,
//                workspace, stream) -> status
PyObject* block_norm_bwd(PyObject*, PyObject* const* a, Py_ssize_t n) {
    if (n != 21) Py_RETURN_NONE;
    int status = 0;
    try {
        Call c;
        const auto f = reinterpret_cast<Backward>(c.pointer(a[0]));
        const int64_t N = c.size(a[2], 0), h = c.size(a[2], 1), rows = c.size(a[8], 0);
        if (!c.ok || a[2] == Py_None || !THPVariable_CheckExact(a[19])) Py_RETURN_NONE;
        const int dt = c.dtype(a[2]), dH_dt = c.dtype(a[1]), grad_dt = c.dtype(a[5]);
        void *dH = c.at(a[1], dH_dt, {N, h}), *r = c.at(a[2], dt, {N, h}), *y = c.at(a[3], dt, {N, h}), *stats = c.at(a[4], 0, {4, N});
        void *dx = c.at(a[5], grad_dt, {N, h}), *dy = c.at(a[6], grad_dt, {N, h}), *dr = c.at(a[7], grad_dt, {N, h});
        void *gate = c.at(a[8], dt, {rows, h}), *w = c.at(a[9], dt, {h}), *w_post = c.at(a[10], dt, {h}), *b_post = c.at(a[11], dt, {h});
        const float scale = (float)c.real(a[12]);
        const uint32_t flags = (uint32_t)c.integer(a[13]);
        float *dgate = static_cast<float*>(c.at(a[14], 0, {rows, h})), *dw = static_cast<float*>(c.at(a[15], 0, {h}));
        float *db = static_cast<float*>(c.at(a[16], 0, {h})), *dw_post = static_cast<float*>(c.at(a[17], 0, {h}));
        float* db_post = static_cast<float*>(c.at(a[18], 0, {h}));
        const at::Tensor& ws = THPVariable_Unpack(a[19]);
        if (!c.ok || !ws.defined() || !ws.is_cuda() || ws.get_device() != c.here || !ws.is_contiguous()) Py_RETURN_NONE;
        void *workspace = ws.data_ptr(), *stream = c.stream(a[20]);
        const size_t bytes = ws.nbytes();
        if (!c.ok) Py_RETURN_NONE;
        Py_BEGIN_ALLOW_THREADS
        status = f(dH, dH_dt, dr, r, y, gate, rows, w_post, b_post, w, static_cast<const float*>(stats), N, h, dt, flags, scale,
                   grad_dt, dx, dy, dgate, dw_post, db_post, dw, db, workspace, bytes, stream);
        Py_END_ALLOW_THREADS
    } catch (...) {
        Py_RETURN_NONE;
    }
    return PyLong_FromLong(status);
}

PyMethodDef methods[] = {
    {"block_norm_fwd", reinterpret_cast<PyCFunction>(reinterpret_cast<void*>(block_norm_fwd)), METH_FASTCALL, nullptr},
    {"block_norm_bwd", reinterpret_cast<PyCFunction>(reinterpret_cast<void*>(block_norm_bwd)), METH_FASTCALL, nullptr},
    {"ptr", reinterpret_cast<PyCFunction>(reinterpret_cast<void*>(ptr)), METH_FASTCALL, nullptr},
    {"ptrs", reinterpret_cast<PyCFunction>(reinterpret_cast<void*>(ptrs)), METH_FASTCALL, nullptr},
    {"same_shapes", same_shapes, METH_O, nullptr},
    {"on_current_device", on_current_device, METH_O, nullptr},
    {"unchanged", reinterpret_cast<PyCFunction>(reinterpret_cast<void*>(unchanged)), METH_FASTCALL, nullptr},
    {"stream", stream, METH_NOARGS, nullptr},
    {nullptr, nullptr, 0, nullptr},
};

PyModuleDef module = {PyModuleDef_HEAD_INIT, "_vphost", nullptr, -1, methods, nullptr, nullptr, nullptr, nullptr};

}  // namespace

PyMODINIT_FUNC PyInit__vphost(void) {
    PyObject* m = PyModule_Create(&module);
    // the PyTorch whose objects this code reads: another one's may be laid out otherwise
    if (m && PyModule_AddStringConstant(m, "torch_version", TORCH_VERSION) < 0) Py_CLEAR(m);
    return m;
}
