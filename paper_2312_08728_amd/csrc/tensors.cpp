// What the library's calls need to know of torch tensors, asked for in one go: type, device, sizes, strides and address of a tensor cost 0.4 us from Python,
// as much as some of these calls take for all their work (64 tensors with moments in 8 bits: 128 tensors, 36 us; here 1.6).
//
//   matrices(tensors, shapes, dtype, device[, written])    bytes: address and row stride (int64) of each, zeros for None; those from index `written` on are told
//                                               that they are written, as torch's own in-place operations tell (autograd then refuses values that it has kept)
//   vectors(tensors, numels, dtype, device)     bytes: the addresses of contiguous tensors; numels: bytes of int64
//   pairs(pairs, numels, dtype, device)         (bytes, bytes): the same of the first and of the second tensors
//   same(groups)                                True if the tensors of every group are what they were when their addresses were read.  A group: (list, item, numels, dtype,
//                                               addresses), the bytes as above; item: which of the tuple that the list has for each, or -1 for tensors themselves
//
//   touch(tensors)                              tells the tensors of a list that they have been written
//
// The first three return the index of the first tensor (of pairs: the first pair) that is not what was asked for instead, an int: the caller says what is wrong with it.
#define PY_SSIZE_T_CLEAN
#include <Python.h>

#include <torch/csrc/Dtype.h>
#include <torch/csrc/autograd/python_variable.h>

#include <cstdint>
#include <cstring>

namespace {

struct Kind {
    c10::ScalarType type;
    int64_t device;
};

bool kind_of(PyObject* dtype, PyObject* device, Kind* k)
{
    if (!THPDtype_Check(dtype)) {
        PyErr_SetString(PyExc_TypeError, "a torch.dtype is wanted");
        return false;
    }
    k->type = reinterpret_cast<THPDtype*>(dtype)->scalar_type;
    k->device = PyLong_AsLongLong(device);
    return !PyErr_Occurred();
}

const at::Tensor* tensor_of(PyObject* o, const Kind& k)
{
    if (!THPVariable_Check(o)) return nullptr;
    const at::Tensor& t = THPVariable_Unpack(o);
    if (t.scalar_type() != k.type || t.layout() != c10::kStrided || !t.has_storage() || t.is_neg()) return nullptr;
    if (t.is_cuda() ? t.get_device() != k.device : k.device != -1 || !t.is_cpu()) return nullptr;
    return &t;
}

void touch(const at::Tensor& t)
{
    if (!t.is_inference()) t.unsafeGetTensorImpl()->bump_version();             // (inference tensors have no count)
}

PyObject* matrices_(PyObject* const* args, Py_ssize_t n)
{
    Kind k;
    if ((n != 4 && n != 5) || !PyTuple_Check(args[0]) || !PyTuple_Check(args[1]) || PyTuple_GET_SIZE(args[0]) != PyTuple_GET_SIZE(args[1])) {
        PyErr_SetString(PyExc_TypeError, "matrices(tensors, shapes, dtype, device): two tuples of one length");
        return nullptr;
    }
    if (!kind_of(args[2], args[3], &k)) return nullptr;
    const Py_ssize_t count = PyTuple_GET_SIZE(args[0]), written = n == 5 ? PyLong_AsSsize_t(args[4]) : count;
    if (written < 0) {
        if (!PyErr_Occurred()) PyErr_SetString(PyExc_ValueError, "matrices(): written must not be negative");
        return nullptr;
    }
    PyObject* out = PyBytes_FromStringAndSize(nullptr, count * 16);
    if (!out) return nullptr;
    char* to = PyBytes_AS_STRING(out);
    for (Py_ssize_t i = 0; i < count; ++i, to += 16) {
        PyObject* o = PyTuple_GET_ITEM(args[0], i);
        int64_t v[2] = {0, 0};
        if (o != Py_None) {
            PyObject* shape = PyTuple_GET_ITEM(args[1], i);
            if (!PyTuple_Check(shape) || PyTuple_GET_SIZE(shape) != 2) {
                Py_DECREF(out);
                PyErr_SetString(PyExc_TypeError, "matrices(): a shape is a pair");
                return nullptr;
            }
            const int64_t rows = PyLong_AsLongLong(PyTuple_GET_ITEM(shape, 0)), cols = PyLong_AsLongLong(PyTuple_GET_ITEM(shape, 1));
            const at::Tensor* t = PyErr_Occurred() ? nullptr : tensor_of(o, k);
            if (PyErr_Occurred()) {
                Py_DECREF(out);
                return nullptr;
            }
            if (!t || t->dim() != 2 || t->size(0) != rows || t->size(1) != cols || (t->stride(1) != 1 && cols != 1)) {
                Py_DECREF(out);
                return PyLong_FromSsize_t(i);
            }
            v[0] = (int64_t)(uintptr_t)t->data_ptr();
            v[1] = t->stride(0);
        }
        std::memcpy(to, v, 16);
    }
    for (Py_ssize_t i = written; i < count; ++i)
        if (PyTuple_GET_ITEM(args[0], i) != Py_None) touch(THPVariable_Unpack(PyTuple_GET_ITEM(args[0], i)));
    return out;
}

PyObject* vectors_(PyObject* const* args, Py_ssize_t n)
{
    Kind k;
    if (n != 4 || !PyList_Check(args[0]) || !PyBytes_Check(args[1]) || PyBytes_GET_SIZE(args[1]) != 8 * PyList_GET_SIZE(args[0])) {
        PyErr_SetString(PyExc_TypeError, "vectors(tensors, numels, dtype, device): a list and eight bytes for each of its tensors");
        return nullptr;
    }
    if (!kind_of(args[2], args[3], &k)) return nullptr;
    const Py_ssize_t count = PyList_GET_SIZE(args[0]);
    PyObject* out = PyBytes_FromStringAndSize(nullptr, count * 8);
    for (Py_ssize_t i = 0; i < count && out; ++i) {
        const at::Tensor* t = tensor_of(PyList_GET_ITEM(args[0], i), k);
        int64_t numel;
        std::memcpy(&numel, PyBytes_AS_STRING(args[1]) + 8 * i, 8);
        if (!t || t->numel() != numel || !t->is_contiguous()) {
            Py_DECREF(out);
            return PyLong_FromSsize_t(i);
        }
        const int64_t at = (int64_t)(uintptr_t)t->data_ptr();
        std::memcpy(PyBytes_AS_STRING(out) + 8 * i, &at, 8);
    }
    return out;
}

PyObject* pairs_(PyObject* const* args, Py_ssize_t n)
{
    Kind k;
    if (n != 4 || !PyList_Check(args[0]) || !PyBytes_Check(args[1]) || PyBytes_GET_SIZE(args[1]) != 8 * PyList_GET_SIZE(args[0])) {
        PyErr_SetString(PyExc_TypeError, "pairs(pairs, numels, dtype, device): a list and eight bytes for each of its pairs");
        return nullptr;
    }
    if (!kind_of(args[2], args[3], &k)) return nullptr;
    const Py_ssize_t count = PyList_GET_SIZE(args[0]);
    PyObject* out[2] = {PyBytes_FromStringAndSize(nullptr, count * 8), PyBytes_FromStringAndSize(nullptr, count * 8)};
    PyObject* answer = nullptr;
    for (Py_ssize_t i = 0; i < count && out[0] && out[1] && !answer; ++i) {
        PyObject* pair = PyList_GET_ITEM(args[0], i);
        const bool tuple = PyTuple_Check(pair) && PyTuple_GET_SIZE(pair) == 2, list = PyList_Check(pair) && PyList_GET_SIZE(pair) == 2;
        int64_t numel;
        std::memcpy(&numel, PyBytes_AS_STRING(args[1]) + 8 * i, 8);
        for (int j = 0; j < 2 && !answer; ++j) {
            const at::Tensor* t = tuple ? tensor_of(PyTuple_GET_ITEM(pair, j), k) : list ? tensor_of(PyList_GET_ITEM(pair, j), k) : nullptr;
            if (!t || t->numel() != numel || !t->is_contiguous()) {
                answer = PyLong_FromSsize_t(i);
                break;
            }
            const int64_t at = (int64_t)(uintptr_t)t->data_ptr();
            std::memcpy(PyBytes_AS_STRING(out[j]) + 8 * i, &at, 8);
        }
    }
    if (!answer && out[0] && out[1]) answer = PyTuple_Pack(2, out[0], out[1]);
    Py_XDECREF(out[0]);
    Py_XDECREF(out[1]);
    return answer;
}

PyObject* same_(PyObject* const* args, Py_ssize_t n)
{
    if (n != 1 || !PyTuple_Check(args[0])) {
        PyErr_SetString(PyExc_TypeError, "same(groups): a tuple of groups");
        return nullptr;
    }
    uint64_t plain = 0;                                        // what kind of tensor the last one was, in torch's words
    for (Py_ssize_t j = 0; j < PyTuple_GET_SIZE(args[0]); ++j) {
        PyObject* const group = PyTuple_GET_ITEM(args[0], j);
        PyObject* g[5] = {};
        for (Py_ssize_t i = 0; i < 5 && PyTuple_Check(group) && PyTuple_GET_SIZE(group) == 5; ++i) g[i] = PyTuple_GET_ITEM(group, i);
        const Py_ssize_t bytes = g[4] && PyBytes_Check(g[4]) ? PyBytes_GET_SIZE(g[4]) : -1;
        if (bytes < 0 || !PyList_Check(g[0]) || !PyBytes_Check(g[2]) || PyBytes_GET_SIZE(g[2]) != bytes) {
            PyErr_SetString(PyExc_TypeError, "same(): a group is (list, item, numels, dtype, addresses)");
            return nullptr;
        }
        if (!THPDtype_Check(g[3])) {
            PyErr_SetString(PyExc_TypeError, "a torch.dtype is wanted");
            return nullptr;
        }
        const caffe2::TypeMeta type = c10::scalarTypeToTypeMeta(reinterpret_cast<THPDtype*>(g[3])->scalar_type);
        const int64_t size = (int64_t)type.itemsize();
        const Py_ssize_t item = PyLong_AsSsize_t(g[1]);
        if (item == -1 && PyErr_Occurred()) return nullptr;
        if (8 * PyList_GET_SIZE(g[0]) != bytes) Py_RETURN_FALSE;
        for (Py_ssize_t i = 0; 8 * i < bytes; ++i) {
            PyObject* o = PyList_GET_ITEM(g[0], i);
            if (item >= 0) o = PyTuple_Check(o) && item < PyTuple_GET_SIZE(o) ? PyTuple_GET_ITEM(o, item) : Py_None;
            if (!THPVariable_Check(o)) Py_RETURN_FALSE;
            // (no device is asked for: memory at the address that was read is on the device that was read)
            const c10::TensorImpl* const t = THPVariable_Unpack(o).unsafeGetTensorImpl();
            int64_t numel, at;
            std::memcpy(&numel, PyBytes_AS_STRING(g[2]) + 8 * i, 8);
            std::memcpy(&at, PyBytes_AS_STRING(g[4]) + 8 * i, 8);
            const uint64_t kind = t->key_set().raw_repr();
            if (kind != plain) {
                if (t->layout() != c10::kStrided || !t->has_storage() || t->is_neg()) Py_RETURN_FALSE;
                plain = kind;
            }
            if (t->dtype() != type || t->numel() != numel || !t->is_contiguous()) Py_RETURN_FALSE;
            const char* const data = static_cast<const char*>(t->storage().mutable_data());     // (a lazy copy is made now)
            if ((int64_t)(uintptr_t)(numel ? data + t->storage_offset() * size : nullptr) != at) Py_RETURN_FALSE;
        }
    }
    Py_RETURN_TRUE;
}

PyObject* touch_(PyObject* const* args, Py_ssize_t n)
{
    if (n != 1 || !PyList_Check(args[0])) {
        PyErr_SetString(PyExc_TypeError, "touch(tensors): a list");
        return nullptr;
    }
    for (Py_ssize_t i = 0; i < PyList_GET_SIZE(args[0]); ++i)
        if (THPVariable_Check(PyList_GET_ITEM(args[0], i))) touch(THPVariable_Unpack(PyList_GET_ITEM(args[0], i)));
    Py_RETURN_NONE;
}

// (no C++ exception leaves these)
template <PyObject* F(PyObject* const*, Py_ssize_t)> PyObject* guarded(PyObject*, PyObject* const* args, Py_ssize_t n)
{
    try {
        return F(args, n);
    } catch (const std::exception& e) {
        PyErr_SetString(PyExc_RuntimeError, e.what());
        return nullptr;
    }
}

PyMethodDef methods[] = {
    {"matrices", reinterpret_cast<PyCFunction>(reinterpret_cast<void (*)()>(&guarded<matrices_>)), METH_FASTCALL, "addresses and row strides of matrices"},
    {"vectors", reinterpret_cast<PyCFunction>(reinterpret_cast<void (*)()>(&guarded<vectors_>)), METH_FASTCALL, "addresses of contiguous tensors"},
    {"pairs", reinterpret_cast<PyCFunction>(reinterpret_cast<void (*)()>(&guarded<pairs_>)), METH_FASTCALL, "addresses of pairs of contiguous tensors"},
    {"same", reinterpret_cast<PyCFunction>(reinterpret_cast<void (*)()>(&guarded<same_>)), METH_FASTCALL, "whether tensors are where they were"},
    {"touch", reinterpret_cast<PyCFunction>(reinterpret_cast<void (*)()>(&guarded<touch_>)), METH_FASTCALL, "tells tensors that they have been written"},
    {nullptr, nullptr, 0, nullptr}};
PyModuleDef module = {PyModuleDef_HEAD_INIT, "_tensors", nullptr, -1, methods, nullptr, nullptr, nullptr, nullptr};

}  // namespace

PyMODINIT_FUNC PyInit__tensors() { return PyModule_Create(&module); }
