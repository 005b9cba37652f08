// The usual calls of the key-value cache from Python (kv.py): tensors on the
// current device as the library takes them, outputs and workspace new. What they
// take there, checks, outputs and the library's call, is 4 to 7 us of the host's
// time in Python beyond the launches' own, as much as the small calls take on the
// GPU; here it is about 1. Anything else, errors in the arguments among it, is
// answered by None, and kv.py goes through it step by step, as it does with all
// calls where this module is not there.
#include <Python.h>

#include <ATen/ops/empty.h>
#include <c10/core/GradMode.h>
#include <torch/csrc/Exceptions.h>
#include <torch/csrc/autograd/python_variable.h>

#include "../../include/kmeans.h"

namespace {

decltype(&kmeans_kv_write) write_fn;
decltype(&kmeans_kv_read) read_fn;
decltype(&kmeans_kv_attend_workspace_bytes) bytes_fn;
decltype(&kmeans_kv_attend) attend_fn;

// A plain tensor of this type on the centres' GPU, or null.
const at::Tensor *plain(PyObject *o, const at::Tensor &centres, at::ScalarType type, int64_t dim)
{
    if (!THPVariable_CheckExact(o)) return nullptr;
    const at::Tensor &t = THPVariable_Unpack(o);
    return t.layout() == at::kStrided && t.device() == centres.device() && t.scalar_type() == type &&
                   t.dim() == dim
               ? &t
               : nullptr;
}

// [n][heads][dim] with its rows on 16 bytes, or null.
const at::Tensor *rows(PyObject *o, const at::Tensor &centres, const kmeans_kv_t *kv)
{
    const at::Tensor *t = plain(o, centres, centres.scalar_type(), 3);
    return t && t->size(0) > 0 && t->size(2) == kv->dim && t->stride(2) == 1 &&
                   ((t->stride(0) | t->stride(1)) & 7) == 0 &&
                   (reinterpret_cast<uintptr_t>(t->data_ptr()) & 15) == 0
               ? t
               : nullptr;
}

const at::Tensor *ints(PyObject *o, const at::Tensor &centres, at::ScalarType type, int64_t n)
{
    const at::Tensor *t = plain(o, centres, type, 1);
    return t && t->size(0) == n && (t->stride(0) == 1 || n == 1) ? t : nullptr;
}

const kmeans_kv_t *desc_of(PyObject *o) { return static_cast<const kmeans_kv_t *>(PyLong_AsVoidPtr(o)); }

// bind(write, read, bytes, attend): where the library's functions are.
PyObject *bind(PyObject *, PyObject *const *a, Py_ssize_t n)
{
    if (n != 4) {
        PyErr_SetString(PyExc_TypeError, "bind takes 4 addresses");
        return nullptr;
    }
    write_fn = reinterpret_cast<decltype(write_fn)>(PyLong_AsVoidPtr(a[0]));
    read_fn = reinterpret_cast<decltype(read_fn)>(PyLong_AsVoidPtr(a[1]));
    bytes_fn = reinterpret_cast<decltype(bytes_fn)>(PyLong_AsVoidPtr(a[2]));
    attend_fn = reinterpret_cast<decltype(attend_fn)>(PyLong_AsVoidPtr(a[3]));
    if (PyErr_Occurred()) return nullptr;
    Py_RETURN_NONE;
}

// write(description, centres, stream, k, v, slots) -> status
PyObject *write(PyObject *, PyObject *const *a, Py_ssize_t n)
{
    HANDLE_TH_ERRORS
    if (n != 6 || !THPVariable_CheckExact(a[1])) Py_RETURN_NONE;
    const kmeans_kv_t *kv = desc_of(a[0]);
    const at::Tensor &centres = THPVariable_Unpack(a[1]);
    const at::Tensor *k = rows(a[3], centres, kv), *v = rows(a[4], centres, kv);
    if (!k || !v || k->size(1) != kv->heads || k->sizes() != v->sizes()) Py_RETURN_NONE;
    const at::Tensor *slots = ints(a[5], centres, at::kLong, k->size(0));
    if (!slots) Py_RETURN_NONE;
    return PyLong_FromLong(write_fn(kv, k->data_ptr(), k->stride(0), k->stride(1), v->data_ptr(),
                                    v->stride(0), v->stride(1), slots->data_ptr<int64_t>(),
                                    k->size(0), PyLong_AsVoidPtr(a[2])));
    END_HANDLE_TH_ERRORS
}

// read(description, centres, stream, slots) -> (k, v) or a status
PyObject *read(PyObject *, PyObject *const *a, Py_ssize_t n)
{
    HANDLE_TH_ERRORS
    if (n != 4 || !THPVariable_CheckExact(a[1])) Py_RETURN_NONE;
    const kmeans_kv_t *kv = desc_of(a[0]);
    const at::Tensor &centres = THPVariable_Unpack(a[1]);
    const at::Tensor *slots = plain(a[3], centres, at::kLong, 1);
    if (!slots || slots->size(0) == 0 || (slots->stride(0) != 1 && slots->size(0) != 1)) Py_RETURN_NONE;
    const int64_t tokens = slots->size(0), head = kv->dim, token = head * kv->heads;
    at::Tensor k = at::empty({tokens, kv->heads, head}, centres.options());
    at::Tensor v = at::empty({tokens, kv->heads, head}, centres.options());
    const int rc = read_fn(kv, slots->data_ptr<int64_t>(), tokens, k.data_ptr(), token, head,
                           v.data_ptr(), token, head, PyLong_AsVoidPtr(a[2]));
    if (rc) return PyLong_FromLong(rc);
    return Py_BuildValue("(NN)", THPVariable_Wrap(std::move(k)), THPVariable_Wrap(std::move(v)));
    END_HANDLE_TH_ERRORS
}

// attend(description, centres, stream, q, table, lengths, scale, starts) -> (out, lse) or a status
PyObject *attend(PyObject *, PyObject *const *a, Py_ssize_t n)
{
    HANDLE_TH_ERRORS
    if (n != 8 || !THPVariable_CheckExact(a[1]) || !PyFloat_CheckExact(a[6])) Py_RETURN_NONE;
    const kmeans_kv_t *kv = desc_of(a[0]);
    const at::Tensor &centres = THPVariable_Unpack(a[1]);
    const at::Tensor *q = rows(a[3], centres, kv), *table = plain(a[4], centres, at::kInt, 2);
    if (!q || !table) Py_RETURN_NONE;
    if ((q->requires_grad() && c10::GradMode::is_enabled()) || q->_fw_grad(0).defined())
        Py_RETURN_NONE;
    const int64_t seqs = q->size(0), q_heads = q->size(1), width = table->size(1);
    if (table->size(0) != seqs || width == 0 || table->stride(1) != 1) Py_RETURN_NONE;
    const at::Tensor *lengths = ints(a[5], centres, at::kInt, seqs), *starts = nullptr;
    if (!lengths) Py_RETURN_NONE;
    if (a[7] != Py_None && !(starts = ints(a[7], centres, at::kInt, seqs))) Py_RETURN_NONE;
    if (seqs > INT32_MAX || q_heads < 1 || q_heads > INT32_MAX || q_heads % kv->heads) Py_RETURN_NONE;
    const size_t bytes = bytes_fn(kv, (int32_t)seqs, (int32_t)q_heads, width);
    if (bytes == 0) Py_RETURN_NONE;
    at::Tensor out = at::empty(q->sizes(), centres.options());
    at::Tensor lse = at::empty({seqs, q_heads}, centres.options().dtype(at::kFloat));
    at::Tensor ws = at::empty({(int64_t)bytes}, centres.options().dtype(at::kByte));
    const int rc = attend_fn(kv, q->data_ptr(), q->stride(0), q->stride(1), (int32_t)seqs,
                             (int32_t)q_heads, table->data_ptr<int32_t>(), table->stride(0), width,
                             lengths->data_ptr<int32_t>(),
                             starts ? starts->data_ptr<int32_t>() : nullptr,
                             (float)PyFloat_AS_DOUBLE(a[6]), out.data_ptr(), out.stride(0),
                             out.stride(1), lse.data_ptr<float>(), ws.data_ptr(), bytes,
                             PyLong_AsVoidPtr(a[2]));
    if (rc) return PyLong_FromLong(rc);
    return Py_BuildValue("(NN)", THPVariable_Wrap(std::move(out)), THPVariable_Wrap(std::move(lse)));
    END_HANDLE_TH_ERRORS
}

template <typename F>
PyCFunction fast(F *f) { return reinterpret_cast<PyCFunction>(reinterpret_cast<void (*)()>(f)); }

PyMethodDef methods[] = {{"bind", fast(bind), METH_FASTCALL, nullptr},
                         {"write", fast(write), METH_FASTCALL, nullptr},
                         {"read", fast(read), METH_FASTCALL, nullptr},
                         {"attend", fast(attend), METH_FASTCALL, nullptr},
                         {nullptr, nullptr, 0, nullptr}};
PyModuleDef module = {PyModuleDef_HEAD_INIT, "_kv_call", nullptr, -1, methods,
                      nullptr, nullptr, nullptr, nullptr};

}  // namespace

// torch_version: the torch whose headers this was built with; kv.py takes no other.
PyMODINIT_FUNC PyInit__kv_call()
{
    PyObject *m = PyModule_Create(&module);
    if (m && PyModule_AddStringConstant(m, "torch_version", KV_TORCH) < 0) {
        Py_DECREF(m);
        return nullptr;
    }
    return m;
}
