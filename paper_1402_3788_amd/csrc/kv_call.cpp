// The usual calls of the key-value cache from Python (kv.py, kv_serve.py): tensors on the
// current device as the library takes them, outputs and workspace new. What they
// take there, checks, outputs and the library's call, is 4 to 7 us of the host's
// time in Python beyond the launches' own, as much as the small calls take on the
// GPU; here it is about 1. Anything else, errors in the arguments among it, is
// answered by None, and the Python modules go through it step by step, as they do with
// all calls where this module is not there.
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
decltype(&kmeans_kv_rotate) rotate_fn;
decltype(&kmeans_kv_attend_tokens_workspace_bytes) tokens_bytes_fn;
decltype(&kmeans_kv_attend_tokens) tokens_fn;
decltype(&kmeans_kv_weigh) weigh_fn;
decltype(&kmeans_kv_evict) evict_fn;

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

// bind_serve(rotate, attend_tokens_workspace_bytes, attend_tokens, weigh, evict)
PyObject *bind_serve(PyObject *, PyObject *const *a, Py_ssize_t n)
{
    if (n != 5) {
        PyErr_SetString(PyExc_TypeError, "bind_serve takes 5 addresses");
        return nullptr;
    }
    rotate_fn = reinterpret_cast<decltype(rotate_fn)>(PyLong_AsVoidPtr(a[0]));
    tokens_bytes_fn = reinterpret_cast<decltype(tokens_bytes_fn)>(PyLong_AsVoidPtr(a[1]));
    tokens_fn = reinterpret_cast<decltype(tokens_fn)>(PyLong_AsVoidPtr(a[2]));
    weigh_fn = reinterpret_cast<decltype(weigh_fn)>(PyLong_AsVoidPtr(a[3]));
    evict_fn = reinterpret_cast<decltype(evict_fn)>(PyLong_AsVoidPtr(a[4]));
    if (PyErr_Occurred()) return nullptr;
    Py_RETURN_NONE;
}

bool needs_gradient(const at::Tensor &t)
{
    return (t.requires_grad() && c10::GradMode::is_enabled()) || t._fw_grad(0).defined();
}

// A number that is a float or an int, exactly.
bool number(PyObject *o, double *x)
{
    if (PyFloat_CheckExact(o)) {
        *x = PyFloat_AS_DOUBLE(o);
        return true;
    }
    if (!PyLong_CheckExact(o)) return false;
    *x = PyLong_AsDouble(o);
    if (*x != -1.0 || !PyErr_Occurred()) return true;
    PyErr_Clear();
    return false;
}

// A whole number of 0 to 2^31 - 1.
bool whole(PyObject *o, int32_t *x)
{
    if (!PyLong_CheckExact(o)) return false;
    int over = 0;
    const long v = PyLong_AsLongAndOverflow(o, &over);
    if (over || v < 0 || v > INT32_MAX) return false;
    *x = (int32_t)v;
    return true;
}

// rotate(device, stream, q, k, positions, frequencies, flags, amplitude) -> (q, k) or a status
PyObject *rotate(PyObject *, PyObject *const *a, Py_ssize_t n)
{
    HANDLE_TH_ERRORS
    double amplitude;
    if (n != 8 || !THPVariable_CheckExact(a[2]) || !number(a[7], &amplitude)) Py_RETURN_NONE;
    const at::Tensor &q = THPVariable_Unpack(a[2]);
    if (!q.is_cuda() || q.get_device() != PyLong_AsLong(a[0]) || q.dim() != 3 || q.size(0) == 0 ||
        (q.scalar_type() != at::kBFloat16 && q.scalar_type() != at::kHalf))
        Py_RETURN_NONE;
    const at::Tensor *k = nullptr;
    if (a[3] != Py_None && !(k = plain(a[3], q, q.scalar_type(), 3))) Py_RETURN_NONE;
    const at::Tensor *positions = ints(a[4], q, at::kLong, q.size(0));
    const at::Tensor *frequencies = plain(a[5], q, at::kDouble, 1);
    if (!positions || !frequencies || !frequencies->is_contiguous() || 2 * frequencies->size(0) > q.size(2) ||
        q.size(2) > INT32_MAX || frequencies->is_conj() || needs_gradient(*frequencies))
        Py_RETURN_NONE;
    if (k && (k->size(0) != q.size(0) || k->size(2) != q.size(2))) Py_RETURN_NONE;
    for (const at::Tensor *t : {&q, k})
        if (t && (t->size(1) == 0 || t->size(1) > INT32_MAX || t->stride(2) != 1 || ((t->stride(0) | t->stride(1)) & 7) ||
                  (reinterpret_cast<uintptr_t>(t->data_ptr()) & 15) || needs_gradient(*t)))
            Py_RETURN_NONE;
    kmeans_kv_turn_t turn{};
    turn.positions = positions->data_ptr<int64_t>();
    turn.frequencies = frequencies->data_ptr<double>();
    turn.tokens = q.size(0);
    turn.dim = (int32_t)q.size(2);
    turn.half = (int32_t)frequencies->size(0);
    turn.type = q.scalar_type() == at::kHalf ? KMEANS_KV_FP16 : KMEANS_KV_BF16;
    turn.flags = (uint32_t)PyLong_AsUnsignedLong(a[6]);
    turn.amplitude = (float)amplitude;
    at::Tensor qo = at::empty(q.sizes(), q.options()), ko;
    if (k) ko = at::empty(k->sizes(), k->options());
    const int rc = rotate_fn(&turn, q.data_ptr(), q.stride(0), q.stride(1), (int32_t)q.size(1),
                             qo.data_ptr(), qo.stride(0), qo.stride(1), k ? k->data_ptr() : nullptr,
                             k ? k->stride(0) : 0, k ? k->stride(1) : 0, k ? (int32_t)k->size(1) : 0,
                             k ? ko.data_ptr() : nullptr, k ? ko.stride(0) : 0, k ? ko.stride(1) : 0,
                             PyLong_AsVoidPtr(a[1]));
    if (rc) return PyLong_FromLong(rc);
    if (k) return Py_BuildValue("(NN)", THPVariable_Wrap(std::move(qo)), THPVariable_Wrap(std::move(ko)));
    return Py_BuildValue("(NO)", THPVariable_Wrap(std::move(qo)), Py_None);
    END_HANDLE_TH_ERRORS
}

// What attend_tokens and weigh have alike: q, bounds, table and lengths, then scale, cap,
// slopes, window, prefixes and starts. False: not a usual call.
bool new_tokens(kmeans_kv_tokens_t *t, const at::Tensor **q_of, const kmeans_kv_t *kv, const at::Tensor &centres,
                PyObject *q_o, PyObject *bounds_o, PyObject *table_o, PyObject *lengths_o, PyObject *const *more)
{
    const at::Tensor *q = rows(q_o, centres, kv), *table = plain(table_o, centres, at::kInt, 2);
    if (!q || !table || needs_gradient(*q)) return false;
    const int64_t seqs = table->size(0);
    if (seqs == 0 || seqs > INT32_MAX || table->size(1) == 0 || table->stride(1) != 1) return false;
    const at::Tensor *lengths = ints(lengths_o, centres, at::kInt, seqs);
    const at::Tensor *bounds = ints(bounds_o, centres, at::kInt, seqs + 1);
    if (!lengths || !bounds || q->size(1) < 1 || q->size(1) > INT32_MAX || q->size(1) % kv->heads) return false;
    double scale, cap;
    if (!number(more[0], &scale) || !number(more[1], &cap) || !whole(more[3], &t->window)) return false;
    const at::Tensor *slopes = nullptr, *prefixes = nullptr, *starts = nullptr;
    if (more[2] != Py_None && (!(slopes = ints(more[2], centres, at::kFloat, q->size(1))) || needs_gradient(*slopes)))
        return false;
    if (more[4] != Py_None && !(prefixes = ints(more[4], centres, at::kInt, seqs))) return false;
    if (more[5] != Py_None && !(starts = ints(more[5], centres, at::kInt, q->size(0)))) return false;
    t->bounds = bounds->data_ptr<int32_t>();
    t->table = table->data_ptr<int32_t>();
    t->table_stride = table->stride(0);
    t->table_pages = table->size(1);
    t->lengths = lengths->data_ptr<int32_t>();
    t->starts = starts ? starts->data_ptr<int32_t>() : nullptr;
    t->prefixes = prefixes ? prefixes->data_ptr<int32_t>() : nullptr;
    t->slopes = slopes ? slopes->data_ptr<float>() : nullptr;
    t->tokens = q->size(0);
    t->seqs = (int32_t)seqs;
    t->q_heads = (int32_t)q->size(1);
    t->scale = (float)scale;
    t->cap = (float)cap;
    *q_of = q;
    return true;
}

// attend_tokens(description, centres, stream, q, bounds, table, lengths, scale, cap, slopes, window,
// prefixes, starts) -> (out, lse) or a status
PyObject *attend_tokens(PyObject *, PyObject *const *a, Py_ssize_t n)
{
    HANDLE_TH_ERRORS
    if (n != 13 || !THPVariable_CheckExact(a[1])) Py_RETURN_NONE;
    const kmeans_kv_t *kv = desc_of(a[0]);
    const at::Tensor &centres = THPVariable_Unpack(a[1]);
    kmeans_kv_tokens_t t{};
    const at::Tensor *q;
    if (!new_tokens(&t, &q, kv, centres, a[3], a[4], a[5], a[6], a + 7)) Py_RETURN_NONE;
    const size_t bytes = tokens_bytes_fn(kv, &t);
    if (bytes == 0) Py_RETURN_NONE;
    at::Tensor out = at::empty(q->sizes(), centres.options());
    at::Tensor lse = at::empty({q->size(0), q->size(1)}, centres.options().dtype(at::kFloat));
    at::Tensor ws = at::empty({(int64_t)bytes}, centres.options().dtype(at::kByte));
    const int rc = tokens_fn(kv, &t, q->data_ptr(), q->stride(0), q->stride(1), out.data_ptr(), out.stride(0),
                             out.stride(1), lse.data_ptr<float>(), ws.data_ptr(), bytes, PyLong_AsVoidPtr(a[2]));
    if (rc) return PyLong_FromLong(rc);
    return Py_BuildValue("(NN)", THPVariable_Wrap(std::move(out)), THPVariable_Wrap(std::move(lse)));
    END_HANDLE_TH_ERRORS
}

// weigh(description, centres, stream, q, bounds, table, lengths, lse, scale, cap, slopes, window,
// prefixes, starts) -> (weights,) or a status
PyObject *weigh(PyObject *, PyObject *const *a, Py_ssize_t n)
{
    HANDLE_TH_ERRORS
    if (n != 14 || !THPVariable_CheckExact(a[1])) Py_RETURN_NONE;
    const kmeans_kv_t *kv = desc_of(a[0]);
    const at::Tensor &centres = THPVariable_Unpack(a[1]);
    kmeans_kv_tokens_t t{};
    const at::Tensor *q;
    if (!new_tokens(&t, &q, kv, centres, a[3], a[4], a[5], a[6], a + 8)) Py_RETURN_NONE;
    const at::Tensor *lse = plain(a[7], centres, at::kFloat, 2);
    if (!lse || lse->size(0) != t.tokens || lse->size(1) != t.q_heads || !lse->is_contiguous() || needs_gradient(*lse))
        Py_RETURN_NONE;
    const int64_t positions = t.table_pages * kv->page;
    at::Tensor w = at::empty({t.seqs, kv->heads, positions}, centres.options().dtype(at::kFloat));
    const int rc = weigh_fn(kv, &t, q->data_ptr(), q->stride(0), q->stride(1), lse->data_ptr<float>(),
                            w.data_ptr<float>(), w.stride(0), w.stride(1), positions, 0, PyLong_AsVoidPtr(a[2]));
    if (rc) return PyLong_FromLong(rc);
    return Py_BuildValue("(N)", THPVariable_Wrap(std::move(w)));
    END_HANDLE_TH_ERRORS
}

// evict(description, centres, stream, weights, table, lengths, keep, recent, first, to)
// -> (kept, lengths, weights) or a status
PyObject *evict(PyObject *, PyObject *const *a, Py_ssize_t n)
{
    HANDLE_TH_ERRORS
    if (n != 10 || !THPVariable_CheckExact(a[1])) Py_RETURN_NONE;
    const kmeans_kv_t *kv = desc_of(a[0]);
    const at::Tensor &centres = THPVariable_Unpack(a[1]);
    const at::Tensor *w = plain(a[3], centres, at::kFloat, 3), *table = plain(a[4], centres, at::kInt, 2), *to = nullptr;
    if (!w || !table || table->size(0) == 0 || table->size(0) > INT32_MAX || table->size(1) == 0 || table->stride(1) != 1)
        Py_RETURN_NONE;
    const int64_t seqs = table->size(0);
    const at::Tensor *lengths = ints(a[5], centres, at::kInt, seqs);
    if (!lengths || w->size(0) != seqs || w->size(1) != kv->heads || !w->is_contiguous() || needs_gradient(*w))
        Py_RETURN_NONE;
    if (a[9] != Py_None &&
        (!(to = plain(a[9], centres, at::kInt, 2)) || to->size(0) != seqs || to->size(1) == 0 || to->stride(1) != 1))
        Py_RETURN_NONE;
    kmeans_kv_evict_t e{};
    if (!whole(a[6], &e.keep) || !whole(a[7], &e.recent) || !whole(a[8], &e.first) || e.keep < 1 ||
        (int64_t)e.recent + e.first > e.keep)
        Py_RETURN_NONE;
    e.table = table->data_ptr<int32_t>();
    e.table_stride = table->stride(0);
    e.table_pages = table->size(1);
    e.lengths = lengths->data_ptr<int32_t>();
    e.weights = w->data_ptr<float>();
    e.positions = w->size(2);
    e.weights_head = e.positions;
    e.weights_seq = e.positions * kv->heads;
    e.seqs = (int32_t)seqs;
    e.to = to ? to->data_ptr<int32_t>() : nullptr;
    e.to_stride = to ? to->stride(0) : 0;
    e.to_pages = to ? to->size(1) : 0;
    at::Tensor kept = at::empty({seqs, kv->heads, e.keep}, centres.options().dtype(at::kInt));
    at::Tensor left = to ? at::empty({seqs}, lengths->options()) : *lengths;
    at::Tensor out = to ? at::empty(w->sizes(), w->options()) : *w;
    const int rc = evict_fn(kv, &e, kept.data_ptr<int32_t>(), left.data_ptr<int32_t>(), out.data_ptr<float>(),
                            e.weights_seq, e.weights_head, PyLong_AsVoidPtr(a[2]));
    if (rc) return PyLong_FromLong(rc);
    if (to)
        return Py_BuildValue("(NNN)", THPVariable_Wrap(std::move(kept)), THPVariable_Wrap(std::move(left)),
                             THPVariable_Wrap(std::move(out)));
    return Py_BuildValue("(NOO)", THPVariable_Wrap(std::move(kept)), a[5], a[3]);
    END_HANDLE_TH_ERRORS
}

template <typename F>
PyCFunction fast(F *f) { return reinterpret_cast<PyCFunction>(reinterpret_cast<void (*)()>(f)); }

PyMethodDef methods[] = {{"bind", fast(bind), METH_FASTCALL, nullptr},
                         {"write", fast(write), METH_FASTCALL, nullptr},
                         {"read", fast(read), METH_FASTCALL, nullptr},
                         {"attend", fast(attend), METH_FASTCALL, nullptr},
                         {"bind_serve", fast(bind_serve), METH_FASTCALL, nullptr},
                         {"rotate", fast(rotate), METH_FASTCALL, nullptr},
                         {"attend_tokens", fast(attend_tokens), METH_FASTCALL, nullptr},
                         {"weigh", fast(weigh), METH_FASTCALL, nullptr},
                         {"evict", fast(evict), METH_FASTCALL, nullptr},
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
