// The decoding operators' calls on plain torch tensors, without the Python in between: checks, outputs, workspace, stream and the call into the C ABI, as atk_torch.cpp does for the
// selections.  Each function returns its results, the library's status where that is not 0, or None for whatever is not a plain call - a subclass, a mode, a trace, a type or shape that
// decode.py refuses - which decode.py then does, or refuses, itself.
//
// Of a call of 18 us on two short sequences (two kernels of 7 and 4) Python took 11: a dozen attributes of each tensor, the argument structure, three tensors made.
#include <Python.h>

#include <cmath>
#include <vector>

#include <ATen/ATen.h>
#include <ATen/PythonTorchFunctionTLS.h>
#include <c10/core/impl/TorchDispatchModeTLS.h>
#include <c10/hip/HIPFunctions.h>
#include <c10/hip/HIPStream.h>
#include <torch/csrc/autograd/python_variable.h>
#include <torch/csrc/jit/frontend/tracer.h>
#include <torch/version.h>

#include "../../include/atk_decode.h"

namespace {

struct {
    decltype(&atk_attention_workspace_bytes) attention_bytes;
    decltype(&atk_shared_prefix_attention) attention;
    decltype(&atk_verify_workspace_bytes) verify_bytes;
    decltype(&atk_verify_drafts) verify;
    decltype(&atk_copy_pages) copy;
    decltype(&atk_fork_sequences) fork;
    decltype(&atk_append_tokens) append;
    decltype(&atk_free_sequences) free;
    decltype(&atk_compact_pages) compact;
} lib;  // of the library that binding.py has loaded

bool plain_mode() {
    return lib.attention && !at::impl::torch_function_mode_enabled() && !c10::impl::TorchDispatchModeTLS::any_modes_set() && !torch::jit::tracer::isTracing();
}
// a plain tensor on that device (-1: any GPU, which it becomes); NULL if it is none
const at::Tensor *tensor(PyObject *o, int *device) {
    if (!THPVariable_CheckExact(o)) return nullptr;
    const at::Tensor &t = THPVariable_Unpack(o);
    if (!t.is_cuda() || t.layout() != at::kStrided || !t.has_storage() ||
        t.key_set().has_any(c10::DispatchKeySet({c10::DispatchKey::Python, c10::DispatchKey::FuncTorchBatched, c10::DispatchKey::FuncTorchGradWrapper, c10::DispatchKey::Functionalize})))
        return nullptr;
    if (*device < 0) *device = t.get_device();
    return t.get_device() == *device ? &t : nullptr;
}
const at::Tensor *ints(PyObject *o, int *device, std::initializer_list<int64_t> shape) {
    const at::Tensor *t = tensor(o, device);
    return t && t->scalar_type() == at::kInt && t->sizes() == at::IntArrayRef(shape) && t->is_contiguous() ? t : nullptr;
}
int type_of(const at::Tensor &t) {
    return t.scalar_type() == at::kFloat ? ATK_F32 : t.scalar_type() == at::kBFloat16 ? ATK_BF16 : t.scalar_type() == at::kHalf ? ATK_F16 : -1;
}
bool integer(PyObject *o, int64_t *out) {
    if (!PyLong_CheckExact(o)) return false;
    int over = 0;
    *out = PyLong_AsLongLongAndOverflow(o, &over);
    return over == 0;
}
void *stream_of(int device) { return c10::hip::getCurrentHIPStream((c10::DeviceIndex)device).stream(); }

PyObject *pair(at::Tensor &&a, at::Tensor &&b) {
    PyObject *x = THPVariable_Wrap(std::move(a));
    if (!x) return nullptr;
    PyObject *y = THPVariable_Wrap(std::move(b));
    PyObject *both = y ? PyTuple_New(2) : nullptr;
    if (!both) {
        Py_DECREF(x);
        Py_XDECREF(y);
        return nullptr;
    }
    PyTuple_SET_ITEM(both, 0, x);
    PyTuple_SET_ITEM(both, 1, y);
    return both;
}

// None for what `body` throws (no memory, say: the Python path meets the same and says so in torch's words)
template <typename BODY>
PyObject *plain(BODY body) {
    try {
        if (!plain_mode()) Py_RETURN_NONE;
        return body();
    } catch (...) {
        PyErr_Clear();
        Py_RETURN_NONE;
    }
}

// attention(q, k_pages, v_pages, page_table, lens, prefix_len, seqs, scale, return_lse, status)
PyObject *attention(PyObject *, PyObject *const *x, Py_ssize_t n) {
    return plain([&]() -> PyObject * {
        int device = -1;
        int64_t prefix;
        if (n != 10 || !integer(x[5], &prefix) || (x[7] != Py_None && !PyFloat_CheckExact(x[7])) || !PyBool_Check(x[8])) Py_RETURN_NONE;
        const at::Tensor *q = tensor(x[0], &device), *k = tensor(x[1], &device), *v = tensor(x[2], &device), *table = tensor(x[3], &device);
        if (!q || !k || !v || !table || device != c10::hip::current_device() || q->dim() != 4 || k->dim() != 4 || v->sizes() != k->sizes() || table->dim() != 2) Py_RETURN_NONE;
        atk_attention_args a = {};
        a.dtype = type_of(*q);
        a.batch = q->size(0), a.tokens = q->size(1), a.heads = q->size(2), a.dim = q->size(3);
        a.n_pages = k->size(0), a.page_size = k->size(1), a.kv_heads = k->size(2), a.rows = table->size(0), a.row_pages = table->size(1), a.prefix_len = prefix;
        const at::Tensor *lens = ints(x[4], &device, {a.rows}), *seqs = x[6] == Py_None ? nullptr : ints(x[6], &device, {a.batch}), *status = x[9] == Py_None ? nullptr : ints(x[9], &device, {1});
        if (!lens || (x[6] != Py_None && !seqs) || (x[9] != Py_None && !status) || (!seqs && a.batch > a.rows)) Py_RETURN_NONE;
        if (a.dtype < 0 || k->scalar_type() != q->scalar_type() || v->scalar_type() != q->scalar_type() || k->size(3) != a.dim || q->numel() == 0 || k->numel() == 0 || table->numel() == 0 ||
            a.heads % a.kv_heads || table->scalar_type() != at::kInt || table->stride(1) != 1 || q->stride(3) != 1 || k->stride(3) != 1 || v->stride(3) != 1 || prefix < 0 ||
            prefix > a.row_pages * a.page_size)
            Py_RETURN_NONE;
        a.table_stride = a.rows > 1 ? table->stride(0) : a.row_pages;
        at::Tensor out = at::empty({a.batch, a.tokens, a.heads, a.dim}, q->options());
        for (int i = 0; i < 3; ++i) a.q_stride[i] = q->stride(i), a.k_stride[i] = k->stride(i), a.v_stride[i] = v->stride(i), a.out_stride[i] = out.stride(i);
        a.scale = x[7] == Py_None ? 1.0 / std::sqrt((double)a.dim) : PyFloat_AS_DOUBLE(x[7]);
        const bool with_lse = x[8] == Py_True;
        at::Tensor lse;
        if (with_lse) lse = at::empty({a.batch, a.tokens, a.heads}, q->options().dtype(at::kFloat));
        a.q = q->data_ptr(), a.k = k->data_ptr(), a.v = v->data_ptr(), a.out = out.data_ptr(), a.lse = with_lse ? (float *)lse.data_ptr() : nullptr;
        a.page_table = (const int32_t *)table->data_ptr(), a.lens = (const int32_t *)lens->data_ptr(), a.seqs = seqs ? (const int32_t *)seqs->data_ptr() : nullptr;
        a.status = status ? (int32_t *)status->data_ptr() : nullptr;
        const int64_t bytes = lib.attention_bytes(&a);
        if (bytes < 0) return PyLong_FromLongLong(bytes);
        at::Tensor work = at::empty({bytes}, q->options().dtype(at::kByte));
        void *const stream = stream_of(device), *const wp = work.data_ptr();
        int code;
        Py_BEGIN_ALLOW_THREADS
        code = lib.attention(&a, wp, bytes, stream);
        Py_END_ALLOW_THREADS
        if (code != ATK_OK) return PyLong_FromLong(code);
        return with_lse ? pair(std::move(out), std::move(lse)) : THPVariable_Wrap(std::move(out));
    });
}

// verify(target_probs, draft_tokens, draft_probs, accept_random, final_random, n_drafts)
PyObject *verify(PyObject *, PyObject *const *x, Py_ssize_t n) {
    return plain([&]() -> PyObject * {
        int device = -1;
        if (n != 6) Py_RETURN_NONE;
        const at::Tensor *p = tensor(x[0], &device), *tokens = tensor(x[1], &device), *d = x[2] == Py_None ? nullptr : tensor(x[2], &device), *u = tensor(x[3], &device), *r = tensor(x[4], &device);
        if (!p || !tokens || (x[2] != Py_None && !d) || !u || !r || device != c10::hip::current_device() || p->dim() != 3 || tokens->dim() != 2) Py_RETURN_NONE;
        const int64_t B = tokens->size(0), L = tokens->size(1), V = p->size(2);
        const int type = type_of(*p);
        const at::Tensor *count = x[5] == Py_None ? nullptr : ints(x[5], &device, {B});
        if (type < 0 || B == 0 || L == 0 || V == 0 || p->size(0) != B || p->size(1) != L + 1 || p->stride(2) != 1 || !ints(x[1], &device, {B, L}) || (x[5] != Py_None && !count) ||
            u->scalar_type() != at::kFloat || r->scalar_type() != at::kFloat || u->sizes() != at::IntArrayRef({B, L}) || r->sizes() != at::IntArrayRef({B}) || !u->is_contiguous() ||
            !r->is_contiguous())
            Py_RETURN_NONE;
        if (d && (d->scalar_type() != p->scalar_type() || d->sizes() != at::IntArrayRef({B, L, V}) || d->stride(2) != 1)) Py_RETURN_NONE;
        at::Tensor accepted = at::empty({B}, tokens->options()), out = at::empty({B, L + 1}, tokens->options());
        const int64_t bytes = lib.verify_bytes(B, L, V);
        if (bytes < 0) return PyLong_FromLongLong(bytes);
        at::Tensor work = at::empty({bytes}, tokens->options().dtype(at::kByte));
        const int64_t ps[2] = {p->stride(0), p->stride(1)}, ds[2] = {d ? d->stride(0) : 0, d ? d->stride(1) : 0};
        const int code = lib.verify(p->data_ptr(), ps, d ? d->data_ptr() : nullptr, ds, (const int32_t *)tokens->data_ptr(), (const float *)u->data_ptr(), (const float *)r->data_ptr(),
                                    count ? (const int32_t *)count->data_ptr() : nullptr, B, L, V, type, (int32_t *)accepted.data_ptr(), (int32_t *)out.data_ptr(), work.data_ptr(), bytes,
                                    stream_of(device));
        if (code != ATK_OK) return PyLong_FromLong(code);
        return pair(std::move(accepted), std::move(out));
    });
}

// The pools of a list: their addresses, and the bytes of a token in each; false if they are not as the calls take them.
bool pools_of(PyObject *list, int *device, int64_t pages, int64_t page_size, std::vector<void *> *at, int64_t *token_bytes) {
    if (!PyList_CheckExact(list) || pages < 1 || page_size < 1) return false;
    const Py_ssize_t n = PyList_GET_SIZE(list);
    at->resize(n);
    *token_bytes = 0;
    for (Py_ssize_t i = 0; i < n; ++i) {
        const at::Tensor *t = tensor(PyList_GET_ITEM(list, i), device);
        if (!t || t->dim() < 2 || t->size(0) != pages || t->size(1) != page_size || !t->is_contiguous()) return false;
        const int64_t bytes = t->numel() / (pages * page_size) * t->element_size();
        if (i && bytes != *token_bytes) return false;
        *token_bytes = bytes;
        (*at)[i] = t->data_ptr();
    }
    return n > 0 && *token_bytes > 0;
}
// The table of a PageTables object, by the address of its argument structure.
const atk_page_tables *tables_of(PyObject *o) {
    int64_t at;
    return integer(o, &at) ? (const atk_page_tables *)(intptr_t)at : nullptr;
}
PyObject *said(int code) {  // 0 is a result here: what is None is not done yet
    return PyLong_FromLong(code);
}

// fork(tables' address, device, pools, parents, children)
PyObject *fork(PyObject *, PyObject *const *x, Py_ssize_t n) {
    return plain([&]() -> PyObject * {
        int64_t device_no, token_bytes;
        const atk_page_tables *t = n == 5 ? tables_of(x[0]) : nullptr;
        if (!t || !integer(x[1], &device_no) || device_no != c10::hip::current_device()) Py_RETURN_NONE;
        int device = (int)device_no;
        const at::Tensor *parents = tensor(x[3], &device);
        if (!parents || parents->dim() != 1) Py_RETURN_NONE;
        const int64_t count = parents->size(0);
        std::vector<void *> pools;
        if (count == 0 || count > t->rows || !ints(x[3], &device, {count}) || !ints(x[4], &device, {count}) || !pools_of(x[2], &device, t->n_pages, t->page_size, &pools, &token_bytes)) Py_RETURN_NONE;
        return said(lib.fork(t, pools.data(), (int64_t)pools.size(), token_bytes, (const int32_t *)parents->data_ptr(), (const int32_t *)THPVariable_Unpack(x[4]).data_ptr(), count, stream_of(device)));
    });
}

// append(tables' address, device, pools, seqs, values)
PyObject *append(PyObject *, PyObject *const *x, Py_ssize_t n) {
    return plain([&]() -> PyObject * {
        int64_t device_no, token_bytes;
        const atk_page_tables *t = n == 5 ? tables_of(x[0]) : nullptr;
        if (!t || !integer(x[1], &device_no) || device_no != c10::hip::current_device() || !PyList_CheckExact(x[4]) || !PyList_CheckExact(x[2])) Py_RETURN_NONE;
        int device = (int)device_no;
        const at::Tensor *seqs = tensor(x[3], &device);
        if (!seqs || seqs->dim() != 1) Py_RETURN_NONE;
        const int64_t count = seqs->size(0);
        std::vector<void *> pools;
        if (count == 0 || count > t->rows || !ints(x[3], &device, {count}) || !pools_of(x[2], &device, t->n_pages, t->page_size, &pools, &token_bytes) || PyList_GET_SIZE(x[4]) != (Py_ssize_t)pools.size())
            Py_RETURN_NONE;
        std::vector<void *> values(pools.size());
        std::vector<int64_t> strides(pools.size());
        int64_t tokens = 0;
        for (size_t i = 0; i < pools.size(); ++i) {
            const at::Tensor *v = tensor(PyList_GET_ITEM(x[4], i), &device);
            const at::Tensor &p = THPVariable_Unpack(PyList_GET_ITEM(x[2], i));
            if (!v || v->dim() < 2 || v->size(0) != count || v->scalar_type() != p.scalar_type() || v->sizes().slice(2) != p.sizes().slice(2) || (i && v->size(1) != tokens)) Py_RETURN_NONE;
            tokens = v->size(1);
            if (tokens == 0 || !(v->is_contiguous() || (*v)[0].is_contiguous())) Py_RETURN_NONE;
            values[i] = v->data_ptr();
            strides[i] = count > 1 ? v->stride(0) * v->element_size() : tokens * token_bytes;
        }
        return said(lib.append(t, pools.data(), (const void *const *)values.data(), strides.data(), (int64_t)pools.size(), token_bytes, (const int32_t *)seqs->data_ptr(), count, tokens,
                               stream_of(device)));
    });
}

// free(tables' address, device, seqs, drop)
PyObject *release(PyObject *, PyObject *const *x, Py_ssize_t n) {
    return plain([&]() -> PyObject * {
        int64_t device_no;
        const atk_page_tables *t = n == 4 ? tables_of(x[0]) : nullptr;
        if (!t || !integer(x[1], &device_no) || device_no != c10::hip::current_device()) Py_RETURN_NONE;
        int device = (int)device_no;
        const at::Tensor *seqs = tensor(x[2], &device);
        if (!seqs || seqs->dim() != 1) Py_RETURN_NONE;
        const int64_t count = seqs->size(0);
        const at::Tensor *drop = x[3] == Py_None ? nullptr : ints(x[3], &device, {count});
        if (count == 0 || count > t->rows || !ints(x[2], &device, {count}) || (x[3] != Py_None && !drop)) Py_RETURN_NONE;
        return said(lib.free(t, (const int32_t *)seqs->data_ptr(), drop ? (const int32_t *)drop->data_ptr() : nullptr, count, stream_of(device)));
    });
}

// compact(tables' address, device, pools): remap
PyObject *compact(PyObject *, PyObject *const *x, Py_ssize_t n) {
    return plain([&]() -> PyObject * {
        int64_t device_no, token_bytes;
        const atk_page_tables *t = n == 3 ? tables_of(x[0]) : nullptr;
        if (!t || !integer(x[1], &device_no) || device_no != c10::hip::current_device()) Py_RETURN_NONE;
        int device = (int)device_no;
        std::vector<void *> pools;
        if (!pools_of(x[2], &device, t->n_pages, t->page_size, &pools, &token_bytes)) Py_RETURN_NONE;
        at::Tensor remap = at::empty({t->n_pages}, THPVariable_Unpack(PyList_GET_ITEM(x[2], 0)).options().dtype(at::kInt));
        const int code = lib.compact(t, pools.data(), (int64_t)pools.size(), token_bytes, (int32_t *)remap.data_ptr(), stream_of(device));
        return code != ATK_OK ? PyLong_FromLong(code) : THPVariable_Wrap(std::move(remap));
    });
}

// copy(src_pools, src_ids, dst_pools, dst_ids, status)
PyObject *copy(PyObject *, PyObject *const *x, Py_ssize_t n) {
    return plain([&]() -> PyObject * {
        int device = -1;
        if (n != 5 || !PyList_CheckExact(x[0]) || !PyList_CheckExact(x[2]) || PyList_GET_SIZE(x[0]) == 0 || PyList_GET_SIZE(x[0]) != PyList_GET_SIZE(x[2])) Py_RETURN_NONE;
        const at::Tensor *src_ids = tensor(x[1], &device);
        if (!src_ids || src_ids->dim() != 1 || device != c10::hip::current_device()) Py_RETURN_NONE;
        const int64_t count = src_ids->size(0);
        const at::Tensor *s = tensor(PyList_GET_ITEM(x[0], 0), &device), *d = tensor(PyList_GET_ITEM(x[2], 0), &device), *status = x[4] == Py_None ? nullptr : ints(x[4], &device, {1});
        if (count == 0 || !ints(x[1], &device, {count}) || !ints(x[3], &device, {count}) || (x[4] != Py_None && !status) || !s || !d || s->dim() < 2 || d->dim() < 2) Py_RETURN_NONE;
        std::vector<void *> src, dst;
        int64_t token_bytes, other;
        const int64_t sp = s->size(0), dp = d->size(0), page_size = s->size(1);
        if (!pools_of(x[0], &device, sp, page_size, &src, &token_bytes) || !pools_of(x[2], &device, dp, page_size, &dst, &other) || token_bytes != other) Py_RETURN_NONE;
        for (size_t i = 0; i < src.size(); ++i) {
            const at::Tensor &a = THPVariable_Unpack(PyList_GET_ITEM(x[0], i)), &b = THPVariable_Unpack(PyList_GET_ITEM(x[2], i));
            if (a.scalar_type() != b.scalar_type() || a.sizes().slice(1) != b.sizes().slice(1)) Py_RETURN_NONE;
        }
        return said(lib.copy((const void *const *)src.data(), dst.data(), (int64_t)src.size(), token_bytes * page_size, sp, dp, (const int32_t *)src_ids->data_ptr(),
                             (const int32_t *)THPVariable_Unpack(x[3]).data_ptr(), count, status ? (int32_t *)status->data_ptr() : nullptr, stream_of(device)));
    });
}

// use(the addresses of the C ABI's functions, in the order of `lib`)
PyObject *use(PyObject *, PyObject *const *args, Py_ssize_t n) {
    void *at[9];
    if (n != 9) {
        PyErr_SetString(PyExc_TypeError, "nine addresses");
        return nullptr;
    }
    for (int i = 0; i < 9; ++i) {
        at[i] = PyLong_AsVoidPtr(args[i]);
        if (PyErr_Occurred()) return nullptr;
    }
    lib.attention_bytes = (decltype(lib.attention_bytes))at[0], lib.attention = (decltype(lib.attention))at[1], lib.verify_bytes = (decltype(lib.verify_bytes))at[2];
    lib.verify = (decltype(lib.verify))at[3], lib.copy = (decltype(lib.copy))at[4], lib.fork = (decltype(lib.fork))at[5], lib.append = (decltype(lib.append))at[6];
    lib.free = (decltype(lib.free))at[7], lib.compact = (decltype(lib.compact))at[8];
    Py_RETURN_NONE;
}

#define ATK_METHOD(name, f) {name, (PyCFunction)(void (*)())f, METH_FASTCALL, nullptr}
PyMethodDef methods[] = {
    ATK_METHOD("attention", attention), ATK_METHOD("verify", verify), ATK_METHOD("fork", fork), ATK_METHOD("append", append), ATK_METHOD("free", release),
    ATK_METHOD("compact", compact),     ATK_METHOD("copy", copy),     ATK_METHOD("use", use),   {nullptr, nullptr, 0, nullptr},
};
PyModuleDef module = {PyModuleDef_HEAD_INIT, "_atk_decode", nullptr, -1, methods, nullptr, nullptr, nullptr, nullptr};

}  // namespace

PyMODINIT_FUNC PyInit__atk_decode() {
    PyObject *m = PyModule_Create(&module);
    if (m && PyModule_AddStringConstant(m, "torch_version", TORCH_VERSION) < 0) {  // (this file knows torch's own structures: for that release alone)
        Py_DECREF(m);
        return nullptr;
    }
    return m;
}
