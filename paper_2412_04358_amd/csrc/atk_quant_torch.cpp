// The calls of quantized.py and scores.py on plain torch tensors, without the Python in between, as atk_decode_torch.cpp does for decode.py: results, the library's status where that is
// not 0, or None for whatever is not a plain call, which the Python code then does, or refuses, itself.
//
// Of a call of 16 us on two short sequences (one kernel of 7) Python took 10.
#include "atk_plain_torch.h"

#include "../../include/atk_quant.h"
#include "../../include/atk_scores.h"

namespace {

struct {
    decltype(&atk_quant_token_bytes) token_bytes;
    decltype(&atk_append_quantized) append;
    decltype(&atk_read_quantized) read;
    decltype(&atk_quant_attention_workspace_bytes) attention_bytes;
    decltype(&atk_quant_attention) attention;
    decltype(&atk_token_logprobs_workspace_bytes) logprobs_bytes;
    decltype(&atk_token_logprobs) logprobs;
    decltype(&atk_token_logprobs_grad) grad;
} lib;  // of the library that binding.py has loaded

const at::Tensor *pool(PyObject *o, int *device, int64_t pages, int64_t page_size, int64_t token_bytes) {
    const at::Tensor *t = tensor(o, device);
    return t && t->scalar_type() == at::kByte && t->sizes() == at::IntArrayRef({pages, page_size, token_bytes}) && t->is_contiguous() ? t : nullptr;
}
const at::Tensor *floats(PyObject *o, int *device, int64_t rows, int64_t tokens) {
    const at::Tensor *t = tensor(o, device);
    return t && t->scalar_type() == at::kFloat && t->sizes() == at::IntArrayRef({rows, tokens}) && t->is_contiguous() ? t : nullptr;
}
template <typename T>
T *address(const at::Tensor *t) { return t ? (T *)t->data_ptr() : nullptr; }

// A tuple (or list) of tensors that are handed over.
PyObject *several(std::vector<at::Tensor> &&all, bool list) {
    PyObject *out = list ? PyList_New((Py_ssize_t)all.size()) : PyTuple_New((Py_ssize_t)all.size());
    if (!out) return nullptr;
    for (size_t i = 0; i < all.size(); ++i) {
        PyObject *t = THPVariable_Wrap(std::move(all[i]));
        if (!t) {
            Py_DECREF(out);
            return nullptr;
        }
        if (list)
            PyList_SET_ITEM(out, (Py_ssize_t)i, t);
        else
            PyTuple_SET_ITEM(out, (Py_ssize_t)i, t);
    }
    return out;
}

// attention(q, k_pages, v_pages, page_table, lens, kv_heads, bits, seqs, scale, return_lse, status)
PyObject *attention(PyObject *, PyObject *const *x, Py_ssize_t n) {
    return plain([&]() -> PyObject * {
        int device = -1;
        int64_t kv_heads, bits;
        if (n != 11 || !integer(x[5], &kv_heads) || !integer(x[6], &bits) || (x[8] != Py_None && !PyFloat_CheckExact(x[8])) || !PyBool_Check(x[9])) Py_RETURN_NONE;
        const at::Tensor *q = tensor(x[0], &device), *k = tensor(x[1], &device), *table = tensor(x[3], &device);
        if (!q || !k || !table || device != c10::hip::current_device() || q->dim() != 4 || k->dim() != 3 || table->dim() != 2 || (bits != 4 && bits != 8)) Py_RETURN_NONE;
        atk_quant_attention_args a = {};
        a.dtype = type_of(*q), a.bits = (int32_t)bits;
        a.batch = q->size(0), a.tokens = q->size(1), a.heads = q->size(2), a.dim = q->size(3), a.kv_heads = kv_heads;
        a.n_pages = k->size(0), a.page_size = k->size(1), a.rows = table->size(0), a.row_pages = table->size(1);
        const int64_t token_bytes = lib.token_bytes(kv_heads, a.dim, a.bits);
        if (token_bytes < 0 || a.dtype < 0 || a.heads % kv_heads || q->numel() == 0 || k->numel() == 0 || table->numel() == 0 || table->scalar_type() != at::kInt || table->stride(1) != 1 ||
            q->stride(3) != 1 || !pool(x[1], &device, a.n_pages, a.page_size, token_bytes))
            Py_RETURN_NONE;
        const at::Tensor *v = pool(x[2], &device, a.n_pages, a.page_size, token_bytes), *lens = ints(x[4], &device, {a.rows});
        const at::Tensor *seqs = x[7] == Py_None ? nullptr : ints(x[7], &device, {a.batch}), *status = x[10] == Py_None ? nullptr : ints(x[10], &device, {1});
        if (!v || !lens || (x[7] != Py_None && !seqs) || (x[10] != Py_None && !status) || (!seqs && a.batch > a.rows)) Py_RETURN_NONE;
        a.table_stride = a.rows > 1 ? table->stride(0) : a.row_pages;
        std::vector<at::Tensor> outs;
        outs.push_back(at::empty({a.batch, a.tokens, a.heads, a.dim}, q->options()));
        if (x[9] == Py_True) outs.push_back(at::empty({a.batch, a.tokens, a.heads}, q->options().dtype(at::kFloat)));
        for (int i = 0; i < 3; ++i) a.q_stride[i] = q->stride(i), a.out_stride[i] = outs[0].stride(i);
        a.scale = x[8] == Py_None ? 1.0 / std::sqrt((double)a.dim) : PyFloat_AS_DOUBLE(x[8]);
        a.q = q->data_ptr(), a.k = k->data_ptr(), a.v = v->data_ptr(), a.out = outs[0].data_ptr(), a.lse = outs.size() > 1 ? (float *)outs[1].data_ptr() : nullptr;
        a.page_table = address<const int32_t>(table), a.lens = address<const int32_t>(lens), a.seqs = address<const int32_t>(seqs), a.status = address<int32_t>(status);
        const int64_t bytes = lib.attention_bytes(&a);
        if (bytes < 0) return PyLong_FromLongLong(bytes);
        const at::Tensor work = at::empty({bytes}, k->options());
        void *const stream = stream_of(device), *const wp = work.data_ptr();
        int code;
        Py_BEGIN_ALLOW_THREADS
        code = lib.attention(&a, wp, bytes, stream);
        Py_END_ALLOW_THREADS
        if (code != ATK_OK) return PyLong_FromLong(code);
        return outs.size() > 1 ? several(std::move(outs), false) : THPVariable_Wrap(std::move(outs[0]));
    });
}

// The addresses of a list of pools.
bool pools_of(PyObject *list, int *device, const atk_page_tables *t, int64_t token_bytes, std::vector<void *> *at) {
    if (!PyList_CheckExact(list) || PyList_GET_SIZE(list) == 0) return false;
    at->resize(PyList_GET_SIZE(list));
    for (size_t i = 0; i < at->size(); ++i) {
        const at::Tensor *p = pool(PyList_GET_ITEM(list, (Py_ssize_t)i), device, t->n_pages, t->page_size, token_bytes);
        if (!p) return false;
        (*at)[i] = p->data_ptr();
    }
    return true;
}

// append(tables' address, device, pools, seqs, values, bits)
PyObject *append(PyObject *, PyObject *const *x, Py_ssize_t n) {
    return plain([&]() -> PyObject * {
        int64_t device_no, bits;
        const atk_page_tables *t = n == 6 ? tables_of(x[0]) : nullptr;
        if (!t || !integer(x[1], &device_no) || device_no != c10::hip::current_device() || !integer(x[5], &bits) || (bits != 4 && bits != 8) || !PyList_CheckExact(x[4]) || PyList_GET_SIZE(x[4]) == 0)
            Py_RETURN_NONE;
        int device = (int)device_no;
        const at::Tensor *seqs = tensor(x[3], &device), *first = tensor(PyList_GET_ITEM(x[4], 0), &device);
        if (!seqs || seqs->dim() != 1 || !first || first->dim() != 4 || type_of(*first) < 0) Py_RETURN_NONE;
        const int64_t count = seqs->size(0), tokens = first->size(1), heads = first->size(2), dim = first->size(3), token_bytes = lib.token_bytes(heads, dim, (int)bits);
        std::vector<void *> pools;
        if (count == 0 || tokens == 0 || count > t->rows || token_bytes < 0 || !ints(x[3], &device, {count}) || !pools_of(x[2], &device, t, token_bytes, &pools) ||
            PyList_GET_SIZE(x[4]) != (Py_ssize_t)pools.size())
            Py_RETURN_NONE;
        std::vector<void *> values(pools.size());
        std::vector<int64_t> strides(2 * pools.size());
        for (size_t i = 0; i < pools.size(); ++i) {
            const at::Tensor *v = tensor(PyList_GET_ITEM(x[4], (Py_ssize_t)i), &device);
            if (!v || v->sizes() != at::IntArrayRef({count, tokens, heads, dim}) || v->scalar_type() != first->scalar_type() || v->stride(3) != 1 || (heads > 1 && v->stride(2) != dim)) Py_RETURN_NONE;
            values[i] = v->data_ptr();
            strides[2 * i] = v->stride(0) * v->element_size(), strides[2 * i + 1] = v->stride(1) * v->element_size();
        }
        return PyLong_FromLong(lib.append(t, pools.data(), (const void *const *)values.data(), strides.data(), (int64_t)pools.size(), heads, dim, (int)bits, type_of(*first),
                                          address<const int32_t>(seqs), count, tokens, stream_of(device)));  // (0 is a result here: what is None is not done yet)
    });
}

// read(tables' address, device, pools, seqs, starts, tokens, kv_heads, dim, bits, type's code)
PyObject *read(PyObject *, PyObject *const *x, Py_ssize_t n) {
    return plain([&]() -> PyObject * {
        int64_t device_no, tokens, heads, dim, bits, type;
        const atk_page_tables *t = n == 10 ? tables_of(x[0]) : nullptr;
        if (!t || !integer(x[1], &device_no) || device_no != c10::hip::current_device() || !integer(x[5], &tokens) || !integer(x[6], &heads) || !integer(x[7], &dim) || !integer(x[8], &bits) ||
            !integer(x[9], &type) || (bits != 4 && bits != 8))
            Py_RETURN_NONE;
        int device = (int)device_no;
        const at::Tensor *seqs = tensor(x[3], &device);
        if (!seqs || seqs->dim() != 1) Py_RETURN_NONE;
        const int64_t count = seqs->size(0), token_bytes = lib.token_bytes(heads, dim, (int)bits);
        const at::Tensor *starts = x[4] == Py_None ? nullptr : ints(x[4], &device, {count});
        std::vector<void *> pools;
        if (count == 0 || tokens < 1 || token_bytes < 0 || !ints(x[3], &device, {count}) || (x[4] != Py_None && !starts) || !pools_of(x[2], &device, t, token_bytes, &pools)) Py_RETURN_NONE;
        const at::TensorOptions options = seqs->options().dtype(type == ATK_F32 ? at::kFloat : type == ATK_BF16 ? at::kBFloat16 : at::kHalf);
        std::vector<at::Tensor> outs;
        std::vector<void *> at_outs;
        for (size_t i = 0; i < pools.size(); ++i) {
            outs.push_back(at::empty({count, tokens, heads, dim}, options));
            at_outs.push_back(outs[i].data_ptr());
        }
        const int code = lib.read(t, (const void *const *)pools.data(), at_outs.data(), (int64_t)pools.size(), heads, dim, (int)bits, (int)type, address<const int32_t>(seqs),
                                  address<const int32_t>(starts), count, tokens, stream_of(device));
        return code != ATK_OK ? PyLong_FromLong(code) : several(std::move(outs), true);
    });
}

// logprobs(logits, tokens, top)
PyObject *logprobs(PyObject *, PyObject *const *x, Py_ssize_t n) {
    return plain([&]() -> PyObject * {
        int device = -1;
        int64_t top;
        if (n != 3 || !integer(x[2], &top)) Py_RETURN_NONE;
        const at::Tensor *p = tensor(x[0], &device);
        if (!p || device != c10::hip::current_device() || p->dim() != 3 || p->numel() == 0 || p->stride(2) != 1 || type_of(*p) < 0) Py_RETURN_NONE;
        const int64_t B = p->size(0), T = p->size(1), V = p->size(2);
        const at::Tensor *tokens = ints(x[1], &device, {B, T});
        if (!tokens || top < 0 || top > 32 || top > V) Py_RETURN_NONE;
        const int type = type_of(*p);
        const int64_t bytes = lib.logprobs_bytes(B, T, V, top, type);
        if (bytes < 0) return PyLong_FromLongLong(bytes);
        const at::TensorOptions f32 = tokens->options().dtype(at::kFloat);
        std::vector<at::Tensor> outs;
        for (int i = 0; i < 3; ++i) outs.push_back(at::empty({B, T}, f32));
        outs.push_back(at::empty({B, T, top}, f32));
        outs.push_back(at::empty({B, T, top}, tokens->options()));
        const at::Tensor work = at::empty({bytes}, tokens->options().dtype(at::kByte));
        const int64_t strides[2] = {p->stride(0), p->stride(1)};
        const int code = lib.logprobs(p->data_ptr(), strides, address<const int32_t>(tokens), B, T, V, top, type, address<float>(&outs[0]), address<float>(&outs[1]), address<float>(&outs[2]),
                                      address<float>(&outs[3]), address<int32_t>(&outs[4]), work.data_ptr(), bytes, stream_of(device));
        return code != ATK_OK ? PyLong_FromLong(code) : several(std::move(outs), false);
    });
}

// grad(logits, tokens, lse, entropy, grad_logprobs, grad_entropy)
PyObject *grad(PyObject *, PyObject *const *x, Py_ssize_t n) {
    return plain([&]() -> PyObject * {
        int device = -1;
        if (n != 6) Py_RETURN_NONE;
        const at::Tensor *p = tensor(x[0], &device);
        if (!p || device != c10::hip::current_device() || p->dim() != 3 || p->numel() == 0 || p->stride(2) != 1 || type_of(*p) < 0) Py_RETURN_NONE;
        const int64_t B = p->size(0), T = p->size(1), V = p->size(2);
        const at::Tensor *tokens = ints(x[1], &device, {B, T}), *some[4];
        for (int i = 0; i < 4; ++i) {
            some[i] = x[2 + i] == Py_None ? nullptr : floats(x[2 + i], &device, B, T);
            if (x[2 + i] != Py_None && !some[i]) Py_RETURN_NONE;
        }
        if (!tokens || !some[0] || (some[3] && !some[1])) Py_RETURN_NONE;
        at::Tensor out = at::empty({B, T, V}, p->options());
        const int64_t strides[2] = {p->stride(0), p->stride(1)}, out_strides[2] = {out.stride(0), out.stride(1)};
        const int code = lib.grad(p->data_ptr(), strides, address<const int32_t>(tokens), address<const float>(some[0]), address<const float>(some[1]), address<const float>(some[2]),
                                  address<const float>(some[3]), B, T, V, type_of(*p), out.data_ptr(), out_strides, stream_of(device));
        return code != ATK_OK ? PyLong_FromLong(code) : THPVariable_Wrap(std::move(out));
    });
}

// use(the addresses of the C ABI's functions, in the order of `lib`)
PyObject *use(PyObject *, PyObject *const *args, Py_ssize_t n) {
    void *at[8];
    if (n != 8) {
        PyErr_SetString(PyExc_TypeError, "eight addresses");
        return nullptr;
    }
    for (int i = 0; i < 8; ++i) {
        at[i] = PyLong_AsVoidPtr(args[i]);
        if (PyErr_Occurred()) return nullptr;
    }
    lib.token_bytes = (decltype(lib.token_bytes))at[0], lib.append = (decltype(lib.append))at[1], lib.read = (decltype(lib.read))at[2];
    lib.attention_bytes = (decltype(lib.attention_bytes))at[3], lib.attention = (decltype(lib.attention))at[4];
    lib.logprobs_bytes = (decltype(lib.logprobs_bytes))at[5], lib.logprobs = (decltype(lib.logprobs))at[6], lib.grad = (decltype(lib.grad))at[7];
    Py_RETURN_NONE;
}

#define ATK_METHOD(name, f) {name, (PyCFunction)(void (*)())f, METH_FASTCALL, nullptr}
PyMethodDef methods[] = {
    ATK_METHOD("attention", attention), ATK_METHOD("append", append), ATK_METHOD("read", read), ATK_METHOD("logprobs", logprobs), ATK_METHOD("grad", grad), ATK_METHOD("use", use),
    {nullptr, nullptr, 0, nullptr},
};
PyModuleDef module = {PyModuleDef_HEAD_INIT, "_atk_quant", nullptr, -1, methods, nullptr, nullptr, nullptr, nullptr};

}  // namespace

PyMODINIT_FUNC PyInit__atk_quant() {
    PyObject *m = PyModule_Create(&module);
    if (m && PyModule_AddStringConstant(m, "torch_version", TORCH_VERSION) < 0) {  // (this file knows torch's own structures: for that release alone)
        Py_DECREF(m);
        return nullptr;
    }
    return m;
}
