// What attend.py asks of torch tensors, in one call each instead of one for each property: a decoding step's calls are
// bound by the host, and a property costs as much from Python as all of them do here.
//
// Each function answers for tensors that are as they should be, and returns None for any other, whatever is wrong with
// it: attend.py then looks again, and says what it is.
#include <Python.h>

#include <ATen/core/Tensor.h>
#include <ATen/ops/empty.h>
#include <torch/csrc/autograd/python_variable.h>

#include <algorithm>
#include <cstdint>

#include "kvx_attend.h"

namespace {

// The tensor behind an argument on `device`, without a gradient to record or a forward-mode tangent (there is one level
// of them), or NULL.
const at::Tensor *tensor_of(PyObject *x, int device) {
    if (!THPVariable_Check(x))
        return nullptr;
    const at::Tensor &t = THPVariable_Unpack(x);
    if (!t.defined() || t.layout() != at::kStrided || t.requires_grad() || t._fw_grad(0).defined() ||
        (t.is_cpu() ? -1 : static_cast<int>(t.get_device())) != device)
        return nullptr;
    return &t;
}

int row_type(const at::Tensor &t) {
    return t.scalar_type() == at::kBFloat16 ? KV_DTYPE_BF16 : t.scalar_type() == at::kHalf ? KV_DTYPE_F16 : 0;
}

PyObject *bytes_of(const void *x, size_t size) {
    return PyBytes_FromStringAndSize(static_cast<const char *>(x), static_cast<Py_ssize_t>(size));
}

// rows(tensor, head_dim, device): (kv_rows, shape)
PyObject *rows(PyObject *, PyObject *const *args, Py_ssize_t count) {
    if (count != 3)
        Py_RETURN_NONE;
    const int64_t head_dim = PyLong_AsLongLong(args[1]);
    const at::Tensor *t = tensor_of(args[0], static_cast<int>(PyLong_AsLong(args[2])));
    if (PyErr_Occurred())
        return nullptr;
    if (!t || t->dim() != 3 || !row_type(*t) || t->size(2) != head_dim || t->stride(2) != 1 || t->size(1) > INT32_MAX)
        Py_RETURN_NONE;
    kv_rows r{};
    r.data = t->data_ptr();
    r.token_stride = t->stride(0);
    r.head_stride = t->stride(1);
    r.heads = static_cast<int32_t>(t->size(1));
    r.dtype = row_type(*t);
    return Py_BuildValue("(N(LLL))", bytes_of(&r, sizeof(r)), static_cast<long long>(t->size(0)),
                         static_cast<long long>(t->size(1)), static_cast<long long>(t->size(2)));
}

// A dense int32 tensor of `dims` dimensions and so many rows, or NULL.
const at::Tensor *ints_of(PyObject *x, int dims, int device, int64_t rows) {
    const at::Tensor *t = tensor_of(x, device);
    return t && t->scalar_type() == at::kInt && t->dim() == dims && (t->stride(-1) == 1 || t->size(-1) <= 1) &&
                   (rows < 0 || t->size(0) == rows)
               ? t
               : nullptr;
}

// ints(tensor, dims, device, rows): the address of a contiguous one
PyObject *ints(PyObject *, PyObject *const *args, Py_ssize_t count) {
    if (count != 4)
        Py_RETURN_NONE;
    const int64_t rows = PyLong_AsLongLong(args[3]);
    const at::Tensor *t = ints_of(args[0], static_cast<int>(PyLong_AsLong(args[1])),
                                  static_cast<int>(PyLong_AsLong(args[2])), rows);
    if (PyErr_Occurred())
        return nullptr;
    if (!t || !t->is_contiguous())
        Py_RETURN_NONE;
    return PyLong_FromUnsignedLongLong(reinterpret_cast<uintptr_t>(t->data_ptr()));
}

// batch(block_size, device, tables, lens, starts, tokens, max_q, max_len): (kv_batch, sequences, max_queries, max_len)
PyObject *batch(PyObject *, PyObject *const *args, Py_ssize_t count) {
    if (count != 8)
        Py_RETURN_NONE;
    const int64_t block_size = PyLong_AsLongLong(args[0]), tokens = PyLong_AsLongLong(args[5]);
    const int device = static_cast<int>(PyLong_AsLong(args[1]));
    if (PyErr_Occurred())
        return nullptr;
    for (const int i : {6, 7})
        if (args[i] != Py_None && !PyLong_CheckExact(args[i]))
            Py_RETURN_NONE;
    const at::Tensor *tables = ints_of(args[2], 2, device, -1);
    if (!tables || tokens >= INT64_C(1) << 31)
        Py_RETURN_NONE;
    const int64_t B = tables->size(0), pages = tables->size(1);
    const at::Tensor *lens = ints_of(args[3], 1, device, B), *starts = nullptr;
    if (!lens || B > INT32_MAX || pages > INT32_MAX)
        Py_RETURN_NONE;
    kv_batch x{};
    x.max_queries = 1;
    if (args[4] == Py_None) {
        if (tokens != B)
            Py_RETURN_NONE;
    } else {
        starts = ints_of(args[4], 1, device, B + 1);
        if (!starts)
            Py_RETURN_NONE;
        int64_t most = tokens;
        if (args[6] != Py_None) {
            int beyond = 0;
            const int64_t asked = PyLong_AsLongLongAndOverflow(args[6], &beyond);
            most = beyond > 0 ? tokens : beyond < 0 ? 0 : std::min(tokens, asked);
        }
        x.max_queries = static_cast<int32_t>(std::max<int64_t>(most, 1));
        x.starts = static_cast<const int32_t *>(starts->data_ptr());
    }
    constexpr int64_t kEnd = INT64_C(1) << 31;
    int64_t most = pages > kEnd / std::max<int64_t>(block_size, 1) ? kEnd : pages * block_size;
    most = std::min<int64_t>(most, kEnd - 1024);
    if (args[7] != Py_None) {
        int beyond = 0;
        const int64_t asked = PyLong_AsLongLongAndOverflow(args[7], &beyond);
        most = beyond > 0 ? most : beyond < 0 ? -1 : std::min(most, std::max<int64_t>(asked, -1));
    }
    x.num_seqs = static_cast<int32_t>(B);
    x.num_queries = static_cast<int32_t>(tokens);
    x.max_len = static_cast<int32_t>(most);
    x.table_len = static_cast<int32_t>(pages);
    x.table_stride = tables->stride(0);
    x.block_tables = static_cast<const int32_t *>(tables->data_ptr());
    x.lens = static_cast<const int32_t *>(lens->data_ptr());
    return Py_BuildValue("(NLLL)", bytes_of(&x, sizeof(x)), static_cast<long long>(B),
                         static_cast<long long>(x.max_queries), static_cast<long long>(most));
}

// scales(tensor, heads, blocks, device): (address, block stride, K to V)
PyObject *scales(PyObject *, PyObject *const *args, Py_ssize_t count) {
    if (count != 4)
        Py_RETURN_NONE;
    const int64_t heads = PyLong_AsLongLong(args[1]), blocks = PyLong_AsLongLong(args[2]);
    const at::Tensor *t = tensor_of(args[0], static_cast<int>(PyLong_AsLong(args[3])));
    if (PyErr_Occurred())
        return nullptr;
    if (!t || (t->scalar_type() != at::kByte && t->scalar_type() != at::ScalarType::Float8_e8m0fnu) || t->dim() != 3 ||
        t->size(0) < std::max<int64_t>(blocks, 2) || t->size(1) != 2 || t->size(2) != heads || t->stride(2) != 1)
        Py_RETURN_NONE;
    return Py_BuildValue("(KLL)", static_cast<unsigned long long>(reinterpret_cast<uintptr_t>(t->data_ptr())),
                         static_cast<long long>(t->stride(0)), static_cast<long long>(t->stride(1)));
}

// lists(pages, counts, tokens, device): (kv_page_list, budget)
PyObject *lists(PyObject *, PyObject *const *args, Py_ssize_t count) {
    if (count != 4)
        Py_RETURN_NONE;
    const int64_t tokens = PyLong_AsLongLong(args[2]);
    const int device = static_cast<int>(PyLong_AsLong(args[3]));
    if (PyErr_Occurred())
        return nullptr;
    const at::Tensor *pages = ints_of(args[0], 3, device, tokens), *counts = ints_of(args[1], 1, device, tokens);
    if (!pages || !counts || !counts->is_contiguous() || pages->size(1) > INT32_MAX || pages->size(2) > INT32_MAX)
        Py_RETURN_NONE;
    kv_page_list x{};
    x.pages = static_cast<const int32_t *>(pages->data_ptr());
    x.counts = static_cast<const int32_t *>(counts->data_ptr());
    x.token_stride = pages->stride(0);
    x.head_stride = pages->stride(1);
    x.heads = static_cast<int32_t>(pages->size(1));
    x.budget = static_cast<int32_t>(pages->size(2));
    return Py_BuildValue("(NL)", bytes_of(&x, sizeof(x)), static_cast<long long>(pages->size(2)));
}

// A contiguous tensor of one dimension and so many elements (any, if negative), or NULL.
const at::Tensor *vector_of(PyObject *x, int64_t elements, int device) {
    const at::Tensor *t = tensor_of(x, device);
    return t && t->dim() == 1 && (elements < 0 || t->size(0) == elements) && t->is_contiguous() ? t : nullptr;
}

// rotation(row type, head_dim, tokens, device, freqs, positions, q_weight, k_weight): (rotary_dim, weights' type,
// freqs, positions, q_weight, k_weight), as kv_rotate_options has them; None for those that are not given
PyObject *rotation(PyObject *, PyObject *const *args, Py_ssize_t count) {
    if (count != 8)
        Py_RETURN_NONE;
    const long type = PyLong_AsLong(args[0]);
    const int64_t head_dim = PyLong_AsLongLong(args[1]), tokens = PyLong_AsLongLong(args[2]);
    const int device = static_cast<int>(PyLong_AsLong(args[3]));
    if (PyErr_Occurred())
        return nullptr;
    int64_t rotary = 0;
    int of_weights = 0;
    const void *at[4] = {};
    if (args[4] != Py_None) {
        const at::Tensor *freqs = vector_of(args[4], -1, device);
        if (!freqs || freqs->scalar_type() != at::kDouble || freqs->size(0) > head_dim)
            Py_RETURN_NONE;
        rotary = 2 * freqs->size(0);
        at[0] = freqs->data_ptr();
    }
    if (args[5] != Py_None) {
        const at::Tensor *positions = vector_of(args[5], tokens, device);
        if (!positions || positions->scalar_type() != at::kInt)
            Py_RETURN_NONE;
        at[1] = positions->data_ptr();
    }
    for (int i = 0; i < 2; ++i) {
        if (args[6 + i] == Py_None)
            continue;
        const at::Tensor *weight = vector_of(args[6 + i], head_dim, device);
        const int is = !weight ? 0 : weight->scalar_type() == at::kFloat ? KV_DTYPE_F32 : row_type(*weight);
        if (!is || (is != KV_DTYPE_F32 && is != type) || (of_weights && of_weights != is))
            Py_RETURN_NONE;
        of_weights = is;
        at[2 + i] = weight->data_ptr();
    }
    const auto address = [&](int i) { return static_cast<unsigned long long>(reinterpret_cast<uintptr_t>(at[i])); };
    return Py_BuildValue("(LiKKKK)", static_cast<long long>(rotary), of_weights, address(0), address(1), address(2),
                         address(3));
}

PyObject *failed(const std::exception &e) {
    PyErr_SetString(PyExc_RuntimeError, e.what());
    return nullptr;
}

// empty(like, type, sizes...), zeros(...): (a contiguous tensor on like's device, its address); type: 0 like's, 1
// float32, 2 int32, 3 bytes
template <bool ZEROS>
PyObject *make(PyObject *, PyObject *const *args, Py_ssize_t count) {
    if (count < 3 || count > 5 || !THPVariable_Check(args[0])) {
        PyErr_SetString(PyExc_TypeError, "a tensor, a type, and up to 3 sizes are needed");
        return nullptr;
    }
    const at::Tensor &like = THPVariable_Unpack(args[0]);
    const long type = PyLong_AsLong(args[1]);
    int64_t sizes[3];
    for (Py_ssize_t i = 2; i < count; ++i)
        sizes[i - 2] = PyLong_AsLongLong(args[i]);
    if (PyErr_Occurred())
        return nullptr;
    const at::ScalarType of = type == 0   ? like.scalar_type()
                              : type == 1 ? at::kFloat
                              : type == 2 ? at::kInt
                                          : at::kByte;
    try {
        const at::IntArrayRef shape(sizes, static_cast<size_t>(count - 2));
        at::Tensor t = at::empty(shape, like.options().dtype(of));
        if (ZEROS)
            t.zero_();
        const auto address = static_cast<unsigned long long>(reinterpret_cast<uintptr_t>(t.data_ptr()));
        PyObject *wrapped = THPVariable_Wrap(std::move(t));
        return wrapped ? Py_BuildValue("(NK)", wrapped, address) : nullptr;
    } catch (const std::exception &e) {
        return failed(e);
    }
}

template <PyObject *(*F)(PyObject *, PyObject *const *, Py_ssize_t)>
PyObject *guarded(PyObject *self, PyObject *const *args, Py_ssize_t count) {
    try {
        return F(self, args, count);
    } catch (const std::exception &) {  // a tensor that does not answer is not as it should be
        PyErr_Clear();
        Py_RETURN_NONE;
    }
}

PyMethodDef methods[] = {
    {"rows", reinterpret_cast<PyCFunction>(reinterpret_cast<void (*)()>(guarded<rows>)), METH_FASTCALL, nullptr},
    {"ints", reinterpret_cast<PyCFunction>(reinterpret_cast<void (*)()>(guarded<ints>)), METH_FASTCALL, nullptr},
    {"batch", reinterpret_cast<PyCFunction>(reinterpret_cast<void (*)()>(guarded<batch>)), METH_FASTCALL, nullptr},
    {"scales", reinterpret_cast<PyCFunction>(reinterpret_cast<void (*)()>(guarded<scales>)), METH_FASTCALL, nullptr},
    {"lists", reinterpret_cast<PyCFunction>(reinterpret_cast<void (*)()>(guarded<lists>)), METH_FASTCALL, nullptr},
    {"rotation", reinterpret_cast<PyCFunction>(reinterpret_cast<void (*)()>(guarded<rotation>)), METH_FASTCALL, nullptr},
    {"empty", reinterpret_cast<PyCFunction>(reinterpret_cast<void (*)()>(make<false>)), METH_FASTCALL, nullptr},
    {"zeros", reinterpret_cast<PyCFunction>(reinterpret_cast<void (*)()>(make<true>)), METH_FASTCALL, nullptr},
    {nullptr, nullptr, 0, nullptr}};

PyModuleDef module = {PyModuleDef_HEAD_INIT, "_tensors", nullptr, -1, methods, nullptr, nullptr, nullptr, nullptr};

}  // namespace

PyMODINIT_FUNC PyInit__tensors() { return PyModule_Create(&module); }
