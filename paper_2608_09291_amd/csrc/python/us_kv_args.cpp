// What the Python binding of the key/value cache asks its tensors for, in one
// call per argument: a small step's launches take the GPU 5 us, and every
// property that Python asks a tensor for takes it 0.1 us (a read of one
// sequence: 8.4 us a call with the questions in Python).
#define PY_SSIZE_T_CLEAN
#include <Python.h>

#include <torch/csrc/autograd/python_variable.h>

namespace {

// Argument i as a tensor, or NULL with a TypeError set.
const at::Tensor *tensor(PyObject *const *args, Py_ssize_t i, const char *name) {
    if (THPVariable_Check(args[i])) return &THPVariable_Unpack(args[i]);
    PyErr_Format(PyExc_TypeError, "%s: a tensor is wanted", name);
    return nullptr;
}

bool count(Py_ssize_t n, Py_ssize_t want) {
    if (n != want) PyErr_Format(PyExc_TypeError, "%zd arguments are wanted, got %zd", want, n);
    return n == want;
}

PyObject *refuse(const char *name, const char *what) {
    return PyErr_Format(PyExc_TypeError, "%s: %s", name, what);
}

unsigned long long address(const at::Tensor &t) { return (unsigned long long)(uintptr_t)t.data_ptr(); }

PyObject *guarded(PyObject *(*f)(PyObject *const *, Py_ssize_t), PyObject *const *args, Py_ssize_t n) {
    try {
        return f(args, n);
    } catch (const std::exception &e) {
        PyErr_SetString(PyExc_TypeError, e.what());
        return nullptr;
    }
}

// Whether t is on GPU `device`, or on any where that is negative.
bool on(const at::Tensor &t, long long device) { return t.is_cuda() && (device < 0 || t.get_device() == device); }

// (k, v, k_scale, v_scale) -> addresses, blocks, heads, bytes of a block, number of the GPU that holds them (-1: not all are on one)
PyObject *cache_of(PyObject *const *args, Py_ssize_t n) {
    if (!count(n, 4)) return nullptr;
    const char *names[4] = {"k", "v", "k_scale", "v_scale"};
    const at::Tensor *t[4];
    bool one = true;
    for (int i = 0; i < 4; ++i) {
        t[i] = tensor(args, i, names[i]);
        if (!t[i]) return nullptr;
        const bool codes = i < 2;
        if (t[i]->dim() != (codes ? 3 : 2) || t[i]->scalar_type() != (codes ? at::kByte : at::kFloat) || !t[i]->is_contiguous() ||
            t[i]->size(0) != t[0]->size(0) || t[i]->size(1) != t[0]->size(1) || (codes && t[i]->size(2) != t[0]->size(2)))
            return refuse(names[i], codes ? "a contiguous uint8 tensor (blocks, heads, bytes of a block) is wanted"
                                          : "a contiguous float32 tensor (blocks, heads) is wanted");
        one = one && t[i]->is_cuda() && t[i]->get_device() == t[0]->get_device();
    }
    return Py_BuildValue("KKKKLLLL", address(*t[0]), address(*t[1]), address(*t[2]), address(*t[3]), (long long)t[0]->size(0),
                         (long long)t[0]->size(1), (long long)t[0]->size(2), one ? (long long)t[0]->get_device() : -1ll);
}

// (blocks, lens, starts or None, device) -> address of blocks, stride, width, batch, addresses of lens and starts
PyObject *seqs_of(PyObject *const *args, Py_ssize_t n) {
    if (!count(n, 4)) return nullptr;
    const at::Tensor *blocks = tensor(args, 0, "blocks"), *lens = blocks ? tensor(args, 1, "lens") : nullptr, *starts = nullptr;
    if (!lens) return nullptr;
    if (args[2] != Py_None && !(starts = tensor(args, 2, "starts"))) return nullptr;
    const long long device = PyLong_AsLongLong(args[3]);
    if (PyErr_Occurred()) return nullptr;
    if (blocks->dim() != 2 || blocks->scalar_type() != at::kInt || (blocks->size(1) > 1 && blocks->stride(1) != 1))
        return refuse("blocks", "an int32 table with contiguous rows is wanted");
    const int64_t batch = blocks->size(0), width = blocks->size(1);
    const auto numbers = [](const at::Tensor &t, int64_t n) {
        return t.dim() == 1 && t.size(0) == n && t.scalar_type() == at::kInt && t.is_contiguous();
    };
    if (!numbers(*lens, batch)) return refuse("lens", "a contiguous int32 number for every sequence is wanted");
    if (starts && !numbers(*starts, batch + 1)) return refuse("starts", "contiguous int32 numbers, one more than sequences, are wanted");
    if (!on(*blocks, device) || !on(*lens, device) || (starts && !on(*starts, device)))
        return refuse("blocks, lens, starts", "tensors on the cache's GPU are wanted");
    return Py_BuildValue("KLLLKK", address(*blocks), (long long)(batch > 1 ? blocks->stride(0) : width), (long long)width,
                         (long long)batch, address(*lens), starts ? address(*starts) : 0ull);
}

// (rows, heads, head_dim, name, device) -> address, token stride, head stride, tokens, type
PyObject *rows_of(PyObject *const *args, Py_ssize_t n) {
    if (!count(n, 5)) return nullptr;
    const char *name = PyUnicode_AsUTF8(args[3]);
    const at::Tensor *t = name ? tensor(args, 0, name) : nullptr;
    if (!t) return nullptr;
    const long long heads = PyLong_AsLongLong(args[1]), head_dim = PyLong_AsLongLong(args[2]), device = PyLong_AsLongLong(args[4]);
    if (PyErr_Occurred()) return nullptr;
    const auto type = t->scalar_type();
    const int dtype = type == at::kFloat ? 0 : type == at::kBFloat16 ? 1 : type == at::kHalf ? 2 : -1;
    if (dtype < 0 || t->dim() != 3 || t->size(1) != heads || t->size(2) != head_dim || (head_dim > 1 && t->stride(2) != 1))
        return PyErr_Format(PyExc_TypeError, "%s: (tokens, %lld, %lld) float32, bfloat16 or float16 with contiguous values is wanted",
                            name, heads, head_dim);
    if (!on(*t, device)) return refuse(name, "a tensor on the cache's GPU is wanted");
    return Py_BuildValue("KLLLi", address(*t), (long long)t->stride(0), (long long)t->stride(1), (long long)t->size(0), dtype);
}

// (freq or None, positions, tokens, device) -> address of freq, pairs, axes, address of positions, their stride
PyObject *turns_of(PyObject *const *args, Py_ssize_t n) {
    if (!count(n, 4)) return nullptr;
    if (args[0] == Py_None) return Py_BuildValue("KiiKL", 0ull, 0, 0, 0ull, 0ll);
    const at::Tensor *f = tensor(args, 0, "freq"), *p = f ? tensor(args, 1, "positions") : nullptr;
    if (!p) return nullptr;
    const long long tokens = PyLong_AsLongLong(args[2]), device = PyLong_AsLongLong(args[3]);
    if (PyErr_Occurred()) return nullptr;
    if (f->scalar_type() != at::kFloat || f->dim() < 1 || f->dim() > 2 || !f->is_contiguous() || !on(*f, device))
        return refuse("freq", "a contiguous float32 tensor (axes, pairs) on the rows' GPU is wanted");
    const int64_t axes = f->dim() == 1 ? 1 : f->size(0), pairs = f->size(f->dim() - 1), last = p->dim() - 1;
    if (p->scalar_type() != at::kInt || last < 0 || last > 1 || p->size(last) != tokens || (tokens > 1 && p->stride(last) != 1) ||
        axes != (last ? p->size(0) : 1) || axes > 1000 || pairs > 1000 || !on(*p, device))
        return PyErr_Format(PyExc_TypeError, "positions: int32 numbers (%lld, %lld) in contiguous rows on the rows' GPU are wanted",
                            (long long)axes, tokens);
    return Py_BuildValue("KiiKL", address(*f), (int)pairs, (int)axes, address(*p), (long long)(axes > 1 ? p->stride(0) : tokens));
}

// (tensor, rows, heads, name, device) -> address and length of the last dimension of a contiguous (rows, heads, n) tensor
PyObject *table_of(PyObject *const *args, Py_ssize_t n, at::ScalarType type, const char *what) {
    if (!count(n, 5)) return nullptr;
    const char *name = PyUnicode_AsUTF8(args[3]);
    const at::Tensor *t = name ? tensor(args, 0, name) : nullptr;
    if (!t) return nullptr;
    const long long rows = PyLong_AsLongLong(args[1]), heads = PyLong_AsLongLong(args[2]), device = PyLong_AsLongLong(args[4]);
    if (PyErr_Occurred()) return nullptr;
    if (t->dim() != 3 || t->scalar_type() != type || t->size(0) != rows || t->size(1) != heads || !t->is_contiguous())
        return PyErr_Format(PyExc_TypeError, "%s: a contiguous %s tensor (%lld, %lld, blocks) is wanted", name, what, rows, heads);
    if (!on(*t, device)) return refuse(name, "a tensor on the cache's GPU is wanted");
    return Py_BuildValue("KL", address(*t), (long long)t->size(2));
}
PyObject *ints_of(PyObject *const *args, Py_ssize_t n) { return table_of(args, n, at::kInt, "int32"); }
PyObject *floats_of(PyObject *const *args, Py_ssize_t n) { return table_of(args, n, at::kFloat, "float32"); }

// (summary, blocks, heads, row, device) -> address of a contiguous uint8 (blocks, heads, 2, row) tensor
PyObject *summary_of(PyObject *const *args, Py_ssize_t n) {
    if (!count(n, 5)) return nullptr;
    const at::Tensor *t = tensor(args, 0, "summary");
    if (!t) return nullptr;
    long long size[4] = {PyLong_AsLongLong(args[1]), PyLong_AsLongLong(args[2]), 2, PyLong_AsLongLong(args[3])};
    const long long device = PyLong_AsLongLong(args[4]);
    if (PyErr_Occurred()) return nullptr;
    bool same = t->dim() == 4 && t->scalar_type() == at::kByte && t->is_contiguous();
    for (int i = 0; i < 4 && same; ++i) same = t->size(i) == size[i];
    if (!same)
        return PyErr_Format(PyExc_TypeError, "summary: a contiguous uint8 tensor (%lld, %lld, 2, %lld) is wanted", size[0], size[1], size[3]);
    if (!on(*t, device)) return refuse("summary", "a tensor on the cache's GPU is wanted");
    return Py_BuildValue("K", address(*t));
}

PyObject *py_ints(PyObject *, PyObject *const *args, Py_ssize_t n) { return guarded(ints_of, args, n); }
PyObject *py_floats(PyObject *, PyObject *const *args, Py_ssize_t n) { return guarded(floats_of, args, n); }
PyObject *py_summary(PyObject *, PyObject *const *args, Py_ssize_t n) { return guarded(summary_of, args, n); }
PyObject *py_turns(PyObject *, PyObject *const *args, Py_ssize_t n) { return guarded(turns_of, args, n); }
PyObject *py_cache(PyObject *, PyObject *const *args, Py_ssize_t n) { return guarded(cache_of, args, n); }
PyObject *py_seqs(PyObject *, PyObject *const *args, Py_ssize_t n) { return guarded(seqs_of, args, n); }
PyObject *py_rows(PyObject *, PyObject *const *args, Py_ssize_t n) { return guarded(rows_of, args, n); }

PyMethodDef methods[] = {{"cache", (PyCFunction)(void (*)(void))py_cache, METH_FASTCALL, nullptr},
                         {"seqs", (PyCFunction)(void (*)(void))py_seqs, METH_FASTCALL, nullptr},
                         {"rows", (PyCFunction)(void (*)(void))py_rows, METH_FASTCALL, nullptr},
                         {"ints", (PyCFunction)(void (*)(void))py_ints, METH_FASTCALL, nullptr},
                         {"floats", (PyCFunction)(void (*)(void))py_floats, METH_FASTCALL, nullptr},
                         {"summary", (PyCFunction)(void (*)(void))py_summary, METH_FASTCALL, nullptr},
                         {"turns", (PyCFunction)(void (*)(void))py_turns, METH_FASTCALL, nullptr},
                         {nullptr, nullptr, 0, nullptr}};
PyModuleDef module = {PyModuleDef_HEAD_INIT, "_kv_args", "Checks and addresses of the key/value cache's tensors.", -1, methods,
                      nullptr, nullptr, nullptr, nullptr};

}  // namespace

PyMODINIT_FUNC PyInit__kv_args(void) { return PyModule_Create(&module); }
