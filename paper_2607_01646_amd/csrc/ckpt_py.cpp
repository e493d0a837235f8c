// ckpt_py.cpp -- CPython module _ckpt_py: the argument marshalling of
// ckpt_pack_noalloc for lists of torch tensors, and of the training-step
// operators.  A pack of 64 fragments spent 25 us of its 41 reading the
// tensors' attributes one Python call at a time; a loss 22 us of its 40.
// Whatever is not plain (other types, subclasses, arguments to refuse) is
// answered None: the Python code beside it takes the call, or raises.
#include <Python.h>

#include <ATen/ops/empty.h>
#include <torch/csrc/autograd/python_variable.h>
#include <torch/version.h>

#include <vector>

#include "../../include/ckpt.h"
#include "../../include/ckpt_ops.h"

namespace {

using PackFn = ckpt_status (*)(const ckpt_tensor*, uint32_t, uint64_t, uint32_t, int32_t, void*, uint64_t, uint64_t*,
                               uint64_t, void*, uint64_t*, uint64_t*);

// Read one tensor's address and bytes.  False for whatever the Python path
// answers better: other types and subclasses (their attributes may be
// overridden), tensors without plain storage, and those it refuses.
bool read(PyObject* o, bool contiguous, void** ptr, uint64_t* nbytes)
{
    if (!THPVariable_CheckExact(o)) return false;
    const at::Tensor& t = THPVariable_Unpack(o);
    if (!t.is_cuda() || (contiguous && !t.is_contiguous())) return false;
    *nbytes = (uint64_t)t.numel() * t.element_size();
    *ptr = t.data_ptr();
    return true;
}

// pack_noalloc(function address, tensors, image, sums, chunk_bytes,
// align_bytes, device, stream handle) -> (status, image bytes, chunks), or
// None when an argument needs the Python path.
PyObject* pack_noalloc(PyObject*, PyObject* const* args, Py_ssize_t n_args)
{
    if (n_args != 8) {
        PyErr_SetString(PyExc_TypeError, "pack_noalloc takes 8 arguments");
        return nullptr;
    }
    if (!PyList_CheckExact(args[1]) && !PyTuple_CheckExact(args[1])) Py_RETURN_NONE;
    const unsigned long long fn = PyLong_AsUnsignedLongLong(args[0]), chunk = PyLong_AsUnsignedLongLong(args[4]);
    const unsigned long long align = PyLong_AsUnsignedLongLong(args[5]), stream = PyLong_AsUnsignedLongLong(args[7]);
    const long device = PyLong_AsLong(args[6]);
    if (PyErr_Occurred() || align > UINT32_MAX || device < INT32_MIN || device > INT32_MAX) {
        PyErr_Clear();
        Py_RETURN_NONE;
    }
    const Py_ssize_t n = PySequence_Fast_GET_SIZE(args[1]);
    PyObject* const* items = PySequence_Fast_ITEMS(args[1]);
    uint64_t image_cap = 0, sums_cap = 0, image_bytes = 0, n_chunks = 0;
    void *image = nullptr, *sums = nullptr;
    std::vector<ckpt_tensor> t;
    if (n == 0 || (uint64_t)n > UINT32_MAX) Py_RETURN_NONE;
    try {
        t.resize((size_t)n);
        for (Py_ssize_t k = 0; k < n; ++k) {
            void* p = nullptr;
            if (!read(items[k], true, &p, &t[k].nbytes)) Py_RETURN_NONE;
            t[k].dev_ptr = t[k].nbytes ? p : nullptr;
            t[k].dtype = t[k].cls = 0;
        }
        if (!read(args[2], false, &image, &image_cap) || !read(args[3], false, &sums, &sums_cap)) Py_RETURN_NONE;
    } catch (...) { // no storage behind the tensor, out of memory: the Python path raises its own error
        Py_RETURN_NONE;
    }
    ckpt_status rc;
    Py_BEGIN_ALLOW_THREADS;
    rc = ((PackFn)(uintptr_t)fn)(t.data(), (uint32_t)n, chunk, (uint32_t)align, (int32_t)device, image, image_cap,
                                 (uint64_t*)sums, sums_cap / 8, (void*)(uintptr_t)stream, &image_bytes, &n_chunks);
    Py_END_ALLOW_THREADS;
    return Py_BuildValue("iKK", (int)rc, (unsigned long long)image_bytes, (unsigned long long)n_chunks);
}

// CKPT_TYPE_* of a tensor, 0 for others.
uint32_t type_of(const at::Tensor& t)
{
    return t.scalar_type() == at::kBFloat16 ? CKPT_TYPE_BF16 : t.scalar_type() == at::kFloat ? CKPT_TYPE_F32 : 0;
}

const at::Tensor* plain(PyObject* o)
{
    if (!THPVariable_CheckExact(o)) return nullptr;
    const at::Tensor& t = THPVariable_Unpack(o);
    return t.is_cuda() && t.layout() == at::kStrided ? &t : nullptr;
}

// A device scalar, or None.
bool read_scalar(PyObject* o, const float** p)
{
    *p = nullptr;
    if (o == Py_None) return true;
    const at::Tensor* t = plain(o);
    if (!t || t->scalar_type() != at::kFloat || t->numel() != 1) return false;
    *p = (const float*)t->data_ptr();
    return true;
}

using AdamFn = ckpt_status (*)(const ckpt_adamw_fragment*, uint32_t, uint32_t, uint32_t, uint64_t, double, double, double,
                               double, double, const float*, int32_t, void*);

// adamw(function address, params, masters, exp_avgs, exp_avg_sqs, grads, step,
// lr, beta1, beta2, eps, weight_decay, grad_scale, stream handle) -> status.
PyObject* adamw(PyObject*, PyObject* const* args, Py_ssize_t n_args)
{
    if (n_args != 14) {
        PyErr_SetString(PyExc_TypeError, "adamw takes 14 arguments");
        return nullptr;
    }
    for (int k = 1; k < 6; ++k)
        if (!PyList_CheckExact(args[k]) && !PyTuple_CheckExact(args[k])) Py_RETURN_NONE;
    const unsigned long long fn = PyLong_AsUnsignedLongLong(args[0]), step = PyLong_AsUnsignedLongLong(args[6]);
    double x[5];
    for (int k = 0; k < 5; ++k) x[k] = PyFloat_AsDouble(args[7 + k]);
    const unsigned long long stream = PyLong_AsUnsignedLongLong(args[13]);
    if (PyErr_Occurred()) {
        PyErr_Clear();
        Py_RETURN_NONE;
    }
    const Py_ssize_t n = PySequence_Fast_GET_SIZE(args[1]);
    if (n == 0 || (uint64_t)n > UINT32_MAX) Py_RETURN_NONE;
    uint32_t types[2] = {0, 0};
    int32_t device = 0;
    const float* scale = nullptr;
    std::vector<ckpt_adamw_fragment> f;
    try {
        f.resize((size_t)n);
        if (!read_scalar(args[12], &scale)) Py_RETURN_NONE;
        for (int k = 0; k < 5; ++k) {
            if (PySequence_Fast_GET_SIZE(args[1 + k]) != n) Py_RETURN_NONE;
            PyObject* const* items = PySequence_Fast_ITEMS(args[1 + k]);
            for (Py_ssize_t i = 0; i < n; ++i) {
                const at::Tensor* t = plain(items[i]);
                if (!t || !t->is_contiguous()) Py_RETURN_NONE;
                const uint32_t type = type_of(*t);
                if (k == 0 || k == 4) {
                    uint32_t& want = types[k == 4];
                    if (i == 0) want = type;
                    if (type == 0 || type != want) Py_RETURN_NONE;
                } else if (type != CKPT_TYPE_F32) {
                    Py_RETURN_NONE;
                }
                if (k == 0) {
                    if (i == 0) device = t->get_device();
                    f[i].numel = (uint64_t)t->numel();
                }
                if ((uint64_t)t->numel() != f[i].numel) Py_RETURN_NONE;
                void* p = f[i].numel ? t->data_ptr() : nullptr;
                if (k == 0) f[i].param = p;
                if (k == 1) f[i].master = (float*)p;
                if (k == 2) f[i].exp_avg = (float*)p;
                if (k == 3) f[i].exp_avg_sq = (float*)p;
                if (k == 4) f[i].grad = p;
            }
        }
    } catch (...) {
        Py_RETURN_NONE;
    }
    ckpt_status rc;
    Py_BEGIN_ALLOW_THREADS;
    rc = ((AdamFn)(uintptr_t)fn)(f.data(), (uint32_t)n, types[0], types[1], step, x[0], x[1], x[2], x[3], x[4], scale,
                                 device, (void*)(uintptr_t)stream);
    Py_END_ALLOW_THREADS;
    return PyLong_FromLong(rc);
}

using NormFn = ckpt_status (*)(const ckpt_tensor*, uint32_t, uint32_t, float, float*, void*, int32_t, void*);

// grad_norm(function address, grads, max_norm, stream handle) -> (status, the
// two values).  Allocates on torch's current stream.
PyObject* grad_norm(PyObject*, PyObject* const* args, Py_ssize_t n_args)
{
    if (n_args != 4) {
        PyErr_SetString(PyExc_TypeError, "grad_norm takes 4 arguments");
        return nullptr;
    }
    if (!PyList_CheckExact(args[1]) && !PyTuple_CheckExact(args[1])) Py_RETURN_NONE;
    const unsigned long long fn = PyLong_AsUnsignedLongLong(args[0]), stream = PyLong_AsUnsignedLongLong(args[3]);
    const double max_norm = PyFloat_AsDouble(args[2]);
    if (PyErr_Occurred()) {
        PyErr_Clear();
        Py_RETURN_NONE;
    }
    const Py_ssize_t n = PySequence_Fast_GET_SIZE(args[1]);
    PyObject* const* items = PySequence_Fast_ITEMS(args[1]);
    if (n == 0 || (uint64_t)n > UINT32_MAX) Py_RETURN_NONE;
    std::vector<ckpt_tensor> t;
    uint32_t type = 0;
    int32_t device = 0;
    at::Tensor out, scratch;
    try {
        t.resize((size_t)n);
        for (Py_ssize_t i = 0; i < n; ++i) {
            const at::Tensor* x = plain(items[i]);
            if (!x || !x->is_contiguous()) Py_RETURN_NONE;
            if (i == 0) {
                type = type_of(*x);
                device = x->get_device();
                out = at::empty({2}, x->options().dtype(at::kFloat));
                scratch = at::empty({CKPT_GRAD_NORM_SCRATCH / 8}, x->options().dtype(at::kDouble));
            }
            if (type == 0 || type_of(*x) != type) Py_RETURN_NONE;
            t[i].nbytes = (uint64_t)x->numel() * x->element_size();
            t[i].dev_ptr = t[i].nbytes ? x->data_ptr() : nullptr;
            t[i].dtype = t[i].cls = 0;
        }
    } catch (...) {
        Py_RETURN_NONE;
    }
    ckpt_status rc;
    Py_BEGIN_ALLOW_THREADS;
    rc = ((NormFn)(uintptr_t)fn)(t.data(), (uint32_t)n, type, (float)max_norm, (float*)out.data_ptr(), scratch.data_ptr(),
                                 device, (void*)(uintptr_t)stream);
    Py_END_ALLOW_THREADS;
    return Py_BuildValue("iN", (int)rc, THPVariable_Wrap(out));
}

// Rows of the last dimension: false unless it is contiguous and the rows are
// one run (contiguous tensors and plain matrices).
bool read_rows(const at::Tensor& t, uint64_t* rows, uint64_t* cols, uint64_t* stride)
{
    const int64_t d = t.dim();
    if (d < 1 || t.size(d - 1) < 1) return false;
    *cols = (uint64_t)t.size(d - 1);
    *rows = (uint64_t)t.numel() / *cols;
    *stride = *cols;
    if (t.is_contiguous()) return true;
    if (d != 2 || t.stride(1) != 1 || t.size(0) < 2) return false;
    *stride = (uint64_t)t.stride(0);
    return true;
}

using WorkFn = ckpt_status (*)(const ckpt_linear_loss_args*, uint64_t*);
using LossFn = ckpt_status (*)(const ckpt_linear_loss_args*, int32_t, void*, uint64_t, void*);

// linear_loss(workspace function's address, loss function's address, hidden,
// weight, target, teacher_index, teacher_logits, temperature, alpha,
// token_weight, ignore_index, reduction, grad, grad_scale, piece_bytes, stream
// handle) -> (status, loss, token_loss, lse, d_hidden, d_weight).  Allocates on
// torch's current stream.
PyObject* linear_loss(PyObject*, PyObject* const* args, Py_ssize_t n_args)
{
    if (n_args != 16) {
        PyErr_SetString(PyExc_TypeError, "linear_loss takes 16 arguments");
        return nullptr;
    }
    const unsigned long long work_fn = PyLong_AsUnsignedLongLong(args[0]), fn = PyLong_AsUnsignedLongLong(args[1]);
    ckpt_linear_loss_args a = {};
    a.temperature = (float)PyFloat_AsDouble(args[7]);
    a.alpha = (float)PyFloat_AsDouble(args[8]);
    a.ignore_index = PyLong_AsLongLong(args[10]);
    a.reduction = (uint32_t)PyLong_AsUnsignedLong(args[11]);
    const int grad = PyObject_IsTrue(args[12]);
    a.piece_bytes = PyLong_AsUnsignedLongLong(args[14]);
    const unsigned long long stream = PyLong_AsUnsignedLongLong(args[15]);
    if (PyErr_Occurred()) {
        PyErr_Clear();
        Py_RETURN_NONE;
    }
    const at::Tensor *h = plain(args[2]), *w = plain(args[3]);
    if (!h || !w) Py_RETURN_NONE;
    at::Tensor loss, token_loss, lse, d_hidden, d_weight, work;
    uint64_t bytes = 0;
    ckpt_status rc;
    int32_t device = 0;
    try {
        uint64_t dim = 0;
        a.dtype = type_of(*h);
        if (a.dtype == 0 || type_of(*w) != a.dtype || w->dim() != 2 || h->device() != w->device()) Py_RETURN_NONE;
        if (!read_rows(*h, &a.tokens, &a.dim, &a.hidden_stride) || !read_rows(*w, &a.vocab, &dim, &a.weight_stride) ||
            dim != a.dim)
            Py_RETURN_NONE;
        device = h->get_device();
        a.hidden = h->data_ptr();
        a.weight = w->data_ptr();
        const auto shape = h->sizes().slice(0, h->dim() - 1);
        const struct {
            PyObject* o;
            at::ScalarType type;
            const void** to;
        } each[] = {{args[4], at::kLong, (const void**)&a.target}, {args[9], at::kFloat, (const void**)&a.token_weight}};
        for (const auto& x : each) {
            if (x.o == Py_None) continue;
            const at::Tensor* t = plain(x.o);
            if (!t || t->scalar_type() != x.type || (uint64_t)t->numel() != a.tokens || !t->is_contiguous() ||
                (t->dim() != 1 && t->sizes() != shape))
                Py_RETURN_NONE;
            *x.to = a.tokens ? t->data_ptr() : nullptr;
        }
        if (args[5] != Py_None) {
            const at::Tensor *i = plain(args[5]), *t = plain(args[6]);
            uint64_t rows = 0, k = 0;
            if (!i || !t || i->scalar_type() != at::kLong || !(a.teacher_dtype = type_of(*t)) || i->sizes() != t->sizes() ||
                i->dim() != h->dim() || i->sizes().slice(0, i->dim() - 1) != shape)
                Py_RETURN_NONE;
            if (!read_rows(*i, &rows, &k, &a.teacher_index_stride) || !read_rows(*t, &rows, &k, &a.teacher_logits_stride) ||
                k > UINT32_MAX)
                Py_RETURN_NONE;
            a.topk = (uint32_t)k;
            a.teacher_index = (const int64_t*)i->data_ptr();
            a.teacher_logits = t->data_ptr();
        }
        if (!read_scalar(args[13], &a.grad_scale)) Py_RETURN_NONE;
        const auto fp32 = h->options().dtype(at::kFloat);
        loss = at::empty({}, fp32);
        token_loss = at::empty(shape, fp32);
        lse = at::empty(shape, fp32);
        a.loss = (float*)loss.data_ptr();
        a.token_loss = (float*)token_loss.data_ptr();
        a.lse = (float*)lse.data_ptr();
        if (grad) {
            d_hidden = at::empty(h->sizes(), h->options());
            d_weight = at::empty(w->sizes(), w->options());
            a.d_hidden = d_hidden.data_ptr();
            a.d_weight = d_weight.data_ptr();
            a.d_hidden_stride = a.d_weight_stride = a.dim;
        }
        rc = ((WorkFn)(uintptr_t)work_fn)(&a, &bytes);
        if (rc == CKPT_OK) work = at::empty({(int64_t)bytes}, h->options().dtype(at::kByte));
    } catch (...) {
        Py_RETURN_NONE;
    }
    if (rc == CKPT_OK) {
        Py_BEGIN_ALLOW_THREADS;
        rc = ((LossFn)(uintptr_t)fn)(&a, device, work.data_ptr(), bytes, (void*)(uintptr_t)stream);
        Py_END_ALLOW_THREADS;
    }
    const auto wrap = [](const at::Tensor& t) {
        if (t.defined()) return THPVariable_Wrap(t);
        Py_INCREF(Py_None);
        return Py_None;
    };
    return Py_BuildValue("iNNNNN", (int)rc, wrap(loss), wrap(token_loss), wrap(lse), wrap(d_hidden), wrap(d_weight));
}

PyMethodDef methods[] = {{"adamw", (PyCFunction)(void (*)(void))adamw, METH_FASTCALL, nullptr},
                         {"grad_norm", (PyCFunction)(void (*)(void))grad_norm, METH_FASTCALL, nullptr},
                         {"linear_loss", (PyCFunction)(void (*)(void))linear_loss, METH_FASTCALL, nullptr},
                         {"pack_noalloc", (PyCFunction)(void (*)(void))pack_noalloc, METH_FASTCALL, nullptr},
                         {nullptr, nullptr, 0, nullptr}};
PyModuleDef module = {PyModuleDef_HEAD_INIT, "_ckpt_py", nullptr, -1, methods, nullptr, nullptr, nullptr, nullptr};

} // namespace

// torch_version: what it was compiled against; another torch lays tensors out
// differently.
PyMODINIT_FUNC PyInit__ckpt_py()
{
    PyObject* m = PyModule_Create(&module);
    if (m && PyModule_AddStringConstant(m, "torch_version", TORCH_VERSION) != 0) Py_CLEAR(m);
    return m;
}
