// The tensor calls' native path: checks plain CUDA tensors, plans, takes a
// workspace from torch's caching allocator and makes the C call, in one step
// from Python. The same work in Python (attribute reads, two ctypes calls, the
// plan as a dict) took 13 to 14 us a call, more than most small and mid-size
// products take on the device.
//
// Each function returns the igemm status, or None for anything but the plain
// case (other types, layouts, devices or streams, tensor subclasses, transforms
// and modes in effect, empty products): the Python code then handles the call,
// with its own checks and messages.
#include <Python.h>

#include <ATen/ATen.h>
#include <ATen/PythonTorchFunctionTLS.h>
#include <ATen/hip/HIPContextLight.h>
#include <ATen/hip/impl/HIPStreamMasqueradingAsCUDA.h>
#include <c10/core/GradMode.h>
#include <c10/core/impl/TorchDispatchModeTLS.h>
#include <pybind11/gil.h>
#include <torch/csrc/Exceptions.h>
#include <torch/csrc/autograd/python_variable.h>

#include "igemm.h"
#include "igemm_rows.h"

namespace {

// A strided CUDA tensor of type dt with dim dimensions, not a subclass and
// under no functorch transform; nullptr otherwise.
const at::Tensor *plain(PyObject *o, at::ScalarType dt, int64_t dim) {
    if (!THPVariable_CheckExact(o)) return nullptr;
    const at::Tensor &t = THPVariable_Unpack(o);
    if (!t.defined() || !t.is_cuda() || t.layout() != at::kStrided || t.scalar_type() != dt ||
        t.dim() != dim)
        return nullptr;
    static const c10::DispatchKeySet other(
        {c10::DispatchKey::Python, c10::DispatchKey::PythonTLSSnapshot,
         c10::DispatchKey::FuncTorchBatched, c10::DispatchKey::FuncTorchGradWrapper,
         c10::DispatchKey::Batched, c10::DispatchKey::Functionalize, c10::DispatchKey::Negative,
         c10::DispatchKey::Conjugate, c10::DispatchKey::ZeroTensor});
    return t.key_set().has_any(other) ? nullptr : &t;
}

// Leading dimension of a 2-D tensor with unit stride along rows (any stride
// for a single column), as the Python checks take it; false otherwise.
bool leading(const at::Tensor &t, int64_t *ld) {
    if (t.size(1) > 1 && t.stride(1) != 1) return false;
    *ld = t.size(0) > 1 ? t.stride(0) : (t.size(1) > 1 ? t.size(1) : 1);
    return true;
}

bool modes_active() {
    return c10::impl::TorchDispatchModeTLS::any_modes_set() ||
           at::impl::PythonTorchFunctionTLS::stack_len() > 0;
}

// The stream of the current device if the tensors live there.
bool here(const at::Tensor &c, std::initializer_list<const at::Tensor *> others, void **stream) {
    const auto s = c10::hip::getCurrentHIPStreamMasqueradingAsCUDA();
    if (c.device() != s.device()) return false;
    for (const at::Tensor *t : others)
        if (t->device() != c.device()) return false;
    *stream = (void *)s.stream();
    return true;
}

int num_cu(const at::Tensor &c) {
    return at::cuda::getDeviceProperties(c.device().index())->multiProcessorCount;
}

// bytes of device memory from the caching allocator, 256-byte aligned.
at::Tensor workspace(const at::Tensor &c, int64_t bytes, void **p) {
    at::Tensor ws = at::empty({bytes + 256}, c.options().dtype(at::kByte));
    *p = (void *)(((uintptr_t)ws.data_ptr() + 255) & ~(uintptr_t)255);
    return ws;
}

bool as_i64(PyObject *o, int64_t *v) {
    if (!PyLong_Check(o)) return false;
    int overflow = 0;
    *v = PyLong_AsLongLongAndOverflow(o, &overflow);
    return overflow == 0;
}
bool as_int(PyObject *o, int *v) {
    int64_t x;
    if (!as_i64(o, &x) || x != (int)x) return false;
    *v = (int)x;
    return true;
}
bool as_pair(PyObject *o, int64_t *a, int64_t *b) {
    return PyTuple_Check(o) && PyTuple_GET_SIZE(o) == 2 && as_i64(PyTuple_GET_ITEM(o, 0), a) &&
           as_i64(PyTuple_GET_ITEM(o, 1), b);
}

struct Product {
    const at::Tensor *a, *b, *c;
    int64_t m, n, k, lda, ldb, ldc;
    void *stream;
};

// A (m x k), B (k x n) of type et, C (m x n) of type ct, nothing empty.
bool product(PyObject *A, PyObject *B, PyObject *C, at::ScalarType et, at::ScalarType ct,
             Product *p) {
    p->a = plain(A, et, 2);
    p->b = p->a ? plain(B, et, 2) : nullptr;
    p->c = p->b ? plain(C, ct, 2) : nullptr;
    if (!p->c || modes_active()) return false;
    p->m = p->a->size(0);
    p->k = p->a->size(1);
    p->n = p->b->size(1);
    return p->m > 0 && p->n > 0 && p->k > 0 && p->b->size(0) == p->k && p->c->size(0) == p->m &&
           p->c->size(1) == p->n && leading(*p->a, &p->lda) && leading(*p->b, &p->ldb) &&
           leading(*p->c, &p->ldc) && here(*p->c, {p->a, p->b}, &p->stream);
}

// gemm(elem_bytes, A, B, C, kernel, split)
PyObject *gemm(PyObject *, PyObject *const *args, Py_ssize_t nargs) {
    HANDLE_TH_ERRORS
    int es, kernel, split, st;
    Product p;
    if (nargs != 6 || !as_int(args[0], &es) || !as_int(args[4], &kernel) ||
        !as_int(args[5], &split) ||
        !product(args[1], args[2], args[3], es == 2 ? at::kShort : at::kChar, at::kInt, &p))
        Py_RETURN_NONE;
    {
        pybind11::gil_scoped_release no_gil;
        const void *A = p.a->data_ptr(), *B = p.b->data_ptr();
        int32_t *C = (int32_t *)p.c->data_ptr();
        igemm_plan plan;
        st = igemm_query_plan(es, p.m, p.n, p.k, A, p.lda, B, p.ldb, C, p.ldc, num_cu(*p.c),
                              kernel, split, &plan);
        at::Tensor ws;
        void *wp = nullptr;
        if (st == IGEMM_OK && plan.workspace_bytes > 0) ws = workspace(*p.c, plan.workspace_bytes, &wp);
        const int64_t wb = wp ? plan.workspace_bytes : 0;
        if (st == IGEMM_OK)
            st = es == 2 ? igemm_i16_ws(p.m, p.n, p.k, (const int16_t *)A, p.lda,
                                        (const int16_t *)B, p.ldb, C, p.ldc, p.stream, kernel,
                                        split, wp, wb)
                         : igemm_i8_ws(p.m, p.n, p.k, (const int8_t *)A, p.lda, (const int8_t *)B,
                                       p.ldb, C, p.ldc, p.stream, kernel, split, wp, wb);
        else
            st = INT_MIN;  // the plan's refusal: raised by the Python code
    }
    if (st == INT_MIN) Py_RETURN_NONE;
    return PyLong_FromLong(st);
    END_HANDLE_TH_ERRORS
}

// srs(A, B, C, kc, shift, round_half_up, kernel)
PyObject *srs(PyObject *, PyObject *const *args, Py_ssize_t nargs) {
    HANDLE_TH_ERRORS
    int64_t kc;
    int shift, kernel, st;
    Product p;
    if (nargs != 7 || !as_i64(args[3], &kc) || !as_int(args[4], &shift) ||
        !as_int(args[6], &kernel) || !THPVariable_CheckExact(args[0]))
        Py_RETURN_NONE;
    const int half_up = PyObject_IsTrue(args[5]);
    if (half_up < 0) return nullptr;
    const at::ScalarType et = THPVariable_Unpack(args[0]).scalar_type();
    if ((et != at::kShort && et != at::kChar) ||
        !product(args[0], args[1], args[2], et, at::kShort, &p))
        Py_RETURN_NONE;
    const int es = et == at::kShort ? 2 : 1;
    {
        pybind11::gil_scoped_release no_gil;
        const void *A = p.a->data_ptr(), *B = p.b->data_ptr();
        int16_t *C = (int16_t *)p.c->data_ptr();
        int64_t wb = 0;
        st = igemm_srs_query(es, p.m, p.n, p.k, A, p.lda, B, p.ldb, C, p.ldc, kc, num_cu(*p.c),
                             kernel, &wb);
        at::Tensor ws;
        void *wp = nullptr;
        if (st == IGEMM_OK && wb > 0) ws = workspace(*p.c, wb, &wp);
        if (st == IGEMM_OK)
            st = igemm_srs_ws(es, p.m, p.n, p.k, A, p.lda, B, p.ldb, C, p.ldc, kc, shift, half_up,
                              p.stream, kernel, wp, wb);
        else
            st = INT_MIN;
    }
    if (st == INT_MIN) Py_RETURN_NONE;
    return PyLong_FromLong(st);
    END_HANDLE_TH_ERRORS
}

// packed_b(elem_bytes, A, packed_b, packed_b_bytes, n, k, C, kernel)
PyObject *packed_b(PyObject *, PyObject *const *args, Py_ssize_t nargs) {
    HANDLE_TH_ERRORS
    int es, kernel, st;
    int64_t pb_bytes, n, k, lda, ldc;
    void *stream;
    if (nargs != 8 || !as_int(args[0], &es) || !as_i64(args[3], &pb_bytes) ||
        !as_i64(args[4], &n) || !as_i64(args[5], &k) || !as_int(args[7], &kernel))
        Py_RETURN_NONE;
    const at::Tensor *a = plain(args[1], es == 2 ? at::kShort : at::kChar, 2);
    const at::Tensor *pb = a ? plain(args[2], at::kByte, 1) : nullptr;
    const at::Tensor *c = pb ? plain(args[6], at::kInt, 2) : nullptr;
    if (!c || modes_active() || n <= 0 || k <= 0 || a->size(0) <= 0 || a->size(1) != k ||
        c->size(0) != a->size(0) || c->size(1) != n || !leading(*a, &lda) || !leading(*c, &ldc) ||
        !here(*c, {a, pb}, &stream))
        Py_RETURN_NONE;
    const int64_t m = a->size(0);
    {
        pybind11::gil_scoped_release no_gil;
        const void *A = a->data_ptr(), *PB = pb->data_ptr();
        int32_t *C = (int32_t *)c->data_ptr();
        const void *fake = (const void *)(uintptr_t)4096;  // B was consumed by the pack call
        igemm_plan plan;
        st = igemm_query_plan(es, m, n, k, A, lda, fake, n, C, ldc, num_cu(*c), kernel, -1, &plan);
        at::Tensor ws;
        void *wp = nullptr;
        if (st == IGEMM_OK && plan.packed_a_bytes > 0) ws = workspace(*c, plan.packed_a_bytes, &wp);
        const int64_t wb = wp ? plan.packed_a_bytes : 0;
        if (st == IGEMM_OK)
            st = es == 2 ? igemm_i16_packed_b(m, n, k, (const int16_t *)A, lda, PB, pb_bytes, C,
                                              ldc, kernel, wp, wb, stream)
                         : igemm_i8_packed_b(m, n, k, (const int8_t *)A, lda, PB, pb_bytes, C, ldc,
                                             kernel, wp, wb, stream);
        else
            st = INT_MIN;
    }
    if (st == INT_MIN) Py_RETURN_NONE;
    return PyLong_FromLong(st);
    END_HANDLE_TH_ERRORS
}

// conv2d(X, W, Y, stride, pad, dil, kernel, split)
PyObject *conv2d(PyObject *, PyObject *const *args, Py_ssize_t nargs) {
    HANDLE_TH_ERRORS
    igemm_conv2d_desc d;
    int kernel, split, st;
    void *stream;
    if (nargs != 8 || !as_pair(args[3], &d.stride_h, &d.stride_w) ||
        !as_pair(args[4], &d.pad_h, &d.pad_w) || !as_pair(args[5], &d.dil_h, &d.dil_w) ||
        !as_int(args[6], &kernel) || !as_int(args[7], &split) || !THPVariable_CheckExact(args[0]))
        Py_RETURN_NONE;
    const at::ScalarType et = THPVariable_Unpack(args[0]).scalar_type();
    if (et != at::kShort && et != at::kChar) Py_RETURN_NONE;
    const at::Tensor *x = plain(args[0], et, 4);
    const at::Tensor *w = x ? plain(args[1], et, 4) : nullptr;
    const at::Tensor *y = w ? plain(args[2], at::kInt, 4) : nullptr;
    if (!y || modes_active() || !x->is_contiguous() || !w->is_contiguous() ||
        !y->is_contiguous() || y->numel() == 0 || x->numel() == 0 || w->numel() == 0 ||
        !here(*y, {x, w}, &stream))
        Py_RETURN_NONE;
    d.n = x->size(0);
    d.h = x->size(1);
    d.w = x->size(2);
    d.c = x->size(3);
    d.r = w->size(0);
    d.s = w->size(1);
    d.k = w->size(3);
    if (w->size(2) != d.c || y->size(0) != d.n || y->size(3) != d.k ||
        y->size(1) != igemm_conv2d_out_dim(d.h, d.r, d.stride_h, d.pad_h, d.dil_h) ||
        y->size(2) != igemm_conv2d_out_dim(d.w, d.s, d.stride_w, d.pad_w, d.dil_w))
        Py_RETURN_NONE;
    {
        pybind11::gil_scoped_release no_gil;
        st = igemm_conv2d_ex(et == at::kShort ? 2 : 1, &d, x->data_ptr(), w->data_ptr(),
                             (int32_t *)y->data_ptr(), stream, kernel, split);
    }
    return PyLong_FromLong(st);
    END_HANDLE_TH_ERRORS
}

// ---- products whose rows choose their weights --------------------------------------

// Whether a gradient, or a derivative along a tangent, would be asked of what is made of t.
bool wants_derivative(const at::Tensor &t) {
    return (t.requires_grad() && c10::GradMode::is_enabled()) || t._fw_grad(/*level=*/0).defined();
}
// Autograd's note that t has been written.
void wrote(const at::Tensor &t) {
    if (!t.is_inference()) t.unsafeGetTensorImpl()->bump_version();
}
// None, or a plain tensor: *t stays null for None.
bool plain_or_none(PyObject *o, at::ScalarType dt, int64_t dim, const at::Tensor **t) {
    *t = nullptr;
    if (o == Py_None) return true;
    *t = plain(o, dt, dim);
    return *t != nullptr && !wants_derivative(**t);
}
// A plain float, bfloat16 or half tensor that no gradient is asked of; its igemm_type
// in *type.
const at::Tensor *plain_real(PyObject *o, int64_t dim, int *type) {
    if (!THPVariable_CheckExact(o)) return nullptr;
    const at::ScalarType dt = THPVariable_Unpack(o).scalar_type();
    if (dt == at::kFloat) *type = IGEMM_F32;
    else if (dt == at::kBFloat16) *type = IGEMM_BF16;
    else if (dt == at::kHalf) *type = IGEMM_F16;
    else return nullptr;
    const at::Tensor *t = plain(o, dt, dim);
    return t && !wants_derivative(*t) ? t : nullptr;
}
// A dense tensor of one or two dimensions of these extents (null: fine).
bool dense(const at::Tensor *t, int64_t d0, int64_t d1 = -1) {
    return t == nullptr || (t->is_contiguous() && t->size(0) == d0 &&
                            (d1 < 0 || t->size(1) == d1));
}
// The stream of the current device if all tensors (some may be null) live there.
bool all_here(std::initializer_list<const at::Tensor *> ts, void **stream) {
    const auto s = c10::hip::getCurrentHIPStreamMasqueradingAsCUDA();
    for (const at::Tensor *t : ts)
        if (t != nullptr && t->device() != s.device()) return false;
    *stream = (void *)s.stream();
    return true;
}
template <class T>
T *data(const at::Tensor *t) {
    return t != nullptr ? (T *)t->data_ptr() : nullptr;
}
// Strides of a stack of matrices with unit stride along rows.
bool stacked(const at::Tensor &t, int64_t *ld, int64_t *stride) {
    if (t.size(2) > 1 && t.stride(2) != 1) return false;
    *ld = t.size(1) > 1 ? t.stride(1) : (t.size(2) > 1 ? t.size(2) : 1);
    *stride = t.size(0) > 1 ? t.stride(0) : 0;
    return true;
}
PyObject *status(int st) { return PyLong_FromLong(st); }

// route(logits, top_k, bias, groups, top_groups, group_best, sigmoid, renormalise, scale,
//       plan) -> None, a status, or (ids, weights, offsets, order)
PyObject *route(PyObject *, PyObject *const *args, Py_ssize_t nargs) {
    HANDLE_TH_ERRORS
    igemm_route_desc d;
    int sigmoid, renormalise, plan, st;
    void *stream;
    const at::Tensor *l = nargs == 10 ? plain_real(args[0], 2, &d.type) : nullptr, *bias;
    int64_t ld;
    if (!l || modes_active() || !as_int(args[1], &d.top_k) ||
        !plain_or_none(args[2], at::kFloat, 1, &bias) || !as_int(args[3], &d.groups) ||
        !as_int(args[4], &d.top_groups) || !as_int(args[5], &d.group_best) ||
        !as_int(args[6], &sigmoid) || !as_int(args[7], &renormalise) ||
        !PyFloat_Check(args[8]) || !as_int(args[9], &plan) || l->numel() == 0 ||
        l->size(1) > INT_MAX || !leading(*l, &ld) || !dense(bias, l->size(1)) ||
        !all_here({l, bias}, &stream))
        Py_RETURN_NONE;
    d.tokens = l->size(0);
    d.experts = (int)l->size(1);
    d.score = sigmoid ? IGEMM_SIGMOID : IGEMM_SOFTMAX;
    d.renormalise = renormalise;
    d.scale = (float)PyFloat_AS_DOUBLE(args[8]);
    at::Tensor ids, weights, offsets, order;
    {
        pybind11::gil_scoped_release no_gil;
        int64_t wb = 0;
        st = igemm_route_query(&d, &wb);
        if (st == IGEMM_OK) {
            const auto ints = l->options().dtype(at::kInt);
            ids = at::empty({d.tokens, d.top_k}, ints);
            weights = at::empty({d.tokens, d.top_k}, l->options().dtype(at::kFloat));
            if (plan) {
                offsets = at::empty({d.experts + 1}, ints);
                order = at::empty({d.tokens * d.top_k}, ints);
            }
            at::Tensor ws;
            void *wp = nullptr;
            if (plan && wb > 0) ws = workspace(*l, wb, &wp);
            st = igemm_route(&d, l->data_ptr(), ld, data<float>(bias), (int32_t *)ids.data_ptr(),
                             (float *)weights.data_ptr(),
                             plan ? (int32_t *)offsets.data_ptr() : nullptr,
                             plan ? (int32_t *)order.data_ptr() : nullptr, wp, wp ? wb : 0,
                             stream);
        }
    }
    if (st != IGEMM_OK) return status(st);
    PyObject *r = PyTuple_New(4);
    if (r == nullptr) return nullptr;
    PyTuple_SET_ITEM(r, 0, THPVariable_Wrap(std::move(ids)));
    PyTuple_SET_ITEM(r, 1, THPVariable_Wrap(std::move(weights)));
    for (int i = 0; i < 2; ++i) {
        PyObject *o = Py_None;
        if (plan) o = THPVariable_Wrap(std::move(i == 0 ? offsets : order));
        else Py_INCREF(o);
        PyTuple_SET_ITEM(r, 2 + i, o);
    }
    for (int i = 0; i < 4; ++i)
        if (PyTuple_GET_ITEM(r, i) == nullptr) {
            Py_DECREF(r);
            return nullptr;
        }
    return r;
    END_HANDLE_TH_ERRORS
}

// grouped(A, B, offsets, order, scale_a, scale_b, slots, scatter, out) -> None or a status
PyObject *grouped(PyObject *, PyObject *const *args, Py_ssize_t nargs) {
    HANDLE_TH_ERRORS
    if (nargs != 9) Py_RETURN_NONE;
    igemm_grouped_desc d;
    const at::Tensor *a = plain(args[0], at::kChar, 2);
    const at::Tensor *b = a ? plain(args[1], at::kChar, 3) : nullptr;
    const at::Tensor *off = b ? plain(args[2], at::kInt, 1) : nullptr;
    const at::Tensor *out = off ? plain_real(args[8], 2, &d.type) : nullptr, *order, *sa, *sb;
    int64_t lda, ldb, ldo, stride_b;
    int st;
    void *stream;
    if (!out || modes_active() || !plain_or_none(args[3], at::kInt, 1, &order) ||
        !plain_or_none(args[4], at::kFloat, 1, &sa) ||
        !plain_or_none(args[5], at::kFloat, 2, &sb) || !as_i64(args[6], &d.slots) ||
        !as_int(args[7], &d.scatter) || a->numel() == 0 || b->numel() == 0 || out->numel() == 0)
        Py_RETURN_NONE;
    d.a_rows = a->size(0);
    d.k = a->size(1);
    d.groups = b->size(0);
    d.n = b->size(2);
    d.out_rows = out->size(0);
    d.rows = order ? order->size(0) : d.a_rows;
    if (b->size(1) != d.k || out->size(1) != d.n || !dense(off, d.groups + 1) ||
        !dense(order, d.rows) || !dense(sa, d.a_rows) || !dense(sb, d.groups, d.n) ||
        !leading(*a, &lda) || !stacked(*b, &ldb, &stride_b) || !leading(*out, &ldo) ||
        !all_here({a, b, off, order, sa, sb, out}, &stream))
        Py_RETURN_NONE;
    {
        pybind11::gil_scoped_release no_gil;
        int64_t wb = 0;
        st = igemm_i8_grouped_query(&d, num_cu(*a), &wb);
        at::Tensor ws;
        void *wp = nullptr;
        if (st == IGEMM_OK && wb > 0) ws = workspace(*a, wb, &wp);
        if (st == IGEMM_OK)
            st = igemm_i8_grouped(&d, data<int32_t>(off), data<int32_t>(order), data<int8_t>(a),
                                  lda, data<float>(sa), data<int8_t>(b), ldb, stride_b,
                                  data<float>(sb), out->data_ptr(), ldo, wp, wb, stream);
    }
    if (st == IGEMM_OK) wrote(*out);
    return status(st);
    END_HANDLE_TH_ERRORS
}

// combine(Z, weights, ids, base, out) -> None or a status
PyObject *combine(PyObject *, PyObject *const *args, Py_ssize_t nargs) {
    HANDLE_TH_ERRORS
    int type, w_type, out_type, st;
    const at::Tensor *z = nargs == 5 ? plain_real(args[0], 2, &type) : nullptr;
    const at::Tensor *w = z ? plain_real(args[1], 2, &w_type) : nullptr, *ids, *base;
    const at::Tensor *out = w ? plain_real(args[4], 2, &out_type) : nullptr;
    int64_t ldz, ld_base = 0, ldo;
    void *stream;
    if (!out || modes_active() || w_type != IGEMM_F32 || out_type != type ||
        !plain_or_none(args[2], at::kInt, 2, &ids) ||
        !plain_or_none(args[3], z->scalar_type(), 2, &base) || z->numel() == 0)
        Py_RETURN_NONE;
    const int64_t tokens = w->size(0), top_k = w->size(1), n = z->size(1);
    if (z->size(0) != tokens * top_k || !dense(w, tokens, top_k) || !dense(ids, tokens, top_k) ||
        out->size(0) != tokens || out->size(1) != n ||
        (base && (base->size(0) != tokens || base->size(1) != n || !leading(*base, &ld_base))) ||
        !leading(*z, &ldz) || !leading(*out, &ldo) || !all_here({z, w, ids, base, out}, &stream))
        Py_RETURN_NONE;
    {
        pybind11::gil_scoped_release no_gil;
        st = igemm_combine(tokens, top_k, n, type, z->data_ptr(), ldz, data<float>(w),
                           data<int32_t>(ids), data<void>(base), ld_base, out->data_ptr(), ldo,
                           stream);
    }
    if (st == IGEMM_OK) wrote(*out);
    return status(st);
    END_HANDLE_TH_ERRORS
}

// adapters(A, B, ids, down, up, scale_a, scale_b, ranks, scaling, out) -> None or a status
PyObject *adapters(PyObject *, PyObject *const *args, Py_ssize_t nargs) {
    HANDLE_TH_ERRORS
    if (nargs != 10) Py_RETURN_NONE;
    igemm_adapters_desc d;
    const at::Tensor *a = plain(args[0], at::kChar, 2);
    const at::Tensor *b = a ? plain(args[1], at::kChar, 2) : nullptr;
    const at::Tensor *ids = b ? plain(args[2], at::kInt, 1) : nullptr;
    const at::Tensor *down = ids ? plain_real(args[3], 3, &d.weight_type) : nullptr;
    int up_type;
    const at::Tensor *up = down ? plain_real(args[4], 3, &up_type) : nullptr;
    const at::Tensor *out = up ? plain_real(args[9], 2, &d.type) : nullptr;
    const at::Tensor *sa, *sb, *ranks, *scaling;
    int64_t lda, ldb, ldo, ldd, ldu, stride_d, stride_u;
    int st;
    void *stream;
    if (!out || modes_active() || d.weight_type == IGEMM_F32 || up_type != d.weight_type ||
        !plain_or_none(args[5], at::kFloat, 1, &sa) ||
        !plain_or_none(args[6], at::kFloat, 1, &sb) ||
        !plain_or_none(args[7], at::kInt, 1, &ranks) ||
        !plain_or_none(args[8], at::kFloat, 1, &scaling) || a->numel() == 0 || b->numel() == 0 ||
        down->numel() == 0 || up->numel() == 0)
        Py_RETURN_NONE;
    d.m = a->size(0);
    d.k = a->size(1);
    d.n = b->size(1);
    d.adapters = down->size(0);
    d.rank = down->size(1);
    if (b->size(0) != d.k || down->size(2) != d.k || up->size(0) != d.adapters ||
        up->size(1) != d.n || up->size(2) != d.rank || out->size(0) != d.m ||
        out->size(1) != d.n || !dense(ids, d.m) || !dense(sa, d.m) || !dense(sb, d.n) ||
        !dense(ranks, d.adapters) || !dense(scaling, d.adapters) || !leading(*a, &lda) ||
        !leading(*b, &ldb) || !stacked(*down, &ldd, &stride_d) ||
        !stacked(*up, &ldu, &stride_u) || !leading(*out, &ldo) ||
        !all_here({a, b, ids, down, up, sa, sb, ranks, scaling, out}, &stream))
        Py_RETURN_NONE;
    {
        pybind11::gil_scoped_release no_gil;
        int64_t wb = 0;
        st = igemm_i8_adapters_query(&d, num_cu(*a), &wb);
        at::Tensor ws;
        void *wp = nullptr;
        if (st == IGEMM_OK && wb > 0) ws = workspace(*a, wb, &wp);
        if (st == IGEMM_OK)
            st = igemm_i8_adapters(&d, data<int8_t>(a), lda, data<float>(sa), data<int8_t>(b), ldb,
                                   data<float>(sb), data<int32_t>(ids), down->data_ptr(), ldd,
                                   stride_d, up->data_ptr(), ldu, stride_u, data<int32_t>(ranks),
                                   data<float>(scaling), out->data_ptr(), ldo, wp, wb, stream);
    }
    if (st == IGEMM_OK) wrote(*out);
    return status(st);
    END_HANDLE_TH_ERRORS
}

#define IGEMM_FAST(f) (PyCFunction)(void (*)(void))f, METH_FASTCALL, nullptr
PyMethodDef methods[] = {{"gemm", IGEMM_FAST(gemm)},
                         {"srs", IGEMM_FAST(srs)},
                         {"packed_b", IGEMM_FAST(packed_b)},
                         {"conv2d", IGEMM_FAST(conv2d)},
                         {"route", IGEMM_FAST(route)},
                         {"grouped", IGEMM_FAST(grouped)},
                         {"combine", IGEMM_FAST(combine)},
                         {"adapters", IGEMM_FAST(adapters)},
                         {nullptr, nullptr, 0, nullptr}};
PyModuleDef module = {PyModuleDef_HEAD_INIT, "_igemm_torch", nullptr, -1, methods,
                      nullptr, nullptr, nullptr, nullptr};

}  // namespace

PyMODINIT_FUNC PyInit__igemm_torch(void) { return PyModule_Create(&module); }
