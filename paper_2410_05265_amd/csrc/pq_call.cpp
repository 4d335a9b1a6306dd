// The call path of the smallest calls, pq_linear and pq_linear2 with the caller's own output and workspace and the three calls of a step on
// the paged 4-bit cache with the caller's own outputs, in native code: argument checks, pointers and the current stream.  A decoded token's kernel takes 4.0 us (1 x 4096 -> 4096), the call through
// Python attributes and ctypes 5.5 us of host time, of which 3.5 are ctypes and the launch; here the whole call takes 3.4 us
// (1 x 4096 -> 4096, eager, weights in turn: 5.95 -> 4.33 us a call).
//
// Only the plain case is taken: exact Tensor objects, contiguous, of the types and shapes that the binding asks for.  For anything else
// the functions return -1 and have done nothing, and the Python path decides (and words the error).
#include <Python.h>

#include <c10/hip/HIPStream.h>
#include <torch/csrc/autograd/python_variable.h>

#include <cstdint>

#include "../../include/pq.h"

namespace {

using Linear = int (*)(const void*, const void*, const float*, float, int32_t, int64_t, int64_t, int64_t, void*, void*, size_t, void*);
using Linear2 = int (*)(const void*, const void*, const float*, int64_t, void*, const void*, const float*, int64_t, void*, float, int32_t,
                        int64_t, int64_t, void*, size_t, void*);
Linear g_linear = nullptr;
Linear2 g_linear2 = nullptr;

// a tensor that the library reads: on the GPU, contiguous, of this type
bool operand(PyObject* o, at::ScalarType type, const at::Tensor** t)
{
    if (!THPVariable_CheckExact(o)) return false;
    *t = &THPVariable_Unpack(o);
    return (*t)->is_cuda() && (*t)->scalar_type() == type && (*t)->is_contiguous();
}

// the caller's fp16 output, with room for M x N values
bool result(PyObject* o, int64_t M, int64_t N, const at::Tensor** t) { return operand(o, at::kHalf, t) && (*t)->numel() >= M * N; }

// the caller's workspace, of any type (the library compares its elements, taken as bytes, with what it needs)
bool workspace(PyObject* o, const at::Tensor** t)
{
    if (!THPVariable_CheckExact(o)) return false;
    *t = &THPVariable_Unpack(o);
    return (*t)->is_cuda() && (*t)->is_contiguous();
}

bool number(PyObject* step, PyObject* block, double* s, long* h)
{
    if (!PyFloat_Check(step) || !PyLong_Check(block)) return false;
    *s = PyFloat_AS_DOUBLE(step);
    *h = PyLong_AsLong(block);
    if (*h == -1 && PyErr_Occurred()) {
        PyErr_Clear();
        return false;
    }
    return *h >= INT32_MIN && *h <= INT32_MAX;
}

// weights of K input channels and their steps
bool matrix(PyObject* w, PyObject* sw, int64_t K, const at::Tensor** wt, const at::Tensor** st)
{
    return operand(w, at::kByte, wt) && operand(sw, at::kFloat, st) && (*wt)->dim() == 2 && (*wt)->size(1) * 2 == K &&
           (*st)->numel() == (*wt)->size(0);
}

void* stream() { return c10::hip::getCurrentHIPStream().stream(); }

// (x, wq, w_scale, act_scale, had_block, out, workspace) -> status, or -1
PyObject* linear(PyObject*, PyObject* const* a, Py_ssize_t n)
{
    try {
        const at::Tensor *x, *w, *s, *out, *ws;
        double step;
        long h;
        if (n == 7 && g_linear && operand(a[0], at::kHalf, &x) && x->dim() == 2 && matrix(a[1], a[2], x->size(1), &w, &s) &&
            number(a[3], a[4], &step, &h) && result(a[5], x->size(0), w->size(0), &out) && workspace(a[6], &ws)) {
            const void *xp = x->data_ptr(), *wp = w->data_ptr();
            const float* sp = static_cast<const float*>(s->data_ptr());
            void *op = out->data_ptr(), *wsp = ws->data_ptr(), *st = stream();
            const int64_t M = x->size(0), K = x->size(1), N = w->size(0);
            const size_t bytes = (size_t)ws->numel();
            int rc;
            Py_BEGIN_ALLOW_THREADS
            rc = g_linear(xp, wp, sp, (float)step, (int32_t)h, M, N, K, op, wsp, bytes, st);
            Py_END_ALLOW_THREADS
            return PyLong_FromLong(rc);
        }
    } catch (...) {        // (a tensor without memory of its own: the Python path reports it)
    }
    return PyLong_FromLong(-1);
}

// (x, wq_a, w_scale_a, wq_b, w_scale_b, act_scale, had_block, out_a, out_b, workspace) -> status, or -1
PyObject* linear2(PyObject*, PyObject* const* a, Py_ssize_t n)
{
    try {
        const at::Tensor *x, *wa, *sa, *wb, *sb, *oa, *ob, *ws;
        double step;
        long h;
        if (n == 10 && g_linear2 && operand(a[0], at::kHalf, &x) && x->dim() == 2 && matrix(a[1], a[2], x->size(1), &wa, &sa) &&
            matrix(a[3], a[4], x->size(1), &wb, &sb) && number(a[5], a[6], &step, &h) &&
            result(a[7], x->size(0), wa->size(0), &oa) && result(a[8], x->size(0), wb->size(0), &ob) && workspace(a[9], &ws)) {
            const void *xp = x->data_ptr(), *wap = wa->data_ptr(), *wbp = wb->data_ptr();
            const float *sap = static_cast<const float*>(sa->data_ptr()), *sbp = static_cast<const float*>(sb->data_ptr());
            void *oap = oa->data_ptr(), *obp = ob->data_ptr(), *wsp = ws->data_ptr(), *st = stream();
            const int64_t M = x->size(0), K = x->size(1), Na = wa->size(0), Nb = wb->size(0);
            const size_t bytes = (size_t)ws->numel();
            int rc;
            Py_BEGIN_ALLOW_THREADS
            rc = g_linear2(xp, wap, sap, Na, oap, wbp, sbp, Nb, obp, (float)step, (int32_t)h, M, K, wsp, bytes, st);
            Py_END_ALLOW_THREADS
            return PyLong_FromLong(rc);
        }
    } catch (...) {
    }
    return PyLong_FromLong(-1);
}

// ---- the paged 4-bit cache.  Here every tensor has to lie on the current device, whose stream the kernels go to.
using Slots = decltype(&pq_kv4_slots);
using Append = decltype(&pq_kv4_append);
using Attention = decltype(&pq_kv4_attention);
Slots g_slots = nullptr;
Append g_append = nullptr;
Attention g_attention = nullptr;

bool here(const at::Tensor& t) { return t.get_device() == c10::hip::current_device(); }
bool operand_here(PyObject* o, at::ScalarType type, const at::Tensor** t) { return operand(o, type, t) && here(**t); }
// None gives a null pointer
bool optional_here(PyObject* o, at::ScalarType type, const at::Tensor** t)
{
    *t = nullptr;
    return o == Py_None || operand_here(o, type, t);
}
void* pointer(const at::Tensor* t) { return t ? t->data_ptr() : nullptr; }
// fp16 rows that may lie apart
bool rows_here(PyObject* o, const at::Tensor** t)
{
    if (!THPVariable_CheckExact(o)) return false;
    *t = &THPVariable_Unpack(o);
    return (*t)->is_cuda() && (*t)->scalar_type() == at::kHalf && (*t)->dim() == 2 && (*t)->stride(1) == 1 && here(**t);
}
int64_t row_stride(const at::Tensor& t) { return t.size(0) > 1 ? t.stride(0) : t.size(1); }

bool whole(PyObject* o, int64_t lo, int64_t hi, int64_t* v)
{
    if (!PyLong_CheckExact(o)) return false;
    *v = PyLong_AsLongLong(o);
    if (*v == -1 && PyErr_Occurred()) {
        PyErr_Clear();
        return false;
    }
    return *v >= lo && *v <= hi;
}

bool cache_here(PyObject* const* a, int64_t group, pq_kv4_cache* c)
{
    const at::Tensor *kc, *vc, *ks, *vs;
    if (!operand_here(a[0], at::kByte, &kc) || !operand_here(a[1], at::kByte, &vc) || !operand_here(a[2], at::kFloat, &ks) ||
        !operand_here(a[3], at::kFloat, &vs) || kc->dim() != 4 || vc->sizes() != kc->sizes() || group < 0)
        return false;
    const int64_t pages = kc->size(0), heads = kc->size(1), ps = kc->size(2), D = 2 * kc->size(3);
    const int64_t steps = group == 0 ? heads : pages * heads * ps * (D / group);
    if (ks->numel() != steps || vs->numel() != steps || heads > INT32_MAX || ps > INT32_MAX || D > INT32_MAX) return false;
    *c = {kc->data_ptr(), vc->data_ptr(), static_cast<float*>(ks->data_ptr()), static_cast<float*>(vs->data_ptr()), pages, (int32_t)heads,
          (int32_t)D, (int32_t)ps, (int32_t)group};
    return true;
}

template <typename T> T* as(const at::Tensor* t) { return static_cast<T*>(pointer(t)); }

// (kv_len, q_len, block_table, free_pages, page_size, T, taken or None, position_offset, cu_q, kv_len_out, positions, slots, taken_out)
PyObject* kv4_slots(PyObject*, PyObject* const* a, Py_ssize_t n)
{
    try {
        const at::Tensor *kv, *q, *table, *free_pages, *taken, *cu, *kv_out, *pos, *slots, *taken_out;
        int64_t ps, T, offset;
        if (n == 13 && g_slots && operand_here(a[0], at::kInt, &kv) && operand_here(a[1], at::kInt, &q) && operand_here(a[2], at::kInt, &table) &&
            operand_here(a[3], at::kInt, &free_pages) && whole(a[4], 0, INT32_MAX, &ps) && whole(a[5], 0, INT32_MAX, &T) &&
            optional_here(a[6], at::kInt, &taken) && whole(a[7], 0, INT32_MAX, &offset) && operand_here(a[8], at::kInt, &cu) &&
            operand_here(a[9], at::kInt, &kv_out) && operand_here(a[10], at::kInt, &pos) && operand_here(a[11], at::kLong, &slots) &&
            operand_here(a[12], at::kInt, &taken_out)) {
            const int64_t B = kv->numel();
            if (q->numel() == B && table->dim() == 2 && table->size(0) == B && cu->numel() > B && kv_out->numel() >= B && pos->numel() >= T &&
                slots->numel() >= T && taken_out->numel() >= 1 && (!taken || taken->numel() >= 1) && B <= INT32_MAX &&
                table->size(1) <= INT32_MAX && free_pages->numel() <= INT32_MAX) {
                void* const st = stream();
                int rc;
                Py_BEGIN_ALLOW_THREADS
                rc = g_slots(as<int32_t>(kv), as<int32_t>(q), (int32_t)B, as<int32_t>(table), (int32_t)table->size(1), as<int32_t>(free_pages),
                             (int32_t)free_pages->numel(), as<int32_t>(taken), (int32_t)ps, T, (int32_t)offset, as<int32_t>(cu), as<int32_t>(kv_out),
                             as<int32_t>(pos), as<int64_t>(slots), as<int32_t>(taken_out), st);
                Py_END_ALLOW_THREADS
                return PyLong_FromLong(rc);
            }
        }
    } catch (...) {
    }
    return PyLong_FromLong(-1);
}

// (qkv, n_heads, positions or None, slots, k_codes, v_codes, k_scale, v_scale, q_weight or None, k_weight or None, eps, cos_sin or None,
//  interleaved, rotate, group, clip, out)
PyObject* kv4_append(PyObject*, PyObject* const* a, Py_ssize_t n)
{
    try {
        const at::Tensor *x, *pos, *slots, *qw, *kw, *cs, *out;
        int64_t heads, group;
        pq_kv4_cache c;
        if (n == 17 && g_append && rows_here(a[0], &x) && whole(a[1], 1, INT32_MAX, &heads) && optional_here(a[2], at::kInt, &pos) &&
            operand_here(a[3], at::kLong, &slots) && whole(a[14], 0, INT32_MAX, &group) && cache_here(a + 4, group, &c) &&
            optional_here(a[8], at::kHalf, &qw) && optional_here(a[9], at::kHalf, &kw) && PyFloat_CheckExact(a[10]) &&
            optional_here(a[11], at::kFloat, &cs) && PyBool_Check(a[12]) && PyBool_Check(a[13]) && PyFloat_CheckExact(a[15]) &&
            operand_here(a[16], at::kHalf, &out)) {
            const int64_t T = x->size(0), D = c.head_dim;
            if (x->size(1) == (heads + 2ll * c.n_kv_heads) * D && slots->numel() == T && (!qw || qw->numel() == D) && (!kw || kw->numel() == D) &&
                (!cs || (cs->dim() == 2 && cs->size(1) <= INT32_MAX && pos && pos->numel() == T)) && out->numel() >= T * heads * D) {
                const float eps = (float)PyFloat_AS_DOUBLE(a[10]), clip = (float)PyFloat_AS_DOUBLE(a[15]);
                const int interleaved = a[12] == Py_True, rotate = a[13] == Py_True;
                void* const st = stream();
                int rc;
                Py_BEGIN_ALLOW_THREADS
                rc = g_append(x->data_ptr(), row_stride(*x), T, (int32_t)heads, as<int32_t>(pos), as<int64_t>(slots), pointer(qw), pointer(kw), eps,
                              as<float>(cs), cs ? cs->size(0) : 0, cs ? (int32_t)cs->size(1) : 0, interleaved, rotate, clip, &c, out->data_ptr(), st);
                Py_END_ALLOW_THREADS
                return PyLong_FromLong(rc);
            }
        }
    } catch (...) {
    }
    return PyLong_FromLong(-1);
}

// (q, cu_q, kv_len, block_table, k_codes, v_codes, k_scale, v_scale, softmax_scale, max_q, group, prefix_k or None, prefix_v or None, causal,
//  out, workspace)
PyObject* kv4_attention(PyObject*, PyObject* const* a, Py_ssize_t n)
{
    try {
        const at::Tensor *q, *cu, *kv, *table, *pk, *pv, *out, *ws;
        int64_t max_q, group;
        pq_kv4_cache c;
        if (n == 16 && g_attention && rows_here(a[0], &q) && operand_here(a[1], at::kInt, &cu) && operand_here(a[2], at::kInt, &kv) &&
            operand_here(a[3], at::kInt, &table) && PyFloat_CheckExact(a[8]) && whole(a[9], 1, INT32_MAX, &max_q) &&
            whole(a[10], 0, INT32_MAX, &group) && cache_here(a + 4, group, &c) && optional_here(a[11], at::kHalf, &pk) &&
            optional_here(a[12], at::kHalf, &pv) && PyBool_Check(a[13]) && operand_here(a[14], at::kHalf, &out) &&
            operand_here(a[15], at::kByte, &ws)) {
            const int64_t T = q->size(0), D = c.head_dim, B = kv->numel(), heads = D ? q->size(1) / D : 0;
            const bool prefix = pk && pk->dim() == 3 && pk->size(1) == c.n_kv_heads && pk->size(2) == D && pv && pv->sizes() == pk->sizes();
            if (heads > 0 && heads * D == q->size(1) && heads <= INT32_MAX && cu->numel() == B + 1 && table->dim() == 2 && table->size(0) == B &&
                table->size(1) <= INT32_MAX && B <= INT32_MAX && (prefix || (!pk && !pv)) && (!prefix || pk->size(0) <= INT32_MAX) &&
                out->numel() >= T * heads * D) {
                const float scale = (float)PyFloat_AS_DOUBLE(a[8]);
                const int causal = a[13] == Py_True;
                void* const st = stream();
                int rc;
                Py_BEGIN_ALLOW_THREADS
                rc = g_attention(q->data_ptr(), row_stride(*q), T, (int32_t)heads, as<int32_t>(cu), as<int32_t>(kv), (int32_t)B, (int32_t)max_q,
                                 as<int32_t>(table), (int32_t)table->size(1), &c, pointer(pk), pointer(pv), prefix ? (int32_t)pk->size(0) : 0, scale,
                                 causal, out->data_ptr(), ws->data_ptr(), (size_t)ws->numel(), st);
                Py_END_ALLOW_THREADS
                return PyLong_FromLong(rc);
            }
        }
    } catch (...) {
    }
    return PyLong_FromLong(-1);
}

// (addresses of pq_kv4_slots, pq_kv4_append and pq_kv4_attention)
PyObject* bind_kv4(PyObject*, PyObject* args)
{
    unsigned long long s, ap, at;
    if (!PyArg_ParseTuple(args, "KKK", &s, &ap, &at)) return nullptr;
    g_slots = reinterpret_cast<Slots>(static_cast<uintptr_t>(s));
    g_append = reinterpret_cast<Append>(static_cast<uintptr_t>(ap));
    g_attention = reinterpret_cast<Attention>(static_cast<uintptr_t>(at));
    Py_RETURN_NONE;
}

// (address of pq_linear, address of pq_linear2): the library that the binding has loaded
PyObject* bind(PyObject*, PyObject* args)
{
    unsigned long long l, l2;
    if (!PyArg_ParseTuple(args, "KK", &l, &l2)) return nullptr;
    g_linear = reinterpret_cast<Linear>(static_cast<uintptr_t>(l));
    g_linear2 = reinterpret_cast<Linear2>(static_cast<uintptr_t>(l2));
    Py_RETURN_NONE;
}

PyMethodDef methods[] = {{"bind", bind, METH_VARARGS, nullptr},
                         {"linear", reinterpret_cast<PyCFunction>(reinterpret_cast<void*>(linear)), METH_FASTCALL, nullptr},
                         {"linear2", reinterpret_cast<PyCFunction>(reinterpret_cast<void*>(linear2)), METH_FASTCALL, nullptr},
                         {"bind_kv4", bind_kv4, METH_VARARGS, nullptr},
                         {"kv4_slots", reinterpret_cast<PyCFunction>(reinterpret_cast<void*>(kv4_slots)), METH_FASTCALL, nullptr},
                         {"kv4_append", reinterpret_cast<PyCFunction>(reinterpret_cast<void*>(kv4_append)), METH_FASTCALL, nullptr},
                         {"kv4_attention", reinterpret_cast<PyCFunction>(reinterpret_cast<void*>(kv4_attention)), METH_FASTCALL, nullptr},
                         {nullptr, nullptr, 0, nullptr}};
PyModuleDef module = {PyModuleDef_HEAD_INIT, "_pq_call", nullptr, -1, methods, nullptr, nullptr, nullptr, nullptr};

}  // namespace

PyMODINIT_FUNC PyInit__pq_call(void) { return PyModule_Create(&module); }
