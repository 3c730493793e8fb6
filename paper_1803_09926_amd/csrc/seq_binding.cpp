// The calls of sequence.py and delta.py in native code, as binding.cpp has those of the convolutions: what is checked of plain device tensors, and the library call.
// Every function takes the descriptor, the operands in the order of its entry below (None where one is left out), the workspace where there is one, and the
// stream; it returns the library's status, or None where an argument is anything but what it takes for granted.
#include "binding.hpp"

#include "../../include/deltaops.h"

namespace {

enum Op { LNORM, CCONV, SSCAN, GDELTA, HNORM, RNORM, OPS };
enum Type { STORED, F32, I32, BYTES };
// Sizes of a descriptor that operands refer to: rows of a width and a stride, or a number of elements (BYTES: what the library says that `kept` needs)
struct Sizes { int64_t T; int64_t width[6], stride[6]; int64_t flat[5]; at::ScalarType stored; };
struct Field { int at; Type type; bool rows; int size; };   // its place in the struct of tensors; size: an index into width and stride, or into flat

#define AT(S, F) (int)(offsetof(S, F) / sizeof(void *))
constexpr int END = -1;

struct Entry { const char *symbol; Op op; bool workspace; Field fields[24]; };
#define L(F, ...) {AT(lnorm_tensors, F), __VA_ARGS__}
#define K(F, ...) {AT(cconv_tensors, F), __VA_ARGS__}
#define S(F, ...) {AT(sscan_tensors, F), __VA_ARGS__}
#define G(F, ...) {AT(gdelta_tensors, F), __VA_ARGS__}
#define H(F, ...) {AT(hnorm_tensors, F), __VA_ARGS__}
#define R(F, ...) {AT(rnorm_tensors, F), __VA_ARGS__}
#define STOP {END, STORED, false, 0}
const Entry ENTRIES[] = {
    {"lnorm_fwd", LNORM, false, {L(x, STORED, true, 0), L(residual, STORED, true, 0), L(w, STORED, false, 0), L(b, STORED, false, 0), L(y, STORED, true, 0),
                                 L(total, STORED, true, 0), L(mean, F32, false, 1), L(rstd, F32, false, 1), STOP}},
    {"lnorm_bwd", LNORM, true, {L(x, STORED, true, 0), L(w, STORED, false, 0), L(mean, F32, false, 1), L(rstd, F32, false, 1), L(dy, STORED, true, 0),
                                L(dtotal, STORED, true, 0), L(dx, STORED, true, 0), L(dw, F32, false, 0), L(db, F32, false, 0), STOP}},
    {"cconv_fwd", CCONV, false, {K(x, STORED, true, 0), K(w, STORED, false, 0), K(b, STORED, false, 1), K(starts, I32, false, 2), K(init, STORED, false, 3),
                                 K(y, STORED, true, 1), K(final, STORED, false, 3), STOP}},
    {"cconv_bwd", CCONV, true, {K(x, STORED, true, 0), K(w, STORED, false, 0), K(b, STORED, false, 1), K(starts, I32, false, 2), K(init, STORED, false, 3),
                                K(dy, STORED, true, 1), K(dx, STORED, true, 0), K(dw, F32, false, 0), K(db, F32, false, 1), STOP}},
    {"cconv_step", CCONV, false, {K(x, STORED, true, 0), K(w, STORED, false, 0), K(b, STORED, false, 1), K(slots, I32, false, 4), K(state, STORED, false, 3),
                                  K(y, STORED, true, 1), STOP}},
    {"sscan_fwd", SSCAN, true, {S(x, STORED, true, 0), S(dt, STORED, true, 1), S(A, F32, false, 0), S(B, STORED, true, 3), S(C, STORED, true, 4),
                                S(D, F32, false, 1), S(z, STORED, true, 2), S(dt_bias, F32, false, 1), S(starts, I32, false, 2), S(init, F32, false, 3),
                                S(y, STORED, true, 5), S(final, F32, false, 3), S(kept, BYTES, false, 0), STOP}},
    {"sscan_bwd", SSCAN, true, {S(x, STORED, true, 0), S(dt, STORED, true, 1), S(A, F32, false, 0), S(B, STORED, true, 3), S(C, STORED, true, 4),
                                S(D, F32, false, 1), S(z, STORED, true, 2), S(dt_bias, F32, false, 1), S(starts, I32, false, 2), S(init, F32, false, 3),
                                S(kept, BYTES, false, 0), S(dy, STORED, true, 5), S(dx, STORED, true, 0), S(ddt, STORED, true, 1), S(dA, F32, false, 0),
                                S(dB, STORED, true, 3), S(dC, STORED, true, 4), S(dD, F32, false, 1), S(dz, STORED, true, 2), S(ddt_bias, F32, false, 1), STOP}},
    {"sscan_step", SSCAN, false, {S(x, STORED, true, 0), S(dt, STORED, true, 1), S(A, F32, false, 0), S(B, STORED, true, 3), S(C, STORED, true, 4),
                                  S(D, F32, false, 1), S(z, STORED, true, 2), S(dt_bias, F32, false, 1), S(slots, I32, false, 4), S(state, F32, false, 3),
                                  S(y, STORED, true, 5), STOP}},
    {"gdelta_fwd", GDELTA, true, {G(q, STORED, true, 0), G(k, STORED, true, 1), G(v, STORED, true, 2), G(a, STORED, true, 3), G(b, STORED, true, 4),
                                  G(A, F32, false, 0), G(a_bias, F32, false, 0), G(starts, I32, false, 2), G(init, F32, false, 3), G(y, STORED, true, 5),
                                  G(final, F32, false, 3), G(kept, BYTES, false, 0), STOP}},
    {"gdelta_bwd", GDELTA, true, {G(q, STORED, true, 0), G(k, STORED, true, 1), G(v, STORED, true, 2), G(a, STORED, true, 3), G(b, STORED, true, 4),
                                  G(A, F32, false, 0), G(a_bias, F32, false, 0), G(starts, I32, false, 2), G(kept, BYTES, false, 0), G(dy, STORED, true, 5),
                                  G(dq, STORED, true, 0), G(dk, STORED, true, 1), G(dv, STORED, true, 2), G(da, STORED, true, 3), G(db, STORED, true, 4),
                                  G(dA, F32, false, 0), G(da_bias, F32, false, 0), STOP}},
    {"gdelta_step", GDELTA, false, {G(q, STORED, true, 0), G(k, STORED, true, 1), G(v, STORED, true, 2), G(a, STORED, true, 3), G(b, STORED, true, 4),
                                    G(A, F32, false, 0), G(a_bias, F32, false, 0), G(slots, I32, false, 4), G(state, F32, false, 3), G(y, STORED, true, 5),
                                    STOP}},
    {"hnorm_fwd", HNORM, false, {H(x, STORED, true, 0), H(z, STORED, true, 1), H(w, STORED, false, 0), H(y, STORED, true, 2), H(rstd, F32, false, 1), STOP}},
    {"hnorm_bwd", HNORM, true, {H(x, STORED, true, 0), H(z, STORED, true, 1), H(w, STORED, false, 0), H(rstd, F32, false, 1), H(dy, STORED, true, 2),
                                H(dx, STORED, true, 0), H(dz, STORED, true, 1), H(dw, F32, false, 0), STOP}},
    {"rnorm_fwd", RNORM, false, {R(x, STORED, true, 0), R(z, STORED, true, 1), R(residual, STORED, true, 2), R(w1, STORED, false, 0),
                                 R(scale, STORED, false, 0), R(w2, STORED, false, 0), R(total, STORED, true, 2), R(y, STORED, true, 2),
                                 R(rstd1, F32, false, 1), R(rstd2, F32, false, 1), STOP}},
    {"rnorm_bwd", RNORM, true, {R(x, STORED, true, 0), R(z, STORED, true, 1), R(w1, STORED, false, 0), R(scale, STORED, false, 0), R(w2, STORED, false, 0),
                                R(total, STORED, true, 2), R(rstd1, F32, false, 1), R(rstd2, F32, false, 1), R(dy, STORED, true, 2),
                                R(dtotal, STORED, true, 2), R(dx, STORED, true, 0), R(dz, STORED, true, 1), R(dresidual, STORED, true, 2),
                                R(dw1, F32, false, 0), R(dscale, F32, false, 0), R(dw2, F32, false, 0), STOP}},
};
constexpr int NENTRIES = sizeof ENTRIES / sizeof ENTRIES[0];
constexpr size_t SLOTS = sizeof(sscan_tensors) / sizeof(void *);     // the largest struct of tensors
static_assert(SLOTS * sizeof(void *) >= sizeof(cconv_tensors) && SLOTS * sizeof(void *) >= sizeof(lnorm_tensors) && SLOTS * sizeof(void *) >= sizeof(gdelta_tensors) &&
              SLOTS * sizeof(void *) >= sizeof(hnorm_tensors) && SLOTS * sizeof(void *) >= sizeof(rnorm_tensors), "the largest struct");

typedef int (*call_fn)(const void *, const void *, void *);
typedef int (*call_ws_fn)(const void *, const void *, void *, size_t, void *);
typedef size_t (*bytes_fn)(const void *);

// set once by bind(), under the interpreter's lock
void *entry_points[NENTRIES];
constexpr const char *KEPT[2] = {"sscan_kept_bytes", "gdelta_kept_bytes"};   // of the operators that have a `kept`, the second one's GDELTA
bytes_fn kept_bytes[2];
PyObject *desc_type[OPS];
constexpr size_t DESC_SIZE[OPS] = {sizeof(lnorm_desc), sizeof(cconv_desc), sizeof(sscan_desc), sizeof(gdelta_desc), sizeof(hnorm_desc), sizeof(rnorm_desc)};

union Desc { lnorm_desc l; cconv_desc k; sscan_desc s; gdelta_desc g; hnorm_desc h; rnorm_desc r; };

// false: left to the checks of the library by way of Python
bool sizes_of(Op op, const Desc &d, Sizes *s)
{
    int32_t dtype;
    if (op == LNORM) {
        if (d.l.T < 0 || d.l.C < 1) return false;
        *s = {d.l.T, {d.l.C}, {d.l.C}, {d.l.C, d.l.T}, at::kFloat};
        dtype = d.l.dtype;
    } else if (op == CCONV) {
        const cconv_desc &c = d.k;
        if (c.T < 0 || c.C < 1 || c.K < 2 || c.K > CCONV_MAX_K || c.sequences < 1) return false;
        *s = {c.T, {c.C, c.C}, {c.x_stride, c.y_stride},
              {(int64_t)c.K * c.C, c.C, (int64_t)c.sequences + 1, (int64_t)c.sequences * (c.K - 1) * c.C, c.T}, at::kFloat};
        dtype = c.dtype;
    } else if (op == GDELTA) {
        const gdelta_desc &c = d.g;
        if (c.T < 0 || c.H < 1 || c.K < 1 || c.K > GDELTA_MAX_K || c.V < 1 || c.V > GDELTA_MAX_V || c.key_heads < 1 || c.sequences < 1) return false;
        const int64_t keys = (int64_t)c.key_heads * c.K, values = (int64_t)c.H * c.V;
        *s = {c.T, {keys, keys, values, c.H, c.H, values}, {c.q_stride, c.k_stride, c.v_stride, c.a_stride, c.b_stride, c.y_stride},
              {c.H, 0, (int64_t)c.sequences + 1, 0, c.T}, at::kFloat};
        if (__builtin_mul_overflow((int64_t)c.sequences * c.H, (int64_t)c.K * c.V, &s->flat[3])) return false;
        dtype = c.dtype;
    } else if (op == HNORM) {
        const hnorm_desc &c = d.h;
        if (c.T < 0 || c.H < 1 || c.D < 1 || c.D > HNORM_MAX_D) return false;
        const int64_t width = (int64_t)c.H * c.D;
        *s = {c.T, {width, width, width}, {c.x_stride, c.z_stride, c.y_stride}, {c.D, (int64_t)c.T * c.H}, at::kFloat};
        dtype = c.dtype;
    } else if (op == RNORM) {
        const rnorm_desc &c = d.r;
        if (c.T < 0 || c.C < 1) return false;
        *s = {c.T, {c.C, c.C, c.C}, {c.x_stride, c.z_stride, c.C}, {c.C, c.T}, at::kFloat};
        dtype = c.dtype;
    } else {
        const sscan_desc &c = d.s;
        if (c.T < 0 || c.C < 1 || c.N < 1 || c.N > SSCAN_MAX_N || c.groups < 1 || c.sequences < 1) return false;
        const int64_t shared = (int64_t)c.groups * c.N;
        *s = {c.T, {c.C, c.C, c.C, shared, shared, c.C}, {c.x_stride, c.dt_stride, c.z_stride, c.b_stride, c.c_stride, c.y_stride},
              {(int64_t)c.C * c.N, c.C, (int64_t)c.sequences + 1, 0, c.T}, at::kFloat};
        if (__builtin_mul_overflow((int64_t)c.sequences * c.C, (int64_t)c.N, &s->flat[3])) return false;
        dtype = c.dtype;
    }
    s->stored = dtype == DWCONV_F32 ? at::kFloat : at::kBFloat16;
    return dtype == DWCONV_F32 || dtype == DWCONV_BF16;
}

// T rows of `width`, `stride` apart, whatever the dimensions are called
bool is_rows(const at::Tensor &t, int64_t T, int64_t width, int64_t stride)
{
    if (t.numel() != T * width) return false;
    if (t.numel() == 0) return true;
    int64_t inner = 1, expected = 1;
    bool outer = width == 1;
    if (outer) expected = stride;
    for (int64_t i = t.dim() - 1; i >= 0; --i) {
        const int64_t n = t.size(i);
        if (n == 1) continue;
        if (t.stride(i) != expected) return false;
        if (!outer) {
            inner *= n;
            if (inner > width) return stride == width && t.is_contiguous();
            expected *= n;
            if (inner == width) { outer = true; expected = stride; }
        } else expected *= n;
    }
    return true;
}

template <int E>
PyObject *call(PyObject *, PyObject *const *args, Py_ssize_t nargs)
{
    HANDLE_TH_ERRORS
    const Entry &e = ENTRIES[E];
    int fields = 0;
    while (e.fields[fields].at != END) ++fields;
    if (nargs != 1 + fields + e.workspace + 1) {
        PyErr_SetString(PyExc_TypeError, "wrong number of arguments");
        return nullptr;
    }
    if ((PyObject *)Py_TYPE(args[0]) != desc_type[e.op] || at::impl::torch_function_mode_enabled()) Py_RETURN_NONE;
    DescView v;
    if (PyObject_GetBuffer(args[0], &v.view, PyBUF_SIMPLE) != 0) return nullptr;
    if (v.view.len != (Py_ssize_t)DESC_SIZE[e.op]) Py_RETURN_NONE;
    Desc d = {};                             // a copy: another thread may write to the descriptor while the library reads it
    memcpy(&d, v.view.buf, v.view.len);
    Sizes s;
    if (!sizes_of(e.op, d, &s)) Py_RETURN_NONE;

    void *p[SLOTS] = {};
    for (int i = 0; i < fields; ++i) {
        const Field &f = e.fields[i];
        if (args[1 + i] == Py_None) continue;
        const at::Tensor *t = plain(args[1 + i]);
        if (!t) Py_RETURN_NONE;
        if (f.type == BYTES) {
            // (asked for here: the library works it out anew, and calls without it do not need it)
            if (!t->is_contiguous() || (size_t)t->numel() * t->itemsize() < kept_bytes[e.op == GDELTA](&d)) Py_RETURN_NONE;
        } else {
            if (t->scalar_type() != (f.type == F32 ? at::kFloat : f.type == I32 ? at::kInt : s.stored)) Py_RETURN_NONE;
            if (f.rows ? !is_rows(*t, s.T, s.width[f.size], s.stride[f.size]) : t->numel() != s.flat[f.size] || !t->is_contiguous()) Py_RETURN_NONE;
        }
        p[f.at] = t->data_ptr();
    }
    void *ws = nullptr;
    size_t bytes = 0;
    if (e.workspace && args[1 + fields] != Py_None) {
        const at::Tensor *t = plain(args[1 + fields]);
        if (!t || !t->is_contiguous()) Py_RETURN_NONE;
        ws = t->data_ptr();
        bytes = (size_t)t->numel() * t->itemsize();
    }
    void *stream;
    switch (stream_of(args[nargs - 1], &stream)) {
    case STREAM_ERROR: return nullptr;
    case STREAM_OTHER: Py_RETURN_NONE;
    case STREAM_TAKEN: break;
    }
    int rc;
    void *const fn = entry_points[E];
    Py_BEGIN_ALLOW_THREADS                   // (the launch may wait for room in the stream's queue)
    if (e.workspace) rc = ((call_ws_fn)fn)(&d, p, ws, bytes, stream);
    else rc = ((call_fn)fn)(&d, p, stream);
    Py_END_ALLOW_THREADS
    return PyLong_FromLong(rc);
    END_HANDLE_TH_ERRORS
}

// bind(lookup, the descriptors' types in the order of Op, Tensor, Parameter): lookup(symbol) gives the address of one of the library's functions
PyObject *bind(PyObject *, PyObject *args)
{
    if (PyTuple_GET_SIZE(args) != 1 + OPS + 2) {
        PyErr_SetString(PyExc_TypeError, "wrong number of arguments");
        return nullptr;
    }
    void *found[NENTRIES + 2];
    for (int i = 0; i < NENTRIES + 2; ++i) {
        PyObject *a = PyObject_CallFunction(PyTuple_GET_ITEM(args, 0), "s", i < NENTRIES ? ENTRIES[i].symbol : KEPT[i - NENTRIES]);
        found[i] = a ? PyLong_AsVoidPtr(a) : nullptr;
        Py_XDECREF(a);
        if (PyErr_Occurred()) return nullptr;
        if (!found[i]) { PyErr_SetString(PyExc_RuntimeError, "no such function"); return nullptr; }
    }
    for (int i = 0; i < NENTRIES; ++i) entry_points[i] = found[i];
    for (int i = 0; i < 2; ++i) kept_bytes[i] = (bytes_fn)found[NENTRIES + i];
    for (int i = 1; i < 1 + OPS + 2; ++i) Py_INCREF(PyTuple_GET_ITEM(args, i));   // (kept until the process ends)
    for (int i = 0; i < OPS; ++i) desc_type[i] = PyTuple_GET_ITEM(args, 1 + i);
    tensor_type = PyTuple_GET_ITEM(args, 1 + OPS);
    parameter_type = PyTuple_GET_ITEM(args, 2 + OPS);
    Py_RETURN_NONE;
}

#define CALL(E) {ENTRIES[E].symbol, (PyCFunction)(void (*)(void))call<E>, METH_FASTCALL, nullptr}
PyMethodDef methods[] = {CALL(0), CALL(1), CALL(2), CALL(3), CALL(4), CALL(5), CALL(6), CALL(7), CALL(8), CALL(9), CALL(10), CALL(11),
                         CALL(12), CALL(13), CALL(14),
                         {"bind", bind, METH_VARARGS, nullptr}, {nullptr, nullptr, 0, nullptr}};
static_assert(NENTRIES == 15, "one method each");
PyModuleDef module = {PyModuleDef_HEAD_INIT, "_seq_binding", "checks and library calls of the sequence operators", -1, methods, nullptr, nullptr, nullptr, nullptr};

}  // namespace

PyMODINIT_FUNC PyInit__seq_binding() { return PyModule_Create(&module); }
