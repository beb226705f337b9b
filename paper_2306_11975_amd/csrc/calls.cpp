// The Python calls of the operators in 8-bit floating point and of those for mixtures of experts: a tensor's sizes, strides, type and address are
// read, checked and handed to the C entry in one step. Bound: the host. Reading them from Python and converting two dozen arguments were half of
// what a call took: one token through 2048 x 2048 7.5 us so, 5.0 here (which is the kernel); choice, order and gradient of 16 tokens 18.7, 10.5.
// The functions of ozimmu.py that carry their names say what they take; here every argument is there, by position.
#include <torch/csrc/autograd/python_variable.h>

#include <algorithm>
#include <cstdint>
#include <stdexcept>
#include <string>

#include "ozimmu.h"

namespace {

using at::Tensor;

struct PythonError {};      // set already
[[noreturn]] void bad(const std::string& what) { throw std::invalid_argument(what); }
void expect(bool condition, const char* what) {
    if (!condition) bad(what);
}

const Tensor& tensor(PyObject* o) {
    if (!THPVariable_Check(o)) {
        PyErr_SetString(PyExc_TypeError, "expected a tensor");
        throw PythonError();
    }
    return THPVariable_Unpack(o);
}
const Tensor* maybe(PyObject* o) { return o == Py_None ? nullptr : &tensor(o); }
void* address(const Tensor& t) { return t.data_ptr(); }
void* address(const Tensor* t) { return t ? t->data_ptr() : nullptr; }
int64_t integer(PyObject* o) {
    const int64_t x = PyLong_AsLongLong(o);
    if (x == -1 && PyErr_Occurred()) throw PythonError();
    return x;
}
int small(PyObject* o) {
    const int64_t x = integer(o);
    return (int)std::min<int64_t>(std::max<int64_t>(x, INT32_MIN), INT32_MAX);
}
double real(PyObject* o) {
    const double x = PyFloat_AsDouble(o);
    if (x == -1.0 && PyErr_Occurred()) throw PythonError();
    return x;
}
int truth(PyObject* o) {
    const int x = PyObject_IsTrue(o);
    if (x < 0) throw PythonError();
    return x;
}

// Rows, columns and row stride of a matrix with unit stride along its rows.
struct Matrix {
    int64_t rows, cols, ld;
};
Matrix matrix(const Tensor& t) {
    expect(t.dim() == 2, "expected a 2-D tensor");
    const Matrix m{t.size(0), t.size(1), t.stride(0)};
    expect(t.stride(1) == 1 || m.cols <= 1, "expected a row-major tensor (unit stride along the second dimension)");
    return {m.rows, m.cols, m.rows > 1 ? m.ld : std::max<int64_t>(m.cols, 1)};
}
// The rows of all experts of a tensor whose first dimension they are.
Matrix matrices(const Tensor& t, int64_t& experts) {
    if (t.dim() != 3 || (t.size(0) > 1 && t.size(1) > 0 && t.stride(0) != t.stride(1) * t.size(1)) || (t.size(2) > 1 && t.stride(2) != 1))
        bad("over experts, weights, scales and weights' gradients have three dimensions, the experts' rows one behind the other");
    experts = t.size(0);
    const int64_t rows = t.size(0) * t.size(1), cols = t.size(2), one = std::max<int64_t>(cols, 1);
    return {rows, cols, rows <= 1 ? one : t.size(1) > 1 ? t.stride(1) : t.stride(0)};
}
int wide_type(const Tensor& t) {   // -1: none of them
    switch (t.scalar_type()) {
        case at::kFloat: return OZIMMU_F32;
        case at::kBFloat16: return OZIMMU_BF16;
        case at::kHalf: return OZIMMU_F16;
        default: return -1;
    }
}
ozimmu_type_t type_of(const Tensor& t) {
    const int x = wide_type(t);
    if (x < 0) bad(std::string("expected float32, bfloat16 or float16, got ") + c10::toString(t.scalar_type()));
    return (ozimmu_type_t)x;
}
bool holds_codes(const Tensor& t) { return t.scalar_type() == at::kByte || t.scalar_type() == at::kFloat8_e4m3fn; }
int scale_type(const Tensor& t) {   // -1: none of them
    if (t.scalar_type() == at::kFloat) return OZIMMU_F32;
    return t.scalar_type() == at::kByte || t.scalar_type() == at::kFloat8_e8m0fnu ? OZIMMU_E8M0 : -1;
}
template <class T, at::ScalarType TYPE>
T* values(const Tensor& t, int64_t count, const char* what) {
    if (t.scalar_type() != TYPE || t.numel() != count || !t.is_contiguous())
        bad(std::string(what) + ": expected " + std::to_string(count) + " contiguous " + (TYPE == at::kInt ? "int32" : "float32") + " values");
    return static_cast<T*>(t.data_ptr());
}
int* ints(const Tensor& t, int64_t count, const char* what) { return values<int, at::kInt>(t, count, what); }
float* floats(const Tensor& t, int64_t count, const char* what) { return values<float, at::kFloat>(t, count, what); }
const int* ints(const Tensor* t, int64_t count, const char* what) { return t ? ints(*t, count, what) : nullptr; }
Matrix pairs(const Tensor& t, const char* what) {
    if (t.dim() != 2) bad(std::string(what) + ": expected a row for each token");
    return {t.size(0), std::min<int64_t>(t.size(1), OZIMMU_MAX_CHOICES + 1), 0};      // (more are refused by the C entry)
}
size_t bytes_of(const Tensor* workspace) {
    if (!workspace) return 0;
    expect(workspace->is_contiguous(), "expected a contiguous workspace");
    return (size_t)workspace->numel() * workspace->element_size();
}

// Codes and scales of an n x k matrix in blocks of block_rows x 128 (experts: matrices of that, one behind the other).
struct Codes {
    int64_t ldq, lds;
    ozimmu_type_t scale_type;
};
Codes check_codes(const char* what, const Matrix& q, const Tensor& codes, const Matrix& s, const Tensor& scales, int64_t n, int64_t k, int64_t block_rows, int64_t experts) {
    const int64_t each = std::max<int64_t>(experts, 1), groups = (k + 127) / 128, srows = (n + block_rows - 1) / block_rows;
    const std::string per = experts ? " for each expert" : "";
    if (q.rows != n * each || q.cols < 128 * groups || !holds_codes(codes))
        bad(std::string(what) + ": expected " + std::to_string(n) + " rows" + per + " of at least " + std::to_string(128 * groups) + " codes (uint8 or float8_e4m3fn)");
    const int kind = scale_type(scales);
    const int64_t most = kind == OZIMMU_F32 ? groups : (groups + 3) / 4 * 4;
    if (kind < 0 || s.rows != srows * each || s.cols < most)
        bad(std::string(what) + "' scales: expected " + std::to_string(srows) + " rows" + per + " of at least " + std::to_string(most) + " (float8_e8m0fnu or uint8: multiples of four) or " +
            std::to_string(groups) + " (float32)");
    return {q.rows > 1 ? q.ld : 128 * groups, s.rows > 1 ? s.ld : most, (ozimmu_type_t)kind};
}

// torch's functions for the current device and its current stream.
PyObject *get_device, *raw_stream, *exchange_device, *exchange_back;
int64_t ask(PyObject* f, int64_t index) {
    PyObject* at = PyLong_FromLongLong(index);
    PyObject* r = at ? PyObject_CallOneArg(f, at) : nullptr;
    Py_XDECREF(at);
    if (!r) throw PythonError();
    const int64_t x = (int64_t)PyLong_AsUnsignedLongLongMask(r);
    Py_DECREF(r);
    if (PyErr_Occurred()) throw PythonError();
    return x;
}
int64_t attribute(PyObject* o, const char* name, const char* then) {
    PyObject* a = PyObject_GetAttrString(o, name);
    PyObject* b = a && then ? PyObject_GetAttrString(a, then) : a;
    if (then) Py_XDECREF(a);
    if (!b) throw PythonError();
    const int64_t x = (int64_t)PyLong_AsUnsignedLongLongMask(b);
    Py_DECREF(b);
    if (PyErr_Occurred()) throw PythonError();
    return x;
}

// f(stream) with the tensors' device current: all must be on one GPU. Without a stream, torch's current one of that device is taken. f is the C
// entry, with addresses read before: it throws nothing.
template <class F>
PyObject* call(std::initializer_list<const Tensor*> tensors, PyObject* stream, F&& f) {
    int64_t index = -2;
    for (const Tensor* t : tensors)
        if (t) {
            const int64_t at = t->is_cuda() ? t->get_device() : -1;
            if (index == -2) index = at;
            expect(at == index, "all tensors must be on one device");
        }
    expect(index >= 0, "expected tensors on a GPU");
    void* raw;
    if (stream == Py_None) {
        raw = reinterpret_cast<void*>(ask(raw_stream, index));
    } else {
        expect(attribute(stream, "device", "index") == index, "the stream belongs to another device than the tensors");
        raw = reinterpret_cast<void*>(attribute(stream, "cuda_stream", nullptr));
    }
    PyObject* current = PyObject_CallNoArgs(get_device);
    if (!current) throw PythonError();
    const bool other = PyLong_AsLongLong(current) != index;
    Py_DECREF(current);
    const int64_t before = other ? ask(exchange_device, index) : 0;
    ozimmu_status_t code;
    {
        struct Unlocked {
            PyThreadState* state = PyEval_SaveThread();
            ~Unlocked() { PyEval_RestoreThread(state); }
        } unlocked;
        code = f(raw);
    }
    if (other) ask(exchange_back, before);
    return PyLong_FromLong(code);
}

// ---- the operators
PyObject* f8_split(PyObject* const* a) {   // W, codes, scales, block_rows, stream
    const Tensor &W = tensor(a[0]), &codes = tensor(a[1]), &scales = tensor(a[2]);
    const Matrix w = matrix(W);
    const int64_t block = integer(a[3]);
    expect(block == 1 || block == 128, "block_rows: expected 1 or 128");
    const Codes c = check_codes("codes", matrix(codes), codes, matrix(scales), scales, w.rows, w.cols, block, 0);
    expect(c.scale_type == OZIMMU_E8M0, "the cut makes scales of a byte (uint8 or float8_e8m0fnu)");
    const ozimmu_type_t type = type_of(W);
    void* pw = address(W);
    uint8_t *pq = static_cast<uint8_t*>(address(codes)), *ps = static_cast<uint8_t*>(address(scales));
    return call({&W, &codes, &scales}, a[4], [&](void* st) { return ozimmu_f8_split(w.rows, w.cols, (int)block, type, pw, w.ld, pq, c.ldq, ps, c.lds, st); });
}
PyObject* f8_expand(PyObject* const* a) {   // codes, scales, W, block_rows, stream
    const Tensor &codes = tensor(a[0]), &scales = tensor(a[1]), &W = tensor(a[2]);
    const Matrix w = matrix(W);
    const int64_t block = integer(a[3]);
    expect(block == 1 || block == 128, "block_rows: expected 1 or 128");
    const Codes c = check_codes("codes", matrix(codes), codes, matrix(scales), scales, w.rows, w.cols, block, 0);
    const ozimmu_type_t type = type_of(W);
    const uint8_t* pq = static_cast<const uint8_t*>(address(codes));
    void *pw = address(W), *ps = address(scales);
    return call({&W, &codes, &scales}, a[4], [&](void* st) { return ozimmu_f8_expand(w.rows, w.cols, (int)block, pq, c.ldq, c.scale_type, ps, c.lds, type, pw, w.ld, st); });
}

PyObject* f8_product(bool gradient, const Tensor& V, const Tensor& codes, const Tensor& scales, const Tensor& R, const Tensor* workspace, const Tensor* v_scales, const Tensor* offsets,
                     const Tensor* source, PyObject* stream) {
    const Matrix v = matrix(V), r = matrix(R);
    int64_t experts = 0, experts_s = 0;
    const Matrix q = offsets ? matrices(codes, experts) : matrix(codes), s = offsets ? matrices(scales, experts_s) : matrix(scales);
    expect(experts == experts_s, "codes and scales must have the same number of experts");
    int64_t inner = v.cols, ldv = v.ld, ldvs = 0;
    int type = wide_type(V);
    if (type < 0) {
        if (!holds_codes(V)) type_of(V);      // (throws)
        expect(v_scales && v_scales->scalar_type() != at::kFloat, "codes of tokens need their scales, which are bytes");
        type = OZIMMU_E4M3;
        // the width of codes is padded: the other sizes tell it
        inner = gradient ? q.rows / std::max<int64_t>(experts, 1) : std::min(inner, q.cols);
        const Codes c = check_codes("tokens", v, V, matrix(*v_scales), *v_scales, v.rows, inner, 1, 0);
        ldv = c.ldq;
        ldvs = c.lds;
    } else {
        expect(!v_scales, "only codes have scales");
    }
    const int64_t n = gradient ? inner : r.cols, k = gradient ? r.cols : inner;
    const Codes c = check_codes("codes", q, codes, s, scales, n, k, 128, experts);
    expect(r.rows == v.rows || (!gradient && source), "tokens and result must have the same number of rows");
    const ozimmu_type_t out = type_of(R);
    const size_t size = bytes_of(workspace);
    const int *po = ints(offsets, experts + 1, "offsets"), *ps = ints(source, r.rows, "source");
    const uint8_t *pq = static_cast<const uint8_t*>(address(codes)), *pvs = static_cast<const uint8_t*>(address(v_scales));
    void *pv = address(V), *psc = address(scales), *pr = address(R), *pws = address(workspace);
    return call({&V, &codes, &scales, &R, workspace, v_scales, offsets, source}, stream, [&](void* st) {
        if (gradient)
            return ozimmu_f8_gemm_grad(r.rows, n, k, experts, (ozimmu_type_t)type, pv, ldv, pvs, ldvs, pq, c.ldq, c.scale_type, psc, c.lds, po, out, pr, r.ld, pws, size, st);
        return ozimmu_f8_gemm(v.rows, r.rows, n, k, experts, (ozimmu_type_t)type, pv, ldv, pvs, ldvs, pq, c.ldq, c.scale_type, psc, c.lds, po, ps, out, pr, r.ld, pws, size, st);
    });
}
PyObject* f8_gemm(PyObject* const* a) {   // X, codes, scales, Y, workspace, x_scales, offsets, source, stream
    return f8_product(false, tensor(a[0]), tensor(a[1]), tensor(a[2]), tensor(a[3]), maybe(a[4]), maybe(a[5]), maybe(a[6]), maybe(a[7]), a[8]);
}
PyObject* f8_gemm_grad(PyObject* const* a) {   // dY, codes, scales, dX, workspace, dy_scales, offsets, stream
    return f8_product(true, tensor(a[0]), tensor(a[1]), tensor(a[2]), tensor(a[3]), maybe(a[4]), maybe(a[5]), maybe(a[6]), nullptr, a[7]);
}
PyObject* f8_weight_grad(PyObject* const* a) {   // dY, X, dW, workspace, offsets, source, stream
    const Tensor &dY = tensor(a[0]), &X = tensor(a[1]), &dW = tensor(a[2]);
    const Tensor *workspace = maybe(a[3]), *offsets = maybe(a[4]), *source = maybe(a[5]);
    const Matrix dy = matrix(dY), x = matrix(X);
    int64_t experts = 0;
    const Matrix dw = offsets ? matrices(dW, experts) : matrix(dW);
    expect(dY.scalar_type() == X.scalar_type(), "dY and X must have one type");
    if (dw.rows != dy.cols * std::max<int64_t>(experts, 1) || dw.cols != x.cols)
        bad("dW: expected " + std::to_string(dy.cols) + " x " + std::to_string(x.cols) + (experts ? " for each expert" : ""));
    expect(source || dy.rows == x.rows, "dY and X must have the same number of rows");
    const int *po = ints(offsets, experts + 1, "offsets"), *ps = ints(source, dy.rows, "source");
    const ozimmu_type_t type = type_of(X), out = type_of(dW);
    const size_t size = bytes_of(workspace);
    void *pdy = address(dY), *px = address(X), *pdw = address(dW), *pws = address(workspace);
    return call({&dY, &X, &dW, workspace, offsets, source}, a[6],
                [&](void* st) { return ozimmu_f8_weight_grad(x.rows, dy.rows, dy.cols, x.cols, experts, type, pdy, dy.ld, px, x.ld, po, ps, out, pdw, dw.ld, pws, size, st); });
}

PyObject* route(PyObject* const* a) {   // logits, indices, weights, bias, score, groups, top_groups, renormalize, scale, stream
    const Tensor &logits = tensor(a[0]), &indices = tensor(a[1]), &weights = tensor(a[2]);
    const Tensor* bias = maybe(a[3]);
    const Matrix l = matrix(logits), p = pairs(indices, "indices");
    expect(p.rows == l.rows, "logits and indices must have the same number of rows");
    const ozimmu_type_t type = type_of(logits);
    const float* b = bias ? floats(*bias, l.cols, "bias") : nullptr;
    int* i = ints(indices, p.rows * p.cols, "indices");
    float* w = floats(weights, p.rows * p.cols, "weights");
    const int score = small(a[4]), groups = small(a[5]), top_groups = small(a[6]), renormalize = truth(a[7]);
    const double scale = real(a[8]);
    void* pl = address(logits);
    return call({&logits, &indices, &weights, bias}, a[9], [&](void* st) {
        return ozimmu_route(l.rows, l.cols, (int)p.cols, type, pl, l.ld, b, (ozimmu_score_t)score, groups, top_groups, renormalize, scale, i, w, st);
    });
}
PyObject* route_grad(PyObject* const* a) {   // logits, indices, dweights, dlogits, score, renormalize, scale, stream
    const Tensor &logits = tensor(a[0]), &indices = tensor(a[1]), &dweights = tensor(a[2]), &dlogits = tensor(a[3]);
    const Matrix l = matrix(logits), p = pairs(indices, "indices"), d = matrix(dlogits);
    expect(p.rows == l.rows, "logits and indices must have the same number of rows");
    expect(d.rows == l.rows && d.cols == l.cols && dlogits.scalar_type() == logits.scalar_type(), "dlogits must have the shape and type of the logits");
    const ozimmu_type_t type = type_of(logits);
    const int* i = ints(indices, p.rows * p.cols, "indices");
    const float* w = floats(dweights, p.rows * p.cols, "dweights");
    const int score = small(a[4]), renormalize = truth(a[5]);
    const double scale = real(a[6]);
    void *pl = address(logits), *pd = address(dlogits);
    return call({&logits, &indices, &dweights, &dlogits}, a[7],
                [&](void* st) { return ozimmu_route_grad(l.rows, l.cols, (int)p.cols, type, pl, l.ld, i, w, (ozimmu_score_t)score, renormalize, scale, pd, d.ld, st); });
}

PyObject* expert_order(PyObject* const* a) {   // indices, experts, offsets, source, place, workspace, stream
    const Tensor &indices = tensor(a[0]), &offsets = tensor(a[2]), &source = tensor(a[3]), &place = tensor(a[4]);
    const Tensor* workspace = maybe(a[5]);
    const Matrix p = pairs(indices, "indices");
    const int64_t experts = integer(a[1]), count = p.rows * p.cols;
    const int* i = ints(indices, count, "indices");
    int *o = ints(offsets, experts + 1, "offsets"), *s = ints(source, count, "source"), *pl = ints(place, count, "place");
    const size_t size = bytes_of(workspace);
    void* pws = address(workspace);
    return call({&indices, &offsets, &source, &place, workspace}, a[6], [&](void* st) { return ozimmu_expert_order(p.rows, (int)p.cols, experts, i, o, s, pl, pws, size, st); });
}
PyObject* expert_combine(PyObject* const* a) {   // O, place, weights, Y, stream
    const Tensor &O = tensor(a[0]), &place = tensor(a[1]), &Y = tensor(a[3]);
    const Tensor* weights = maybe(a[2]);
    const Matrix o = matrix(O), y = matrix(Y), p = pairs(place, "place");
    expect(p.rows == y.rows && o.cols == y.cols && O.scalar_type() == Y.scalar_type(), "O and Y must have one type and width, place and Y the same number of rows");
    const ozimmu_type_t type = type_of(O);
    const int* pl = ints(place, p.rows * p.cols, "place");
    const float* w = weights ? floats(*weights, p.rows * p.cols, "weights") : nullptr;
    void *po = address(O), *py = address(Y);
    return call({&O, &place, weights, &Y}, a[4], [&](void* st) { return ozimmu_expert_combine(y.rows, (int)p.cols, o.rows, o.cols, type, po, o.ld, pl, w, py, y.ld, st); });
}
PyObject* expert_combine_grad(PyObject* const* a) {   // dY, O, place, weights, dO, dweights, stream
    const Tensor &dY = tensor(a[0]), &O = tensor(a[1]), &place = tensor(a[2]), &weights = tensor(a[3]), &dO = tensor(a[4]), &dweights = tensor(a[5]);
    const Matrix dy = matrix(dY), o = matrix(O), d = matrix(dO), p = pairs(place, "place");
    expect(p.rows == dy.rows && o.cols == dy.cols && d.rows == o.rows && d.cols == dy.cols && O.scalar_type() == dY.scalar_type() && dO.scalar_type() == dY.scalar_type(),
           "dY, O and dO must have one type and width, dO the rows of O, place those of dY");
    const ozimmu_type_t type = type_of(O);
    const int* pl = ints(place, p.rows * p.cols, "place");
    const float* w = floats(weights, p.rows * p.cols, "weights");
    float* dw = floats(dweights, p.rows * p.cols, "dweights");
    void *pdy = address(dY), *po = address(O), *pd = address(dO);
    return call({&dY, &O, &place, &weights, &dO, &dweights}, a[6],
                [&](void* st) { return ozimmu_expert_combine_grad(dy.rows, (int)p.cols, o.rows, dy.cols, type, pdy, dy.ld, po, o.ld, pl, w, pd, d.ld, dw, st); });
}

template <PyObject* (*OPERATOR)(PyObject* const*), int ARGUMENTS>
PyObject* entry(PyObject*, PyObject* const* args, Py_ssize_t count) {
    if (count != ARGUMENTS) return PyErr_Format(PyExc_TypeError, "expected %d arguments, got %zd", ARGUMENTS, count);
    try {
        return OPERATOR(args);
    } catch (const PythonError&) {
        return nullptr;
    } catch (const std::invalid_argument& e) {
        PyErr_SetString(PyExc_ValueError, e.what());
    } catch (const std::exception& e) {
        PyErr_SetString(PyExc_RuntimeError, e.what());
    }
    return nullptr;
}
#define CALL(name, arguments) {#name, reinterpret_cast<PyCFunction>(reinterpret_cast<void (*)()>(&entry<name, arguments>)), METH_FASTCALL, nullptr}
PyMethodDef methods[] = {CALL(f8_split, 5),   CALL(f8_expand, 5),  CALL(f8_gemm, 9),      CALL(f8_gemm_grad, 8),   CALL(f8_weight_grad, 7), CALL(route, 10),
                         CALL(route_grad, 8), CALL(expert_order, 7), CALL(expert_combine, 5), CALL(expert_combine_grad, 7), {nullptr, nullptr, 0, nullptr}};
PyModuleDef module = {PyModuleDef_HEAD_INIT, "_calls", nullptr, -1, methods, nullptr, nullptr, nullptr, nullptr};

bool take(PyObject*& to, const char* from, const char* name) {
    PyObject* m = PyImport_ImportModule(from);
    to = m ? PyObject_GetAttrString(m, name) : nullptr;
    Py_XDECREF(m);
    return to != nullptr;
}

}  // namespace

PyMODINIT_FUNC PyInit__calls() {
    if (!take(get_device, "torch._C", "_cuda_getDevice") || !take(raw_stream, "torch._C", "_cuda_getCurrentRawStream") || !take(exchange_device, "torch.cuda", "_exchange_device") ||
        !take(exchange_back, "torch.cuda", "_maybe_exchange_device"))
        return nullptr;
    return PyModule_Create(&module);
}
