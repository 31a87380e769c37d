// The calls of binding.py that a program makes per layer, marshalled in C++: a ctypes call of 10 to 20 arguments takes
// 1.5 to 4 us of Python beside the 2.3 us a kernel launch costs the host, which is what a small layer waits for.
//
// bind(name, address, fallback) returns a function that takes what `fallback` (the Python form of the call) takes.
// The ordinary call -- device tensors, Python integers within the C types, the current stream -- goes straight to
// the C entry point at `address`; any other one (addresses as integers, host tensors, tensor subclasses, wrapped
// tensors, a given stream, numbers of other types, a wrong argument list) is handed to `fallback` unchanged, so what
// such calls do and raise is written in one place.  us per call on the host, ctypes / here: bwta_linear 4.3 / 3.1, the
// eleven calls of a decoder block 53 / 38, the nine of an attention layer 38 / 26.
#define PY_SSIZE_T_CLEAN
#include <Python.h>

#include <torch/csrc/autograd/python_variable.h>

#include <climits>
#include <cstdint>
#include <cstring>
#include <new>

#include "../../include/bwta.h"

namespace {

constexpr int kMaxParams = 24;

struct Bound;
// fills the call's arguments from `v` (one slot per parameter, null where not given) and makes it; false: not an
// ordinary call, nothing was done
typedef bool (*Marshal)(const Bound &b, PyObject *const *v, PyObject **result);

struct Spec {
    const char *name;
    int positional;  // parameters before the keyword-only ones
    const char *params[kMaxParams + 1];
    Marshal marshal;
};

struct Bound {
    PyObject_HEAD
    vectorcallfunc call;
    const Spec *spec;
    PyObject *names[kMaxParams];  // interned parameter names
    int count;
    void *address;
    PyObject *fallback;
    PyObject *weak;  // weak references
};

PyObject *g_check = nullptr, *g_raw_stream = nullptr, *g_device = nullptr;  // binding._check, torch's two stream calls
PyTypeObject *g_cache = nullptr;                                             // binding.Cache

struct NotOrdinary {};

// ---- argument readers: throw NotOrdinary for anything but the ordinary form

const at::Tensor *tensor(PyObject *o)
{
    if (o == nullptr || o == Py_None) return nullptr;
    if (!THPVariable_CheckExact(o)) throw NotOrdinary{};
    const at::Tensor &t = THPVariable_Unpack(o);
    if (!t.defined() || !t.is_cuda()) throw NotOrdinary{};
    return &t;
}

void *address(const at::Tensor *t) { return t ? t->data_ptr() : nullptr; }  // throws for tensors without storage

int64_t int64(PyObject *o)
{
    if (o == nullptr || !PyLong_CheckExact(o)) throw NotOrdinary{};
    int overflow = 0;
    const long long v = PyLong_AsLongLongAndOverflow(o, &overflow);
    if (overflow) throw NotOrdinary{};
    return v;
}

int int32(PyObject *o)
{
    const int64_t v = int64(o);
    if (v < INT_MIN || v > INT_MAX) throw NotOrdinary{};
    return (int)v;
}

bool given(PyObject *o) { return o != nullptr && o != Py_None; }
int64_t int64_or(PyObject *o, int64_t otherwise) { return given(o) ? int64(o) : otherwise; }

int scale_mode(PyObject *o, const at::Tensor *s)
{
    if (given(o)) return int32(o);
    return s == nullptr ? BWTA_SCALE_NONE : s->numel() == 1 ? BWTA_SCALE_SCALAR : BWTA_SCALE_VECTOR;
}

size_t bytes_of(PyObject *o, const at::Tensor *t)
{
    if (!given(o)) return t ? t->nbytes() : 0;
    const int64_t v = int64(o);
    if (v < 0) throw NotOrdinary{};
    return (size_t)v;
}

float number(PyObject *o, float otherwise)
{
    if (o == nullptr) return otherwise;
    if (!PyFloat_CheckExact(o)) throw NotOrdinary{};
    return (float)PyFloat_AS_DOUBLE(o);
}

// the current stream of the current device, as binding._stream finds it
void *current_stream(PyObject *o)
{
    if (given(o)) throw NotOrdinary{};
    PyObject *device = PyObject_CallNoArgs(g_device);
    PyObject *raw = device ? PyObject_CallOneArg(g_raw_stream, device) : nullptr;
    Py_XDECREF(device);
    void *st = raw ? PyLong_AsVoidPtr(raw) : nullptr;
    Py_XDECREF(raw);
    if (PyErr_Occurred()) {
        PyErr_Clear();
        throw NotOrdinary{};
    }
    return st;
}

// ---- the operators on heads: tensors of the current device alone, as binding._here has it

struct Here {
    long device;
    void *stream;
    const at::Tensor *tensor(PyObject *o) const
    {
        const at::Tensor *t = ::tensor(o);
        if (t && t->get_device() != device) throw NotOrdinary{};
        return t;
    }
    // what binding._dtype and binding._dense refuse is theirs to refuse
    const at::Tensor *rows(PyObject *o) const
    {
        const at::Tensor *t = tensor(o);
        if (t && t->dim() && t->stride(-1) != 1 && t->size(-1) > 1) throw NotOrdinary{};
        return t;
    }
    const at::Tensor *rows_like(PyObject *o, const at::Tensor *first) const
    {
        const at::Tensor *t = rows(o);
        if (t && first && t->scalar_type() != first->scalar_type()) throw NotOrdinary{};
        return t;
    }
    const at::Tensor *dense(PyObject *o, at::ScalarType type) const
    {
        const at::Tensor *t = tensor(o);
        if (t && (t->scalar_type() != type || !t->is_contiguous())) throw NotOrdinary{};
        return t;
    }
    const at::Tensor *ints(PyObject *o) const { return dense(o, at::kInt); }
    const at::Tensor *floats(PyObject *o) const { return dense(o, at::kFloat); }
    const at::Tensor *table(PyObject *o) const
    {
        const at::Tensor *t = rows(o);
        if (t && t->scalar_type() != at::kInt) throw NotOrdinary{};
        return t;
    }
};

Here here(PyObject *stream)
{
    if (given(stream)) throw NotOrdinary{};
    PyObject *device = PyObject_CallNoArgs(g_device);
    PyObject *raw = device ? PyObject_CallOneArg(g_raw_stream, device) : nullptr;
    Here h{device ? PyLong_AsLong(device) : -1, raw ? PyLong_AsVoidPtr(raw) : nullptr};
    Py_XDECREF(device);
    Py_XDECREF(raw);
    if (PyErr_Occurred()) throw NotOrdinary{};
    return h;
}

struct Cache {  // binding.Cache: the C struct, and one more than the number of its tensors' device (0: not known)
    bwta_cache c;
    int32_t place;
};

Cache cache_of(PyObject *o, const Here &h)
{
    if (!o || Py_TYPE(o) != g_cache) throw NotOrdinary{};
    Py_buffer view;
    if (PyObject_GetBuffer(o, &view, PyBUF_SIMPLE) != 0) throw NotOrdinary{};
    Cache c;
    const bool fits = view.len >= (Py_ssize_t)sizeof c;
    if (fits) memcpy(&c, view.buf, sizeof c);
    PyBuffer_Release(&view);
    if (!fits || (c.place > 0 && c.place - 1 != h.device)) throw NotOrdinary{};
    return c;
}

int head_dtype(PyObject *o, const at::Tensor *t)  // (that the others are of the first tensor's type is rows_like's to see)
{
    if (t && t->scalar_type() != at::kHalf && t->scalar_type() != at::kBFloat16) throw NotOrdinary{};
    const int named = given(o) ? int32(o) : -1;
    if (!t) return given(o) ? named : throw NotOrdinary{};
    const int mine = t->scalar_type() == at::kHalf ? BWTA_DTYPE_FP16 : BWTA_DTYPE_BF16;
    if ((named == BWTA_DTYPE_FP16 || named == BWTA_DTYPE_BF16) && named != mine) throw NotOrdinary{};
    return given(o) ? named : mine;
}

int flag(PyObject *o, bool otherwise)
{
    if (o == nullptr) return otherwise;
    if (o != Py_True && o != Py_False) throw NotOrdinary{};
    return o == Py_True;
}

// binding._apart
int64_t rows_apart(PyObject *o, const at::Tensor *t, int64_t width)
{
    if (t && t->numel() && width > 0) {
        int64_t size = 1, i = t->dim();
        while (i > 0 && size < width) {
            --i;
            if (t->size(i) > 1 && t->stride(i) != size) throw NotOrdinary{};
            size *= t->size(i);
        }
        if (!given(o)) {
            int64_t apart = 0, step = 0;
            while (i-- > 0) {
                if (t->size(i) <= 1) continue;
                if (step && t->stride(i) != step) throw NotOrdinary{};
                if (!step) apart = t->stride(i);
                step = t->stride(i) * t->size(i);
                if (step == 0) throw NotOrdinary{};
            }
            return step ? apart : width;
        }
    }
    return given(o) ? int64(o) : width;
}

// binding._holds (in 128 bits: what does not fit 64 is the Python form's to refuse)
void holds(const at::Tensor *t, int64_t apart, int64_t rows, int64_t width, int64_t size)
{
    if (!t || rows <= 0 || width <= 0) return;
    __int128 span = t->numel() ? 1 : 0;
    if (span)
        for (int64_t i = 0; i < t->dim(); ++i) span += (__int128)(t->size(i) - 1) * t->stride(i);
    if (span * (int64_t)t->element_size() < ((__int128)(rows - 1) * apart + width) * size) throw NotOrdinary{};
}

void sequences_hold(const Cache &cache, const at::Tensor *table, int64_t ldt, const at::Tensor *lens, const at::Tensor *cu, int M, int batch, int max_new, int max_len)
{
    if (M <= 0 || batch <= 0 || max_new <= 0) return;
    holds(lens, 0, 1, batch, 4);
    holds(cu, 0, 1, (int64_t)batch + 1, 4);
    if (cache.c.block > 0) holds(table, ldt, batch, ((int64_t)max_len + cache.c.block - 1) / cache.c.block, 4);
}

int64_t blocks_apart(PyObject *o, const at::Tensor *table, int batch)
{
    if (given(o)) return int64(o);
    if (!table || table->dim() == 0) throw NotOrdinary{};
    return batch == 1 && (table->dim() == 1 || table->size(0) == 1) ? table->numel() : table->stride(0);
}

// the C call without the interpreter lock (a launch waits where the queue is full), its code turned into what the Python
// form returns or raises
template <typename F>
bool finish(F f, PyObject **result, const int *value = nullptr)
{
    int code;
    Py_BEGIN_ALLOW_THREADS
    code = f();
    Py_END_ALLOW_THREADS
    if (code != BWTA_OK) {
        PyObject *c = PyLong_FromLong(code);
        PyObject *r = c ? PyObject_CallOneArg(g_check, c) : nullptr;  // raises
        Py_XDECREF(c);
        Py_XDECREF(r);
        *result = nullptr;
        if (!PyErr_Occurred()) PyErr_SetString(PyExc_RuntimeError, "bwta call failed");
        return true;
    }
    if (value) {
        *result = PyLong_FromLong(*value);
    } else {
        Py_INCREF(Py_None);
        *result = Py_None;
    }
    return true;
}

#define BWTA_FN(fn) auto *call = (decltype(&fn))b.address

bool linear(const Bound &b, PyObject *const *v, PyObject **result)
{
    const at::Tensor *A = tensor(v[0]), *s_a = tensor(v[1]), *w = tensor(v[2]), *s_w = tensor(v[3]), *out = tensor(v[4]), *ws = tensor(v[5]);
    const int M = int32(v[6]), N = int32(v[7]), K = int32(v[8]);
    const int64_t lda = int64_or(v[9], K), ldo = int64_or(v[10], N);
    const int am = scale_mode(v[11], s_a), wm = scale_mode(v[12], s_w);
    const size_t bytes = bytes_of(v[13], ws);
    void *const pA = address(A), *const psa = address(s_a), *const pw = address(w), *const psw = address(s_w), *const po = address(out), *const pws = address(ws);
    void *const st = current_stream(v[14]);
    BWTA_FN(bwta_linear);
    return finish([&] { return call(pA, lda, psa, am, (const uint32_t *)pw, psw, wm, M, N, K, po, ldo, pws, bytes, st); }, result);
}

bool gemm(const Bound &b, PyObject *const *v, PyObject **result)
{
    const at::Tensor *mask = tensor(v[0]), *sign = tensor(v[1]), *w = tensor(v[2]), *s_a = tensor(v[3]), *s_w = tensor(v[4]), *acc = tensor(v[5]),
                     *out = tensor(v[6]), *ws = tensor(v[7]);
    const int M = int32(v[8]), N = int32(v[9]), K = int32(v[10]);
    const int64_t ldo = int64_or(v[11], N);
    const int am = scale_mode(v[12], s_a), wm = scale_mode(v[13], s_w);
    const size_t bytes = bytes_of(v[14], ws);
    void *const pm = address(mask), *const ps = address(sign), *const pw = address(w), *const psa = address(s_a), *const psw = address(s_w),
               *const pacc = address(acc), *const po = address(out), *const pws = address(ws);
    void *const st = current_stream(v[15]);
    BWTA_FN(bwta_gemm);
    return finish([&] { return call((const uint32_t *)pm, (const uint32_t *)ps, (const uint32_t *)pw, M, N, K, psa, am, psw, wm, (int32_t *)pacc, po, ldo, pws, bytes, st); }, result);
}

bool gemm_prepared(const Bound &b, PyObject *const *v, PyObject **result)
{
    const at::Tensor *prep = tensor(v[0]), *w = tensor(v[1]), *s_a = tensor(v[2]), *s_w = tensor(v[3]), *acc = tensor(v[4]), *out = tensor(v[5]);
    const int fmt = int32(v[6]), M = int32(v[7]), N = int32(v[8]), K = int32(v[9]);
    const int64_t ldo = int64_or(v[10], N);
    const int am = scale_mode(v[11], s_a), wm = scale_mode(v[12], s_w);
    const size_t bytes = bytes_of(v[13], prep);
    void *const pp = address(prep), *const pw = address(w), *const psa = address(s_a), *const psw = address(s_w), *const pacc = address(acc), *const po = address(out);
    void *const st = current_stream(v[14]);
    BWTA_FN(bwta_gemm_prepared);
    return finish([&] { return call(pp, bytes, fmt, (const uint32_t *)pw, M, N, K, psa, am, psw, wm, (int32_t *)pacc, po, ldo, st); }, result);
}

bool prepare_act(const Bound &b, PyObject *const *v, PyObject **result)
{
    const at::Tensor *A = tensor(v[0]), *s_a = tensor(v[1]), *prep = tensor(v[2]);
    const int M = int32(v[3]), K = int32(v[4]);
    const int64_t lda = int64_or(v[5], K);
    const int am = scale_mode(v[6], s_a);
    const size_t bytes = bytes_of(v[7], prep);
    void *const pA = address(A), *const psa = address(s_a), *const pp = address(prep);
    void *const st = current_stream(v[8]);
    int fmt = 0;
    BWTA_FN(bwta_prepare_act);
    return finish([&] { return call(pA, lda, psa, am, M, K, pp, bytes, &fmt, st); }, result, &fmt);
}

bool prepare_act_autoscale(const Bound &b, PyObject *const *v, PyObject **result)
{
    const at::Tensor *A = tensor(v[0]), *s_a = tensor(v[1]), *prep = tensor(v[2]);
    const int M = int32(v[3]), K = int32(v[4]);
    const int64_t lda = int64_or(v[5], K);
    const size_t bytes = bytes_of(v[6], prep);
    void *const pA = address(A), *const psa = address(s_a), *const pp = address(prep);
    void *const st = current_stream(v[7]);
    int fmt = 0;
    BWTA_FN(bwta_prepare_act_autoscale);
    return finish([&] { return call(pA, lda, M, K, psa, pp, bytes, &fmt, st); }, result, &fmt);
}

bool quantize_pack_act(const Bound &b, PyObject *const *v, PyObject **result)
{
    const at::Tensor *A = tensor(v[0]), *s_a = tensor(v[1]), *mask = tensor(v[2]), *sign = tensor(v[3]), *nnz = tensor(v[4]);
    const int M = int32(v[5]), K = int32(v[6]);
    const int64_t lda = int64_or(v[7], K);
    const int dtype = v[8] ? int32(v[8]) : BWTA_DTYPE_FP16;
    const int am = scale_mode(v[9], s_a);
    void *const pA = address(A), *const psa = address(s_a), *const pm = address(mask), *const ps = address(sign), *const pn = address(nnz);
    void *const st = current_stream(v[10]);
    BWTA_FN(bwta_quantize_pack_act);
    return finish([&] { return call(pA, dtype, lda, psa, am, M, K, (uint32_t *)pm, (uint32_t *)ps, (int32_t *)pn, st); }, result);
}

bool quantize_pack_bool(const Bound &b, PyObject *const *v, PyObject **result)
{
    const at::Tensor *A = tensor(v[0]), *s_a = tensor(v[1]), *mask = tensor(v[2]);
    const int M = int32(v[3]), K = int32(v[4]);
    const int64_t lda = int64_or(v[5], K);
    const int am = scale_mode(v[6], s_a);
    void *const pA = address(A), *const psa = address(s_a), *const pm = address(mask);
    void *const st = current_stream(v[7]);
    BWTA_FN(bwta_quantize_pack_bool);
    return finish([&] { return call(pA, lda, psa, am, M, K, (uint32_t *)pm, st); }, result);
}

bool act_scale(const Bound &b, PyObject *const *v, PyObject **result)
{
    const at::Tensor *A = tensor(v[0]), *s = tensor(v[1]);
    const int M = int32(v[2]), K = int32(v[3]);
    const int64_t lda = int64_or(v[4], K);
    void *const pA = address(A), *const ps = address(s);
    void *const st = current_stream(v[5]);
    BWTA_FN(bwta_act_scale);
    return finish([&] { return call(pA, lda, M, K, ps, st); }, result);
}

bool prepare_weights(const Bound &b, PyObject *const *v, PyObject **result)
{
    const at::Tensor *W = tensor(v[0]), *w = tensor(v[1]), *s_w = tensor(v[2]);
    const int N = int32(v[3]), K = int32(v[4]);
    const int64_t ldw = int64_or(v[5], K);
    void *const pW = address(W), *const pw = address(w), *const psw = address(s_w);
    void *const st = current_stream(v[6]);
    BWTA_FN(bwta_prepare_weights);
    return finish([&] { return call(pW, ldw, N, K, (uint32_t *)pw, psw, st); }, result);
}

int64_t row_words(int K) { return 4 * (((int64_t)K + 127) / 128); }  // bwta_plane_row_words of a positive K

bool matmul_tt(const Bound &b, PyObject *const *v, PyObject **result)
{
    const at::Tensor *ma = tensor(v[0]), *sa = tensor(v[1]), *mb = tensor(v[2]), *sb = tensor(v[3]), *s_a = tensor(v[4]), *s_b = tensor(v[5]),
                     *acc = tensor(v[6]), *out = tensor(v[7]);
    const int batch = int32(v[8]), M = int32(v[9]), N = int32(v[10]), K = int32(v[11]);
    if (M <= 0 || N <= 0 || K <= 0) throw NotOrdinary{};
    const float alpha = number(v[12], 1.0f);
    const int64_t strideA = int64_or(v[13], M * row_words(K)), strideB = int64_or(v[14], N * row_words(K)), ldo = int64_or(v[15], N);
    if (ldo < 0 || ldo > INT_MAX) throw NotOrdinary{};
    const int64_t stride_out = int64_or(v[16], M * ldo);
    const int am = scale_mode(v[17], s_a), bm = scale_mode(v[18], s_b);
    void *const pma = address(ma), *const psa = address(sa), *const pmb = address(mb), *const psb = address(sb), *const pa = address(s_a), *const pb = address(s_b),
               *const pacc = address(acc), *const po = address(out);
    void *const st = current_stream(v[19]);
    BWTA_FN(bwta_matmul_tt);
    return finish([&] { return call((const uint32_t *)pma, (const uint32_t *)psa, strideA, (const uint32_t *)pmb, (const uint32_t *)psb, strideB, batch, M, N, K, pa, am, pb, bm,
                                    alpha, (int32_t *)pacc, po, ldo, stride_out, st); }, result);
}

bool matmul_bool_prepared(const Bound &b, PyObject *const *v, PyObject **result)
{
    const at::Tensor *ma = tensor(v[0]), *prep = tensor(v[1]), *s_a = tensor(v[2]), *s_b = tensor(v[3]), *out = tensor(v[4]);
    const int fmt = int32(v[5]), batch = int32(v[6]), M = int32(v[7]), N = int32(v[8]), K = int32(v[9]);
    if (M <= 0 || N <= 0 || K <= 0) throw NotOrdinary{};
    const float alpha = number(v[10], 1.0f);
    const int64_t strideA = int64_or(v[11], M * row_words(K)), ldo = int64_or(v[12], N);
    if (ldo < 0 || ldo > INT_MAX) throw NotOrdinary{};
    const int64_t stride_out = int64_or(v[13], M * ldo);
    const int am = scale_mode(v[14], s_a), bm = scale_mode(v[15], s_b);
    const size_t bytes = bytes_of(v[16], prep);
    void *const pma = address(ma), *const pp = address(prep), *const pa = address(s_a), *const pb = address(s_b), *const po = address(out);
    void *const st = current_stream(v[17]);
    BWTA_FN(bwta_matmul_bool_prepared);
    return finish([&] { return call((const uint32_t *)pma, strideA, pp, bytes, fmt, batch, M, N, K, pa, am, pb, bm, alpha, po, ldo, stride_out, st); }, result);
}

bool head_norm_rope(const Bound &b, PyObject *const *v, PyObject **result)
{
    const Here h = here(v[21]);
    const at::Tensor *Q = h.rows(v[0]), *K = h.rows(v[1]), *first = Q ? Q : K;
    h.rows_like(v[1], first);
    const at::Tensor *wqt = h.rows_like(v[2], first), *wkt = h.rows_like(v[3], first), *Qout = h.rows_like(v[6], first), *Kout = h.rows_like(v[7], first);
    const int M = int32(v[8]), heads = int32(v[9]), kv = int32(v[10]), dim = int32(v[11]), rot = given(v[12]) ? int32(v[12]) : dim;
    const float eps = number(v[13], 1e-6f);
    const int norm = flag(v[14], true), interleaved = flag(v[15], false);
    const int64_t wq = (int64_t)heads * dim, wk = (int64_t)kv * dim;
    const int64_t ldq = rows_apart(v[16], Q, wq), ldk = rows_apart(v[17], K, wk), ldqo = rows_apart(v[18], Qout, wq), ldko = rows_apart(v[19], Kout, wk);
    const int dtype = head_dtype(v[20], first);
    void *const pq = address(Q), *const pk = address(K), *const pwq = address(wqt), *const pwk = address(wkt), *const qo = address(Qout), *const ko = address(Kout);
    const at::Tensor *const positions = h.ints(v[4]), *const inv_freq = h.floats(v[5]);
    holds(Q, ldq, M, wq, 2), holds(K, ldk, M, wk, 2), holds(Qout, ldqo, M, wq, 2), holds(Kout, ldko, M, wk, 2);
    if (M > 0) {
        holds(wqt, 0, norm && heads > 0, dim, 2), holds(wkt, 0, norm && kv > 0, dim, 2);
        holds(positions, 0, rot > 0, M, 4), holds(inv_freq, 0, 1, rot / 2, 4);
    }
    const int32_t *const pos = (const int32_t *)address(positions);
    const float *const freq = (const float *)address(inv_freq);
    BWTA_FN(bwta_head_norm_rope);
    return finish([&] { return call(pq, ldq, heads, pwq, pk, ldk, kv, pwk, dtype, M, dim, norm, eps, pos, freq, rot, interleaved, qo, ldqo, ko, ldko, h.stream); }, result);
}

template <typename F>
bool cache_rows(F *call, PyObject *const *v, PyObject **result)
{
    const Here h = here(v[14]);
    const Cache cache = cache_of(v[0], h);
    const at::Tensor *K = h.rows(v[1]), *V = h.rows_like(v[2], K), *table = h.table(v[3]);
    const int M = int32(v[6]), batch = int32(v[7]), max_new = int32(v[8]), max_len = int32(v[9]);
    const int64_t width = (int64_t)cache.c.kv_heads * cache.c.dim, ldk = rows_apart(v[10], K, width), ldv = rows_apart(v[11], V, width);
    const int64_t ldt = blocks_apart(v[12], table, batch);
    const int dtype = head_dtype(v[13], K);
    const at::Tensor *const lt = h.ints(v[4]), *const ct = h.ints(v[5]);
    holds(K, ldk, M, width, 2), holds(V, ldv, M, width, 2);
    sequences_hold(cache, table, ldt, lt, ct, M, batch, max_new, max_len);
    void *const pk = address(K), *const pv = address(V), *const pt = address(table);
    const int32_t *const lens = (const int32_t *)address(lt), *const cu = (const int32_t *)address(ct);
    return finish([&] { return call(&cache.c, pk, ldk, pv, ldv, dtype, (const int32_t *)pt, ldt, lens, cu, batch, M, max_new, max_len, h.stream); }, result);
}

bool cache_write(const Bound &b, PyObject *const *v, PyObject **result)
{
    BWTA_FN(bwta_cache_write);
    return cache_rows(call, v, result);
}

bool cache_read(const Bound &b, PyObject *const *v, PyObject **result)
{
    BWTA_FN(bwta_cache_read);
    return cache_rows(call, v, result);
}

bool cache_attention(const Bound &b, PyObject *const *v, PyObject **result)
{
    const Here h = here(v[21]);
    const Cache cache = cache_of(v[0], h);
    const at::Tensor *Q = h.rows(v[1]), *out = h.rows_like(v[2], Q), *table = h.table(v[4]), *ws = h.tensor(v[7]);
    const int M = int32(v[8]), batch = int32(v[9]), max_new = int32(v[10]), max_len = int32(v[11]), heads = int32(v[12]);
    if (!v[13]) throw NotOrdinary{};
    const float alpha = number(v[13], 0.0f);
    const int causal = flag(v[14], true), window = v[15] ? int32(v[15]) : 0;
    const int64_t width = (int64_t)heads * cache.c.dim, ldq = rows_apart(v[16], Q, width), ldo = rows_apart(v[17], out, width);
    const int64_t ldt = blocks_apart(v[18], table, batch);
    const int dtype = head_dtype(v[19], Q);
    const size_t bytes = bytes_of(v[20], ws);
    if (ws && (!ws->is_contiguous() || bytes > ws->nbytes())) throw NotOrdinary{};  // binding._room
    void *const pq = address(Q), *const po = address(out), *const pt = address(table), *const pws = address(ws);
    const at::Tensor *const logs = h.floats(v[3]), *const lt = h.ints(v[5]), *const ct = h.ints(v[6]);
    holds(Q, ldq, M, width, 2), holds(out, ldo, M, width, 2), holds(logs, heads, M, heads, 4);
    sequences_hold(cache, table, ldt, lt, ct, M, batch, max_new, max_len);
    float *const lse = (float *)address(logs);
    const int32_t *const lens = (const int32_t *)address(lt), *const cu = (const int32_t *)address(ct);
    BWTA_FN(bwta_cache_attention);
    return finish([&] { return call(&cache.c, pq, ldq, po, ldo, dtype, lse, (const int32_t *)pt, ldt, lens, cu, batch, M, max_new, max_len,
                                    heads, alpha, causal, window, pws, bytes, h.stream); }, result);
}

const Spec kSpecs[] = {
    {"bwta_linear", 6, {"A", "s_a", "wsign", "s_w", "out", "workspace", "M", "N", "K", "lda", "ldo", "a_scale_mode", "w_scale_mode", "workspace_bytes", "stream"}, linear},
    {"bwta_gemm", 8, {"mask", "sign", "wsign", "s_a", "s_w", "acc", "out", "workspace", "M", "N", "K", "ldo", "a_scale_mode", "w_scale_mode", "workspace_bytes", "stream"}, gemm},
    {"bwta_gemm_prepared", 6, {"prepared", "wsign", "s_a", "s_w", "acc", "out", "fmt", "M", "N", "K", "ldo", "a_scale_mode", "w_scale_mode", "prepared_bytes", "stream"}, gemm_prepared},
    {"bwta_prepare_act", 3, {"A", "s_a", "prepared", "M", "K", "lda", "a_scale_mode", "prepared_bytes", "stream"}, prepare_act},
    {"bwta_prepare_act_autoscale", 3, {"A", "s_a", "prepared", "M", "K", "lda", "prepared_bytes", "stream"}, prepare_act_autoscale},
    {"bwta_quantize_pack_act", 5, {"A", "s_a", "mask", "sign", "nnz", "M", "K", "lda", "a_dtype", "scale_mode", "stream"}, quantize_pack_act},
    {"bwta_quantize_pack_bool", 3, {"A", "s_a", "mask", "M", "K", "lda", "scale_mode", "stream"}, quantize_pack_bool},
    {"bwta_act_scale", 2, {"A", "s", "M", "K", "lda", "stream"}, act_scale},
    {"bwta_prepare_weights", 3, {"W", "wsign", "s_w", "N", "K", "ldw", "stream"}, prepare_weights},
    {"bwta_matmul_tt", 8, {"maskA", "signA", "maskB", "signB", "s_a", "s_b", "acc", "out", "batch", "M", "N", "K", "alpha", "strideA", "strideB", "ldo", "stride_out", "a_scale_mode", "b_scale_mode", "stream"}, matmul_tt},
    {"bwta_matmul_bool_prepared", 5, {"maskA", "preparedB", "s_a", "s_b", "out", "fmt", "batch", "M", "N", "K", "alpha", "strideA", "ldo", "stride_out", "a_scale_mode", "b_scale_mode", "prepared_bytes", "stream"}, matmul_bool_prepared},
};

const Spec kHeadSpecs[] = {
    {"bwta_head_norm_rope", 8, {"Q", "K", "wq", "wk", "positions", "inv_freq", "Qout", "Kout", "M", "heads", "kv_heads", "dim", "rot_dim", "eps", "norm", "interleaved", "ldq", "ldk", "ldqo", "ldko", "dtype", "stream"}, head_norm_rope},
    {"bwta_cache_write", 6, {"cache", "K", "V", "table", "lens", "cu", "M", "batch", "max_new", "max_len", "ldk", "ldv", "ldt", "dtype", "stream"}, cache_write},
    {"bwta_cache_read", 6, {"cache", "K", "V", "table", "lens", "cu", "M", "batch", "max_new", "max_len", "ldk", "ldv", "ldt", "dtype", "stream"}, cache_read},
    {"bwta_cache_attention", 8, {"cache", "Q", "out", "lse", "table", "lens", "cu", "workspace", "M", "batch", "max_new", "max_len", "heads", "alpha", "causal", "window", "ldq", "ldo", "ldt", "dtype", "workspace_bytes", "stream"}, cache_attention},
};

constexpr int kSpecCount = sizeof kSpecs / sizeof kSpecs[0], kHeadSpecCount = sizeof kHeadSpecs / sizeof kHeadSpecs[0];

// positional parameters that may be left out
bool may_be_left_out(const char *name) { return strcmp(name, "nnz") == 0 || strcmp(name, "cu") == 0 || strcmp(name, "workspace") == 0; }

// the arguments to their parameters' slots; false where the Python form would raise or this table does not know better
bool place(const Bound &b, PyObject *const *args, Py_ssize_t nargs, PyObject *kwnames, PyObject **v)
{
    if (nargs > b.spec->positional) return false;
    for (int i = 0; i < b.count; ++i) v[i] = i < nargs ? args[i] : nullptr;
    const Py_ssize_t nkw = kwnames ? PyTuple_GET_SIZE(kwnames) : 0;
    int at = (int)nargs;
    for (Py_ssize_t k = 0; k < nkw; ++k) {
        PyObject *name = PyTuple_GET_ITEM(kwnames, k);
        int i = 0;
        for (; i < b.count; ++i, at = at + 1 < b.count ? at + 1 : 0)  // names come in order as a rule, and interned
            if (b.names[at] == name) break;
        if (i == b.count || v[at]) return false;
        v[at] = args[nargs + k];
    }
    // the tensors all have to be given, except some (bwta_linear's and bwta_gemm's workspace are not among them)
    for (int i = 0; i < b.spec->positional; ++i)
        if (!v[i] && (i < b.spec->positional - 2 || !may_be_left_out(b.spec->params[i]) || (strcmp(b.spec->params[i], "workspace") == 0 && b.spec->marshal != cache_attention))) return false;
    return true;
}

PyObject *bound_call(PyObject *self, PyObject *const *args, size_t nargsf, PyObject *kwnames)
{
    const Bound &b = *(const Bound *)self;
    PyObject *v[kMaxParams], *result = nullptr;
    if (place(b, args, PyVectorcall_NARGS(nargsf), kwnames, v)) {
        try {
            if (b.spec->marshal(b, v, &result)) return result;
        } catch (const std::bad_alloc &) {
            return PyErr_NoMemory();
        } catch (...) {  // not the ordinary form, or a tensor without an address: the Python form's business
            PyErr_Clear();
        }
    }
    return PyObject_Vectorcall(b.fallback, args, nargsf & ~PY_VECTORCALL_ARGUMENTS_OFFSET, kwnames);
}

void bound_dealloc(PyObject *self)
{
    Bound *b = (Bound *)self;
    if (b->weak) PyObject_ClearWeakRefs(self);
    for (int i = 0; i < b->count; ++i) Py_XDECREF(b->names[i]);
    Py_XDECREF(b->fallback);
    Py_TYPE(self)->tp_free(self);
}

// Everything a program may do with a Python function besides calling it: its attributes, __class__ among them, are those
// of the Python form and are set there, it binds as a method, and is pickled and copied by its name.
PyObject *bound_getattro(PyObject *self, PyObject *name)
{
    if (PyUnicode_Check(name)) {
        const char *s = PyUnicode_AsUTF8(name);
        if (!s) return nullptr;
        if (strcmp(s, "__reduce_ex__") == 0 || strcmp(s, "__reduce__") == 0 || strcmp(s, "__get__") == 0) return PyObject_GenericGetAttr(self, name);
    }
    return PyObject_GetAttr(((Bound *)self)->fallback, name);
}

int bound_setattro(PyObject *self, PyObject *name, PyObject *value) { return PyObject_SetAttr(((Bound *)self)->fallback, name, value); }

PyObject *bound_descr_get(PyObject *self, PyObject *object, PyObject *)
{
    if (object == nullptr || object == Py_None) {
        Py_INCREF(self);
        return self;
    }
    return PyMethod_New(self, object);
}

PyObject *bound_repr(PyObject *self) { return PyObject_Repr(((Bound *)self)->fallback); }

PyObject *bound_reduce(PyObject *self, PyObject *) { return PyObject_GetAttrString(((Bound *)self)->fallback, "__qualname__"); }

PyMethodDef kBoundMethods[] = {{"__reduce_ex__", bound_reduce, METH_O, nullptr}, {"__reduce__", bound_reduce, METH_NOARGS, nullptr}, {nullptr, nullptr, 0, nullptr}};

PyTypeObject BoundType = {PyVarObject_HEAD_INIT(nullptr, 0)};

PyObject *bind(PyObject *, PyObject *args)
{
    const char *name;
    PyObject *addr, *fallback;
    if (!PyArg_ParseTuple(args, "sOO", &name, &addr, &fallback)) return nullptr;
    for (int n = 0; n < kSpecCount + kHeadSpecCount; ++n) {
        const Spec &s = n < kSpecCount ? kSpecs[n] : kHeadSpecs[n - kSpecCount];
        if (strcmp(s.name, name) != 0) continue;
        void *const address = PyLong_AsVoidPtr(addr);
        if (PyErr_Occurred()) return nullptr;
        Bound *b = PyObject_New(Bound, &BoundType);
        if (!b) return nullptr;
        b->call = bound_call, b->spec = &s, b->count = 0, b->address = address, b->fallback = fallback, b->weak = nullptr;
        Py_INCREF(fallback);
        for (; s.params[b->count]; ++b->count) {
            b->names[b->count] = PyUnicode_InternFromString(s.params[b->count]);
            if (!b->names[b->count]) {
                Py_DECREF(b);
                return nullptr;
            }
        }
        return (PyObject *)b;
    }
    PyErr_Format(PyExc_KeyError, "%s", name);
    return nullptr;
}

PyObject *setup(PyObject *, PyObject *args)  // (check, raw_stream, device, cache type)
{
    PyObject *c, *r, *d, *t;
    if (!PyArg_ParseTuple(args, "OOOO!", &c, &r, &d, &PyType_Type, &t)) return nullptr;
    Py_INCREF(c), Py_INCREF(r), Py_INCREF(d), Py_INCREF(t);
    Py_XDECREF(g_check), Py_XDECREF(g_raw_stream), Py_XDECREF(g_device), Py_XDECREF(g_cache);
    g_check = c, g_raw_stream = r, g_device = d, g_cache = (PyTypeObject *)t;
    Py_RETURN_NONE;
}

PyObject *table_of(const Spec *specs, int count)  // {name: (positional parameters, all parameters)}
{
    PyObject *out = PyDict_New();
    for (int n = 0; n < count; ++n) {
        const Spec &s = specs[n];
        PyObject *l = out ? PyList_New(0) : nullptr;
        if (!l) break;
        for (int i = 0; s.params[i]; ++i) {
            PyObject *p = PyUnicode_FromString(s.params[i]);
            if (p) PyList_Append(l, p);
            Py_XDECREF(p);
        }
        PyObject *t = Py_BuildValue("(iN)", s.positional, l);
        if (t) PyDict_SetItemString(out, s.name, t);
        Py_XDECREF(t);
    }
    if (PyErr_Occurred()) {
        Py_XDECREF(out);
        return nullptr;
    }
    return out;
}

PyObject *parameters(PyObject *, PyObject *) { return table_of(kSpecs, kSpecCount); }
PyObject *head_parameters(PyObject *, PyObject *) { return table_of(kHeadSpecs, kHeadSpecCount); }

#ifndef BWTA_IDENTITY
#define BWTA_IDENTITY "unknown"
#endif
PyObject *identity(PyObject *, PyObject *) { return PyUnicode_FromString(BWTA_IDENTITY); }

PyMethodDef kMethods[] = {{"identity", identity, METH_NOARGS, "identity() -> \"<digest of the sources> <torch version> <Python version>\""},
                          {"bind", bind, METH_VARARGS, "bind(name, address, fallback) -> function"},
                          {"setup", setup, METH_VARARGS, "setup(check, raw_stream, device, cache type)"},
                          {"head_parameters", head_parameters, METH_NOARGS, "as parameters(), of the operators on heads"},
                          {"parameters", parameters, METH_NOARGS, "{name: (positional parameters, all parameters)}"},
                          {nullptr, nullptr, 0, nullptr}};
PyModuleDef kModule = {PyModuleDef_HEAD_INIT, "_bwta_native", "Marshalling of the per-layer calls.", -1, kMethods};

}  // namespace

PyMODINIT_FUNC PyInit__bwta_native(void)
{
#define BWTA_STR2(x) #x
#define BWTA_STR(x) BWTA_STR2(x)
    constexpr char built_for[] = BWTA_STR(PY_MAJOR_VERSION) "." BWTA_STR(PY_MINOR_VERSION) ".";
    if (strncmp(Py_GetVersion(), built_for, sizeof built_for - 1) != 0) {
        PyErr_SetString(PyExc_ImportError, "built for another version of Python");
        return nullptr;
    }
    BoundType.tp_name = "_bwta_native.function";
    BoundType.tp_basicsize = sizeof(Bound);
    BoundType.tp_dealloc = bound_dealloc;
    BoundType.tp_call = PyVectorcall_Call;
    BoundType.tp_vectorcall_offset = offsetof(Bound, call);
    BoundType.tp_getattro = bound_getattro;
    BoundType.tp_setattro = bound_setattro;
    BoundType.tp_descr_get = bound_descr_get;
    BoundType.tp_repr = bound_repr;
    BoundType.tp_methods = kBoundMethods;
    BoundType.tp_weaklistoffset = offsetof(Bound, weak);
    BoundType.tp_flags = Py_TPFLAGS_DEFAULT | Py_TPFLAGS_HAVE_VECTORCALL;
    if (PyType_Ready(&BoundType) < 0) return nullptr;
    return PyModule_Create(&kModule);
}
