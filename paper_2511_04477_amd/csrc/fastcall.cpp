// What a device call of binding.py does before the library's function, without the interpreter: the tensors' types and sizes, the current
// stream, the call.  A Python extension module; binding.py has the same in Python and is what decides.
//
// What bounds an eager call: the host.  Of 4.65 us for spqt_gather and 6.2 for spqt_gemv 2.7 were the launch inside the runtime; five tensors
// with five attribute reads each, the size formulas, ctypes and its structure were the rest.  Here they take 0.3 to 0.6 (a gather and a GEMV,
// 512 x 1024: 11.0 us in Python, 6.8 here; 4 of each on 11001 x 4224, with the GPU's share, 45.7 / 34.3).
//
// Every function returns the library's status, or None where anything is other than what it knows for certain - a tensor that is not plainly a
// dense one of the type asked for, another size, an int or a threshold of another type, a stream given, a torch-function mode, which the Python code's reads of
// the tensors would reach - and then has done nothing.  The caller goes on with the Python code, which accepts or refuses as it always did.
#include <Python.h>

#include <ATen/PythonTorchFunctionTLS.h>
#include <ATen/core/TensorBase.h>
#include <c10/hip/HIPStream.h>
#include <torch/csrc/autograd/python_variable.h>

#include <cmath>
#include <cstdint>

#include "spqt.h"
#include "spqt_colblock.h"
#include "spqt_kv.h"

namespace {

struct NotPlain {};      // anything that the Python code is to look at

// A dense tensor on the GPU, in memory order, of this type.
const at::Tensor &tensor(PyObject *o, at::ScalarType type) {
    if (!THPVariable_CheckExact(o)) throw NotPlain();
    const at::Tensor &t = THPVariable_Unpack(o);
    const c10::TensorImpl *impl = t.unsafeGetTensorImpl();
    if (!t.defined() || impl->is_python_dispatch() || !impl->has_storage() || t.layout() != at::kStrided || !t.is_cuda() || t.scalar_type() != type ||
        !t.is_contiguous())
        throw NotPlain();
    return t;
}
int64_t whole(PyObject *o) {
    if (!PyLong_CheckExact(o)) throw NotPlain();
    int overflow = 0;
    const long long v = PyLong_AsLongLongAndOverflow(o, &overflow);
    if (overflow) throw NotPlain();
    return v;
}
int small(PyObject *o) {
    const int64_t v = whole(o);
    if (v < -(1 << 30) || v > (1 << 30)) throw NotPlain();
    return (int)v;
}
float threshold(PyObject *o) {
    if (!PyFloat_CheckExact(o)) throw NotPlain();
    return (float)PyFloat_AS_DOUBLE(o);
}
void *current_stream(PyObject *o) {
    if (o != Py_None) throw NotPlain();
    return c10::hip::getCurrentHIPStream().stream();
}
template <class F>
F function(PyObject *o) {
    void *p = PyLong_AsVoidPtr(o);
    if (!p) throw NotPlain();
    return reinterpret_cast<F>(p);
}

// The packed matrix: chunks of `chunk` bytes for `high` x `columns` weights.
void *packed_matrix(PyObject *o, int64_t M, int64_t K, int64_t high, int64_t columns, int64_t chunk) {
    const at::Tensor &t = tensor(o, at::kByte);
    if (M <= 0 || M > 1 << 24 || K <= 0 || K > 1 << 24 || K % SPQT_GROUP != 0 || (columns != SPQT_GROUP && columns != SPQT_GROUP / 2)) throw NotPlain();
    if (t.numel() < (M + high - 1) / high * (K / columns) * chunk) throw NotPlain();
    return t.data_ptr();
}

struct Output {
    void *p;
    int64_t n;
    int flags;
};
Output output(PyObject *o) {
    const bool half = THPVariable_CheckExact(o) && THPVariable_Unpack(o).scalar_type() == at::kHalf;
    const at::Tensor &t = tensor(o, half ? at::kHalf : at::kFloat);
    return {t.data_ptr(), t.numel(), half ? SPQT_CFG_Y_FP16 : 0};
}
struct Space {
    void *p = nullptr;
    size_t n = 0;
};
Space workspace(PyObject *o) {
    if (o == Py_None) return {};
    const at::Tensor &t = tensor(o, at::kByte);
    return {t.data_ptr(), (size_t)t.numel()};
}
struct List {
    const int32_t *idx = nullptr, *count = nullptr;
};
List list(PyObject *idx, PyObject *count) {
    if (idx == Py_None) return {};
    return {(const int32_t *)tensor(idx, at::kInt).data_ptr(), (const int32_t *)tensor(count, at::kInt).data_ptr()};
}
// x[K] or x[batch][K]
struct Rows {
    void *p;
    int batch;
    int64_t K;
};
Rows rows(PyObject *o) {
    const at::Tensor &t = tensor(o, at::kHalf);
    if (t.dim() != 1 && t.dim() != 2) throw NotPlain();
    const int64_t batch = t.dim() == 1 ? 1 : t.size(0);
    if (batch < 1 || batch > SPQT_MAX_BATCH) throw NotPlain();
    return {t.data_ptr(), (int)batch, t.size(t.dim() - 1)};
}

template <class Body>
PyObject *guarded(Py_ssize_t given, Py_ssize_t expected, Body body) {
    if (given != expected) {
        PyErr_SetString(PyExc_TypeError, "wrong number of arguments");
        return nullptr;
    }
    try {
        if (at::impl::torch_function_mode_enabled()) Py_RETURN_NONE;
        return PyLong_FromLong(body());
    } catch (...) {                       // NotPlain, and whatever torch throws at a tensor without memory
        PyErr_Clear();
        Py_RETURN_NONE;
    }
}
// The library's function, with the interpreter free for other threads as ctypes leaves it.
template <class F, class... A>
int call(F f, A... a) {
    PyThreadState *held = PyEval_SaveThread();
    const int rc = f(a...);
    PyEval_RestoreThread(held);
    return rc;
}

// gather(function, x, threshold, idx_out, count_out, stream)
PyObject *gather(PyObject *, PyObject *const *a, Py_ssize_t n) {
    return guarded(n, 6, [&]() {
        const Rows x = rows(a[1]);
        const at::Tensor &idx = tensor(a[3], at::kInt), &count = tensor(a[4], at::kInt);
        if (idx.numel() < x.K || count.numel() < 1) throw NotPlain();
        return call(function<decltype(&spqt_gather)>(a[0]), x.p, x.K, x.batch, threshold(a[2]), (int32_t *)idx.data_ptr(), (int32_t *)count.data_ptr(),
                    current_stream(a[5]));
    });
}
// gather_rows(function, x, threshold, idx_out, count_out, x_masked_out, stream)
PyObject *gather_rows(PyObject *, PyObject *const *a, Py_ssize_t n) {
    return guarded(n, 7, [&]() {
        const Rows x = rows(a[1]);
        const at::Tensor &idx = tensor(a[3], at::kInt), &count = tensor(a[4], at::kInt), &masked = tensor(a[5], at::kHalf);
        if (idx.numel() < x.K || count.numel() < 1 || masked.numel() != x.batch * x.K) throw NotPlain();
        return call(function<decltype(&spqt_gather_rows)>(a[0]), x.p, x.K, x.batch, threshold(a[2]), (int32_t *)idx.data_ptr(),
                    (int32_t *)count.data_ptr(), masked.data_ptr(), current_stream(a[6]));
    });
}
// The launch configuration of a call: splits and waves, and the flags with the output's type.
spqt_launch_cfg config(PyObject *splits, PyObject *waves, int flags) {
    spqt_launch_cfg c;
    c.splits = small(splits);
    c.waves = small(waves);
    c.flags = flags;
    return c;
}
// gemv(function of spqt_gemv_ex's type, packed, M, K, x, idx, count, y, workspace, stream, group, splits, waves, flags)
PyObject *gemv(PyObject *, PyObject *const *a, Py_ssize_t n) {
    return guarded(n, 14, [&]() {
        const int64_t M = whole(a[2]), K = whole(a[3]), group = whole(a[10]);
        void *packed = packed_matrix(a[1], M, K, SPQT_TILE_ROWS, group, 2 * SPQT_TILE_ROWS + 128 * group);
        const Rows x = rows(a[4]);
        const Output y = output(a[7]);
        if (x.K != K || y.n != x.batch * M) throw NotPlain();
        const List l = list(a[5], a[6]);
        const Space ws = workspace(a[8]);
        const spqt_launch_cfg cfg = config(a[11], a[12], small(a[13]) | y.flags);
        return call(function<decltype(&spqt_gemv_ex)>(a[0]), packed, M, K, (int)group, x.p, x.batch, l.idx, l.count, y.p, ws.p, ws.n,
                    current_stream(a[9]), &cfg);
    });
}

// gemv_fused(function, packed, M, K, x, threshold, y, workspace, stream, group, splits, waves, flags)
PyObject *gemv_fused(PyObject *, PyObject *const *a, Py_ssize_t n) {
    return guarded(n, 13, [&]() {
        const int64_t M = whole(a[2]), K = whole(a[3]), group = whole(a[9]);
        void *packed = packed_matrix(a[1], M, K, SPQT_TILE_ROWS, group, 2 * SPQT_TILE_ROWS + 128 * group);
        const at::Tensor &x = tensor(a[4], at::kHalf);
        const Output y = output(a[6]);
        if (x.numel() != K || y.n != M) throw NotPlain();
        const Space ws = workspace(a[7]);
        const spqt_launch_cfg cfg = config(a[10], a[11], small(a[12]) | y.flags);
        return call(function<decltype(&spqt_gemv_fused)>(a[0]), packed, M, K, (int)group, x.data_ptr(), threshold(a[5]), y.p, ws.p, ws.n,
                    current_stream(a[8]), &cfg);
    });
}
// gemv_fused_rows(function, packed, M, K, x, threshold, own_sets, y, workspace, stream, group, splits, waves)
PyObject *gemv_fused_rows(PyObject *, PyObject *const *a, Py_ssize_t n) {
    return guarded(n, 13, [&]() {
        const int64_t M = whole(a[2]), K = whole(a[3]), group = whole(a[10]);
        void *packed = packed_matrix(a[1], M, K, SPQT_TILE_ROWS, group, 2 * SPQT_TILE_ROWS + 128 * group);
        const Rows x = rows(a[4]);
        const Output y = output(a[7]);
        if (x.K != K || y.n != x.batch * M || !PyBool_Check(a[6])) throw NotPlain();
        const Space ws = workspace(a[8]);
        const spqt_launch_cfg cfg = config(a[11], a[12], y.flags);
        return call(function<decltype(&spqt_gemv_fused_rows)>(a[0]), packed, M, K, (int)group, x.p, x.batch, threshold(a[5]), (int)(a[6] == Py_True), y.p,
                    ws.p, ws.n, current_stream(a[9]), &cfg);
    });
}
// The column-block layouts, whose rows per block-row and bytes per chunk come with the call.
// cb_gemv(function, packed, M, K, x, idx, count, y, workspace, stream, splits, waves, high, chunk)
PyObject *cb_gemv(PyObject *, PyObject *const *a, Py_ssize_t n) {
    return guarded(n, 14, [&]() {
        const int64_t M = whole(a[2]), K = whole(a[3]);
        void *packed = packed_matrix(a[1], M, K, whole(a[12]), SPQT_GROUP, whole(a[13]));
        const Rows x = rows(a[4]);
        const Output y = output(a[7]);
        if (x.K != K || y.n != x.batch * M) throw NotPlain();
        const List l = list(a[5], a[6]);
        const Space ws = workspace(a[8]);
        const spqt_launch_cfg cfg = config(a[10], a[11], y.flags);
        return call(function<decltype(&spqt_cb_gemv)>(a[0]), packed, M, K, x.p, x.batch, l.idx, l.count, y.p, ws.p, ws.n, current_stream(a[9]), &cfg);
    });
}
// cb_gemv_one(the same): the functions that take one activation row
PyObject *cb_gemv_one(PyObject *, PyObject *const *a, Py_ssize_t n) {
    return guarded(n, 14, [&]() {
        const int64_t M = whole(a[2]), K = whole(a[3]);
        void *packed = packed_matrix(a[1], M, K, whole(a[12]), SPQT_GROUP, whole(a[13]));
        const at::Tensor &x = tensor(a[4], at::kHalf);
        const Output y = output(a[7]);
        if (x.numel() != K || y.n != M) throw NotPlain();
        const List l = list(a[5], a[6]);
        const Space ws = workspace(a[8]);
        const spqt_launch_cfg cfg = config(a[10], a[11], y.flags);
        return call(function<decltype(&spqt_cb8_gemv)>(a[0]), packed, M, K, x.data_ptr(), l.idx, l.count, y.p, ws.p, ws.n, current_stream(a[9]), &cfg);
    });
}
// cb_gemv_fused(function, packed, M, K, x, threshold, y, workspace, stream, splits, waves, high, chunk)
PyObject *cb_gemv_fused(PyObject *, PyObject *const *a, Py_ssize_t n) {
    return guarded(n, 13, [&]() {
        const int64_t M = whole(a[2]), K = whole(a[3]);
        void *packed = packed_matrix(a[1], M, K, whole(a[11]), SPQT_GROUP, whole(a[12]));
        const at::Tensor &x = tensor(a[4], at::kHalf);
        const Output y = output(a[6]);
        if (x.numel() != K || y.n != M) throw NotPlain();
        const Space ws = workspace(a[7]);
        const spqt_launch_cfg cfg = config(a[9], a[10], y.flags);
        return call(function<decltype(&spqt_cb_gemv_fused)>(a[0]), packed, M, K, x.data_ptr(), threshold(a[5]), y.p, ws.p, ws.n, current_stream(a[8]),
                    &cfg);
    });
}

// The key/value cache (kv.py). A cache's tensors: on one GPU, dense, of the shapes that the codes and the table ask for.
struct KvTensors {
    spqt_kv_cache c;
    c10::Device device;
};
const at::Tensor &kv_tensor(PyObject *o, at::ScalarType type, c10::Device device, c10::IntArrayRef shape) {
    const at::Tensor &t = tensor(o, type);
    if (t.device() != device || t.sizes() != shape) throw NotPlain();
    return t;
}
KvTensors kv_cache(PyObject *codes, PyObject *scales, PyObject *table, PyObject *lengths, PyObject *tail, PyObject *weights, at::ScalarType type) {
    const at::Tensor &k = tensor(codes, at::kByte), &b = tensor(table, at::kInt);
    if (type != at::kHalf && type != at::kBFloat16) throw NotPlain();
    if (k.dim() != 5 || k.size(2) != 2 || k.size(3) != SPQT_KV_BLOCK || b.dim() != 2 || b.device() != k.device()) throw NotPlain();
    const int64_t pages = k.size(0), heads = k.size(1), dim = k.size(4), sequences = b.size(0), blocks = b.size(1);
    if (heads > 1 << 20 || dim > 1 << 20 || sequences > 1 << 20 || blocks > 1 << 30) throw NotPlain();
    KvTensors r = {{}, k.device()};
    r.c.codes = k.data_ptr();
    r.c.scales = (float *)kv_tensor(scales, at::kFloat, r.device, {pages, heads, 2}).data_ptr();
    r.c.tail = tail == Py_None ? nullptr : kv_tensor(tail, type, r.device, {sequences, heads, 2, SPQT_KV_BLOCK, dim}).data_ptr();
    r.c.weights = weights == Py_None ? nullptr : (float *)kv_tensor(weights, at::kFloat, r.device, {pages, heads, SPQT_KV_BLOCK}).data_ptr();
    r.c.table = (const int32_t *)b.data_ptr();
    r.c.lengths = (const int32_t *)kv_tensor(lengths, at::kInt, r.device, {sequences}).data_ptr();
    r.c.pages = pages;
    r.c.sequences = (int)sequences;
    r.c.max_blocks = (int)blocks;
    r.c.kv_heads = (int)heads;
    r.c.head_dim = (int)dim;
    r.c.type = type == at::kBFloat16 ? SPQT_KV_BF16 : SPQT_KV_FP16;
    return r;
}
// A 16-bit tensor whose last dimension is dense; heads 0: any number of them.
struct KvRows {
    spqt_kv_rows r;
    int64_t rows, heads;
};
at::ScalarType kv_type(PyObject *o) {
    if (!THPVariable_CheckExact(o) || !THPVariable_Unpack(o).defined()) throw NotPlain();
    return THPVariable_Unpack(o).scalar_type();
}
KvRows kv_rows(PyObject *o, at::ScalarType type, const KvTensors &k, int64_t heads) {
    if (!THPVariable_CheckExact(o)) throw NotPlain();
    const at::Tensor &t = THPVariable_Unpack(o);
    const c10::TensorImpl *impl = t.unsafeGetTensorImpl();
    if (!t.defined() || impl->is_python_dispatch() || !impl->has_storage() || t.layout() != at::kStrided || !t.is_cuda() || t.scalar_type() != type ||
        t.device() != k.device || t.dim() != 4)
        throw NotPlain();
    if (t.size(0) != k.c.sequences || t.size(3) != k.c.head_dim || t.stride(3) != 1 || (heads && t.size(2) != heads)) throw NotPlain();
    if (t.size(1) > 1 << 30 || t.size(2) > 1 << 30) throw NotPlain();
    auto stride = [&](int d) { return t.size(d) > 1 ? t.stride(d) : 0; };
    return {{t.data_ptr(), stride(0), stride(1), stride(2)}, t.size(1), t.size(2)};
}
const int32_t *kv_counts(PyObject *o, const KvTensors &k) {
    return o == Py_None ? nullptr : (const int32_t *)kv_tensor(o, at::kInt, k.device, {k.c.sequences}).data_ptr();
}
// kv_append(function, codes, scales, tail, table, lengths, k, v, counts, weights, stream)
PyObject *kv_append(PyObject *, PyObject *const *a, Py_ssize_t n) {
    return guarded(n, 11, [&]() {
        const at::ScalarType type = kv_type(a[6]);
        if (a[3] == Py_None) throw NotPlain();
        const KvTensors c = kv_cache(a[1], a[2], a[4], a[5], a[3], a[9], type);
        const KvRows k = kv_rows(a[6], type, c, c.c.kv_heads), v = kv_rows(a[7], type, c, c.c.kv_heads);
        if (k.rows != v.rows) throw NotPlain();
        return call(function<decltype(&spqt_kv_append)>(a[0]), &c.c, &k.r, &v.r, (int)k.rows, kv_counts(a[8], c), current_stream(a[10]));
    });
}
// kv_read(function, codes, scales, table, lengths, k_out, v_out, counts, stream)
PyObject *kv_read(PyObject *, PyObject *const *a, Py_ssize_t n) {
    return guarded(n, 9, [&]() {
        const at::ScalarType type = kv_type(a[5]);
        const KvTensors c = kv_cache(a[1], a[2], a[3], a[4], Py_None, Py_None, type);
        const KvRows k = kv_rows(a[5], type, c, c.c.kv_heads), v = kv_rows(a[6], type, c, c.c.kv_heads);
        if (k.rows != v.rows) throw NotPlain();
        return call(function<decltype(&spqt_kv_read)>(a[0]), &c.c, &k.r, &v.r, (int)k.rows, kv_counts(a[7], c), current_stream(a[8]));
    });
}
// kv_attention(function, codes, scales, table, lengths, q, out, workspace, scale, counts, window, lse, weights, decay, stream)
PyObject *kv_attention(PyObject *, PyObject *const *a, Py_ssize_t n) {
    return guarded(n, 15, [&]() {
        const at::ScalarType type = kv_type(a[5]);
        const KvTensors c = kv_cache(a[1], a[2], a[3], a[4], Py_None, a[12], type);
        const KvRows q = kv_rows(a[5], type, c, 0), out = kv_rows(a[6], type, c, q.heads);
        if (q.rows != out.rows || a[7] == Py_None) throw NotPlain();
        float *lse = a[11] == Py_None ? nullptr : (float *)kv_tensor(a[11], at::kFloat, c.device, {c.c.sequences, q.rows, q.heads}).data_ptr();
        const at::Tensor &space = tensor(a[7], at::kByte);
        if (space.device() != c.device || space.dim() != 1) throw NotPlain();
        const float scale = a[8] == Py_None ? (float)std::pow((double)c.c.head_dim, -0.5) : threshold(a[8]);
        return call(function<decltype(&spqt_kv_attention)>(a[0]), &c.c, &q.r, &out.r, lse, (int)q.rows, kv_counts(a[9], c), (int)q.heads, scale,
                    small(a[10]), threshold(a[13]), space.data_ptr(), (size_t)space.numel(), current_stream(a[14]));
    });
}
// kv_evict(function, codes, scales, tail, weights, table, lengths, keep, recent, new_table, new_lengths, kept, stream)
PyObject *kv_evict(PyObject *, PyObject *const *a, Py_ssize_t n) {
    return guarded(n, 13, [&]() {
        if (a[3] == Py_None || a[4] == Py_None) throw NotPlain();
        const KvTensors c = kv_cache(a[1], a[2], a[5], a[6], a[3], a[4], kv_type(a[3]));
        const int keep = small(a[7]), recent = small(a[8]);
        const at::Tensor &table = tensor(a[9], at::kInt);
        if (table.device() != c.device || table.dim() != 2 || table.size(0) != c.c.sequences || table.size(1) > 1 << 30) throw NotPlain();
        int32_t *lengths = (int32_t *)kv_tensor(a[10], at::kInt, c.device, {c.c.sequences}).data_ptr();
        int32_t *kept = (int32_t *)kv_tensor(a[11], at::kInt, c.device, {c.c.sequences, c.c.kv_heads, keep}).data_ptr();
        return call(function<decltype(&spqt_kv_evict)>(a[0]), &c.c, keep, recent, (const int32_t *)table.data_ptr(), (int)table.size(1), lengths, kept,
                    current_stream(a[12]));
    });
}

#define SPQT_METHOD(name) {#name, (PyCFunction)(void (*)(void))name, METH_FASTCALL, nullptr}
PyMethodDef methods[] = {SPQT_METHOD(gather),  SPQT_METHOD(gather_rows), SPQT_METHOD(gemv),         SPQT_METHOD(gemv_fused), SPQT_METHOD(gemv_fused_rows),
                         SPQT_METHOD(cb_gemv), SPQT_METHOD(cb_gemv_one), SPQT_METHOD(cb_gemv_fused),
                         SPQT_METHOD(kv_append), SPQT_METHOD(kv_read), SPQT_METHOD(kv_attention), SPQT_METHOD(kv_evict), {nullptr, nullptr, 0, nullptr}};
PyModuleDef module = {PyModuleDef_HEAD_INIT, "_fastcall", "Device calls of binding.py without the interpreter.", -1, methods, nullptr, nullptr, nullptr, nullptr};

}  // namespace

PyMODINIT_FUNC PyInit__fastcall() {
    PyObject *m = PyModule_Create(&module);
    // binding.py uses the module only with the torch whose headers it was compiled against
    if (m && PyModule_AddStringConstant(m, "torch_version", SPQT_TORCH_VERSION) < 0) Py_CLEAR(m);
    return m;
}
