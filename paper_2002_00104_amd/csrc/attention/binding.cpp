// The operators of pwlq_attention.h for Python, on tensors: _pwlq_attention.append and the others that attention.py documents.
// C++ for the same reason as the block's operators: a call for one token has a dozen tensors to check.
#include "../block/binding.h"

#include "../../../include/pwlq_attention.h"

namespace {

bool is_half(ScalarType t) { return t == at::kBFloat16 || t == at::kHalf; }

const int32_t *integers(const Call &c, const char *name, const Tensor *t, at::IntArrayRef sizes)
{
    c.dense(name, t, sizes, at::kInt);
    return t ? static_cast<const int32_t *>(t->data_ptr()) : nullptr;
}

// a[0..6]: keys, values, key_step or None, value_step or None, table, lengths, starts or None; T: rows of the call, or -1 for one
// of each sequence
constexpr int kShared = 7;
void shared(const Call &c, PyObject *const *a, int64_t T, pwlq_cache &cache, pwlq_batch &batch)
{
    const Tensor &keys = needed("keys", a[0]), &values = needed("values", a[1]);
    const ScalarType type = keys.scalar_type();
    if (!is_half(type) && type != at::kChar) refuse("keys must be bfloat16, float16 or int8");
    const int64_t pages = keys.size(0), heads = keys.size(1), page = keys.size(2), D = keys.size(3);
    if (heads > INT32_MAX || page > INT32_MAX || D > INT32_MAX) refuse("keys is too large");
    c.dense("keys", &keys, {pages, heads, page, D}, type);
    c.dense("values", &values, {pages, heads, page, D}, type);
    const Tensor *key_step = tensor("key_step", a[2]), *value_step = tensor("value_step", a[3]);
    if ((type == at::kChar) != (key_step != nullptr) || !key_step != !value_step) refuse("steps go with keys and values of int8");
    cache.keys = keys.data_ptr();
    cache.values = values.data_ptr();
    cache.key_step = const_cast<float *>(c.floats("key_step", key_step, {pages, heads, page}));
    cache.value_step = const_cast<float *>(c.floats("value_step", value_step, {pages, heads, page}));
    cache.pages = pages;
    cache.heads = (int)heads;
    cache.page = (int)page;
    cache.D = (int)D;
    cache.type = type_of(type);
    const Tensor &table = needed("table", a[4]), &lengths = needed("lengths", a[5]), *starts = tensor("starts", a[6]);
    if (!(table.device() == c.device && table.scalar_type() == at::kInt && table.dim() == 2)) refuse("table must be an int32 matrix on the device of the cache");
    batch.S = table.size(0);
    batch.table_pages = table.size(1);
    if ((batch.table_pages > 1 && table.stride(1) != 1) || (batch.S > 1 && table.stride(0) < batch.table_pages))
        refuse("table must have its columns next to each other, and rows that do not overlap");
    batch.table_stride = batch.S > 1 ? table.stride(0) : batch.table_pages;
    batch.T = T < 0 ? batch.S : T;
    batch.table = static_cast<const int32_t *>(table.data_ptr());
    batch.lengths = integers(c, "lengths", &lengths, {batch.S});
    batch.starts = integers(c, "starts", starts, {batch.S + 1});
}

pwlq_heads heads_of(const Call &c, const char *name, const Tensor *t, int64_t T, int64_t heads, int64_t D, ScalarType type)
{
    pwlq_heads h = {nullptr, 0, 0, 0};
    if (!t) return h;
    if (!(t->device() == c.device && t->scalar_type() == type && t->dim() == 3 && t->size(0) == T && t->size(1) == heads && t->size(2) == D))
        refuse("%s must be [rows, heads, D], of the sizes, the type and the device that go with the other arguments", name);
    if (t->stride(2) != 1) refuse("%s must have its channels next to each other", name);
    h.data = t->data_ptr();
    h.stride = T > 1 ? t->stride(0) : 0;
    h.head_stride = heads > 1 ? t->stride(1) : 0;
    h.type = type_of(type);
    return h;
}

int truth(PyObject *o)
{
    const int v = PyObject_IsTrue(o);
    if (v < 0) throw python_error();
    return v;
}
int64_t integer(PyObject *o)
{
    const long long v = PyLong_AsLongLong(o);
    if (v == -1 && PyErr_Occurred()) throw python_error();
    return v;
}

// the shared arguments, k, v, q or None, positions or None, frequencies or None, interleaved, out or None, stream
PyObject *append(PyObject *, PyObject *const *a, Py_ssize_t n)
{
    HANDLE_TH_ERRORS
    count("append", n, kShared + 8);
    PyObject *const *const m = a + kShared;
    const Tensor &k = needed("k", m[0]), &v = needed("v", m[1]), *q = tensor("q", m[2]), *out = tensor("out", m[6]);
    const Call c("keys", needed("keys", a[0]), 4);
    untracked(nullptr, {{"keys", tensor("keys", a[0])}, {"values", tensor("values", a[1])}, {"key_step", tensor("key_step", a[2])},
                        {"value_step", tensor("value_step", a[3])}, {"k", &k}, {"v", &v}, {"q", q},
                        {"frequencies", tensor("frequencies", m[4])}, {"out", out}});
    if (k.dim() != 3 || !is_half(k.scalar_type())) refuse("k must be [rows, heads, D] of bfloat16 or float16");
    const ScalarType type = k.scalar_type();
    const int64_t T = k.size(0);
    pwlq_append_args args = {};
    shared(c, a, T, args.cache, args.batch);
    if (args.cache.type != PWLQ_I8 && args.cache.type != type_of(type)) refuse("k must be of the cache's type, or the cache of int8");
    const int64_t heads = args.cache.heads, D = args.cache.D;
    args.k = heads_of(c, "k", &k, T, heads, D, type);
    args.v = heads_of(c, "v", &v, T, heads, D, type);
    Tensor turned;
    if (q) {
        if (q->dim() != 3 || q->size(1) > INT32_MAX) refuse("q must be [rows, heads, D]");
        args.q_heads = (int)q->size(1);
        args.q = heads_of(c, "q", q, T, args.q_heads, D, type);
        turned = out ? *out : c.make({T, args.q_heads, D}, type);
        args.q_out = heads_of(c, "out", &turned, T, args.q_heads, D, type);
    } else if (out) {
        refuse("out goes with q");
    }
    args.positions = integers(c, "positions", tensor("positions", m[3]), {T});
    if (const Tensor *f = tensor("frequencies", m[4])) {
        if (f->dim() != 1 || f->size(0) > D) refuse("frequencies must be one for each pair of rotated channels");
        args.frequencies = c.floats("frequencies", f, {f->size(0)});
        args.rotated = 2 * (int)f->size(0);
    }
    args.interleaved = truth(m[5]);
    void *stream = stream_of(m[7]);
    call([&] { return pwlq_append(&args, stream); });
    return wrap(turned);
    END_HANDLE_TH_ERRORS
}

// the shared arguments, rows or None, dtype or None, k or None, v or None, stream
PyObject *read(PyObject *, PyObject *const *a, Py_ssize_t n)
{
    HANDLE_TH_ERRORS
    count("read", n, kShared + 5);
    PyObject *const *const m = a + kShared;
    const Tensor &keys = needed("keys", a[0]), *k = tensor("k", m[2]), *v = tensor("v", m[3]);
    const Call c("keys", keys, 4);
    untracked(nullptr, {{"keys", &keys}, {"values", tensor("values", a[1])}, {"key_step", tensor("key_step", a[2])},
                        {"value_step", tensor("value_step", a[3])}, {"k", k}, {"v", v}});
    pwlq_read_args args = {};
    const int64_t rows = m[0] == Py_None ? -1 : integer(m[0]);
    if (m[0] != Py_None && rows < 0) refuse("rows is negative");
    if (a[6] != Py_None && m[0] == Py_None) refuse("rows must be given with starts");
    shared(c, a, rows, args.cache, args.batch);
    const int64_t T = args.batch.T, heads = args.cache.heads, D = args.cache.D;
    const ScalarType type = dtype_of(m[1], k ? k->scalar_type() : v ? v->scalar_type() : keys.scalar_type() == at::kChar ? at::kBFloat16 : keys.scalar_type());
    if (!is_half(type) || (args.cache.type != PWLQ_I8 && args.cache.type != type_of(type))) refuse("rows are read as the cache's type, or from int8 as bfloat16 or float16");
    Tensor to_k = k ? *k : c.make({T, heads, D}, type), to_v = v ? *v : c.make({T, heads, D}, type);
    args.k = heads_of(c, "k", &to_k, T, heads, D, type);
    args.v = heads_of(c, "v", &to_v, T, heads, D, type);
    void *stream = stream_of(m[4]);
    call([&] { return pwlq_read(&args, stream); });
    return tuple(to_k, to_v);
    END_HANDLE_TH_ERRORS
}

// the shared arguments, q, longest or None, scale or None, cap, slopes or None, window, prefix or None, tree or None, out or None,
// workspace or None, stream
PyObject *attend(PyObject *, PyObject *const *a, Py_ssize_t n)
{
    HANDLE_TH_ERRORS
    count("attend", n, kShared + 11);
    PyObject *const *const m = a + kShared;
    const Tensor &q = needed("q", m[0]), *given = tensor("out", m[8]), *slopes = tensor("slopes", m[4]), *tree = tensor("tree", m[7]);
    const Call c("keys", needed("keys", a[0]), 4);
    untracked(nullptr, {{"keys", tensor("keys", a[0])}, {"values", tensor("values", a[1])}, {"key_step", tensor("key_step", a[2])},
                        {"value_step", tensor("value_step", a[3])}, {"q", &q}, {"slopes", slopes}, {"out", given}});
    if (q.dim() != 3 || !is_half(q.scalar_type()) || q.size(1) > INT32_MAX) refuse("q must be [rows, heads, D] of bfloat16 or float16");
    const ScalarType type = q.scalar_type();
    const int64_t T = q.size(0), H = q.size(1);
    pwlq_attend_args args = {};
    shared(c, a, T, args.cache, args.batch);
    if (args.cache.type != PWLQ_I8 && args.cache.type != type_of(type)) refuse("q must be of the cache's type, or the cache of int8");
    const int64_t D = args.cache.D;
    args.q_heads = (int)H;
    args.q = heads_of(c, "q", &q, T, H, D, type);
    args.longest = m[1] == Py_None ? 0 : integer(m[1]);
    args.scale = m[2] == Py_None ? 1.0f / __builtin_sqrtf((float)D) : real(m[2]);
    args.cap = real(m[3]);
    args.slopes = c.floats("slopes", slopes, {H});
    args.window = integer(m[5]);
    args.prefix = integers(c, "prefix", tensor("prefix", m[6]), {args.batch.S});
    if (tree) {
        if (tree->dim() != 2) refuse("tree must be a matrix");
        args.tree_words = tree->size(1);
        c.dense("tree", tree, {T, args.tree_words}, at::kLong);
        args.tree = static_cast<const uint64_t *>(tree->data_ptr());
    }
    void *stream = stream_of(m[10]);
    Tensor out = given ? *given : c.make({T, H, D}, type), keep;
    args.out = heads_of(c, "out", &out, T, H, D, type);
    size_t bytes = 0;
    void *room = c.room(m[9], pwlq_attend_workspace_bytes(&args), keep, bytes);
    call([&] { return pwlq_attend(&args, room, bytes, stream); });
    return wrap(out);
    END_HANDLE_TH_ERRORS
}

PyMethodDef g_methods[] = {METHOD(append), METHOD(read), METHOD(attend), {"raises", raises, METH_O, nullptr}, {nullptr, nullptr, 0, nullptr}};
PyModuleDef g_module = {PyModuleDef_HEAD_INIT, "_pwlq_attention", nullptr, -1, g_methods, nullptr, nullptr, nullptr, nullptr};

} // namespace

PyMODINIT_FUNC PyInit__pwlq_attention(void) { return PyModule_Create(&g_module); }
