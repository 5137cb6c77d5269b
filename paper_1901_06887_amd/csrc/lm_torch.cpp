// From torch tensors to the calls of the operators behind language models' answers: the checks of shapes, types and strides, the argument blocks and the calls.
//
// A small call takes the GPU 3 to 5 us and the library's launch 3 us of the host.  The same checks in Python, with an attribute lookup or a method call for every
// fact about a tensor, took 0.5 us a tensor and 2 to 4 us a call; here they are loads.  Host code only (g++); the library's entry points come
// from the binding, which has it open (bind).
#include <Python.h>
#include <torch/csrc/autograd/python_variable.h>

#include <algorithm>
#include <cmath>
#include <initializer_list>
#include <sstream>
#include <stdexcept>

#include "../../include/mt.h"

namespace {

typedef mt_status (*NormCall)(mt_ctx*, void*, const mt_norm_args*);
typedef mt_status (*LinearCall)(mt_ctx*, void*, const mt_linear4_args*, const mt_row_group*, uint32_t, uint32_t, uint32_t);
typedef mt_status (*ScoreCall)(mt_ctx*, void*, const mt_score_args*);
typedef mt_status (*WriteCall)(mt_ctx*, void*, const mt_kv_cache*, const mt_kv_batch*, const mt_kv_write_args*);
typedef mt_status (*AttendCall)(mt_ctx*, void*, const mt_kv_cache*, const mt_kv_batch*, const mt_attend_args*);
typedef mt_status (*GrowCall)(mt_ctx*, void*, const mt_kv_cache*, const int32_t*, const int32_t*, uint32_t, int32_t*);       // mt_kv_fork too
typedef mt_status (*FreeCall)(mt_ctx*, void*, const mt_kv_cache*, const int32_t*, uint32_t);
typedef mt_status (*CompactCall)(mt_ctx*, void*, const mt_kv_cache*, int32_t*);
typedef mt_status (*CopyCall)(mt_ctx*, void*, const mt_kv_cache*, const int32_t*, const int32_t*, uint32_t);
typedef mt_status (*SampleCall)(mt_ctx*, void*, const mt_sample_args*);
NormCall norm_call;
LinearCall linear_call;
ScoreCall score_call;
WriteCall write_call;
AttendCall attend_call;
GrowCall grow_call, fork_call;
FreeCall free_call;
CompactCall compact_call;
CopyCall copy_call;
SampleCall sample_call;

struct Refused : std::runtime_error { using std::runtime_error::runtime_error; };      // a ValueError

constexpr auto kF32 = at::kFloat;
constexpr auto kBf16 = at::kBFloat16;
constexpr auto kInt = at::kInt;
constexpr auto kE4m3 = at::kFloat8_e4m3fn;
constexpr auto kE8m0 = at::kFloat8_e8m0fnu;

const at::Tensor& tensor(PyObject* o, const char* what)
{
    if (!THPVariable_Check(o)) throw Refused(std::string(what) + ": a tensor is wanted");
    return THPVariable_Unpack(o);
}

[[noreturn]] void refuse(const at::Tensor& t, const char* what, const char* wanted, uint64_t rows, uint64_t width, at::ScalarType type, int64_t device)
{
    std::ostringstream s;
    s << what << ": " << t.sizes() << " of " << c10::toString(t.scalar_type()) << " on " << t.device() << " with strides " << t.strides() << "; " << wanted << " [" << rows << ", " << width
      << "] of " << c10::toString(type) << " on cuda:" << device << " is wanted";
    throw Refused(s.str());
}

bool here(const at::Tensor& t, int64_t device) { return t.is_cuda() && t.get_device() == device; }

uint32_t dtype_of(const at::Tensor& t, const char* what)
{
    if (t.scalar_type() == kF32) return MT_F32;
    if (t.scalar_type() == kBf16) return MT_BF16;
    throw Refused(std::string(what) + " of " + c10::toString(t.scalar_type()) + ": float32 or bfloat16 is wanted");
}

struct Size { uint32_t rows, width; };
Size matrix(const at::Tensor& t, const char* what)
{
    if (t.dim() != 2 || t.size(0) > UINT32_MAX || t.size(1) > UINT32_MAX) {
        std::ostringstream s;
        s << what << ": " << t.sizes() << "; two dimensions (of less than 2^32) are wanted";
        throw Refused(s.str());
    }
    return Size{(uint32_t)t.size(0), (uint32_t)t.size(1)};
}

// The elements between consecutive rows of a [rows][width] tensor on the device, whose rows are contiguous.
uint64_t row_stride(const at::Tensor& t, const char* what, uint64_t rows, uint64_t width, at::ScalarType type, int64_t device)
{
    const bool fits = t.scalar_type() == type || (type == kE8m0 && t.scalar_type() == at::kByte);       // (scales also as bytes)
    if (t.dim() != 2 || (uint64_t)t.size(0) != rows || (uint64_t)t.size(1) != width || !fits || !here(t, device) || (width > 1 && t.stride(1) != 1))
        refuse(t, what, "contiguous rows", rows, width, type, device);
    return rows > 1 ? (uint64_t)t.stride(0) : width;
}

// Its address, too; nothing for None.
template <typename P>
void rows_of(PyObject* o, const char* what, uint64_t rows, uint64_t width, at::ScalarType type, int64_t device, P** p, uint64_t* stride)
{
    if (o == Py_None) return;
    const at::Tensor& t = tensor(o, what);
    *stride = row_stride(t, what, rows, width, type, device);
    *p = (P*)t.data_ptr();
}

// A contiguous [rows][width] tensor; a contiguous list of `rows`.
template <typename P>
void table_of(PyObject* o, const char* what, uint64_t rows, uint64_t width, at::ScalarType type, int64_t device, P** p)
{
    if (o == Py_None) return;
    const at::Tensor& t = tensor(o, what);
    if (row_stride(t, what, rows, width, type, device) != width) refuse(t, what, "contiguous", rows, width, type, device);
    *p = (P*)t.data_ptr();
}
template <typename P>
void list_of(PyObject* o, const char* what, uint64_t rows, at::ScalarType type, int64_t device, P** p)
{
    if (o == Py_None) return;
    const at::Tensor& t = tensor(o, what);
    if (t.dim() != 1 || (uint64_t)t.size(0) != rows || t.scalar_type() != type || !here(t, device) || (rows > 1 && t.stride(0) != 1))
        refuse(t, what, "a contiguous list", 1, rows, type, device);
    *p = (P*)t.data_ptr();
}

// The first three arguments of every call here: context, stream, device.
struct Where { mt_ctx* ctx; void* stream; int64_t device; };
Where where(PyObject* const* a)
{
    const Where w{(mt_ctx*)PyLong_AsVoidPtr(a[0]), PyLong_AsVoidPtr(a[1]), PyLong_AsLongLong(a[2])};
    if (PyErr_Occurred()) throw std::bad_alloc();       // (the Python error stands)
    return w;
}
float number(PyObject* o, const char* what)
{
    const double v = PyFloat_AsDouble(o);
    if (v == -1.0 && PyErr_Occurred()) { PyErr_Clear(); throw Refused(std::string(what) + ": a number is wanted"); }
    return (float)v;
}

// The call's status as a Python int; errors of the checks as Python's.
template <typename F> PyObject* guarded(Py_ssize_t n, Py_ssize_t wanted, F f)
{
    if (n != wanted) { PyErr_Format(PyExc_TypeError, "%zd arguments instead of %zd", n, wanted); return nullptr; }
    try {
        return PyLong_FromLong(f());
    } catch (const Refused& e) {
        PyErr_SetString(PyExc_ValueError, e.what());
    } catch (const std::exception& e) {
        if (!PyErr_Occurred()) PyErr_SetString(PyExc_RuntimeError, e.what());
    }
    return nullptr;
}
template <typename F> long without_gil(F f)
{
    long st;
    Py_BEGIN_ALLOW_THREADS
    st = (long)f();
    Py_END_ALLOW_THREADS
    return st;
}

// Outputs of a call that went through count as changed, so that autograd notices where it had kept one.  (Tensors of inference mode carry no versions.)
long written(long status, std::initializer_list<PyObject*> outputs)
{
    if (status == MT_OK)
        for (PyObject* o : outputs) {
            if (o == Py_None) continue;
            const at::Tensor& t = THPVariable_Unpack(o);
            if (!t.is_inference()) t.unsafeGetTensorImpl()->bump_version();
        }
    return status;
}

// x, residual, gain, gain_ids, eps, sum, y, y8, y8_scales
PyObject* add_norm(PyObject*, PyObject* const* o, Py_ssize_t n)
{
    return guarded(n, 12, [&] {
        const Where w = where(o);
        mt_norm_args a{};
        const at::Tensor& x = tensor(o[3], "x");
        const Size s = matrix(x, "x");
        const auto type = x.scalar_type();
        a.dtype = dtype_of(x, "rows");
        a.rows = s.rows; a.width = s.width;
        rows_of(o[3], "x", s.rows, s.width, type, w.device, &a.x, &a.x_stride);
        rows_of(o[4], "residual", s.rows, s.width, type, w.device, &a.residual, &a.residual_stride);
        if (o[5] != Py_None) {
            const at::Tensor& g = tensor(o[5], "gain");
            if (g.dim() == 1) {
                a.n_gains = 1; a.gain_stride = s.width;
                list_of(o[5], "gain", s.width, kF32, w.device, &a.gain);
            } else {
                a.n_gains = matrix(g, "gain").rows;
                rows_of(o[5], "gain", a.n_gains, s.width, kF32, w.device, &a.gain, &a.gain_stride);
            }
        }
        list_of(o[6], "gain_ids", s.rows, kInt, w.device, &a.gain_ids);
        a.eps = number(o[7], "eps");
        rows_of(o[8], "sum_out", s.rows, s.width, type, w.device, &a.sum, &a.sum_stride);
        rows_of(o[9], "out", s.rows, s.width, type, w.device, &a.y, &a.y_stride);
        rows_of(o[10], "out8", s.rows, s.width, kE4m3, w.device, &a.y8, &a.y8_stride);
        rows_of(o[11], "out8_scales", s.rows, ((uint64_t)s.width + 31) / 32, kE8m0, w.device, &a.y8_scales, &a.y8_scales_stride);
        return written(without_gil([&] { return norm_call(w.ctx, w.stream, &a); }), {o[8], o[9], o[10], o[11]});
    });
}

// groups, x, out, x_scales, act
PyObject* linear4(PyObject*, PyObject* const* o, Py_ssize_t n)
{
    return guarded(n, 8, [&] {
        const Where w = where(o);
        mt_linear4_args a{};
        const at::Tensor &x = tensor(o[4], "x"), &y = tensor(o[5], "out");
        const Size s = matrix(x, "x");
        a.rows = s.rows;
        const auto type = x.scalar_type();
        if (type == kE4m3) {
            a.x_dtype = MT_MX8;
            if (o[6] == Py_None) throw Refused("8-bit rows come with their scales");
            rows_of(o[6], "x_scales", s.rows, ((uint64_t)s.width + 31) / 32, kE8m0, w.device, &a.x_scales, &a.x_scales_stride);
        } else {
            a.x_dtype = dtype_of(x, "rows");
            if (o[6] != Py_None) throw Refused("scales come with 8-bit rows only");
        }
        // (a matrix may be narrower than the rows; that none is wider than the tensors, the library checks for every group)
        rows_of(o[4], "x", s.rows, s.width, type, w.device, &a.x, &a.x_stride);
        a.y_dtype = dtype_of(y, "out");
        const uint32_t y_width = matrix(y, "out").width;
        rows_of(o[5], "out", s.rows, y_width, y.scalar_type(), w.device, &a.y, &a.y_stride);
        const unsigned long act = PyLong_AsUnsignedLong(o[7]);
        if (PyErr_Occurred()) { PyErr_Clear(); throw Refused("act: one of MT_ACT_... is wanted"); }
        a.act = (uint32_t)std::min<unsigned long>(act, UINT32_MAX);
        Py_buffer groups;
        if (PyObject_GetBuffer(o[3], &groups, PyBUF_SIMPLE) != 0) { PyErr_Clear(); throw Refused("groups: what row_groups makes is wanted"); }
        const bool whole = groups.len % sizeof(mt_row_group) == 0;
        const long st = whole ? without_gil([&] { return linear_call(w.ctx, w.stream, &a, (const mt_row_group*)groups.buf, (uint32_t)(groups.len / sizeof(mt_row_group)), s.width, y_width); }) : 0;
        PyBuffer_Release(&groups);
        if (!whole) throw Refused("groups: what row_groups makes is wanted");
        return written(st, {o[5]});
    });
}

// logits, given, n_classes, allowed, temperature, given_logprobs, given_ranks, entropy, top_ids, top_logprobs, scratch
PyObject* score(PyObject*, PyObject* const* o, Py_ssize_t n)
{
    return guarded(n, 14, [&] {
        const Where w = where(o);
        mt_score_args a{};
        const at::Tensor& x = tensor(o[3], "logits");
        const Size s = matrix(x, "logits");
        a.dtype = dtype_of(x, "logits");
        a.rows = s.rows; a.classes = s.width;
        rows_of(o[3], "logits", s.rows, s.width, x.scalar_type(), w.device, &a.logits, &a.row_stride);
        list_of(o[5], "n_classes", s.rows, kInt, w.device, &a.n_classes);
        if (o[6] != Py_None) {
            const Size words = matrix(tensor(o[6], "allowed"), "allowed");
            if (words.width < ((uint64_t)s.width + 31) / 32) throw Refused("allowed: less than a bit for every class");
            rows_of(o[6], "allowed", s.rows, words.width, kInt, w.device, &a.allowed, &a.allowed_stride);
        }
        a.temperature = number(o[7], "temperature");
        // (outputs may be left out: how many classes are given, and how many alternatives are wanted, either of a pair says)
        const auto either = [&](int i, int j) { return o[i] != Py_None ? o[i] : o[j]; };
        if ((o[4] == Py_None) != (either(8, 9) == Py_None)) throw Refused("given classes and their outputs come together");
        if (o[4] != Py_None) {
            a.n_given = matrix(tensor(either(8, 9), "outputs of given classes"), "outputs of given classes").width;
            table_of(o[4], "given", s.rows, a.n_given, kInt, w.device, &a.given);
            table_of(o[8], "given_logprobs", s.rows, a.n_given, kF32, w.device, &a.given_logprobs);
            table_of(o[9], "given_ranks", s.rows, a.n_given, kInt, w.device, &a.given_ranks);
        }
        list_of(o[10], "entropy", s.rows, kF32, w.device, &a.entropy);
        if (either(11, 12) != Py_None) {
            a.top = matrix(tensor(either(11, 12), "alternatives"), "alternatives").width;
            table_of(o[11], "top_ids", s.rows, a.top, kInt, w.device, &a.top_ids);
            table_of(o[12], "top_logprobs", s.rows, a.top, kF32, w.device, &a.top_logprobs);
        }
        const at::Tensor& scratch = tensor(o[13], "scratch");
        list_of(o[13], "scratch", scratch.numel(), at::kByte, w.device, &a.scratch);
        a.scratch_bytes = scratch.numel();
        return written(without_gil([&] { return score_call(w.ctx, w.stream, &a); }), {o[8], o[9], o[10], o[11], o[12], o[13]});
    });
}

// ---- caches of language models: the fourth argument is a cache's description (mt_kv_cache, kept by its owner with the tensors it names), the fifth those tensors ----
struct OfCache { mt_kv_cache c; PyObject* tensors; };
OfCache cache_of(PyObject* o, PyObject* tensors, int64_t device)
{
    Py_buffer b;
    if (PyObject_GetBuffer(o, &b, PyBUF_SIMPLE) != 0) { PyErr_Clear(); throw Refused("cache: what alloc_kv makes is wanted"); }
    OfCache k;
    const bool whole = b.len == sizeof(k.c) && PyTuple_Check(tensors);
    if (whole) k.c = *(const mt_kv_cache*)b.buf;
    PyBuffer_Release(&b);
    if (!whole) throw Refused("cache: what alloc_kv makes is wanted");
    for (Py_ssize_t i = 0; i < PyTuple_GET_SIZE(tensors); ++i)
        if (PyTuple_GET_ITEM(tensors, i) != Py_None && !here(tensor(PyTuple_GET_ITEM(tensors, i), "cache"), device))
            throw Refused("cache: tensors on cuda:" + std::to_string(device) + " are wanted");
    k.tensors = tensors;
    return k;
}
// A call that went through has changed the cache's tensors (those that there are) in the given places of its tuple: k, v, k_scales, v_scales, table, lengths, refs.
long cache_written(long status, const OfCache& k, Py_ssize_t first, Py_ssize_t last)
{
    for (Py_ssize_t i = first; i < last && i < PyTuple_GET_SIZE(k.tensors); ++i) written(status, {PyTuple_GET_ITEM(k.tensors, i)});
    return status;
}

// A contiguous list of int32 of any length; its length.
template <typename P> uint32_t any_list(PyObject* o, const char* what, int64_t device, P** p)
{
    if (o == Py_None) return 0;
    const at::Tensor& t = tensor(o, what);
    list_of(o, what, t.numel(), kInt, device, p);
    if (t.numel() > INT32_MAX) throw Refused(std::string(what) + ": less than 2^31 entries are wanted");
    return (uint32_t)t.numel();
}

// Rows and whose they are.
mt_kv_batch batch_of(PyObject* seqs, PyObject* first_row, PyObject* max_new, uint32_t rows, int64_t device)
{
    mt_kv_batch b{};
    b.rows = rows;
    const uint32_t named = any_list(seqs, "seqs", device, &b.seqs);
    if (first_row != Py_None) {
        const uint32_t n = any_list(first_row, "first_row", device, &b.first_row);
        if (n == 0) throw Refused("first_row: an entry more than there are sequences is wanted");
        b.n_seqs = n - 1;
    } else b.n_seqs = rows;
    if (seqs != Py_None && named != b.n_seqs) throw Refused("seqs: one for every sequence of the batch is wanted");
    const unsigned long n = PyLong_AsUnsignedLong(max_new);
    if (PyErr_Occurred()) { PyErr_Clear(); throw Refused("max_new: a number is wanted"); }
    b.max_new = (uint32_t)std::min<unsigned long>(n, UINT32_MAX);
    return b;
}
uint32_t number_of(PyObject* o, const char* what)
{
    const unsigned long v = PyLong_AsUnsignedLong(o);
    if (PyErr_Occurred() || v > UINT32_MAX) { PyErr_Clear(); throw Refused(std::string(what) + ": a number of 0 or more is wanted"); }
    return (uint32_t)v;
}

// cache, its tensors, k, v, seqs, first_row, max_new, layer
PyObject* kv_write(PyObject*, PyObject* const* o, Py_ssize_t n)
{
    return guarded(n, 11, [&] {
        const Where w = where(o);
        const OfCache c = cache_of(o[3], o[4], w.device);
        mt_kv_write_args a{};
        const at::Tensor &k = tensor(o[5], "k"), &v = tensor(o[6], "v");
        const uint32_t rows = matrix(k, "k").rows;
        const uint64_t width = (uint64_t)c.c.heads * c.c.head_dim;
        a.dtype = dtype_of(k, "keys");
        a.k_stride = row_stride(k, "k", rows, width, k.scalar_type(), w.device);
        a.v_stride = row_stride(v, "v", rows, width, k.scalar_type(), w.device);
        a.k = k.data_ptr(); a.v = v.data_ptr();
        a.layer = number_of(o[10], "layer");
        const mt_kv_batch b = batch_of(o[7], o[8], o[9], rows, w.device);
        return cache_written(without_gil([&] { return write_call(w.ctx, w.stream, &c.c, &b, &a); }), c, 0, 4);
    });
}

// cache, its tensors, q, out, seqs, first_row, max_new, layer, window, max_length, scale (None: head_dim^-0.5), lse, scratch
PyObject* attend(PyObject*, PyObject* const* o, Py_ssize_t n)
{
    return guarded(n, 16, [&] {
        const Where w = where(o);
        const OfCache c = cache_of(o[3], o[4], w.device);
        mt_attend_args a{};
        const at::Tensor &q = tensor(o[5], "q"), &out = tensor(o[6], "out");
        const Size s = matrix(q, "q");
        if (c.c.head_dim == 0 || s.width % c.c.head_dim) throw Refused("q: rows of whole heads are wanted");
        a.dtype = dtype_of(q, "rows");
        a.q_heads = s.width / c.c.head_dim;
        a.q_stride = row_stride(q, "q", s.rows, s.width, q.scalar_type(), w.device);
        a.out_stride = row_stride(out, "out", s.rows, s.width, q.scalar_type(), w.device);
        a.q = q.data_ptr(); a.out = out.data_ptr();
        a.layer = number_of(o[10], "layer"); a.window = number_of(o[11], "window"); a.max_length = number_of(o[12], "max_length");
        a.scale = o[13] == Py_None ? (float)(1.0 / std::sqrt((double)c.c.head_dim)) : number(o[13], "scale");
        table_of(o[14], "lse", s.rows, a.q_heads, kF32, w.device, &a.lse);
        if (o[15] != Py_None) {
            const at::Tensor& scratch = tensor(o[15], "scratch");
            list_of(o[15], "scratch", scratch.numel(), at::kByte, w.device, &a.scratch);
            a.scratch_bytes = scratch.numel();
        }
        const mt_kv_batch b = batch_of(o[7], o[8], o[9], s.rows, w.device);
        return written(without_gil([&] { return attend_call(w.ctx, w.stream, &c.c, &b, &a); }), {o[6], o[14], o[15]});
    });
}

// cache, its tensors, two lists (the first may be None where `either`), granted
template <bool FORK> PyObject* take_pages(PyObject*, PyObject* const* o, Py_ssize_t n)
{
    return guarded(n, 8, [&] {
        const Where w = where(o);
        const OfCache c = cache_of(o[3], o[4], w.device);
        const int32_t *first = nullptr, *second = nullptr;
        int32_t* granted = nullptr;
        const uint32_t m = any_list((tensor(o[6], FORK ? "children" : "tokens"), o[6]), FORK ? "children" : "tokens", w.device, &second);
        if (FORK || o[5] != Py_None) list_of((tensor(o[5], FORK ? "parents" : "seqs"), o[5]), FORK ? "parents" : "seqs", m, kInt, w.device, &first);
        list_of(o[7], "granted", m, kInt, w.device, &granted);
        return cache_written(written(without_gil([&] { return (FORK ? fork_call : grow_call)(w.ctx, w.stream, &c.c, first, second, m, granted); }), {o[7]}), c, FORK ? 0 : 4, 7);
    });
}
PyObject* kv_grow(PyObject* m, PyObject* const* o, Py_ssize_t n) { return take_pages<false>(m, o, n); }
PyObject* kv_fork(PyObject* m, PyObject* const* o, Py_ssize_t n) { return take_pages<true>(m, o, n); }

// cache, its tensors, seqs
PyObject* kv_free(PyObject*, PyObject* const* o, Py_ssize_t n)
{
    return guarded(n, 6, [&] {
        const Where w = where(o);
        const OfCache c = cache_of(o[3], o[4], w.device);
        const int32_t* seqs = nullptr;
        const uint32_t m = any_list((tensor(o[5], "seqs"), o[5]), "seqs", w.device, &seqs);
        return cache_written(without_gil([&] { return free_call(w.ctx, w.stream, &c.c, seqs, m); }), c, 4, 7);
    });
}

// cache, its tensors, live
PyObject* kv_compact(PyObject*, PyObject* const* o, Py_ssize_t n)
{
    return guarded(n, 6, [&] {
        const Where w = where(o);
        const OfCache c = cache_of(o[3], o[4], w.device);
        int32_t* live = nullptr;
        list_of(o[5], "live", 1, kInt, w.device, &live);
        return cache_written(written(without_gil([&] { return compact_call(w.ctx, w.stream, &c.c, live); }), {o[5]}), c, 0, 7);
    });
}

// cache, its tensors, from, to
PyObject* kv_copy(PyObject*, PyObject* const* o, Py_ssize_t n)
{
    return guarded(n, 7, [&] {
        const Where w = where(o);
        const OfCache c = cache_of(o[3], o[4], w.device);
        const int32_t *from = nullptr, *to = nullptr;
        const uint32_t m = any_list((tensor(o[5], "from"), o[5]), "from", w.device, &from);
        list_of((tensor(o[6], "to"), o[6]), "to", m, kInt, w.device, &to);
        return cache_written(without_gil([&] { return copy_call(w.ctx, w.stream, &c.c, from, to, m); }), c, 0, 4);
    });
}

// logits, uniform, temperature, top_k, top_p, min_p, n_classes, allowed, ids, logprobs, kept, scratch
PyObject* sample(PyObject*, PyObject* const* o, Py_ssize_t n)
{
    return guarded(n, 15, [&] {
        const Where w = where(o);
        mt_sample_args a{};
        const at::Tensor& x = tensor(o[3], "logits");
        const Size s = matrix(x, "logits");
        a.dtype = dtype_of(x, "logits");
        a.rows = s.rows; a.classes = s.width;
        rows_of(o[3], "logits", s.rows, s.width, x.scalar_type(), w.device, &a.logits, &a.row_stride);
        list_of((tensor(o[4], "uniform"), o[4]), "uniform", s.rows, kF32, w.device, &a.uniform);
        list_of(o[5], "temperature", s.rows, kF32, w.device, &a.temperature);
        list_of(o[6], "top_k", s.rows, kInt, w.device, &a.top_k);
        list_of(o[7], "top_p", s.rows, kF32, w.device, &a.top_p);
        list_of(o[8], "min_p", s.rows, kF32, w.device, &a.min_p);
        list_of(o[9], "n_classes", s.rows, kInt, w.device, &a.n_classes);
        if (o[10] != Py_None) {
            const Size words = matrix(tensor(o[10], "allowed"), "allowed");
            if (words.width < ((uint64_t)s.width + 31) / 32) throw Refused("allowed: less than a bit for every class");
            rows_of(o[10], "allowed", s.rows, words.width, kInt, w.device, &a.allowed, &a.allowed_stride);
        }
        list_of(o[11], "ids", s.rows, kInt, w.device, &a.ids);
        list_of(o[12], "logprobs", s.rows, kF32, w.device, &a.logprobs);
        list_of(o[13], "kept", s.rows, kInt, w.device, &a.kept);
        if (o[14] != Py_None) list_of(o[14], "scratch", tensor(o[14], "scratch").numel(), at::kByte, w.device, &a.scratch);
        return written(without_gil([&] { return sample_call(w.ctx, w.stream, &a); }), {o[11], o[12], o[13]});
    });
}

// The addresses of mt_add_norm, mt_linear4_within, mt_score and the calls on caches, in the order of their types above.
PyObject* bind(PyObject*, PyObject* const* o, Py_ssize_t n)
{
    return guarded(n, 11, [&] {
        void* p[11];
        for (int i = 0; i < 11; ++i)
            if (!(p[i] = PyLong_AsVoidPtr(o[i]))) throw Refused("null entry point");
        norm_call = (NormCall)p[0]; linear_call = (LinearCall)p[1]; score_call = (ScoreCall)p[2];
        write_call = (WriteCall)p[3]; attend_call = (AttendCall)p[4]; grow_call = (GrowCall)p[5]; fork_call = (GrowCall)p[6];
        free_call = (FreeCall)p[7]; compact_call = (CompactCall)p[8]; copy_call = (CopyCall)p[9]; sample_call = (SampleCall)p[10];
        return 0L;
    });
}

#define MT_METHOD(name) {#name, (PyCFunction)(void*)name, METH_FASTCALL, nullptr}
PyMethodDef methods[] = {MT_METHOD(add_norm), MT_METHOD(linear4), MT_METHOD(score), MT_METHOD(kv_write), MT_METHOD(attend), MT_METHOD(kv_grow), MT_METHOD(kv_fork), MT_METHOD(kv_free), MT_METHOD(kv_compact),
                        MT_METHOD(kv_copy), MT_METHOD(sample), MT_METHOD(bind), {nullptr, nullptr, 0, nullptr}};
PyModuleDef module = {PyModuleDef_HEAD_INIT, "_answers", "Calls of the operators behind language models' answers on torch tensors.", -1, methods, nullptr, nullptr, nullptr, nullptr};

}  // namespace

PyMODINIT_FUNC PyInit__answers() { return PyModule_Create(&module); }
