// CPython binding of the C ABI in include/amq.h: argument marshalling only, in native code.
//
// A call through ctypes costs some 9 us of interpreter time (argument conversion, data_ptr per tensor, current_stream), twice a
// short kernel's duration; here it costs about one.  Entry points of the header are Python functions of the same name without the trailing
// stream argument (the calling thread's current stream is used): pointers take None, a tensor (checked: CUDA, contiguous, the element
// type of the pointer) or an integer address (unchecked: strided views, host memory), sizes take integers.  The operators of a decoder step
// take tensors instead, whose shapes and strides are looked at here (second half of this file).  The library is opened by path, so that an
// instrumented build can take its place.
#define PY_SSIZE_T_CLEAN
#include <Python.h>

#include <dlfcn.h>

#include <algorithm>
#include <climits>
#include <tuple>
#include <type_traits>
#include <utility>

#include <ATen/ATen.h>
#include <c10/core/Storage.h>
#include <c10/cuda/CUDAGuard.h>
#include <c10/cuda/CUDAStream.h>
#include <torch/csrc/autograd/python_variable.h>

#include "amq.h"

namespace {

template <typename T> struct Element;
template <> struct Element<float> { static constexpr at::ScalarType type = at::kFloat; static constexpr const char* name = "float32"; };
template <> struct Element<uint32_t> { static constexpr at::ScalarType type = at::kInt; static constexpr const char* name = "int32"; };
template <> struct Element<int32_t> { static constexpr at::ScalarType type = at::kInt; static constexpr const char* name = "int32"; };
template <> struct Element<void> { static constexpr at::ScalarType type = at::kByte; static constexpr const char* name = "uint8"; };    // (any)

// one argument; on a mismatch sets a Python error
template <typename T, typename = void> struct Arg;

template <typename T>
struct Arg<T*> {
    static T* get(PyObject* o, Py_ssize_t index)
    {
        using E = Element<std::remove_const_t<T>>;
        if (o == Py_None) return nullptr;
        if (THPVariable_Check(o)) {
            const at::Tensor& t = THPVariable_Unpack(o);
            if (t.is_cuda() && (std::is_void_v<std::remove_const_t<T>> || t.scalar_type() == E::type) && t.is_contiguous()) return static_cast<T*>(t.data_ptr());
            PyErr_Format(PyExc_TypeError, "argument %zd must be a contiguous CUDA tensor of dtype %s", index, E::name);
            return nullptr;
        }
        void* p = PyLong_AsVoidPtr(o);
        return static_cast<T*>(p);
    }
};

template <typename T>
struct Arg<T, std::enable_if_t<std::is_integral_v<T>>> {
    static T get(PyObject* o, Py_ssize_t index)
    {
        const long long v = PyLong_AsLongLong(o);
        const T r = static_cast<T>(v);
        if (static_cast<long long>(r) != v && !PyErr_Occurred())
            PyErr_Format(PyExc_OverflowError, "argument %zd is out of range", index);
        return r;
    }
};

template <typename... A, size_t... I>
PyObject* call_checked(amq_status (*f)(A...), PyObject* const* args, std::index_sequence<I...>)
{
    using Tuple = std::tuple<A...>;
    // all arguments but the last, which is the stream
    // (none is looked at behind one that was refused: asking an object's type with an error pending is an error of its own)
    std::tuple<std::tuple_element_t<I, Tuple>...> v{
        (PyErr_Occurred() ? std::tuple_element_t<I, Tuple>{} : Arg<std::tuple_element_t<I, Tuple>>::get(args[I], (Py_ssize_t)I))...};
    if (PyErr_Occurred()) return nullptr;
    void* stream = c10::cuda::getCurrentCUDAStream().stream();
    amq_status s;
    Py_BEGIN_ALLOW_THREADS
    s = f(std::get<I>(v)..., stream);
    Py_END_ALLOW_THREADS
    return PyLong_FromLong(s);
}

template <typename... A>
PyObject* call(amq_status (*f)(A...), PyObject* const* args, Py_ssize_t nargs)
{
    constexpr size_t N = sizeof...(A) - 1;
    if (!f) { PyErr_SetString(PyExc_RuntimeError, "the library has not been opened"); return nullptr; }
    if (nargs != (Py_ssize_t)N) {
        PyErr_Format(PyExc_TypeError, "expected %zu arguments, got %zd", N, nargs);
        return nullptr;
    }
    try {
        return call_checked(f, args, std::make_index_sequence<N>{});
    } catch (const std::exception& e) {
        PyErr_SetString(PyExc_RuntimeError, e.what());
        return nullptr;
    }
}

#define AMQ_ENTRIES(X)                                                                                                          \
    X(amq_quantize) X(amq_pack) X(amq_unpack) X(amq_binary_dots) X(amq_binary_gemm) X(amq_quantized_gemv) X(amq_lstm_step)      \
    X(amq_lstm_step_static) X(amq_gru_step) X(amq_lstm_sequence) X(amq_gru_sequence) X(amq_lstm_sequence_host)                  \
    X(amq_gru_sequence_host) X(amq_selftest_sequence_give_up) X(amq_selftest_batched_sequence) X(amq_selftest_decode_give_up) X(amq_selftest_binary_gemm) \
    X(amq_gru_step_original) X(amq_quantize_variant) X(amq_lm_greedy_decode) X(amq_log_softmax_argmax) X(amq_beam_select) X(amq_embedding_rows) X(amq_lstm_step_paper) X(amq_lstm_sequence_paper)

#define AMQ_WRAP(name)                                                                          \
    decltype(&::name) p_##name = nullptr;                                                       \
    PyObject* py_##name(PyObject*, PyObject* const* args, Py_ssize_t nargs) { return call(p_##name, args, nargs); }
AMQ_ENTRIES(AMQ_WRAP)

// ---- calls whose arguments are looked at and whose results are made here as well -----------------------------------------------------
// (short kernels: shapes, strides and results cost the interpreter more than the kernel takes).  Each answers with its results, or with the status
// of a call that the library refused, as an integer.

// a tensor argument, or null (with a Python error) where it is none
const at::Tensor* tensor(PyObject* o, const char* name)
{
    if (THPVariable_Check(o)) return &THPVariable_Unpack(o);
    PyErr_Format(PyExc_TypeError, "%s must be a tensor", name);
    return nullptr;
}

bool refuse(const char* what) { PyErr_SetString(PyExc_TypeError, what); return false; }

bool shaped(const at::Tensor& t, at::ScalarType type, std::initializer_list<int64_t> shape)
{
    if (!t.is_cuda() || t.scalar_type() != type || t.dim() != (int64_t)shape.size()) return false;
    int64_t d = 0;
    for (int64_t s : shape)
        if (t.size(d++) != s) return false;
    return true;
}

// the same, and contiguous
bool packed(const at::Tensor& t, at::ScalarType type, std::initializer_list<int64_t> shape) { return shaped(t, type, shape) && t.is_contiguous(); }

// rows of a matrix: contiguous, at any stride that is no shorter; their stride, or -1
int64_t leading(const at::Tensor& t)
{
    const int64_t rows = t.size(0), cols = t.size(1);
    if (cols > 1 && t.stride(1) != 1) return -1;
    if (rows <= 1) return std::max(cols, t.stride(0));
    return t.stride(0) >= cols ? t.stride(0) : -1;
}

bool same_device(std::initializer_list<const at::Tensor*> ts)
{
    const at::Tensor* first = nullptr;
    for (const at::Tensor* t : ts) {
        if (!t) continue;
        if (first && t->device() != first->device()) return refuse("all tensors must be on one device");
        first = t;
    }
    return true;
}

int64_t fits(int64_t v) { return v <= INT_MAX ? v : -1; }       // (a size that the library refuses)

at::Tensor fresh(at::IntArrayRef size, at::ScalarType type, const at::Tensor& like) { return at::empty(size, at::TensorOptions().dtype(type).device(like.device())); }

template <typename F>
PyObject* guarded(F&& f)
{
    try {
        return f();
    } catch (const std::exception& e) {
        if (!PyErr_Occurred()) PyErr_SetString(PyExc_RuntimeError, e.what());
        return nullptr;
    }
}

// The library's call without the interpreter's lock (a launch waits where the device's queue is full).  Its arguments are numbers and addresses, made before
// the lock goes: other threads may change a list of tensors meanwhile.
template <typename... P, typename... A>
amq_status unlocked(amq_status (*f)(P...), A... args)
{
    amq_status s;
    Py_BEGIN_ALLOW_THREADS
    s = f(args...);
    Py_END_ALLOW_THREADS
    return s;
}

// the device of the call's tensors made current, and its current stream
struct On {
    c10::cuda::CUDAGuard guard;
    explicit On(const at::Tensor& t) : guard(t.device()) {}
    void* stream() const { return c10::cuda::getCurrentCUDAStream().stream(); }
};

decltype(&::amq_binary_gemm_act) p_amq_binary_gemm_act = nullptr;

// binary_gemm_act(Wcodes, Walpha, xcodes, xbeta, n, bias, activation, residual, y)
PyObject* py_binary_gemm_act(PyObject*, PyObject* const* args, Py_ssize_t nargs)
{
    if (!p_amq_binary_gemm_act || nargs != 9) { PyErr_SetString(PyExc_TypeError, "binary_gemm_act takes nine arguments of an opened library"); return nullptr; }
    return guarded([&]() -> PyObject* {
        const at::Tensor *Wc = tensor(args[0], "Wcodes"), *Wa = Wc ? tensor(args[1], "Walpha") : nullptr, *xc = Wa ? tensor(args[2], "xcodes") : nullptr,
                         *xb = xc ? tensor(args[3], "xbeta") : nullptr;
        if (!xb) return nullptr;
        const at::Tensor *bias = nullptr, *residual = nullptr, *y = nullptr;
        if (args[5] != Py_None && !(bias = tensor(args[5], "bias"))) return nullptr;
        if (args[7] != Py_None && !(residual = tensor(args[7], "residual"))) return nullptr;
        if (args[8] != Py_None && !(y = tensor(args[8], "y"))) return nullptr;
        const long long n = PyLong_AsLongLong(args[4]), act = PyLong_AsLongLong(args[6]);
        if (PyErr_Occurred()) return nullptr;
        if (Wc->dim() != 3 || xc->dim() != 3) { refuse("codes must have the shape (rows, bits, words of a plane)"); return nullptr; }
        const int64_t m = Wc->size(0), kw = Wc->size(1), batch = xc->size(0), ka = xc->size(1), words = 4 * ((n + 127) / 128);
        if (!packed(*Wc, at::kInt, {m, kw, words}) || !packed(*xc, at::kInt, {batch, ka, words})) {
            refuse("codes must be contiguous CUDA int32 tensors (rows, bits, words of a plane of n)");
            return nullptr;
        }
        if (!packed(*Wa, at::kFloat, {m, kw}) || !packed(*xb, at::kFloat, {batch, ka}) || (bias && !packed(*bias, at::kFloat, {m}))) {
            refuse("coefficients (rows, bits) and bias (rows of W) must be contiguous CUDA float32 tensors");
            return nullptr;
        }
        if ((residual && (!shaped(*residual, at::kFloat, {batch, m}) || leading(*residual) < 0)) || (y && (!shaped(*y, at::kFloat, {batch, m}) || leading(*y) < 0))) {
            refuse("residual and y must be CUDA float32 tensors (vectors, rows of W) with contiguous rows");
            return nullptr;
        }
        if (!same_device({Wc, Wa, xc, xb, bias, residual, y})) return nullptr;
        const On on(*Wc);
        at::Tensor out = y ? *y : fresh({batch, m}, at::kFloat, *Wc);
        const amq_status s = unlocked(
            p_amq_binary_gemm_act, static_cast<const uint32_t*>(Wc->data_ptr()), static_cast<const float*>(Wa->data_ptr()), (int)fits(m), (int)fits(n), (int)kw,
            static_cast<const uint32_t*>(xc->data_ptr()), static_cast<const float*>(xb->data_ptr()), (int)fits(batch), (int)ka,
            bias ? static_cast<const float*>(bias->data_ptr()) : nullptr, act == (int)act ? (int)act : -1, residual ? static_cast<const float*>(residual->data_ptr()) : nullptr,
            residual ? (int)fits(leading(*residual)) : 0, static_cast<float*>(out.data_ptr()), (int)fits(leading(out)), on.stream());
        return s == AMQ_OK ? THPVariable_Wrap(out) : PyLong_FromLong(s);
    });
}

// a cache (kcodes, kcoeffs, vcodes, vcoeffs), block table and lengths, checked against one another
struct Cache {
    const at::Tensor *t[4], *table, *lengths;
    int64_t pages, page_size, heads, k, d, batch, max_pages, ld_table;
};

bool cache_of(PyObject* cache, PyObject* table, PyObject* lengths, int64_t d, Cache* out)
{
    if (!PyTuple_Check(cache) && !PyList_Check(cache)) return refuse("a cache is (kcodes, kcoeffs, vcodes, vcoeffs)");
    if (PySequence_Fast_GET_SIZE(cache) != 4) return refuse("a cache is (kcodes, kcoeffs, vcodes, vcoeffs)");
    for (int i = 0; i < 4; ++i)
        if (!(out->t[i] = tensor(PySequence_Fast_GET_ITEM(cache, i), "each part of a cache"))) return false;
    if (!(out->table = tensor(table, "table")) || !(out->lengths = tensor(lengths, "lengths"))) return false;
    const at::Tensor& k = *out->t[0];
    if (k.dim() != 5) return refuse("cached codes must have the shape (pages, page_size, heads, bits, words of a plane)");
    out->pages = k.size(0); out->page_size = k.size(1); out->heads = k.size(2); out->k = k.size(3); out->d = d;
    const int64_t words = 4 * ((d + 127) / 128);
    for (int i = 0; i < 4; ++i) {
        const bool ok = i % 2 == 0 ? packed(*out->t[i], at::kInt, {out->pages, out->page_size, out->heads, out->k, words})
                                   : packed(*out->t[i], at::kFloat, {out->pages, out->page_size, out->heads, out->k});
        if (!ok) return refuse("a cache is four contiguous CUDA tensors: int32 codes (pages, page_size, heads, bits, words of a plane of d), float32 coefficients "
                               "(pages, page_size, heads, bits), of the keys and of the values");
    }
    const at::Tensor& t = *out->table;
    if (!t.is_cuda() || t.scalar_type() != at::kInt || t.dim() != 2 || leading(t) < 0)
        return refuse("table must be a CUDA int32 tensor (batch, pages of a sequence) with contiguous rows");
    out->batch = t.size(0); out->max_pages = t.size(1); out->ld_table = leading(t);
    if (!packed(*out->lengths, at::kInt, {out->batch})) return refuse("lengths must be a contiguous CUDA int32 tensor (batch,)");
    return same_device({out->t[0], out->t[1], out->t[2], out->t[3], out->table, out->lengths});
}

template <typename T> T* data(const at::Tensor* t) { return static_cast<T*>(t->data_ptr()); }

decltype(&::amq_cache_append) p_amq_cache_append = nullptr;

// cache_append(kcodes, kcoeffs, vcodes, vcoeffs, cache, table, lengths, d)
PyObject* py_cache_append(PyObject*, PyObject* const* args, Py_ssize_t nargs)
{
    if (!p_amq_cache_append || nargs != 8) { PyErr_SetString(PyExc_TypeError, "cache_append takes eight arguments of an opened library"); return nullptr; }
    return guarded([&]() -> PyObject* {
        const long long d = PyLong_AsLongLong(args[7]);
        Cache c;
        if (PyErr_Occurred() || !cache_of(args[4], args[5], args[6], d, &c)) return nullptr;
        const at::Tensor* rows[4];
        for (int i = 0; i < 4; ++i)
            if (!(rows[i] = tensor(args[i], "each of the new rows' parts"))) return nullptr;
        const int64_t count = rows[0]->dim() == 5 ? rows[0]->size(1) : -1, words = 4 * ((d + 127) / 128);
        for (int i = 0; i < 4; ++i) {
            const bool ok = i % 2 == 0 ? packed(*rows[i], at::kInt, {c.batch, count, c.heads, c.k, words}) : packed(*rows[i], at::kFloat, {c.batch, count, c.heads, c.k});
            if (!ok) { refuse("new rows are contiguous CUDA tensors (batch, count, heads, bits[, words of a plane]), as the cache and the table have them"); return nullptr; }
        }
        if (!same_device({c.t[0], rows[0], rows[1], rows[2], rows[3]})) return nullptr;
        const On on(*c.t[0]);
        return PyLong_FromLong(unlocked(p_amq_cache_append, data<const uint32_t>(rows[0]), data<const float>(rows[1]), data<const uint32_t>(rows[2]), data<const float>(rows[3]),
                                                  data<uint32_t>(c.t[0]), data<float>(c.t[1]), data<uint32_t>(c.t[2]), data<float>(c.t[3]),
                                                  (int)fits(c.pages), (int)fits(c.page_size), (int)fits(c.heads), (int)fits(d), (int)c.k, data<const int32_t>(c.table),
                                                  (int)fits(c.ld_table), (int)fits(c.max_pages), data<const int32_t>(c.lengths), (int)fits(c.batch), (int)fits(count),
                                                  on.stream()));
    });
}

decltype(&::amq_cache_attention) p_amq_cache_attention = nullptr;
decltype(&::amq_cache_attention_workspace_bytes) p_amq_cache_attention_workspace_bytes = nullptr;

// cache_attention(q, cache, table, lengths, scale, workspace, out)
PyObject* py_cache_attention(PyObject*, PyObject* const* args, Py_ssize_t nargs)
{
    if (!p_amq_cache_attention || nargs != 7) { PyErr_SetString(PyExc_TypeError, "cache_attention takes seven arguments of an opened library"); return nullptr; }
    return guarded([&]() -> PyObject* {
        const at::Tensor* q = tensor(args[0], "q");
        if (!q) return nullptr;
        if (!q->is_cuda() || q->scalar_type() != at::kFloat || q->dim() != 4 || (q->size(3) > 1 && q->stride(3) != 1)) {
            refuse("q must be a CUDA float32 tensor (batch, q_len, q_heads, d) with contiguous rows");
            return nullptr;
        }
        const int64_t batch = q->size(0), q_len = q->size(1), q_heads = q->size(2), d = q->size(3);
        Cache c;
        if (!cache_of(args[1], args[2], args[3], d, &c)) return nullptr;
        if (c.batch != batch) { refuse("q and table must agree in their first dimension"); return nullptr; }
        const float scale = (float)PyFloat_AsDouble(args[4]);
        if (PyErr_Occurred()) return nullptr;
        const at::Tensor *workspace = nullptr, *given = nullptr;
        if (args[5] != Py_None && !(workspace = tensor(args[5], "workspace"))) return nullptr;
        if (args[6] != Py_None && !(given = tensor(args[6], "out"))) return nullptr;
        if (workspace && (!workspace->is_cuda() || !workspace->is_contiguous())) { refuse("workspace must be a contiguous CUDA tensor"); return nullptr; }
        if (given && !packed(*given, at::kFloat, {batch, q_len, q_heads, d})) { refuse("out must be a contiguous CUDA float32 tensor of q's shape"); return nullptr; }
        if (!same_device({q, c.t[0], workspace, given})) return nullptr;
        const On on(*q);
        at::Tensor own, out = given ? *given : fresh({batch, q_len, q_heads, d}, at::kFloat, *q);
        if (!workspace) {
            const size_t bytes = p_amq_cache_attention_workspace_bytes((int)fits(batch), (int)fits(q_len), (int)fits(q_heads), (int)fits(c.heads), (int)fits(d),
                                                                       (int)fits(c.max_pages * c.page_size));
            if (bytes) { own = fresh({(int64_t)bytes}, at::kByte, *q); workspace = &own; }
        }
        const amq_status s = unlocked(
            p_amq_cache_attention, data<const float>(q), q->stride(0), q->stride(1), q->stride(2), data<const uint32_t>(c.t[0]), data<const float>(c.t[1]), data<const uint32_t>(c.t[2]),
            data<const float>(c.t[3]), (int)fits(c.pages), (int)fits(c.page_size), (int)fits(c.heads), (int)fits(d), (int)c.k, data<const int32_t>(c.table),
            (int)fits(c.ld_table), (int)fits(c.max_pages), data<const int32_t>(c.lengths), (int)fits(batch), (int)fits(q_len), (int)fits(q_heads), scale,
            static_cast<float*>(out.data_ptr()), workspace ? workspace->data_ptr() : nullptr, workspace ? workspace->nbytes() : 0, on.stream());
        return s == AMQ_OK ? THPVariable_Wrap(out) : PyLong_FromLong(s);
    });
}

// a contiguous part of a buffer as a tensor of its own
PyObject* part_of(const at::Tensor& buffer, int64_t first, at::IntArrayRef size, at::ScalarType type)
{
    at::Tensor t = at::detail::make_tensor<c10::TensorImpl>(c10::Storage(buffer.storage()), buffer.key_set(), c10::scalarTypeToTypeMeta(type));
    t.unsafeGetTensorImpl()->set_storage_offset(first);
    t.unsafeGetTensorImpl()->set_sizes_contiguous(size);
    return THPVariable_Wrap(t);
}

// beam_select(logits, scores, finished, eos) -> (scores, parents, tokens, finished), four parts of one allocation
PyObject* py_beam_select(PyObject*, PyObject* const* args, Py_ssize_t nargs)
{
    if (!p_amq_beam_select || nargs != 4) { PyErr_SetString(PyExc_TypeError, "beam_select takes four arguments of an opened library"); return nullptr; }
    return guarded([&]() -> PyObject* {
        const at::Tensor *logits = tensor(args[0], "logits"), *scores = logits ? tensor(args[1], "scores") : nullptr, *finished = nullptr;
        if (!scores || (args[2] != Py_None && !(finished = tensor(args[2], "finished")))) return nullptr;
        const long long eos = PyLong_AsLongLong(args[3]);
        if (PyErr_Occurred()) return nullptr;
        if (scores->dim() != 2 || !packed(*scores, at::kFloat, {scores->size(0), scores->size(1)})) {
            refuse("scores must be a contiguous CUDA float32 tensor (batch, beams)");
            return nullptr;
        }
        const int64_t batch = scores->size(0), beams = scores->size(1);
        if (logits->dim() != 2 || !shaped(*logits, at::kFloat, {batch * beams, logits->size(1)}) || leading(*logits) < 0) {
            refuse("logits must be a CUDA float32 tensor (batch * beams, vocabulary) with contiguous rows");
            return nullptr;
        }
        if (finished && !packed(*finished, at::kInt, {batch, beams})) { refuse("finished must be a contiguous CUDA int32 tensor (batch, beams)"); return nullptr; }
        if (!same_device({logits, scores, finished})) return nullptr;
        const On on(*scores);
        const int64_t n = batch * beams, step = (n + 3) / 4 * 4;         // (each part on 16 bytes)
        at::Tensor buffer = fresh({4 * step}, at::kInt, *scores);
        int32_t* at = static_cast<int32_t*>(buffer.data_ptr());
        const amq_status s = unlocked(p_amq_beam_select, data<const float>(logits), (int)fits(leading(*logits)), (int)fits(logits->size(1)), data<const float>(scores),
                                               finished ? data<const int32_t>(finished) : nullptr, eos == (int)eos ? (int)eos : -2, (int)fits(batch), (int)fits(beams),
                                               reinterpret_cast<float*>(at), at + step, at + 2 * step, at + 3 * step, on.stream());
        if (s != AMQ_OK) return PyLong_FromLong(s);
        PyObject* parts[4];
        for (int i = 0; i < 4; ++i) parts[i] = part_of(buffer, i * step, {batch, beams}, i == 0 ? at::kFloat : at::kInt);
        PyObject* answer = PyTuple_Pack(4, parts[0], parts[1], parts[2], parts[3]);
        for (PyObject* q : parts) Py_XDECREF(q);
        return answer;
    });
}

// amq_beam_reorder(states, out, parents): two sequences of tensors (batch, beams, ..), rows contiguous and at one stride, and the parents;
// the call's HOST arrays are made from them here
decltype(&::amq_beam_reorder) p_amq_beam_reorder = nullptr;

// row of a state: its bytes and the stride between rows; false (with a Python error) where it has none
bool state_rows(PyObject* o, const char* name, int64_t batch, int64_t beams, void** at, size_t* bytes, size_t* stride, at::Tensor* out)
{
    if (THPVariable_Check(o)) {
        const at::Tensor& t = THPVariable_Unpack(o);
        if (t.is_cuda() && t.dim() >= 2 && t.size(0) == batch && t.size(1) == beams) {
            int64_t row = 1;
            bool packed = true;
            for (int64_t d = t.dim() - 1; d >= 2; --d) {
                if (t.size(d) != 1 && t.stride(d) != row) packed = false;
                row *= t.size(d);
            }
            // the stride of one dimension where the other is not walked along
            int64_t step = beams > 1 ? t.stride(1) : batch > 1 ? t.stride(0) : row;
            if (batch > 1 && beams > 1 && t.stride(0) != beams * step) packed = false;
            if (packed && step >= row) {
                const size_t e = t.element_size();
                *at = t.data_ptr(); *bytes = row * e; *stride = step * e; *out = t;
                return true;
            }
        }
    }
    PyErr_Format(PyExc_TypeError, "%s must be CUDA tensors of shape (batch, beams, ..), as the parents have it, with contiguous rows at one stride", name);
    return false;
}

PyObject* py_amq_beam_reorder(PyObject*, PyObject* const* args, Py_ssize_t nargs)
{
    if (!p_amq_beam_reorder) { PyErr_SetString(PyExc_RuntimeError, "the library has not been opened"); return nullptr; }
    if (nargs != 3 || !THPVariable_Check(args[2])) { PyErr_SetString(PyExc_TypeError, "amq_beam_reorder(states, out, parents)"); return nullptr; }
    try {
        const at::Tensor& parents = THPVariable_Unpack(args[2]);
        if (!parents.is_cuda() || parents.scalar_type() != at::kInt || parents.dim() != 2 || !parents.is_contiguous()) {
            PyErr_SetString(PyExc_TypeError, "parents must be a contiguous CUDA tensor (batch, beams) of dtype int32");
            return nullptr;
        }
        PyObject* seq[2] = {PySequence_Fast(args[0], "states must be a sequence of tensors"), nullptr};
        if (seq[0]) seq[1] = PySequence_Fast(args[1], "out must be a sequence of tensors");
        PyObject* answer = nullptr;
        if (seq[1]) {
            const Py_ssize_t count = PySequence_Fast_GET_SIZE(seq[0]);
            if (PySequence_Fast_GET_SIZE(seq[1]) != count) {
                PyErr_SetString(PyExc_TypeError, "as many tensors to write as states");
            } else if (count > AMQ_MAX_STATES) {
                answer = PyLong_FromLong(AMQ_ERR_UNSUPPORTED);
            } else {
                void *src[AMQ_MAX_STATES], *dst[AMQ_MAX_STATES];
                size_t bytes[AMQ_MAX_STATES], from[AMQ_MAX_STATES], to[AMQ_MAX_STATES], same;
                bool ok = true;
                for (Py_ssize_t i = 0; ok && i < count; ++i) {
                    at::Tensor a, b;
                    ok = state_rows(PySequence_Fast_GET_ITEM(seq[0], i), "states", parents.size(0), parents.size(1), &src[i], &bytes[i], &from[i], &a) &&
                         state_rows(PySequence_Fast_GET_ITEM(seq[1], i), "the tensors to write", parents.size(0), parents.size(1), &dst[i], &same, &to[i], &b);
                    if (ok && (a.sizes() != b.sizes() || a.scalar_type() != b.scalar_type() || a.device() != b.device() || a.device() != parents.device())) {
                        PyErr_SetString(PyExc_TypeError, "a state and what it is written to must agree in shape, dtype and device, which is that of the parents");
                        ok = false;
                    }
                }
                if (ok) {
                    const On on(parents);
                    answer = PyLong_FromLong(unlocked(p_amq_beam_reorder, src, dst, bytes, from, to, (int)count, static_cast<const int32_t*>(parents.data_ptr()),
                                                      (int)parents.size(0), (int)parents.size(1), on.stream()));
                }
            }
        }
        Py_XDECREF(seq[0]);
        Py_XDECREF(seq[1]);
        return answer;
    } catch (const std::exception& e) {
        PyErr_SetString(PyExc_RuntimeError, e.what());
        return nullptr;
    }
}

// open(path): the library whose entry points the functions call
PyObject* py_open(PyObject*, PyObject* path)
{
    const char* p = PyUnicode_AsUTF8(path);
    if (!p) return nullptr;
    void* lib = dlopen(p, RTLD_NOW | RTLD_LOCAL);
    if (!lib) { PyErr_SetString(PyExc_ImportError, dlerror()); return nullptr; }
#define AMQ_LOOKUP(name)                                                                        \
    p_##name = reinterpret_cast<decltype(&::name)>(dlsym(lib, #name));                          \
    if (!p_##name) { PyErr_SetString(PyExc_ImportError, "missing entry point " #name); return nullptr; }
    AMQ_ENTRIES(AMQ_LOOKUP)
    AMQ_LOOKUP(amq_binary_gemm_act)
    AMQ_LOOKUP(amq_cache_append)
    AMQ_LOOKUP(amq_cache_attention)
    AMQ_LOOKUP(amq_beam_reorder)
    AMQ_LOOKUP(amq_cache_attention_workspace_bytes)
    Py_RETURN_NONE;
}

// empty(like, kind, d0, d1, ..): an uninitialised contiguous tensor on the device of `like`; kind 0 float32, 1 int32
PyObject* py_empty(PyObject*, PyObject* const* args, Py_ssize_t nargs)
{
    if (nargs < 2 || nargs > 8 || !THPVariable_Check(args[0])) {
        PyErr_SetString(PyExc_TypeError, "empty(like, kind, sizes..)");
        return nullptr;
    }
    int64_t size[6];
    const long kind = PyLong_AsLong(args[1]);
    for (Py_ssize_t i = 2; i < nargs; ++i) size[i - 2] = PyLong_AsLongLong(args[i]);
    if (PyErr_Occurred()) return nullptr;
    try {
        const at::Tensor& like = THPVariable_Unpack(args[0]);
        return THPVariable_Wrap(at::empty(at::IntArrayRef(size, nargs - 2),
                                          at::TensorOptions().dtype(kind ? at::kInt : at::kFloat).device(like.device())));
    } catch (const std::exception& e) {
        PyErr_SetString(PyExc_RuntimeError, e.what());
        return nullptr;
    }
}

#define AMQ_METHOD(name) {#name, (PyCFunction)(void (*)(void))py_##name, METH_FASTCALL, nullptr},
PyMethodDef methods[] = {
    AMQ_ENTRIES(AMQ_METHOD)
    AMQ_METHOD(amq_beam_reorder)
    AMQ_METHOD(binary_gemm_act) AMQ_METHOD(cache_append) AMQ_METHOD(cache_attention) AMQ_METHOD(beam_select)
    {"open", py_open, METH_O, nullptr},
    {"empty", (PyCFunction)(void (*)(void))py_empty, METH_FASTCALL, nullptr},
    {nullptr, nullptr, 0, nullptr},
};
PyModuleDef module = {PyModuleDef_HEAD_INIT, "_amq_binding", nullptr, -1, methods, nullptr, nullptr, nullptr, nullptr};

}  // namespace

PyMODINIT_FUNC PyInit__amq_binding() { return PyModule_Create(&module); }
