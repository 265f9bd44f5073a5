// Binding of the calls around the KV cache: checks torch tensors, allocates results, passes pointers to
// the C interface (include/retopk.h).  In C++ because the same in Python costs twice as much as a launch:
// a rotation of one token took 11.5 us of host time a call.
#include <torch/csrc/autograd/python_variable.h>
#include <torch/csrc/Exceptions.h>

#include <ATen/ATen.h>
#include <ATen/core/grad_mode.h>
#include <c10/cuda/CUDAGuard.h>
#include <c10/cuda/CUDAStream.h>

#include <map>
#include <memory>
#include <sstream>
#include <tuple>
#include <vector>

#include "../../include/retopk.h"

namespace {

PyObject* g_error = nullptr;                 // RetopkError

struct Failure { PyObject* type; std::string what; };

template <class... T> std::string text(const T&... parts) {
    std::ostringstream s;
    (s << ... << parts);
    return s.str();
}
template <class... T> [[noreturn]] void type_error(const T&... p) { throw Failure{PyExc_TypeError, text(p...)}; }
template <class... T> [[noreturn]] void value_error(const T&... p) { throw Failure{PyExc_ValueError, text(p...)}; }

void check(int64_t rc, const char* what) {
    if (rc < 0) throw Failure{g_error, text(what, " failed: ", retopk_strerror((int)rc), " (", rc, ")")};
}

const at::Tensor& tensor(PyObject* o, const char* what) {
    if (!THPVariable_Check(o)) type_error(what, ": expected a tensor, got ", Py_TYPE(o)->tp_name);
    return THPVariable_Unpack(o);
}
bool given(PyObject* o) { return o != Py_None; }

bool half_type(at::ScalarType t) { return t == at::kBFloat16 || t == at::kHalf; }
int type_code(at::ScalarType t) { return t == at::kBFloat16 ? RETOPK_BF16 : (t == at::kHalf ? RETOPK_FP16 : RETOPK_FP32); }

// A token-major tensor [n, heads, d] of 16-bit values whose heads lie d apart.
struct Rows { void* p; int64_t stride; };
Rows rows(const at::Tensor& t, const char* what, at::Device dev, at::ScalarType dt, int64_t n, int64_t heads, int64_t d) {
    if (t.device() != dev || t.scalar_type() != dt) type_error(what, ": expected ", dt, " on ", dev, ", got ", t.scalar_type(), " on ", t.device());
    if (t.dim() != 3 || t.size(0) != n || t.size(1) != heads || t.size(2) != d)
        value_error(what, ": expected shape [", n, ", ", heads, ", ", d, "], got ", t.sizes());
    if (t.stride(2) != 1 || (heads > 1 && t.stride(1) != d))
        value_error(what, ": the heads of a token have to lie ", d, " elements apart, strides are ", t.strides());
    return {t.data_ptr(), n > 1 ? t.stride(0) : heads * d};
}
const at::Tensor& half_rows(PyObject* o, const char* what) {
    const at::Tensor& t = tensor(o, what);
    if (!t.is_cuda() || !half_type(t.scalar_type())) type_error(what, ": expected a bf16 or fp16 CUDA tensor, got ", t.scalar_type(), " on ", t.device());
    if (t.dim() != 3) value_error(what, ": expected [tokens, heads, d], got ", t.sizes());
    return t;
}
const int32_t* ints(PyObject* o, const char* what, at::Device dev, int64_t n) {
    const at::Tensor& t = tensor(o, what);
    if (t.device() != dev || t.scalar_type() != at::kInt || !t.is_contiguous())
        type_error(what, ": expected a contiguous int32 tensor on ", dev, ", got ", t.scalar_type(), " on ", t.device());
    if (t.dim() != 1 || t.size(0) != n) value_error(what, ": expected shape [", n, "], got ", t.sizes());
    return t.data_ptr<int32_t>();
}
int64_t count(PyObject* o, const char* what) {
    const at::Tensor& t = tensor(o, what);
    if (t.dim() != 1) value_error(what, ": expected one dimension, got ", t.sizes());
    return t.size(0);
}
at::Tensor empty(at::IntArrayRef shape, const at::Tensor& like, at::ScalarType dt) { return at::empty(shape, like.options().dtype(dt)); }
void* stream_of(at::Device dev) { return c10::cuda::getCurrentCUDAStream(dev.index()).stream(); }

// Whether autograd would have to record a call on these tensors.
bool wants_gradient(std::initializer_list<const at::Tensor*> all) {
    if (!at::GradMode::is_enabled()) return false;
    for (const at::Tensor* t : all)
        if (t->defined() && t->requires_grad()) return true;
    return false;
}
// For calls without a backward pass: a gradient that would be lost is refused.
void no_gradient(const char* what, std::initializer_list<const at::Tensor*> all) {
    if (wants_gradient(all)) throw Failure{g_error, text(what, " has no gradient, but a tensor requires one: call it under torch.no_grad(), or detach")};
}

// Tells autograd that a tensor was written in place, so that a backward pass that saved it is refused.
void written(const at::Tensor& t) {
    if (t.defined() && !t.is_inference()) t.unsafeGetTensorImpl()->bump_version();
}

// The pages of one cache, as KVPages made them out.  It owns the tensors that `pages` points into.
struct Cache {
    retopk_pages_t pages;
    at::Device dev;
    at::Tensor tensors[4];                   // k, v, and of 4-bit pages k_scale, v_scale
    void* at[4];
    int64_t numel[4];
    std::map<std::tuple<int64_t, int64_t, int64_t>, int64_t> needs;      // workspace bytes by (B, T, H_q)
};
constexpr const char* CACHE = "retopk_cache";
Cache& cache_of(PyObject* o) {
    auto* c = static_cast<Cache*>(PyCapsule_GetPointer(o, CACHE));
    if (!c) throw python_error();
    for (int i = 0; i < 4; ++i) {
        const at::Tensor& t = c->tensors[i];
        if (t.defined() && (t.data_ptr() != c->at[i] || t.numel() != c->numel[i] || !t.is_contiguous() ||
                            t.storage().nbytes() < (size_t)(t.storage_offset() + t.numel()) * t.element_size()))
            throw Failure{g_error, "a tensor of the cache was resized or given other memory: wrap the tensors again"};
    }
    return *c;
}
retopk_pages_t pages_of(const Cache& c, int64_t B, PyObject* table) {
    retopk_pages_t p = c.pages;
    if (given(table)) {
        const at::Tensor& t = tensor(table, "block_table");
        if (t.device() != c.dev || t.scalar_type() != at::kInt || !t.is_contiguous())
            type_error("block_table: expected a contiguous int32 tensor on ", c.dev, ", got ", t.scalar_type(), " on ", t.device());
        if (t.dim() != 2 || t.size(0) != B) value_error("block_table: expected [", B, ", pages], got ", t.sizes());
        p.block_table = t.data_ptr<int32_t>();
        p.max_pages = t.size(1);
    }
    return p;
}

template <class F> PyObject* guarded(F f) {
    HANDLE_TH_ERRORS
    try {
        return f();
    } catch (const Failure& e) {
        PyErr_SetString(e.type, e.what.c_str());
        return nullptr;
    }
    END_HANDLE_TH_ERRORS
}
bool arity(Py_ssize_t n, Py_ssize_t want) {
    if (n != want) PyErr_Format(PyExc_TypeError, "expected %zd arguments, got %zd", want, n);
    return n == want;
}

// rope_apply(handle, d, q, k, positions, q_out, k_out, inverse) -> (q_out, k_out), or None where autograd has
// to record the call
PyObject* rope_apply(PyObject*, PyObject* const* a, Py_ssize_t n_args) {
    if (!arity(n_args, 8)) return nullptr;
    return guarded([&]() -> PyObject* {
        const auto* rope = static_cast<const retopk_rope*>(PyLong_AsVoidPtr(a[0]));
        if (!rope) { PyErr_Clear(); throw Failure{g_error, "the rotation was closed"}; }
        const int64_t d = PyLong_AsLongLong(a[1]);
        const at::Tensor& q = half_rows(a[2], "q");
        const at::Device dev = q.device();
        const at::ScalarType dt = q.scalar_type();
        const int64_t n = q.size(0), H_q = q.size(1);
        const Rows qi = rows(q, "q", dev, dt, n, H_q, d);
        const int32_t* pos = ints(a[4], "positions", dev, n);
        const int inverse = PyObject_IsTrue(a[7]);
        const at::Tensor none, &k_in = given(a[3]) ? tensor(a[3], "k") : none;
        if (given(a[5]) || given(a[6]))
            no_gradient("a rotation into given outputs", {&q, &k_in, given(a[5]) ? &tensor(a[5], "q_out") : &none, given(a[6]) ? &tensor(a[6], "k_out") : &none});
        else if (wants_gradient({&q, &k_in}))
            return Py_NewRef(Py_None);
        const c10::cuda::CUDAGuard guard(dev);
        const at::Tensor qo = given(a[5]) ? tensor(a[5], "q_out") : empty({n, H_q, d}, q, dt);
        const Rows qr = rows(qo, "q_out", dev, dt, n, H_q, d);
        at::Tensor ko;
        Rows ki = {nullptr, 0}, kr = {nullptr, 0};
        int64_t H_k = 0;
        if (given(a[3])) {
            const at::Tensor& k = half_rows(a[3], "k");
            H_k = k.size(1);
            ki = rows(k, "k", dev, dt, n, H_k, d);
            ko = given(a[6]) ? tensor(a[6], "k_out") : empty({n, H_k, d}, q, dt);
            kr = rows(ko, "k_out", dev, dt, n, H_k, d);
        }
        if (n > 0)
            check(retopk_rope_apply(rope, type_code(dt), n, pos, qi.p, qi.stride, qr.p, qr.stride, (int)H_q, ki.p, ki.stride, kr.p,
                                    kr.stride, (int)H_k, inverse, stream_of(dev)), "retopk_rope_apply");
        if (given(a[5])) written(qo);
        if (given(a[6])) written(ko);
        PyObject* out = PyTuple_New(2);
        PyTuple_SET_ITEM(out, 0, THPVariable_Wrap(qo));
        PyObject* second = ko.defined() ? THPVariable_Wrap(ko) : Py_NewRef(Py_None);
        PyTuple_SET_ITEM(out, 1, second);
        return out;
    });
}

// cache_new(format, H_kv, d, page_size, n_pages, k, v, k_scale or None, v_scale or None) -> capsule
PyObject* cache_new(PyObject*, PyObject* const* a, Py_ssize_t n_args) {
    if (!arity(n_args, 9)) return nullptr;
    return guarded([&]() -> PyObject* {
        int64_t v[5];
        for (int i = 0; i < 5; ++i) {
            v[i] = PyLong_AsLongLong(a[i]);
            if (v[i] == -1 && PyErr_Occurred()) throw python_error();
        }
        auto c = std::unique_ptr<Cache>(new Cache{{(int)v[0], (int)v[1], (int)v[2], (int)v[3], v[4], nullptr, nullptr, nullptr, nullptr, nullptr, 0},
                                                  tensor(a[5], "k").device(), {}, {}, {}, {}});
        for (int i = 0; i < 4; ++i)
            if (given(a[5 + i])) {
                c->tensors[i] = tensor(a[5 + i], "k, v, k_scale, v_scale");
                c->at[i] = c->tensors[i].data_ptr();
                c->numel[i] = c->tensors[i].numel();
            }
        c->pages.k = c->at[0];
        c->pages.v = c->at[1];
        c->pages.k_scale = c->at[2];
        c->pages.v_scale = c->at[3];
        PyObject* capsule = PyCapsule_New(c.get(), CACHE, [](PyObject* o) { delete static_cast<Cache*>(PyCapsule_GetPointer(o, CACHE)); });
        if (capsule) c.release();
        return capsule;
    });
}

// append(cache, k_new, v_new, seq_lens, block_table, cu_new, rope handle or 0, q, q_out) -> q_out
PyObject* append(PyObject*, PyObject* const* a, Py_ssize_t n_args) {
    if (!arity(n_args, 9)) return nullptr;
    return guarded([&]() -> PyObject* {
        const Cache& c = cache_of(a[0]);
        const at::Tensor &k = half_rows(a[1], "k_new"), &v = half_rows(a[2], "v_new");
        const at::ScalarType dt = k.scalar_type();
        const int64_t n = k.size(0), H = c.pages.H_kv, d = c.pages.d, B = count(a[3], "seq_lens");
        const int32_t* lens = ints(a[3], "seq_lens", c.dev, B);
        const Rows kr = rows(k, "k_new", c.dev, dt, n, H, d), vr = rows(v, "v_new", c.dev, dt, n, H, d);
        const int32_t* cu = given(a[5]) ? ints(a[5], "cu_new", c.dev, B + 1) : nullptr;
        if (!cu && B > 0 && n % B) value_error(n, " new tokens do not divide among ", B, " sequences: pass cu_new");
        const auto* rope = static_cast<const retopk_rope*>(PyLong_AsVoidPtr(a[6]));
        const retopk_pages_t pages = pages_of(c, B, a[4]);
        const at::Tensor none;
        const at::Tensor* pg = c.tensors;
        no_gradient("append", {&k, &v, &pg[0], &pg[1], &pg[2], &pg[3], given(a[7]) ? &tensor(a[7], "q") : &none, given(a[8]) ? &tensor(a[8], "q_out") : &none});
        const c10::cuda::CUDAGuard guard(c.dev);
        at::Tensor qo;
        Rows qi = {nullptr, 0}, qr = {nullptr, 0};
        int64_t H_q = 0;
        if (given(a[7])) {
            if (!rope) value_error("q is rotated with the keys: pass rope");
            const at::Tensor& q = half_rows(a[7], "q");
            H_q = q.size(1);
            qi = rows(q, "q", c.dev, dt, n, H_q, d);
            qo = given(a[8]) ? tensor(a[8], "q_out") : empty({n, H_q, d}, q, dt);
            qr = rows(qo, "q_out", c.dev, dt, n, H_q, d);
        }
        if (n > 0)
            check(retopk_kv_append(&pages, (int)B, lens, cu, n, type_code(dt), kr.p, kr.stride, vr.p, vr.stride, rope, qi.p, qi.stride, qr.p,
                                   qr.stride, (int)H_q, stream_of(c.dev)), "retopk_kv_append");
        for (const at::Tensor& t : c.tensors) written(t);
        if (given(a[7]) && given(a[8])) written(qo);
        return qo.defined() ? THPVariable_Wrap(qo) : Py_NewRef(given(a[8]) ? a[8] : Py_None);
    });
}

// gather(cache, k_out, v_out, seq_lens, block_table, first)
PyObject* gather(PyObject*, PyObject* const* a, Py_ssize_t n_args) {
    if (!arity(n_args, 6)) return nullptr;
    return guarded([&]() -> PyObject* {
        const Cache& c = cache_of(a[0]);
        if (!given(a[1]) && !given(a[2])) value_error("gather: pass k_out, v_out or both");
        const at::Tensor& ref = tensor(given(a[1]) ? a[1] : a[2], "k_out, v_out");
        if (ref.dim() != 4 || ref.size(1) != c.pages.H_kv || ref.size(3) != c.pages.d)
            value_error("k_out, v_out: expected [B, ", c.pages.H_kv, ", rows, ", c.pages.d, "], got ", ref.sizes());
        const at::ScalarType dt = ref.scalar_type();
        if (!half_type(dt) && dt != at::kFloat) type_error("k_out, v_out: bf16, fp16 or fp32, got ", dt);
        void* out[2] = {nullptr, nullptr};
        for (int i = 0; i < 2; ++i)
            if (given(a[1 + i])) {
                const at::Tensor& t = tensor(a[1 + i], "k_out, v_out");
                if (t.device() != c.dev || t.scalar_type() != dt || t.sizes() != ref.sizes() || !t.is_contiguous())
                    type_error("k_out, v_out: contiguous ", dt, " ", ref.sizes(), " on ", c.dev);
                no_gradient("gather", {&t, &c.tensors[0], &c.tensors[1]});
                out[i] = t.data_ptr();
            }
        const int64_t B = ref.size(0);
        const int32_t* lens = ints(a[3], "seq_lens", c.dev, B);
        const int32_t* first = given(a[5]) ? ints(a[5], "first", c.dev, B) : nullptr;
        const retopk_pages_t pages = pages_of(c, B, a[4]);
        if (ref.numel() > 0) {
            const c10::cuda::CUDAGuard guard(c.dev);
            check(retopk_kv_gather(&pages, (int)B, lens, first, ref.size(2), type_code(dt), out[0], out[1], stream_of(c.dev)), "retopk_kv_gather");
            for (int i = 0; i < 2; ++i)
                if (given(a[1 + i])) written(tensor(a[1 + i], "k_out, v_out"));
        }
        return Py_NewRef(Py_None);
    });
}

// Rows that a sequence can have.
int64_t keys_of(const retopk_pages_t& p) { return p.block_table ? p.max_pages * p.page_size : p.page_size; }

// Queries [B, H_q, d] or [B, T, H_q, d], and results of their shape.
struct Queries {
    const at::Tensor& q;
    int64_t B, T, H_q, stride;
    at::ScalarType dt;
};
Queries queries(PyObject* o, const Cache& c) {
    const int64_t d = c.pages.d;
    const at::Tensor& q = tensor(o, "q");
    if (q.device() != c.dev || !half_type(q.scalar_type())) type_error("q: expected bf16 or fp16 on ", c.dev, ", got ", q.scalar_type(), " on ", q.device());
    if ((q.dim() != 3 && q.dim() != 4) || q.size(-1) != d) value_error("q: expected [B, H_q, ", d, "] or [B, T, H_q, ", d, "], got ", q.sizes());
    const bool four = q.dim() == 4;
    const int64_t B = q.size(0), T = four ? q.size(1) : 1, H_q = q.size(-2);
    if (q.stride(-1) != 1 || (H_q > 1 && q.stride(-2) != d) || (four && T > 1 && B > 1 && q.stride(0) != T * q.stride(1)))
        value_error("q: tokens have to lie one stride apart and heads ", d, " elements apart, strides are ", q.strides());
    return {q, B, T, H_q, B * T <= 1 ? H_q * d : (T == 1 ? q.stride(0) : q.stride(1)), q.scalar_type()};
}
Queries queries_of_pages(PyObject* o, const Cache& c) {
    const Queries q = queries(o, c);
    if (q.dt != c.tensors[0].scalar_type()) type_error("q: this cache holds ", c.tensors[0].scalar_type(), ", got ", q.dt);
    return q;
}
void sixteen_bits(const Cache& c, const char* what) {
    if (c.pages.format == RETOPK_PAGES_Q4) type_error(what, " reads 16-bit pages, this cache holds 4-bit values");
}
at::Tensor output(PyObject* o, const Queries& x, const Cache& c) {
    if (!given(o)) return empty(x.q.sizes(), x.q, x.dt);
    const at::Tensor& out = tensor(o, "out");
    if (out.device() != c.dev || out.scalar_type() != x.dt || out.sizes() != x.q.sizes() || !out.is_contiguous())
        type_error("out: contiguous ", x.dt, " ", x.q.sizes(), " on ", c.dev);
    return out;
}
float* log_sums(PyObject* o, const Queries& x, const Cache& c) {
    if (!given(o)) return nullptr;
    const at::Tensor& l = tensor(o, "lse");
    if (l.device() != c.dev || l.scalar_type() != at::kFloat || l.sizes() != x.q.sizes().slice(0, x.q.dim() - 1) || !l.is_contiguous())
        type_error("lse: contiguous fp32 ", x.q.sizes().slice(0, x.q.dim() - 1), " on ", c.dev);
    return l.data_ptr<float>();
}
double scale_of(PyObject* o, int64_t d) { return given(o) ? PyFloat_AsDouble(o) : 1.0 / std::sqrt((double)d); }
// from torch's allocator: tied to this stream (and, under capture, to the graph's own pool)
at::Tensor workspace(int64_t bytes, const at::Tensor& like) { return empty({bytes}, like, at::kByte); }

// attend(cache, q, seq_lens, block_table, scale or None, window, out, lse) -> out
PyObject* attend(PyObject*, PyObject* const* a, Py_ssize_t n_args) {
    if (!arity(n_args, 8)) return nullptr;
    return guarded([&]() -> PyObject* {
        Cache& c = cache_of(a[0]);
        if (c.pages.format != RETOPK_PAGES_Q4) type_error("attend reads 4-bit pages, this cache holds 16-bit values");
        const Queries x = queries(a[1], c);
        const int32_t* lens = ints(a[2], "seq_lens", c.dev, x.B);
        const retopk_pages_t pages = pages_of(c, x.B, a[3]);
        const at::Tensor none;
        no_gradient("attend", {&x.q, &c.tensors[2], &c.tensors[3], given(a[6]) ? &tensor(a[6], "out") : &none, given(a[7]) ? &tensor(a[7], "lse") : &none});
        const double scale = scale_of(a[4], c.pages.d);
        const int64_t window = PyLong_AsLongLong(a[5]);
        if (PyErr_Occurred()) throw python_error();
        const c10::cuda::CUDAGuard guard(c.dev);
        const at::Tensor out = output(a[6], x, c);
        float* lse = log_sums(a[7], x, c);
        if (x.B > 0) {
            int64_t& need = c.needs[{x.B, x.T, x.H_q}];
            if (need <= 0) {
                need = retopk_q4_attention_workspace((int)x.B, (int)x.T, (int)x.H_q, c.pages.H_kv, c.pages.d);
                check(need, "retopk_q4_attention_workspace");
            }
            const at::Tensor ws = workspace(need, x.q);
            check(retopk_q4_attention(&pages, (int)x.B, (int)x.T, (int)x.H_q, lens, type_code(x.dt), x.q.data_ptr(), x.stride, (float)scale,
                                      window, out.data_ptr(), lse, ws.data_ptr(), need, stream_of(c.dev)), "retopk_q4_attention");
            if (given(a[6])) written(out);
            if (given(a[7])) written(tensor(a[7], "lse"));
        }
        return THPVariable_Wrap(out);
    });
}

// attend_shared(cache, q, seq_lens, block_table, cu_groups or None, shared_lens or None, scale or None, out, lse) -> out
PyObject* attend_shared(PyObject*, PyObject* const* a, Py_ssize_t n_args) {
    if (!arity(n_args, 9)) return nullptr;
    return guarded([&]() -> PyObject* {
        const Cache& c = cache_of(a[0]);
        sixteen_bits(c, "attend_shared");
        const Queries x = queries_of_pages(a[1], c);
        const int32_t* lens = ints(a[2], "seq_lens", c.dev, x.B);
        const retopk_pages_t pages = pages_of(c, x.B, a[3]);
        if (given(a[4]) != given(a[5])) value_error("cu_groups and shared_lens go together");
        int64_t groups = 0;
        const int32_t *cu = nullptr, *shared = nullptr;
        if (given(a[4])) {
            const at::Tensor& t = tensor(a[5], "shared_lens");
            if (t.dim() != 1) value_error("shared_lens: expected one length per group, got ", t.sizes());
            groups = t.size(0);
            shared = ints(a[5], "shared_lens", c.dev, groups);
            cu = ints(a[4], "cu_groups", c.dev, groups + 1);
            if (groups > x.B) value_error(groups, " groups of ", x.B, " sequences");
        }
        const at::Tensor none;
        no_gradient("attend_shared", {&x.q, &c.tensors[0], &c.tensors[1], given(a[7]) ? &tensor(a[7], "out") : &none, given(a[8]) ? &tensor(a[8], "lse") : &none});
        const double scale = scale_of(a[6], c.pages.d);
        if (PyErr_Occurred()) throw python_error();
        const c10::cuda::CUDAGuard guard(c.dev);
        const at::Tensor out = output(a[7], x, c);
        float* lse = log_sums(a[8], x, c);
        if (x.B > 0) {
            const int64_t need = retopk_shared_attention_workspace((int)x.B, (int)groups, (int)x.T, (int)x.H_q, c.pages.H_kv, c.pages.d, keys_of(pages));
            check(need, "retopk_shared_attention_workspace");
            const at::Tensor ws = workspace(need, x.q);
            check(retopk_shared_attention(&pages, (int)x.B, (int)x.T, (int)x.H_q, lens, (int)groups, cu, shared, x.q.data_ptr(), x.stride,
                                          (float)scale, out.data_ptr(), lse, ws.data_ptr(), need, stream_of(c.dev)), "retopk_shared_attention");
            if (given(a[7])) written(out);
            if (given(a[8])) written(tensor(a[8], "lse"));
        }
        return THPVariable_Wrap(out);
    });
}

// The bounds of a cache's blocks [n_pages, H_kv, page_size / block, 2, d].
const at::Tensor& bounds_of(PyObject* o, const Cache& c, int64_t block) {
    sixteen_bits(c, "a block index");
    const at::Tensor& t = tensor(o, "bounds");
    if (t.device() != c.dev || t.scalar_type() != c.tensors[0].scalar_type() || !t.is_contiguous())
        type_error("bounds: contiguous ", c.tensors[0].scalar_type(), " on ", c.dev);
    const int64_t want[5] = {c.pages.n_pages, c.pages.H_kv, block > 0 ? c.pages.page_size / block : 0, 2, c.pages.d};
    if (t.sizes() != at::IntArrayRef(want, 5)) value_error("bounds: expected ", at::IntArrayRef(want, 5), ", got ", t.sizes());
    return t;
}
int64_t integer(PyObject* o) {
    const int64_t v = PyLong_AsLongLong(o);
    if (v == -1 && PyErr_Occurred()) throw python_error();
    return v;
}
// A count as the C interface takes it; one that it would not hold is one that it refuses.
int clipped(int64_t n) { return (int)(n < 2147483647 ? n : 2147483647); }
int small(PyObject* o, const char* what) {
    const int64_t v = integer(o);
    if (v < -2147483647 || v > 2147483647) value_error(what, ": out of range, got ", v);
    return (int)v;
}

// block_update(cache, bounds, block, seq_lens, block_table, n_new)
PyObject* block_update(PyObject*, PyObject* const* a, Py_ssize_t n_args) {
    if (!arity(n_args, 6)) return nullptr;
    return guarded([&]() -> PyObject* {
        const Cache& c = cache_of(a[0]);
        const int block = small(a[2], "block");
        const at::Tensor& bounds = bounds_of(a[1], c, block);
        const int64_t B = count(a[3], "seq_lens"), n_new = integer(a[5]);
        const int32_t* lens = ints(a[3], "seq_lens", c.dev, B);
        const retopk_pages_t pages = pages_of(c, B, a[4]);
        no_gradient("update", {&bounds, &c.tensors[0]});
        if (B > 0) {
            const c10::cuda::CUDAGuard guard(c.dev);
            check(retopk_block_update(&pages, block, bounds.data_ptr(), clipped(B), lens, n_new, stream_of(c.dev)), "retopk_block_update");
            written(bounds);
        }
        return Py_NewRef(Py_None);
    });
}

// block_select(cache, bounds, block, q, seq_lens, block_table, keep, first, last, out) -> blocks
PyObject* block_select(PyObject*, PyObject* const* a, Py_ssize_t n_args) {
    if (!arity(n_args, 10)) return nullptr;
    return guarded([&]() -> PyObject* {
        const Cache& c = cache_of(a[0]);
        const int block = small(a[2], "block"), keep = small(a[6], "keep"), first = small(a[7], "first"), last = small(a[8], "last");
        const at::Tensor& bounds = bounds_of(a[1], c, block);
        const Queries x = queries_of_pages(a[3], c);
        const int32_t* lens = ints(a[4], "seq_lens", c.dev, x.B);
        const retopk_pages_t pages = pages_of(c, x.B, a[5]);
        if (keep < 1 || first < 0 || last < 1 || first > keep - last) value_error("keep ", keep, ", first ", first, ", last ", last, ": last >= 1, first + last <= keep");
        no_gradient("select", {&x.q, &bounds});
        const c10::cuda::CUDAGuard guard(c.dev);
        std::vector<int64_t> shape = {x.B};
        if (x.q.dim() == 4) shape.push_back(x.T);
        shape.push_back(c.pages.H_kv);
        shape.push_back(keep);
        at::Tensor out;
        if (given(a[9])) {
            out = tensor(a[9], "out");
            if (out.device() != c.dev || out.scalar_type() != at::kInt || out.sizes() != shape || !out.is_contiguous())
                type_error("out: contiguous int32 ", at::IntArrayRef(shape), " on ", c.dev);
        } else {
            out = empty(shape, x.q, at::kInt);
        }
        if (x.B > 0) {
            const int64_t capacity = keys_of(pages);
            const int64_t need = retopk_block_select_workspace((int)x.B, (int)x.T, (int)x.H_q, c.pages.H_kv, c.pages.d, (capacity + block - 1) / block);
            check(need, "retopk_block_select_workspace");
            const at::Tensor ws = workspace(need, x.q);
            check(retopk_block_select(&pages, block, bounds.data_ptr(), (int)x.B, (int)x.T, (int)x.H_q, lens, x.q.data_ptr(), x.stride, keep, first,
                                      last, out.data_ptr<int32_t>(), ws.data_ptr(), need, stream_of(c.dev)), "retopk_block_select");
            if (given(a[9])) written(out);
        }
        return THPVariable_Wrap(out);
    });
}

// block_attend(cache, block, q, seq_lens, blocks, block_table, scale or None, out, lse) -> out
PyObject* block_attend(PyObject*, PyObject* const* a, Py_ssize_t n_args) {
    if (!arity(n_args, 9)) return nullptr;
    return guarded([&]() -> PyObject* {
        const Cache& c = cache_of(a[0]);
        sixteen_bits(c, "attend");
        const int block = small(a[1], "block");
        const Queries x = queries_of_pages(a[2], c);
        const int32_t* lens = ints(a[3], "seq_lens", c.dev, x.B);
        const at::Tensor& blocks = tensor(a[4], "blocks");
        if (blocks.device() != c.dev || blocks.scalar_type() != at::kInt || !blocks.is_contiguous())
            type_error("blocks: expected a contiguous int32 tensor on ", c.dev, ", got ", blocks.scalar_type(), " on ", blocks.device());
        std::vector<int64_t> shape = {x.B};
        if (x.q.dim() == 4) shape.push_back(x.T);
        shape.push_back(c.pages.H_kv);
        if (blocks.dim() != (int64_t)shape.size() + 1 || blocks.sizes().slice(0, shape.size()) != shape || blocks.size(-1) < 1 || blocks.size(-1) > 2147483647)
            value_error("blocks: expected ", at::IntArrayRef(shape), " and a list of blocks each, got ", blocks.sizes());
        const int keep = (int)blocks.size(-1);
        const retopk_pages_t pages = pages_of(c, x.B, a[5]);
        const at::Tensor none;
        no_gradient("attend", {&x.q, &c.tensors[0], &c.tensors[1], given(a[7]) ? &tensor(a[7], "out") : &none, given(a[8]) ? &tensor(a[8], "lse") : &none});
        const double scale = scale_of(a[6], c.pages.d);
        if (PyErr_Occurred()) throw python_error();
        const c10::cuda::CUDAGuard guard(c.dev);
        const at::Tensor out = output(a[7], x, c);
        float* lse = log_sums(a[8], x, c);
        if (x.B > 0) {
            const int64_t need = retopk_block_attention_workspace((int)x.B, (int)x.T, (int)x.H_q, c.pages.H_kv, c.pages.d, keep, block);
            check(need, "retopk_block_attention_workspace");
            const at::Tensor ws = workspace(need, x.q);
            check(retopk_block_attention(&pages, block, (int)x.B, (int)x.T, (int)x.H_q, lens, keep, blocks.data_ptr<int32_t>(), x.q.data_ptr(),
                                         x.stride, (float)scale, out.data_ptr(), lse, ws.data_ptr(), need, stream_of(c.dev)), "retopk_block_attention");
            if (given(a[7])) written(out);
            if (given(a[8])) written(tensor(a[8], "lse"));
        }
        return THPVariable_Wrap(out);
    });
}

// copy_pages(cache, src, dst, rows or None); block_copy(cache, bounds, block, src, dst)
PyObject* copy_pages(PyObject*, PyObject* const* a, Py_ssize_t n_args) {
    if (!arity(n_args, 4)) return nullptr;
    return guarded([&]() -> PyObject* {
        const Cache& c = cache_of(a[0]);
        const int64_t n = count(a[1], "src");
        const int32_t *src = ints(a[1], "src", c.dev, n), *dst = ints(a[2], "dst", c.dev, n);
        const int32_t* rows_ = given(a[3]) ? ints(a[3], "rows", c.dev, n) : nullptr;
        no_gradient("copy_pages", {&c.tensors[0], &c.tensors[1], &c.tensors[2], &c.tensors[3]});
        if (n > 0) {
            const c10::cuda::CUDAGuard guard(c.dev);
            check(retopk_pages_copy(&c.pages, n, src, dst, rows_, stream_of(c.dev)), "retopk_pages_copy");
            for (const at::Tensor& t : c.tensors) written(t);
        }
        return Py_NewRef(Py_None);
    });
}
PyObject* block_copy(PyObject*, PyObject* const* a, Py_ssize_t n_args) {
    if (!arity(n_args, 5)) return nullptr;
    return guarded([&]() -> PyObject* {
        const Cache& c = cache_of(a[0]);
        const int block = small(a[2], "block");
        const at::Tensor& bounds = bounds_of(a[1], c, block);
        const int64_t n = count(a[3], "src");
        const int32_t *src = ints(a[3], "src", c.dev, n), *dst = ints(a[4], "dst", c.dev, n);
        no_gradient("copy_pages", {&bounds});
        if (n > 0) {
            const c10::cuda::CUDAGuard guard(c.dev);
            check(retopk_block_copy(&c.pages, block, bounds.data_ptr(), n, src, dst, stream_of(c.dev)), "retopk_block_copy");
            written(bounds);
        }
        return Py_NewRef(Py_None);
    });
}

// The pool of a call, its table and its sequences: (refs, scratch, page_size, block_table, lens).
struct Pooled {
    retopk_pool_t pool;
    at::Device dev;
    const at::Tensor& table;
    int64_t B;
    int32_t* lens;
};
Pooled pooled(PyObject* const* a, const char* lens_name) {
    const at::Tensor &refs = tensor(a[0], "refs"), &scratch = tensor(a[1], "scratch"), &table = tensor(a[3], "block_table");
    const at::Device dev = refs.device();
    if (!refs.is_cuda()) type_error("refs: expected a CUDA tensor, got one on ", dev);
    const int64_t n = count(a[0], "refs");
    ints(a[0], "refs", dev, n);
    ints(a[1], "scratch", dev, n + RETOPK_POOL_SCRATCH);
    if (table.device() != dev || table.scalar_type() != at::kInt || !table.is_contiguous())
        type_error("block_table: expected a contiguous int32 tensor on ", dev, ", got ", table.scalar_type(), " on ", table.device());
    if (table.dim() != 2) value_error("block_table: expected [sequences, pages], got ", table.sizes());
    const int64_t B = table.size(0);
    if (B > 0 && table.size(1) == 0) value_error("block_table has no room: ", table.sizes());
    const int32_t* lens = ints(a[4], lens_name, dev, B);
    return {{refs.data_ptr<int32_t>(), scratch.data_ptr<int32_t>(), n, small(a[2], "page_size")}, dev, table, B, const_cast<int32_t*>(lens)};
}

// pool_reserve(refs, scratch, page_size, block_table, old_lens, new_lens)
PyObject* pool_reserve(PyObject*, PyObject* const* a, Py_ssize_t n_args) {
    if (!arity(n_args, 6)) return nullptr;
    return guarded([&]() -> PyObject* {
        const Pooled p = pooled(a, "old_lens");
        const int32_t* now = ints(a[5], "new_lens", p.dev, p.B);
        if (p.B > 0) {
            const c10::cuda::CUDAGuard guard(p.dev);
            check(retopk_pool_reserve(&p.pool, clipped(p.B), p.lens, now, p.table.data_ptr<int32_t>(), p.table.size(1), stream_of(p.dev)), "retopk_pool_reserve");
            for (int i : {0, 1, 3}) written(tensor(a[i], "refs, block_table"));
        }
        return Py_NewRef(Py_None);
    });
}

// pool_fork(refs, scratch, page_size, block_table, seq_lens, parents, children) -> (src, dst, rows)
PyObject* pool_fork(PyObject*, PyObject* const* a, Py_ssize_t n_args) {
    if (!arity(n_args, 7)) return nullptr;
    return guarded([&]() -> PyObject* {
        const Pooled p = pooled(a, "seq_lens");
        const int64_t n = count(a[5], "parents");
        const int32_t *parents = ints(a[5], "parents", p.dev, n), *children = ints(a[6], "children", p.dev, n);
        if (n > 65535) value_error("at most 65535 forks, got ", n);
        const c10::cuda::CUDAGuard guard(p.dev);
        at::Tensor out[3];
        for (at::Tensor& t : out) t = empty({n}, p.table, at::kInt);
        if (n > 0 && p.B == 0) value_error("forks in a block_table of no sequences");
        if (n > 0) {
            check(retopk_pool_fork(&p.pool, clipped(p.B), p.lens, p.table.data_ptr<int32_t>(), p.table.size(1), (int)n, parents, children,
                                   out[0].data_ptr<int32_t>(), out[1].data_ptr<int32_t>(), out[2].data_ptr<int32_t>(), stream_of(p.dev)), "retopk_pool_fork");
            for (int i : {0, 1, 3, 4}) written(tensor(a[i], "refs, block_table, seq_lens"));
        }
        PyObject* r = PyTuple_New(3);
        for (int i = 0; i < 3; ++i) PyTuple_SET_ITEM(r, i, THPVariable_Wrap(out[i]));
        return r;
    });
}

// pool_free(refs, scratch, page_size, block_table, seq_lens, rows or None)
PyObject* pool_free(PyObject*, PyObject* const* a, Py_ssize_t n_args) {
    if (!arity(n_args, 6)) return nullptr;
    return guarded([&]() -> PyObject* {
        const Pooled p = pooled(a, "seq_lens");
        const int64_t n = given(a[5]) ? count(a[5], "rows") : p.B;
        const int32_t* rows_ = given(a[5]) ? ints(a[5], "rows", p.dev, n) : nullptr;
        if (n > 2147483647) value_error("rows: too many, ", n);
        if (n > 0 && p.B > 0) {
            const c10::cuda::CUDAGuard guard(p.dev);
            check(retopk_pool_free(&p.pool, clipped(p.B), p.lens, p.table.data_ptr<int32_t>(), p.table.size(1), (int)n, rows_, stream_of(p.dev)), "retopk_pool_free");
            for (int i : {0, 1, 4}) written(tensor(a[i], "refs, seq_lens"));
        }
        return Py_NewRef(Py_None);
    });
}

// pool_compact(refs, scratch, page_size, block_table, seq_lens) -> (src, dst)
PyObject* pool_compact(PyObject*, PyObject* const* a, Py_ssize_t n_args) {
    if (!arity(n_args, 5)) return nullptr;
    return guarded([&]() -> PyObject* {
        const Pooled p = pooled(a, "seq_lens");
        if (p.B == 0) value_error("block_table of no sequences");
        const c10::cuda::CUDAGuard guard(p.dev);
        const at::Tensor src = empty({p.pool.n_pages / 2}, p.table, at::kInt), dst = empty({p.pool.n_pages / 2}, p.table, at::kInt);
        check(retopk_pool_compact(&p.pool, clipped(p.B), p.lens, p.table.data_ptr<int32_t>(), p.table.size(1), src.data_ptr<int32_t>(),
                                  dst.data_ptr<int32_t>(), stream_of(p.dev)), "retopk_pool_compact");
        for (int i : {0, 1, 3}) written(tensor(a[i], "refs, block_table"));
        PyObject* r = PyTuple_New(2);
        PyTuple_SET_ITEM(r, 0, THPVariable_Wrap(src));
        PyTuple_SET_ITEM(r, 1, THPVariable_Wrap(dst));
        return r;
    });
}

PyObject* set_error(PyObject*, PyObject* type) {
    Py_XSETREF(g_error, Py_NewRef(type));
    return Py_NewRef(Py_None);
}

#define FAST(f) {#f, reinterpret_cast<PyCFunction>(reinterpret_cast<void (*)()>(f)), METH_FASTCALL, nullptr}
PyMethodDef METHODS[] = {FAST(rope_apply), FAST(cache_new), FAST(append), FAST(gather), FAST(attend), FAST(attend_shared), FAST(block_update), FAST(block_select),
                         FAST(block_attend), FAST(block_copy), FAST(copy_pages), FAST(pool_reserve), FAST(pool_fork), FAST(pool_free), FAST(pool_compact),
                         {"set_error", set_error, METH_O, nullptr}, {nullptr, nullptr, 0, nullptr}};
PyModuleDef MODULE = {PyModuleDef_HEAD_INIT, "_paged", "Calls around the KV cache (see paged.py).", -1, METHODS, nullptr, nullptr, nullptr, nullptr};

}  // namespace

PyMODINIT_FUNC PyInit__paged() {
    PyObject* m = PyModule_Create(&MODULE);
    if (m && PyModule_AddStringConstant(m, "built_for", BUILT_FOR) != 0) Py_CLEAR(m);      // compared by paged.py
    return m;
}
