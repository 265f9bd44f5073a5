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
int64_t sequences(PyObject* lens) {
    const at::Tensor& t = tensor(lens, "seq_lens");
    if (t.dim() != 1) value_error("seq_lens: expected one length per sequence, got ", t.sizes());
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
        const int64_t n = k.size(0), H = c.pages.H_kv, d = c.pages.d, B = sequences(a[3]);
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

// attend(cache, q, seq_lens, block_table, scale or None, window, out, lse) -> out
PyObject* attend(PyObject*, PyObject* const* a, Py_ssize_t n_args) {
    if (!arity(n_args, 8)) return nullptr;
    return guarded([&]() -> PyObject* {
        Cache& c = cache_of(a[0]);
        if (c.pages.format != RETOPK_PAGES_Q4) type_error("attend reads 4-bit pages, this cache holds 16-bit values");
        const int64_t d = c.pages.d;
        const at::Tensor& q = tensor(a[1], "q");
        if (q.device() != c.dev || !half_type(q.scalar_type())) type_error("q: expected bf16 or fp16 on ", c.dev, ", got ", q.scalar_type(), " on ", q.device());
        if ((q.dim() != 3 && q.dim() != 4) || q.size(-1) != d) value_error("q: expected [B, H_q, ", d, "] or [B, T, H_q, ", d, "], got ", q.sizes());
        const bool four = q.dim() == 4;
        const int64_t B = q.size(0), T = four ? q.size(1) : 1, H_q = q.size(-2);
        if (q.stride(-1) != 1 || (H_q > 1 && q.stride(-2) != d) || (four && T > 1 && B > 1 && q.stride(0) != T * q.stride(1)))
            value_error("q: tokens have to lie one stride apart and heads ", d, " elements apart, strides are ", q.strides());
        const int64_t q_stride = B * T <= 1 ? H_q * d : (T == 1 ? q.stride(0) : q.stride(1));
        const int32_t* lens = ints(a[2], "seq_lens", c.dev, B);
        const retopk_pages_t pages = pages_of(c, B, a[3]);
        const at::Tensor none;
        no_gradient("attend", {&q, &c.tensors[2], &c.tensors[3], given(a[6]) ? &tensor(a[6], "out") : &none, given(a[7]) ? &tensor(a[7], "lse") : &none});
        const double scale = given(a[4]) ? PyFloat_AsDouble(a[4]) : 1.0 / std::sqrt((double)d);
        const int64_t window = PyLong_AsLongLong(a[5]);
        if (PyErr_Occurred()) throw python_error();
        const c10::cuda::CUDAGuard guard(c.dev);
        at::Tensor out;
        if (given(a[6])) {
            out = tensor(a[6], "out");
            if (out.device() != c.dev || out.scalar_type() != q.scalar_type() || out.sizes() != q.sizes() || !out.is_contiguous())
                type_error("out: contiguous ", q.scalar_type(), " ", q.sizes(), " on ", c.dev);
        } else {
            out = empty(q.sizes(), q, q.scalar_type());
        }
        float* lse = nullptr;
        if (given(a[7])) {
            const at::Tensor& l = tensor(a[7], "lse");
            if (l.device() != c.dev || l.scalar_type() != at::kFloat || l.sizes() != q.sizes().slice(0, q.dim() - 1) || !l.is_contiguous())
                type_error("lse: contiguous fp32 ", q.sizes().slice(0, q.dim() - 1), " on ", c.dev);
            lse = l.data_ptr<float>();
        }
        if (B > 0) {
            int64_t& need = c.needs[{B, T, H_q}];
            if (need <= 0) {
                need = retopk_q4_attention_workspace((int)B, (int)T, (int)H_q, c.pages.H_kv, c.pages.d);
                check(need, "retopk_q4_attention_workspace");
            }
            // from torch's allocator: tied to this stream (and, under capture, to the graph's own pool)
            const at::Tensor ws = empty({need}, q, at::kByte);
            check(retopk_q4_attention(&pages, (int)B, (int)T, (int)H_q, lens, type_code(q.scalar_type()), q.data_ptr(), q_stride, (float)scale,
                                      window, out.data_ptr(), lse, ws.data_ptr(), need, stream_of(c.dev)), "retopk_q4_attention");
            if (given(a[6])) written(out);
            if (given(a[7])) written(tensor(a[7], "lse"));
        }
        return THPVariable_Wrap(out);
    });
}

PyObject* set_error(PyObject*, PyObject* type) {
    Py_XSETREF(g_error, Py_NewRef(type));
    return Py_NewRef(Py_None);
}

#define FAST(f) {#f, reinterpret_cast<PyCFunction>(reinterpret_cast<void (*)()>(f)), METH_FASTCALL, nullptr}
PyMethodDef METHODS[] = {FAST(rope_apply), FAST(cache_new), FAST(append), FAST(gather), FAST(attend),
                         {"set_error", set_error, METH_O, nullptr}, {nullptr, nullptr, 0, nullptr}};
PyModuleDef MODULE = {PyModuleDef_HEAD_INIT, "_paged", "Calls around the KV cache (see paged.py).", -1, METHODS, nullptr, nullptr, nullptr, nullptr};

}  // namespace

PyMODINIT_FUNC PyInit__paged() {
    PyObject* m = PyModule_Create(&MODULE);
    if (m && PyModule_AddStringConstant(m, "built_for", BUILT_FOR) != 0) Py_CLEAR(m);      // compared by paged.py
    return m;
}
