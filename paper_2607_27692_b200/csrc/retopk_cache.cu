// Host side of the calls around the KV cache: argument checks, frequencies, launches, C interface.
#include "retopk_cache_host.cuh"

#include <math.h>
#include <mutex>
#include <new>

using namespace retopk_cache;

struct retopk_rope {
    int d, rot_dim, layout;
    double amp;
    double w[MAX_PAIRS];        // radians per position
    double turns[MAX_PAIRS];    // w / (2 pi)
};

namespace {

constexpr double PI = 3.14159265358979323846;
constexpr int MAX_HEADS = 65535;         // of a tensor that is rotated or appended

// SM count, looked up once per device; and the attention kernels' opt-in to large shared memory.
constexpr int MAX_DEVICES = 64;
struct DeviceSetup { bool ready; int num_sms; };
DeviceSetup g_setup[MAX_DEVICES];
std::mutex g_setup_mutex;

template <int DT, int D, int SHAPE> bool opt_in_one() {
    return cudaFuncSetAttribute(q4_attend_kernel<DT, D, SHAPE>, cudaFuncAttributeMaxDynamicSharedMemorySize,
                                q4_smem_bytes(D, SHAPE)) == cudaSuccess;
}
template <int DT, int D> bool opt_in_all() { return opt_in_one<DT, D, COLS_4>() && opt_in_one<DT, D, COLS_8>() && opt_in_one<DT, D, COLS_16>(); }

int device_sms(int* num_sms) {
    int dev = -1;
    if (cudaGetDevice(&dev) != cudaSuccess) { cudaGetLastError(); return RETOPK_ECUDA; }
    if (dev < 0 || dev >= MAX_DEVICES) return RETOPK_EUNSUPPORTED;
    std::lock_guard<std::mutex> lock(g_setup_mutex);
    DeviceSetup& st = g_setup[dev];
    if (!st.ready) {
        if (cudaDeviceGetAttribute(&st.num_sms, cudaDevAttrMultiProcessorCount, dev) != cudaSuccess ||
            !opt_in_all<TYPE_BF16, 64>() || !opt_in_all<TYPE_BF16, 128>() || !opt_in_all<TYPE_FP16, 64>() || !opt_in_all<TYPE_FP16, 128>()) {
            cudaGetLastError();
            return RETOPK_ECUDA;
        }
        st.ready = true;
    }
    *num_sms = st.num_sms;
    return RETOPK_OK;
}

void set_rotation(RowsArgs& a, const retopk_rope* rope, int inverse) {
    if (!rope) return;
    memcpy(a.turns, rope->turns, sizeof a.turns);
    a.amp = rope->amp;
    a.pairs = rope->rot_dim / 2;
    a.inverse = inverse;
}

// CTAs for n tokens of R rows each: a warp per token where that gives every SM warps enough, several
// warps or CTAs per token below.
template <int DEST> int launch_rows(RowsArgs& a, const retopk_rope* rope, int dtype, int d, int num_sms, cudaStream_t s) {
    const int rpw = 32 / (d / 16);
    a.gq = (a.Hq + rpw - 1) / rpw;
    a.groups = a.gq + (a.Hk + a.Hv + rpw - 1) / rpw;
    const long long want = 16ll * num_sms;               // warps
    a.tokens_per_cta = a.n_tokens >= want ? 4 : (2 * a.n_tokens >= want ? 2 : 1);
    // two groups of rows to a warp, if the tokens alone do not fill the device
    const int per_tok = ROWS_WARPS / a.tokens_per_cta, most = (a.groups + 2 * per_tok - 1) / (2 * per_tok);
    const long long need = (want + a.n_tokens * per_tok - 1) / (a.n_tokens * per_tok);
    a.units = (int)(need < most ? need : most);
    if (a.units < 1) a.units = 1;
    const long long gx = (a.n_tokens + a.tokens_per_cta - 1) / a.tokens_per_cta;
    if (gx > 2147483647ll || a.units > 65535) return RETOPK_EUNSUPPORTED;
    const dim3 grid((unsigned)gx, (unsigned)a.units);
    auto go = [&](auto bf128, auto bf64, auto fp128, auto fp64) {
        return launch(dtype == RETOPK_BF16 ? (d == 128 ? bf128 : bf64) : (d == 128 ? fp128 : fp64), grid, ROWS_THREADS, 0, s, a);
    };
    constexpr int BF = TYPE_BF16, FP = TYPE_FP16;
    if (!rope || (rope->layout == RETOPK_ROPE_HALF && rope->rot_dim % 16 != 0))
        return go(rows_kernel<BF, 128, DEST, ROT_OTHER>, rows_kernel<BF, 64, DEST, ROT_OTHER>,
                  rows_kernel<FP, 128, DEST, ROT_OTHER>, rows_kernel<FP, 64, DEST, ROT_OTHER>);
    if (rope->layout == RETOPK_ROPE_HALF)
        return go(rows_kernel<BF, 128, DEST, ROT_HALF>, rows_kernel<BF, 64, DEST, ROT_HALF>,
                  rows_kernel<FP, 128, DEST, ROT_HALF>, rows_kernel<FP, 64, DEST, ROT_HALF>);
    return go(rows_kernel<BF, 128, DEST, ROT_INTERLEAVED>, rows_kernel<BF, 64, DEST, ROT_INTERLEAVED>,
              rows_kernel<FP, 128, DEST, ROT_INTERLEAVED>, rows_kernel<FP, 64, DEST, ROT_INTERLEAVED>);
}

template <int SRC, int DT> int launch_gather(const GatherArgs& a, int d, dim3 grid, cudaStream_t s) {
    return d == 128 ? launch(gather_kernel<SRC, DT, 128>, grid, GATHER_THREADS, 0, s, a)
                    : launch(gather_kernel<SRC, DT, 64>, grid, GATHER_THREADS, 0, s, a);
}

int q4_shape(int columns) { return columns <= 4 ? COLS_4 : (columns <= 8 ? COLS_8 : COLS_16); }
int q4_ctas(int shape, int num_sms) { return num_sms * q4_ctas_per_sm(shape); }

int check_q4_shape(int B, int T, int H_q, int H_kv, int d) {
    if (B < 1 || T < 1 || H_q < 1 || H_kv < 1 || H_q % H_kv != 0) return RETOPK_EINVAL;
    if ((d != 64 && d != 128) || H_q / H_kv > 16 || T > 16 || (long long)B * H_kv > MAX_SEQ_GROUPS) return RETOPK_EUNSUPPORTED;
    return RETOPK_OK;
}

template <int DT, int D, int SHAPE> int launch_q4(const Q4Args& a, int items, cudaStream_t s) {
    const int rc = launch(q4_attend_kernel<DT, D, SHAPE>, dim3((unsigned)a.grid), Q4_THREADS, q4_smem_bytes(D, SHAPE), s, a);
    if (rc != RETOPK_OK) return rc;
    return launch(q4_combine_kernel<DT, D, SHAPE>, dim3((unsigned)items, (unsigned)q4_cols(SHAPE)), D, 0, s, a);
}
template <int DT, int D> int launch_q4_shape(const Q4Args& a, int shape, int items, cudaStream_t s) {
    if (shape == COLS_4) return launch_q4<DT, D, COLS_4>(a, items, s);
    if (shape == COLS_8) return launch_q4<DT, D, COLS_8>(a, items, s);
    return launch_q4<DT, D, COLS_16>(a, items, s);
}

}  // namespace

extern "C" {

int retopk_rope_create(retopk_rope** rope, const retopk_rope_config_t* c) {
    if (!rope) return RETOPK_EINVAL;
    *rope = nullptr;
    if (!c) return RETOPK_EINVAL;
    if (c->rot_dim < 2 || c->rot_dim % 2 != 0 || c->rot_dim > c->d) return RETOPK_EINVAL;
    if (c->layout != RETOPK_ROPE_HALF && c->layout != RETOPK_ROPE_INTERLEAVED) return RETOPK_EINVAL;
    if (c->scaling < RETOPK_ROPE_PLAIN || c->scaling > RETOPK_ROPE_YARN) return RETOPK_EINVAL;
    if (!(c->base > 1.0) || !isfinite(c->base) || !(c->attn_factor >= 0.0) || c->attn_factor > 1e30) return RETOPK_EINVAL;
    if (c->scaling != RETOPK_ROPE_PLAIN && (!(c->factor >= 1.0) || !isfinite(c->factor))) return RETOPK_EINVAL;
    if (c->scaling == RETOPK_ROPE_NTK && c->rot_dim == 2) return RETOPK_EINVAL;
    const double lowf = c->low_freq_factor != 0.0 ? c->low_freq_factor : 1.0;
    const double highf = c->high_freq_factor != 0.0 ? c->high_freq_factor : 4.0;
    const double fast = c->beta_fast != 0.0 ? c->beta_fast : 32.0;
    const double slow = c->beta_slow != 0.0 ? c->beta_slow : 1.0;
    if (c->scaling == RETOPK_ROPE_LLAMA3 || c->scaling == RETOPK_ROPE_YARN)
        if (!(c->original_len >= 1.0) || !isfinite(c->original_len)) return RETOPK_EINVAL;
    if (c->scaling == RETOPK_ROPE_LLAMA3 && !(lowf > 0.0 && highf > lowf && isfinite(highf))) return RETOPK_EINVAL;
    if (c->scaling == RETOPK_ROPE_YARN && !(slow > 0.0 && fast >= slow && isfinite(fast))) return RETOPK_EINVAL;
    if (c->d != 64 && c->d != 128) return RETOPK_EUNSUPPORTED;

    retopk_rope* r = new (std::nothrow) retopk_rope;
    if (!r) return RETOPK_ENOMEM;
    memset(r, 0, sizeof *r);
    r->d = c->d;
    r->rot_dim = c->rot_dim;
    r->layout = c->layout;
    r->amp = 1.0;
    const double rot = c->rot_dim, f = c->factor;
    double base = c->base;
    if (c->scaling == RETOPK_ROPE_NTK) base *= pow(f, rot / (rot - 2.0));
    double ramp_lo = 0.0, ramp_hi = 0.0;
    if (c->scaling == RETOPK_ROPE_YARN) {
        // pair whose angle turns x times over the original length: base^(-2i/rot) * len = 2 pi x
        ramp_lo = floor(rot * log(c->original_len / (fast * 2.0 * PI)) / (2.0 * log(base)));
        ramp_hi = ceil(rot * log(c->original_len / (slow * 2.0 * PI)) / (2.0 * log(base)));
        if (ramp_lo < 0.0) ramp_lo = 0.0;
        if (ramp_hi > rot - 1.0) ramp_hi = rot - 1.0;
        r->amp = 0.1 * log(f) + 1.0;
    }
    if (c->attn_factor > 0.0) r->amp = c->attn_factor;
    for (int i = 0; i < c->rot_dim / 2; ++i) {
        double w = pow(base, -2.0 * i / rot);
        if (c->scaling == RETOPK_ROPE_LINEAR) {
            w /= f;
        } else if (c->scaling == RETOPK_ROPE_LLAMA3) {
            const double ratio = c->original_len * w / (2.0 * PI);        // original_len / wavelength
            double t = (ratio - lowf) / (highf - lowf);
            t = t < 0.0 ? 0.0 : (t > 1.0 ? 1.0 : t);
            w = (1.0 - t) * w / f + t * w;
        } else if (c->scaling == RETOPK_ROPE_YARN) {
            double width = ramp_hi - ramp_lo;
            if (width < 1e-3) width = 1e-3;
            double t = (i - ramp_lo) / width;
            t = t < 0.0 ? 0.0 : (t > 1.0 ? 1.0 : t);
            w = t * w / f + (1.0 - t) * w;
        }
        r->w[i] = w;
        r->turns[i] = w / (2.0 * PI);
    }
    *rope = r;
    return RETOPK_OK;
}

int retopk_rope_destroy(retopk_rope* rope) {
    if (!rope) return RETOPK_EINVAL;
    delete rope;
    return RETOPK_OK;
}

int retopk_rope_frequencies(const retopk_rope* rope, double* inv_freq_host, double* attn_factor_host) {
    if (!rope) return RETOPK_EINVAL;
    if (inv_freq_host) memcpy(inv_freq_host, rope->w, sizeof(double) * (rope->rot_dim / 2));
    if (attn_factor_host) *attn_factor_host = rope->amp;
    return RETOPK_OK;
}

int retopk_rope_apply(const retopk_rope* rope, int dtype, int64_t n_tokens, const int32_t* positions, const void* q,
                      int64_t q_stride, void* q_out, int64_t q_out_stride, int H_q, const void* k, int64_t k_stride,
                      void* k_out, int64_t k_out_stride, int H_k, int inverse, void* stream) {
    if (!rope || n_tokens < 0 || (!q && !k) || (inverse != 0 && inverse != 1) || bad_half_type(dtype)) return RETOPK_EINVAL;
    const int d = rope->d;
    if (q && (!rows_ok(q, q_stride, H_q, d) || !rows_ok(q_out, q_out_stride, H_q, d))) return RETOPK_EINVAL;
    if (k && (!rows_ok(k, k_stride, H_k, d) || !rows_ok(k_out, k_out_stride, H_k, d))) return RETOPK_EINVAL;
    if ((q && H_q > MAX_HEADS) || (k && H_k > MAX_HEADS)) return RETOPK_EUNSUPPORTED;
    if (n_tokens == 0) return RETOPK_OK;
    if (!positions) return RETOPK_EINVAL;
    const Strided qi = {q, q_stride, H_q}, qo = {q_out, q_out_stride, H_q}, ki = {k, k_stride, H_k}, ko = {k_out, k_out_stride, H_k};
    if (q && !in_place_or_apart(qi, qo, n_tokens, d)) return RETOPK_EINVAL;
    if (k && !in_place_or_apart(ki, ko, n_tokens, d)) return RETOPK_EINVAL;
    if (q && k && !(rows_apart(qo, ki, n_tokens, d) && rows_apart(ko, qi, n_tokens, d) && rows_apart(qo, ko, n_tokens, d))) return RETOPK_EINVAL;
    int num_sms = 0;
    const int rc = device_sms(&num_sms);
    if (rc != RETOPK_OK) return rc;
    RowsArgs a;
    memset(&a, 0, sizeof a);
    set_rotation(a, rope, inverse);
    a.n_tokens = n_tokens;
    a.positions = positions;
    a.q = static_cast<const uint16_t*>(q); a.q_stride = q_stride;
    a.q_out = static_cast<uint16_t*>(q_out); a.q_out_stride = q_out_stride;
    a.k = static_cast<const uint16_t*>(k); a.k_stride = k_stride;
    a.k_out = static_cast<uint16_t*>(k_out); a.k_out_stride = k_out_stride;
    a.Hq = q ? H_q : 0;
    a.Hk = k ? H_k : 0;
    return launch_rows<DEST_ROWS>(a, rope, dtype, d, num_sms, static_cast<cudaStream_t>(stream));
}

int retopk_kv_append(const retopk_pages_t* pages, int B, const int32_t* seq_lens, const int32_t* cu_new, int64_t n_new,
                     int dtype, const void* k_new, int64_t k_stride, const void* v_new, int64_t v_stride,
                     const retopk_rope* rope, const void* q, int64_t q_stride, void* q_out, int64_t q_out_stride, int H_q,
                     void* stream) {
    int rc = check_pages(pages, B);
    if (rc != RETOPK_OK) return rc;
    const int d = pages->d, H = pages->H_kv;
    if (!seq_lens || n_new < 0 || bad_half_type(dtype)) return RETOPK_EINVAL;
    if (pages->format != RETOPK_PAGES_Q4 && (pages->format == RETOPK_PAGES_BF16) != (dtype == RETOPK_BF16)) return RETOPK_EINVAL;
    if (!cu_new && n_new % B != 0) return RETOPK_EINVAL;
    if (!rows_ok(k_new, k_stride, H, d) || !rows_ok(v_new, v_stride, H, d)) return RETOPK_EINVAL;
    if (rope && rope->d != d) return RETOPK_EINVAL;
    if (q && (!rope || !rows_ok(q, q_stride, H_q, d) || !rows_ok(q_out, q_out_stride, H_q, d))) return RETOPK_EINVAL;
    if (B > 65535 || n_new > 2147483647ll || H > MAX_HEADS || (q && H_q > MAX_HEADS)) return RETOPK_EUNSUPPORTED;
    if (n_new == 0) return RETOPK_OK;
    const Strided qi = {q, q_stride, H_q}, qo = {q_out, q_out_stride, H_q}, ki = {k_new, k_stride, H}, vi = {v_new, v_stride, H};
    if (q && !(in_place_or_apart(qi, qo, n_new, d) && rows_apart(qo, ki, n_new, d) && rows_apart(qo, vi, n_new, d))) return RETOPK_EINVAL;
    Memory pg[4];
    memory_of(pages, pg);
    for (int i = 0; i < 4; ++i)
        for (int j = i + 1; j < 4; ++j)
            if (!apart(pg[i], pg[j])) return RETOPK_EINVAL;
    if (!all_apart(memory_of(ki, n_new, d), pg) || !all_apart(memory_of(vi, n_new, d), pg)) return RETOPK_EINVAL;
    if (q && (!all_apart(memory_of(qi, n_new, d), pg) || !all_apart(memory_of(qo, n_new, d), pg))) return RETOPK_EINVAL;
    int num_sms = 0;
    rc = device_sms(&num_sms);
    if (rc != RETOPK_OK) return rc;
    RowsArgs a;
    memset(&a, 0, sizeof a);
    set_rotation(a, rope, 0);
    a.n_tokens = n_new;
    a.seq_lens = seq_lens;
    a.cu = cu_new;
    a.B = B;
    a.T = cu_new ? 0 : (int)(n_new / B);
    a.q = static_cast<const uint16_t*>(q); a.q_stride = q_stride;
    a.q_out = static_cast<uint16_t*>(q_out); a.q_out_stride = q_out_stride;
    a.k = static_cast<const uint16_t*>(k_new); a.k_stride = k_stride;
    a.v = static_cast<const uint16_t*>(v_new); a.v_stride = v_stride;
    a.Hq = q ? H_q : 0;
    a.Hk = a.Hv = H;
    a.pg = device_pages(pages);
    cudaStream_t s = static_cast<cudaStream_t>(stream);
    if (pages->format == RETOPK_PAGES_Q4) return launch_rows<DEST_PAGES4>(a, rope, dtype, d, num_sms, s);
    return launch_rows<DEST_PAGES16>(a, rope, dtype, d, num_sms, s);
}

int retopk_kv_gather(const retopk_pages_t* pages, int B, const int32_t* seq_lens, const int32_t* first, int64_t max_rows,
                     int dtype, void* k_out, void* v_out, void* stream) {
    const int rc = check_pages(pages, B);
    if (rc != RETOPK_OK) return rc;
    if (!seq_lens || max_rows < 0 || (!k_out && !v_out) || dtype < RETOPK_BF16 || dtype > RETOPK_FP32) return RETOPK_EINVAL;
    if ((k_out && !aligned16(k_out)) || (v_out && !aligned16(v_out))) return RETOPK_EINVAL;
    const bool q4 = pages->format == RETOPK_PAGES_Q4;
    if (!q4 && dtype != RETOPK_FP32 && (pages->format == RETOPK_PAGES_BF16) != (dtype == RETOPK_BF16)) return RETOPK_EINVAL;
    if (B > 65535 || pages->H_kv > 65535) return RETOPK_EUNSUPPORTED;
    if (max_rows == 0) return RETOPK_OK;
    Memory pg[4];
    memory_of(pages, pg);
    const uint64_t out_bytes = (uint64_t)B * pages->H_kv * max_rows * pages->d * (dtype == RETOPK_FP32 ? 4 : 2);
    const Memory ko = {k_out, out_bytes}, vo = {v_out, out_bytes};
    if (!all_apart(ko, pg) || !all_apart(vo, pg) || !apart(ko, vo)) return RETOPK_EINVAL;
    GatherArgs a;
    memset(&a, 0, sizeof a);
    a.pg = device_pages(pages);
    a.seq_lens = seq_lens;
    a.first = first;
    a.max_rows = max_rows;
    a.k_out = k_out;
    a.v_out = v_out;
    // no sequence has more rows than the cache holds (unless it begins before the first)
    const long long rows = first || max_rows < a.pg.capacity ? max_rows : a.pg.capacity;
    if (rows > 2147483647ll * GATHER_ROWS) return RETOPK_EUNSUPPORTED;
    const dim3 grid((unsigned)((rows + GATHER_ROWS - 1) / GATHER_ROWS), (unsigned)pages->H_kv, (unsigned)B);
    cudaStream_t s = static_cast<cudaStream_t>(stream);
    if (q4) {
        if (dtype == RETOPK_BF16) return launch_gather<2, TYPE_BF16>(a, pages->d, grid, s);
        if (dtype == RETOPK_FP16) return launch_gather<2, TYPE_FP16>(a, pages->d, grid, s);
        return launch_gather<2, TYPE_FP32>(a, pages->d, grid, s);
    }
    if (pages->format == RETOPK_PAGES_BF16)
        return dtype == RETOPK_FP32 ? launch_gather<0, TYPE_FP32>(a, pages->d, grid, s) : launch_gather<0, TYPE_BF16>(a, pages->d, grid, s);
    return dtype == RETOPK_FP32 ? launch_gather<1, TYPE_FP32>(a, pages->d, grid, s) : launch_gather<1, TYPE_FP16>(a, pages->d, grid, s);
}

int64_t retopk_q4_attention_workspace(int B, int T, int H_q, int H_kv, int d) {
    int rc = check_q4_shape(B, T, H_q, H_kv, d), num_sms = 0;
    if (rc == RETOPK_OK) rc = device_sms(&num_sms);
    if (rc != RETOPK_OK) return rc;
    const int shape = q4_shape(T * (H_q / H_kv));
    return 2ll * q4_ctas(shape, num_sms) * q4_cols(shape) * (d + 2) * 4;
}

int retopk_q4_attention(const retopk_pages_t* pages, int B, int T, int H_q, const int32_t* seq_lens, int dtype,
                        const void* q, int64_t q_stride, float scale, int64_t window, void* out, float* lse,
                        void* workspace, int64_t workspace_bytes, void* stream) {
    int rc = check_pages(pages, B);
    if (rc != RETOPK_OK) return rc;
    if (pages->format != RETOPK_PAGES_Q4 || !seq_lens || !out || !workspace || bad_half_type(dtype)) return RETOPK_EINVAL;
    if (window < 0 || !isfinite(scale)) return RETOPK_EINVAL;
    rc = check_q4_shape(B, T, H_q, pages->H_kv, pages->d);
    if (rc != RETOPK_OK) return rc;
    if (!rows_ok(q, q_stride, H_q, pages->d) || !aligned16(workspace)) return RETOPK_EINVAL;
    Q4Args a;
    memset(&a, 0, sizeof a);
    a.pg = device_pages(pages);
    if (a.pg.capacity > MAX_KEYS || pages->n_pages > 0xfffffffell / ((long long)pages->H_kv * pages->page_size)) return RETOPK_EUNSUPPORTED;
    const long long n = (long long)B * T;
    const Strided qi = {q, q_stride, H_q}, qo = {out, (long long)H_q * pages->d, H_q};
    Memory pg[4];
    memory_of(pages, pg);
    const Memory out_m = memory_of(qo, n, pages->d), lse_m = {lse, (uint64_t)n * H_q * 4}, ws_m = {workspace, (uint64_t)workspace_bytes};
    if (!in_place_or_apart(qi, qo, n, pages->d) || !all_apart(out_m, pg) || !all_apart(lse_m, pg) || !all_apart(ws_m, pg)) return RETOPK_EINVAL;
    if (!all_apart(lse_m, {out_m, memory_of(qi, n, pages->d), ws_m}) || !all_apart(ws_m, {out_m, memory_of(qi, n, pages->d)})) return RETOPK_EINVAL;
    int num_sms = 0;
    rc = device_sms(&num_sms);
    if (rc != RETOPK_OK) return rc;
    a.seq_lens = seq_lens;
    a.q = static_cast<const uint16_t*>(q);
    a.out = static_cast<uint16_t*>(out);
    a.lse = lse;
    a.part = static_cast<float*>(workspace);
    a.q_stride = q_stride;
    a.window = window <= MAX_KEYS ? window : 0;         // a wider one leaves no key out (nor may sums with it overflow)
    a.two16 = 1u << 16;
    a.scale_log2 = (float)((double)scale * 1.44269504088896340736);
    a.B = B; a.T = T; a.Hq = H_q; a.G = H_q / pages->H_kv;
    const int columns = T * a.G, shape = q4_shape(columns);
    a.col_tiles = (columns + q4_cols(shape) - 1) / q4_cols(shape);
    if (workspace_bytes < 2ll * q4_ctas(shape, num_sms) * q4_cols(shape) * (pages->d + 2) * 4) return RETOPK_EINVAL;
    const long long most = (long long)B * pages->H_kv * a.col_tiles * ((a.pg.capacity + Q4_UNIT - 1) / Q4_UNIT);
    const int ctas = q4_ctas(shape, num_sms);
    a.grid = (int)(most < ctas ? most : ctas);
    const int items = B * pages->H_kv * a.col_tiles;
    cudaStream_t s = static_cast<cudaStream_t>(stream);
    if (dtype == RETOPK_BF16)
        return pages->d == 128 ? launch_q4_shape<TYPE_BF16, 128>(a, shape, items, s) : launch_q4_shape<TYPE_BF16, 64>(a, shape, items, s);
    return pages->d == 128 ? launch_q4_shape<TYPE_FP16, 128>(a, shape, items, s) : launch_q4_shape<TYPE_FP16, 64>(a, shape, items, s);
}

}  // extern "C"
