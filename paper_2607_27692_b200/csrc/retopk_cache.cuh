// Device code around the KV cache (sm_100a): rotary positions, append to 16-bit or 4-bit pages,
// read-back of pages, and decode attention over 4-bit pages.
//
//   rows_kernel       rotates rows of q and k and stores k and v (rotation alone, append to 16-bit
//                     pages and append to 4-bit pages are three instances of it)
//   gather_kernel     rows of a paged cache -> contiguous [B,H_kv,rows,d]
//   q4_attend_kernel  streams the 4-bit pages once through the tensor cores
//   q4_combine_kernel joins the parts of sequences that several CTAs shared
#pragma once
#include <cuda_bf16.h>
#include <cuda_fp16.h>
#include <cuda_runtime.h>
#include <stdint.h>

namespace retopk_cache {

constexpr int TYPE_BF16 = 0, TYPE_FP16 = 1, TYPE_FP32 = 2;
constexpr int GROUP = 64;                // channels that share a step and a minimum
constexpr int MAX_PAIRS = 64;            // rotated pairs of a head (d <= 128)

// ---------------------------------------------------------------------------------------
// Small helpers
// ---------------------------------------------------------------------------------------
template <int DT> __device__ __forceinline__ float to_f32(uint16_t u) {
    if (DT == TYPE_BF16) return __uint_as_float((uint32_t)u << 16);
    return __half2float(__ushort_as_half(u));
}
template <int DT> __device__ __forceinline__ float2 unpack2(uint32_t u) {
    if (DT == TYPE_BF16) return make_float2(__uint_as_float(u << 16), __uint_as_float(u & 0xffff0000u));
    return __half22float2(*reinterpret_cast<const __half2*>(&u));
}
template <int DT> __device__ __forceinline__ uint32_t pack2(float lo, float hi) {
    if (DT == TYPE_BF16) {
        __nv_bfloat162 v = __floats2bfloat162_rn(lo, hi);
        return *reinterpret_cast<uint32_t*>(&v);
    }
    __half2 v = __floats2half2_rn(lo, hi);
    return *reinterpret_cast<uint32_t*>(&v);
}
template <int DT> __device__ __forceinline__ void unpack8(const uint4& x, float* f) {
    const uint32_t w[4] = {x.x, x.y, x.z, x.w};
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        const float2 p = unpack2<DT>(w[i]);
        f[2 * i] = p.x;
        f[2 * i + 1] = p.y;
    }
}
template <int DT> __device__ __forceinline__ uint4 pack8(const float* f) {
    return make_uint4(pack2<DT>(f[0], f[1]), pack2<DT>(f[2], f[3]), pack2<DT>(f[4], f[5]), pack2<DT>(f[6], f[7]));
}

// Minimum and maximum that are NaN if one operand is.
__device__ __forceinline__ float min_nan(float a, float b) {
    float c;
    asm("min.NaN.f32 %0, %1, %2;" : "=f"(c) : "f"(a), "f"(b));
    return c;
}
__device__ __forceinline__ float max_nan(float a, float b) {
    float c;
    asm("max.NaN.f32 %0, %1, %2;" : "=f"(c) : "f"(a), "f"(b));
    return c;
}

__device__ __forceinline__ uint32_t bf16x2_fma(uint32_t a, uint32_t b, uint32_t c) {
    uint32_t d;
    asm("fma.rn.bf16x2 %0, %1, %2, %3;" : "=r"(d) : "r"(a), "r"(b), "r"(c));
    return d;
}
__device__ __forceinline__ uint32_t bf16x2_sub(uint32_t a, uint32_t b) {
    uint32_t d;
    asm("sub.rn.bf16x2 %0, %1, %2;" : "=r"(d) : "r"(a), "r"(b));
    return d;
}

__device__ __forceinline__ void cp_async16(uint32_t smem_dst, const void* src) {
    asm volatile("cp.async.cg.shared.global [%0], [%1], 16;" ::"r"(smem_dst), "l"(src) : "memory");
}
// Programmatic dependent launch: every kernel here is launched with the stream-serialisation attribute
// and waits before it touches memory; a kernel that lets its successor start does so after its own wait.
__device__ __forceinline__ void pdl_wait() { asm volatile("griddepcontrol.wait;" ::: "memory"); }
__device__ __forceinline__ void pdl_start_next() { asm volatile("griddepcontrol.launch_dependents;" ::: "memory"); }
__device__ __forceinline__ void cp_async_commit() { asm volatile("cp.async.commit_group;" ::: "memory"); }
template <int N> __device__ __forceinline__ void cp_async_wait() { asm volatile("cp.async.wait_group %0;" ::"n"(N) : "memory"); }

// The cache as the kernels see it (retopk_pages_t with 64-bit strides worked out).
struct Pages {
    unsigned char *k, *v, *ks, *vs;
    const int32_t* table;       // null: sequence b owns page b
    long long n_pages, max_pages, capacity;   // capacity: rows a sequence can have
    int H_kv, page_size, page_shift;          // page_shift: log2 of page_size, or -1
};

// Row index of position `pos` of sequence b for KV head 0 (head h: + h * page_size), or -1 when
// the position is outside the cache or its page number is not a page.
__device__ __forceinline__ long long cache_row(const Pages& pg, int b, long long pos) {
    if (pos < 0 || pos >= pg.capacity) return -1;
    const int slot = pg.page_shift >= 0 ? (int)pos >> pg.page_shift : (int)pos / pg.page_size, off = (int)pos - slot * pg.page_size;
    long long page = b;
    if (pg.table) page = pg.table[(long long)b * pg.max_pages + slot];
    if (page < 0 || page >= pg.n_pages) return -1;
    return page * pg.H_kv * pg.page_size + off;
}

// Codes round((x - m) / s) within 0..15 of eight values, the first in the low bits; c: a power of two
// that brings s well into the normal range, y: 1 / (s c) rounded, 0 if s is.  The quotient is rounded as
// the division is (P. Markstein's theorem: from the rounded reciprocal y and a quotient q within one unit,
// q + (a - b q) y rounds correctly).  Adding 1.5 * 2^23 rounds to a whole number, ties to even, and leaves
// it in the low bits.  A step that is not subnormal is at least (1 - 2^-8) of a fifteenth of the span, so
// no quotient reaches 15.5; below 0 it can be, if the minimum was rounded up.
template <bool SCALED>
__device__ __forceinline__ uint32_t eight_codes(const float* x, float m, float s, float y, float c) {
    const float b = SCALED ? s * c : s;
    uint32_t w = 0;
#pragma unroll
    for (int e = 7; e >= 0; --e) {
        const float a = SCALED ? (x[e] - m) * c : x[e] - m, q0 = a * y;
        float q = fmaxf(fmaf(fmaf(-q0, b, a), y, q0), 0.f);
        if (SCALED) q = fminf(q, 15.f);
        w = w * 16u + (__float_as_uint(q + 12582912.f) - 0x4b400000u);
    }
    return w;
}
// The rare steps below 2^-60 or above 2^60, out of line.
__device__ __noinline__ uint32_t eight_codes_scaled(float x0, float x1, float x2, float x3, float x4, float x5, float x6, float x7, float m, float s) {
    const float c = s < 1.f ? 18446744073709551616.f : 5.4210109e-20f;       // 2^64, 2^-64
    const float x[8] = {x0, x1, x2, x3, x4, x5, x6, x7};
    return eight_codes<true>(x, m, s, s > 0.f ? __frcp_rn(s * c) : 0.f, c);
}
__device__ __forceinline__ uint32_t codes_of(const float* x, float m, float s) {
    if (s > 8.6736174e-19f && s < 1.1529215e18f) return eight_codes<false>(x, m, s, __frcp_rn(s), 1.f);
    return eight_codes_scaled(x[0], x[1], x[2], x[3], x[4], x[5], x[6], x[7], m, s);
}

// ---------------------------------------------------------------------------------------
// rows_kernel: rotate and store
// ---------------------------------------------------------------------------------------
enum { ROT_HALF = 0, ROT_INTERLEAVED = 1, ROT_OTHER = 2 };    // OTHER: none (pairs = 0), or a half layout of any even size
enum { DEST_ROWS = 0, DEST_PAGES16 = 1, DEST_PAGES4 = 2 };
constexpr int ROWS_THREADS = 128, ROWS_WARPS = ROWS_THREADS / 32, ROWS_CTAS = 6;

struct RowsArgs {
    double turns[MAX_PAIRS];    // turns per position of each pair: w_i / (2 pi)
    double amp;                 // factor on cosine and sine
    int pairs, inverse;         // pairs = 0: no rotation
    int tokens_per_cta, units;  // a CTA takes 1, 2 or 4 tokens; blockIdx.y of `units` shares their rows
    long long n_tokens;
    const int32_t* positions;   // DEST_ROWS
    const int32_t *seq_lens, *cu;
    int B, T;                   // T: new tokens per sequence when cu is null
    const uint16_t *q, *k, *v;
    uint16_t *q_out, *k_out;
    long long q_stride, k_stride, v_stride, q_out_stride, k_out_stride;
    int Hq, Hk, Hv;
    int gq, groups;             // groups of rows of q; of q, and of k and v one after the other
    Pages pg;
};

// x as the sum of a head of 16 (bf16) or 13 (fp16) bits and a rest.  Both have x's sign (cut off, not
// rounded) and neither is 0 unless x is (a rest of 2^-100 is nothing next to the head), so that an
// infinity times x is that infinity in both products and in their sum.
template <int DT> __device__ __forceinline__ float2 head_and_rest(double x) {
    constexpr uint32_t HEAD = DT == TYPE_BF16 ? 0xffffff00u : 0xfffff800u;
    const float h = __uint_as_float(__float_as_uint(__double2float_rz(x)) & HEAD);
    float r = (float)(x - h);
    if (r == 0.f && h != 0.f) r = copysignf(7.8886091e-31f, h);
    return make_float2(h, r);
}

// One row is held by D / 16 lanes, two chunks of 8 channels each, so that a warp has 4 rows (d = 128) or
// 8; a warp stays with one token, whose cosines and sines it keeps in shared memory, and goes through the
// heads, the next groups of rows on their way.  Where a half-layout rotation covers a multiple of 16
// channels, a lane's chunks are partners of each other (c and c + rot/2), so that no value crosses
// lanes; otherwise they are channels 8l and D/2 + 8l.
//
// Bound: HBM (two bytes read and written per value).  The angle is reduced and its cosine and sine are
// taken in fp64: at far positions an fp32 angle is useless.  The rotation itself: cosine and sine are
// split into a head of so few bits that its product with a 16-bit value is exact in fp32 (16 bits for
// bf16, 13 for fp16) and a rest, so that x ch - y sh is rounded once, whatever cancels, and the rests
// add what is missing: 2^-23 of the result, before it is rounded to 16 bits.  Keys that are quantised
// afterwards are rotated in fp64: a 16-bit value that is one step off could change a code.  (All in
// fp64, 16K tokens of 40 heads took 71 us: the conversions from and to fp32 fill their pipe.)
template <int DT, int D, int DEST, int ROT>
__global__ void __launch_bounds__(ROWS_THREADS, ROWS_CTAS) rows_kernel(const __grid_constant__ RowsArgs a) {
    constexpr int LANES = D / 16, RPW = 32 / LANES;      // lanes per row, rows per warp
    __shared__ float4 s_tab[ROWS_WARPS][MAX_PAIRS];      // heads and rests of cosine and sine
    __shared__ double2 s_tab64[DEST == DEST_PAGES4 ? ROWS_WARPS : 1][MAX_PAIRS];

    const int lane = threadIdx.x & 31, sub = lane % LANES, row_in = lane / LANES;
    const int warp = __shfl_sync(0xffffffffu, (int)threadIdx.x >> 5, 0);      // (known to be the same for all lanes)
    const int per_tok = ROWS_WARPS / a.tokens_per_cta;   // warps per token; each keeps a table of its own
    const long long tok = (long long)blockIdx.x * a.tokens_per_cta + warp / per_tok;
    pdl_wait();
    if (tok >= a.n_tokens) return;

    const int half = a.pairs;                            // rot / 2
    int ca = 8 * sub, cb = D / 2 + 8 * sub;
    if (ROT == ROT_HALF) {
        if (8 * sub < half) cb = half + 8 * sub;
        else { ca = 16 * sub; cb = ca + 8; }             // behind the rotated part
    }

    // ---- where this warp's rows are -------------------------------------------------------------
    // Groups of RPW rows of q, then of k and v one after the other (a group may end in k and begin in v),
    // are dealt out in turn to the warps of a token, which take PER of them at a time, the next ones on
    // their way.
    // (quantising twice over is too much code: 16 against 14.3 us, 5938 tokens of 16 + 4 + 4 heads of 64; so are
    // partners in other lanes)
    constexpr int PER = DEST == DEST_PAGES4 || ROT == ROT_OTHER ? 1 : 2;
    const int step = per_tok * a.units;
    const uint16_t *const q_src = a.q + tok * a.q_stride, *const k_src = a.k + tok * a.k_stride, *const v_src = a.v + tok * a.v_stride;
    struct Rows { int which, h; bool on; const uint16_t* src; };
    auto rows_of = [&](int g) {                          // this lane's row of group g: 0 q, 1 k, 2 v
        Rows r;
        r.h = (g < a.gq ? g : g - a.gq) * RPW + row_in;
        r.on = g < a.groups && r.h < (g < a.gq ? a.Hq : a.Hk + a.Hv);
        r.which = g < a.gq ? 0 : (DEST == DEST_ROWS || r.h < a.Hk ? 1 : 2);
        if (r.which == 2) r.h -= a.Hk;
        r.src = (r.which == 0 ? q_src : (r.which == 1 ? k_src : v_src)) + r.h * D;
        return r;
    };
    auto fetch = [&](int g, Rows (&r)[PER], uint4 (&fa)[PER], uint4 (&fb)[PER]) {
#pragma unroll
        for (int i = 0; i < PER; ++i) {
            r[i] = rows_of(g + i * step);
            if (r[i].on) {
                fa[i] = *reinterpret_cast<const uint4*>(r[i].src + ca);
                fb[i] = *reinterpret_cast<const uint4*>(r[i].src + cb);
            }
        }
    };
    Rows here[PER];
    uint4 ya[PER], yb[PER];
    const int g0 = (int)blockIdx.y * per_tok + warp % per_tok;
    fetch(g0, here, ya, yb);                             // on their way while position and page are looked up

    // ---- position and page row, by the whole warp -----------------------------------------------
    int pos = 0;
    long long row0 = -1;                                 // page row for head 0, -1: not stored
    if (DEST == DEST_ROWS) {
        pos = a.positions[tok];
    } else {
        long long p = -1;
        int b = 0;
        if (a.cu) {
            // largest b < B with cu[b] <= tok, 32 candidates at a time
            int lo = 0, n = a.B;
            while (n > 1) {
                const int hop = (n + 31) / 32, at = lane * hop;
                const uint32_t le = __ballot_sync(0xffffffffu, at < n && a.cu[lo + at] <= tok);
                const int last = le ? 31 - __clz((int)le) : 0;
                lo += last * hop;
                n = n - last * hop < hop ? n - last * hop : hop;
            }
            b = lo;
            const int first = a.cu[b], end = a.cu[b + 1], len = a.seq_lens[b];
            if (tok >= first && tok < end) p = (long long)len - end + tok;
        } else {
            b = (int)tok / a.T;
            p = (long long)a.seq_lens[b] - a.T + ((int)tok - b * a.T);
        }
        if (p < 0) return;                               // belongs to no sequence, or has no place
        pos = (int)p;
        row0 = cache_row(a.pg, b, p);
    }

    // ---- cosines and sines of this position -----------------------------------------------------
    for (int i = lane; i < a.pairs; i += 32) {
        // angle in turns, reduced before it is rounded: position * turns as a product and its rest
        const double p = (double)pos, w = a.turns[i];
        const double hi = p * w, lo = fma(p, w, -hi);
        const double r = (hi - rint(hi)) + lo;
        double sn, cs;
        sincospi(2.0 * r, &sn, &cs);
        sn *= a.amp;
        cs *= a.amp;
        if (a.inverse) sn = -sn;
        // a lane reads 8 neighbouring pairs one after the other; the exclusive-or keeps the lanes of a
        // row in different banks
        const int at = i ^ ((i >> 3) & 7);
        const float2 c = head_and_rest<DT>(cs), s = head_and_rest<DT>(sn);
        s_tab[warp][at] = make_float4(c.x, c.y, s.x, s.y);
        if (DEST == DEST_PAGES4) s_tab64[DEST == DEST_PAGES4 ? warp : 0][at] = make_double2(cs, sn);
    }
    __syncwarp();

    // pair i turned: (x, y) -> (x c - y s, y c + x s)
    auto turn = [&](bool exact, int i, float& x, float& y) {
        const int at = i ^ ((i >> 3) & 7);
        if (DEST == DEST_PAGES4 && exact) {
            const double2 c = s_tab64[DEST == DEST_PAGES4 ? warp : 0][at];
            const double u = x, v = y;
            x = (float)(u * c.x - v * c.y);
            y = (float)(v * c.x + u * c.y);
        } else {
            const float4 c = s_tab[warp][at];
            const float u = x, v = y;
            x = fmaf(-v, c.z, u * c.x) + fmaf(-v, c.w, u * c.y);
            y = fmaf(u, c.z, v * c.x) + fmaf(u, c.w, v * c.y);
        }
    };
    // 16 channels of one row, in place; src: the row itself (for partners in other lanes), on: it exists
    auto rotate = [&](bool exact, uint4& ya, uint4& yb, const uint16_t* src, bool on) {
        if (ROT == ROT_OTHER && a.pairs == 0) return;
        float xa[8], xb[8];
        unpack8<DT>(ya, xa);
        unpack8<DT>(yb, xb);
        if (ROT == ROT_HALF) {
            if (8 * sub >= half) return;
#pragma unroll
            for (int e = 0; e < 8; ++e) turn(exact, ca + e, xa[e], xb[e]);
        } else if (ROT == ROT_INTERLEAVED) {
#pragma unroll
            for (int e = 0; e < 4; ++e) {
                if (ca / 2 + e < half) turn(exact, ca / 2 + e, xa[2 * e], xa[2 * e + 1]);
                if (cb / 2 + e < half) turn(exact, cb / 2 + e, xb[2 * e], xb[2 * e + 1]);
            }
        } else {
            // a rotated part that is no multiple of 16 channels: partners lie in other lanes
            float pa[8], pb[8];
            if (on) {
                auto partner = [&](int c) { return c < half ? to_f32<DT>(src[c + half]) : (c < 2 * half ? to_f32<DT>(src[c - half]) : 0.f); };
#pragma unroll
                for (int e = 0; e < 8; ++e) { pa[e] = partner(ca + e); pb[e] = partner(cb + e); }
            }
            __syncwarp();                 // in place: every lane of the row has read before one writes
#pragma unroll
            for (int e = 0; e < 8; ++e) {
#pragma unroll
                for (int s = 0; s < 2; ++s) {
                    const int c = (s ? cb : ca) + e;
                    float& x = s ? xb[e] : xa[e];
                    float other = s ? pb[e] : pa[e];
                    if (on && c < half) turn(exact, c, x, other);
                    else if (on && c < 2 * half) turn(exact, c - half, other, x);
                }
            }
        }
        ya = pack8<DT>(xa);
        yb = pack8<DT>(xb);
    };
    // quantise one row's 16-bit values and store codes, step and minimum
    auto quantise = [&](const uint4& ya, const uint4& yb, unsigned char* codes, unsigned char* scales, long long row, bool store) {
            constexpr int NG = D / GROUP;
            float xa[8], xb[8];
            // quantise the 16-bit values: minimum and maximum of each group over the lanes of the row
            unpack8<DT>(ya, xa);
            unpack8<DT>(yb, xb);
            float mna = xa[0], mxa = xa[0], mnb = xb[0], mxb = xb[0];
#pragma unroll
            for (int e = 1; e < 8; ++e) {
                mna = min_nan(mna, xa[e]); mxa = max_nan(mxa, xa[e]);
                mnb = min_nan(mnb, xb[e]); mxb = max_nan(mxb, xb[e]);
            }
            const int ga = ca / GROUP, gb = cb / GROUP;
            float low[NG], step_[NG];
#pragma unroll
            for (int g = 0; g < NG; ++g) {
                float mn = min_nan(ga == g ? mna : INFINITY, gb == g ? mnb : INFINITY);
                float mx = max_nan(ga == g ? mxa : -INFINITY, gb == g ? mxb : -INFINITY);
#pragma unroll
                for (int o = 1; o < LANES; o <<= 1) {
                    mn = min_nan(mn, __shfl_xor_sync(0xffffffffu, mn, o));
                    mx = max_nan(mx, __shfl_xor_sync(0xffffffffu, mx, o));
                }
                low[g] = __bfloat162float(__float2bfloat16_rn(mn));
                // the minimum may have been rounded up past the maximum of a narrow group; no finite code stands
                // for NaN or an infinity, so a group that holds one gets a step of NaN or inf, which makes all of it NaN
                step_[g] = __bfloat162float(__float2bfloat16_rn(max_nan(__fdiv_rn(mx - low[g], 15.f), 0.f)));
            }
            const uint32_t wa = codes_of(xa, ga == 0 ? low[0] : low[NG - 1], ga == 0 ? step_[0] : step_[NG - 1]);
            const uint32_t wb = codes_of(xb, gb == 0 ? low[0] : low[NG - 1], gb == 0 ? step_[0] : step_[NG - 1]);
            if (store) {
                unsigned char* dst = codes + row * (D / 2);
                *reinterpret_cast<uint32_t*>(dst + ca / 2) = wa;
                *reinterpret_cast<uint32_t*>(dst + cb / 2) = wb;
                if (sub < NG)
                    reinterpret_cast<uint32_t*>(scales)[row * NG + sub] = pack2<TYPE_BF16>(sub == 0 ? step_[0] : step_[NG - 1], sub == 0 ? low[0] : low[NG - 1]);
            }
    };

#pragma unroll 1
    for (int g = g0; g < a.groups; g += PER * step) {
        Rows next[PER];
        uint4 na[PER], nb[PER];
        fetch(g + PER * step, next, na, nb);
#pragma unroll
        for (int i = 0; i < PER; ++i) {
            if (i > 0 && g + i * step >= a.groups) break;
            const Rows r = here[i];
            // (values go in as they are; their chunks are where the lane's are)
            const int gi = g + i * step;
            if (DEST == DEST_ROWS) {
                rotate(false, ya[i], yb[i], r.src, r.on);
            } else if (gi < a.gq || (gi - a.gq) * RPW < a.Hk) {
                uint4 za = ya[i], zb = yb[i];
                rotate(DEST == DEST_PAGES4 && gi >= a.gq, za, zb, r.src, r.on && r.which != 2);
                if (r.which != 2) { ya[i] = za; yb[i] = zb; }
            }
            if (DEST == DEST_ROWS || gi < a.gq) {
                if (r.on) {
                    uint16_t* dst = (r.which == 0 ? a.q_out + tok * a.q_out_stride : a.k_out + tok * a.k_out_stride) + r.h * D;
                    *reinterpret_cast<uint4*>(dst + ca) = ya[i];
                    *reinterpret_cast<uint4*>(dst + cb) = yb[i];
                }
            } else {
                const long long row = row0 + (long long)r.h * a.pg.page_size;
                unsigned char* pages = r.which == 1 ? a.pg.k : a.pg.v;
                const bool store = r.on && row0 >= 0;
                if (DEST == DEST_PAGES4) {
                    quantise(ya[i], yb[i], pages, r.which == 1 ? a.pg.ks : a.pg.vs, row, store);
                } else if (store) {
                    uint16_t* dst = reinterpret_cast<uint16_t*>(pages) + row * D;
                    *reinterpret_cast<uint4*>(dst + ca) = ya[i];
                    *reinterpret_cast<uint4*>(dst + cb) = yb[i];
                }
            }
        }
#pragma unroll
        for (int i = 0; i < PER; ++i) {
            here[i] = next[i];
            ya[i] = na[i];
            yb[i] = nb[i];
        }
    }
}

// ---------------------------------------------------------------------------------------
// gather_kernel: rows of a paged cache -> contiguous rows
// ---------------------------------------------------------------------------------------
constexpr int GATHER_THREADS = 256;
constexpr int GATHER_ROWS = 64;          // rows per CTA

struct GatherArgs {
    Pages pg;
    const int32_t *seq_lens, *first;
    long long max_rows;
    void *k_out, *v_out;
};

// One row is held by D / 8 lanes with 8 channels each, for fp32 results 4 in each half of the row, so
// that every store instruction writes whole sectors.  All of a thread's loads, keys and values, are
// asked for before the first is used.  Bound: HBM, mostly the writes; but a code at a time through
// integer conversion it was the ALU (4 x 32K rows to bf16: 127 us at 76% ALU).  bf16 results take two
// codes to a packed multiply-add, s n + m with its one rounding; 128 + n is a mask away.
template <int SRC /* 0 bf16, 1 fp16, 2: four bits */, int DT, int D>
__global__ void __launch_bounds__(GATHER_THREADS) gather_kernel(const __grid_constant__ GatherArgs a) {
    constexpr int LANES = D / 8, RPP = GATHER_THREADS / LANES, PASSES = GATHER_ROWS / RPP;
    constexpr bool SPLIT = DT == TYPE_FP32;              // 4 + 4 channels instead of 8
    pdl_wait();
    const int b = blockIdx.z, h = blockIdx.y;
    const long long row0 = (long long)blockIdx.x * GATHER_ROWS;
    const long long first = a.first ? a.first[b] : 0;
    long long len = a.seq_lens[b];
    if (len > a.pg.capacity) len = a.pg.capacity;
    if (first + row0 >= len) return;
    const int sub = threadIdx.x % LANES, r0 = threadIdx.x / LANES;
    const int c0 = SPLIT ? 4 * sub : 8 * sub, c1 = SPLIT ? D / 2 + 4 * sub : 8 * sub + 4;
    long long src_row[PASSES];
#pragma unroll
    for (int p = 0; p < PASSES; ++p) {
        const long long i = row0 + r0 + p * RPP;
        src_row[p] = -1;
        if (i < a.max_rows && first + i < len) {
            src_row[p] = cache_row(a.pg, b, first + i);
            if (src_row[p] >= 0) src_row[p] += (long long)h * a.pg.page_size;
        }
    }
    uint2 x0[2][PASSES], x1[2][PASSES];                  // 16 bits: four values each; 4 bits: codes and scale
#pragma unroll
    for (int kv = 0; kv < 2; ++kv) {
        if (!(kv ? a.v_out : a.k_out)) continue;
        const unsigned char* base = kv ? a.pg.v : a.pg.k;
        const unsigned char* sbase = kv ? a.pg.vs : a.pg.ks;
#pragma unroll
        for (int p = 0; p < PASSES; ++p) {
            if (src_row[p] < 0) continue;
            if (SRC == 2) {
                const unsigned char* row = base + src_row[p] * (D / 2);
                const unsigned char* sc = sbase + src_row[p] * (D / GROUP * 4);
                if (SPLIT) {
                    x0[kv][p].x = *reinterpret_cast<const uint16_t*>(row + c0 / 2);
                    x1[kv][p].x = *reinterpret_cast<const uint16_t*>(row + c1 / 2);
                } else {
                    x0[kv][p].x = *reinterpret_cast<const uint32_t*>(row + c0 / 2);
                    x1[kv][p].x = x0[kv][p].x >> 16;
                }
                x0[kv][p].y = *reinterpret_cast<const uint32_t*>(sc + c0 / GROUP * 4);
                x1[kv][p].y = SPLIT ? *reinterpret_cast<const uint32_t*>(sc + c1 / GROUP * 4) : x0[kv][p].y;
            } else {
                const unsigned char* row = base + src_row[p] * (D * 2);
                if (SPLIT) {
                    x0[kv][p] = *reinterpret_cast<const uint2*>(row + c0 * 2);
                    x1[kv][p] = *reinterpret_cast<const uint2*>(row + c1 * 2);
                } else {
                    const uint4 x = *reinterpret_cast<const uint4*>(row + c0 * 2);
                    x0[kv][p] = make_uint2(x.x, x.y);
                    x1[kv][p] = make_uint2(x.z, x.w);
                }
            }
        }
    }
#pragma unroll
    for (int kv = 0; kv < 2; ++kv) {
        void* out = kv ? a.v_out : a.k_out;
        if (!out) continue;
#pragma unroll
        for (int p = 0; p < PASSES; ++p) {
            if (src_row[p] < 0) continue;
            const long long at = (((long long)b * a.pg.H_kv + h) * a.max_rows + row0 + r0 + p * RPP) * D;
            if constexpr (SRC == 2 && DT == TYPE_BF16) {
                const uint32_t x = x0[kv][p].x, sm = x0[kv][p].y;
                uint32_t v[4];                           // values (0,4) (1,5) (2,6) (3,7)
#pragma unroll
                for (int e = 0; e < 4; ++e) {
                    const uint32_t n = ((x >> (4 * e)) & 0x000f000fu) | 0x43004300u;
                    v[e] = bf16x2_fma(bf16x2_sub(n, 0x43004300u), __byte_perm(sm, sm, 0x1010), __byte_perm(sm, sm, 0x3232));
                }
                *reinterpret_cast<uint4*>(static_cast<uint16_t*>(out) + at + c0) =
                    make_uint4(__byte_perm(v[0], v[1], 0x5410), __byte_perm(v[2], v[3], 0x5410),
                               __byte_perm(v[0], v[1], 0x7632), __byte_perm(v[2], v[3], 0x7632));
            } else {
                float f[8];
#pragma unroll
                for (int half = 0; half < 2; ++half) {
                    const uint2 x = half ? x1[kv][p] : x0[kv][p];
                    if (SRC == 2) {
                        const float2 sm = unpack2<TYPE_BF16>(x.y);
#pragma unroll
                        for (int e = 0; e < 4; ++e) {        // 2^23 + n is a mask away too
                            const float n = __uint_as_float(((x.x >> (4 * e)) & 15u) | 0x4b000000u) - 8388608.f;
                            f[4 * half + e] = fmaf(n, sm.x, sm.y);
                        }
                    } else if (SPLIT) {
                        const float2 lo = unpack2<SRC == 2 ? 0 : SRC>(x.x), hi = unpack2<SRC == 2 ? 0 : SRC>(x.y);
                        f[4 * half] = lo.x; f[4 * half + 1] = lo.y; f[4 * half + 2] = hi.x; f[4 * half + 3] = hi.y;
                    }
                }
                if (SPLIT) {
                    float* o = static_cast<float*>(out) + at;
                    *reinterpret_cast<float4*>(o + c0) = make_float4(f[0], f[1], f[2], f[3]);
                    *reinterpret_cast<float4*>(o + c1) = make_float4(f[4], f[5], f[6], f[7]);
                } else {
                    *reinterpret_cast<uint4*>(static_cast<uint16_t*>(out) + at + c0) =
                        SRC == 2 ? pack8<SPLIT ? 0 : DT>(f) : make_uint4(x0[kv][p].x, x0[kv][p].y, x1[kv][p].x, x1[kv][p].y);
                }
            }
        }
    }
}

// ---------------------------------------------------------------------------------------
// q4_attend_kernel
// ---------------------------------------------------------------------------------------
constexpr int Q4_THREADS = 128, Q4_WARPS = Q4_THREADS / 32;
constexpr int Q4_TILE = 16;              // keys of one tile
constexpr int Q4_STEP = 3;               // tiles that a warp takes in one step
constexpr int Q4_UNIT = Q4_TILE * Q4_WARPS;
constexpr int Q4_STAGES = 2;             // steps a warp has in flight or in use
constexpr int Q4_AHEAD = 32 / Q4_STEP * Q4_STEP;   // tiles whose rows the lanes of a warp look up at once
constexpr float Q4_NONE = -3.402823466e38f;   // reference of a column that has seen no key: no score is below it

// Columns (query token, head of the group) of one CTA by shape: four columns, each as two parts of
// its weights, or 8 or 16 columns.
enum { COLS_4 = 0, COLS_8 = 1, COLS_16 = 2 };
__host__ __device__ constexpr int q4_cols(int shape) { return shape == COLS_4 ? 4 : (shape == COLS_8 ? 8 : 16); }
// bytes of one tile: key codes, value codes, key scales, value scales of 16 rows
__host__ __device__ constexpr int q4_tile_bytes(int d) { return Q4_TILE * (d + d / GROUP * 8); }
__host__ __device__ constexpr int q4_ring_bytes(int d, int shape) {      // the ring, later the join of the warps
    const int ring = Q4_WARPS * Q4_STAGES * Q4_STEP * q4_tile_bytes(d);
    const int merge = Q4_WARPS * q4_cols(shape) * (d + 4) * 4;
    return ring > merge ? ring : merge;
}
// The tensor core cuts what it adds to an accumulator off at that accumulator's last place: after 150
// tiles the sums were 5e-6 too small, and where many keys average out to little that is the first thing
// wrong with the result.  Every Q4_FLUSH steps the sums move on to shared memory, by rounded additions.
constexpr int Q4_FLUSH = 4;
__host__ __device__ constexpr int q4_smem_bytes(int d, int shape) { return q4_ring_bytes(d, shape) + Q4_WARPS * q4_cols(shape) * d * 4; }

// Few warps with many registers: three tiles at a time keep the ALU and the tensor cores busier than
// more warps with one or two tiles would (4 x 131584 keys, graph replays: 4 heads a group 107..115 us, 8 heads 137;
// 16 warps an SM with two tiles 113..120 and 146; 20 with one 137 and 171).  16 columns take what two CTAs
// leave.  At d = 128 a third does not fit (86 KB of shared memory each).  At d = 64 it would, in fewer registers,
// and is better for long shares but not for short ones: 16 heads a group, 4 x 131584 keys 127 us with two and 124
// with three; four draft tokens, 4 x 64K keys 72 and 70; 8 x 8K 28.7 and 28.7; a window of 8K 22.6 and 24.6;
// three draft tokens of 8 heads, 8 x 8K 43 and 45.
__host__ __device__ constexpr int q4_ctas_per_sm(int shape) { return shape == COLS_16 ? 2 : 3; }

struct Q4Args {
    Pages pg;
    const int32_t* seq_lens;
    const uint16_t* q;
    uint16_t* out;
    float* lse;
    float* part;                // [2 * grid][cols][d + 2]
    long long q_stride, window;
    float scale_log2;
    int B, T, Hq, G, col_tiles, grid;
    uint32_t two16;             // 2^16: a shift as a product
};

// What beginning an item costs a CTA (page look-up, queries, first tiles, join), in units: a share counts
// that much more for every item that begins in it, else the CTAs that get the short sequences of a mixed
// batch finish last.
constexpr int Q4_BEGIN = 10;

// keys of a sequence: first one read (multiple of 16), end, units, and what an item counts (0 if empty)
struct Span { int lo, len, units, weight; };
__device__ __forceinline__ Span q4_span(const Q4Args& a, int seq_len) {
    Span s;
    // a length that the block table cannot hold does not tell which rows hold keys: none counts
    s.len = seq_len > 0 && seq_len <= a.pg.capacity ? seq_len : 0;
    long long lo = a.window > 0 ? (long long)s.len - a.T + 1 - a.window : 0;
    if (lo < 0) lo = 0;
    s.lo = (int)lo & ~(Q4_TILE - 1);
    s.units = s.len > s.lo ? (s.len - s.lo + Q4_UNIT - 1) / Q4_UNIT : 0;
    s.weight = s.units > 0 ? s.units + Q4_BEGIN : 0;
    return s;
}
// Share c of `grid` in U >= grid units begins here (no share is empty).
__device__ __forceinline__ long long q4_share(long long U, int grid, int c) { return U * c / grid; }

__device__ __forceinline__ float ex2(float x) {
    float y;
    asm("ex2.approx.ftz.f32 %0, %1;" : "=f"(y) : "f"(x));
    return y;
}
__device__ __forceinline__ uint32_t movmatrix(uint32_t x) {
    uint32_t y;
    asm("movmatrix.sync.aligned.m8n8.trans.b16 %0, %1;" : "=r"(y) : "r"(x));
    return y;
}
// c += a * b, and c = a * b
template <int DT>
__device__ __forceinline__ void mma16816(float (&c)[4], uint32_t a0, uint32_t a1, uint32_t a2, uint32_t a3, uint32_t b0, uint32_t b1) {
    if (DT == TYPE_BF16)
        asm("mma.sync.aligned.m16n8k16.row.col.f32.bf16.bf16.f32 {%0,%1,%2,%3}, {%4,%5,%6,%7}, {%8,%9}, {%0,%1,%2,%3};"
            : "+f"(c[0]), "+f"(c[1]), "+f"(c[2]), "+f"(c[3]) : "r"(a0), "r"(a1), "r"(a2), "r"(a3), "r"(b0), "r"(b1));
    else
        asm("mma.sync.aligned.m16n8k16.row.col.f32.f16.f16.f32 {%0,%1,%2,%3}, {%4,%5,%6,%7}, {%8,%9}, {%0,%1,%2,%3};"
            : "+f"(c[0]), "+f"(c[1]), "+f"(c[2]), "+f"(c[3]) : "r"(a0), "r"(a1), "r"(a2), "r"(a3), "r"(b0), "r"(b1));
}
__device__ __forceinline__ void mma16816_first(float (&c)[4], uint32_t a0, uint32_t a1, uint32_t a2, uint32_t a3, uint32_t b0, uint32_t b1) {
    asm("mma.sync.aligned.m16n8k16.row.col.f32.f16.f16.f32 {%0,%1,%2,%3}, {%4,%5,%6,%7}, {%8,%9}, {%10,%10,%10,%10};"
        : "=f"(c[0]), "=f"(c[1]), "=f"(c[2]), "=f"(c[3]) : "r"(a0), "r"(a1), "r"(a2), "r"(a3), "r"(b0), "r"(b1), "f"(0.f));
}

// Codes as operands: the bits of a code ARE a small number.  In bf16 bits 0..7 count in steps of 2^-133
// (subnormals, then the first exponent), in fp16 bits 0..10 in steps of 2^-24, and the tensor core
// multiplies subnormals exactly.  So a mask makes the operand and no offset has to be taken out of the
// sums again.  A byte b = n0 + 16 n1 goes in as n0 and as b: four instructions for the eight codes of a
// word instead of the seven of four masks and three shifts.  What b brings too much is put right in the
// other operand (keys) or once at the end (values).
//
// What bounds the kernel short of HBM is instructions, on the ALU most of all, where masks, shifts and byte
// permutations go, and the power that they take: 4 x 131584 keys take 107 us in short runs, 88% of the copy rate,
// and 118..125 us back to back, where the card is at 1000 W and 1.6 GHz.  Measured when this form was chosen, against
// its 121 us: n0, 16 n1 and a shift for the upper bytes of keys and values 132 us; that shift as a product 142 us
// (its two issue slots cost more); e4m3 operands for the keys 143 us (mma converts them to fp16, on the ALU).
// Queries as whole numbers against 8-bit integer operands take 6% less than this form, but hold only 2^-15 of a
// row's largest element.
__device__ __forceinline__ void code_bytes(uint32_t x, uint32_t (&c)[4]) {
    c[0] = x & 0x000f000fu;                      // codes (0,4)
    c[1] = __byte_perm(x, 0u, 0x4240);           // bytes 0 and 2: (0,4) + 16 (1,5)
    c[3] = __byte_perm(x, 0u, 0x4341);           // bytes 1 and 3: (2,6) + 16 (3,7)
    c[2] = c[3] & 0x000f000fu;                   // codes (2,6)
}
__device__ __forceinline__ void code_words(uint32_t x, uint32_t (&c)[4]) {
    const uint32_t y = x >> 8;
    c[0] = x & 0x000f000fu;                      // codes (0,4)
    c[1] = x & 0x00f000f0u;                      // 16 times codes (1,5)
    c[2] = y & 0x000f000fu;                      // codes (2,6)
    c[3] = y & 0x00f000f0u;                      // 16 times codes (3,7)
}
// n0 and b of the lower or upper half words of two keys: codes 0..3 of the first, of the second.
__device__ __forceinline__ void pair_bytes(uint32_t z, uint32_t (&c)[4]) {
    c[0] = z & 0x000f000fu;
    c[1] = z & 0x00ff00ffu;
    c[3] = __byte_perm(z, 0u, 0x4341);
    c[2] = c[3] & 0x000f000fu;
}
__device__ __forceinline__ float2 step_min(uint32_t x, uint32_t two16) {
    return make_float2(__uint_as_float(x * two16), __uint_as_float(x & 0xffff0000u));
}
// Whether one of two bf16 values is an infinity or NaN.
__device__ __forceinline__ bool not_finite(uint32_t x) { return (x & 0x7f80u) == 0x7f80u || (x & 0x7f800000u) == 0x7f800000u; }
__device__ __forceinline__ uint32_t lds32(uint32_t addr) {
    uint32_t x;
    asm volatile("ld.shared.u32 %0, [%1];" : "=r"(x) : "r"(addr) : "memory");
    return x;
}
__device__ __forceinline__ void sts32(uint32_t addr, uint32_t x) { asm volatile("st.shared.u32 [%0], %1;" ::"r"(addr), "r"(x) : "memory"); }
__device__ __forceinline__ uint2 lds64(uint32_t addr) {
    uint2 x;
    asm volatile("ld.shared.v2.u32 {%0,%1}, [%2];" : "=r"(x.x), "=r"(x.y) : "r"(addr) : "memory");
    return x;
}
// Weights carry 2^64 through the reference of their exponentials: it keeps their products with the
// subnormals in the middle of the fp32 range.  With steps s, a weight (up to 2^72) times s has to be finite
// (s < 2^55) and 2^64 s 2^-133 normal (s >= 2^-57); 2^20 weights of 2^72 times minima are below 2^128 for
// minima below 2^36.
constexpr float TWO64 = 18446744073709551616.f, TWO69 = 32.f * TWO64;     // 2^-133 * 2^64 = 1 / TWO69

// One warp's running state over the keys that it has seen.
template <int D, int NT, bool PACKED>
struct Q4State {
    static constexpr int NG = D / GROUP, NC = PACKED ? 1 : 2;
    float o[NG][4][NT][4];      // codes and bytes times weights: channel pairs x columns
    float msum[NG][NT][NC];     // weights times minima, over this lane's rows
    float l[NT][NC], ref[NT][NC];   // sum of weights; reference of the exponentials minus 64
};

// Mathematics.  With a key row held as s_g n_c + m_g per group g of 64 channels,
//     q . k = sum_g ( s_g (q . n)_g + m_g (sum of q)_g )
// so the codes go into the tensor core as they are and step and minimum are applied to the 16 x 8
// result.  The same for values: sum_j p_j v_j = sum_j (p_j s_j) n_j + sum_j p_j m_j, the weight p_j s_j
// entering as two bf16 parts (hi cut off, lo rounded: within 2^-16).  Keys are the M side of both products (16 keys
// or 16 channels), the columns the N side: with 4 columns the two parts of a weight fill the 8 columns
// of one product, so the second part is free.
//
// A warp works alone on tiles of 16 keys (2.3 KB at d = 128), three at a time, through its own ring of
// cp.async stages; warps meet only when a sequence's share ends.  The reference of the exponentials
// moves only when a score exceeds it by 2^8: one vote per step instead of a reduction.
//
// Channels are matched to the fragments so that no code moves between lanes: key codes of lane quarter
// t are channels 64 g + 16 t .. + 15, value codes of lane group r channels 64 g + 8 r .. + 7.
template <int DT, int D, int SHAPE>
__global__ void __launch_bounds__(Q4_THREADS, q4_ctas_per_sm(SHAPE)) q4_attend_kernel(const __grid_constant__ Q4Args a) {
    constexpr bool PACKED = SHAPE == COLS_4;
    constexpr int NT = SHAPE == COLS_16 ? 2 : 1, U = Q4_STEP;
    constexpr int COLS = q4_cols(SHAPE), NG = D / GROUP, NC = PACKED ? 1 : 2, PARTS = PACKED ? 1 : 2;
    constexpr int TILE = q4_tile_bytes(D), KB = Q4_TILE * D / 2, SB = Q4_TILE * NG * 4, RING = Q4_STAGES * U * TILE;
    extern __shared__ __align__(128) unsigned char smem[];

    const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5, t4 = lane & 3, r8 = lane >> 2;
    const int per_seq = a.pg.H_kv * a.col_tiles;

    pdl_wait();
    pdl_start_next();
    // Every warp adds up the weights of the sequences by itself, 128 at a time: first the total, then
    // the sequence in which this CTA's share begins (up to 128 lengths are still in registers then).
    long long total = 0, u = 0, u_end = 0, before = 0;   // before: weight before sequence b
    int shares = 0, b = 0, b_len = 0;
    {
        constexpr int EACH = 4;
        int len[EACH], w[EACH], mine = 0, incl = 0;
        for (int pass = 0; pass < 2; ++pass) {
            long long run = 0;
            for (int b0 = 0; b0 < a.B; b0 += 32 * EACH) {
                const int first = b0 + lane * EACH;
                if (pass == 0 || a.B > 32 * EACH) {
                    mine = 0;
#pragma unroll
                    for (int i = 0; i < EACH; ++i) len[i] = first + i < a.B ? a.seq_lens[first + i] : 0;
#pragma unroll
                    for (int i = 0; i < EACH; ++i) {
                        w[i] = q4_span(a, len[i]).weight * per_seq;
                        mine += w[i];
                    }
                    incl = mine;
#pragma unroll
                    for (int o = 1; o < 32; o <<= 1) {
                        const int x = __shfl_up_sync(0xffffffffu, incl, o);
                        if (lane >= o) incl += x;
                    }
                }
                const int all = __shfl_sync(0xffffffffu, incl, 31);
                if (pass == 1) {
                    const long long lo = run + incl - mine;
                    const uint32_t hit = __ballot_sync(0xffffffffu, u >= lo && u < lo + mine);
                    if (hit) {                           // one lane has it
                        long long at = lo;
                        int bb = first, ll = len[0];
#pragma unroll
                        for (int i = 0; i < EACH - 1; ++i)
                            if (bb == first + i && u >= at + w[i]) { at += w[i]; bb = first + i + 1; ll = len[i + 1]; }
                        const int src = __ffs(hit) - 1;
                        before = __shfl_sync(0xffffffffu, at, src);
                        b = __shfl_sync(0xffffffffu, bb, src);
                        b_len = __shfl_sync(0xffffffffu, ll, src);
                        break;
                    }
                }
                run += all;
            }
            if (pass == 0) {
                total = run;
                shares = total < a.grid ? (int)total : a.grid;
                if ((int)blockIdx.x >= shares) return;
                u = q4_share(total, shares, blockIdx.x);
                u_end = q4_share(total, shares, blockIdx.x + 1);
            }
        }
    }
    Span sp = q4_span(a, b_len);
    const long long u_begin = u;

    const uint32_t ring = (uint32_t)__cvta_generic_to_shared(smem) + warp * RING;
    float* s_merge = reinterpret_cast<float*>(smem);
    // this lane's sums over the earlier steps: pairs of channels, [group][pair][tile][column][lane]
    float2* const s_sum = reinterpret_cast<float2*>(smem + q4_ring_bytes(D, SHAPE)) + warp * (COLS * D / 2) + lane;

    // Where this lane's codes lie in a block of 16 rows whose 128-byte lines have their 16-byte slots
    // exchanged by line (slot ^ 2 (line mod 4)), so that every read below touches each bank once.
    // Keys: row r8, byte 8 t4 of a group's 32.  Values: row 2 t4, byte 4 r8.
    auto swz = [](int r, int x) -> int {
        const int lin = r * (D / 2) + x, line = lin >> 7;
        return (line << 7) + ((((lin >> 4) & 7) ^ (2 * (line & 3))) << 4) + (lin & 15);
    };
    constexpr int ROW8 = 8 * D / 2;                      // 8 rows on: for d = 64 the exchange differs by 4 slots
    constexpr int ROW8_X = D == 64 ? 64 : 0;
    constexpr int ROW1_X = D / 2;                        // the odd row of a pair: its slot bit
    const uint32_t k_at = ring + swz(r8, 8 * t4), v_at = ring + KB + swz(2 * t4, 4 * r8);
    // the same with the exchanged slots, relative to the first: group 1, the odd row, 8 rows on
    auto moved = [](uint32_t at, uint32_t base, int x) { return base + ((at - base) ^ x); };
    uint32_t k_addr[NG][2], v_addr[NG][2][2];            // [group][8 rows on], [group][odd row][8 rows on]
#pragma unroll
    for (int g = 0; g < NG; ++g)
#pragma unroll
        for (int e = 0; e < 2; ++e) {
            k_addr[g][e] = moved(k_at, ring, 32 * g ^ (e ? ROW8_X : 0));
#pragma unroll
            for (int odd = 0; odd < 2; ++odd) v_addr[g][odd][e] = moved(v_at, ring + KB, 32 * g ^ (odd ? ROW1_X : 0) ^ (e ? ROW8_X : 0));
        }
    const uint32_t s_addr = ring + 2 * KB + r8 * (NG * 4);
    // what this lane copies: 16 bytes of every 512 of the codes, and a piece of the scales
    const uint32_t c_dst = ring + swz(lane * 16 / (D / 2), lane * 16 % (D / 2));
    const unsigned char* const k_src = a.pg.k + lane * 16;
    const unsigned char* const v_src = a.pg.v + lane * 16;
    const unsigned char* const s_src = (lane < SB / 16 ? a.pg.ks : a.pg.vs - SB) + lane * 16;

    while (u < u_end) {
        while (u >= before + (long long)sp.weight * per_seq) {
            before += (long long)sp.weight * per_seq;
            ++b;
            sp = q4_span(a, a.seq_lens[b]);
        }
        const int in_seq = (int)(u - before);
        const int item = in_seq / sp.weight, at = in_seq - item * sp.weight;
        const int h = item / a.col_tiles, ct = item - h * a.col_tiles;
        const int here = u_end - u < sp.weight - at ? (int)(u_end - u) : sp.weight - at;
        u += here;
        const int k_unit = at > Q4_BEGIN ? at - Q4_BEGIN : 0, n_units = at + here - Q4_BEGIN - k_unit;
        if (n_units <= 0) continue;                      // a share that ends within an item's beginning
        const long long item_start = before + (long long)item * sp.weight;
        const int key0 = sp.lo + k_unit * Q4_UNIT;
        int key_end = key0 + n_units * Q4_UNIT;
        if (key_end > sp.len) key_end = sp.len;
        // this warp's tiles: key0 + (i * warps + warp) * 16
        const int n_all = (key_end - key0 + Q4_TILE - 1) / Q4_TILE;
        const int n_tiles = n_all > warp ? (n_all - warp + Q4_WARPS - 1) / Q4_WARPS : 0;

        // ---- queries of this column tile: asked for here, used below ---------------------------
        const int cols_here = a.T * a.G - ct * COLS < COLS ? a.T * a.G - ct * COLS : COLS;
        uint4 q_raw[NT][NG][2];
#pragma unroll
        for (int nt = 0; nt < NT; ++nt) {
            const int col = PACKED ? r8 >> 1 : nt * 8 + r8;
            const int cc = ct * COLS + (col < cols_here ? col : 0);
            const int tok = cc / a.G, head = h * a.G + (cc - tok * a.G);
            const uint16_t* qp = a.q + ((long long)b * a.T + tok) * a.q_stride + (long long)head * D;
#pragma unroll
            for (int g = 0; g < NG; ++g)
#pragma unroll
                for (int j = 0; j < 2; ++j) q_raw[nt][g][j] = *reinterpret_cast<const uint4*>(qp + g * GROUP + 16 * t4 + 8 * j);
        }

        // ---- page rows of the next tiles, one per lane ---------------------------------------
        // (32 bits: the host refuses caches of 2^32 rows or more.)  A tile whose page is out of range
        // is read from row 0 and masked; that such a tile exists is remembered for the whole share.
        bool bad = false;
        auto row_of = [&](int i) -> long long { return cache_row(a.pg, b, key0 + ((long long)i * Q4_WARPS + warp) * Q4_TILE); };
        auto tile_row = [&](int i) -> uint32_t {
            if (i >= n_tiles) return 0u;
            const long long r = row_of(i);
            bad |= r < 0;
            return r < 0 ? 0u : (uint32_t)(r + (long long)h * a.pg.page_size);
        };
        uint32_t rows_now = tile_row(lane), rows_next = tile_row(Q4_AHEAD + lane);
        bool some_bad = __any_sync(0xffffffffu, bad);
        int ahead = 0;                                   // tiles issued from rows_now

        auto issue = [&](int step, int st) {             // tiles of `step` into stage st
            if (ahead == Q4_AHEAD) {
                ahead = 0;
                rows_now = rows_next;
                rows_next = tile_row(step * U + Q4_AHEAD + lane);
                some_bad = __any_sync(0xffffffffu, bad);
            }
#pragma unroll
            for (int x = 0; x < U; ++x) {
                const int i = step * U + x;
                const uint32_t row = __shfl_sync(0xffffffffu, rows_now, ahead + x);
                if (i < n_tiles) {
                    const uint32_t dst = c_dst + (st * U + x) * TILE;
                    const unsigned char* kp = k_src + (uint64_t)row * (D / 2);
                    const unsigned char* vp = v_src + (uint64_t)row * (D / 2);
#pragma unroll
                    for (int c = 0; c < KB / 512; ++c) {
                        cp_async16(dst + c * 512, kp + c * 512);
                        cp_async16(dst + KB + c * 512, vp + c * 512);
                    }
                    if (lane < SB / 8) cp_async16(ring + (st * U + x) * TILE + 2 * KB + lane * 16, s_src + (uint64_t)row * (NG * 4));
                }
            }
            ahead += U;
            cp_async_commit();
        };
        const int n_steps = (n_tiles + U - 1) / U;
#pragma unroll
        for (int i = 0; i < Q4_STAGES - 1; ++i) issue(i, i);

        // ---- query fragments --------------------------------------------------------------------
        // Fragment column n of tile nt is column (PACKED: n / 2, else nt * 8 + n).  Queries enter as
        // fp16, scaled by the power of two that brings the column's largest element to 2^14..2^15: exact
        // but for elements below 2^-24 of the largest (off by 2^-35 of it).
        uint32_t qf[NT][NG][4][2];
        float qsum[NT][NG][NC], unit[NT][NC];            // sum of q in units of the products; their value in powers of two
#pragma unroll
        for (int nt = 0; nt < NT; ++nt) {
            float f[NG][2][8], big = 0.f, sum[NG];
#pragma unroll
            for (int g = 0; g < NG; ++g) {
                sum[g] = 0.f;
#pragma unroll
                for (int j = 0; j < 2; ++j) {
                    unpack8<DT>(q_raw[nt][g][j], f[g][j]);
#pragma unroll
                    for (int e = 0; e < 8; ++e) { sum[g] += f[g][j][e]; big = fmaxf(big, fabsf(f[g][j][e])); }
                }
                sum[g] += __shfl_xor_sync(0xffffffffu, sum[g], 1);
                sum[g] += __shfl_xor_sync(0xffffffffu, sum[g], 2);
            }
            big = fmaxf(big, __shfl_xor_sync(0xffffffffu, big, 1));
            big = fmaxf(big, __shfl_xor_sync(0xffffffffu, big, 2));
            // 2^(14 - exponent of the largest), kept within what a float can hold both ways
            int e2 = 141 - (int)(__float_as_uint(big) >> 23);
            e2 = e2 > 100 ? 100 : (e2 < -103 ? -103 : e2);
            const float to_unit = __uint_as_float((uint32_t)(127 + e2) << 23);
            const float of_unit = __uint_as_float((uint32_t)(127 + 24 - e2) << 23);      // products: n q 2^-24
            // PACKED: q0 n0 + q1 n1 = (q0 - q1 / 16) n0 + (q1 / 16) b.  The difference needs more bits than
            // fp16 has: the odd columns take what it leaves over (2^-23 of the larger of the two is lost).
            // Otherwise that would be a product more, dearer than the masks it saves: q1 / 16 against 16 n1.
#pragma unroll
            for (int g = 0; g < NG; ++g)
#pragma unroll
                for (int j = 0; j < 2; ++j)
#pragma unroll
                    for (int e = 0; e < 2; ++e) {        // channels (0,4) (1,5), then (2,6) (3,7) of the eight
                        float q0[2], q1[2];
#pragma unroll
                        for (int i = 0; i < 2; ++i) {
                            q0[i] = f[g][j][2 * e + 4 * i] * to_unit;
                            q1[i] = f[g][j][2 * e + 4 * i + 1] * (0.0625f * to_unit);
                        }
                        if (PACKED) {
                            const float d0 = q0[0] - q1[0], d1 = q0[1] - q1[1];
                            const uint32_t hi = pack2<TYPE_FP16>(d0, d1);
                            const float2 hf = unpack2<TYPE_FP16>(hi);
                            const bool rest = r8 & 1;
                            qf[nt][g][2 * j + e][0] = rest ? pack2<TYPE_FP16>(d0 - hf.x, d1 - hf.y) : hi;
                            qf[nt][g][2 * j + e][1] = rest ? 0u : pack2<TYPE_FP16>(q1[0], q1[1]);
                        } else {
                            qf[nt][g][2 * j + e][0] = pack2<TYPE_FP16>(q0[0], q0[1]);
                            qf[nt][g][2 * j + e][1] = pack2<TYPE_FP16>(q1[0], q1[1]);
                        }
                    }
            // lanes hold columns 2 t4 + c of the result
#pragma unroll
            for (int c = 0; c < NC; ++c) {
                const float of = __shfl_sync(0xffffffffu, of_unit, (2 * t4 + c) * 4);
                unit[nt][c] = a.scale_log2 * of;
#pragma unroll
                for (int g = 0; g < NG; ++g) qsum[nt][g][c] = __shfl_sync(0xffffffffu, sum[g], (2 * t4 + c) * 4) / of;
            }
        }
        // keys below safe_end and from safe_lo on count for every column, and are in the ring
        const int safe_end = sp.len - a.T + 1 < key_end ? sp.len - a.T + 1 : key_end;
        const int safe_lo = a.window > 0 && sp.len > a.window ? (int)(sp.len - a.window) : 0;

        Q4State<D, NT, PACKED> st;
#pragma unroll
        for (int nt = 0; nt < NT; ++nt) {
#pragma unroll
            for (int g = 0; g < NG; ++g) {
#pragma unroll
                for (int m = 0; m < 4; ++m)
#pragma unroll
                    for (int e = 0; e < 4; ++e) st.o[g][m][nt][e] = 0.f;
#pragma unroll
                for (int c = 0; c < NC; ++c) st.msum[g][nt][c] = 0.f;
            }
#pragma unroll
            for (int c = 0; c < NC; ++c) { st.l[nt][c] = 0.f; st.ref[nt][c] = Q4_NONE; }
        }

        int stage = 0, since = 0;
        bool flushed = false;
        auto flush = [&]() {
#pragma unroll
            for (int nt = 0; nt < NT; ++nt)
#pragma unroll
                for (int c = 0; c < NC; ++c)
#pragma unroll
                    for (int g = 0; g < NG; ++g)
#pragma unroll
                        for (int m = 0; m < 4; ++m) {    // accumulator rows r8 and r8 + 8: n0 and n0 + 16 n1 of
                            float (&o)[4] = st.o[g][m][nt];          // channels 2 m, 2 m + 1
                            float x = o[c], y = o[2 + c];
                            if (PACKED) { x += o[1]; y += o[3]; }
                            float2* at = s_sum + (((g * 4 + m) * NT + nt) * NC + c) * 32;
                            float2 v = make_float2(x * TWO69, (y - x) * (TWO69 / 16.f));
                            if (flushed) { const float2 w = *at; v.x += w.x; v.y += w.y; }
                            *at = v;
                            if (PACKED) { o[0] = o[1] = o[2] = o[3] = 0.f; } else { o[c] = o[2 + c] = 0.f; }
                        }
            flushed = true;
            since = 0;
        };
#pragma unroll 1
        for (int step = 0; step < n_steps; ++step) {
            if (since == Q4_FLUSH) flush();
            ++since;
            cp_async_wait<Q4_STAGES - 2>();
            __syncwarp();
            const int ring_at = stage * (U * TILE);
            // the next tiles go into the stage that the previous step left
            issue(step + Q4_STAGES - 1, stage == 0 ? Q4_STAGES - 1 : stage - 1);
            stage = stage == Q4_STAGES - 1 ? 0 : stage + 1;
            const int kbase = key0 + (step * U * Q4_WARPS + warp) * Q4_TILE;

            // ---- scores --------------------------------------------------------------------------
            float sc[U][NT][2][NC];                      // rows r8 and r8 + 8, in powers of two
#pragma unroll
            for (int x = 0; x < U; ++x) {
                constexpr int NGW = NG;
                const int blk = ring_at + x * TILE;
                uint32_t w_s[2][NGW];                    // step and minimum of rows r8 and r8 + 8, per group
#pragma unroll
                for (int r = 0; r < 2; ++r) {
                    const uint32_t at = s_addr + blk + r * (8 * NG * 4);
                    if (NG == 2) {
                        const uint2 z = lds64(at);
                        w_s[r][0] = z.x;
                        w_s[r][NG - 1] = z.y;
                    } else {
                        w_s[r][0] = lds32(at);
                    }
                }
#pragma unroll
                for (int g = 0; g < NG; ++g) {
                    const uint2 w0 = lds64(k_addr[g][0] + blk), w8 = lds64(k_addr[g][1] + blk + ROW8);
                    float acc[NT][4];
#pragma unroll
                    for (int j = 0; j < 2; ++j) {
                        uint32_t c0[4], c8[4];
                        if (PACKED) {
                            code_bytes(j ? w0.y : w0.x, c0);
                            code_bytes(j ? w8.y : w8.x, c8);
                        } else {
                            code_words(j ? w0.y : w0.x, c0);
                            code_words(j ? w8.y : w8.x, c8);
                        }
#pragma unroll
                        for (int nt = 0; nt < NT; ++nt) {
                            if (j == 0) mma16816_first(acc[nt], c0[0], c8[0], c0[1], c8[1], qf[nt][g][0][0], qf[nt][g][0][1]);
                            else mma16816<TYPE_FP16>(acc[nt], c0[0], c8[0], c0[1], c8[1], qf[nt][g][2][0], qf[nt][g][2][1]);
                            mma16816<TYPE_FP16>(acc[nt], c0[2], c8[2], c0[3], c8[3], qf[nt][g][2 * j + 1][0], qf[nt][g][2 * j + 1][1]);
                        }
                    }
#pragma unroll
                    for (int r = 0; r < 2; ++r) {
                        const float2 s = step_min(w_s[r][g], a.two16);
#pragma unroll
                        for (int nt = 0; nt < NT; ++nt)
#pragma unroll
                            for (int c = 0; c < NC; ++c)
                                sc[x][nt][r][c] = fmaf(s.x, PACKED ? acc[nt][2 * r] + acc[nt][2 * r + 1] : acc[nt][2 * r + c],
                                                       g == 0 ? s.y * qsum[nt][g][c] : fmaf(s.y, qsum[nt][g][c], sc[x][nt][r][c]));
                    }
                }
            }

            // ---- weights -------------------------------------------------------------------------
            // An infinite score becomes NaN (times 0, plus itself): +inf leaves no weights to speak of, and
            // -inf, which stands for a key that does not count, would drop this one without a trace.
#pragma unroll
            for (int x = 0; x < U; ++x)
#pragma unroll
                for (int nt = 0; nt < NT; ++nt)
#pragma unroll
                    for (int r = 0; r < 2; ++r)
#pragma unroll
                        for (int c = 0; c < NC; ++c) {
                            const float y = sc[x][nt][r][c] * unit[nt][c];
                            sc[x][nt][r][c] = fmaf(y, 0.f, y);
                        }
            if (some_bad || kbase + (U - 1) * Q4_UNIT + Q4_TILE > safe_end || kbase < safe_lo) {
                // Keys that do not count for a column: score -inf, so weight 0.
#pragma unroll
                for (int x = 0; x < U; ++x) {
                    const int key = kbase + x * Q4_UNIT + r8;
                    const bool none = some_bad && row_of(step * U + x) < 0;
#pragma unroll
                    for (int nt = 0; nt < NT; ++nt)
#pragma unroll
                        for (int c = 0; c < NC; ++c) {
                            const int mycol = PACKED ? t4 : nt * 8 + 2 * t4 + c;
                            const int tk = (ct * COLS + (mycol < cols_here ? mycol : 0)) / a.G;
                            const int lim = sp.len - a.T + 1 + tk;          // keys [low, lim) count
                            const int low = a.window > 0 && lim > a.window ? (int)(lim - a.window) : 0;
                            const int end = lim < key_end ? lim : key_end;  // beyond key_end the ring holds no tile
#pragma unroll
                            for (int r = 0; r < 2; ++r)
                                if (none || key + 8 * r >= end || key + 8 * r < low) sc[x][nt][r][c] = -INFINITY;
                        }
                }
                // Rows that do not count may hold anything, and 0 times NaN is NaN: a row whose value step or
                // minimum is no finite number leaves the ring, and the columns for which it does count get NaN.
                bool wild = false;
#pragma unroll
                for (int x = 0; x < U; ++x)
#pragma unroll
                    for (int r = 0; r < 2; ++r)
#pragma unroll
                        for (int g = 0; g < NG; ++g) wild |= not_finite(lds32(s_addr + ring_at + x * TILE + SB + (r * 8 * NG + g) * 4));
                if (__any_sync(0xffffffffu, wild)) {
#pragma unroll
                    for (int x = 0; x < U; ++x)
#pragma unroll
                        for (int r = 0; r < 2; ++r) {
                            const uint32_t at = s_addr + ring_at + x * TILE + SB + r * (8 * NG * 4);
                            bool clear[NG];
#pragma unroll
                            for (int g = 0; g < NG; ++g) {
                                clear[g] = not_finite(lds32(at + 4 * g));
#pragma unroll
                                for (int nt = 0; nt < NT; ++nt)
#pragma unroll
                                    for (int c = 0; c < NC; ++c)
                                        if (clear[g] && sc[x][nt][r][c] != -INFINITY) st.msum[g][nt][c] = NAN;
                            }
                            __syncwarp();                // the four lanes of a row have read it
#pragma unroll
                            for (int g = 0; g < NG; ++g)
                                if (clear[g] && t4 == 0) sts32(at + 4 * g, 0u);
                        }
                    __syncwarp();
                }
            }
            bool grow = false;
#pragma unroll
            for (int nt = 0; nt < NT; ++nt)
#pragma unroll
                for (int c = 0; c < NC; ++c) {
                    float mx = fmaxf(sc[0][nt][0][c], sc[0][nt][1][c]);
#pragma unroll
                    for (int x = 1; x < U; ++x) mx = fmaxf(mx, fmaxf(sc[x][nt][0][c], sc[x][nt][1][c]));
                    grow |= mx > st.ref[nt][c] + 72.f;                      // 8 above the reference
                }
            if (__any_sync(0xffffffffu, grow)) {
#pragma unroll
                for (int nt = 0; nt < NT; ++nt) {
                    float f[NC];
#pragma unroll
                    for (int c = 0; c < NC; ++c) {
                        float mx = fmaxf(sc[0][nt][0][c], sc[0][nt][1][c]);
#pragma unroll
                        for (int x = 1; x < U; ++x) mx = fmaxf(mx, fmaxf(sc[x][nt][0][c], sc[x][nt][1][c]));
                        mx = fmaxf(mx, __shfl_xor_sync(0xffffffffu, mx, 4));
                        mx = fmaxf(mx, __shfl_xor_sync(0xffffffffu, mx, 8));
                        mx = fmaxf(mx, __shfl_xor_sync(0xffffffffu, mx, 16));
                        mx = fmaxf(mx - 64.f, st.ref[nt][c]);
                        f[c] = ex2(st.ref[nt][c] - mx);
                        st.ref[nt][c] = mx;
                        st.l[nt][c] *= f[c];
                    }
#pragma unroll
                    for (int g = 0; g < NG; ++g) {
#pragma unroll
                        for (int c = 0; c < NC; ++c) st.msum[g][nt][c] *= f[c];
#pragma unroll
                        for (int m = 0; m < 4; ++m)
#pragma unroll
                            for (int e = 0; e < 4; ++e) st.o[g][m][nt][e] *= f[PACKED ? 0 : (e & 1)];
                        if (flushed) {
#pragma unroll
                            for (int m = 0; m < 4; ++m)
#pragma unroll
                                for (int c = 0; c < NC; ++c) {
                                    float2* at = s_sum + (((g * 4 + m) * NT + nt) * NC + c) * 32;
                                    const float2 w = *at;
                                    *at = make_float2(w.x * f[c], w.y * f[c]);
                                }
                        }
                    }
                }
            }
#pragma unroll
            for (int x = 0; x < U; ++x)
#pragma unroll
                for (int nt = 0; nt < NT; ++nt)
#pragma unroll
                    for (int c = 0; c < NC; ++c) {
                        sc[x][nt][0][c] = ex2(sc[x][nt][0][c] - st.ref[nt][c]);
                        sc[x][nt][1][c] = ex2(sc[x][nt][1][c] - st.ref[nt][c]);
                        st.l[nt][c] += sc[x][nt][0][c] + sc[x][nt][1][c];
                    }

            // ---- values --------------------------------------------------------------------------
#pragma unroll
            for (int x = 0; x < U; ++x) {
                const int blk = ring_at + x * TILE;
                uint32_t w_s[2][NG];
#pragma unroll
                for (int r = 0; r < 2; ++r) {
                    const uint32_t at = s_addr + blk + SB + r * (8 * NG * 4);
                    if (NG == 2) {
                        const uint2 z = lds64(at);
                        w_s[r][0] = z.x;
                        w_s[r][NG - 1] = z.y;
                    } else {
                        w_s[r][0] = lds32(at);
                    }
                }
#pragma unroll
                for (int g = 0; g < NG; ++g) {
                    const float2 v0 = step_min(w_s[0][g], a.two16), v8 = step_min(w_s[1][g], a.two16);
                    // weights transposed to the N side: [part][rows 0-7, 8-15]; the second part is what
                    // cutting the first to 16 bits left over
                    uint32_t bw[NT][PARTS][2];
#pragma unroll
                    for (int nt = 0; nt < NT; ++nt)
#pragma unroll
                        for (int r = 0; r < 2; ++r) {
                            const float2 v = r ? v8 : v0;
                            const float w0 = sc[x][nt][r][0] * v.x;
                            const float h0 = __uint_as_float(__float_as_uint(w0) & 0xffff0000u), d0 = w0 - h0;
                            st.msum[g][nt][0] = fmaf(sc[x][nt][r][0], v.y, st.msum[g][nt][0]);
                            if (PACKED) {
                                bw[nt][0][r] = movmatrix(pack2<TYPE_BF16>(h0, d0));
                            } else {
                                const float w1 = sc[x][nt][r][NC - 1] * v.x;
                                const float d1 = w1 - __uint_as_float(__float_as_uint(w1) & 0xffff0000u);
                                st.msum[g][nt][NC - 1] = fmaf(sc[x][nt][r][NC - 1], v.y, st.msum[g][nt][NC - 1]);
                                bw[nt][0][r] = movmatrix(__byte_perm(__float_as_uint(w0), __float_as_uint(w1), 0x7632));
                                bw[nt][PARTS - 1][r] = movmatrix(pack2<TYPE_BF16>(d0, d1));
                            }
                        }
                    // codes of keys 2 t4, 2 t4 + 1, + 8, + 9 for channels 64 g + 8 r8 .. + 7
                    const uint32_t w0 = lds32(v_addr[g][0][0] + blk), w1 = lds32(v_addr[g][1][0] + blk);
                    const uint32_t w8 = lds32(v_addr[g][0][1] + blk + ROW8), w9 = lds32(v_addr[g][1][1] + blk + ROW8);
#pragma unroll
                    for (int hh = 0; hh < 2; ++hh) {
                        uint32_t c0[4], c8[4];
                        pair_bytes(__byte_perm(w0, w1, hh ? 0x7632 : 0x5410), c0);
                        pair_bytes(__byte_perm(w8, w9, hh ? 0x7632 : 0x5410), c8);
#pragma unroll
                        for (int nt = 0; nt < NT; ++nt)
#pragma unroll
                            for (int part = 0; part < PARTS; ++part) {
                                mma16816<TYPE_BF16>(st.o[g][2 * hh][nt], c0[0], c0[1], c8[0], c8[1], bw[nt][part][0], bw[nt][part][1]);
                                mma16816<TYPE_BF16>(st.o[g][2 * hh + 1][nt], c0[2], c0[3], c8[2], c8[3], bw[nt][part][0], bw[nt][part][1]);
                            }
                    }
                }
            }
        }
        cp_async_wait<0>();
        flush();

        // ---- join the warps ---------------------------------------------------------------------
        // sums over the lanes that share columns (rows of the tiles); the 2^64 of the weights goes here
#pragma unroll
        for (int nt = 0; nt < NT; ++nt)
#pragma unroll
            for (int c = 0; c < NC; ++c) {
#pragma unroll
                for (int o = 4; o < 32; o <<= 1) {
                    st.l[nt][c] += __shfl_xor_sync(0xffffffffu, st.l[nt][c], o);
#pragma unroll
                    for (int g = 0; g < NG; ++g) st.msum[g][nt][c] += __shfl_xor_sync(0xffffffffu, st.msum[g][nt][c], o);
                }
                st.l[nt][c] *= 1.f / TWO64;
#pragma unroll
                for (int g = 0; g < NG; ++g) st.msum[g][nt][c] *= 1.f / TWO64;
            }
        __syncthreads();                                 // every warp is done with its ring
        // [warp][col][D + 2] (the two keep the columns of a store in different banks), then [warp][col]
        // reference and sum
        constexpr int LD = D + 2;
        float* s_ref = s_merge + Q4_WARPS * COLS * LD;
        float* s_l = s_ref + Q4_WARPS * COLS;
#pragma unroll
        for (int nt = 0; nt < NT; ++nt)
#pragma unroll
            for (int c = 0; c < NC; ++c) {
                const int col = PACKED ? t4 : nt * 8 + 2 * t4 + c;
                float* dst = s_merge + (warp * COLS + col) * LD + 8 * r8;
#pragma unroll
                for (int g = 0; g < NG; ++g)
#pragma unroll
                    for (int m = 0; m < 4; ++m)
                    {
                        const float2 v = s_sum[(((g * 4 + m) * NT + nt) * NC + c) * 32];
                        *reinterpret_cast<float2*>(dst + g * GROUP + 2 * m) = make_float2(v.x + st.msum[g][nt][c], v.y + st.msum[g][nt][c]);
                    }
                if (r8 == 0) { s_ref[warp * COLS + col] = st.ref[nt][c]; s_l[warp * COLS + col] = st.l[nt][c]; }
            }
        __syncthreads();
        // per column: common reference, the warps' factors to it (in place of their references), sum
        if (tid < COLS) {
            float mx = Q4_NONE, l = 0.f;
#pragma unroll
            for (int w = 0; w < Q4_WARPS; ++w) mx = fmaxf(mx, s_ref[w * COLS + tid]);
#pragma unroll
            for (int w = 0; w < Q4_WARPS; ++w) {
                const float f = ex2(s_ref[w * COLS + tid] - mx);
                l = fmaf(f, s_l[w * COLS + tid], l);
                s_ref[w * COLS + tid] = f;
            }
            s_l[tid] = l;
            s_l[COLS + tid] = mx;
        }
        __syncthreads();
        const bool whole = n_units == sp.units;
        float* part = a.part + (long long)(2 * blockIdx.x + (item_start > u_begin ? 1 : 0)) * COLS * (D + 2);
        const int ch = tid % D;                          // a thread keeps its channel
        for (int col = tid / D; col < cols_here; col += Q4_THREADS / D) {
            float o = 0.f;
#pragma unroll
            for (int w = 0; w < Q4_WARPS; ++w) o = fmaf(s_ref[w * COLS + col], s_merge[(w * COLS + col) * LD + ch], o);
            const float l = s_l[col], mx = s_l[COLS + col];
            if (whole) {
                const int cc = ct * COLS + col, tok = cc / a.G, head = h * a.G + (cc - tok * a.G);
                const long long row = ((long long)b * a.T + tok) * a.Hq + head;
                const float y = l == 0.f ? 0.f : o / l;         // (no key; a NaN goes on)
                a.out[row * D + ch] = (uint16_t)(pack2<DT>(y, 0.f) & 0xffffu);
                if (a.lse && ch == 0) a.lse[row] = l == 0.f ? -INFINITY : (mx + 64.f + log2f(l)) * 0.6931471805599453f;
            } else {
                part[col * (D + 2) + ch] = o;
                if (ch == 0) { part[col * (D + 2) + D] = mx; part[col * (D + 2) + D + 1] = l; }
            }
        }
        __syncthreads();                                 // the ring is free for the next share
    }
}

// Joins the parts of items (sequence, KV head, column tile) that more than one CTA worked on, and
// writes the rows of sequences without keys.  One CTA of D threads per item and column.
template <int DT, int D, int SHAPE>
__global__ void __launch_bounds__(D) q4_combine_kernel(const __grid_constant__ Q4Args a) {
    constexpr int COLS = q4_cols(SHAPE), WARPS = D / 32, AHEAD = 8;
    __shared__ long long s_sum[2][WARPS];
    const int tid = threadIdx.x, per_seq = a.pg.H_kv * a.col_tiles;
    const int b = blockIdx.x / per_seq, item = blockIdx.x - b * per_seq;
    const int h = item / a.col_tiles, ct = item - h * a.col_tiles, col = blockIdx.y;
    const int cols_here = a.T * a.G - ct * COLS < COLS ? a.T * a.G - ct * COLS : COLS;
    if (col >= cols_here) { pdl_wait(); return; }        // (a grid that ends is one whose predecessor has)
    long long mine = 0, all = 0;
    for (int bb = tid; bb < a.B; bb += D) {
        const int n = q4_span(a, a.seq_lens[bb]).weight;
        all += n;
        if (bb < b) mine += n;
    }
    const int weight = q4_span(a, a.seq_lens[b]).weight;
#pragma unroll
    for (int o = 16; o > 0; o >>= 1) {
        mine += __shfl_down_sync(0xffffffffu, mine, o);
        all += __shfl_down_sync(0xffffffffu, all, o);
    }
    if ((tid & 31) == 0) { s_sum[0][tid >> 5] = mine; s_sum[1][tid >> 5] = all; }
    __syncthreads();
    mine = all = 0;
#pragma unroll
    for (int w = 0; w < WARPS; ++w) { mine += s_sum[0][w]; all += s_sum[1][w]; }
    const long long total = all * per_seq, ua = mine * per_seq + (long long)item * weight, ub = ua + weight;
    const int shares = total < a.grid ? (int)total : a.grid;
    int c0 = 0, c1 = -1;
    if (weight > 0) {
        // CTA whose share holds x: the largest c with total * c / shares <= x; the first key's, the last key's
        c0 = (int)(((ua + Q4_BEGIN + 1) * shares + total - 1) / total) - 1;
        c1 = (int)((ub * shares + total - 1) / total) - 1;
    }
    // only the first CTA can have begun another item before this one
    const float* p0 = a.part + ((long long)(2 * c0 + (weight > 0 && ua > q4_share(total, shares, c0) ? 1 : 0)) * COLS + col) * (D + 2);
    const float* p1 = a.part + ((long long)(2 * (c0 + 1)) * COLS + col) * (D + 2);
    constexpr long long NEXT = 2ll * COLS * (D + 2);
    pdl_wait();                                          // (the lengths were there before the first kernel began)
    if (weight > 0 && c0 == c1) return;                  // one CTA had it all and wrote it
    float mx = Q4_NONE, l = 0.f, o = 0.f;
    for (int c = c0; c <= c1; c += AHEAD) {
        float m[AHEAD], s[AHEAD], x[AHEAD];
#pragma unroll
        for (int i = 0; i < AHEAD; ++i) {
            const bool in = c + i <= c1;
            const float* p = c + i == c0 ? p0 : p1 + (long long)(c + i - c0 - 1) * NEXT;
            m[i] = in ? p[D] : Q4_NONE;
            s[i] = in ? p[D + 1] : 0.f;
            x[i] = in ? p[tid] : 0.f;
        }
        float top = mx;
#pragma unroll
        for (int i = 0; i < AHEAD; ++i) top = fmaxf(top, m[i]);
        const float f = ex2(mx - top);
        l *= f;
        o *= f;
        mx = top;
#pragma unroll
        for (int i = 0; i < AHEAD; ++i) {
            const float g = ex2(m[i] - top);
            l = fmaf(g, s[i], l);
            o = fmaf(g, x[i], o);
        }
    }
    const int cc = ct * COLS + col, tok = cc / a.G, head = h * a.G + (cc - tok * a.G);
    const long long row = ((long long)b * a.T + tok) * a.Hq + head;
    const float y = l == 0.f ? 0.f : o / l;         // (no key; a NaN goes on)
    a.out[row * D + tid] = (uint16_t)(pack2<DT>(y, 0.f) & 0xffffu);
    if (a.lse && tid == 0) a.lse[row] = l == 0.f ? -INFINITY : (mx + 64.f + log2f(l)) * 0.6931471805599453f;
}

}  // namespace retopk_cache
