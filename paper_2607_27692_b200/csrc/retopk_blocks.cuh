// Device code that selects blocks of keys by a cheap score (sm_100a).
//
//   bounds_kernel   least and largest key of each block, channel by channel
//   score_kernel    upper bound of a block's scores from its bounds
//   pick_kernel     the blocks with the largest bounds
#pragma once
#include "retopk_attend.cuh"

namespace retopk_cache {

// ---------------------------------------------------------------------------------------
// bounds_kernel
// ---------------------------------------------------------------------------------------
template <int DT> __device__ __forceinline__ uint32_t min2_nan(uint32_t a, uint32_t b) {
    uint32_t c;
    if (DT == TYPE_BF16) asm("min.NaN.bf16x2 %0, %1, %2;" : "=r"(c) : "r"(a), "r"(b));
    else asm("min.NaN.f16x2 %0, %1, %2;" : "=r"(c) : "r"(a), "r"(b));
    return c;
}
template <int DT> __device__ __forceinline__ uint32_t max2_nan(uint32_t a, uint32_t b) {
    uint32_t c;
    if (DT == TYPE_BF16) asm("max.NaN.bf16x2 %0, %1, %2;" : "=r"(c) : "r"(a), "r"(b));
    else asm("max.NaN.f16x2 %0, %1, %2;" : "=r"(c) : "r"(a), "r"(b));
    return c;
}

struct BoundsArgs {
    Pages pg;
    int block;                  // rows of a block
    const int32_t* seq_lens;
    long long n_new;            // blocks that overlap the last n_new rows
    uint16_t* bounds;           // [n_pages, H_kv, page_size / block, 2, d]
};
constexpr int BOUNDS_THREADS = 128, BOUNDS_WARPS = BOUNDS_THREADS / 32;

// A warp for a block of one head: D / 8 lanes hold a row, the others of the warp further rows.
template <int DT, int D> __global__ void __launch_bounds__(BOUNDS_THREADS) bounds_kernel(const __grid_constant__ BoundsArgs a) {
    constexpr int LANES = D / 8, RPW = 32 / LANES;       // lanes per row, rows per load of the warp
    pdl_wait();
    const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5, b = blockIdx.z, h = blockIdx.y;
    const long long n = keys_seen(a.pg, a.seq_lens[b], 1, 0);
    const long long first = a.n_new < n ? n - a.n_new : 0;
    const long long j = first / a.block + (long long)blockIdx.x * BOUNDS_WARPS + warp;
    if (j >= n / a.block) return;
    const long long row0 = cache_row(a.pg, b, j * a.block);
    if (row0 < 0) return;
    const unsigned char* src = a.pg.k + (row0 + (long long)h * a.pg.page_size) * (D * 2) + lane * 16;
    uint4 lo = make_uint4(0, 0, 0, 0), hi = lo;
    for (int r = 0; r < a.block; r += RPW * 8) {
        uint4 x[8];
#pragma unroll
        for (int i = 0; i < 8; ++i)
            if (r + i * RPW < a.block) x[i] = *reinterpret_cast<const uint4*>(src + (long long)(r + i * RPW) * (D * 2));
#pragma unroll
        for (int i = 0; i < 8; ++i) {
            if (r + i * RPW >= a.block) break;
            if (r + i == 0) {
                lo = hi = x[0];
            } else {
                lo = make_uint4(min2_nan<DT>(lo.x, x[i].x), min2_nan<DT>(lo.y, x[i].y), min2_nan<DT>(lo.z, x[i].z), min2_nan<DT>(lo.w, x[i].w));
                hi = make_uint4(max2_nan<DT>(hi.x, x[i].x), max2_nan<DT>(hi.y, x[i].y), max2_nan<DT>(hi.z, x[i].z), max2_nan<DT>(hi.w, x[i].w));
            }
        }
    }
#pragma unroll
    for (int o = LANES; o < 32; o <<= 1) {
        auto other = [&](uint32_t v) { return __shfl_xor_sync(0xffffffffu, v, o); };
        lo = make_uint4(min2_nan<DT>(lo.x, other(lo.x)), min2_nan<DT>(lo.y, other(lo.y)), min2_nan<DT>(lo.z, other(lo.z)), min2_nan<DT>(lo.w, other(lo.w)));
        hi = make_uint4(max2_nan<DT>(hi.x, other(hi.x)), max2_nan<DT>(hi.y, other(hi.y)), max2_nan<DT>(hi.z, other(hi.z)), max2_nan<DT>(hi.w, other(hi.w)));
    }
    // blocks of a page and head follow one another, as its rows do
    uint16_t* dst = a.bounds + (row0 + (long long)h * a.pg.page_size) / a.block * (2 * D);
    if (lane < LANES) *reinterpret_cast<uint4*>(dst + lane * 8) = lo;
    else if (lane < 2 * LANES) *reinterpret_cast<uint4*>(dst + D + (lane - LANES) * 8) = hi;
}

// ---------------------------------------------------------------------------------------
// score_kernel, pick_kernel
// ---------------------------------------------------------------------------------------
struct SelectArgs {
    Pages pg;
    int block, T, Hq, G, keep, first, last;
    const int32_t* seq_lens;
    const uint16_t* bounds;
    const uint16_t* q;
    long long q_stride;
    float* scores;              // [B, T, H_kv, max_blocks]
    long long max_blocks;
    int32_t* blocks;            // [B, T, H_kv, keep]
};
constexpr int SCORE_THREADS = 128, SCORE_BLOCKS = 32, SCORE_COLS = 4;
constexpr int PICK_THREADS = 512;

// Four threads to a block of keys, a share of the channels each; sums of exact products in 64 bits, so that
// the order of blocks does not hang on the order of additions.
template <int DT, int D> __global__ void __launch_bounds__(SCORE_THREADS) score_kernel(const __grid_constant__ SelectArgs a) {
    __shared__ double s_q[SCORE_COLS][D];
    pdl_wait();
    pdl_start_next();
    const int b = blockIdx.z, h = blockIdx.y, sub = threadIdx.x & 3;
    const long long j = (long long)blockIdx.x * SCORE_BLOCKS + (threadIdx.x >> 2);
    const long long seen = keys_seen(a.pg, a.seq_lens[b], a.T, a.T - 1), N = (seen + a.block - 1) / a.block;
    if (N <= a.keep || (long long)blockIdx.x * SCORE_BLOCKS >= N - a.last) return;
    uint4 lo[D / 32], hi[D / 32];
    bool on = j < N - a.last;
    if (on) {
        const long long row = cache_row(a.pg, b, j * a.block);
        on = row >= 0;
        if (on) {
            const uint16_t* src = a.bounds + (row + (long long)h * a.pg.page_size) / a.block * (2 * D);
#pragma unroll
            for (int i = 0; i < D / 32; ++i) {
                lo[i] = *reinterpret_cast<const uint4*>(src + (4 * i + sub) * 8);
                hi[i] = *reinterpret_cast<const uint4*>(src + D + (4 * i + sub) * 8);
            }
        }
    }
    float best = 0.f;
    for (int c0 = 0; c0 < a.T * a.G; c0 += SCORE_COLS) {
        __syncthreads();
        for (int i = threadIdx.x; i < SCORE_COLS * D; i += SCORE_THREADS) {
            const int c = c0 + i / D;
            double x = 0.0;
            if (c < a.T * a.G) x = to_f32<DT>(a.q[((long long)b * a.T + c / a.G) * a.q_stride + (h * a.G + c % a.G) * D + i % D]);
            s_q[i / D][i % D] = x;
        }
        __syncthreads();
        double acc[SCORE_COLS] = {};
        if (on) {
#pragma unroll
            for (int i = 0; i < D / 32; ++i) {
                float l[8], u[8];
                unpack8<DT>(lo[i], l);
                unpack8<DT>(hi[i], u);
#pragma unroll
                for (int e = 0; e < 8; ++e) {
                    const double dl = l[e], du = u[e];
#pragma unroll
                    for (int c = 0; c < SCORE_COLS; ++c) {
                        const double q = s_q[c][(4 * i + sub) * 8 + e];
                        acc[c] = fma(q, q < 0.0 ? dl : du, acc[c]);
                    }
                }
            }
        }
#pragma unroll
        for (int c = 0; c < SCORE_COLS; ++c) {
            acc[c] += __shfl_xor_sync(0xffffffffu, acc[c], 1);
            acc[c] += __shfl_xor_sync(0xffffffffu, acc[c], 2);
            if (c0 + c >= a.T * a.G) break;
            float s = (float)acc[c];
            if (!on) s = -INFINITY;
            else if (s != s) s = INFINITY;
            const int g = (c0 + c) % a.G;
            best = g == 0 ? s : fmaxf(best, s);
            if (g == a.G - 1 && sub == 0 && j < N - a.last)
                a.scores[(((long long)b * a.T + (c0 + c) / a.G) * a.pg.H_kv + h) * a.max_blocks + j] = best;
        }
    }
}

// Order of scores as unsigned numbers.
__device__ __forceinline__ uint32_t order_of(float s) {
    const uint32_t u = __float_as_uint(s + 0.f);          // (-0 becomes 0)
    return u & 0x80000000u ? ~u : u | 0x80000000u;
}

// One CTA for a token and KV head: the threshold byte by byte, then the numbers above it, ascending.
__global__ void __launch_bounds__(PICK_THREADS) pick_kernel(const __grid_constant__ SelectArgs a) {
    __shared__ int s_hist[256], s_digit, s_above;
    pdl_wait();
    const int h = blockIdx.x, t = blockIdx.y, b = blockIdx.z, tid = threadIdx.x;
    const long long seen = keys_seen(a.pg, a.seq_lens[b], a.T, t);
    const int N = (int)((seen + a.block - 1) / a.block);
    const long long item = ((long long)b * a.T + t) * a.pg.H_kv + h;
    int32_t* out = a.blocks + item * a.keep;
    if (N <= a.keep) {
        for (int i = tid; i < a.keep; i += PICK_THREADS) out[i] = i < N ? i : -1;
        return;
    }
    const int want = a.keep - a.first - a.last, m = N - a.first - a.last;
    for (int i = tid; i < a.first; i += PICK_THREADS) out[i] = i;
    for (int i = tid; i < a.last; i += PICK_THREADS) out[a.keep - a.last + i] = N - a.last + i;
    if (want == 0) return;
    const float* scores = a.scores + item * a.max_blocks + a.first;
    uint32_t limit = 0;                                   // digits of the want-th largest, as far as they are known
    int rest = want;                                      // how many of those that share them are taken
    for (int shift = 24; shift >= 0; shift -= 8) {
        for (int i = tid; i < 256; i += PICK_THREADS) s_hist[i] = 0;
        __syncthreads();
        for (int i = tid; i < m; i += PICK_THREADS) {
            const uint32_t u = order_of(scores[i]);
            if (shift == 24 || u >> (shift + 8) == limit >> (shift + 8)) atomicAdd(&s_hist[(u >> shift) & 255], 1);
        }
        __syncthreads();
        if (tid < 32) {                                   // from the largest digit down, 8 digits to a lane
            int mine = 0;
            for (int k = 0; k < 8; ++k) mine += s_hist[255 - (tid * 8 + k)];
            int sum = mine;
#pragma unroll
            for (int o = 1; o < 32; o <<= 1) {
                const int y = __shfl_up_sync(0xffffffffu, sum, o);
                if (tid >= o) sum += y;
            }
            int above = sum - mine;
            if (above < rest && rest <= sum) {
                int k = 0;
                while (above + s_hist[255 - (tid * 8 + k)] < rest) above += s_hist[255 - (tid * 8 + k++)];
                s_digit = 255 - (tid * 8 + k);
                s_above = above;
            }
        }
        __syncthreads();
        limit |= (uint32_t)s_digit << shift;
        rest -= s_above;
        __syncthreads();
    }
    // taken: above the limit, or equal to it and among the first `rest` of those
    int taken = 0, equal = 0;
    for (int i0 = 0; i0 < m; i0 += PICK_THREADS) {
        const int i = i0 + tid;
        const uint32_t u = i < m ? order_of(scores[i]) : 0;
        const bool eq = i < m && u == limit, gt = i < m && u > limit;
        int total;
        const int before = scan_cta<PICK_THREADS>((int)gt | (int)eq << 16, &total);
        const int e = equal + (before >> 16), at = taken + (before & 65535) + (e < rest ? e : rest);
        if (gt || (eq && e < rest)) out[a.first + at] = a.first + i;
        taken += total & 65535;
        equal += total >> 16;
    }
}

}  // namespace retopk_cache
