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
    int block, shift;           // rows of a block, and as a power of two
    const int32_t* seq_lens;
    long long n_new;            // blocks that overlap the last n_new rows
    uint16_t* bounds;           // [n_pages, H_kv, page_size / block, 2, d]
};
constexpr int BOUNDS_THREADS = 128, BOUNDS_WARPS = BOUNDS_THREADS / 32;

// A warp for a block of one head: D / 8 lanes hold a row, the others of the warp further rows; 8 loads of a lane are under way at
// once.  Bound by memory: 4 sequences of 128K keys, 8 heads of 128 channels, 1.1 GB in 162 us, 6.8 TB/s.
template <int DT, int D> __global__ void __launch_bounds__(BOUNDS_THREADS) bounds_kernel(const __grid_constant__ BoundsArgs a) {
    constexpr int LANES = D / 8, RPW = 32 / LANES;       // lanes per row, rows per load of the warp
    pdl_wait();
    const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5, b = blockIdx.z, h = blockIdx.y;
    const int n = keys_seen(a.pg, a.seq_lens[b], 1, 0), first = a.n_new < n ? n - (int)a.n_new : 0;
    const int j = (first >> a.shift) + (int)blockIdx.x * BOUNDS_WARPS + warp;
    if (j >= n >> a.shift) return;
    const long long row0 = cache_row(a.pg, b, j << a.shift);
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
    uint16_t* dst = a.bounds + ((row0 + (long long)h * a.pg.page_size) >> a.shift) * (2 * D);
    if (lane < LANES) *reinterpret_cast<uint4*>(dst + lane * 8) = lo;
    else if (lane < 2 * LANES) *reinterpret_cast<uint4*>(dst + D + (lane - LANES) * 8) = hi;
}

// ---------------------------------------------------------------------------------------
// score_kernel, pick_kernel
// ---------------------------------------------------------------------------------------
struct SelectArgs {
    Pages pg;
    int block, shift, T, Hq, G, keep, first, last;       // (block: 1 << shift)
    float per_G;                // 1 / G
    const int32_t* seq_lens;
    const uint16_t* bounds;
    const uint16_t* q;
    long long q_stride;
    float2* scores;             // [B, T, H_kv, max_blocks]: a score in fp32 and how far it may be off
    long long max_blocks;
    int32_t* blocks;            // [B, T, H_kv, keep]
    bool scored;                // score_kernel runs before
};
constexpr int SCORE_THREADS = 128, SCORE_WARPS = SCORE_THREADS / 32, SCORE_ROWS = 16, SCORE_COLS = 8;
constexpr int PICK_THREADS = 512, PICK_WARPS = PICK_THREADS / 32, PICK_DEEP = 8, PICK_LIST = 512;

__device__ __forceinline__ uint32_t word(const uint4& x, int i) { return i == 0 ? x.x : (i == 1 ? x.y : (i == 2 ? x.z : x.w)); }

// Scores in fp32, and a bound on their errors; pick_kernel works out exactly those that the bound leaves open.
// Bound by reading the bounds, once for all queries of a KV head: at 4 x 8 x 2048 blocks of 128 channels and 4 queries 34 MB and 8 us,
// with three waits for memory one after the other (length, page, bounds).  All of them in 64 bits were 22 us.
//
// max(q lo, q hi) = q+ hi + q- lo with the positive and the negative part of q.  A warp has 16 blocks as the rows
// of A, up to 8 queries as the columns of B.  The channels that a lane loads at once (8 of 32) are
// those that it holds in A and in B of two products: sums do not care for their order.
// Error: products of 16-bit numbers are exact in fp32.  Two products of depth 16 go into a sum, each of whose 34 additions
// cuts off at most 2^-23 of what was summed so far, below the sum's share of size = sum |q| times the largest |bound| of the
// block; at most 8 such sums are added with 2^-24 of size each: 34 * 2^-23 + 8 * 2^-24 < 2^-17 of size.
template <int DT, int D> __global__ void __launch_bounds__(SCORE_THREADS, 7) score_kernel(const __grid_constant__ SelectArgs a) {
    constexpr int STEPS = D / 32;
    __shared__ float s_score[SCORE_WARPS][SCORE_COLS][SCORE_ROWS], s_size[SCORE_WARPS][SCORE_COLS];
    pdl_wait();
    pdl_start_next();
    const int b = blockIdx.z, h = blockIdx.y, lane = threadIdx.x & 31, warp = threadIdx.x >> 5, g = lane >> 2, part = lane & 3;
    const int j0 = (blockIdx.x * SCORE_WARPS + warp) * SCORE_ROWS;
    const int seen = (int)keys_seen(a.pg, a.seq_lens[b], a.T, a.T - 1), end = ((seen + a.block - 1) >> a.shift) - a.last;
    if (end + a.last <= a.keep || j0 >= end) return;
    constexpr int DEEP = 2;                              // groups of 32 channels that are loaded at once
    const uint16_t* src[2];
#pragma unroll
    for (int y = 0; y < 2; ++y) {
        const int j = j0 + g + 8 * y;
        const long long r = j < end ? cache_row(a.pg, b, j << a.shift) : -1;
        src[y] = r < 0 ? nullptr : a.bounds + ((r + (long long)h * a.pg.page_size) >> a.shift) * (2 * D) + part * 8;
    }
    uint32_t largest2[2] = {0, 0};                       // of the bounds' magnitudes
    float largest[2] = {0.f, 0.f};
    const int cols = a.T * a.G;
    float best = 0.f, size = 0.f;
    for (int c0 = 0; c0 < cols; c0 += SCORE_COLS) {
        float c[4] = {0.f, 0.f, 0.f, 0.f}, sum = 0.f;
        const int col = c0 + g, t = small_div(col, a.per_G);
        const uint16_t* q = a.q + ((long long)b * a.T + t) * a.q_stride + (h * a.G + col - t * a.G) * D + part * 8;
#pragma unroll
        for (int i0 = 0; i0 < STEPS; i0 += DEEP) {
            uint4 lo[2][DEEP], hi[2][DEEP], x[DEEP];
#pragma unroll
            for (int i = 0; i < DEEP; ++i) {
#pragma unroll
                for (int y = 0; y < 2; ++y) {
                    lo[y][i] = hi[y][i] = make_uint4(0, 0, 0, 0);
                    if (src[y]) {
                        lo[y][i] = *reinterpret_cast<const uint4*>(src[y] + (i0 + i) * 32);
                        hi[y][i] = *reinterpret_cast<const uint4*>(src[y] + D + (i0 + i) * 32);
                    }
                }
                x[i] = col < cols ? *reinterpret_cast<const uint4*>(q + (i0 + i) * 32) : make_uint4(0, 0, 0, 0);
            }
#pragma unroll
            for (int i = 0; i < DEEP; ++i) {
                uint32_t up[4], down[4];
#pragma unroll
                for (int w = 0; w < 4; ++w) {
                    up[w] = max2_nan<DT>(word(x[i], w), 0u);
                    down[w] = min2_nan<DT>(word(x[i], w), 0u);
                    const float2 f = unpack2<DT>(word(x[i], w));
                    sum += fabsf(f.x) + fabsf(f.y);
                    if (c0 == 0)
#pragma unroll
                        for (int y = 0; y < 2; ++y)
                            largest2[y] = __vmaxu2(__vmaxu2(largest2[y], word(lo[y][i], w) & 0x7fff7fffu), word(hi[y][i], w) & 0x7fff7fffu);
                }
                float u[4] = {0.f, 0.f, 0.f, 0.f}, v[4] = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
                for (int w = 0; w < 4; w += 2) {
                    mma16816<DT>(u, word(hi[0][i], w), word(hi[1][i], w), word(hi[0][i], w + 1), word(hi[1][i], w + 1), up[w], up[w + 1]);
                    mma16816<DT>(v, word(lo[0][i], w), word(lo[1][i], w), word(lo[0][i], w + 1), word(lo[1][i], w + 1), down[w], down[w + 1]);
                }
#pragma unroll
                for (int k = 0; k < 4; ++k) c[k] += u[k] + v[k];
            }
        }
        if (c0 == 0)
#pragma unroll
            for (int y = 0; y < 2; ++y) {
                uint32_t m = largest2[y];
                m = __vmaxu2(m, __shfl_xor_sync(0xffffffffu, m, 1));
                m = __vmaxu2(m, __shfl_xor_sync(0xffffffffu, m, 2));
                const float2 f = unpack2<DT>(m);
                largest[y] = f.x != f.x || f.y != f.y ? INFINITY : fmaxf(f.x, f.y);
            }
        sum += __shfl_xor_sync(0xffffffffu, sum, 1);
        sum += __shfl_xor_sync(0xffffffffu, sum, 2);
        if (part == 0) s_size[warp][g] = sum;
#pragma unroll
        for (int y = 0; y < 2; ++y) {
            s_score[warp][2 * part][g + 8 * y] = c[2 * y];
            s_score[warp][2 * part + 1][g + 8 * y] = c[2 * y + 1];
        }
        __syncwarp();
        // lane x < 16: block x of the warp
        const int from = (lane & 7) * 4;
        const float most0 = __shfl_sync(0xffffffffu, largest[0], from), most1 = __shfl_sync(0xffffffffu, largest[1], from);
        const int none0 = __shfl_sync(0xffffffffu, (int)(src[0] == nullptr), from), none1 = __shfl_sync(0xffffffffu, (int)(src[1] == nullptr), from);
        if (lane < SCORE_ROWS && j0 + lane < end) {
            const float most = lane & 8 ? most1 : most0;
            const bool out = (lane & 8 ? none1 : none0) != 0;
            for (int k = 0; k < SCORE_COLS && c0 + k < cols; ++k) {
                const int t = small_div(c0 + k, a.per_G), head = c0 + k - t * a.G;
                const float s = s_score[warp][k][lane], z = s_size[warp][k];
                best = head == 0 ? s : fmaxf(best, s);
                size = head == 0 || z != z ? z : (size != size ? size : fmaxf(size, z));          // (NaN stays)
                if (head == a.G - 1) {
                    float off = size * most * 0x1p-17f + 1e-35f;
                    if (!(off < 1e37f) || !(fabsf(best) < 1e37f)) off = INFINITY;
                    a.scores[(((long long)b * a.T + t) * a.pg.H_kv + h) * a.max_blocks + j0 + lane] =
                        out ? make_float2(-INFINITY, 0.f) : (off == INFINITY ? make_float2(0.f, INFINITY) : make_float2(best, off));
                }
            }
        }
        __syncwarp();
    }
}

// Order of scores as unsigned numbers, from 1 on.
__device__ __forceinline__ uint32_t order_of(float s) {
    const uint32_t u = __float_as_uint(s + 0.f);          // (-0 becomes 0)
    return u & 0x80000000u ? ~u : u | 0x80000000u;
}

// The want-th largest of the CTA's numbers: `limit`, and how many of those equal to it are among the want.  Each thread calls
// f for its numbers.  Digits of what the numbers have above the least of them, 8 bits at a time; without EXACT over when
// a digit's numbers are all taken (then the limit is at most the want-th largest, and above all that are smaller).
template <bool EXACT, class Each> __device__ __forceinline__ void find_limit(Each each, int want, uint32_t* limit, int* rest_out) {
    __shared__ int s_hist[256], s_digit, s_above, s_inside;
    __shared__ uint32_t s_low[PICK_WARPS], s_high[PICK_WARPS];
    const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5;
    uint32_t low = ~0u, high = 0;
    each([&](uint32_t u) {
        low = u < low ? u : low;
        high = u > high ? u : high;
    });
    low = __reduce_min_sync(0xffffffffu, low);
    high = __reduce_max_sync(0xffffffffu, high);
    __syncthreads();
    if (lane == 0) { s_low[warp] = low; s_high[warp] = high; }
    __syncthreads();
    low = __reduce_min_sync(0xffffffffu, s_low[lane % PICK_WARPS]);
    high = __reduce_max_sync(0xffffffffu, s_high[lane % PICK_WARPS]);
    int bits = high > low ? 32 - __clz(high - low) : 0;
    uint32_t prefix = 0;                                  // digits known so far, of u - low
    int rest = want, shift = bits;
    while (shift > 0) {
        const int width = shift < 8 ? shift : 8, next = shift - width;
        for (int i = tid; i < 256; i += PICK_THREADS) s_hist[i] = 0;
        __syncthreads();
        each([&](uint32_t u) {
            u -= low;
            if (shift == bits || u >> shift == prefix) atomicAdd(&s_hist[(u >> next) & ((1 << width) - 1)], 1);
        });
        __syncthreads();
        if (warp == 0) {                                  // from the largest digit down, 8 digits to a lane
            int digits[8], mine = 0;
#pragma unroll
            for (int k = 0; k < 8; ++k) mine += digits[k] = s_hist[255 - (lane * 8 + k)];
            int sum = mine;
#pragma unroll
            for (int o = 1; o < 32; o <<= 1) {
                const int y = __shfl_up_sync(0xffffffffu, sum, o);
                if (lane >= o) sum += y;
            }
            int above = sum - mine;
            if (above < rest && rest <= sum) {
                bool found = false;
#pragma unroll
                for (int k = 0; k < 8; ++k) {
                    if (!found && above + digits[k] >= rest) {
                        found = true;
                        s_digit = 255 - (lane * 8 + k);
                        s_above = above;
                        s_inside = digits[k];
                    }
                    above += digits[k];
                }
            }
        }
        __syncthreads();
        prefix = prefix << width | (uint32_t)s_digit;
        rest -= s_above;
        shift = next;
        if (!EXACT && s_inside == rest) break;                      // all that share the digits so far: the limit is the least of them
        __syncthreads();
    }
    *limit = low + (prefix << shift);
    // cut short: numbers of the last digit may lie above the limit; they are taken as larger ones, none as equal
    *rest_out = shift > 0 ? 0x7fffffff : rest;
}

// The score of block j for a head, in 64 bits and rounded once to fp32, by a warp: D / 32 channels to a lane.
template <int DT, int D> __device__ __forceinline__ float exact_score(const SelectArgs& a, int b, int t, int h, int g, int j) {
    constexpr int WORDS = D / 64;
    const int lane = threadIdx.x & 31;
    const long long r = cache_row(a.pg, b, j << a.shift);
    if (r < 0) return -INFINITY;
    const uint32_t* src = reinterpret_cast<const uint32_t*>(a.bounds + ((r + (long long)h * a.pg.page_size) >> a.shift) * (2 * D)) + lane;
    const uint32_t* q = reinterpret_cast<const uint32_t*>(a.q + ((long long)b * a.T + t) * a.q_stride + ((long long)h * a.G + g) * D) + lane;
    double sum = 0.0;
#pragma unroll
    for (int w = 0; w < WORDS; ++w) {
        const float2 x = unpack2<DT>(q[w * 32]), lo = unpack2<DT>(src[w * 32]), hi = unpack2<DT>(src[D / 2 + w * 32]);
#pragma unroll
        for (int e = 0; e < 2; ++e) {
            const double y = e ? x.y : x.x, p = y * (e ? lo.y : lo.x), z = y * (e ? hi.y : hi.x);
            sum += p != p || z != z ? p + z : (p > z ? p : z);
        }
    }
#pragma unroll 1
    for (int o = 16; o > 0; o >>= 1) sum += __shfl_xor_sync(0xffffffffu, sum, o);
    const float f = (float)sum;
    return f != f ? INFINITY : f;
}

// Any number of blocks to choose from, any number of equal scores.  A block whose upper end
// is below the want-th largest lower end is out, and one whose lower end is above the (want + 1)-th largest
// upper end is in; those between are scored exactly.
template <int DT, int D> __device__ __noinline__ void pick_any(const SelectArgs& a, float2* at, int b, int t, int h, int m, int want, int32_t* out) {
    const int tid = threadIdx.x, lane = tid & 31;
    uint32_t lowest, limit;
    int rest;
    find_limit<false>([&](auto f) {
        for (int i = tid; i < m; i += PICK_THREADS) f(order_of(__fsub_rd(at[i].x, at[i].y)));
    }, want, &lowest, &rest);
    int left = 0, all_left;
    for (int i = tid; i < m; i += PICK_THREADS) left += order_of(__fadd_ru(at[i].x, at[i].y)) >= lowest;
    scan_cta<PICK_THREADS>(left, &all_left);
    uint32_t highest = 0;                                 // (as many left as wanted: all of them are in)
    if (all_left > want)
        find_limit<true>([&](auto f) {
            for (int i = tid; i < m; i += PICK_THREADS) {
                const uint32_t u = order_of(__fadd_ru(at[i].x, at[i].y));
                if (u >= lowest) f(u);
            }
        }, want + 1, &highest, &rest);

    // From here on x holds a number's bits: 0 for a block that is out, the largest for one that is in, else the order
    // of its exact score.
#pragma unroll 1
    for (int i0 = 0; i0 < m; i0 += PICK_THREADS) {
        const int i = i0 + tid;
        const float2 s = i < m ? at[i] : make_float2(0.f, 0.f);
        const bool some = i < m && order_of(__fadd_ru(s.x, s.y)) >= lowest, in = some && order_of(__fsub_rd(s.x, s.y)) > highest;
        uint32_t mine = in ? ~0u : 0u;
        for (uint32_t todo = __ballot_sync(0xffffffffu, some && !in); todo; todo &= todo - 1) {
            const int x = __ffs(todo) - 1, j = a.first + (i - lane) + x;
            float score = -INFINITY;
#pragma unroll 1
            for (int g = 0; g < a.G; ++g) score = fmaxf(score, exact_score<DT, D>(a, b, t, h, g, j));
            if (lane == x) mine = order_of(score);
        }
        if (i < m) at[i].x = __uint_as_float(mine);
    }
    __syncthreads();
    limit = 1;
    rest = 0x7fffffff;
    if (all_left > want)
        find_limit<false>([&](auto f) {
            for (int i = tid; i < m; i += PICK_THREADS) {
                const uint32_t u = __float_as_uint(at[i].x);
                if (u) f(u);
            }
        }, want, &limit, &rest);
    // taken: above the limit, or equal to it and among the first `rest` of those
    int taken = 0, equal = 0;
#pragma unroll 1
    for (int i0 = 0; i0 < m; i0 += PICK_THREADS) {
        const int i = i0 + tid;
        const uint32_t u = i < m ? __float_as_uint(at[i].x) : 0;
        const bool eq = i < m && u == limit, gt = i < m && u > limit;
        int total;
        const int before = scan_cta<PICK_THREADS>((int)gt | (int)eq << 16, &total);
        const int e = equal + (before >> 16), place = taken + (before & 65535) + (e < rest ? e : rest);
        if (gt || (eq && e < rest)) out[a.first + place] = a.first + i;
        taken += total & 65535;
        equal += total >> 16;
    }
}

// One CTA for a token and KV head; `want` blocks are to be chosen, whose scores are known as intervals.  A bin of the want-th
// largest lower end gives a limit that few blocks reach with their upper end; among those, each is compared with
// all others, and those that stay open are scored exactly.  Bound by waiting: 4 us for 61 of 2045, of 61 to 63 candidates and up to 2 open
// ones.  (Ranks among all candidates, one after the other, were 3.5 us more, and 7 at 125 of 911.)
template <int DT, int D> __global__ void __launch_bounds__(PICK_THREADS, 1) pick_kernel(const __grid_constant__ SelectArgs a) {
    constexpr int BITS = 10, BINS = 1 << BITS, DEEP = PICK_DEEP;
    __shared__ int s_bin[BINS], s_count, s_found[3];
    __shared__ __align__(16) uint32_t s_cand[PICK_LIST], s_lower[PICK_LIST], s_upper[PICK_LIST], s_key[PICK_LIST];
    __shared__ uint32_t s_low[PICK_WARPS], s_high[PICK_WARPS];
    __shared__ int s_opened;
    int* const s_open = s_bin;                           // (the bins are done with by then)
    const int h = blockIdx.x, t = blockIdx.y, b = blockIdx.z, tid = threadIdx.x, lane = tid & 31, warp = tid >> 5;
    if (!a.scored) pdl_wait();                           // (else score_kernel has waited for all but its own scores)
    const int seen = keys_seen(a.pg, a.seq_lens[b], a.T, t), N = (seen + a.block - 1) >> a.shift;
    const long long item = ((long long)b * a.T + t) * a.pg.H_kv + h;
    int32_t* out = a.blocks + item * a.keep;
    if (N <= a.keep) {
#pragma unroll 1
        for (int i = tid; i < a.keep; i += PICK_THREADS) out[i] = i < N ? i : -1;
        if (a.scored) pdl_wait();                        // (no CTA ends before score_kernel has: what follows may rely on it)
        return;
    }
    const int want = a.keep - a.first - a.last, m = N - a.first - a.last;
#pragma unroll 1
    for (int i = tid; i < a.first; i += PICK_THREADS) out[i] = i;
#pragma unroll 1
    for (int i = tid; i < a.last; i += PICK_THREADS) out[a.keep - a.last + i] = N - a.last + i;
#pragma unroll
    for (int i = 0; i < BINS / PICK_THREADS; ++i) s_bin[i * PICK_THREADS + tid] = 0;
    if (tid == 0) s_count = s_opened = 0;
    if (a.scored) pdl_wait();
    pdl_start_next();
    if (want == 0) return;
    float2* const at = a.scores + item * a.max_blocks + a.first;
    auto lower = [](float2 s) { return order_of(__fsub_rd(s.x, s.y)); };
    auto upper = [](float2 s) { return order_of(__fadd_ru(s.x, s.y)); };
    float2 x[DEEP];                                      // the first scores of this thread; others are read again where they are wanted
#pragma unroll
    for (int k = 0; k < DEEP; ++k)
        if (k * PICK_THREADS + tid < m) x[k] = at[k * PICK_THREADS + tid];
    auto each = [&](auto f) {
#pragma unroll
        for (int k = 0; k < DEEP; ++k)
            if (k * PICK_THREADS + tid < m) f(k * PICK_THREADS + tid, x[k]);
#pragma unroll 1
        for (int i = DEEP * PICK_THREADS + tid; i < m; i += PICK_THREADS) f(i, at[i]);
    };
    {
        uint32_t low = ~0u, high = 0;
        each([&](int, float2 v) {
            low = min(low, lower(v));
            high = max(high, lower(v));
        });
        low = __reduce_min_sync(0xffffffffu, low);
        high = __reduce_max_sync(0xffffffffu, high);
        if (lane == 0) { s_low[warp] = low; s_high[warp] = high; }
    }
    __syncthreads();
    const uint32_t low = __reduce_min_sync(0xffffffffu, s_low[lane % PICK_WARPS]), high = __reduce_max_sync(0xffffffffu, s_high[lane % PICK_WARPS]);
    // bins, BITS of what the lower ends have above the least of them at a time, until one holds few
    const int bits = high > low ? 32 - __clz(high - low) : 0;
    uint32_t prefix = 0;
    int rest = want, shift = bits;
#pragma unroll 1
    while (shift > 0) {
        const int width = shift < BITS ? shift : BITS, next = shift - width;
        each([&](int, float2 v) {
            const uint32_t u = lower(v) - low;
            if (shift == bits || u >> shift == prefix) atomicAdd(&s_bin[(u >> next) & (BINS - 1)], 1);
        });
        __syncthreads();
        constexpr int PER = BINS / PICK_THREADS;          // bins of a thread, from the largest down
        int n[PER], mine = 0, total;
#pragma unroll
        for (int k = 0; k < PER; ++k) {
            mine += n[k] = s_bin[BINS - 1 - (tid * PER + k)];
            s_bin[BINS - 1 - (tid * PER + k)] = 0;
        }
        int above = scan_cta<PICK_THREADS>(mine, &total);
#pragma unroll
        for (int k = 0; k < PER; ++k) {
            if (above < rest && rest <= above + n[k]) {
                s_found[0] = BINS - 1 - (tid * PER + k);
                s_found[1] = above;
                s_found[2] = n[k];
            }
            above += n[k];
        }
        __syncthreads();
        prefix = prefix << width | (uint32_t)s_found[0];
        rest -= s_found[1];
        shift = next;
        if (s_found[2] <= 32) break;
        __syncthreads();
    }
    const uint32_t limit = low + (prefix << shift);
    // the blocks that reach the limit, in any order
    each([&](int i, float2 v) {
        const uint32_t u = upper(v);
        if (u < limit) return;
        const int c = atomicAdd(&s_count, 1);
        if (c >= PICK_LIST) return;
        s_cand[c] = i;
        s_lower[c] = lower(v);
        s_upper[c] = u;
    });
    __syncthreads();
    const int C = s_count;
    if (C > PICK_LIST) {
        pick_any<DT, D>(a, at, b, t, h, m, want, out);
        return;
    }
    // 1 to 4 threads to a candidate, who go through the others four at a time (filled up with ones that count for nothing)
    const int C4 = (C + 3) / 4, fan = C <= PICK_THREADS / 4 ? 2 : (C <= PICK_THREADS / 2 ? 1 : 0), mine = tid >> fan, share = tid & ((1 << fan) - 1);
    const bool on = mine < C;
    auto count = [&](const uint32_t* list, auto f) {
        int n = 0;
        if (on)
#pragma unroll 4
            for (int k = share; k < C4; k += 1 << fan) {
                const uint4 v = reinterpret_cast<const uint4*>(list)[k];
                n += (int)f(v.x) + (int)f(v.y) + (int)f(v.z) + (int)f(v.w);
            }
        if (fan > 0) n += __shfl_xor_sync(0xffffffffu, n, 1);
        if (fan > 1) n += __shfl_xor_sync(0xffffffffu, n, 2);
        return n;
    };
    if (tid < 4 * C4 - C) {
        s_lower[C + tid] = s_upper[C + tid] = 0;
        s_cand[C + tid] = ~0u;
    }
    __syncthreads();
    const uint32_t me = on ? s_cand[mine] : ~0u;
    bool in = on;
    if (C > want) {
        const uint32_t lo = on ? s_lower[mine] : 0, hi = on ? s_upper[mine] : 0;
        const int better = count(s_lower, [&](uint32_t u) { return u > hi; }), rivals = count(s_upper, [&](uint32_t u) { return u >= lo; });
        in = on && rivals <= want;
        const bool open = on && better < want && rivals > want;
        if (open && share == 0) s_open[atomicAdd(&s_opened, 1)] = mine;
        const int free = want - __syncthreads_count(in && share == 0), opened = s_opened;
        // those that stay open: the largest of the heads' exact scores
        if (tid < opened) s_key[s_open[tid]] = 0;
        __syncthreads();
#pragma unroll 1
        for (int y = warp; y < opened * a.G; y += PICK_WARPS) {
            const int k = small_div(y, a.per_G), c = s_open[k];
            const float score = exact_score<DT, D>(a, b, t, h, y - k * a.G, a.first + (int)s_cand[c]);
            if (lane == 0) atomicMax(&s_key[c], order_of(score));
        }
        __syncthreads();
        if (open) {
            const uint32_t key = s_key[mine];
            int rank = 0;
#pragma unroll 1
            for (int k = 0; k < opened; ++k) {
                const int c = s_open[k];
                rank += s_key[c] > key || (s_key[c] == key && s_cand[c] < me);
            }
            in = rank < free;
        }
        __syncthreads();
        if (on && !in && share == 0) s_cand[mine] = ~0u;
        __syncthreads();
    }
    const int place = count(s_cand, [&](uint32_t u) { return u < me; });
    if (in && share == 0) out[a.first + place] = a.first + (int)me;
}

}  // namespace retopk_cache
