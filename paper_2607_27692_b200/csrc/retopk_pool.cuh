// Device code that manages the pages of a cache (sm_100a): which are in use, and moving their rows.
//
//   reserve_kernel       gives sequences the pages that their new rows need
//   fork_kernel          lets a sequence continue another one's pages
//   free_kernel          gives the pages of sequences back
//   compact_kernel       decides which pages move to the front, renumber_kernel follows in the block table
//   copy_pages_kernel    moves rows of pages
#pragma once
#include "retopk_cache.cuh"

namespace retopk_cache {

struct PoolArgs {
    int32_t* refs;              // entries of block tables that hold a page; 0 and below: free
    int32_t* scratch;           // [0] pages that were missing, [1] CTAs that are done, [2] pages in use, then a list of n_pages
    long long n_pages;
    int page_size;
    int32_t* table;
    long long max_pages, capacity;
    int B, n;
    int32_t* lens;              // fork, free: the lengths, written; reserve, compact: read
    const int32_t* other;       // reserve: the new lengths; fork: parents; free: rows or null
    const int32_t* children;
    int32_t *src, *dst, *rows;
    long long pairs;            // compact: size of src and dst
};
constexpr int POOL_SHORT = 0, POOL_TICKET = 1, POOL_USED = 2, POOL_LIST = 4;
constexpr int POOL_THREADS = 1024, POOL_WARPS = POOL_THREADS / 32;
constexpr int FORK_THREADS = 256;

__device__ __forceinline__ long long pages_held(long long len, int page_size) { return len <= 0 ? 0 : (len + page_size - 1) / page_size; }

// The lowest `want` free pages, ascending, into `list`; how many there are.  One CTA: a warp has 512 pages at a time, 32 of
// them side by side, so that a CTA of 256 threads looks through 4096 with one wait for memory and one barrier.
template <int THREADS> __device__ int lowest_free(const PoolArgs& a, int32_t* list, int want) {
    constexpr int PER = 16, WARPS = THREADS / 32;
    __shared__ int s_found[2][WARPS];
    const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
    int found = 0, turn = 0;
#pragma unroll 1
    for (long long at = 0; at < a.n_pages && found < want; at += (long long)THREADS * PER, turn ^= 1) {
        const long long p0 = at + warp * (32 * PER) + lane;
        int refs[PER], mine = 0;
#pragma unroll
        for (int k = 0; k < PER; ++k) refs[k] = p0 + k * 32 < a.n_pages ? __ldcg(a.refs + p0 + k * 32) : 1;
#pragma unroll
        for (int k = 0; k < PER; ++k) mine += __popc(__ballot_sync(0xffffffffu, refs[k] <= 0));
        if (lane == 0) s_found[turn][warp] = mine;
        __syncthreads();
        const int n = lane < WARPS ? s_found[turn][lane] : 0;
        int r = found + __reduce_add_sync(0xffffffffu, lane < warp ? n : 0);
        found += __reduce_add_sync(0xffffffffu, n);
#pragma unroll
        for (int k = 0; k < PER; ++k) {
            const uint32_t who = __ballot_sync(0xffffffffu, refs[k] <= 0);
            const int place = r + __popc(who & ((1u << lane) - 1));
            if (refs[k] <= 0 && place < want) list[place] = (int)(p0 + k * 32);
            r += __popc(who);
        }
    }
    __syncthreads();
    return found < want ? found : want;
}

// Pages that were missing, by one thread: the count stays at the largest number.
__device__ __forceinline__ void count_missing(const PoolArgs& a, long long n) {
    const int have = __ldcg(a.scratch + POOL_SHORT), room = have > 0 ? 0x7fffffff - have : 0x7fffffff;
    if (n > 0) atomicAdd(a.scratch + POOL_SHORT, n < room ? (int)n : room);
}

// One CTA: how many pages each sequence needs, the lowest free ones, and their places in the table.  A
// sequence gets all of its pages or none: then its new entries are -1, all of them, however few pages there are.  Before that
// sequences that shrink give back what they no longer hold, so that a page may go from one to another in a call.
// Bound by waiting: 6.5 us for a page each of 64 sequences out of 8192, 3.1 with nothing to do; where nearly all pages are in use the
// walk over their counts shows, 16 us of 65 536 and 115 of 2^20.
__global__ void __launch_bounds__(POOL_THREADS) reserve_kernel(const __grid_constant__ PoolArgs a) {
    __shared__ int s_base[POOL_THREADS], s_need[POOL_THREADS];
    pdl_wait();
    const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
    int32_t* list = a.scratch + POOL_LIST;
    // A sequence's new places, and the pages that it lacks for them: as a number to add up it is cut at n_pages + 1 (more
    // than there are); negative: more than its row has places for.  `gone`: the places from `first` on that it no longer holds.
    struct Need { long long first, places, lack, gone; int n; };
    auto need_of = [&](int b) {
        const long long had = pages_held(a.lens[b], a.page_size), get = pages_held(a.other[b], a.page_size);
        const long long from = had < a.max_pages ? had : a.max_pages, to = get < a.max_pages ? get : a.max_pages;
        Need x = {from, 0, 0, 0, 0};
        if (get <= had) {
            x.first = to;
            x.gone = from - to;
            return x;
        }
        x.places = to - from;
        x.lack = get - had;
        x.n = (int)(x.lack <= a.n_pages ? x.lack : a.n_pages + 1);
        if (get > a.max_pages) x.n = -x.n;
        return x;
    };
    long long want = 0;
    bool less = false;
    for (int b0 = 0; b0 < a.B; b0 += POOL_THREADS) {
        const int b = b0 + threadIdx.x;
        int total;
        Need x = {0, 0, 0, 0, 0};
        if (b < a.B) x = need_of(b);
        less |= x.gone > 0;
        scan_cta<POOL_THREADS>(x.n < 0 ? 0 : x.n, &total);
        want += total;
    }
    if (__syncthreads_or(less)) {
        for (int b = warp; b < a.B; b += POOL_WARPS) {
            const Need x = need_of(b);
            int32_t* row = a.table + (long long)b * a.max_pages + x.first;
            for (long long s = lane; s < x.gone; s += 32) {
                const int p = row[s];
                if (p >= 0 && p < a.n_pages) atomicSub(a.refs + p, 1);
                row[s] = -1;
            }
        }
        __syncthreads();
    }
    const int found = lowest_free<POOL_THREADS>(a, list, (int)(want < a.n_pages ? want : a.n_pages));
    __shared__ unsigned long long s_missing;
    if (threadIdx.x == 0) s_missing = 0;
    long long base = 0;
    for (int b0 = 0; b0 < a.B; b0 += POOL_THREADS) {
        const int b = b0 + threadIdx.x;
        int total;
        Need x = {0, 0, 0, 0, 0};
        if (b < a.B) x = need_of(b);
        const int at = scan_cta<POOL_THREADS>(x.n < 0 ? 0 : x.n, &total);
        const bool ok = x.n >= 0 && base + at + x.n <= found;
        if (!ok && x.lack > 0) atomicAdd(&s_missing, (unsigned long long)x.lack);
        s_base[threadIdx.x] = ok ? (int)(base + at) : -1;
        s_need[threadIdx.x] = x.n;
        __syncthreads();
        const int here = a.B - b0 < POOL_THREADS ? a.B - b0 : POOL_THREADS;
        for (int i = warp; i < here; i += POOL_WARPS) {
            if (s_need[i] == 0) continue;
            const Need x = need_of(b0 + i);
            int32_t* row = a.table + (long long)(b0 + i) * a.max_pages + x.first;
            for (long long s = lane; s < x.places; s += 32) {
                const int p = s_base[i] < 0 ? -1 : list[s_base[i] + s];
                row[s] = p;
                if (p >= 0) a.refs[p] = 1;
            }
        }
        base += total;
        __syncthreads();
    }
    if (threadIdx.x == 0) count_missing(a, (long long)s_missing);
}

// Bound by waiting, about ten times for memory one after the other: 4.6 us for 3 forks, 8 for 64 of up to 2048 pages.
// One CTA for a fork copies the table row and counts the full pages, one more finds free pages meanwhile (full pages
// are in use, so that the counts of free ones stay as they are); the CTA that is done last hands them out
// for the partial pages, in the order of the forks.
__global__ void __launch_bounds__(FORK_THREADS) fork_kernel(const __grid_constant__ PoolArgs a) {
    constexpr int DEEP = 8;
    __shared__ int s_last;
    pdl_wait();
    const int tid = threadIdx.x, i = blockIdx.x;
    int32_t* list = a.scratch + POOL_LIST;
    if (i == a.n) {
        const int found = lowest_free<FORK_THREADS>(a, list, a.n < a.n_pages ? a.n : (int)a.n_pages);
        if (tid == 0) a.scratch[POOL_USED] = found;
    } else {
        const int c = a.children[i], p = a.other[i];
        // what holds for a fork does not depend on the others' progress: no child is anyone's parent, and of
        // several forks to one child the first counts
        bool ok = c >= 0 && c < a.B && p >= 0 && p < a.B;
        bool clash = false;
        for (int j = tid; j < a.n; j += FORK_THREADS) {
            const int x = a.children[j];
            clash |= (x == c && j < i) || x == p;
        }
        ok = !__syncthreads_or(clash) && ok;
        const int len = ok ? a.lens[p] : 0;
        ok = ok && len > 0 && len <= a.capacity && a.lens[c] <= 0;
        const int full = ok ? len / a.page_size : 0, rest = ok ? len % a.page_size : 0;
        const int32_t* from = a.table + (long long)p * a.max_pages;
        int32_t* to = a.table + (long long)c * a.max_pages;
        for (int s0 = tid; s0 < full; s0 += FORK_THREADS * DEEP) {
            int page[DEEP];
#pragma unroll
            for (int k = 0; k < DEEP; ++k) page[k] = s0 + k * FORK_THREADS < full ? from[s0 + k * FORK_THREADS] : -1;
#pragma unroll
            for (int k = 0; k < DEEP; ++k) {
                if (s0 + k * FORK_THREADS < full) to[s0 + k * FORK_THREADS] = page[k];
                if (page[k] >= 0 && page[k] < a.n_pages) atomicAdd(a.refs + page[k], 1);
            }
        }
        if (tid == 0) {
            a.src[i] = rest ? from[full] : -1;
            a.dst[i] = !ok ? -3 : (rest ? -2 : -1);          // -2: waits for a page, -3: not made
            a.rows[i] = rest;
        }
    }
    __threadfence();
    __syncthreads();
    if (tid == 0) s_last = atomicAdd(a.scratch + POOL_TICKET, 1) == (int)gridDim.x - 1;
    __syncthreads();
    if (!s_last) return;
    __threadfence();
    if (tid == 0) a.scratch[POOL_TICKET] = 0;

    const int found = __ldcg(a.scratch + POOL_USED);
    int base = 0;
    for (int i0 = 0; i0 < a.n; i0 += FORK_THREADS) {
        const int k = i0 + tid, state = k < a.n ? __ldcg(a.dst + k) : -3;
        int total;
        const int at = base + scan_cta<FORK_THREADS>(state == -2, &total);
        base += total;
        if (k >= a.n) continue;
        if (state == -3) {
            a.dst[k] = -1;
            continue;
        }
        const int child = a.children[k], n = a.lens[a.other[k]], whole = n / a.page_size;
        int32_t* row = a.table + (long long)child * a.max_pages;
        if (state == -1 || at < found) {
            if (state == -2) {
                const int page = __ldcg(list + at);
                row[whole] = page;
                a.refs[page] = 1;
                a.dst[k] = page;
            }
            a.lens[child] = n;
        } else {                                          // no page left: the fork is not made
            for (int s = 0; s < whole; ++s) {
                const int page = __ldcg(row + s);
                if (page >= 0 && page < a.n_pages) atomicSub(a.refs + page, 1);
            }
            a.src[k] = a.dst[k] = -1;
            a.rows[k] = 0;
        }
    }
    if (tid == 0) count_missing(a, base - found);        // (each fork that found no page lacks one)
}

// One CTA for a sequence.  Whoever takes the length takes the pages: a row that is named twice is freed once.
__global__ void __launch_bounds__(FORK_THREADS) free_kernel(const __grid_constant__ PoolArgs a) {
    __shared__ int s_len;
    pdl_wait();
    const int b = a.other ? a.other[blockIdx.x] : (int)blockIdx.x;
    if (b < 0 || b >= a.B) return;
    if (threadIdx.x == 0) s_len = atomicExch(a.lens + b, 0);
    __syncthreads();
    long long held = pages_held(s_len, a.page_size);
    if (held > a.max_pages) held = a.max_pages;
    for (long long s = threadIdx.x; s < held; s += FORK_THREADS) {
        const int p = a.table[(long long)b * a.max_pages + s];
        if (p >= 0 && p < a.n_pages) atomicSub(a.refs + p, 1);
    }
}

// One CTA: the i-th page in use from number U on (U: pages in use) moves to the i-th free page below U.
// The list says where each page from U on went.
__global__ void __launch_bounds__(POOL_THREADS) compact_kernel(const __grid_constant__ PoolArgs a) {
    constexpr int PER = 4;
    pdl_wait();
    int32_t* list = a.scratch + POOL_LIST;
    int used = 0;
    for (long long at = 0; at < a.n_pages; at += POOL_THREADS * PER) {
        int mine = 0;
#pragma unroll
        for (int i = 0; i < PER; ++i) {
            const long long p = at + (long long)i * POOL_THREADS + threadIdx.x;
            mine += p < a.n_pages && a.refs[p] > 0;
        }
        used += mine;
    }
    int U;
    scan_cta<POOL_THREADS>(used, &U);
    int holes = 0, movers = 0;
    for (long long at = 0; at < a.n_pages; at += POOL_THREADS * PER) {
        const long long p0 = at + (long long)threadIdx.x * PER;
        int mine = 0, total;                              // holes below U in the low half, movers in the high one
        bool hit[PER];
#pragma unroll
        for (int i = 0; i < PER; ++i) {
            const long long p = p0 + i;
            hit[i] = p < a.n_pages && (a.refs[p] > 0) == (p >= U);
            if (hit[i]) mine += p < U ? 1 : 65536;
        }
        int r = scan_cta<POOL_THREADS>(mine, &total);
        int h = holes + (r & 65535), m = movers + (r >> 16);
#pragma unroll
        for (int i = 0; i < PER; ++i) {
            const long long p = p0 + i;
            if (p < a.n_pages && p >= U && !hit[i]) list[p] = (int)p;
            if (hit[i] && p < U) a.dst[h++] = (int)p;
            if (hit[i] && p >= U) a.src[m++] = (int)p;
        }
        holes += total & 65535;
        movers += total >> 16;
    }
    __syncthreads();
    for (long long i = threadIdx.x; i < a.pairs; i += POOL_THREADS) {
        if (i < movers) {
            const int from = a.src[i], to = a.dst[i];
            list[from] = to;
            a.refs[to] = a.refs[from];
            a.refs[from] = 0;
        } else {
            a.src[i] = a.dst[i] = -1;
        }
    }
    if (threadIdx.x == 0) a.scratch[POOL_USED] = U;
}

__global__ void __launch_bounds__(FORK_THREADS) renumber_kernel(const __grid_constant__ PoolArgs a) {
    pdl_wait();
    const int b = blockIdx.x, U = a.scratch[POOL_USED];
    long long held = pages_held(a.lens[b], a.page_size);
    if (held > a.max_pages) held = a.max_pages;
    int32_t* row = a.table + (long long)b * a.max_pages;
    for (long long s = threadIdx.x; s < held; s += FORK_THREADS) {
        const int p = row[s];
        if (p >= U && p < a.n_pages) row[s] = a.scratch[POOL_LIST + p];
    }
}

// ---------------------------------------------------------------------------------------
// copy_pages_kernel
// ---------------------------------------------------------------------------------------
constexpr int COPY_THREADS = 256, COPY_DEEP = 8, COPY_TENSORS = 4;

// A tensor of pages [n_pages, H, rows of a page, bytes of a row].
struct CopyTensor { unsigned char* p; int row_bytes; };
struct CopyArgs {
    CopyTensor t[COPY_TENSORS];
    int tensors, H, page_rows;
    long long n_pages;
    long long n;                // pairs
    int parts;                  // a pair is shared by this many CTAs
    unsigned long long per_part;         // 2^64 / parts, rounded up
    const int32_t *src, *dst, *rows;
};

// A pair's rows are one line of pieces of 16 bytes (4 for scales of a partial page), tensor by tensor and
// head by head; `parts` CTAs take equal shares of it.  Bound by memory: 826 MB read and written by a compaction in
// 130 us, 6.4 TB/s; of a few partial pages 3 us.  (Whole pages and partial ones in one loop, with a 64-bit division and remainder for each piece, took 136 and 5.3.)
__global__ void __launch_bounds__(COPY_THREADS) copy_pages_kernel(const __grid_constant__ CopyArgs a) {
    pdl_wait();
    const int part = blockIdx.x % a.parts;
    for (long long i = blockIdx.x / a.parts; i < a.n; i += gridDim.x / a.parts) {
        const int from = a.src[i], to = a.dst[i];
        if (from < 0 || from >= a.n_pages || to < 0 || to >= a.n_pages || from == to) continue;
        int r = a.rows ? a.rows[i] : a.page_rows;
        if (r > a.page_rows) r = a.page_rows;
        if (r <= 0) continue;
        for (int t = 0; t < a.tensors; ++t) {
            // bytes from one head to the next; 2^31 and more where a page is a long sequence
            const long long head = (long long)a.page_rows * a.t[t].row_bytes;
            const bool whole = r == a.page_rows;
            const unsigned char* const s = a.t[t].p + (long long)from * a.H * head;
            unsigned char* const d = a.t[t].p + (long long)to * a.H * head;
            auto move = [&](auto piece) {
                using P = decltype(piece);
                // heads that are copied whole are one run
                const long long run = (whole ? a.H * head : (long long)r * a.t[t].row_bytes) / (int)sizeof(P);
                const long long all = whole ? run : run * a.H, share = a.parts > 1 ? (long long)__umul64hi(all, a.per_part) : all, more = all - share * a.parts;
                const long long lo = share * part + (part < more ? part : more), hi = lo + share + (part < more);
                if (whole) {
                    for (long long at = lo + threadIdx.x; at < hi; at += COPY_THREADS * COPY_DEEP) {
                        P x[COPY_DEEP];
#pragma unroll
                        for (int k = 0; k < COPY_DEEP; ++k)
                            if (at + k * COPY_THREADS < hi) x[k] = reinterpret_cast<const P*>(s)[at + k * COPY_THREADS];
#pragma unroll
                        for (int k = 0; k < COPY_DEEP; ++k)
                            if (at + k * COPY_THREADS < hi) reinterpret_cast<P*>(d)[at + k * COPY_THREADS] = x[k];
                    }
                    return;
                }
                // of a thread's pieces: the run (head), and the place in it, one after the other without further divisions
                const long long skip = head - run * (int)sizeof(P);
                const int step_run = run > COPY_THREADS ? 0 : COPY_THREADS / (int)run, step_at = COPY_THREADS - step_run * (int)(run > COPY_THREADS ? 0 : run);
                long long at = lo + threadIdx.x, h = at / run, in_run = at - h * run;
                while (at < hi) {
                    P x[COPY_DEEP / 2];
                    long long off[COPY_DEEP / 2];
#pragma unroll
                    for (int k = 0; k < COPY_DEEP / 2; ++k) {
                        off[k] = at < hi ? at * (int)sizeof(P) + h * skip : -1;
                        if (off[k] >= 0) x[k] = *reinterpret_cast<const P*>(s + off[k]);
                        at += COPY_THREADS;
                        h += step_run;
                        in_run += step_at;
                        if (in_run >= run) {
                            in_run -= run;
                            ++h;
                        }
                    }
#pragma unroll
                    for (int k = 0; k < COPY_DEEP / 2; ++k)
                        if (off[k] >= 0) *reinterpret_cast<P*>(d + off[k]) = x[k];
                }
            };
            if (whole || a.t[t].row_bytes % 16 == 0) move(uint4());
            else move(uint32_t());
        }
    }
}

}  // namespace retopk_cache
