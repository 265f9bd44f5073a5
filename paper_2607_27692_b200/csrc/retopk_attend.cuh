// Attention over 16-bit pages on the fifth-generation tensor cores (sm_100a).
//
//   plan_kernel      what there is to do: entries of work, one behind the other on a line (of many sequences; of few,
//                    attend_kernel works it out itself)
//   attend_kernel    a CTA takes an equal share of the line
//   join_kernel      joins the parts of a row
//
// An entry is a set of query rows that see the same keys: the members of a group and the rows that they share,
// the tokens of a sequence and the rows of its own, or one token and the blocks selected for it.  Keys that only some of a sequence's
// draft tokens see (its last T - 1) are left to join_kernel, so that a tile of 128 keys has one mask for all
// rows.  For each KV head and 256 query rows an entry has a line of tiles; a piece of a line is what one CTA
// takes of it, and leaves fp32 sums for its rows in the workspace.
//
// Measured (bf16, d = 128, 8 KV heads of 4 queries).  Four sequences of 128K keys on their own, 2.1 GB: 320 us, 6.7 TB/s, as fast as a copy.
// Eight sequences that share 32K keys: 43 us, of which 21 are the floor of reading them; 3 pass until all CTAs know their work,
// 3 until the first scores, 8 in join_kernel.  Of 64 sequences that share 128K: 188 us, 730 TFLOP/s, in short runs; 215 to 228 us and 600 to
// 640 TFLOP/s repeated for seconds, at the power limit.  There the softmax bounds it.  256
// rows of a tile take 4900 cycles: 2048 for the exponentials alone (16 a cycle), about 2560 of the tensor
// core (half tiles of keys read Q anew for 64 keys), and neither is hidden wholly behind the other.
#pragma once
#include <cuda.h>

#include "retopk_cache.cuh"

namespace retopk_cache {

// Keys that token t of T sees in a sequence of `len` keys; none if the cache cannot hold the sequence.
__device__ __forceinline__ int keys_seen(const Pages& pg, int len, int T, int t) {
    if (len < 0 || len > pg.capacity) return 0;
    const int n = len - T + 1 + t;
    return n > 0 ? n : 0;
}

constexpr int ATT_TILE = 128;            // keys of a tile, and query rows of a stream
constexpr int ATT_FEW = 64;              // query rows up to which tiles are taken whole
constexpr int ATT_CHUNK = 1024;          // tiles of a line whose sums one part of a CTA holds at most
// What a CTA's work counts: a tile of up to 128 query rows 1 (two of them are at work at once), one of more rows 2, and the
// beginning of a line 3.  (64 sequences that share 128K, the one size at which this was varied: 237, 210, 201, 191 and 195 us with 1.5, 2, 2.5, 3 and 4.5.)
constexpr int ATT_START = 3;
constexpr float ATT_NONE = -3.402823466e38f, ATT_LOW = -3.3e38f;     // reference of a row without keys; lowest of one with keys
constexpr float ATT_LEAST_SCALE = 1.17549435e-38f;        // stands for a scale of 0

struct Entry {
    int u;                      // where its lines begin
    int item;                   // number of its first (line, chunk): in the order of the lines, with places to spare
    int rows, token;            // query rows: heads of a group of the tokens from `token` on
    int b;                      // sequence whose row of the block table holds the keys
    int lo, hi, seen;           // keys lo..hi-1 (of the selected blocks one behind the other: 0..hi-1, below `seen`)
    int tile0, tiles;
    int row_tiles, chunks;      // 256 query rows each: with the KV heads of each, its lines; chunks of a line
};
struct AttendHeader { int units; };

// Keys and values as [rows of all pages, d] for copies of a box of rows (which lie in one page), of 8 and of single rows.
struct AttendMaps { CUtensorMap k, v, v_eight, v_row; };

struct AttendArgs {
    Pages pg;
    const int32_t* seq_lens;
    const uint16_t* q;
    long long q_stride;
    uint16_t* out;
    float* lse;
    float scale_log2;
    int B, T, Hq, G;
    int n_groups;
    const int32_t *cu, *shared_lens;
    const int32_t* blocks;      // [B, T, H_kv, keep], or null: all keys
    int keep, block, block_shift;
    int entries, grid, max_chunks, own_rows;             // max_chunks: of a line at most; own_rows: rows of a half of a part that belongs to one sequence
    AttendHeader* head;
    Entry* entry;
    int32_t *group_of, *flags;  // group of a sequence or -1; CTAs that gave up
    float *shared_parts, *own_parts;
    int box_shift, total_rows;  // rows of a copy: 1 << box_shift
    bool planned;               // by plan_kernel
    bool few_rows;              // no line has more than ATT_FEW query rows
    // join_kernel: float4s of a row that a CTA has, threads to each, and 1 / rows, 1 / (rows * wide), 1 / G
    int join_wide, join_splits;
    float per_row, per_work, per_G;
};
struct AttendParams {
    AttendMaps maps;
    AttendArgs a;
};

// Floats of a half of a part (one stream's): the sums of four rows each lie together, [rows / 4][D / 4][4 rows][4], so
// that join_kernel finds a sequence's rows in one place; then reference and weight sum of each row.
__host__ __device__ constexpr int half_floats(int rows, int d) { return (rows + 3) / 4 * 4 * (d + 2); }
__device__ __forceinline__ int sums_at(int row, int c4, int d) { return (row >> 2) * (4 * d) + c4 * 16 + (row & 3) * 4; }
__device__ __forceinline__ int weight_at(int row, int rows, int d) { return (rows + 3) / 4 * 4 * d + 2 * row; }
__device__ __forceinline__ int tile_shift(int rows) { return rows > ATT_TILE ? 1 : 0; }
__device__ __forceinline__ int line_units(const Entry& e) { return e.tiles > 0 ? (e.tiles << tile_shift(e.rows)) + ATT_START : 0; }
// Equal shares of the line: that of CTA c begins at floor(units * c / n).  None is below 2 units, of a short line fewer
// CTAs have one: so each that lies between two tiles of a line has a tile of it too, and the parts are without holes.
struct Shares {
    int units, n, whole, rest;
    __device__ __forceinline__ Shares(int units_, int grid) {
        units = units_;
        n = units / 2 < grid ? units / 2 : grid;
        whole = n > 0 ? units / n : 0;
        rest = units - whole * n;
    }
    __device__ __forceinline__ int begin(int c) const { return c < n ? whole * c + rest * c / n : units; }
};

// With few query rows, copies of them fill the 128 of a stream: each copy has a share of a tile's keys to itself,
// so that four warps have the work of one.
__host__ __device__ constexpr int copies_of(int rows) { return rows <= ATT_TILE / 4 ? 4 : (rows <= ATT_TILE / 2 ? 2 : 1); }
// Tiles of a piece at most, as a power of two: their sums stay in the tensor core, which cuts each addition off, 2^-23.5 of a
// sum of one sign on average.  8192 additions (1024 tiles of more than 128 rows; both streams and all copies share those of fewer) are
// 6e-4 of the sum: little next to half a step of bf16, 4e-3, but more than one of fp16, 5e-4.  fp16: up to 1024 additions, 1.1e-4, after which
// the next piece of the same part adds its sums to what is there, rounded in fp32.  (152 lines of 1024 tiles of 256 rows, d = 64: 5.9e-4
// and 2505 us without, 1.1e-4 and 2547 us with it.)
template <int DT> __device__ __forceinline__ int piece_shift(int rows) {
    return DT == TYPE_BF16 ? 10 : 7 + (rows <= ATT_TILE) + (copies_of(rows) >> 1);
}
static_assert(ATT_CHUNK == 1 << 10, "pieces divide chunks");
// Whether the sums of a part's copies become one before they are written.  That takes 1 to 2 us at the end of a piece; in
// join_kernel it saves a half or three quarters of the places, in all parts of the line, that the threads which share a row go
// through.  Done where each of them had 6 or more.  (us without and with it: groups of 2, 4, 8 and 16 sequences that share 32K, 18 parts to
// a line, 40.9 and 38.4, 44.1 and 41.0, 47.3 and 42.9, 46.7 and 44.8; blocks of 4 sequences, 5 parts to a line, 21.8 and 22.2;
// 4 sequences that share 704, 19.7 and 20.7.)
__device__ __forceinline__ bool merges_copies(const AttendArgs& a, int line_units, int rows, int units) {
    const int copies = copies_of(rows);
    return copies > 1 && (long long)line_units * (units / 2 < a.grid ? units / 2 : a.grid) * (2 * copies) >= 6ll * a.join_splits * units;
}
// The CTA whose share holds unit u: the last c with floor(units * c / n) <= u.
__device__ __forceinline__ int share_of(int u, int units, int grid) {
    const int n = units / 2 < grid ? units / 2 : grid;
    const long long end = (u + 1ll) * n;
    int c = (int)(__fdividef((float)u, (float)units) * (float)n);
    c = c < 0 ? 0 : (c < n - 1 ? c : n - 1);
#pragma unroll 1
    while (c > 0 && (long long)units * c >= end) --c;
#pragma unroll 1
    while (c < n - 1 && units * (c + 1ll) < end) ++c;
    return c;
}

// ---------------------------------------------------------------------------------------
// plan_kernel
// ---------------------------------------------------------------------------------------
constexpr int PLAN_THREADS = 1024;

// Where the plan is made from: in global memory, or copies of it in shared memory.
struct PlanInput { const int32_t *seq_lens, *cu, *shared_lens; };

// By one CTA: the entries, the group of each sequence, and how long the line is.  Groups: the first member that is not
// empty owns the keys, the fewest rows that any of them sees are shared; a member alone shares nothing.
// s_part: a number for each warp.
template <int THREADS>
__device__ __forceinline__ int make_plan(const AttendArgs& a, const PlanInput& in, Entry* entry, int32_t* group_of, int* s_part) {
    const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5;
    int groups = 0;
    if (a.n_groups > 0) {
        bool bad = false;
#pragma unroll 1
        for (int g = warp; g < a.n_groups; g += THREADS / 32) {
            int b0 = in.cu[g], b1 = in.cu[g + 1];
            const bool wrong = (b0 < 0) | (b1 < b0) | (b1 > a.B) | ((g == 0) & (b0 != 0)) | ((g == a.n_groups - 1) & (b1 != a.B));
            bad |= wrong;
            if (wrong) b0 = b1 = 0;
            int owner = 0x7fffffff, least = 0x7fffffff, members = 0;
#pragma unroll 1
            for (int b = b0 + lane; b < b1; b += 32) {
                group_of[b] = g;
                const int len = in.seq_lens[b];
                if (len <= 0 || len > a.pg.capacity) continue;
                const int n = (int)keys_seen(a.pg, len, a.T, 0);
                owner = b < owner ? b : owner;
                least = n < least ? n : least;
                ++members;
            }
            owner = __reduce_min_sync(0xffffffffu, owner);
            least = __reduce_min_sync(0xffffffffu, least);
            members = __reduce_add_sync(0xffffffffu, members);
            if (lane == 0) {
                int n = in.shared_lens[g];
                n = members < 2 || n < 0 ? 0 : (n < least ? n : least);
                Entry e;
                e.rows = (b1 - b0) * a.T * a.G;
                e.token = b0 * a.T;
                e.b = n > 0 ? owner : 0;
                e.hi = n;
                entry[g] = e;
            }
        }
        groups = __syncthreads_or(bad) ? 0 : a.n_groups;
        if (groups == 0) {
#pragma unroll 1
            for (int b = tid; b < a.B; b += THREADS) group_of[b] = -1;
            __syncthreads();
        }
    } else if (!a.blocks) {
#pragma unroll 1
        for (int b = tid; b < a.B; b += THREADS) group_of[b] = -1;
    }
    int units = 0;
#pragma unroll 1
    for (int e0 = 0; e0 < a.entries; e0 += THREADS) {
        const int i = e0 + tid;
        const bool on = i < a.entries;
        Entry e;
        e.rows = e.token = e.b = e.lo = e.hi = e.item = 0;
        if (i < a.n_groups) {
            if (groups > 0) e = entry[i];
            e.lo = 0;
            e.seen = e.hi;
            // (groups of x rows in all have at most one row tile each more than x / 256, and so do the first of them)
            e.item = (i + e.token * a.G / (2 * ATT_TILE)) * a.pg.H_kv * a.max_chunks;
        } else if (on) {
            const int at = i - a.n_groups, b = a.blocks ? at / a.T : at;
            e.b = b;
            e.item = at * a.pg.H_kv * a.max_chunks;
            e.seen = (int)keys_seen(a.pg, in.seq_lens[b], a.T, a.blocks ? at - b * a.T : 0);
            if (a.blocks) {
                const int N = (e.seen + a.block - 1) >> a.block_shift;
                e.rows = a.G;
                e.token = at;
                e.hi = (N < a.keep ? N : a.keep) << a.block_shift;
            } else {
                e.rows = a.T * a.G;
                e.token = b * a.T;
                e.hi = e.seen;
                if (groups > 0) e.lo = entry[group_of[b]].hi;
                if (e.lo > e.hi) e.lo = e.hi;
            }
        }
        e.tile0 = e.lo / ATT_TILE;
        e.tiles = e.hi > e.lo ? (e.hi + ATT_TILE - 1) / ATT_TILE - e.tile0 : 0;
        e.row_tiles = (e.rows + 2 * ATT_TILE - 1) / (2 * ATT_TILE);
        e.chunks = (e.tiles + ATT_CHUNK - 1) / ATT_CHUNK;
        int all;
        e.u = units + scan_cta<THREADS>(a.pg.H_kv * e.row_tiles * line_units(e), &all, s_part);
        if (on) entry[i] = e;
        units += all;
    }
    return units;
}

__global__ void __launch_bounds__(PLAN_THREADS) plan_kernel(const __grid_constant__ AttendArgs a) {
    __shared__ int s_part[PLAN_THREADS / 32];
    pdl_wait();
    pdl_start_next();
    const int units = make_plan<PLAN_THREADS>(a, {a.seq_lens, a.cu, a.shared_lens}, a.entry, a.group_of, s_part);
    if (threadIdx.x == 0) a.head->units = units;
}

// ---------------------------------------------------------------------------------------
// Barriers and the tensor core
// ---------------------------------------------------------------------------------------
__device__ __forceinline__ uint32_t smem_of(const void* p) { return (uint32_t)__cvta_generic_to_shared(p); }
__device__ __forceinline__ void bar_init(uint32_t bar, int count) { asm volatile("mbarrier.init.shared::cta.b64 [%0], %1;" ::"r"(bar), "r"(count) : "memory"); }
__device__ __forceinline__ void bar_arrive(uint32_t bar) { asm volatile("mbarrier.arrive.shared::cta.b64 _, [%0];" ::"r"(bar) : "memory"); }
__device__ __forceinline__ bool bar_try(uint32_t bar, uint32_t parity) {
    uint32_t ok;
    asm volatile("{\n.reg .pred p;\nmbarrier.try_wait.parity.shared::cta.b64 p, [%1], %2;\nselp.u32 %0, 1, 0, p;\n}" : "=r"(ok) : "r"(bar), "r"(parity) : "memory");
    return ok != 0;
}
__device__ __forceinline__ unsigned long long clock_ns() {
    unsigned long long t;
    asm volatile("mov.u64 %0, %globaltimer;" : "=l"(t));
    return t;
}
// Waits for the phase; gives up after two seconds, or when another part of the CTA has.
__device__ __noinline__ bool bar_wait_long(uint32_t bar, uint32_t parity, volatile int* gave_up) {
    const unsigned long long begin = clock_ns();
    for (;;) {
        for (int i = 0; i < 64; ++i)
            if (bar_try(bar, parity)) return true;
        if (*gave_up) return false;
        if (clock_ns() - begin > 2000000000ull) {
            *gave_up = 1;
            return false;
        }
    }
}
__device__ __forceinline__ bool bar_wait(uint32_t bar, uint32_t parity, volatile int* gave_up) {
    if (bar_try(bar, parity)) return true;
    return bar_wait_long(bar, parity, gave_up);
}

__device__ __forceinline__ void fence_async() { asm volatile("fence.proxy.async.shared::cta;" ::: "memory"); }
__device__ __forceinline__ void tc_before_sync() { asm volatile("tcgen05.fence::before_thread_sync;" ::: "memory"); }
__device__ __forceinline__ void tc_after_sync() { asm volatile("tcgen05.fence::after_thread_sync;" ::: "memory"); }
__device__ __forceinline__ void tc_commit(uint32_t bar, uint32_t issue) {
    asm volatile("{\n.reg .pred q;\nsetp.ne.u32 q, %1, 0;\n@q tcgen05.commit.cta_group::1.mbarrier::arrive::one.shared::cluster.b64 [%0];\n}" ::"r"(bar), "r"(issue) : "memory");
}
__device__ __forceinline__ void tc_wait_ld() { asm volatile("tcgen05.wait::ld.sync.aligned;" ::: "memory"); }
__device__ __forceinline__ void tc_wait_st() { asm volatile("tcgen05.wait::st.sync.aligned;" ::: "memory"); }

// D (+)= A B, 128 x N x 16; A in shared memory or in tensor memory.  The whole warp comes here, the one lane with
// `issue` issues: operands that are the same for all lanes stay in uniform registers, where the instruction takes them from.
__device__ __forceinline__ void tc_mma_ss(uint32_t d, uint64_t a, uint64_t b, uint32_t idesc, bool add, uint32_t issue) {
    asm volatile("{\n.reg .pred p, q;\nsetp.ne.u32 p, %4, 0;\nsetp.ne.u32 q, %5, 0;\n@q tcgen05.mma.cta_group::1.kind::f16 [%0], %1, %2, %3, p;\n}"
                 ::"r"(d), "l"(a), "l"(b), "r"(idesc), "r"((uint32_t)add), "r"(issue) : "memory");
}
__device__ __forceinline__ void tc_mma_ts(uint32_t d, uint32_t a, uint64_t b, uint32_t idesc, bool add, uint32_t issue) {
    asm volatile("{\n.reg .pred p, q;\nsetp.ne.u32 p, %4, 0;\nsetp.ne.u32 q, %5, 0;\n@q tcgen05.mma.cta_group::1.kind::f16 [%0], [%1], %2, %3, p;\n}"
                 ::"r"(d), "r"(a), "l"(b), "r"(idesc), "r"((uint32_t)add), "r"(issue) : "memory");
}
__device__ __forceinline__ uint32_t elect_one() {
    uint32_t one;
    asm volatile("{\n.reg .pred p;\nelect.sync _|p, 0xffffffff;\nselp.u32 %0, 1, 0, p;\n}" : "=r"(one));
    return one;
}

#define TC_R8(x, i) "=r"(x[i]), "=r"(x[i + 1]), "=r"(x[i + 2]), "=r"(x[i + 3]), "=r"(x[i + 4]), "=r"(x[i + 5]), "=r"(x[i + 6]), "=r"(x[i + 7])
#define TC_W8(x, i) "r"(x[i]), "r"(x[i + 1]), "r"(x[i + 2]), "r"(x[i + 3]), "r"(x[i + 4]), "r"(x[i + 5]), "r"(x[i + 6]), "r"(x[i + 7])
#define TC_RW8(x, i) "+r"(x[i]), "+r"(x[i + 1]), "+r"(x[i + 2]), "+r"(x[i + 3]), "+r"(x[i + 4]), "+r"(x[i + 5]), "+r"(x[i + 6]), "+r"(x[i + 7])
// 32 columns of the lanes of this warp; tc_wait_ld and tc_loaded before the values are used.
__device__ __forceinline__ void tc_ld32(uint32_t addr, uint32_t* x) {
    asm volatile("tcgen05.ld.sync.aligned.32x32b.x32.b32 {%0, %1, %2, %3, %4, %5, %6, %7, %8, %9, %10, %11, %12, %13, %14, %15, "
                 "%16, %17, %18, %19, %20, %21, %22, %23, %24, %25, %26, %27, %28, %29, %30, %31}, [%32];"
                 : TC_R8(x, 0), TC_R8(x, 8), TC_R8(x, 16), TC_R8(x, 24) : "r"(addr));
}
// Behind the wait: without it the compiler sees nothing that keeps what uses x from being moved before the wait.
__device__ __forceinline__ void tc_loaded16(uint32_t* x) { asm volatile("" : TC_RW8(x, 0), TC_RW8(x, 8)); }
__device__ __forceinline__ void tc_loaded32(uint32_t* x) { asm volatile("" : TC_RW8(x, 0), TC_RW8(x, 8), TC_RW8(x, 16), TC_RW8(x, 24)); }
__device__ __forceinline__ void tc_st16(uint32_t addr, const uint32_t* x) {
    asm volatile("tcgen05.st.sync.aligned.32x32b.x16.b32 [%0], {%1, %2, %3, %4, %5, %6, %7, %8, %9, %10, %11, %12, %13, %14, %15, %16};"
                 ::"r"(addr), TC_W8(x, 0), TC_W8(x, 8) : "memory");
}
__device__ __forceinline__ void tc_ld16(uint32_t addr, uint32_t* x) {
    asm volatile("tcgen05.ld.sync.aligned.32x32b.x16.b32 {%0, %1, %2, %3, %4, %5, %6, %7, %8, %9, %10, %11, %12, %13, %14, %15}, [%16];"
                 : TC_R8(x, 0), TC_R8(x, 8) : "r"(addr));
}
__device__ __forceinline__ void tc_st32(uint32_t addr, const uint32_t* x) {
    asm volatile("tcgen05.st.sync.aligned.32x32b.x32.b32 [%0], {%1, %2, %3, %4, %5, %6, %7, %8, %9, %10, %11, %12, %13, %14, %15, %16, "
                 "%17, %18, %19, %20, %21, %22, %23, %24, %25, %26, %27, %28, %29, %30, %31, %32};"
                 ::"r"(addr), TC_W8(x, 0), TC_W8(x, 8), TC_W8(x, 16), TC_W8(x, 24) : "memory");
}
__device__ __forceinline__ float exp2_approx(float x) {
    float y;
    asm("ex2.approx.ftz.f32 %0, %1;" : "=f"(y) : "f"(x));
    return y;
}

// Two fp32 operations at once, on pairs of registers.
__device__ __forceinline__ uint64_t pair_of(uint32_t lo, uint32_t hi) { return (uint64_t)hi << 32 | lo; }
__device__ __forceinline__ uint64_t pair_of(float lo, float hi) { return pair_of(__float_as_uint(lo), __float_as_uint(hi)); }
__device__ __forceinline__ float low_of(uint64_t x) { return __uint_as_float((uint32_t)x); }
__device__ __forceinline__ float high_of(uint64_t x) { return __uint_as_float((uint32_t)(x >> 32)); }
__device__ __forceinline__ uint64_t fma2(uint64_t a, uint64_t b, uint64_t c) {
    uint64_t d;
    asm("fma.rn.f32x2 %0, %1, %2, %3;" : "=l"(d) : "l"(a), "l"(b), "l"(c));
    return d;
}
__device__ __forceinline__ uint64_t add2(uint64_t a, uint64_t b) {
    uint64_t d;
    asm("add.rn.f32x2 %0, %1, %2;" : "=l"(d) : "l"(a), "l"(b));
    return d;
}

// Shared memory operand with rows of 128 bytes, 16-byte columns exchanged within 8 rows (128-byte swizzle);
// `lead`: bytes between halves of 64 channels where the operand runs along the channels.
__device__ __forceinline__ uint64_t tc_operand(uint32_t addr, uint32_t lead) {
    return (uint64_t)((addr & 0x3ffff) >> 4) | (uint64_t)(lead >> 4) << 16 | (uint64_t)(1024 >> 4) << 32 | 1ull << 46 | 2ull << 61;
}
// Accumulators in fp32, operands of one 16-bit type, 128 x n; b_along_n: B lies with its rows along k.
template <int DT> __host__ __device__ constexpr uint32_t tc_shape(int n, bool b_along_n) {
    return 1u << 4 | (uint32_t)(DT == TYPE_BF16) << 7 | (uint32_t)(DT == TYPE_BF16) << 10 | (uint32_t)b_along_n << 16 |
           (uint32_t)(n >> 3) << 17 | (uint32_t)(ATT_TILE >> 4) << 24;
}

// ---------------------------------------------------------------------------------------
// attend_kernel
// ---------------------------------------------------------------------------------------
constexpr int ATT_SOFT_WARPS = 8, ATT_LOAD_WARP = ATT_SOFT_WARPS, ATT_MMA_WARP = ATT_LOAD_WARP + 2;      // (two of each)
constexpr int ATT_WARPS = ATT_MMA_WARP + 2, ATT_THREADS = ATT_WARPS * 32;
constexpr int ATT_PIECES = 32;           // pieces that a CTA lists at once
constexpr int ATT_MASKS = 8;             // tiles of a stream whose masks are kept

// Loads of a piece of n tiles, j = 0 .. 2 n - 1: K0, K1, V0, K2, V1, .., K(n-1), V(n-2), V(n-1).
__device__ __forceinline__ int k_load(int t) { return t == 0 ? 0 : 2 * t - 1; }
__device__ __forceinline__ int v_load(int t, int n) { return t == n - 1 ? 2 * n - 1 : 2 * t + 2; }
__device__ __forceinline__ int tile_of_load(int j, int n) { return j == 0 ? 0 : (j == 2 * n - 1 ? n - 1 : (j & 1 ? (j + 1) >> 1 : (j >> 1) - 1)); }

struct Piece {
    int b, h, token, row0, rows, half_rows;
    int lo, hi, seen, tile0, tile1;
    bool merge;                 // the copies' sums become one
    bool more;                  // its sums are added to those that the CTA's piece before left in the same part
    float* part;
};
template <int D> struct AttendSmem {
    static constexpr int TILE_BYTES = ATT_TILE * D * 2;
    static constexpr int SLOTS = 5 * 128 / D;
    unsigned char q[2][TILE_BYTES];
    unsigned char ring[SLOTS][TILE_BYTES];
    uint32_t mask[2][ATT_MASKS][4];                      // of each stream's own tiles, one after the other
    uint64_t full[SLOTS], empty[SLOTS], mask_ready[2][ATT_MASKS], q_ready[2], s_ready[2][2], p_ready[2][2], o_ready[2][2], merged[2], drained[2];         // [stream][half of a tile]
    Piece piece[ATT_PIECES];
    int warp_sum[ATT_WARPS];
    uint32_t issued[SLOTS];     // last load into a slot
    uint32_t tmem;
    int gave_up;
};

// Two streams of four warps each take the softmax of 128 query rows: with up to 128 rows both have the same
// rows and every other tile, with more a stream has 128 of 256 rows and every tile.  While one is at its
// softmax the tensor core works for the other.  One warp fetches keys, one values, by copies of as many rows as
// lie in a page together, into a ring of 5 tiles of 32 KB at d = 128; for each stream one thread issues the products: S = Q K^T into
// tensor memory, O += P V with P over the columns of S.  With many rows half a tile of keys at a time, so that the other half
// is at its softmax; WHOLE, for calls without a line of more than 64 rows (whose copies leave each warp 32 or 64 of a tile's keys): all
// of it at once, with fewer waits.  (us, whole and halves: blocks of 4 sequences 37.3 and 39.4, of ragged ones 35.9 and 39.4, 4 short sequences
// 15.5 and 16.9; with the maxima that it takes, 32 sequences of 128 rows in all would be 56 and 52, 64 of 256 rows 222 and 188.)
// Rows of values that do not count (masked, pages out of range) are read from behind the last row, where a copy
// finds zeros; a weight of 0 would not hide a NaN.
// Weights are taken against a reference that need not be the maximum (halves: as long as their sum stays below 2^14; WHOLE: each below
// 2^8), so that most halves need neither maxima nor a rescaling of O; they are rounded to 16 bits once, for the tensor core.  In
// two parts each, as the attention over 4-bit pages has them, O += P V and the conversions would be twice as much where they and the
// softmax bound the kernel already; rounded once, outputs are 0.0023 (bf16) and 0.0003 (fp16) off on average, 0.0017 and 0.0002 of which
// is the rounding of the output itself.  Their sum is that of the weights before they are rounded.
template <int DT, int D, bool WHOLE>
__global__ void __launch_bounds__(ATT_THREADS, 1) attend_kernel(const __grid_constant__ AttendParams params) {
    using Smem = AttendSmem<D>;
    const AttendArgs& a = params.a;
    const AttendMaps& maps = params.maps;
    extern __shared__ __align__(1024) unsigned char att_smem[];
    Smem& sm = *reinterpret_cast<Smem*>(att_smem);
    const int tid = threadIdx.x, lane = tid & 31, warp = __shfl_sync(0xffffffffu, tid >> 5, 0), cta = blockIdx.x;
    volatile int* gave_up = &sm.gave_up;
    if (tid == 0) {
        sm.gave_up = (smem_of(att_smem) & 1023) != 0;    // operands need the alignment
#pragma unroll 1
        for (int i = 0; i < Smem::SLOTS; ++i) {
            bar_init(smem_of(&sm.full[i]), 1);
            sm.issued[i] = ~0u;
            bar_init(smem_of(&sm.empty[i]), 2);           // one of each stream
        }
#pragma unroll 1
        for (int i = 0; i < 2 * ATT_MASKS; ++i) bar_init(smem_of(&sm.mask_ready[i / ATT_MASKS][i % ATT_MASKS]), 1);
        for (int i = 0; i < 2; ++i) {
            bar_init(smem_of(&sm.q_ready[i]), 4);
            for (int h = 0; h < 2; ++h) {
                bar_init(smem_of(&sm.s_ready[i][h]), 1);
                bar_init(smem_of(&sm.p_ready[i][h]), 4);
                bar_init(smem_of(&sm.o_ready[i][h]), 1);
            }
        }
        for (int i = 0; i < 2; ++i) {
            bar_init(smem_of(&sm.drained[i]), 1);
            bar_init(smem_of(&sm.merged[i]), 4);
        }
        asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
    }
    if (tid == 32) {
        asm volatile("prefetch.tensormap [%0];" ::"l"(&maps.k) : "memory");
        asm volatile("prefetch.tensormap [%0];" ::"l"(&maps.v) : "memory");
    }
    if (warp == ATT_MMA_WARP) {
        asm volatile("tcgen05.alloc.cta_group::1.sync.aligned.shared::cta.b32 [%0], 512;" ::"r"(smem_of(&sm.tmem)) : "memory");
        asm volatile("tcgen05.relinquish_alloc_permit.cta_group::1.sync.aligned;" ::: "memory");
    }
    pdl_wait();
    pdl_start_next();

    // what the roles keep from piece to piece
    uint32_t loads = 0, masks[2] = {0, 0};               // loads issued (or consumed), masks written for each stream
    uint32_t turns = 0, begun = 0, merges = 0;           // of a stream: tiles behind, pieces begun, times its warps waited for each other
    bool ok = true;

    for (int batch = 0;; ++batch) {
        // ---- the pieces of this CTA, ATT_PIECES at a time ------------------------------------------
        // (a plan of this CTA's own is laid out where the ring is, which is empty between batches)
        const Entry* plan = a.entry;
        int units;
        if (a.planned) {
            units = a.head->units;
        } else {
            Entry* own_plan = reinterpret_cast<Entry*>(sm.ring);
            int32_t* const lens = reinterpret_cast<int32_t*>(own_plan + ATT_THREADS);
            int32_t *const cu = lens + ATT_THREADS, *const shared_lens = cu + ATT_THREADS, *const group_of = shared_lens + ATT_THREADS;
            if (tid < a.B) lens[tid] = a.seq_lens[tid];
            if (tid <= a.n_groups && a.n_groups > 0) cu[tid] = a.cu[tid];
            if (tid < a.n_groups) shared_lens[tid] = a.shared_lens[tid];
            __syncthreads();
            units = make_plan<ATT_THREADS>(a, {lens, cu, shared_lens}, own_plan, group_of, sm.warp_sum);
            plan = own_plan;
            if (cta == 0 && batch == 0) {                // for join_kernel
                __syncthreads();
                if (tid < a.entries) a.entry[tid] = own_plan[tid];
                if (tid < a.B && !a.blocks) a.group_of[tid] = group_of[tid];
                if (tid == 0) a.head->units = units;
            }
        }
        const Shares shares(units, a.grid);
        const int u0 = shares.begin(cta), u1 = shares.begin(cta + 1);
        int listed = 0;
#pragma unroll 1
        for (int e0 = 0; e0 < a.entries && u0 < u1; e0 += ATT_THREADS) {
            const int i = e0 + tid;
            Entry e;
            int from = 0, to = 0, len = 1, shift = 0, cut = 0, count = 0, lines0 = 0, lines1 = 0;
            // tiles of this CTA in a line: those that its units stand for
            auto range_of = [&](int line, int& t0, int& t1) {
                const int x0 = from > line * len ? from - line * len : 0, x1 = to - line * len < len ? to - line * len : len;
                t0 = x0 > ATT_START ? (x0 - ATT_START + (1 << shift) - 1) >> shift : 0;
                t1 = x1 > ATT_START ? (x1 - ATT_START + (1 << shift) - 1) >> shift : 0;
            };
            if (i < a.entries) {
                e = plan[i];
                len = line_units(e);
                shift = tile_shift(e.rows);
                cut = piece_shift<DT>(e.rows);
                from = u0 > e.u ? u0 - e.u : 0;
                const int all = len * a.pg.H_kv * e.row_tiles;
                to = u1 - e.u < all ? u1 - e.u : all;
                if (to > from) {
                    lines0 = from / len;
                    lines1 = (to - 1) / len;
#pragma unroll 1
                    for (int line = lines0; line <= lines1; line = line == lines0 && lines1 > lines0 + 1 ? lines1 : line + 1) {
                        int t0, t1;
                        range_of(line, t0, t1);
                        if (t1 > t0) count += ((t1 - 1) >> cut) - (t0 >> cut) + 1;
                    }
                    if (lines1 > lines0 + 1) count += (lines1 - lines0 - 1) * (((e.tiles - 1) >> cut) + 1);
                }
            }
            int total, at = listed + scan_cta<ATT_THREADS>(count, &total, sm.warp_sum) - batch * ATT_PIECES;     // of this entry's first piece
            listed += total;
            if (count > 0 && at < ATT_PIECES && at + count > 0) {
#pragma unroll 1
                for (int line = lines0; line <= lines1 && at < ATT_PIECES; ++line) {
                    int first, t1;
                    range_of(line, first, t1);
#pragma unroll 1
                    for (int t0 = first; t0 < t1; t0 = ((t0 >> cut) + 1) << cut, ++at) {
                        if (at < 0 || at >= ATT_PIECES) continue;
                        const int chunk = t0 / ATT_CHUNK, next = ((t0 >> cut) + 1) << cut, end = next < t1 ? next : t1;
                        Piece p;
                        p.b = e.b;
                        const int row_tile = line / a.pg.H_kv;
                        p.h = line - row_tile * a.pg.H_kv;
                        p.token = e.token;
                        p.row0 = row_tile * (2 * ATT_TILE);
                        p.rows = e.rows - p.row0 < 2 * ATT_TILE ? e.rows - p.row0 : 2 * ATT_TILE;
                        p.lo = e.lo;
                        p.hi = e.hi;
                        p.seen = e.seen;
                        p.merge = merges_copies(a, e.tiles << shift, p.rows, units);
                        p.more = t0 > first && t0 % ATT_CHUNK != 0;
                        p.tile0 = e.tile0 + t0;
                        p.tile1 = e.tile0 + end;
                        const long long slot = (long long)e.item + (long long)line * a.max_chunks + chunk + cta;
                        const bool own = i >= a.n_groups;
                        p.half_rows = own ? a.own_rows : ATT_TILE;
                        p.part = (own ? a.own_parts : a.shared_parts) + slot * (2 * half_floats(p.half_rows, D));
                        sm.piece[at] = p;
                    }
                }
            }
            __syncthreads();
        }
        int pieces = listed - batch * ATT_PIECES;
        pieces = pieces < ATT_PIECES ? pieces : ATT_PIECES;
        fence_async();                                   // the plan has been read: copies may take its place
        tc_before_sync();
        __syncthreads();
        tc_after_sync();
        if (pieces <= 0 || !ok) break;                   // (the same for all threads)
        const uint32_t tmem = sm.tmem;

        if (warp >= ATT_LOAD_WARP && warp < ATT_MMA_WARP) {
            // ---- loads: keys by one warp, values by the other ------------------------------------
            const bool keys = warp == ATT_LOAD_WARP;
            const CUtensorMap* map = keys ? &maps.k : &maps.v;
            const int box_shift = a.box_shift, box = 1 << box_shift;
            // A box of a copy's rows to a lane, of as many tiles as that makes: at 16 rows of 4 tiles.  Its first row or -1,
            // and which of its rows count.
            struct Box { int row, from, to; };
            auto look_up = [&](const Piece& p, int at) -> Box {          // at: its place among the keys
                const int lo = p.lo, hi = p.hi, seen = p.seen;
                int pos = at;                            // position in the sequence
                if (a.blocks && at < hi) {
                    const int j = a.blocks[((long long)p.token * a.pg.H_kv + p.h) * a.keep + (at >> a.block_shift)];
                    pos = j < 0 || j > (seen - 1) >> a.block_shift ? -1 : (j << a.block_shift) + (at & (a.block - 1));
                }
                const long long found = at >= hi || at + box <= lo ? -1 : cache_row(a.pg, p.b, pos);
                Box x;
                x.row = found < 0 ? -1 : (int)(found + (long long)p.h * a.pg.page_size);
                x.from = lo > at ? lo - at : 0;
                x.to = hi - at < seen - pos ? hi - at : seen - pos;
                x.to = x.to < box ? x.to : box;
                if (x.row < 0 || x.to <= x.from) x.from = x.to = 0;
                return x;
            };
            auto copy = [&](const CUtensorMap* m, uint32_t dst, int row, uint32_t bar) {
#pragma unroll
                for (int c = 0; c < D / 64; ++c)
                    asm volatile("cp.async.bulk.tensor.2d.shared::cta.global.tile.mbarrier::complete_tx::bytes [%0], [%1, {%2, %3}], [%4];"
                                 ::"r"(dst + c * (ATT_TILE * 128)), "l"(m), "r"(c * 64), "r"(row), "r"(bar) : "memory");
            };
            // the copies of a box; of values that do not count none but zeros
            auto fetch = [&](const Box& x, uint32_t dst, uint32_t bar) {
                if (x.to == 0 || keys || x.to - x.from == box) {
                    copy(map, dst, x.to == 0 ? a.total_rows : x.row, bar);
                    return;
                }
                const int step = box < 8 ? box : 8;
#pragma unroll 1
                for (int r = 0; r < box; r += step) {
                    const bool none = x.to <= r || x.from >= r + step, all = x.from <= r && x.to >= r + step;
                    if (step == 8 && (none || all)) {
                        copy(&maps.v_eight, dst + r * 128, all ? x.row + r : a.total_rows, bar);
                    } else {
#pragma unroll 1
                        for (int e = r; e < r + step; ++e) copy(&maps.v_row, dst + e * 128, e >= x.from && e < x.to ? x.row + e : a.total_rows, bar);
                    }
                }
            };
            const int boxes = ATT_TILE >> box_shift, tile_shift = 7 - box_shift;         // of a tile
            const int ahead = boxes <= 32 ? 32 >> tile_shift : 1;        // tiles that are looked up at once
            Box next;
            if (boxes <= 32) next = look_up(sm.piece[0], sm.piece[0].tile0 * ATT_TILE + (lane << box_shift));
#pragma unroll 1
            for (int i = 0; i < pieces && ok; ++i) {
                const Piece p = sm.piece[i];
                const int n = p.tile1 - p.tile0;
                const bool both = !WHOLE && p.rows > ATT_TILE;           // every tile is both streams'
                Box mine;
                int at = ahead;                          // of the tiles looked up last
#pragma unroll 1
                for (int t = 0; t < n && ok; ++t, ++at) {
                    if (at == ahead) {                   // (those after them are looked up meanwhile, of the next piece too)
                        at = 0;
                        mine = next;
                        if (boxes <= 32) {
                            const bool more = t + ahead < n;
                            if (more || i + 1 < pieces) {
                                const Piece& c = sm.piece[more ? i : i + 1];
                                next = look_up(c, (c.tile0 + (more ? t + ahead : 0)) * ATT_TILE + (lane << box_shift));
                            }
                        }
                    }
                    const uint32_t load = loads + (keys ? k_load(t) : v_load(t, n)), slot = load % Smem::SLOTS, turn = load / Smem::SLOTS;
                    ok = __all_sync(0xffffffffu, bar_wait(smem_of(&sm.empty[slot]), (turn & 1) ^ 1, gave_up));
                    if (!ok) break;
                    const uint32_t bar = smem_of(&sm.full[slot]), dst = smem_of(sm.ring[slot]);
                    if (lane == 0) asm volatile("mbarrier.arrive.expect_tx.shared::cta.b64 _, [%0], %1;" ::"r"(bar), "r"(Smem::TILE_BYTES) : "memory");
                    __syncwarp();
                    uint32_t valid = 0;                  // of rows 4 * lane on
                    if (boxes <= 32) {
                        if (lane >> tile_shift == at) fetch(mine, dst + (lane << box_shift) * 128 - at * (ATT_TILE * 128), bar);
                        const int range = __shfl_sync(0xffffffffu, mine.from | mine.to << 16, (at << tile_shift) + (lane * 4 >> box_shift));
                        const int first = lane * 4 & (box - 1), from = (range & 0xffff) - first, to = (range >> 16) - first;
#pragma unroll
                        for (int e = 0; e < 4; ++e) valid |= e >= from && e < to ? 1u << e : 0u;
                    } else {                             // boxes of one or two rows
#pragma unroll 1
                        for (int e = 0; e < 4; e += box) {
                            const Box x = look_up(p, (p.tile0 + t) * ATT_TILE + lane * 4 + e);
                            fetch(x, dst + (lane * 4 + e) * 128, bar);
                            valid |= ((1u << x.to) - (1u << x.from)) << e;
                        }
                    }
                    if (lane == 0) sm.issued[slot] = load;
                    if (keys) {
                        // The mask, for the stream or the two that take the tile.  A stream's masks are numbered as its turns are, so that
                        // it waits for each of them and a phase of a barrier cannot be taken for the one before.  That of its turn
                        // 8 back is no longer read: the softmax of that was over before this slot came free.
                        uint32_t m = valid << (lane % 8 * 4);
                        m |= __shfl_xor_sync(0xffffffffu, m, 1);
                        m |= __shfl_xor_sync(0xffffffffu, m, 2);
                        m |= __shfl_xor_sync(0xffffffffu, m, 4);
#pragma unroll
                        for (int s = 0; s < 2; ++s)
                            if (both || (t & 1) == s) {
                                if (lane % 8 == 0) sm.mask[s][masks[s] % ATT_MASKS][lane / 8] = m;
                                __syncwarp();
                                if (lane == 0) bar_arrive(smem_of(&sm.mask_ready[s][masks[s] % ATT_MASKS]));
                                ++masks[s];
                            }
                    }
                }
                loads += 2 * n;
            }
            if (!ok && lane == 0) {                      // copies that are under way end before the memory is given back
                volatile int never = 0;
                for (int x = 0; x < Smem::SLOTS; ++x)
                    if (sm.issued[x] != ~0u) bar_wait(smem_of(&sm.full[x]), sm.issued[x] / Smem::SLOTS & 1, &never);
            }
            __syncwarp();
        } else if (warp >= ATT_MMA_WARP) {
            // ---- products: a warp for each stream ------------------------------------------------
            constexpr uint32_t QK = tc_shape<DT>(WHOLE ? ATT_TILE : ATT_TILE / 2, false), PV = tc_shape<DT>(D, true);
            const uint32_t issue = elect_one();          // always the same lane
            const int s = warp - ATT_MMA_WARP;
            const uint32_t S = tmem + s * ATT_TILE, O = tmem + 2 * ATT_TILE + s * D, q = smem_of(sm.q[s]);
#pragma unroll 1
            for (int i = 0; i < pieces && ok; ++i) {
                const Piece& p = sm.piece[i];
                const int n = __shfl_sync(0xffffffffu, p.tile1 - p.tile0, 0), step = WHOLE ? 2 : __shfl_sync(0xffffffffu, p.rows > ATT_TILE ? 1 : 2, 0);
                auto wait_full = [&](int j) { return bar_wait(smem_of(&sm.full[(loads + j) % Smem::SLOTS]), (loads + j) / Smem::SLOTS & 1, gave_up); };
                auto tile_at = [&](int j) { return __shfl_sync(0xffffffffu, smem_of(sm.ring[(loads + j) % Smem::SLOTS]), 0); };
                auto empty_at = [&](int j) { return smem_of(&sm.empty[(loads + j) % Smem::SLOTS]); };
                // Both warps see all loads go by, so that neither runs away from the other: a phase of a
                // barrier is told from the one after the next by nothing else.  What the other stream has loaded is given back
                // behind the products that this warp has issued, not before they are over: a place of the ring is one warp's
                // and the other's load in turn, and either takes for granted that what was there two loads before has been
                // given back when its own load before has (loads are then given back in their order but for neighbours).
                int seen = 0;
                auto see = [&](int j) -> bool {          // the other stream's loads before j
                    if (step == 2)
                        for (; seen < j; ++seen)
                            if ((tile_of_load(seen, n) & 1) != s) {
                                if (!wait_full(seen)) return false;
                                tc_commit(empty_at(seen), issue);
                            }
                    return true;
                };
                const int first = step == 1 ? 0 : s;
                if constexpr (WHOLE) {
                    auto score = [&](int t) {                // S = Q K^T
                        const uint32_t k = tile_at(k_load(t));
                        tc_after_sync();
#pragma unroll
                        for (int x = 0; x < D / 16; ++x) {
                            const uint32_t off = (x >> 2) * (ATT_TILE * 128) + (x & 3) * 32;
                            tc_mma_ss(S, tc_operand(q + off, 0), tc_operand(k + off, 0), QK, x > 0, issue);
                        }
                        tc_commit(smem_of(&sm.s_ready[s][0]), issue);
                        tc_commit(empty_at(k_load(t)), issue);
                    };
                    if (first < n) {
                        // (weights that S takes the place of have been read)
                        ok = see(k_load(first)) && bar_wait(smem_of(&sm.q_ready[s]), begun & 1, gave_up) && wait_full(k_load(first)) &&
                             (turns == 0 || bar_wait(smem_of(&sm.o_ready[s][0]), (turns - 1) & 1, gave_up));
                        ++begun;
                        if (__all_sync(0xffffffffu, ok)) score(first);
                    }
                    for (int t = first; t < n && __all_sync(0xffffffffu, ok); t += step) {
                        ok = see(v_load(t, n) < k_load(t + step) ? v_load(t, n) : k_load(t + step)) && wait_full(v_load(t, n));
                        const uint32_t v = tile_at(v_load(t, n));
                        ok = __all_sync(0xffffffffu, ok && bar_wait(smem_of(&sm.p_ready[s][0]), turns & 1, gave_up));
                        if (!ok) break;
                        tc_after_sync();
#pragma unroll
                        for (int x = 0; x < ATT_TILE / 16; ++x)              // O += P V
                            tc_mma_ts(O, S + x * 8, tc_operand(v + x * 2048, ATT_TILE * 128), PV, x > 0 || t >= step, issue);
                        tc_commit(smem_of(&sm.o_ready[s][0]), issue);
                        tc_commit(empty_at(v_load(t, n)), issue);
                        if (t + step < n) {
                            ok = __all_sync(0xffffffffu, wait_full(k_load(t + step)) && bar_wait(smem_of(&sm.o_ready[s][0]), turns & 1, gave_up));
                            if (ok) score(t + step);
                        }
                        ++turns;
                    }
                } else {
                    auto score = [&](int t, int h) {         // S = Q K^T of half a tile
                        const uint32_t k = tile_at(k_load(t)) + h * (ATT_TILE / 2 * 128);
                        tc_after_sync();
#pragma unroll
                        for (int x = 0; x < D / 16; ++x) {
                            const uint32_t off = (x >> 2) * (ATT_TILE * 128) + (x & 3) * 32;
                            tc_mma_ss(S + h * (ATT_TILE / 2), tc_operand(q + off, 0), tc_operand(k + off, 0), QK, x > 0, issue);
                        }
                        tc_commit(smem_of(&sm.s_ready[s][h]), issue);
                        if (h == 1) tc_commit(empty_at(k_load(t)), issue);
                    };
                    // weights that S takes the place of have been read
                    auto wait_o = [&](int h) { return turns == 0 || bar_wait(smem_of(&sm.o_ready[s][h]), (turns - 1) & 1, gave_up); };
                    if (first < n) {
                        ok = see(k_load(first)) && bar_wait(smem_of(&sm.q_ready[s]), begun & 1, gave_up) && wait_full(k_load(first));
                        ++begun;
#pragma unroll
                        for (int h = 0; h < 2; ++h) {
                            ok = ok && wait_o(h);
                            if (__all_sync(0xffffffffu, ok)) score(first, h);
                        }
                    }
                    for (int t = first; t < n && __all_sync(0xffffffffu, ok); t += step) {
                        ok = see(v_load(t, n) < k_load(t + step) ? v_load(t, n) : k_load(t + step)) && wait_full(v_load(t, n));
                        const uint32_t v = tile_at(v_load(t, n));
                        const bool more = t + step < n;
#pragma unroll
                        for (int h = 0; h < 2; ++h) {
                            ok = __all_sync(0xffffffffu, ok && bar_wait(smem_of(&sm.p_ready[s][h]), turns & 1, gave_up));
                            if (!ok) break;
                            tc_after_sync();
#pragma unroll
                            for (int x = 0; x < ATT_TILE / 32; ++x)                  // O += P V
                                tc_mma_ts(O, S + h * (ATT_TILE / 2) + x * 8, tc_operand(v + (h * 4 + x) * 2048, ATT_TILE * 128), PV, x > 0 || h > 0 || t >= step, issue);
                            tc_commit(smem_of(&sm.o_ready[s][h]), issue);
                            if (h == 1) tc_commit(empty_at(v_load(t, n)), issue);
                            if (more) {
                                ok = __all_sync(0xffffffffu, (h == 1 || wait_full(k_load(t + step))) && bar_wait(smem_of(&sm.o_ready[s][h]), turns & 1, gave_up));
                                if (ok) score(t + step, h);
                            }
                        }
                        ++turns;
                    }
                }
                ok = ok && see(2 * n);
                ok = __all_sync(0xffffffffu, ok);
                loads += 2 * n;
            }
            if (!ok) {                                   // what was issued ends before the memory is given back
                tc_commit(smem_of(&sm.drained[s]), issue);
                volatile int never = 0;
                bar_wait(smem_of(&sm.drained[s]), 0, &never);
                *gave_up = 1;
            }
            __syncwarp();
        } else {
            // ---- softmax -------------------------------------------------------------------------
            const int s = warp >> 2, row = (warp & 3) * 32 + lane;
            const uint32_t lanes = tmem + ((uint32_t)(warp & 3) << 21);
            const uint32_t S = lanes + s * ATT_TILE, O = lanes + 2 * ATT_TILE + s * D;
            // (a scale of 0 as the smallest: 0 times the -inf of a hidden key is no number)
            const float scale = a.scale_log2 == 0.f ? ATT_LEAST_SCALE : fabsf(a.scale_log2);
            // tiles of this stream in a piece (WHOLE: none has more rows than ATT_FEW)
            auto turns_of = [&](const Piece& p) { return !WHOLE && p.rows > ATT_TILE ? p.tile1 - p.tile0 : (p.tile1 - p.tile0 + 1 - s) / 2; };
            // this thread's query row in a piece, or -1; the copy that it belongs to
            auto row_of = [&](const Piece& p, int* copy) {
                const int copies = copies_of(p.rows), stride = ATT_TILE / copies, r = row % stride + (p.rows > ATT_TILE ? s * ATT_TILE : 0);
                *copy = copies == 1 ? 0 : row / stride;
                return r < p.rows ? r : -1;
            };
            auto fetch_q = [&](const Piece& p) {
                int copy;
                const int r = p.row0 + row_of(p, &copy);
                if (r >= p.row0) {
                    const uint16_t* src = a.q + ((long long)p.token + r / a.G) * a.q_stride + (long long)(p.h * a.G + r % a.G) * D;
                    const uint32_t dst = smem_of(sm.q[s]) + row * 128;
#pragma unroll
                    for (int c = 0; c < D / 8; ++c) cp_async16(dst + (c >> 3) * (ATT_TILE * 128) + (((c & 7) ^ (row & 7)) << 4), src + c * 8);
                }
                cp_async_commit();
            };
            auto give_q = [&](const Piece& p) {
                cp_async_wait<0>();
                int copy;
                if (a.scale_log2 < 0.f && row_of(p, &copy) >= 0)         // a negative scale turns the queries' signs
#pragma unroll 1
                    for (int c = 0; c < D / 8; ++c) {
                        uint4* x = reinterpret_cast<uint4*>(sm.q[s] + (c >> 3) * (ATT_TILE * 128) + row * 128 + ((c & 7) << 4));
                        x->x ^= 0x80008000u; x->y ^= 0x80008000u; x->z ^= 0x80008000u; x->w ^= 0x80008000u;
                    }
                fence_async();
                __syncwarp();
                if (lane == 0) bar_arrive(smem_of(&sm.q_ready[s]));
            };
            bool fetched = false;                        // the queries of the next piece are there
#pragma unroll 1
            for (int i = 0; i < pieces && ok; ++i) {
                const Piece& p = sm.piece[i];
                const int turn_count = turns_of(p), copies = copies_of(p.rows);
                int copy;
                const int r = row_of(p, &copy);
                const bool live = r >= 0, warp_live = __any_sync(0xffffffffu, live);
                const int c0 = copy * (4 / copies), c1 = c0 + 4 / copies;        // columns of this warp, in 32s
                float ref = ATT_NONE, l = 0.f;
                // (the queries of the first tile; those of the next piece are asked for at the last tile, in the same place)
                bool here = fetched || turn_count == 0;
                fetched = false;
#pragma unroll 1
                for (int k = 0; k < turn_count && ok; ++k) {
                    const bool ahead = !p.merge && k == turn_count - 1 && i + 1 < pieces && turns_of(sm.piece[i + 1]) > 0;
                    if (__builtin_expect(!here, 0)) {
                        fetch_q(p);
                        give_q(p);
                        here = true;
                    }
                    ok = bar_wait(smem_of(&sm.mask_ready[s][turns % ATT_MASKS]), turns / ATT_MASKS & 1, gave_up);
                    if constexpr (WHOLE) {
                        ok = __all_sync(0xffffffffu, ok && bar_wait(smem_of(&sm.s_ready[s][0]), turns & 1, gave_up));
                        if (!ok) break;
                        if (__builtin_expect(ahead, 0)) fetch_q(sm.piece[i + 1]);        // the queries of this piece have been read
                        if (warp_live) {
                            tc_after_sync();
                            // this copy's columns, 32 or 64 of them
                            const uint32_t* masks = sm.mask[s][turns % ATT_MASKS] + c0;
                            const bool two = c1 - c0 > 1;
                            uint32_t x[64];
                            tc_ld32(S + c0 * 32, x);
                            if (two) tc_ld32(S + c0 * 32 + 32, x + 32);
                            const uint32_t m0 = masks[0], m1 = two ? masks[1] : 0, any = m0 | m1;
                            tc_wait_ld();
                            tc_loaded32(x);
                            tc_loaded32(x + 32);
                            auto hide = [&](uint32_t* v, uint32_t m) {   // keys that do not count: weight 0
                                if (__builtin_expect(m == ~0u, 1)) return;
#pragma unroll
                                for (int j = 0; j < 32; ++j)
                                    if (!(m >> j & 1)) v[j] = 0xff800000u;
                            };
                            hide(x, m0);
                            hide(x + 32, m1);
                            float most[4] = {-INFINITY, -INFINITY, -INFINITY, -INFINITY};
                            auto larger = [&](const uint32_t* v) {
#pragma unroll
                                for (int j = 0; j < 32; j += 8)
#pragma unroll
                                    for (int e = 0; e < 4; ++e) most[e] = fmaxf(most[e], fmaxf(__uint_as_float(v[j + e]), __uint_as_float(v[j + e + 4])));
                            };
                            larger(x);
                            if (two) larger(x + 32);
                            // The reference need not be the maximum, as long as weights stay below 2^8: where the maximum is 8 above it
                            // (in powers of two), it becomes that, and sums so far follow.
                            const float top = any ? fmaxf(fmaxf(fmaxf(most[0], most[1]), fmaxf(most[2], most[3])) * scale, ATT_LOW) : ATT_NONE;
                            const bool low = live && (top > ref + 8.f || (ref == ATT_NONE && any));
                            if (__builtin_expect(__any_sync(0xffffffffu, low), 0)) {
                                const float f = low ? exp2_approx(ref - top) : 1.f;
                                if (low) ref = top;
                                l *= f;
                                if (k > 0) {             // (scores are there: the product of the tile before is over)
#pragma unroll 1
                                    for (int c = 0; c < D; c += 16) {
                                        uint32_t o[16];
                                        tc_ld16(O + c, o);
                                        tc_wait_ld();
                                        tc_loaded16(o);
#pragma unroll
                                        for (int j = 0; j < 16; ++j) o[j] = __float_as_uint(__uint_as_float(o[j]) * f);
                                        tc_st16(O + c, o);
                                    }
                                }
                            }
                            const uint64_t scale2 = pair_of(scale, scale), ref2 = pair_of(-ref, -ref);
                            uint64_t sum = 0, more = 0;
                            auto weigh = [&](const uint32_t* y, int c) {
                                uint32_t w[16];
#pragma unroll
                                for (int j = 0; j < 32; j += 4) {
                                    const uint64_t u = fma2(pair_of(y[j], y[j + 1]), scale2, ref2), v = fma2(pair_of(y[j + 2], y[j + 3]), scale2, ref2);
                                    const float u0 = exp2_approx(low_of(u)), u1 = exp2_approx(high_of(u));
                                    const float v0 = exp2_approx(low_of(v)), v1 = exp2_approx(high_of(v));
                                    sum = add2(sum, pair_of(u0, u1));
                                    more = add2(more, pair_of(v0, v1));
                                    w[j / 2] = pack2<DT>(u0, u1);
                                    w[j / 2 + 1] = pack2<DT>(v0, v1);
                                }
                                tc_st16(S + c * 16, w);
                            };
                            weigh(x, c0);
                            if (two) weigh(x + 32, c0 + 1);
                            sum = add2(sum, more);
                            l += low_of(sum) + high_of(sum);
                            uint32_t none[16];           // other copies' keys
#pragma unroll
                            for (int j = 0; j < 16; ++j) none[j] = 0;
#pragma unroll 1
                            for (int c = 0; c < 4; ++c)
                                if (c < c0 || c >= c1) tc_st16(S + c * 16, none);
                            tc_wait_st();
                            tc_before_sync();
                        }
                        __syncwarp();
                        if (lane == 0) bar_arrive(smem_of(&sm.p_ready[s][0]));
                    } else {
#pragma unroll 1
                        for (int h = 0; h < 2; ++h) {
                            ok = __all_sync(0xffffffffu, ok && bar_wait(smem_of(&sm.s_ready[s][h]), turns & 1, gave_up));
                            if (!ok) break;
                            if (__builtin_expect(ahead && h == 1, 0)) fetch_q(sm.piece[i + 1]);   // the queries of this piece have been read: the next one's take their place
                            if (warp_live) {
                                tc_after_sync();
                                const uint32_t Sh = S + h * (ATT_TILE / 2);
                                uint32_t x[32], y[32];
                                // this copy's columns: both 32s of the half, one, or none
                                const bool first = 2 * h >= c0 && 2 * h < c1, second = 2 * h + 1 >= c0 && 2 * h + 1 < c1;
                                uint32_t mx = sm.mask[s][turns % ATT_MASKS][2 * h], my = sm.mask[s][turns % ATT_MASKS][2 * h + 1];
                                if (!first) mx = 0;
                                if (!second) my = 0;
                                if (__builtin_expect(first | second, 1)) {
                                    if (__builtin_expect(first, 1)) tc_ld32(Sh, x);
                                    if (__builtin_expect(second, 1)) tc_ld32(Sh + 32, y);
                                    tc_wait_ld();
                                    tc_loaded32(x);
                                    tc_loaded32(y);
                                    auto hide = [&](uint32_t* v, uint32_t m) {       // keys that do not count: weight 0
                                        if (__builtin_expect(m == ~0u, 1)) return;
#pragma unroll
                                        for (int j = 0; j < 32; ++j)
                                            if (!(m >> j & 1)) v[j] = 0xff800000u;
                                    };
                                    hide(x, mx);
                                    hide(y, my);
                                    uint32_t w[32];
                                    float total;
                                    auto weigh = [&]() {
                                        const uint64_t scale2 = pair_of(scale, scale), ref2 = pair_of(-ref, -ref);
                                        uint64_t sum = 0, more = 0;
#pragma unroll
                                        for (int j = 0; j < 32; j += 2) {
                                            const uint64_t u = fma2(pair_of(x[j], x[j + 1]), scale2, ref2), v = fma2(pair_of(y[j], y[j + 1]), scale2, ref2);
                                            const float u0 = exp2_approx(low_of(u)), u1 = exp2_approx(high_of(u));
                                            const float v0 = exp2_approx(low_of(v)), v1 = exp2_approx(high_of(v));
                                            sum = add2(sum, pair_of(u0, u1));
                                            more = add2(more, pair_of(v0, v1));
                                            w[j / 2] = pack2<DT>(u0, u1);
                                            w[16 + j / 2] = pack2<DT>(v0, v1);
                                        }
                                        sum = add2(sum, more);
                                        total = low_of(sum) + high_of(sum);
                                    };
                                    // Weights come first, against the reference that is there: it need not be the maximum, as long
                                    // as no sum leaves 2^14 (what fp16 weights can hold).  Where one does, or there was none
                                    // before, the reference becomes the maximum, and sums so far and weights follow.
                                    weigh();
                                    const bool low = live && (!(total <= 16384.f) || (ref == ATT_NONE && (mx | my)));
                                    if (__builtin_expect(__any_sync(0xffffffffu, low), 0)) {
                                        float most[4] = {-INFINITY, -INFINITY, -INFINITY, -INFINITY};
#pragma unroll
                                        for (int j = 0; j < 32; j += 2) {
                                            most[j & 2] = fmaxf(most[j & 2], fmaxf(__uint_as_float(x[j]), __uint_as_float(x[j + 1])));
                                            most[(j & 2) + 1] = fmaxf(most[(j & 2) + 1], fmaxf(__uint_as_float(y[j]), __uint_as_float(y[j + 1])));
                                        }
                                        const float top = fmaxf(fmaxf(fmaxf(most[0], most[1]), fmaxf(most[2], most[3])) * scale, ATT_LOW);
                                        float f = 1.f;
                                        if (low && top > ref) {
                                            f = exp2_approx(ref - top);
                                            ref = top;
                                            l *= f;
                                        }
                                        if (k > 0 || h > 0) {
                                            // (the product of the half before may be under way)
                                            ok = __all_sync(0xffffffffu, bar_wait(smem_of(&sm.o_ready[s][1 - h]), (h == 0 ? turns - 1 : turns) & 1, gave_up));
                                            if (!ok) break;
                                            tc_after_sync();
#pragma unroll 1
                                            for (int c = 0; c < D; c += 16) {
                                                uint32_t o[16];
                                                tc_ld16(O + c, o);
                                                tc_wait_ld();
                                                tc_loaded16(o);
#pragma unroll
                                                for (int j = 0; j < 16; ++j) o[j] = __float_as_uint(__uint_as_float(o[j]) * f);
                                                tc_st16(O + c, o);
                                            }
                                        }
                                        weigh();
                                    }
                                    l += total;
                                    tc_st32(Sh, w);
                                } else {                     // another copy's keys
#pragma unroll
                                    for (int j = 0; j < 32; ++j) x[j] = 0;
                                    tc_st32(Sh, x);
                                }
                                tc_wait_st();
                                tc_before_sync();
                            }
                            __syncwarp();
                            if (lane == 0) bar_arrive(smem_of(&sm.p_ready[s][h]));
                        }
                    }
                    ++turns;
                    if (__builtin_expect(ok && ahead, 0)) {
                        give_q(sm.piece[i + 1]);
                        fetched = true;
                    }
                }
                // ---- the sums of this piece ------------------------------------------------------
                float* part = p.part + s * half_floats(p.half_rows, D);
                const int at = p.merge ? row % (ATT_TILE / copies) : copy * (p.half_rows / copies) + row % (ATT_TILE / copies);
                if (ok && turn_count > 0) {
                    ok = __all_sync(0xffffffffu, bar_wait(smem_of(&sm.o_ready[s][0]), (turns - 1) & 1, gave_up) &&
                                                     (WHOLE || bar_wait(smem_of(&sm.o_ready[s][1]), (turns - 1) & 1, gave_up)));
                    tc_after_sync();
                }
                // What is there of the part's rows already (with `more`): reference and weight sum, and the factors for its sums and for this piece's.
                const bool adds = DT == TYPE_FP16 && p.more && turn_count > 0;
                float2 old = make_float2(ATT_NONE, 0.f);
                float keep = 0.f, take = 1.f;
                auto add_weights = [&](float& top, float& sum) {
                    if (old.x == ATT_NONE) return;
                    const float now = fmaxf(old.x, top);
                    keep = exp2_approx(old.x - now);
                    take = exp2_approx(top - now);
                    top = now;
                    sum = fmaf(old.y, keep, sum * take);
                };
                if (adds && live) old = *reinterpret_cast<const float2*>(part + weight_at(at, p.half_rows, D));
                if (!p.merge || turn_count == 0) {
                    if (adds) add_weights(ref, l);
                    if (live && (!p.merge || copy == 0) && (turn_count > 0 || !p.more)) *reinterpret_cast<float2*>(part + weight_at(at, p.half_rows, D)) = make_float2(ref, l);
                    if (ok && turn_count > 0 && warp_live) {
#pragma unroll 1
                        for (int c = 0; c < D; c += 32) {
                            uint32_t x[32];
                            tc_ld32(O + c, x);
                            tc_wait_ld();
                            tc_loaded32(x);
                            if (adds && old.x != ATT_NONE) {
#pragma unroll
                                for (int j = 0; j < 32; j += 4) {
                                    const float4 y = *reinterpret_cast<const float4*>(part + sums_at(at, (c + j) / 4, D));
                                    x[j] = __float_as_uint(fmaf(y.x, keep, __uint_as_float(x[j]) * take));
                                    x[j + 1] = __float_as_uint(fmaf(y.y, keep, __uint_as_float(x[j + 1]) * take));
                                    x[j + 2] = __float_as_uint(fmaf(y.z, keep, __uint_as_float(x[j + 2]) * take));
                                    x[j + 3] = __float_as_uint(fmaf(y.w, keep, __uint_as_float(x[j + 3]) * take));
                                }
                            }
                            if (live) {
#pragma unroll
                                for (int j = 0; j < 32; j += 4)
                                    *reinterpret_cast<uint4*>(part + sums_at(at, (c + j) / 4, D)) = make_uint4(x[j], x[j + 1], x[j + 2], x[j + 3]);
                            }
                        }
                    }
                } else {
                    // The copies' sums become one, in the place of the queries, which have been read: references first, then
                    // half of the channels at a time.  A copy adds up a share of the channels.  (Written out as they are, they
                    // would be 2 or 4 times as much to write here and to read in join_kernel.)
                    auto meet = [&]() {                  // the warps of the stream
                        __syncwarp();
                        if (lane == 0) bar_arrive(smem_of(&sm.merged[s]));
                        ok = __all_sync(0xffffffffu, ok && bar_wait(smem_of(&sm.merged[s]), merges & 1, gave_up));
                        ++merges;
                    };
                    constexpr int F4 = D / 8;            // float4s of half a row
                    float4* const sums = reinterpret_cast<float4*>(sm.q[s]);
                    float2* const refs = reinterpret_cast<float2*>(sm.q[s]);
                    if (ok) refs[row] = make_float2(ref, l);
                    meet();
                    float top = ATT_NONE, total = 0.f, e[4];
#pragma unroll
                    for (int c = 0; c < 4; ++c) {
                        e[c] = c < copies ? refs[at + c * (ATT_TILE / copies)].x : ATT_NONE;
                        top = fmaxf(top, e[c]);
                    }
#pragma unroll
                    for (int c = 0; c < 4; ++c) {
                        e[c] = e[c] == ATT_NONE ? 0.f : exp2_approx(e[c] - top);
                        if (c < copies) total = fmaf(refs[at + c * (ATT_TILE / copies)].y, e[c], total);
                    }
                    if (adds) {                          // (all copies have read what copy 0 writes now)
                        add_weights(top, total);
#pragma unroll
                        for (int c = 0; c < 4; ++c) e[c] *= take;
                    }
                    if (ok && live && copy == 0) *reinterpret_cast<float2*>(part + weight_at(at, p.half_rows, D)) = make_float2(top, total);
                    meet();
#pragma unroll 1
                    for (int half = 0; half < 2 && ok; ++half) {
#pragma unroll 1
                        for (int c = 0; c < D / 2; c += 32) {
                            uint32_t x[32];
                            tc_ld32(O + half * (D / 2) + c, x);
                            tc_wait_ld();
                            tc_loaded32(x);
#pragma unroll
                            for (int j = 0; j < 32; j += 4)
                                *reinterpret_cast<uint4*>(&sums[row * F4 + (((c + j) / 4) ^ (row & 7))]) = make_uint4(x[j], x[j + 1], x[j + 2], x[j + 3]);
                        }
                        meet();
                        if (!ok) break;
#pragma unroll 1
                        for (int c4 = copy * (F4 / copies); c4 < (copy + 1) * (F4 / copies); ++c4) {
                            float4 y = make_float4(0.f, 0.f, 0.f, 0.f);
                            if (adds && old.x != ATT_NONE) {
                                y = *reinterpret_cast<const float4*>(part + sums_at(at, half * F4 + c4, D));
                                y = make_float4(y.x * keep, y.y * keep, y.z * keep, y.w * keep);
                            }
#pragma unroll
                            for (int c = 0; c < 4; ++c) {
                                if (c >= copies) break;
                                const float4 v = sums[(at + c * (ATT_TILE / copies)) * F4 + (c4 ^ (row & 7))];
                                y = make_float4(fmaf(v.x, e[c], y.x), fmaf(v.y, e[c], y.y), fmaf(v.z, e[c], y.z), fmaf(v.w, e[c], y.w));
                            }
                            if (live) *reinterpret_cast<float4*>(part + sums_at(at, half * F4 + c4, D)) = y;
                        }
                        meet();
                    }
                }
                if (turn_count > 0) tc_before_sync();
            }
        }
        ok = !__syncthreads_or(!ok) && !*gave_up;
        if (listed <= (batch + 1) * ATT_PIECES || !ok) break;
    }
    tc_before_sync();
    __syncthreads();
    if (warp == ATT_MMA_WARP) asm volatile("tcgen05.dealloc.cta_group::1.sync.aligned.b32 %0, 512;" ::"r"(sm.tmem) : "memory");
    if (tid == 0) a.flags[cta] = !ok;
}

// ---------------------------------------------------------------------------------------
// join_kernel
// ---------------------------------------------------------------------------------------
constexpr int JOIN_THREADS = 256, JOIN_DEEP = 4, JOIN_CTAS = 8;          // (CTAs that share the channels at most)

// x / n for 0 <= x < 2^13 and n <= x or not much more, from 1 / n: an integer division takes several times as long
__device__ __forceinline__ int small_div(int x, float per_n) { return (int)(((float)x + 0.5f) * per_n); }

// A KV head of one sequence (or token), or a share of its channels.  Bound by waiting: 8 us at 148 parts of 8 lines, of which a
// launch, the plan, the parts and the output take about 1, 2, 3 and 1.  The parts that hold its rows lie one behind
// the other: a line's, in the order of the CTAs that had it (its group's line, of which its rows may be in two, and its own).
// Four channels of a row go to a thread, or to several that share the parts.  All orders are fixed, so that
// results do not depend on timing.  What does not need the parts is done before they are there; what is left is a few
// steps that wait for memory one after the other, so each loads all it can.
template <int DT, int D> __global__ void __launch_bounds__(JOIN_THREADS, 4) join_kernel(const __grid_constant__ AttendArgs a) {
    __shared__ float s_late[16 * 16 * 16];               // scores of the keys that the first token does not see, 16 to a row
    __shared__ long long s_late_row[16];
    __shared__ struct { const float* part; int count; } s_line[3];       // parts of a chunk of a line: the first one, and how many
    __shared__ float4 s_o[JOIN_THREADS];
    __shared__ float2 s_ml[JOIN_THREADS];
    const int i = blockIdx.x, h = blockIdx.y, tid = threadIdx.x;         // entry a.n_groups + i
    const int rows = a.blocks ? a.G : a.T * a.G, token0 = a.blocks ? i : i * a.T;
    // later draft tokens: all queries are read before the first output is written, which may take their place
    int late = 0, first_seen = 0;
    if (!a.blocks && a.T > 1) {
        const int len = a.seq_lens[i], end = keys_seen(a.pg, len, a.T, a.T - 1);
        first_seen = keys_seen(a.pg, len, a.T, 0);
        late = end - first_seen;
        if (tid < late) {
            const long long row = cache_row(a.pg, i, first_seen + tid);
            s_late_row[tid] = row < 0 ? -1 : row + (long long)h * a.pg.page_size;
        }
        first_seen = len - a.T + 1 - first_seen;         // (below 0 where the first tokens see nothing)
        __syncthreads();
        const int shift = late > 1 ? 32 - __clz(late - 1) : 0;
        // 8 lanes to a score
#pragma unroll 1
        for (int x0 = 0; x0 < rows << shift && late > 0; x0 += JOIN_THREADS / 8) {
            const int x = x0 + tid / 8, r = x >> shift, k = x - (r << shift), share = tid % 8, t = small_div(r, a.per_G);
            float s = 0.f;
            const bool sees = r < rows && k < late && k < first_seen + t && s_late_row[k] >= 0;
            if (sees) {
                const uint16_t* key = reinterpret_cast<const uint16_t*>(a.pg.k) + s_late_row[k] * D + share * 8;
                const uint16_t* q = a.q + ((long long)token0 + t) * a.q_stride + (long long)(h * a.G + r - t * a.G) * D + share * 8;
#pragma unroll
                for (int c = 0; c < D; c += 64) {
                    float kf[8], qf[8];
                    unpack8<DT>(*reinterpret_cast<const uint4*>(key + c), kf);
                    unpack8<DT>(*reinterpret_cast<const uint4*>(q + c), qf);
#pragma unroll
                    for (int e = 0; e < 8; ++e) s = fmaf(qf[e], kf[e], s);
                }
            }
#pragma unroll
            for (int o = 1; o < 8; o <<= 1) s += __shfl_xor_sync(0xffffffffu, s, o);
            if (sees && share == 0) s_late[r * 16 + k] = s * (a.scale_log2 == 0.f ? ATT_LEAST_SCALE : a.scale_log2);
        }
    }
    pdl_wait();
    const int flag = tid < a.grid ? a.flags[tid] : 0;
    const int units = a.head->units;
    const int g = a.blocks ? -1 : a.group_of[i];
    const Entry* own = a.entry + a.n_groups + i;
    const Entry* group = a.entry + (g >= 0 ? g : 0);
    // (an empty sequence has no part in its group's line)
    const bool shared = g >= 0 && own->hi >= group->hi && group->tiles > 0;
    const int shared_row = shared ? (token0 - group->token) * a.G : 0, m0 = shared_row / (2 * ATT_TILE), group_rows = shared ? group->rows : 0;
    const int group_chunks = shared ? group->chunks : 0, chunks = group_chunks > own->chunks ? group_chunks : own->chunks;
    const int group_units = shared ? group->tiles << tile_shift(group->rows) : 0;
    const bool own_merge = merges_copies(a, own->tiles << tile_shift(rows), rows, units);
    bool failed = false;
    const int work = rows * a.join_wide, splits = a.join_splits;
#pragma unroll 1
    for (int x0 = 0; x0 < work; x0 += JOIN_THREADS) {
        const int split = splits > 1 ? small_div(tid, a.per_work) : 0, x = x0 + tid - split * work, quad = small_div(x, a.per_row);
        const int r = x - quad * rows, c4 = blockIdx.z * a.join_wide + quad;
        const bool on = x < work && split < splits;
        float M = ATT_NONE, L = 0.f;
        float4 O = make_float4(0.f, 0.f, 0.f, 0.f);
        // Chunk by chunk (of lines of more than ATT_CHUNK tiles); a sequence without keys has its late ones
#pragma unroll 1
        for (int chunk = 0; chunk == 0 || chunk < chunks; ++chunk) {
            if (chunk > 0 || x0 > 0) __syncthreads();
            if (tid % 32 == 0 && tid < 96) {             // one warp for each: who had the chunk
                const int which = tid / 32;
                const Entry* e = which < 2 ? group : own;
                int count = 0;
                if (which == 2 || (shared && (which == 0 || (shared_row + rows - 1) / (2 * ATT_TILE) > m0))) {
                    const int line = (which < 2 ? m0 + which : 0) * a.pg.H_kv + h, tile0 = chunk * ATT_CHUNK, left = e->tiles - tile0;
                    const int tiles = left < ATT_CHUNK ? left : ATT_CHUNK, shift = tile_shift(e->rows), u = e->u + line * line_units(*e) + ATT_START + (tile0 << shift);
                    if (tiles > 0) {
                        const int c0 = share_of(u, units, a.grid);
                        count = share_of(u + ((tiles - 1) << shift), units, a.grid) - c0 + 1;
                        s_line[which].part = (which < 2 ? a.shared_parts : a.own_parts) +
                                             ((long long)e->item + (long long)line * a.max_chunks + chunk + c0) * (2 * half_floats(which < 2 ? ATT_TILE : a.own_rows, D));
                    }
                }
                s_line[which].count = count;
            }
            failed = __syncthreads_or(flag != 0);
            if (on) {
                // Row `row` of a row tile: with more than 128 rows in one half of each part, with fewer in both, in
                // `copies` places.  Places of the group's line, then of the own one, then the late keys.
                const int row = shared_row + r - m0 * (2 * ATT_TILE), m = row / (2 * ATT_TILE), tile_rows = group_rows - (m0 + m) * (2 * ATT_TILE);
                const int g_copies = merges_copies(a, group_units, tile_rows, units) ? 0 : copies_of(tile_rows) >> 1;       // as shifts: 0, 1, 2
                const int o_copies = own_merge ? 0 : copies_of(rows) >> 1;
                const int g_shift = tile_rows > ATT_TILE ? 0 : g_copies + 1, o_shift = rows > ATT_TILE ? 0 : o_copies + 1;
                const int n_group = s_line[m].count << g_shift, n_own = n_group + (s_line[2].count << o_shift);
                const int sees = chunk == 0 && late > 0 ? first_seen + small_div(r, a.per_G) : 0, all = n_own + (sees < late ? (sees > 0 ? sees : 0) : late);
                const float *g_part = s_line[m].part, *o_part = s_line[2].part;
                // (a float2 of the row's reference and sum, and its sums)
                const int g_row = row % (2 * ATT_TILE) % ATT_TILE, o_row = r % ATT_TILE;
                const int g_half = half_floats(ATT_TILE, D), o_half = half_floats(a.own_rows, D);
                const int g_skip = row % (2 * ATT_TILE) / ATT_TILE, o_skip = r / ATT_TILE;
#pragma unroll 1
                for (int k0 = split; k0 < all; k0 += splits * JOIN_DEEP) {
                    float2 ml[JOIN_DEEP];
                    float4 o[JOIN_DEEP];
#pragma unroll
                    for (int d = 0; d < JOIN_DEEP; ++d) {
                        const int k = k0 + d * splits;
                        ml[d] = make_float2(ATT_NONE, 0.f);
                        o[d] = make_float4(0.f, 0.f, 0.f, 0.f);
                        if (k < n_own) {
                            const bool of_group = k < n_group;
                            const int shift = of_group ? g_shift : o_shift, j = of_group ? k : k - n_group;
                            const int half_rows = of_group ? ATT_TILE : a.own_rows, place = j & ((1 << shift) - 1);
                            const int at = of_group ? g_row + (place >> 1) * (ATT_TILE >> g_copies) : o_row + (place >> 1) * (a.own_rows >> o_copies);
                            const int which = 2 * (j >> shift) + (of_group ? g_skip : o_skip) + (place & 1);
                            const float* half = (of_group ? g_part : o_part) + (long long)which * (of_group ? g_half : o_half);
                            ml[d] = *reinterpret_cast<const float2*>(half + weight_at(at, half_rows, D));
                            o[d] = *reinterpret_cast<const float4*>(half + sums_at(at, c4, D));
                        } else if (k < all && s_late_row[k - n_own] >= 0) {
                            const uint2 v = *reinterpret_cast<const uint2*>(reinterpret_cast<const uint16_t*>(a.pg.v) + s_late_row[k - n_own] * D + c4 * 4);
                            // (a score of -inf is a weight of 0, one of NaN a weight of NaN: the reference stays a number, as a
                            // tile's does, so that the row is one with keys)
                            const float score = s_late[r * 16 + k - n_own], w = score == -INFINITY ? 0.f : (score != score ? score : 1.f);
                            ml[d] = make_float2(fmaxf(score, ATT_LOW), w);
                            const float2 v0 = unpack2<DT>(v.x), v1 = unpack2<DT>(v.y);
                            o[d] = make_float4(v0.x * w, v0.y * w, v1.x * w, v1.y * w);
                        }
                    }
                    float top = M;
#pragma unroll
                    for (int d = 0; d < JOIN_DEEP; ++d) {
                        if (ml[d].x == ATT_NONE) o[d] = make_float4(0.f, 0.f, 0.f, 0.f);             // (never written)
                        top = fmaxf(top, ml[d].x);
                    }
                    const float f = exp2_approx(M - top);
                    M = top;
                    L *= f;
                    O = make_float4(O.x * f, O.y * f, O.z * f, O.w * f);
#pragma unroll
                    for (int d = 0; d < JOIN_DEEP; ++d) {
                        const float e = exp2_approx(ml[d].x - top);
                        L = fmaf(ml[d].y, e, L);
                        O = make_float4(fmaf(o[d].x, e, O.x), fmaf(o[d].y, e, O.y), fmaf(o[d].z, e, O.z), fmaf(o[d].w, e, O.w));
                    }
                }
            }
        }
        // the splits of an item: by 2 or 4 neighbouring threads, and these by shuffles
        int item = x;
        bool writes = on;
        if (splits > 1) {
            s_ml[tid] = make_float2(M, L);
            s_o[tid] = O;
            __syncthreads();
            const int fan = splits < 4 ? 1 : 2;          // as a shift
            item = tid >> fan;
            writes = item < work && (tid & ((1 << fan) - 1)) == 0;
            M = ATT_NONE, L = 0.f;
            O = make_float4(0.f, 0.f, 0.f, 0.f);
            const int first = item < work ? tid & ((1 << fan) - 1) : splits;
#pragma unroll 4
            for (int k = first; k < splits; k += 1 << fan) M = fmaxf(M, s_ml[item + k * work].x);
#pragma unroll 1
            for (int o = 1; o < 1 << fan; o <<= 1) M = fmaxf(M, __shfl_xor_sync(0xffffffffu, M, o));
#pragma unroll 4
            for (int k = first; k < splits; k += 1 << fan) {
                const float2 ml = s_ml[item + k * work];
                const float4 o = s_o[item + k * work];
                const float e = exp2_approx(ml.x - M);
                L = fmaf(ml.y, e, L);
                O = make_float4(fmaf(o.x, e, O.x), fmaf(o.y, e, O.y), fmaf(o.z, e, O.z), fmaf(o.w, e, O.w));
            }
#pragma unroll 1
            for (int o = 1; o < 1 << fan; o <<= 1) {
                L += __shfl_xor_sync(0xffffffffu, L, o);
                O.x += __shfl_xor_sync(0xffffffffu, O.x, o);
                O.y += __shfl_xor_sync(0xffffffffu, O.y, o);
                O.z += __shfl_xor_sync(0xffffffffu, O.z, o);
                O.w += __shfl_xor_sync(0xffffffffu, O.w, o);
            }
        }
        if (!writes) continue;
        const int column = small_div(item, a.per_row), out_row = item - column * rows, out_c4 = blockIdx.z * a.join_wide + column, t = small_div(out_row, a.per_G);
        const long long at = ((long long)token0 + t) * a.Hq + h * a.G + out_row - t * a.G;
        const float per_L = 1.f / L;
        float4 y = make_float4(0.f, 0.f, 0.f, 0.f);
        if (M != ATT_NONE) y = make_float4(O.x * per_L, O.y * per_L, O.z * per_L, O.w * per_L);
        if (failed) y.x = y.y = y.z = y.w = __int_as_float(0x7fc00000);
        *reinterpret_cast<uint2*>(a.out + at * D + out_c4 * 4) = make_uint2(pack2<DT>(y.x, y.y), pack2<DT>(y.z, y.w));
        if (a.lse && out_c4 == 0) a.lse[at] = failed ? y.x : (M == ATT_NONE ? -INFINITY : (M + log2f(L)) * 0.69314718f);
    }
}

}  // namespace retopk_cache
