// Host side of the attention over 16-bit pages and of the selection of blocks: argument checks, launches,
// C interface.
#include "retopk_blocks.cuh"

#include <math.h>
#include <mutex>

#include "retopk_cache_host.cuh"

using namespace retopk_cache;

namespace {

int check_shape(int B, int T, int H_q, int H_kv, int d) {
    if (B < 1 || T < 1 || H_q < 1 || H_kv < 1 || H_q % H_kv != 0) return RETOPK_EINVAL;
    if ((d != 64 && d != 128) || H_q / H_kv > 16 || T > 16 || (long long)B * H_kv > MAX_SEQ_GROUPS) return RETOPK_EUNSUPPORTED;
    return RETOPK_OK;
}

// SM count, and the kernels' opt-in to large shared memory; once per device.
constexpr int MAX_DEVICES = 64;
using EncodeTiled = CUresult (*)(CUtensorMap*, CUtensorMapDataType, cuuint32_t, void*, const cuuint64_t*, const cuuint64_t*, const cuuint32_t*,
                                 const cuuint32_t*, CUtensorMapInterleave, CUtensorMapSwizzle, CUtensorMapL2promotion, CUtensorMapFloatOOBfill);
struct DeviceSetup { bool ready; int num_sms; EncodeTiled encode; };
DeviceSetup g_setup[MAX_DEVICES];
std::mutex g_setup_mutex;

template <int DT, int D> bool opt_in() {
    return cudaFuncSetAttribute(attend_kernel<DT, D, false>, cudaFuncAttributeMaxDynamicSharedMemorySize, (int)sizeof(AttendSmem<D>)) == cudaSuccess &&
           cudaFuncSetAttribute(attend_kernel<DT, D, true>, cudaFuncAttributeMaxDynamicSharedMemorySize, (int)sizeof(AttendSmem<D>)) == cudaSuccess;
}
int device_setup(DeviceSetup* setup) {
    int dev = -1;
    if (cudaGetDevice(&dev) != cudaSuccess) { cudaGetLastError(); return RETOPK_ECUDA; }
    if (dev < 0 || dev >= MAX_DEVICES) return RETOPK_EUNSUPPORTED;
    std::lock_guard<std::mutex> lock(g_setup_mutex);
    DeviceSetup& st = g_setup[dev];
    if (!st.ready) {
        if (cudaDeviceGetAttribute(&st.num_sms, cudaDevAttrMultiProcessorCount, dev) != cudaSuccess ||
            !opt_in<TYPE_BF16, 64>() || !opt_in<TYPE_BF16, 128>() || !opt_in<TYPE_FP16, 64>() || !opt_in<TYPE_FP16, 128>()) {
            cudaGetLastError();
            return RETOPK_ECUDA;
        }
        void* fn = nullptr;
        cudaDriverEntryPointQueryResult found;
        if (cudaGetDriverEntryPointByVersion("cuTensorMapEncodeTiled", &fn, 12000, cudaEnableDefault, &found) != cudaSuccess ||
            found != cudaDriverEntryPointSuccess || !fn) {
            cudaGetLastError();
            return RETOPK_ECUDA;
        }
        st.encode = reinterpret_cast<EncodeTiled>(fn);
        if (st.num_sms > JOIN_THREADS) st.num_sms = JOIN_THREADS;        // (CTAs of the attention, each with a flag that a thread reads)
        st.ready = true;
    }
    *setup = st;
    return RETOPK_OK;
}

// Rows of a half of a part that belongs to one sequence with `rows` query rows: all copies of them.
int half_rows(int rows) { return rows < ATT_TILE ? rows * copies_of(rows) : ATT_TILE; }

// The workspace: where its parts begin, and its size.  `sequences`: entries that belong to one sequence or token,
// `rows` query rows each; `keys`: the most keys that an entry can have.
struct Workspace { int64_t entry, group_of, flags, shared_parts, own_parts, bytes, chunks; };
Workspace lay_out(int64_t sequences, int64_t rows, int64_t n_groups, int64_t group_rows, int64_t H_kv, int d, int64_t keys, int grid) {
    auto up = [](int64_t x) { return (x + 255) / 256 * 256; };
    const int64_t tiles = (keys + ATT_TILE - 1) / ATT_TILE, chunks = (tiles + ATT_CHUNK - 1) / ATT_CHUNK;
    const int64_t own = sequences * H_kv * chunks + grid;
    // groups of x rows in all have at most one row tile each more than x / 256
    const int64_t shared = n_groups ? H_kv * chunks * (n_groups + group_rows / (2 * ATT_TILE)) + grid : 0;
    Workspace w;
    w.entry = up(sizeof(AttendHeader));
    w.group_of = w.entry + up((n_groups + sequences) * (int64_t)sizeof(Entry));
    w.flags = w.group_of + up(sequences * 4);
    w.shared_parts = w.flags + up(grid * 4);
    w.own_parts = w.shared_parts + up(shared * 2 * half_floats(ATT_TILE, d) * 4);
    w.chunks = chunks;
    w.bytes = w.own_parts + up(own * 2 * half_floats(half_rows((int)rows), d) * 4);
    return w;
}

// What both attentions refuse alike, and their arguments.  cu, shared and blocks: what else is read, or nothing.
int check_attention(const retopk_pages_t* pages, int B, int T, int H_q, const int32_t* seq_lens, const Memory& cu_m, const Memory& shared_m,
                    const Memory& blocks_m, const void* q, int64_t q_stride, float scale, void* out, float* lse, void* workspace,
                    int64_t workspace_bytes, AttendArgs& a) {
    if (pages->format == RETOPK_PAGES_Q4 || !seq_lens || !out || !workspace || !isfinite(scale)) return RETOPK_EINVAL;
    const float scale_log2 = (float)((double)scale * 1.44269504088896340736);
    if (!isfinite(scale_log2)) return RETOPK_EINVAL;     // (0 times it would be no number)
    const int d = pages->d;
    if (!rows_ok(q, q_stride, H_q, d) || !aligned16(workspace) || !aligned16(out)) return RETOPK_EINVAL;
    memset(&a, 0, sizeof a);
    a.pg = device_pages(pages);
    if (a.pg.capacity > MAX_KEYS || pages->n_pages > 0x7fffff00ll / ((long long)pages->H_kv * pages->page_size)) return RETOPK_EUNSUPPORTED;
    const long long n = (long long)B * T;
    const Strided qi = {q, q_stride, H_q}, qo = {out, (long long)H_q * d, H_q};
    Memory pg[4];
    memory_of(pages, pg);
    const Memory q_m = memory_of(qi, n, d), out_m = memory_of(qo, n, d), lse_m = {lse, (uint64_t)n * H_q * 4}, ws_m = {workspace, (uint64_t)workspace_bytes};
    if (!in_place_or_apart(qi, qo, n, d) || !all_apart(out_m, pg) || !all_apart(lse_m, pg) || !all_apart(ws_m, pg)) return RETOPK_EINVAL;
    if (!all_apart(lse_m, {out_m, q_m, ws_m}) || !all_apart(ws_m, {out_m, q_m})) return RETOPK_EINVAL;
    const Memory lens_m = lens_memory(seq_lens, B), table_m = table_memory(pages, B);
    for (const Memory& written : {out_m, lse_m, ws_m})
        if (!all_apart(written, {lens_m, table_m, cu_m, shared_m, blocks_m})) return RETOPK_EINVAL;
    a.seq_lens = seq_lens;
    a.q = static_cast<const uint16_t*>(q);
    a.q_stride = q_stride;
    a.out = static_cast<uint16_t*>(out);
    a.lse = lse;
    a.scale_log2 = scale_log2;
    a.B = B; a.T = T; a.Hq = H_q; a.G = H_q / pages->H_kv;
    return RETOPK_OK;
}

template <int DT, int D> int launch_attention(AttendParams& p, int sequences, cudaStream_t s) {
    AttendArgs& a = p.a;
    // join_kernel has as many CTAs to a head as run at once (4 on an SM); one where outputs take the place of queries that it reads.
    const int rows = a.blocks ? a.G : a.T * a.G;
    int shares = 1;
    while ((a.T == 1 || a.out != a.q) && shares < JOIN_CTAS && 2ll * shares * a.pg.H_kv * sequences <= 4ll * a.grid) shares *= 2;
    a.join_wide = D / 4 / shares;
    a.join_splits = 1;
    while (2 * a.join_splits * rows * a.join_wide <= JOIN_THREADS) a.join_splits *= 2;
    a.per_row = 1.f / rows;
    a.per_work = 1.f / (rows * a.join_wide);
    a.per_G = 1.f / a.G;
    int rc = a.planned ? launch(plan_kernel, dim3(1), PLAN_THREADS, 0, s, a) : RETOPK_OK;
    if (rc != RETOPK_OK) return rc;
    rc = launch(a.few_rows ? attend_kernel<DT, D, true> : attend_kernel<DT, D, false>, dim3((unsigned)a.grid), ATT_THREADS, sizeof(AttendSmem<D>), s, p);
    if (rc != RETOPK_OK) return rc;
    // (tokens with blocks of their own can be 65536, one more than a grid has room for in any dimension but the first)
    return launch(join_kernel<DT, D>, dim3((unsigned)sequences, (unsigned)a.pg.H_kv, (unsigned)shares), JOIN_THREADS, 0, s, a);
}

// Rows of 64 channels each, `box` rows to a copy, into shared memory as the tensor cores' operands lie there.
bool encode_rows(EncodeTiled encode, CUtensorMap* map, const retopk_pages_t* pages, void* base, int64_t rows, int box) {
    const cuuint64_t dims[2] = {(cuuint64_t)pages->d, (cuuint64_t)rows}, strides[1] = {(cuuint64_t)pages->d * 2};
    const cuuint32_t boxes[2] = {64, (cuuint32_t)box}, steps[2] = {1, 1};
    const CUtensorMapDataType type = pages->format == RETOPK_PAGES_BF16 ? CU_TENSOR_MAP_DATA_TYPE_BFLOAT16 : CU_TENSOR_MAP_DATA_TYPE_FLOAT16;
    return encode(map, type, 2, base, dims, strides, boxes, steps, CU_TENSOR_MAP_INTERLEAVE_NONE, CU_TENSOR_MAP_SWIZZLE_128B,
                  CU_TENSOR_MAP_L2_PROMOTION_L2_256B, CU_TENSOR_MAP_FLOAT_OOB_FILL_NONE) == CUDA_SUCCESS;
}
int run_attention(AttendParams& p, const retopk_pages_t* pages, int sequences, int rows, const Workspace& w, const DeviceSetup& dev, void* workspace, cudaStream_t s) {
    AttendArgs& a = p.a;
    // Rows that lie together wherever a tile or a block begins: a block, in a cache without a table a tile, else the power of two in a
    // page's size.  (4 x 128K keys in pages of 128 rows 320 us, with copies of 64, 4, 2 and 1 row 329, 596, 1060 and 1992: pages
    // of an odd size cost up to six times as much.)
    int box = pages->block_table ? pages->page_size & -pages->page_size : ATT_TILE;
    if (a.blocks && box > a.block) box = a.block;
    if (box > ATT_TILE) box = ATT_TILE;
    const int64_t rows_in_all = pages->n_pages * pages->H_kv * pages->page_size;
    if (!encode_rows(dev.encode, &p.maps.k, pages, pages->k, rows_in_all, box) || !encode_rows(dev.encode, &p.maps.v, pages, pages->v, rows_in_all, box) ||
        !encode_rows(dev.encode, &p.maps.v_eight, pages, pages->v, rows_in_all, 8) ||
        !encode_rows(dev.encode, &p.maps.v_row, pages, pages->v, rows_in_all, 1))
        return RETOPK_ECUDA;
    a.box_shift = __builtin_ctz((unsigned)box);
    a.total_rows = (int)rows_in_all;
    char* ws = static_cast<char*>(workspace);
    a.head = reinterpret_cast<AttendHeader*>(ws);
    a.entry = reinterpret_cast<Entry*>(ws + w.entry);
    a.group_of = reinterpret_cast<int32_t*>(ws + w.group_of);
    a.flags = reinterpret_cast<int32_t*>(ws + w.flags);
    a.shared_parts = reinterpret_cast<float*>(ws + w.shared_parts);
    a.own_parts = reinterpret_cast<float*>(ws + w.own_parts);
    a.entries = a.n_groups + sequences;
    a.planned = a.entries >= ATT_THREADS;
    a.grid = dev.num_sms;
    a.max_chunks = (int)w.chunks;
    a.own_rows = half_rows(rows);
    a.few_rows = (a.n_groups > 0 ? (long long)a.B : 1) * rows <= ATT_FEW;
    if (pages->format == RETOPK_PAGES_BF16)
        return pages->d == 128 ? launch_attention<TYPE_BF16, 128>(p, sequences, s) : launch_attention<TYPE_BF16, 64>(p, sequences, s);
    return pages->d == 128 ? launch_attention<TYPE_FP16, 128>(p, sequences, s) : launch_attention<TYPE_FP16, 64>(p, sequences, s);
}

int shared_workspace(int B, int n_groups, int T, int H_q, int H_kv, int d, int64_t max_keys, Workspace* w, DeviceSetup* dev) {
    int rc = check_shape(B, T, H_q, H_kv, d);
    if (rc != RETOPK_OK) return rc;
    if (n_groups < 0 || n_groups > B || max_keys < 1) return RETOPK_EINVAL;
    if (max_keys > MAX_KEYS) return RETOPK_EUNSUPPORTED;
    rc = device_setup(dev);
    if (rc != RETOPK_OK) return rc;
    const int rows = T * (H_q / H_kv);
    *w = lay_out(B, rows, n_groups, (int64_t)B * rows, H_kv, d, max_keys, dev->num_sms);
    return RETOPK_OK;
}
int block_workspace(int B, int T, int H_q, int H_kv, int d, int64_t max_keys, Workspace* w, DeviceSetup* dev) {
    int rc = check_shape(B, T, H_q, H_kv, d);
    if (rc != RETOPK_OK) return rc;
    if (max_keys < 1) return RETOPK_EINVAL;
    if (max_keys > MAX_KEYS + 127) return RETOPK_EUNSUPPORTED;
    rc = device_setup(dev);
    if (rc != RETOPK_OK) return rc;
    *w = lay_out((int64_t)B * T, H_q / H_kv, 0, 0, H_kv, d, max_keys, dev->num_sms);
    return RETOPK_OK;
}

template <class Args, class F>
int by_type(const retopk_pages_t* p, F bf128, F bf64, F fp128, F fp64, dim3 grid, unsigned threads, cudaStream_t s, const Args& a) {
    const bool bf = p->format == RETOPK_PAGES_BF16, wide = p->d == 128;
    return launch(bf ? (wide ? bf128 : bf64) : (wide ? fp128 : fp64), grid, threads, 0, s, a);
}

}  // namespace

extern "C" {

int64_t retopk_shared_attention_workspace(int B, int n_groups, int T, int H_q, int H_kv, int d, int64_t max_keys) {
    Workspace w;
    DeviceSetup dev;
    const int rc = shared_workspace(B, n_groups, T, H_q, H_kv, d, max_keys, &w, &dev);
    return rc == RETOPK_OK ? w.bytes : rc;
}

int retopk_shared_attention(const retopk_pages_t* pages, int B, int T, int H_q, const int32_t* seq_lens, int n_groups,
                            const int32_t* cu_groups, const int32_t* shared_lens, const void* q, int64_t q_stride, float scale,
                            void* out, float* lse, void* workspace, int64_t workspace_bytes, void* stream) {
    int rc = check_pages(pages, B);
    if (rc != RETOPK_OK) return rc;
    rc = check_shape(B, T, H_q, pages->H_kv, pages->d);
    if (rc != RETOPK_OK) return rc;
    if (n_groups < 0 || n_groups > B || (n_groups > 0 && (!cu_groups || !shared_lens))) return RETOPK_EINVAL;
    AttendParams p;
    AttendArgs& a = p.a;
    rc = check_attention(pages, B, T, H_q, seq_lens, {n_groups > 0 ? cu_groups : nullptr, (n_groups + 1ull) * 4},
                         {n_groups > 0 ? shared_lens : nullptr, n_groups * 4ull}, {nullptr, 0}, q, q_stride, scale, out, lse, workspace, workspace_bytes, a);
    if (rc != RETOPK_OK) return rc;
    if (workspace_bytes < 4096) return RETOPK_EINVAL;    // (refused without a device too)
    Workspace w;
    DeviceSetup dev;
    rc = shared_workspace(B, n_groups, T, H_q, pages->H_kv, pages->d, a.pg.capacity, &w, &dev);
    if (rc != RETOPK_OK) return rc;
    if (workspace_bytes < w.bytes) return RETOPK_EINVAL;
    a.n_groups = n_groups;
    a.cu = cu_groups;
    a.shared_lens = shared_lens;
    return run_attention(p, pages, B, T * a.G, w, dev, workspace, static_cast<cudaStream_t>(stream));
}

int retopk_block_update(const retopk_pages_t* pages, int block, void* bounds, int B, const int32_t* seq_lens, int64_t n_new, void* stream) {
    const int rc = check_blocks(pages, B, block, bounds);
    if (rc != RETOPK_OK) return rc;
    if (!seq_lens || n_new < 0) return RETOPK_EINVAL;
    if (B > 65535 || pages->H_kv > 65535) return RETOPK_EUNSUPPORTED;
    if (n_new == 0) return RETOPK_OK;
    if (!all_apart(bounds_memory(pages, block, bounds), {lens_memory(seq_lens, B), table_memory(pages, B)})) return RETOPK_EINVAL;
    BoundsArgs a;
    memset(&a, 0, sizeof a);
    a.pg = device_pages(pages);
    a.block = block;
    a.shift = __builtin_ctz((unsigned)block);
    a.seq_lens = seq_lens;
    a.n_new = n_new;
    a.bounds = static_cast<uint16_t*>(bounds);
    // whole blocks that n_new rows can touch
    const long long all = a.pg.capacity / block, some = n_new >= a.pg.capacity ? all : (n_new + block - 2) / block + 1;
    const long long most = some < all ? some : all;
    if (most == 0) return RETOPK_OK;
    const dim3 grid((unsigned)((most + BOUNDS_WARPS - 1) / BOUNDS_WARPS), (unsigned)pages->H_kv, (unsigned)B);
    return by_type(pages, bounds_kernel<TYPE_BF16, 128>, bounds_kernel<TYPE_BF16, 64>, bounds_kernel<TYPE_FP16, 128>,
                   bounds_kernel<TYPE_FP16, 64>, grid, BOUNDS_THREADS, static_cast<cudaStream_t>(stream), a);
}

int64_t retopk_block_select_workspace(int B, int T, int H_q, int H_kv, int d, int64_t max_blocks) {
    const int rc = check_shape(B, T, H_q, H_kv, d);
    if (rc != RETOPK_OK) return rc;
    if (max_blocks < 1) return RETOPK_EINVAL;
    if (max_blocks > MAX_KEYS) return RETOPK_EUNSUPPORTED;
    return (int64_t)B * T * H_kv * max_blocks * 8;
}

int retopk_block_select(const retopk_pages_t* pages, int block, const void* bounds, int B, int T, int H_q, const int32_t* seq_lens,
                        const void* q, int64_t q_stride, int keep, int first, int last, int32_t* blocks, void* workspace,
                        int64_t workspace_bytes, void* stream) {
    int rc = check_blocks(pages, B, block, bounds);
    if (rc != RETOPK_OK) return rc;
    if (!seq_lens || !blocks || !workspace || keep < 1 || first < 0 || last < 1 || first > keep - last) return RETOPK_EINVAL;
    SelectArgs a;
    memset(&a, 0, sizeof a);
    a.pg = device_pages(pages);
    if (a.pg.capacity > MAX_KEYS) return RETOPK_EUNSUPPORTED;
    a.max_blocks = (a.pg.capacity + block - 1) / block;
    const int64_t need = retopk_block_select_workspace(B, T, H_q, pages->H_kv, pages->d, a.max_blocks);
    if (need < 0) return (int)need;
    if (!rows_ok(q, q_stride, H_q, pages->d) || !aligned16(workspace) || workspace_bytes < need) return RETOPK_EINVAL;
    if (keep > MAX_KEYS) return RETOPK_EUNSUPPORTED;
    const Memory q_m = memory_of(Strided{q, q_stride, H_q}, (long long)B * T, pages->d), ws_m = {workspace, (uint64_t)workspace_bytes};
    const Memory bounds_m = bounds_memory(pages, block, bounds), blocks_m = {blocks, (uint64_t)B * T * pages->H_kv * keep * 4};
    if (!all_apart(blocks_m, {q_m, ws_m, bounds_m}) || !all_apart(ws_m, {q_m, bounds_m})) return RETOPK_EINVAL;
    const Memory lens_m = lens_memory(seq_lens, B), table_m = table_memory(pages, B);
    if (!all_apart(blocks_m, {lens_m, table_m}) || !all_apart(ws_m, {lens_m, table_m})) return RETOPK_EINVAL;
    a.block = block; a.shift = __builtin_ctz((unsigned)block); a.per_G = 1.f / (float)(H_q / pages->H_kv); a.scored = a.max_blocks > keep;
    a.T = T; a.Hq = H_q; a.G = H_q / pages->H_kv; a.keep = keep; a.first = first; a.last = last;
    a.seq_lens = seq_lens;
    a.bounds = static_cast<const uint16_t*>(bounds);
    a.q = static_cast<const uint16_t*>(q);
    a.q_stride = q_stride;
    a.scores = static_cast<float2*>(workspace);
    a.blocks = blocks;
    cudaStream_t s = static_cast<cudaStream_t>(stream);
    if (a.scored) {
        constexpr int PER_CTA = SCORE_WARPS * SCORE_ROWS;
        const dim3 grid((unsigned)((a.max_blocks + PER_CTA - 1) / PER_CTA), (unsigned)pages->H_kv, (unsigned)B);
        rc = by_type(pages, score_kernel<TYPE_BF16, 128>, score_kernel<TYPE_BF16, 64>, score_kernel<TYPE_FP16, 128>,
                     score_kernel<TYPE_FP16, 64>, grid, SCORE_THREADS, s, a);
        if (rc != RETOPK_OK) return rc;
    }
    return by_type(pages, pick_kernel<TYPE_BF16, 128>, pick_kernel<TYPE_BF16, 64>, pick_kernel<TYPE_FP16, 128>, pick_kernel<TYPE_FP16, 64>,
                   dim3((unsigned)pages->H_kv, (unsigned)T, (unsigned)B), PICK_THREADS, s, a);
}

int64_t retopk_block_attention_workspace(int B, int T, int H_q, int H_kv, int d, int keep, int block) {
    const int rc0 = check_shape(B, T, H_q, H_kv, d);
    if (rc0 != RETOPK_OK) return rc0;
    if (keep < 1 || block < 1) return RETOPK_EINVAL;
    if (keep > MAX_KEYS || block > 128) return RETOPK_EUNSUPPORTED;
    const int64_t keys = (int64_t)keep * block, most = MAX_KEYS + block - 1;
    Workspace w;
    DeviceSetup dev;
    const int rc = block_workspace(B, T, H_q, H_kv, d, keys < most ? keys : most, &w, &dev);
    return rc == RETOPK_OK ? w.bytes : rc;
}

int retopk_block_attention(const retopk_pages_t* pages, int block, int B, int T, int H_q, const int32_t* seq_lens, int keep,
                           const int32_t* blocks, const void* q, int64_t q_stride, float scale, void* out, float* lse,
                           void* workspace, int64_t workspace_bytes, void* stream) {
    int rc = check_pages(pages, B);
    if (rc != RETOPK_OK) return rc;
    if (block != 16 && block != 32 && block != 64 && block != 128) return RETOPK_EUNSUPPORTED;
    rc = check_shape(B, T, H_q, pages->H_kv, pages->d);
    if (rc != RETOPK_OK) return rc;
    if (keep < 1 || !blocks || pages->page_size % block != 0) return RETOPK_EINVAL;
    if (keep > MAX_KEYS) return RETOPK_EUNSUPPORTED;
    AttendParams p;
    AttendArgs& a = p.a;
    rc = check_attention(pages, B, T, H_q, seq_lens, {nullptr, 0}, {nullptr, 0}, {blocks, (uint64_t)B * T * pages->H_kv * keep * 4}, q, q_stride,
                         scale, out, lse, workspace, workspace_bytes, a);
    if (rc != RETOPK_OK) return rc;
    if (workspace_bytes < 4096) return RETOPK_EINVAL;
    const int64_t keys = (int64_t)keep * block, most = MAX_KEYS + block - 1;
    Workspace w;
    DeviceSetup dev;
    rc = block_workspace(B, T, H_q, pages->H_kv, pages->d, keys < most ? keys : most, &w, &dev);
    if (rc != RETOPK_OK) return rc;
    if (workspace_bytes < w.bytes) return RETOPK_EINVAL;
    a.blocks = blocks;
    a.keep = keep;
    a.block = block;
    a.block_shift = __builtin_ctz((unsigned)block);
    return run_attention(p, pages, B * T, a.G, w, dev, workspace, static_cast<cudaStream_t>(stream));
}

}  // extern "C"
