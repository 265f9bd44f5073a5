// Host side of the page calls: argument checks, launches, C interface.
#include "retopk_pool.cuh"

#include "retopk_cache_host.cuh"

using namespace retopk_cache;

namespace {

constexpr int64_t MAX_POOL_PAGES = 1 << 20;
constexpr int64_t MAX_ROWS = 65535;      // sequences of a table

// The pool, a table over it, and what both are made of.
int check_pool(const retopk_pool_t* pool, int B, const int32_t* lens, const int32_t* table, int64_t max_pages, Memory (&m)[4]) {
    if (!pool || !pool->refs || !pool->scratch || pool->n_pages < 1 || pool->page_size < 1) return RETOPK_EINVAL;
    if (B < 1 || !lens || !table || max_pages < 1 || max_pages > 2147483647ll / pool->page_size) return RETOPK_EINVAL;
    if (pool->n_pages > MAX_POOL_PAGES || B > MAX_ROWS) return RETOPK_EUNSUPPORTED;
    m[0] = {pool->refs, (uint64_t)pool->n_pages * 4};
    m[1] = {pool->scratch, (uint64_t)(pool->n_pages + RETOPK_POOL_SCRATCH) * 4};
    m[2] = {table, (uint64_t)B * max_pages * 4};
    m[3] = {lens, (uint64_t)B * 4};
    for (int i = 0; i < 4; ++i)
        for (int j = i + 1; j < 4; ++j)
            if (!apart(m[i], m[j])) return RETOPK_EINVAL;
    return RETOPK_OK;
}
PoolArgs pool_args(const retopk_pool_t* pool, int B, const int32_t* lens, int32_t* table, int64_t max_pages) {
    PoolArgs a;
    memset(&a, 0, sizeof a);
    a.refs = pool->refs;
    a.scratch = pool->scratch;
    a.n_pages = pool->n_pages;
    a.page_size = pool->page_size;
    a.table = table;
    a.max_pages = max_pages;
    a.capacity = max_pages * pool->page_size;
    a.B = B;
    a.lens = const_cast<int32_t*>(lens);
    return a;
}

int launch_copy(CopyArgs& a, int64_t n, const int32_t* src, const int32_t* dst, const int32_t* rows, cudaStream_t s) {
    int dev = 0, num_sms = 0;
    if (cudaGetDevice(&dev) != cudaSuccess || cudaDeviceGetAttribute(&num_sms, cudaDevAttrMultiProcessorCount, dev) != cudaSuccess) {
        cudaGetLastError();
        return RETOPK_ECUDA;
    }
    a.n = n;
    a.src = src;
    a.dst = dst;
    a.rows = rows;
    long long pair = 0;
    for (int t = 0; t < a.tensors; ++t) pair += (long long)a.H * a.page_rows * a.t[t].row_bytes;
    // about 8 KB of a pair to a CTA where there are few pairs; many pairs are shared by four each, so that the
    // CTAs end at about the same time
    const long long ctas = 8ll * num_sms, most = pair / 8192 > 1 ? pair / 8192 : 1;
    long long parts = (2 * ctas + n - 1) / n;
    parts = parts < 4 ? 4 : parts;
    a.parts = (int)(parts < most ? parts : most);
    a.per_part = ~0ull / (unsigned)a.parts + 1;
    const long long lines = n < (ctas + a.parts - 1) / a.parts ? n : (ctas + a.parts - 1) / a.parts;
    return launch(copy_pages_kernel, dim3((unsigned)(lines * a.parts)), COPY_THREADS, 0, s, a);
}

}  // namespace

extern "C" {

int retopk_pool_reserve(const retopk_pool_t* pool, int B, const int32_t* old_lens, const int32_t* new_lens, int32_t* block_table,
                        int64_t max_pages, void* stream) {
    Memory m[4];
    const int rc = check_pool(pool, B, old_lens, block_table, max_pages, m);
    if (rc != RETOPK_OK) return rc;
    const Memory lens = {new_lens, (uint64_t)B * 4};
    if (!new_lens || !apart(lens, m[0]) || !apart(lens, m[1]) || !apart(lens, m[2])) return RETOPK_EINVAL;
    PoolArgs a = pool_args(pool, B, old_lens, block_table, max_pages);
    a.other = new_lens;
    return launch(reserve_kernel, dim3(1), POOL_THREADS, 0, static_cast<cudaStream_t>(stream), a);
}

int retopk_pool_fork(const retopk_pool_t* pool, int B, int32_t* seq_lens, int32_t* block_table, int64_t max_pages, int n,
                     const int32_t* parents, const int32_t* children, int32_t* src, int32_t* dst, int32_t* rows, void* stream) {
    Memory m[4];
    const int rc = check_pool(pool, B, seq_lens, block_table, max_pages, m);
    if (rc != RETOPK_OK) return rc;
    if (n < 0) return RETOPK_EINVAL;
    if (n > MAX_ROWS) return RETOPK_EUNSUPPORTED;
    if (n == 0) return RETOPK_OK;
    if (!parents || !children || !src || !dst || !rows) return RETOPK_EINVAL;
    const uint64_t bytes = (uint64_t)n * 4;
    const Memory lists[5] = {{src, bytes}, {dst, bytes}, {rows, bytes}, {parents, bytes}, {children, bytes}};
    for (int i = 0; i < 5; ++i) {
        if (!all_apart(lists[i], m)) return RETOPK_EINVAL;
        for (int j = 0; j < 3; ++j)
            if (j != i && !apart(lists[i], lists[j])) return RETOPK_EINVAL;
    }
    PoolArgs a = pool_args(pool, B, seq_lens, block_table, max_pages);
    a.n = n;
    a.other = parents;
    a.children = children;
    a.src = src;
    a.dst = dst;
    a.rows = rows;
    return launch(fork_kernel, dim3((unsigned)n + 1), FORK_THREADS, 0, static_cast<cudaStream_t>(stream), a);
}

int retopk_pool_free(const retopk_pool_t* pool, int B, int32_t* seq_lens, const int32_t* block_table, int64_t max_pages, int n,
                     const int32_t* rows, void* stream) {
    Memory m[4];
    const int rc = check_pool(pool, B, seq_lens, block_table, max_pages, m);
    if (rc != RETOPK_OK) return rc;
    if (n < 0 || (!rows && n != B) || !all_apart({rows, (uint64_t)n * 4}, m)) return RETOPK_EINVAL;
    if (n == 0) return RETOPK_OK;
    PoolArgs a = pool_args(pool, B, seq_lens, const_cast<int32_t*>(block_table), max_pages);
    a.n = n;
    a.other = rows;
    return launch(free_kernel, dim3((unsigned)n), FORK_THREADS, 0, static_cast<cudaStream_t>(stream), a);
}

int retopk_pool_compact(const retopk_pool_t* pool, int B, const int32_t* seq_lens, int32_t* block_table, int64_t max_pages,
                        int32_t* src, int32_t* dst, void* stream) {
    Memory m[4];
    int rc = check_pool(pool, B, seq_lens, block_table, max_pages, m);
    if (rc != RETOPK_OK) return rc;
    const uint64_t bytes = (uint64_t)(pool->n_pages / 2) * 4;
    if (pool->n_pages < 2) return RETOPK_OK;
    if (!src || !dst || !all_apart({src, bytes}, m) || !all_apart({dst, bytes}, m) || !apart({src, bytes}, {dst, bytes})) return RETOPK_EINVAL;
    PoolArgs a = pool_args(pool, B, seq_lens, block_table, max_pages);
    a.src = src;
    a.dst = dst;
    a.pairs = pool->n_pages / 2;
    cudaStream_t s = static_cast<cudaStream_t>(stream);
    rc = launch(compact_kernel, dim3(1), POOL_THREADS, 0, s, a);
    if (rc != RETOPK_OK) return rc;
    return launch(renumber_kernel, dim3((unsigned)B), FORK_THREADS, 0, s, a);
}

int retopk_pages_copy(const retopk_pages_t* pages, int64_t n, const int32_t* src, const int32_t* dst, const int32_t* rows, void* stream) {
    const int rc = check_pages(pages, 1);
    if (rc != RETOPK_OK) return rc;
    if (n < 0) return RETOPK_EINVAL;
    if (n > MAX_POOL_PAGES) return RETOPK_EUNSUPPORTED;
    if (n == 0) return RETOPK_OK;
    Memory m[4];
    memory_of(pages, m);
    for (int i = 0; i < 4; ++i)
        for (int j = i + 1; j < 4; ++j)
            if (!apart(m[i], m[j])) return RETOPK_EINVAL;
    const uint64_t bytes = (uint64_t)n * 4;
    if (!src || !dst || !all_apart({src, bytes}, m) || !all_apart({dst, bytes}, m) || !all_apart({rows, bytes}, m)) return RETOPK_EINVAL;
    const bool q4 = pages->format == RETOPK_PAGES_Q4;
    CopyArgs a;
    memset(&a, 0, sizeof a);
    const int row = q4 ? pages->d / 2 : pages->d * 2, scale = pages->d / GROUP * 4;
    a.t[0] = {static_cast<unsigned char*>(pages->k), row};
    a.t[1] = {static_cast<unsigned char*>(pages->v), row};
    a.t[2] = {static_cast<unsigned char*>(pages->k_scale), scale};
    a.t[3] = {static_cast<unsigned char*>(pages->v_scale), scale};
    a.tensors = q4 ? 4 : 2;
    a.H = pages->H_kv;
    a.page_rows = pages->page_size;
    a.n_pages = pages->n_pages;
    return launch_copy(a, n, src, dst, rows, static_cast<cudaStream_t>(stream));
}

int retopk_block_copy(const retopk_pages_t* pages, int block, void* bounds, int64_t n, const int32_t* src, const int32_t* dst, void* stream) {
    const int rc = check_blocks(pages, 1, block, bounds);
    if (rc != RETOPK_OK) return rc;
    if (n < 0) return RETOPK_EINVAL;
    if (n > MAX_POOL_PAGES) return RETOPK_EUNSUPPORTED;
    if (n == 0) return RETOPK_OK;
    const Memory b = bounds_memory(pages, block, bounds);
    if (!src || !dst || !apart({src, (uint64_t)n * 4}, b) || !apart({dst, (uint64_t)n * 4}, b)) return RETOPK_EINVAL;
    CopyArgs a;
    memset(&a, 0, sizeof a);
    a.t[0] = {static_cast<unsigned char*>(bounds), pages->d * 4};
    a.tensors = 1;
    a.H = pages->H_kv;
    a.page_rows = pages->page_size / block;
    a.n_pages = pages->n_pages;
    return launch_copy(a, n, src, dst, nullptr, static_cast<cudaStream_t>(stream));
}

}  // extern "C"
