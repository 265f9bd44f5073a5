// Host helpers that the calls around the KV cache share: argument checks, overlaps, launches.
#pragma once
#include <string.h>

#include "../../include/retopk.h"
#include "retopk_cache.cuh"

namespace retopk_cache {

constexpr long long MAX_KEYS = 1048576;  // keys of one sequence in an attention, as in retopk_create
constexpr int MAX_SEQ_GROUPS = 4096;     // B * H_kv, as in retopk_create

inline bool aligned16(const void* p) { return (reinterpret_cast<uintptr_t>(p) & 15u) == 0; }
inline bool bad_half_type(int dtype) { return dtype != RETOPK_BF16 && dtype != RETOPK_FP16; }

// A token-major tensor [n, heads, d] with a stride of its own.
inline bool rows_ok(const void* p, long long stride, int heads, int d) {
    return p && aligned16(p) && heads >= 1 && stride % 8 == 0 && stride >= (long long)heads * d;
}
// Whether two such tensors of n tokens share no element: apart altogether, or with one stride and side by
// side within it (slices of one projection's output).
struct Strided { const void* p; long long stride; int heads; };
inline bool rows_apart(const Strided& x, const Strided& y, long long n, int d) {
    const uintptr_t x0 = reinterpret_cast<uintptr_t>(x.p), y0 = reinterpret_cast<uintptr_t>(y.p);
    const uintptr_t wx = (uintptr_t)x.heads * d * 2, wy = (uintptr_t)y.heads * d * 2;
    if (x0 + (uintptr_t)(n - 1) * x.stride * 2 + wx <= y0 || y0 + (uintptr_t)(n - 1) * y.stride * 2 + wy <= x0) return true;
    if (x.stride != y.stride) return false;
    const uintptr_t step = (uintptr_t)x.stride * 2, off = y0 >= x0 ? (y0 - x0) % step : (step - (x0 - y0) % step) % step;
    return off >= wx && off + wy <= step;
}
// An output may be its own input exactly, or must not touch it.
inline bool in_place_or_apart(const Strided& in, const Strided& out, long long n, int d) {
    return (in.p == out.p && in.stride == out.stride) || rows_apart(in, out, n, d);
}

// A stretch of memory; and whether one that is written keeps clear of others.
struct Memory { const void* p; uint64_t bytes; };
inline bool apart(const Memory& x, const Memory& y) {
    const uintptr_t x0 = reinterpret_cast<uintptr_t>(x.p), y0 = reinterpret_cast<uintptr_t>(y.p);
    return !x.p || !y.p || x0 + x.bytes <= y0 || y0 + y.bytes <= x0;
}
template <size_t N> bool all_apart(const Memory& x, const Memory (&others)[N]) {
    for (const Memory& y : others)
        if (!apart(x, y)) return false;
    return true;
}
inline Memory memory_of(const Strided& x, long long n, int d) { return {x.p, ((uint64_t)(n - 1) * x.stride + (uint64_t)x.heads * d) * 2}; }
inline void memory_of(const retopk_pages_t* p, Memory (&m)[4]) {
    const bool q4 = p->format == RETOPK_PAGES_Q4;
    const uint64_t rows = (uint64_t)p->n_pages * p->H_kv * p->page_size;
    m[0] = {p->k, rows * (q4 ? p->d / 2 : p->d * 2)};
    m[1] = {p->v, m[0].bytes};
    m[2] = {q4 ? p->k_scale : nullptr, rows * (p->d / GROUP * 4)};
    m[3] = {q4 ? p->v_scale : nullptr, m[2].bytes};
}

inline int check_pages(const retopk_pages_t* p, int B) {
    if (!p || B < 1) return RETOPK_EINVAL;
    if (p->format < RETOPK_PAGES_BF16 || p->format > RETOPK_PAGES_Q4) return RETOPK_EINVAL;
    if (p->H_kv < 1 || p->page_size < 1 || p->n_pages < 1 || !p->k || !p->v) return RETOPK_EINVAL;
    if (p->d != 64 && p->d != 128) return RETOPK_EUNSUPPORTED;
    if (!aligned16(p->k) || !aligned16(p->v)) return RETOPK_EINVAL;
    if (p->format == RETOPK_PAGES_Q4) {
        if (!p->k_scale || !p->v_scale || !aligned16(p->k_scale) || !aligned16(p->v_scale)) return RETOPK_EINVAL;
        if (p->page_size % Q4_TILE != 0) return RETOPK_EINVAL;
    }
    if (p->block_table) {
        if (p->max_pages < 1 || p->max_pages > 2147483647ll / p->page_size) return RETOPK_EINVAL;
    } else if (p->n_pages < B) {
        return RETOPK_EINVAL;
    }
    return RETOPK_OK;
}

inline Pages device_pages(const retopk_pages_t* p) {
    Pages g;
    g.k = static_cast<unsigned char*>(p->k);
    g.v = static_cast<unsigned char*>(p->v);
    g.ks = static_cast<unsigned char*>(p->k_scale);
    g.vs = static_cast<unsigned char*>(p->v_scale);
    g.table = p->block_table;
    g.n_pages = p->n_pages;
    g.max_pages = p->block_table ? p->max_pages : 1;
    g.capacity = g.max_pages * p->page_size;
    g.H_kv = p->H_kv;
    g.page_size = p->page_size;
    g.page_shift = (p->page_size & (p->page_size - 1)) == 0 ? __builtin_ctz((unsigned)p->page_size) : -1;
    return g;
}

// What a call reads of the sequences: their lengths and their rows of the block table.
inline Memory lens_memory(const int32_t* seq_lens, int B) { return {seq_lens, (uint64_t)B * 4}; }
inline Memory table_memory(const retopk_pages_t* p, int B) { return {p->block_table, (uint64_t)B * p->max_pages * 4}; }

// Bounds of blocks of keys, and the 16-bit pages that they belong to.
inline Memory bounds_memory(const retopk_pages_t* p, int block, const void* bounds) {
    return {bounds, (uint64_t)p->n_pages * p->H_kv * (p->page_size / block) * p->d * 4};
}
inline int check_blocks(const retopk_pages_t* p, int B, int block, const void* bounds) {
    const int rc = check_pages(p, B);
    if (rc != RETOPK_OK) return rc;
    if (p->format == RETOPK_PAGES_Q4) return RETOPK_EINVAL;
    if (block != 16 && block != 32 && block != 64 && block != 128) return RETOPK_EUNSUPPORTED;
    if (p->page_size % block != 0 || !bounds || !aligned16(bounds)) return RETOPK_EINVAL;
    Memory pg[4];
    memory_of(p, pg);
    return all_apart(bounds_memory(p, block, bounds), pg) ? RETOPK_OK : RETOPK_EINVAL;
}

// Launch with programmatic stream serialisation: the kernel may be set up while its predecessor in
// the stream still runs; it waits (pdl_wait) before it touches memory.
template <class Args>
int launch(void (*kernel)(Args), dim3 grid, unsigned threads, size_t smem, cudaStream_t s, const Args& a) {
    cudaLaunchConfig_t cfg;
    memset(&cfg, 0, sizeof cfg);
    cfg.gridDim = grid;
    cfg.blockDim = dim3(threads);
    cfg.dynamicSmemBytes = smem;
    cfg.stream = s;
    cudaLaunchAttribute attr;
    attr.id = cudaLaunchAttributeProgrammaticStreamSerialization;
    attr.val.programmaticStreamSerializationAllowed = 1;
    cfg.attrs = &attr;
    cfg.numAttrs = 1;
    if (cudaLaunchKernelEx(&cfg, kernel, a) != cudaSuccess) { cudaGetLastError(); return RETOPK_ECUDA; }
    return RETOPK_OK;
}

}  // namespace retopk_cache
