// The 4-bit sequence cache as its kernels see it.
#pragma once

#include <climits>

#include "aif_internal.h"
#include "aif_mx4.cuh"

namespace aif {

// Buffers and sizes of a cache, and where row (page, head, row) of it lies.
struct Cache4 {
    int32_t d, heads, page_shift, n_pages, n_seqs, max_pages;
    uint8_t *codes[2], *scales[2];   // keys, values ([1] of a shared cache: the keys')
    int32_t *table, *lengths, *refs, *free_pages, *n_free;
    int32_t *scratch;
    uint32_t *status;

    __host__ __device__ int page_rows() const { return 1 << page_shift; }
    __device__ size_t row(int page, int head, int row_in_page) const { return (((size_t)page * heads + head) << page_shift) + row_in_page; }
    __device__ int pages_of(int length) const { return (int)(((int64_t)length + page_rows() - 1) >> page_shift); }
    __device__ int longest() const { return max_pages << page_shift; }
    __device__ bool holds(int page) const { return page >= 0 && page < n_pages; }
};

inline Cache4 cache4_of(const aif_cache4 *c)
{
    Cache4 k{};
    k.d = c->d, k.heads = c->heads, k.page_shift = __builtin_ctz((unsigned)c->page_rows), k.n_pages = c->n_pages, k.n_seqs = c->n_seqs, k.max_pages = c->max_pages;
    k.codes[0] = c->k_codes, k.scales[0] = c->k_scales;
    k.codes[1] = c->shared ? c->k_codes : c->v_codes, k.scales[1] = c->shared ? c->k_scales : c->v_scales;
    k.table = c->table, k.lengths = c->lengths, k.refs = c->refs, k.free_pages = c->free_pages, k.n_free = c->n_free;
    k.scratch = c->scratch, k.status = c->status;
    return k;
}

// 32-bit division by a number that the host knows: a multiplication.
struct FastDiv {
    uint32_t by, mul, shift;   // x / by = (x mul) >> (32 + shift)
    static FastDiv of(uint32_t by)
    {
        FastDiv f{by, 0u, 0u};
        while ((1u << f.shift) < by) ++f.shift;
        f.mul = (uint32_t)(((uint64_t)1 << 32) * ((1ull << f.shift) - by) / by + 1);   // round-up multiplier less 2^32
        return f;
    }
    __device__ uint32_t div(uint32_t x) const { return (uint32_t)(((uint64_t)__umulhi(x, mul) + x) >> shift); }
};

int cache4_check(const aif_cache4 *c);   // AIF_OK, AIF_ERR_ARG or AIF_ERR_SHAPE
int cache4_failed(cudaError_t e, const char *what);

}  // namespace aif
