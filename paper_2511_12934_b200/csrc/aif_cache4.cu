// Books and rows of the 4-bit sequence cache: appending, sharing, copying, moving, freeing and reading pages.
//
// A call that changes the books is one small kernel over the listed sequences (k_books) and, where rows or pages move, one more that
// moves them, bound by HBM.  The books are kept by one CTA, or for many pages one cluster of CTAs: its phases hand over through
// barriers, a matter of a microsecond, where separate launches would cost two or three each.  Nothing depends on the order of atomics: pages are
// handed out and taken back by position in the call (prefix sums), so the same calls leave the same books.
// Fork of 48 sequences 9.3 us (phases of one CTA, each some loads that need one another), freeing 3135 pages 21 us (30 thousand scattered accesses of one multiprocessor),
// append of 200 thousand rows (d = 128) with the books of append and free 39 us in bf16, 47 in fp32 (13 of them books of no rows); read of as many 18 and 32 us;
// copy and free of 100 sequences of 2000 rows 29 us, fork and free 23; compaction of those 14.5.
#include <algorithm>
#include <cstdio>

#include "aif_cache4.cuh"
#include "aif_span.h"
#include "aif_tc_ptx.cuh"

namespace aif {
namespace {

enum BooksOp { kFree, kFork, kCopy, kAppend };

// Scratch of a cache, in 32-bit words.  The marks are INT_MAX between calls.
struct Scratch {
    int32_t *mark_page;   // [n_pages] smallest position in the call that gave the page up
    int32_t *mark_seq;    // [n_seqs] first entry that names the sequence
    int32_t *map;         // [n_pages] rank of a page in use within its block (aif_cache4_compact)
    int32_t *count;       // [n_seqs] pages that an entry gives up or needs
    int32_t *before;      // [n_seqs] the same of the entries before it
    int32_t *info;        // [n_seqs] for the kernel that moves rows: first new row (append), pages (copy); -1: undone
    int32_t *from, *to;   // [n_seqs] page to copy before rows are appended, or -1
    int32_t *misc;        // [8]
    int32_t *block_sum;   // [n_pages / kMapBlock + 1]
};
constexpr int kMapBlock = 1024;

__host__ __device__ inline int64_t scratch_ints(int n_pages, int n_seqs) { return 2ll * n_pages + 6ll * n_seqs + 8 + n_pages / kMapBlock + 1; }
__device__ __forceinline__ Scratch scratch_of(const Cache4 &c)
{
    Scratch s;
    s.mark_page = c.scratch, s.mark_seq = s.mark_page + c.n_pages, s.map = s.mark_seq + c.n_seqs, s.count = s.map + c.n_pages;
    s.before = s.count + c.n_seqs, s.info = s.before + c.n_seqs, s.from = s.info + c.n_seqs, s.to = s.from + c.n_seqs, s.misc = s.to + c.n_seqs;
    s.block_sum = s.misc + 8;
    return s;
}

__device__ __forceinline__ int ld(const int32_t *p) { return __ldcg(p); }   // what other CTAs of the cluster wrote: from L2
__device__ __forceinline__ void st(int32_t *p, int v) { __stcg(p, v); }

__device__ __forceinline__ void books_sync()
{
    __threadfence();
    cluster_sync();
}

constexpr int kBookThreads = 512;

// before[i] = count[0] + .. + count[i - 1] for i < n, and the total.  One CTA.
__device__ int scan_counts(const int32_t *count, int32_t *before, int n, int32_t *warp_sum)
{
    const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5;
    int carry = 0;
    for (int i0 = 0; i0 < n; i0 += kBookThreads) {
        const int i = i0 + tid, v = i < n ? ld(count + i) : 0;
        int x = v;
#pragma unroll
        for (int o = 1; o < 32; o <<= 1) {
            const int y = __shfl_up_sync(0xffffffffu, x, o);
            if (lane >= o) x += y;
        }
        if (lane == 31) warp_sum[warp] = x;
        __syncthreads();
        int base = 0, all = 0;
        for (int w = 0; w < kBookThreads / 32; ++w) {
            const int s = warp_sum[w];
            if (w < warp) base += s;
            all += s;
        }
        if (i < n) st(before + i, carry + base + x - v);
        carry += all;
        __syncthreads();
    }
    return carry;
}

struct BooksParams {
    Cache4 c;
    int32_t n;
    const int32_t *dst, *src;     // src: fork, copy
    const int64_t *offsets;       // append
    int64_t rows;
};

// Pages listed by (entry, place in its table).  Every phase goes over the entries warp by warp in the same way.
template <int OP>
__global__ void __launch_bounds__(kBookThreads) k_books(const BooksParams p)
{
    const Cache4 &c = p.c;
    const Scratch s = scratch_of(c);
    __shared__ int32_t warp_sum[kBookThreads / 32];
    const int tid = threadIdx.x, lane = tid & 31, n = p.n;
    const int cta = (int)cluster_rank(), ctas = gridDim.x;   // the grid is one cluster
    const int w0 = cta * (kBookThreads / 32) + (tid >> 5), warps = ctas * (kBookThreads / 32);
    const int t0 = cta * kBookThreads + tid, threads = ctas * kBookThreads;
    uint32_t bits = 0;

    bool offsets_bad = false;
    if (OP == kAppend) {
        for (int i = tid; i < n; i += kBookThreads) {
            const int64_t a = p.offsets[i], b = p.offsets[i + 1];
            offsets_bad |= a < 0 || b < a || b > p.rows;
        }
        offsets_bad = __syncthreads_or(offsets_bad) != 0;
        if (offsets_bad) bits |= AIF_STATUS_BAD_ID;
    }
    for (int i = t0; i < n; i += threads) {
        const int q = p.dst[i];
        if (q >= 0 && q < c.n_seqs) atomicMin(s.mark_seq + q, i);
    }
    books_sync();

    // which entries stand
    for (int i = t0; i < n; i += threads) {
        const int q = p.dst[i];
        bool ok = q >= 0 && q < c.n_seqs && ld(s.mark_seq + q) == i;
        if (OP == kFork || OP == kCopy) {
            const int f = p.src[i];
            ok = ok && f >= 0 && f < c.n_seqs && ld(s.mark_seq + f) == INT_MAX;
        }
        if (!ok) bits |= AIF_STATUS_BAD_ID;
        int need = 0, tail = -1, info = ok && !offsets_bad ? 0 : -1;
        if (OP == kAppend && info == 0) {
            const int64_t r = p.offsets[i + 1] - p.offsets[i];
            const int L = ld(c.lengths + q);
            if (L < 0 || L > c.longest() || r > c.longest() - L) {
                info = -1, bits |= AIF_STATUS_FULL;
            } else {
                info = L;
                need = c.pages_of(L + (int)r) - c.pages_of(L);
                const int fill = L & (c.page_rows() - 1);
                if (r > 0 && fill > 0) {
                    const int pg = ld(c.table + (size_t)q * c.max_pages + (L >> c.page_shift));
                    if (c.holds(pg) && ld(c.refs + pg) > 1) tail = pg, need += 1;
                }
            }
        }
        st(s.info + i, info), st(s.from + i, tail);
        st(s.count + i, need);
    }
    books_sync();
    for (int i = t0; i < n; i += threads) {
        const int q = p.dst[i];
        if (q >= 0 && q < c.n_seqs) st(s.mark_seq + q, INT_MAX);
    }

    if (OP != kAppend) {
        // the pages that the entries' sequences had: one reference less each
        for (int i = w0; i < n; i += warps) {
            if (ld(s.info + i) < 0) continue;
            const int q = p.dst[i], np = min(c.pages_of(max(ld(c.lengths + q), 0)), c.max_pages);
            for (int x = lane; x < np; x += 32) {
                const int pg = ld(c.table + (size_t)q * c.max_pages + x);
                if (c.holds(pg)) atomicSub(c.refs + pg, 1), atomicMin(s.mark_page + pg, i * c.max_pages + x);
            }
        }
        books_sync();
        for (int i = w0; i < n; i += warps) {
            int got = 0;
            if (ld(s.info + i) >= 0) {
                const int q = p.dst[i], np = min(c.pages_of(max(ld(c.lengths + q), 0)), c.max_pages);
                for (int x = lane; x < np; x += 32) {
                    const int pg = ld(c.table + (size_t)q * c.max_pages + x);
                    got += c.holds(pg) && ld(c.refs + pg) == 0 && ld(s.mark_page + pg) == i * c.max_pages + x;
                }
                got = __reduce_add_sync(0xffffffffu, got);
            }
            if (lane == 0) st(s.count + i, got);
        }
        books_sync();
        if (cta == 0) {
            const int total = scan_counts(s.count, s.before, n, warp_sum);
            if (tid == 0) {
                const int free_now = min(max(ld(c.n_free), 0), c.n_pages);
                st(s.misc, total), st(s.misc + 1, free_now), st(c.n_free, free_now + total);
            }
        }
        books_sync();
        const int total = ld(s.misc), base = ld(s.misc + 1);
        for (int i = w0; i < n; i += warps) {
            if (ld(s.info + i) < 0) continue;
            const int q = p.dst[i], np = min(c.pages_of(max(ld(c.lengths + q), 0)), c.max_pages);
            int32_t *row = c.table + (size_t)q * c.max_pages;
            // pages go back in the order opposite to the one in which they are handed out: the last entry's last page first
            int at = base + total - ld(s.before + i) - 1;
            for (int x0 = 0; x0 < np; x0 += 32) {
                const int x = x0 + lane, pg = x < np ? ld(row + x) : -1;
                const bool mine = c.holds(pg) && ld(s.mark_page + pg) == i * c.max_pages + x, back = mine && ld(c.refs + pg) == 0;
                const unsigned who = __ballot_sync(0xffffffffu, back);
                const int pos = at - __popc(who & ((1u << lane) - 1u));
                if (back && pos >= 0 && pos < c.n_pages) st(c.free_pages + pos, pg);
                if (mine) st(s.mark_page + pg, INT_MAX);
                if (x < np) st(row + x, -1);
                at -= __popc(who);
            }
            int length = 0;
            if (OP == kFork) {
                const int f = p.src[i];
                length = ld(c.lengths + f);
                const int nf = min(c.pages_of(max(length, 0)), c.max_pages);
                for (int x = lane; x < nf; x += 32) {
                    const int pg = ld(c.table + (size_t)f * c.max_pages + x);
                    st(row + x, pg);
                    if (c.holds(pg)) atomicAdd(c.refs + pg, 1);
                }
            }
            __syncwarp();
            if (OP != kCopy && lane == 0) st(c.lengths + q, length);
            if (OP == kCopy && lane == 0) {
                const int want = min(c.pages_of(max(ld(c.lengths + p.src[i]), 0)), c.max_pages);
                st(c.lengths + q, 0), st(s.count + i, want);
            }
        }
        if (OP == kCopy) {
            for (int i = t0; i < n; i += threads)
                if (ld(s.info + i) < 0) st(s.count + i, 0);
        }
    }
    if (OP == kCopy || OP == kAppend) {
        if (OP == kCopy) books_sync();
        if (cta == 0) {
            scan_counts(s.count, s.before, n, warp_sum);
            const int free_now = min(max(ld(c.n_free), 0), c.n_pages);
            int taken = 0;   // the entries that are served are a beginning of those that need pages
            for (int i = tid; i < n; i += kBookThreads) {
                const int end = ld(s.before + i) + ld(s.count + i);
                if (end <= free_now) taken = max(taken, end);
            }
            taken = __reduce_max_sync(0xffffffffu, taken);
            if (lane == 0) warp_sum[tid >> 5] = taken;
            __syncthreads();
            if (tid == 0) {
                for (int w = 0; w < kBookThreads / 32; ++w) taken = max(taken, warp_sum[w]);
                st(s.misc + 1, free_now), st(s.misc + 2, 0), st(c.n_free, free_now - taken);
            }
        }
        books_sync();
        const int top = ld(s.misc + 1) - 1;
        for (int i = w0; i < n; i += warps) {
            const int need = ld(s.count + i), first = ld(s.before + i), info = ld(s.info + i);
            if (info < 0) continue;
            if (need > 0 && first + need > top + 1) {
                bits |= AIF_STATUS_FULL;
                __syncwarp();
                if (lane == 0) st(s.info + i, -1), st(s.from + i, -1);
                continue;
            }
            const int q = p.dst[i];
            int32_t *row = c.table + (size_t)q * c.max_pages;
            const int tail = OP == kAppend ? ld(s.from + i) : -1;
            const int have = OP == kAppend ? c.pages_of(info) - (tail >= 0) : 0;   // place of the first new page
            for (int x = lane; x < need; x += 32) {
                const int pg = ld(c.free_pages + top - first - x);
                if (c.holds(pg)) st(c.refs + pg, 1);
                else bits |= AIF_STATUS_BAD_ID;
                st(row + have + x, pg);
                if (x == 0 && tail >= 0) {
                    st(s.to + i, pg), st(s.misc + 2, 1);
                    atomicSub(c.refs + tail, 1), atomicMin(s.mark_page + tail, i);
                }
            }
            if (lane == 0) {
                const int length = OP == kAppend ? info + (int)(p.offsets[i + 1] - p.offsets[i]) : ld(c.lengths + p.src[i]);
                st(c.lengths + q, length);
                if (OP == kCopy) st(s.info + i, need);
            }
        }
        books_sync();
        if (OP == kAppend && ld(s.misc + 2) != 0) {
            // shared last pages that every sequence has copied away in this very call belong to nobody now
            for (int i = t0; i < n; i += threads) {
                const int pg = ld(s.from + i);
                const bool mine = pg >= 0 && ld(s.mark_page + pg) == i;
                st(s.count + i, mine && ld(c.refs + pg) == 0 ? 1 : 0);
            }
            books_sync();
            if (cta == 0) {
                const int total = scan_counts(s.count, s.before, n, warp_sum);
                if (tid == 0) {
                    const int free_now = min(max(ld(c.n_free), 0), c.n_pages);
                    st(s.misc, total), st(s.misc + 1, free_now), st(c.n_free, free_now + total);
                }
            }
            books_sync();
            const int last = ld(s.misc) + ld(s.misc + 1) - 1;
            for (int i = t0; i < n; i += threads) {
                const int pg = ld(s.from + i);
                if (pg < 0) continue;
                const int pos = last - ld(s.before + i);
                if (ld(s.count + i) && pos >= 0 && pos < c.n_pages) st(c.free_pages + pos, pg);
                if (ld(s.mark_page + pg) == i) st(s.mark_page + pg, INT_MAX);
            }
        }
    }
    if (bits) atomicOr(c.status, bits);
}

// The same for a few sequences (n <= kFewSeqs), in one CTA with the entries in shared memory.  Its time is a chain of loads from L2, so none is made twice.
constexpr int kFewSeqs = 128, kFewThreads = 1024;

// before[i] = count[0] + .. + count[i - 1]; the total is left in before[n].  One warp.
__device__ __forceinline__ void scan_few(const int32_t *count, int32_t *before, int n, int lane)
{
    int v[4], mine = 0;
#pragma unroll
    for (int u = 0; u < 4; ++u) v[u] = 4 * lane + u < n ? count[4 * lane + u] : 0, mine += v[u];
    int x = mine;
#pragma unroll
    for (int o = 1; o < 32; o <<= 1) {
        const int y = __shfl_up_sync(0xffffffffu, x, o);
        if (lane >= o) x += y;
    }
    int at = x - mine;
#pragma unroll
    for (int u = 0; u < 4; ++u) {
        if (4 * lane + u <= n) before[4 * lane + u] = at;
        at += v[u];
    }
    if (lane == 31 && n == kFewSeqs) before[n] = at;
}

template <int OP>
__global__ void __launch_bounds__(kFewThreads) k_books_few(const BooksParams p)
{
    const Cache4 &c = p.c;
    const Scratch s = scratch_of(c);
    __shared__ int32_t dst[kFewSeqs], src[kFewSeqs], had[kFewSeqs], now[kFewSeqs], count[kFewSeqs], before[kFewSeqs + 1], info[kFewSeqs], from[kFewSeqs], to[kFewSeqs];
    __shared__ int32_t n_free, given;
    const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5, n = p.n;
    constexpr int kWarps = kFewThreads / 32;
    uint32_t bits = 0;
    bool offsets_bad = false;
    int64_t added = 0;
    if (tid == 0) n_free = min(max(ld(c.n_free), 0), c.n_pages), given = 0;
    if (tid < n) {
        const int q = p.dst[tid], f = OP == kFork || OP == kCopy ? p.src[tid] : 0;
        dst[tid] = q, src[tid] = f;
        if (OP == kAppend) {
            const int64_t a = p.offsets[tid], b = p.offsets[tid + 1];
            offsets_bad = a < 0 || b < a || b > p.rows;
            added = b - a;
        }
        had[tid] = q >= 0 && q < c.n_seqs ? ld(c.lengths + q) : 0;
        now[tid] = (OP == kFork || OP == kCopy) && f >= 0 && f < c.n_seqs ? ld(c.lengths + f) : 0;
    }
    offsets_bad = __syncthreads_or(offsets_bad) != 0;
    if (tid < n) {
        const int q = dst[tid], f = src[tid];
        bool ok = q >= 0 && q < c.n_seqs;
        for (int j = 0; j < tid; ++j) ok = ok && dst[j] != q;   // the first that names a sequence stands
        if (OP == kFork || OP == kCopy) {
            ok = ok && f >= 0 && f < c.n_seqs;
            for (int j = 0; j < n; ++j) ok = ok && dst[j] != f;
        }
        if (!ok || offsets_bad) bits |= AIF_STATUS_BAD_ID;
        int need = 0, tail = -1, in = ok && !offsets_bad ? 0 : -1;
        if (OP == kAppend && in == 0) {
            const int L = had[tid];
            if (L < 0 || L > c.longest() || added > c.longest() - L) {
                in = -1, bits |= AIF_STATUS_FULL;
            } else {
                in = L;
                need = c.pages_of(L + (int)added) - c.pages_of(L);
                now[tid] = L + (int)added;
                if (added > 0 && (L & (c.page_rows() - 1)) > 0) {
                    const int pg = ld(c.table + (size_t)q * c.max_pages + (L >> c.page_shift));
                    if (c.holds(pg) && ld(c.refs + pg) > 1) tail = pg, need += 1;
                }
            }
        }
        if (OP == kCopy && in == 0) need = min(c.pages_of(max(now[tid], 0)), c.max_pages);
        info[tid] = in, from[tid] = tail, to[tid] = -1, count[tid] = need;
    }
    __syncthreads();
    auto pages_had = [&](int i) { return min(c.pages_of(max(had[i], 0)), c.max_pages); };
    if (OP != kAppend) {
        // the pages that the entries' sequences had: one reference less each, then those that nobody has back to the free ones
        __shared__ int32_t back[kFewSeqs];
        for (int i = warp; i < n; i += kWarps) {
            if (info[i] < 0) continue;
            const int32_t *row = c.table + (size_t)dst[i] * c.max_pages;
            const int np = pages_had(i);
            for (int x = lane; x < np; x += 32) {
                const int pg = ld(row + x);
                if (c.holds(pg)) atomicSub(c.refs + pg, 1), atomicMin(s.mark_page + pg, i * c.max_pages + x);
            }
        }
        __syncthreads();
        for (int i = warp; i < n; i += kWarps) {
            int got = 0;
            if (info[i] >= 0) {
                const int32_t *row = c.table + (size_t)dst[i] * c.max_pages;
                const int np = pages_had(i);
                for (int x = lane; x < np; x += 32) {
                    const int pg = ld(row + x);
                    if (!c.holds(pg)) continue;
                    const int refs = ld(c.refs + pg), mark = ld(s.mark_page + pg);
                    got += refs == 0 && mark == i * c.max_pages + x;
                }
                got = __reduce_add_sync(0xffffffffu, got);
            }
            if (lane == 0) back[i] = got;
        }
        __syncthreads();
        if (warp == 0) scan_few(back, before, n, lane);
        __syncthreads();
        const int total = before[n], base = n_free;
        for (int i = warp; i < n; i += kWarps) {
            if (info[i] < 0) continue;
            int32_t *row = c.table + (size_t)dst[i] * c.max_pages;
            const int np = pages_had(i), nf = OP == kFork ? min(c.pages_of(max(now[i], 0)), c.max_pages) : 0;
            const int32_t *row_f = c.table + (size_t)max(src[i], 0) * c.max_pages;
            // pages go back in the order opposite to the one in which they are handed out: the last entry's last page first
            int at = base + total - before[i] - 1;
            for (int x0 = 0; x0 < max(np, nf); x0 += 32) {
                const int x = x0 + lane, pg = x < np ? ld(row + x) : -1, take = x < nf ? ld(row_f + x) : -1;
                int refs = 1, mark = -1;
                if (c.holds(pg)) refs = ld(c.refs + pg), mark = ld(s.mark_page + pg);
                const bool mine = mark == i * c.max_pages + x && c.holds(pg), give = mine && refs == 0;
                const unsigned who = __ballot_sync(0xffffffffu, give);
                const int pos = at - __popc(who & ((1u << lane) - 1u));
                if (give && pos >= 0 && pos < c.n_pages) st(c.free_pages + pos, pg);
                if (mine) st(s.mark_page + pg, INT_MAX);
                if (x < np || x < nf) st(row + x, take);
                if (c.holds(take)) atomicAdd(c.refs + take, 1);
                at -= __popc(who);
            }
            if (lane == 0) st(c.lengths + dst[i], OP == kFork ? now[i] : 0);
        }
        __syncthreads();
        if (tid == 0) n_free = base + total;
        __syncthreads();
    }
    if (OP == kCopy || OP == kAppend) {
        if (warp == 0) scan_few(count, before, n, lane);
        __syncthreads();
        const int top = n_free - 1;
        for (int i = warp; i < n; i += kWarps) {
            const int need = count[i], first = before[i], in = info[i];
            if (in < 0) continue;
            if (need > 0 && first + need > top + 1) {   // the entries that are served are a beginning of those that need pages
                bits |= AIF_STATUS_FULL;
                __syncwarp();
                if (lane == 0) info[i] = -1, from[i] = -1;
                continue;
            }
            int32_t *row = c.table + (size_t)dst[i] * c.max_pages;
            const int tail = from[i], have = OP == kAppend ? c.pages_of(in) - (tail >= 0) : 0;   // place of the first new page
            for (int x = lane; x < need; x += 32) {
                const int pg = ld(c.free_pages + top - first - x);
                if (c.holds(pg)) st(c.refs + pg, 1);
                else bits |= AIF_STATUS_BAD_ID;
                st(row + have + x, pg);
                if (x == 0 && tail >= 0) {
                    to[i] = pg, given = 1;
                    atomicSub(c.refs + tail, 1), atomicMin(s.mark_page + tail, i);
                }
            }
            if (lane == 0) {
                st(c.lengths + dst[i], now[i]);
                if (OP == kCopy) info[i] = need;
            }
        }
        __syncthreads();
        if (tid < n) {
            st(s.info + tid, info[tid]), st(s.from + tid, from[tid]), st(s.to + tid, to[tid]);
        }
        // pages taken: up to the last entry that was served
        int taken = 0;
        if (tid < n && count[tid] > 0 && before[tid] + count[tid] <= top + 1) taken = before[tid] + count[tid];
        taken = __reduce_max_sync(0xffffffffu, taken);
        __shared__ int32_t most;
        if (tid == 0) most = 0;
        __syncthreads();
        if (lane == 0 && taken > 0) atomicMax(&most, taken);
        __syncthreads();
        if (tid == 0) n_free -= most;
        __syncthreads();
        if (OP == kAppend && given) {
            // shared last pages that every sequence has copied away in this very call belong to nobody now
            int pg = -1;
            bool mine = false;
            if (tid < n) {
                pg = from[tid];
                mine = pg >= 0 && ld(s.mark_page + pg) == tid;
                count[tid] = mine && ld(c.refs + pg) == 0 ? 1 : 0;
            }
            __syncthreads();
            if (warp == 0) scan_few(count, before, n, lane);
            __syncthreads();
            if (tid < n) {
                const int pos = n_free + before[n] - 1 - before[tid];
                if (count[tid] && pos >= 0 && pos < c.n_pages) st(c.free_pages + pos, pg);
                if (mine) st(s.mark_page + pg, INT_MAX);
            }
            __syncthreads();
            if (tid == 0) n_free += before[n];
        }
    }
    if (tid == 0) st(c.n_free, n_free);
    if (bits) atomicOr(c.status, bits);
}

// ---- rows -------------------------------------------------------------------------------------------------------

// Entry of a row: the last i with offsets[i] <= row (offsets ascend; row < offsets[n]).
__device__ __forceinline__ int entry_of(const int64_t *offsets, int n, int64_t row)
{
    int lo = 0, hi = n;
    while (hi - lo > 1) {
        const int mid = (lo + hi) >> 1;
        if (__ldg(offsets + mid) <= row) lo = mid;
        else hi = mid;
    }
    return lo;
}

// A CTA of the row kernels takes whole rows, about kRowItems pieces of eight elements.
constexpr int kRowItems = 1024, kRowThreads = 256, kMostRows = kRowItems / 4;   // (a row has four pieces at least)
// Of a call with `rows` rows: as many as spread over eight CTAs of every multiprocessor, between that and kMostRows, since a CTA's rows wait for a search and three loads that need
// one another (read of 944919 rows, d = 128: 77 us with 256 rows to a CTA, 88 with 64).
inline int rows_of_cta(int per_row, int64_t rows)
{
    const int least = std::max(1, kRowItems / per_row), most = std::min(kMostRows, 8 * least);
    return (int)std::clamp<int64_t>((rows + 148 * 8 - 1) / (148 * 8), least, most);
}

struct AppendParams {
    Cache4 c;
    int32_t n;
    const int32_t *seq_ids;
    const int64_t *offsets;
    const void *x[2];
    int64_t rows, stride;
    int32_t row_blocks;   // CTAs that bring rows; the ones behind them copy shared last pages
    int32_t cta_rows;
    FastDiv per_row, per_head;   // pieces of eight elements of a row, of a head's row
};

// Rows to pages: four lanes quantise a block of 32 elements, so a warp reads 512 (bf16) consecutive bytes at a time; where a row goes is looked up once,
// while its elements are on their way.
template <typename T, bool ALIGNED>
__global__ void __launch_bounds__(kRowThreads) k_append(const AppendParams p)
{
    const Cache4 &c = p.c;
    const Scratch s = scratch_of(c);
    __shared__ int64_t place[kMostRows];   // row of a page (of head 0) that a row of the CTA goes to, or -1
    const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5, which = blockIdx.y;
    if ((int)blockIdx.x >= p.row_blocks) {
        // the rows that a copied last page held: codes in 16-byte pieces, scale bytes one by one (the rows behind them are being written)
        for (int i = ((int)blockIdx.x - p.row_blocks) * 8 + warp; i < p.n; i += (gridDim.x - p.row_blocks) * 8) {
            const int from = s.from[i], L = s.info[i];
            if (from < 0 || L < 0 || !c.holds(s.to[i])) continue;
            const int fill = L & (c.page_rows() - 1), to = s.to[i];
            for (int h = 0; h < c.heads; ++h) {
                const size_t a = c.row(from, h, 0), b = c.row(to, h, 0);
                const uint4 *src = reinterpret_cast<const uint4 *>(c.codes[which] + a * (c.d / 2));
                uint4 *dst = reinterpret_cast<uint4 *>(c.codes[which] + b * (c.d / 2));
                for (int x = lane; x < fill * (c.d / 32); x += 32) {
                    dst[x] = src[x];
                    c.scales[which][b * (c.d / 32) + x] = c.scales[which][a * (c.d / 32) + x];
                }
            }
        }
        return;
    }
    const int64_t row0 = (int64_t)blockIdx.x * p.cta_rows;
    const int rows = rows_before(min(p.offsets[p.n], p.rows), row0, p.cta_rows), items = rows * (int)p.per_row.by;   // (offsets that k_books refused come here too)
    if (rows <= 0) return;
    const T *x = static_cast<const T *>(p.x[which]) + row0 * p.stride;
    for (int i0 = 0; i0 < items; i0 += 4 * kRowThreads) {
        Raw8<T> v[4];
        int row[4], part[4];
#pragma unroll
        for (int u = 0; u < 4; ++u) {
            const int i = i0 + u * kRowThreads + tid;
            row[u] = (int)p.per_row.div((uint32_t)i), part[u] = i - row[u] * (int)p.per_row.by;
            v[u] = Raw8<T>{};
            if (i < items) v[u] = load_raw8<T, ALIGNED>(x + row[u] * p.stride + part[u] * 8);
        }
        if (i0 == 0) {
            if (tid < rows) {
                const int64_t r = row0 + tid;
                int64_t to = -1;
                if (r >= p.offsets[0]) {
                    const int e = entry_of(p.offsets, p.n, r), first = s.info[e];
                    if (first >= 0) {   // (offsets ascend then)
                        const int at = first + (int)(r - p.offsets[e]);
                        const int page = c.table[(size_t)p.seq_ids[e] * c.max_pages + (at >> c.page_shift)];
                        if (c.holds(page)) to = (int64_t)c.row(page, 0, at & (c.page_rows() - 1));
                    }
                }
                place[tid] = to;
            }
            __syncthreads();
        }
        uint32_t w[4], byte[4];
        mx_quantise_quad<T>(v, w, byte);
#pragma unroll
        for (int u = 0; u < 4; ++u) {
            if (i0 + u * kRowThreads + tid >= items || place[row[u]] < 0) continue;
            const int head = (int)p.per_head.div((uint32_t)part[u]), sub = part[u] - head * (int)p.per_head.by;
            const size_t r = (size_t)place[row[u]] + ((size_t)head << c.page_shift);
            reinterpret_cast<uint32_t *>(c.codes[which] + r * (c.d / 2))[sub] = w[u];
            if ((sub & 3) == 0) c.scales[which][r * (c.d / 32) + (sub >> 2)] = (uint8_t)byte[u];
        }
    }
}

struct ReadParams {
    Cache4 c;
    int32_t n;
    const int32_t *seq_ids;
    const int64_t *offsets;
    void *out[2];
    int64_t rows, stride;
    int32_t cta_rows;
    FastDiv per_row, per_head;
};

template <typename T, bool ALIGNED>
__global__ void __launch_bounds__(kRowThreads) k_read(const ReadParams p)
{
    const Cache4 &c = p.c;
    __shared__ int64_t place[kMostRows];   // row of a page (of head 0); -1: nobody's row; -2: a row that is not there
    const int tid = threadIdx.x, which = blockIdx.y;
    bool bad = false;
    for (int i = tid; i < p.n; i += kRowThreads) {
        const int64_t a = p.offsets[i], b = p.offsets[i + 1];
        bad |= a < 0 || b < a || b > p.rows;
    }
    if (__syncthreads_or(bad)) {
        if (blockIdx.x == 0 && tid == 0) atomicOr(c.status, AIF_STATUS_BAD_ID);
        return;
    }
    const int64_t row0 = (int64_t)blockIdx.x * p.cta_rows;
    const int rows = rows_before(p.offsets[p.n], row0, p.cta_rows), items = rows * (int)p.per_row.by;
    if (rows <= 0) return;
    if (tid < rows) {
        const int64_t r = row0 + tid;
        int64_t from = -1;
        if (r >= p.offsets[0]) {
            const int e = entry_of(p.offsets, p.n, r), q = p.seq_ids[e];
            const int64_t at = r - p.offsets[e];
            int page = -1;
            if (q >= 0 && q < c.n_seqs && at < c.lengths[q] && at < c.longest()) page = c.table[(size_t)q * c.max_pages + (at >> c.page_shift)];
            from = c.holds(page) ? (int64_t)c.row(page, 0, (int)at & (c.page_rows() - 1)) : -2;
            if (from == -2) atomicOr(c.status, AIF_STATUS_BAD_ID);
        }
        place[tid] = from;
    }
    __syncthreads();
    T *out = static_cast<T *>(p.out[which]) + row0 * p.stride;
    for (int i0 = 0; i0 < items; i0 += 4 * kRowThreads) {
        uint32_t w[4], byte[4];
        int row[4], part[4];
#pragma unroll
        for (int u = 0; u < 4; ++u) {
            const int i = i0 + u * kRowThreads + tid;
            row[u] = (int)p.per_row.div((uint32_t)i), part[u] = i - row[u] * (int)p.per_row.by;
            w[u] = 0u, byte[u] = 0u;
            if (i < items && place[row[u]] >= 0) {
                const int head = (int)p.per_head.div((uint32_t)part[u]), sub = part[u] - head * (int)p.per_head.by;
                const size_t r = (size_t)place[row[u]] + ((size_t)head << c.page_shift);
                w[u] = __ldg(reinterpret_cast<const uint32_t *>(c.codes[which] + r * (c.d / 2)) + sub);
                byte[u] = __ldg(c.scales[which] + r * (c.d / 32) + (sub >> 2));
            }
        }
#pragma unroll
        for (int u = 0; u < 4; ++u) {
            if (i0 + u * kRowThreads + tid >= items || place[row[u]] == -1) continue;
            float v[8];
            mx_values8(w[u], mx_scale(byte[u]), v);
            store8<T, ALIGNED>(out + row[u] * p.stride + part[u] * 8, v);
        }
    }
}

// ---- whole pages ------------------------------------------------------------------------------------------------

// One warp: page `from` of a to page `to` of b, keys or values.
__device__ __forceinline__ void move_page(const Cache4 &a, const Cache4 &b, int which, int from, int to, int lane)
{
    const size_t ra = a.row(from, 0, 0), rb = b.row(to, 0, 0);
    const int rows = a.heads << a.page_shift;
    const uint4 *src = reinterpret_cast<const uint4 *>(a.codes[which] + ra * (a.d / 2));
    uint4 *dst = reinterpret_cast<uint4 *>(b.codes[which] + rb * (b.d / 2));
    const int nc = rows * (a.d / 32);
    for (int x0 = lane; x0 < nc; x0 += 128) {
        uint4 v[4];
#pragma unroll
        for (int u = 0; u < 4; ++u)
            if (x0 + 32 * u < nc) v[u] = __ldg(src + x0 + 32 * u);
#pragma unroll
        for (int u = 0; u < 4; ++u)
            if (x0 + 32 * u < nc) dst[x0 + 32 * u] = v[u];
    }
    // rows of a page: at least 16, so its scale bytes are whole 16-byte pieces too
    const uint4 *ss = reinterpret_cast<const uint4 *>(a.scales[which] + ra * (a.d / 32));
    uint4 *sd = reinterpret_cast<uint4 *>(b.scales[which] + rb * (b.d / 32));
    for (int x = lane; x < rows * (a.d / 32) / 16; x += 32) sd[x] = __ldg(ss + x);
}

struct CopyParams {
    Cache4 c;
    int32_t n, kinds;
    const int32_t *src, *dst;
};
__global__ void __launch_bounds__(256) k_copy_pages(const CopyParams p)
{
    const Cache4 &c = p.c;
    const Scratch s = scratch_of(c);
    const int lane = threadIdx.x & 31;
    const int64_t items = (int64_t)p.n * c.max_pages;
    for (int64_t w = (int64_t)blockIdx.x * 8 + (threadIdx.x >> 5); w < items; w += (int64_t)gridDim.x * 8) {
        const int i = (int)(w / c.max_pages), x = (int)(w - (int64_t)i * c.max_pages);
        if (x >= s.info[i]) continue;   // (-1: undone)
        const int from = c.table[(size_t)p.src[i] * c.max_pages + x], to = c.table[(size_t)p.dst[i] * c.max_pages + x];
        if (!c.holds(from) || !c.holds(to)) continue;
        for (int k = 0; k < p.kinds; ++k) move_page(c, c, k, from, to, lane);
    }
}

// Pages in use per block of kMapBlock, and the rank of each within its block.
__global__ void __launch_bounds__(256) k_map_pages(const Cache4 c)
{
    const Scratch s = scratch_of(c);
    __shared__ int32_t sums[8];
    const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5;
    const int64_t p0 = (int64_t)blockIdx.x * kMapBlock + tid * 4;
    int used[4], mine = 0;
#pragma unroll
    for (int u = 0; u < 4; ++u) used[u] = p0 + u < c.n_pages && c.refs[p0 + u] > 0, mine += used[u];
    int x = mine;
#pragma unroll
    for (int o = 1; o < 32; o <<= 1) {
        const int y = __shfl_up_sync(0xffffffffu, x, o);
        if (lane >= o) x += y;
    }
    if (lane == 31) sums[warp] = x;
    __syncthreads();
    int at = x - mine, all = 0;
    for (int w = 0; w < 8; ++w) at += w < warp ? sums[w] : 0, all += sums[w];
#pragma unroll
    for (int u = 0; u < 4; ++u) {
        if (p0 + u < c.n_pages) s.map[p0 + u] = used[u] ? at : -1;
        at += used[u];
    }
    if (tid == 0) s.block_sum[blockIdx.x] = all;
}
// Exclusive sums over the blocks in place; misc[3] = pages in use.
__global__ void __launch_bounds__(kBookThreads) k_map_blocks(const Cache4 c, int blocks)
{
    const Scratch s = scratch_of(c);
    __shared__ int32_t warp_sum[kBookThreads / 32];
    const int total = scan_counts(s.block_sum, s.block_sum, blocks, warp_sum);
    if (threadIdx.x == 0) s.misc[3] = total;
}
// Pages, tables and books of `into`.
__global__ void __launch_bounds__(256) k_move_pages(const Cache4 c, const Cache4 into, int kinds)
{
    const Scratch s = scratch_of(c), si = scratch_of(into);
    const int lane = threadIdx.x & 31;
    const int live = s.misc[3];
    const bool fits = live <= into.n_pages;
    const int64_t t0 = (int64_t)blockIdx.x * 256 + threadIdx.x, threads = (int64_t)gridDim.x * 256;
    if (fits) {
        for (int64_t pg = t0 >> 5; pg < c.n_pages; pg += threads >> 5) {
            const int rank = s.map[pg];
            if (rank < 0) continue;
            const int to = rank + s.block_sum[pg / kMapBlock];
            for (int k = 0; k < kinds; ++k) move_page(c, into, k, (int)pg, to, lane);
            if (lane == 0) into.refs[to] = c.refs[pg];
        }
    }
    for (int64_t x = t0; x < (int64_t)c.n_seqs * c.max_pages; x += threads) {
        const int pg = c.table[x];
        const bool used = fits && c.holds(pg) && s.map[pg] >= 0;
        into.table[x] = used ? s.map[pg] + s.block_sum[pg / kMapBlock] : -1;
    }
    for (int64_t x = t0; x < c.n_seqs; x += threads) into.lengths[x] = fits ? c.lengths[x] : 0, si.mark_seq[x] = INT_MAX;
    for (int64_t x = t0; x < into.n_pages; x += threads) {
        into.free_pages[x] = into.n_pages - 1 - (int)x;
        si.mark_page[x] = INT_MAX;
        if (!fits || x >= live) into.refs[x] = 0;
    }
    if (t0 == 0) {
        *into.n_free = fits ? into.n_pages - live : into.n_pages;
        if (!fits) atomicOr(into.status, AIF_STATUS_FULL);
    }
}

__global__ void __launch_bounds__(256) k_reset(const Cache4 c)
{
    const Scratch s = scratch_of(c);
    const int64_t t0 = (int64_t)blockIdx.x * 256 + threadIdx.x, threads = (int64_t)gridDim.x * 256;
    for (int64_t x = t0; x < (int64_t)c.n_seqs * c.max_pages; x += threads) c.table[x] = -1;
    for (int64_t x = t0; x < c.n_seqs; x += threads) c.lengths[x] = 0, s.mark_seq[x] = INT_MAX;
    for (int64_t x = t0; x < c.n_pages; x += threads) c.refs[x] = 0, c.free_pages[x] = c.n_pages - 1 - (int)x, s.mark_page[x] = INT_MAX;
    if (t0 == 0) *c.n_free = c.n_pages, *c.status = 0u;
}

template <int OP>
cudaError_t run_books(const BooksParams &p, cudaStream_t st)
{
    count_launch();
    // A few sequences: one CTA, until its 32 warps have some hundred pages each.  us of one CTA and of the cluster, over sequences that share their pages (fork), and with pages taken and
    // given back (append and free of rows, both calls):
    //   sequences x pages  16 x 32     48 x 32     64 x 49     100 x 60    128 x 80    16 x 200    16 x 1000   4 x 4000
    //   fork               5.7   9.9   9.3  11.0   14.1  13.5  21.6  13.4  27.8  15.4  15.5  23.0  49    74    149   234
    //   append + free      13.1  20.6  17.5 21.2   22.6  24.9  32.2  25.7  39.1  28.7  22.1  34.4  56    89    157   254
    if (p.n <= kFewSeqs && (int64_t)p.n * p.c.max_pages <= 32768) {
        k_books_few<OP><<<1, kFewThreads, 0, st>>>(p);
        return cudaGetLastError();
    }
    cudaLaunchConfig_t cfg{};
    cfg.gridDim = dim3(8), cfg.blockDim = dim3(kBookThreads), cfg.stream = st;
    cudaLaunchAttribute attr[1];
    attr[0].id = cudaLaunchAttributeClusterDimension;
    attr[0].val.clusterDim.x = 8, attr[0].val.clusterDim.y = 1, attr[0].val.clusterDim.z = 1;
    cfg.attrs = attr, cfg.numAttrs = 1;
    return cudaLaunchKernelEx(&cfg, k_books<OP>, p);
}

unsigned grid_for(int64_t items, int64_t per_block, int64_t most) { return (unsigned)std::max<int64_t>(1, std::min<int64_t>((items + per_block - 1) / per_block, most)); }

bool at16(const void *p) { return (reinterpret_cast<uintptr_t>(p) & 15) == 0; }

// Checks of a call that names sequences.
int check_call(const aif_cache4 *c, int32_t n, bool distinct)
{
    const int rc = cache4_check(c);
    if (rc != AIF_OK) return rc;
    if (n < 0 || (distinct && n > c->n_seqs)) return AIF_ERR_SHAPE;
    return AIF_OK;
}
// Checks of rows that go in or come out.
int check_rows(const aif_cache4 *c, const void *k, const void *v, int32_t dtype, int64_t rows, int64_t stride)
{
    if (dtype != AIF_F32 && dtype != AIF_BF16) return AIF_ERR_ARG;
    if (rows < 0 || rows > (int64_t)1 << 40 || stride < (int64_t)c->heads * c->d || stride > (int64_t)1 << 31) return AIF_ERR_SHAPE;
    if (rows / rows_of_cta(c->heads * c->d / 8, rows) > INT_MAX - 1024) return AIF_ERR_SHAPE;   // CTAs of a grid
    const unsigned el = dtype == AIF_BF16 ? 2 : 4;
    if ((c->shared != 0) != (v == nullptr)) return AIF_ERR_ARG;
    if (rows > 0 && (!k || reinterpret_cast<uintptr_t>(k) % el != 0 || (v && reinterpret_cast<uintptr_t>(v) % el != 0))) return AIF_ERR_ARG;
    return AIF_OK;
}

int share(const aif_cache4 *c, int32_t n, const int32_t *src, const int32_t *dst, aif_stream stream, bool copy, const char *what)
{
    StageRange range(what);
    const int rc = check_call(c, n, true);
    if (rc != AIF_OK) return rc;
    if (n == 0) return AIF_OK;
    if (!src || !dst) return AIF_ERR_ARG;
    cudaStream_t st = reinterpret_cast<cudaStream_t>(stream);
    BooksParams p{};
    p.c = cache4_of(c), p.n = n, p.src = src, p.dst = dst;
    cudaError_t e = copy ? run_books<kCopy>(p, st) : run_books<kFork>(p, st);
    if (e == cudaSuccess && copy) {
        CopyParams q{};
        q.c = p.c, q.n = n, q.kinds = c->shared ? 1 : 2, q.src = src, q.dst = dst;
        k_copy_pages<<<grid_for((int64_t)n * c->max_pages, 8, 148 * 8), 256, 0, st>>>(q);
        count_launch();
        e = cudaGetLastError();
    }
    return cache4_failed(e, what);
}

}  // namespace

int cache4_failed(cudaError_t e, const char *what)
{
    if (e == cudaSuccess) return AIF_OK;
    char text[256];
    snprintf(text, sizeof(text), "%s: %s", what, cudaGetErrorString(e));
    cudaGetLastError();
    set_last_error(text);
    return AIF_ERR_CUDA;
}

int cache4_check(const aif_cache4 *c)
{
    if (!c || c->struct_size != sizeof(aif_cache4)) return AIF_ERR_ARG;
    if (c->d < 32 || c->d > 256 || c->d % 32 != 0 || c->heads < 1 || c->heads > 64) return AIF_ERR_SHAPE;
    if (c->shared != 0 && c->shared != 1) return AIF_ERR_ARG;
    if (c->page_rows < 16 || c->page_rows > 1024 || (c->page_rows & (c->page_rows - 1)) != 0) return AIF_ERR_SHAPE;
    if (c->n_pages < 1 || c->n_seqs < 1 || c->max_pages < 1) return AIF_ERR_SHAPE;
    if ((int64_t)c->n_seqs * c->max_pages > INT_MAX || (int64_t)c->max_pages * c->page_rows > 1 << 30) return AIF_ERR_SHAPE;
    if (!c->k_codes || !c->k_scales || !c->table || !c->lengths || !c->refs || !c->free_pages || !c->n_free || !c->scratch || !c->status) return AIF_ERR_ARG;
    if ((c->shared != 0) == (c->v_codes != nullptr) || (c->shared != 0) == (c->v_scales != nullptr)) return AIF_ERR_ARG;
    if (!at16(c->k_codes) || !at16(c->k_scales) || !at16(c->v_codes) || !at16(c->v_scales)) return AIF_ERR_ARG;
    return AIF_OK;
}

}  // namespace aif

using namespace aif;

extern "C" {

int64_t aif_cache4_scratch_ints(const aif_cache4 *c)
{
    if (!c || c->struct_size != sizeof(aif_cache4)) return AIF_ERR_ARG;
    if (c->n_pages < 1 || c->n_seqs < 1) return AIF_ERR_SHAPE;
    return scratch_ints(c->n_pages, c->n_seqs);
}

int aif_cache4_reset(const aif_cache4 *c, aif_stream stream)
{
    StageRange range("aif_cache4_reset");
    const int rc = cache4_check(c);
    if (rc != AIF_OK) return rc;
    k_reset<<<grid_for(std::max<int64_t>(c->n_pages, (int64_t)c->n_seqs * c->max_pages), 256, 148 * 8), 256, 0, reinterpret_cast<cudaStream_t>(stream)>>>(cache4_of(c));
    count_launch();
    return cache4_failed(cudaGetLastError(), "aif_cache4_reset");
}

int aif_cache4_append(const aif_cache4 *c, int32_t n, const int32_t *seq_ids, const int64_t *offsets, const void *k, const void *v, int32_t dtype,
                      int64_t rows, int64_t stride, aif_stream stream)
{
    StageRange range("aif_cache4_append");
    int rc = check_call(c, n, true);
    if (rc == AIF_OK) rc = check_rows(c, k, v, dtype, rows, stride);
    if (rc != AIF_OK) return rc;
    if (n == 0) return AIF_OK;
    if (!seq_ids || !offsets) return AIF_ERR_ARG;
    cudaStream_t st = reinterpret_cast<cudaStream_t>(stream);
    BooksParams b{};
    b.c = cache4_of(c), b.n = n, b.dst = seq_ids, b.offsets = offsets, b.rows = rows;
    cudaError_t e = run_books<kAppend>(b, st);
    if (e == cudaSuccess && rows > 0) {
        AppendParams p{};
        p.c = b.c, p.n = n, p.seq_ids = seq_ids, p.offsets = offsets, p.x[0] = k, p.x[1] = v, p.rows = rows, p.stride = stride;
        p.per_row = FastDiv::of(c->heads * c->d / 8), p.per_head = FastDiv::of(c->d / 8), p.cta_rows = rows_of_cta(c->heads * c->d / 8, rows);
        p.row_blocks = (int)grid_for(rows, p.cta_rows, INT_MAX);
        const dim3 grid((unsigned)p.row_blocks + grid_for(n, 8, 148), c->shared ? 1 : 2);
        const int el = dtype == AIF_BF16 ? 2 : 4;
        const bool al = at16(k) && at16(v) && stride * el % 16 == 0;
        auto go = [&](auto kernel) { kernel<<<grid, kRowThreads, 0, st>>>(p); };
        if (dtype == AIF_BF16) al ? go(k_append<__nv_bfloat16, true>) : go(k_append<__nv_bfloat16, false>);
        else al ? go(k_append<float, true>) : go(k_append<float, false>);
        count_launch();
        e = cudaGetLastError();
    }
    return cache4_failed(e, "aif_cache4_append");
}

int aif_cache4_fork(const aif_cache4 *c, int32_t n, const int32_t *src, const int32_t *dst, aif_stream stream)
{
    return share(c, n, src, dst, stream, false, "aif_cache4_fork");
}

int aif_cache4_copy(const aif_cache4 *c, int32_t n, const int32_t *src, const int32_t *dst, aif_stream stream)
{
    return share(c, n, src, dst, stream, true, "aif_cache4_copy");
}

int aif_cache4_free(const aif_cache4 *c, int32_t n, const int32_t *seq_ids, aif_stream stream)
{
    StageRange range("aif_cache4_free");
    const int rc = check_call(c, n, true);
    if (rc != AIF_OK) return rc;
    if (n == 0) return AIF_OK;
    if (!seq_ids) return AIF_ERR_ARG;
    BooksParams p{};
    p.c = cache4_of(c), p.n = n, p.dst = seq_ids;
    return cache4_failed(run_books<kFree>(p, reinterpret_cast<cudaStream_t>(stream)), "aif_cache4_free");
}

int aif_cache4_compact(const aif_cache4 *c, const aif_cache4 *into, aif_stream stream)
{
    StageRange range("aif_cache4_compact");
    int rc = cache4_check(c);
    if (rc == AIF_OK) rc = cache4_check(into);
    if (rc != AIF_OK) return rc;
    if (c->d != into->d || c->heads != into->heads || c->shared != into->shared || c->page_rows != into->page_rows || c->n_seqs != into->n_seqs ||
        c->max_pages != into->max_pages)
        return AIF_ERR_SHAPE;
    if (c->k_codes == into->k_codes || c->k_scales == into->k_scales || c->table == into->table || c->lengths == into->lengths || c->refs == into->refs ||
        c->free_pages == into->free_pages || c->n_free == into->n_free || c->scratch == into->scratch || (!c->shared && (c->v_codes == into->v_codes || c->v_scales == into->v_scales)))
        return AIF_ERR_ARG;
    cudaStream_t st = reinterpret_cast<cudaStream_t>(stream);
    const Cache4 a = cache4_of(c), b = cache4_of(into);
    const int blocks = (int)(((int64_t)c->n_pages + kMapBlock - 1) / kMapBlock);
    k_map_pages<<<blocks, 256, 0, st>>>(a);
    k_map_blocks<<<1, kBookThreads, 0, st>>>(a, blocks);
    k_move_pages<<<grid_for(std::max<int64_t>((int64_t)std::max(c->n_pages, into->n_pages) * 32, (int64_t)c->n_seqs * c->max_pages), 256, 148 * 8), 256, 0, st>>>(a, b, c->shared ? 1 : 2);
    count_launch(3);
    return cache4_failed(cudaGetLastError(), "aif_cache4_compact");
}

int aif_cache4_read(const aif_cache4 *c, int32_t n, const int32_t *seq_ids, const int64_t *offsets, void *k_out, void *v_out, int32_t dtype,
                    int64_t rows, int64_t stride, aif_stream stream)
{
    StageRange range("aif_cache4_read");
    int rc = check_call(c, n, false);
    if (rc == AIF_OK) rc = check_rows(c, k_out, v_out, dtype, rows, stride);
    if (rc != AIF_OK) return rc;
    if (n == 0 || rows == 0) return AIF_OK;
    if (!seq_ids || !offsets) return AIF_ERR_ARG;
    cudaStream_t st = reinterpret_cast<cudaStream_t>(stream);
    ReadParams p{};
    p.c = cache4_of(c), p.n = n, p.seq_ids = seq_ids, p.offsets = offsets, p.out[0] = k_out, p.out[1] = v_out, p.rows = rows, p.stride = stride;
    p.per_row = FastDiv::of(c->heads * c->d / 8), p.per_head = FastDiv::of(c->d / 8), p.cta_rows = rows_of_cta(c->heads * c->d / 8, rows);
    const dim3 grid(grid_for(rows, p.cta_rows, INT_MAX), c->shared ? 1 : 2);
    const int el = dtype == AIF_BF16 ? 2 : 4;
    const bool al = at16(k_out) && at16(v_out) && stride * el % 16 == 0;
    auto go = [&](auto kernel) { kernel<<<grid, kRowThreads, 0, st>>>(p); };
    if (dtype == AIF_BF16) al ? go(k_read<__nv_bfloat16, true>) : go(k_read<__nv_bfloat16, false>);
    else al ? go(k_read<float, true>) : go(k_read<float, false>);
    count_launch();
    return cache4_failed(cudaGetLastError(), "aif_cache4_read");
}

int aif_cache4_poll(const aif_cache4 *c, uint32_t *bits, aif_stream stream)
{
    const int rc = cache4_check(c);
    if (rc != AIF_OK) return rc;
    if (!bits) return AIF_ERR_ARG;
    cudaStream_t st = reinterpret_cast<cudaStream_t>(stream);
    cudaError_t e = cudaMemcpyAsync(bits, c->status, 4, cudaMemcpyDeviceToHost, st);
    if (e == cudaSuccess) e = cudaMemsetAsync(c->status, 0, 4, st);
    if (e == cudaSuccess) e = cudaStreamSynchronize(st);
    return cache4_failed(e, "aif_cache4_poll");
}

}  // extern "C"
