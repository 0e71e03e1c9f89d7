// Division of an attention call over the 4-bit cache among the CTAs of a launch, worked out on the device: lengths, offsets and page
// tables are device memory, so a captured call follows them.
//
// A tile is up to `tile_rows` query rows (row = query x heads of a group) of one sequence and one head of the cache; a unit is one block of `block_keys`
// visible keys of a tile (an empty sequence has one).  The units of all tiles, one after the other, are cut into equal ranges, one per CTA, so a launch
// is even whatever the lengths.  A tile that is cut leaves its pieces in the workspace: every CTA has two records, [2 c] for a piece of
// a tile that began in an earlier CTA and [2 c + 1] for the beginning of one that goes on in the next, and a header that says which tile ends in it.
#pragma once

#include "aif_cache4.cuh"

namespace aif {

struct PieceHeader;

struct AttCall {
    Cache4 c;
    int32_t n, n_heads, group;     // group = n_heads / c.heads
    const int32_t *seq_ids;
    const int64_t *offsets;
    int64_t rows;
    const void *q;
    void *out;
    int64_t q_stride, out_stride;
    float scale_log2;              // scale x log2(e)
    int32_t window, sinks;
    int32_t tile_rows, block_keys, min_units;
    float *records;                // [2 x grid][tile_rows][d] sums, then [tile_rows][2]: exponent offset and weight
    PieceHeader *headers;          // [grid]; nullptr where no tile can have more than one unit
};

// A sequence of the call.
struct Entry {
    int32_t seq, length;       // length < 0: bad (id, length)
    int32_t first, rest;       // visible rows: [0, first) and [rest, length)
    int64_t row0;
    int32_t rows;              // query rows x group
    __device__ int keys() const { return length < 0 ? 0 : first + (length - rest); }
    // row of the visible key v
    __device__ int key(int v) const { return v < first ? v : rest + (v - first); }
    // The same in groups of 16 rows that begin on multiples of 16 (and so lie in one page): groups of the call, and the first row of one.  Rows of a group
    // that are not visible: at or behind `first` in the groups of the first rows, before `rest` in the others.
    __device__ int sink_groups() const { return (first + 15) >> 4; }
    __device__ int groups() const { return length < 0 ? 0 : sink_groups() + ((length + 15) >> 4) - (rest >> 4); }
};

// A tile as the CTA that finishes it hands it to the kernel that joins its pieces.
struct PieceHeader {
    int64_t row0;       // first query row of the sequence
    int32_t first_cta;  // CTA where the tile began; -1: nothing ends here that began elsewhere
    int32_t head, r0, rows;   // head of the cache, first row of the tile (query x group) and rows in it
    int32_t pad_[2];
};

cudaError_t launch_att4_pair(const AttCall &a, int grid, cudaStream_t st);   // aif_cache4_pair.cu: bf16, d = 64, 128; tiles of 256 rows, blocks of 64 keys
cudaError_t launch_att4_tc(const AttCall &a, int grid, cudaStream_t st);     // aif_cache4_tc.cu: bf16, d = 256; 128 rows, 64 keys
cudaError_t launch_att4_few(const AttCall &a, int grid, cudaStream_t st);    // aif_cache4_few.cu: bf16, d = 32, 64, 128, 256; 8 rows, 512 keys

namespace {

__device__ __forceinline__ Entry entry_at(const AttCall &a, int i)
{
    Entry e;
    const int64_t o = a.offsets ? a.offsets[i] : i, o1 = a.offsets ? a.offsets[i + 1] : i + 1;
    e.row0 = o, e.rows = (int)(o1 - o) * a.group;
    e.seq = a.seq_ids ? a.seq_ids[i] : i;
    e.length = -1;
    if (e.seq >= 0 && e.seq < a.c.n_seqs) {
        const int L = a.c.lengths[e.seq];
        if (L >= 0 && L <= a.c.longest()) e.length = L;
    }
    e.first = 0, e.rest = 0;
    if (a.window > 0 && e.length > a.window) e.rest = e.length - a.window, e.first = min(a.sinks, e.rest);
    return e;
}
// (block_keys < 0: blocks of that many groups of 16 rows)
__device__ __forceinline__ int blocks_at(const AttCall &a, const Entry &e)
{
    return max(1, a.block_keys > 0 ? (int)(((int64_t)e.keys() + a.block_keys - 1) / a.block_keys) : (e.groups() - a.block_keys - 1) / -a.block_keys);
}
__device__ __forceinline__ int tiles_at(const AttCall &a, const Entry &e) { return (e.rows + a.tile_rows - 1) / a.tile_rows; }
__device__ __forceinline__ int64_t units_at(const AttCall &a, const Entry &e) { return (int64_t)tiles_at(a, e) * a.c.heads * blocks_at(a, e); }

// Where a CTA's units begin: entry, tile (head x row tile) and block in it.
struct Cursor {
    int32_t i, tile, block;
    Entry e;
    int32_t tiles, blocks;   // of the entry (tiles of all heads)
};

// Shared memory of the division.
template <int THREADS>
struct PlanShared {
    int64_t sum[THREADS];   // units before the entries of every thread
    int64_t total;
    int32_t bad;
};

__device__ __forceinline__ int64_t cut(int64_t total, int ctas, int c) { return total / ctas * c + total % ctas * c / ctas; }

// All threads.  Returns the units of the call (0 with *bad: offsets that cannot be) and the number of CTAs that get any; on return sum[t] holds the
// units before the entries of thread t.
template <int THREADS>
__device__ int64_t plan_total(const AttCall &a, PlanShared<THREADS> &s)
{
    const int tid = threadIdx.x, lane = tid & 31;
    const int per = (a.n + THREADS - 1) / THREADS;
    int64_t mine = 0;
    bool bad = false;
    for (int i = tid * per; i < min(a.n, (tid + 1) * per); ++i) {
        if (a.offsets) {
            const int64_t o = a.offsets[i], o1 = a.offsets[i + 1];
            if (o < 0 || o1 < o || o1 > a.rows) {
                bad = true;
                continue;
            }
        }
        mine += units_at(a, entry_at(a, i));
    }
    int64_t x = mine;
#pragma unroll
    for (int o = 1; o < 32; o <<= 1) {
        const int64_t y = __shfl_up_sync(0xffffffffu, x, o);
        if (lane >= o) x += y;
    }
    __shared__ int64_t warp_sum[THREADS / 32];
    if (lane == 31) warp_sum[tid >> 5] = x;
    const bool any_bad = __syncthreads_or(bad) != 0;
    int64_t base = 0, all = 0;
    for (int w = 0; w < THREADS / 32; ++w) {
        if (w < (tid >> 5)) base += warp_sum[w];
        all += warp_sum[w];
    }
    s.sum[tid] = base + x - mine;
    __syncthreads();
    if (any_bad) {
        if (tid == 0 && blockIdx.x == 0) atomicOr(a.c.status, AIF_STATUS_BAD_ID);
        return 0;
    }
    return all;
}

// The place of unit u (u < total); any thread, after plan_total.
template <int THREADS>
__device__ Cursor plan_find(const AttCall &a, const PlanShared<THREADS> &s, int64_t u)
{
    int lo = 0, hi = THREADS;   // the last thread whose entries begin at or before u
    while (hi - lo > 1) {
        const int mid = (lo + hi) >> 1;
        if (s.sum[mid] <= u) lo = mid;
        else hi = mid;
    }
    const int per = (a.n + THREADS - 1) / THREADS;
    Cursor c;
    c.i = lo * per;
    int64_t left = u - s.sum[lo];
    for (;; ++c.i) {
        c.e = entry_at(a, c.i);
        const int64_t has = units_at(a, c.e);
        if (left < has || c.i >= a.n - 1) break;
        left -= has;
    }
    c.tiles = tiles_at(a, c.e) * a.c.heads, c.blocks = blocks_at(a, c.e);
    c.tile = (int)(left / c.blocks), c.block = (int)(left - (int64_t)c.tile * c.blocks);
    return c;
}
// To the next tile (block 0 of it).
__device__ __forceinline__ void plan_next(const AttCall &a, Cursor &c)
{
    c.block = 0;
    if (++c.tile < c.tiles) return;
    c.tile = 0;
    do {
        if (++c.i >= a.n) return;
        c.e = entry_at(a, c.i);
        c.tiles = tiles_at(a, c.e) * a.c.heads;
    } while (c.tiles == 0);
    c.blocks = blocks_at(a, c.e);
}

}  // namespace
}  // namespace aif
