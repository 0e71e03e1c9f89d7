// Division of an attention call over the 4-bit cache among the CTAs of a launch, worked out on the device: lengths, offsets and page
// tables are device memory, so a captured call follows them.
//
// A tile is up to `tile_rows` query rows (row = query x heads of a group) of one sequence and one head of the cache; a unit is one block of a fixed number of
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
    FastDiv by_group;
    const int32_t *seq_ids;
    const int64_t *offsets;
    int64_t rows;
    const void *q;
    void *out;
    int64_t q_stride, out_stride;
    float scale_log2;              // scale x log2(e)
    int32_t window, sinks;
    int32_t tile_rows, min_units, tile_shift, block_shift, in_groups;   // tiles and blocks by shifts; in_groups: blocks are of groups of 16 rows
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
__device__ __forceinline__ int blocks_at(const AttCall &a, const Entry &e)
{
    return max(1, (int)(((uint32_t)(a.in_groups ? e.groups() : e.keys()) + (1u << a.block_shift) - 1) >> a.block_shift));
}
__device__ __forceinline__ int tiles_at(const AttCall &a, const Entry &e) { return (int)(((uint32_t)e.rows + (1u << a.tile_shift) - 1) >> a.tile_shift); }
// (tiles: their number so far, as far as it matters: up to the CTAs of a launch)
__device__ __forceinline__ int64_t units_at(const AttCall &a, const Entry &e, int &tiles)
{
    const int64_t mine = (int64_t)tiles_at(a, e) * a.c.heads;
    tiles = min(tiles + (int)min(mine, (int64_t)1024), 1024);
    return mine * blocks_at(a, e);
}

// Where a CTA's units begin: entry, tile (head, then tile of query rows) and block in it.
struct Cursor {
    int32_t i, head, row_tile, block;
    Entry e;
    int32_t row_tiles, blocks;   // of the entry (tiles of one head)
};

// Shared memory of the division.
template <int THREADS>
struct PlanShared {
    int64_t sum[THREADS];   // units before the sequences of every thread
};

// Elements before row rr (query x group) of head `head` of the cache, for a sequence whose first query row is row0, in q or out.
__device__ __forceinline__ int64_t row_at(const AttCall &a, int64_t row0, int head, int rr, int64_t stride, int d)
{
    const int query = (int)a.by_group.div((uint32_t)rr);
    return (row0 + query) * stride + (head * a.group + rr - query * a.group) * d;
}

// x / y for y > 0: in 32 bits where that does (a 64-bit division costs some hundred cycles).
__device__ __forceinline__ int64_t divide(int64_t x, int64_t y)
{
    if (((x | y) >> 32) == 0) return (uint32_t)x / (uint32_t)y;
    return x / y;
}
// First unit of CTA c of `ctas`: an even share of `total`.
__device__ __forceinline__ int64_t cut(int64_t total, int ctas, int c)
{
    if (total < (int64_t)1 << 22) return (uint32_t)total * (uint32_t)c / (uint32_t)ctas;   // (ctas <= 444)
    const int64_t each = divide(total, ctas);
    return each * c + divide((total - each * ctas) * c, ctas);
}

// What a CTA of the launch has to do: the units [u0, u1), the first of them at `cur`.  total 0: nothing for anybody.
struct Share {
    int64_t total, u0, u1;
    int32_t ctas;
    Cursor cur;
};

__device__ __forceinline__ bool offsets_ok(const AttCall &a, int i)
{
    if (!a.offsets) return true;
    const int64_t o = a.offsets[i], o1 = a.offsets[i + 1];
    return o >= 0 && o1 >= o && o1 <= a.rows;
}

// All threads.  Up to 128 sequences every warp works it out by itself, four to a lane; beyond that the threads of the CTA share them.
template <int THREADS>
__device__ Share plan_share(const AttCall &a, PlanShared<THREADS> &s)
{
    const int tid = threadIdx.x, lane = tid & 31, cta = blockIdx.x;
    const bool few = a.n <= 128;
    const int per = few ? (a.n + 31) >> 5 : (a.n + THREADS - 1) / THREADS, first = (few ? lane : tid) * per;
    int64_t mine = 0, unit[4] = {0, 0, 0, 0};
    bool bad = false;
    int tiles = 0;
    if (few) {
#pragma unroll
        for (int j = 0; j < 4; ++j) {
            const int i = first + j;
            if (j < per && i < a.n) {
                if (offsets_ok(a, i)) unit[j] = units_at(a, entry_at(a, i), tiles);
                else bad = true;
            }
            mine += unit[j];
        }
    } else {
#pragma unroll 4
        for (int i = first; i < min(a.n, first + per); ++i) {
            if (offsets_ok(a, i)) mine += units_at(a, entry_at(a, i), tiles);
            else bad = true;
        }
    }
    int64_t x = mine;
#pragma unroll
    for (int o = 1; o < 32; o <<= 1) {
        const int64_t y = __shfl_up_sync(0xffffffffu, x, o);
        if (lane >= o) x += y;
    }
    int64_t base = x - mine;
    Share h;
    if (few) {
        h.total = __shfl_sync(0xffffffffu, x, 31);
        bad = __any_sync(0xffffffffu, bad);
        tiles = __reduce_add_sync(0xffffffffu, tiles);
    } else {
        __shared__ int64_t warp_sum[THREADS / 32];
        __shared__ int warp_tiles[THREADS / 32];
        tiles = __reduce_add_sync(0xffffffffu, tiles);
        if (lane == 31) warp_sum[tid >> 5] = x, warp_tiles[tid >> 5] = tiles;
        bad = __syncthreads_or(bad) != 0;
        int64_t before = 0;
        h.total = 0, tiles = 0;
        for (int w = 0; w < THREADS / 32; ++w) {
            if (w < (tid >> 5)) before += warp_sum[w];
            h.total += warp_sum[w], tiles += warp_tiles[w];
        }
        base += before;
        s.sum[tid] = base;
        __syncthreads();
    }
    h.u0 = h.u1 = 0, h.ctas = 1, h.cur = Cursor{};
    if (bad) {
        h.total = 0;
        if (tid == 0 && cta == 0) atomicOr(a.c.status, AIF_STATUS_BAD_ID);
    }
    if (h.total == 0) return h;
    // a CTA has min_units on average at least, or as many as a tile has: tiles beside each other cost nothing to part (148 tiles of one block: 13 us against 35)
    h.ctas = (int)min((int64_t)gridDim.x, max((int64_t)tiles, a.min_units == 1 ? h.total : divide(h.total, a.min_units)));
    if (cta >= h.ctas) return h;
    h.u0 = cut(h.total, h.ctas, cta), h.u1 = cut(h.total, h.ctas, cta + 1);
    // the sequence of unit u0
    int i;
    int64_t left;
    if (few) {
        left = h.u0 - base, i = first;
        const int who = __ffs(__ballot_sync(0xffffffffu, left >= 0 && left < mine)) - 1;
#pragma unroll
        for (int j = 0; j < 3; ++j)
            if (i == first + j && left >= unit[j]) left -= unit[j], ++i;
        i = __shfl_sync(0xffffffffu, i, who), left = __shfl_sync(0xffffffffu, left, who);
    } else {
        int lo = 0, hi = THREADS;   // the last thread whose sequences begin at or before u0
        while (hi - lo > 1) {
            const int mid = (lo + hi) >> 1;
            if (s.sum[mid] <= h.u0) lo = mid;
            else hi = mid;
        }
        i = lo * per, left = h.u0 - s.sum[lo];
        for (; i < a.n - 1; ++i) {
            const int64_t has = units_at(a, entry_at(a, i), tiles);
            if (left < has) break;
            left -= has;
        }
    }
    Cursor &c = h.cur;
    c.i = i, c.e = entry_at(a, i);
    c.row_tiles = tiles_at(a, c.e), c.blocks = blocks_at(a, c.e);
    const int tile = (int)divide(left, c.blocks);
    c.block = (int)(left - (int64_t)tile * c.blocks);
    c.head = a.c.heads == 1 ? 0 : tile / c.row_tiles, c.row_tile = tile - c.head * c.row_tiles;
    return h;
}
// To the next tile (block 0 of it).
__device__ __forceinline__ void plan_next(const AttCall &a, Cursor &c)
{
    c.block = 0;
    if (++c.row_tile < c.row_tiles) return;
    c.row_tile = 0;
    if (++c.head < a.c.heads) return;
    c.head = 0;
    do {
        if (++c.i >= a.n) return;
        c.e = entry_at(a, c.i);
        c.row_tiles = tiles_at(a, c.e);
    } while (c.row_tiles == 0);
    c.blocks = blocks_at(a, c.e);
}

}  // namespace
}  // namespace aif
