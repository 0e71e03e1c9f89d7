// Attention of query rows over sequences in the 4-bit cache: the CUDA-core kernel (fp32 models, and few rows per sequence, where the
// work is to read the cache once), the kernel that joins pieces, and the entry points.
//
// k_att4_rows: R query rows of a sequence against all its visible keys.  A warp takes stages of a few groups of 16 rows (a group lies in one page: its
// codes and scales are two contiguous pieces), copied asynchronously into a ring of its own in shared memory, three stages ahead of
// the one at work.  A key row is spread over P lanes (32 of its elements, one block, to a lane for one query row; 16 elements where R rows share the decoding), 32 / P
// keys to a step, each key group of lanes with a running maximum, weight and sum of its own, so a step needs no exchange but the score's sum over P lanes.
// Codes are decoded once for score and sum where values are the keys; sums are fp32 throughout (f32x2 fused multiply-adds on register pairs).
// Bound: issue slots (about three instructions per element of one row; 55 % of them taken, HBM 19 %).  256 sequences of 10^4 rows: fp32 d = 128 161 us, bf16 d = 96 117 us.
// Many rows are not what it is for: keys are decoded again for every four rows, a CTA's tiles follow one another with nothing in flight between them, and the four-row forms spill
// (334 to 554 bytes of stores a thread at 168 registers; the one-row forms spill nothing).  fp32, d = 64, one sequence of 50 keys: 1000 rows 10.9 us, 10^4 44 us,
// 10^5 386 us; bf16, d = 96, 16 x 1000 rows x 10^4 keys 5.0 ms.
#include <algorithm>
#include <cfloat>
#include <cstdio>

#include "aif_cache4_plan.cuh"
#include "aif_tc_ptx.cuh"

namespace aif {
namespace {

constexpr int kRowThreads = 128;
constexpr int kRowWarps = kRowThreads / 32;
constexpr int kRing = 4;           // stages of a warp's ring
constexpr int kRowGroups = 16;     // groups of 16 rows of a unit

__device__ __forceinline__ uint64_t mul_f32x2(uint64_t a, uint64_t b)
{
    uint64_t d;
    asm("mul.rn.f32x2 %0, %1, %2;" : "=l"(d) : "l"(a), "l"(b));
    return d;
}

template <int R, int P>
struct RowsCfg {
    static constexpr int E = R == 1 ? 32 : 16;                     // elements of a lane
    static constexpr int KS = 32 / P;                              // keys of a step
    static constexpr int kKeys = 4 * KS > 16 ? 4 * KS : 16;        // keys of a stage
    static constexpr int kGroups = kKeys / 16;
};

template <typename T, int R, int P, bool SHARED>
__global__ void __launch_bounds__(kRowThreads, 3) k_att4_rows(const AttCall a)
{
    using C = RowsCfg<R, P>;
    constexpr int E = C::E, KS = C::KS, W = E / 8, kKinds = SHARED ? 1 : 2;   // W: code words of a lane
    const Cache4 &c = a.c;
    const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5, d = c.d, nb = d >> 5;
    const int part = lane % P, sub = lane / P;
    const bool act = part * E < d;
    extern __shared__ __align__(16) unsigned char smem[];   // rings [warps][kRing][kKinds][codes, scales]; then sums [warps][R][d + 2]
    const int stage_bytes = C::kKeys * (d / 2 + nb);
    unsigned char *ring = smem + warp * (kRing * kKinds) * stage_bytes;
    float *sums = reinterpret_cast<float *>(smem + kRowWarps * (kRing * kKinds) * stage_bytes);
    __shared__ PlanShared<kRowThreads> plan;

    grid_dep_wait();
    grid_dep_launch();
    const int cta = blockIdx.x;
    if (tid == 0 && a.headers) a.headers[cta].first_cta = -1;
    const Share share = plan_share(a, plan);
    if (share.u0 >= share.u1) return;
    const int64_t total = share.total, u1 = share.u1;
    const int ctas = share.ctas;
    int64_t u = share.u0;
    Cursor cur = share.cur;
    const int d2 = d + 2;
    bool bad_page = false;
    while (u < u1) {
        const Entry &e = cur.e;
        const int head = cur.head, r0 = cur.row_tile * R, rows = min(R, e.rows - r0);
        const int64_t tile_u0 = u - cur.block;
        const int take = (int)min(u1 - u, (int64_t)(cur.blocks - cur.block));
        const int groups = e.groups(), g0 = cur.block * kRowGroups, g1 = min(groups, (cur.block + take) * kRowGroups);
        const int sink_groups = e.sink_groups(), rest_group = (e.rest >> 4) - sink_groups;
        const int32_t *table = c.table + (size_t)max(e.seq, 0) * c.max_pages;

        // the stage that begins with group `grp` into slot `slot` of the ring
        auto bring = [&](int grp, int slot) {
#pragma unroll
            for (int x = 0; x < C::kGroups; ++x) {
                const int gi = grp + x;
                if (gi >= g1) break;
                const int row = (gi < sink_groups ? gi : gi + rest_group) << 4, page = __ldg(table + (row >> c.page_shift));
                const bool ok = c.holds(page);
                bad_page |= !ok;
                const size_t at = c.row(ok ? page : 0, head, row & (c.page_rows() - 1));
#pragma unroll
                for (int k = 0; k < kKinds; ++k) {
                    unsigned char *codes = ring + (slot * kKinds + k) * stage_bytes + x * 16 * (d / 2), *scales = ring + (slot * kKinds + k) * stage_bytes + C::kKeys * (d / 2) + x * 16 * nb;
                    const uint8_t *from = c.codes[k] + at * (d / 2);
                    for (int y = lane; y < 16 * nb; y += 32) cp_async16(smem_u32(codes + y * 16), from + y * 16, 16u);
                    if (ok) {
                        if (lane < nb) cp_async16(smem_u32(scales + lane * 16), c.scales[k] + at * nb + lane * 16, 16u);
                    } else {   // no such page: no number
                        for (int y = lane; y < 16 * nb; y += 32) scales[y] = (unsigned char)kMxNan;
                    }
                }
            }
            cp_async_commit();
        };
        const int first = g0 + warp * C::kGroups;
        constexpr int kStride = kRowWarps * C::kGroups;
#pragma unroll
        for (int i = 0; i < kRing - 1; ++i) {
            if (first + i * kStride < g1) bring(first + i * kStride, i);
            else cp_async_commit();
        }

        uint64_t q[R][E / 2], o[R][E / 2];
        float m[R], l[R];
#pragma unroll
        for (int r = 0; r < R; ++r) {
            m[r] = -FLT_MAX, l[r] = 0.f;
            const T *src = static_cast<const T *>(a.q) + row_at(a, e.row0, head, min(r, rows - 1) + r0, a.q_stride, d) + part * E;
#pragma unroll
            for (int w = 0; w < W; ++w) {
                float v[8] = {};
                if (act) load8<T, true>(src + w * 8, v);
#pragma unroll
                for (int i = 0; i < 4; ++i) q[r][w * 4 + i] = pack_f32x2(v[2 * i] * a.scale_log2, v[2 * i + 1] * a.scale_log2), o[r][w * 4 + i] = 0ull;
            }
        }
        int slot = 0;
        for (int grp = first; grp < g1; grp += kStride) {
            // (the slot that is filled now was read a whole stage ago)
            const int ahead = grp + (kRing - 1) * kStride;
            if (ahead < g1) bring(ahead, (slot + kRing - 1) % kRing);
            else cp_async_commit();
            cp_async_wait<kRing - 1>();
            __syncwarp();
            const unsigned char *codes = ring + slot * kKinds * stage_bytes, *scales = codes + C::kKeys * (d / 2);
#pragma unroll
            for (int s = 0; s < C::kKeys / KS; ++s) {
                const int k = s * KS + sub, gi = grp + (k >> 4);
                const int row = ((gi < sink_groups ? gi : gi + rest_group) << 4) + (k & 15);
                const bool there = gi < g1 && (gi < sink_groups ? row < e.first : row >= e.rest && row < e.length);
                uint64_t val[E / 2];
                auto decode = [&](const unsigned char *from) {
                    uint32_t w[W];
                    if constexpr (W == 4) {
                        const uint4 x = *reinterpret_cast<const uint4 *>(from);
                        w[0] = x.x, w[1] = x.y, w[2] = x.z, w[3] = x.w;
                    } else {
                        const uint2 x = *reinterpret_cast<const uint2 *>(from);
                        w[0] = x.x, w[1] = x.y;
                    }
#pragma unroll
                    for (int i = 0; i < W; ++i) {
                        uint32_t h[4];
                        mx_decode8_f16(w[i], h);
#pragma unroll
                        for (int j = 0; j < 4; ++j) {
                            const float2 f = half2_to_float2(h[j]);
                            val[i * 4 + j] = pack_f32x2(f.x, f.y);
                        }
                    }
                };
                const int cell = k * (d / 2) + (act ? part * (E / 2) : 0), cell_scale = k * nb + (act ? part * E / 32 : 0);
                decode(codes + cell);
                float scale = there && act ? mx_scale(scales[cell_scale]) : 0.f;   // (what is not there has finite codes and no scale)
                float pr[R];
                bool raise = false;
#pragma unroll
                for (int r = 0; r < R; ++r) {
                    uint64_t acc[2] = {0ull, 0ull};
#pragma unroll
                    for (int i = 0; i < E / 2; ++i) acc[i & 1] = fma_f32x2(val[i], q[r][i], acc[i & 1]);
                    float x, y;
                    unpack_f32x2(add_f32x2(acc[0], acc[1]), x, y);
                    float sc = (x + y) * scale;
#pragma unroll
                    for (int b = 1; b < P; b <<= 1) sc += __shfl_xor_sync(0xffffffffu, sc, b);
                    pr[r] = there ? sc : -INFINITY;
                    raise |= pr[r] > m[r] + 8.f;
                }
                // the offset of the exponent follows the maximum only when that has grown by a factor of 2^8
                if (__any_sync(0xffffffffu, raise)) {
#pragma unroll
                    for (int r = 0; r < R; ++r) {
                        const float mn = pr[r] > m[r] + 8.f ? pr[r] : m[r], f = fast_exp2(m[r] - mn);
                        m[r] = mn, l[r] *= f;
                        const uint64_t ff = pack_f32x2(f, f);
#pragma unroll
                        for (int i = 0; i < E / 2; ++i) o[r][i] = mul_f32x2(o[r][i], ff);
                    }
                }
                if constexpr (!SHARED) {
                    decode(codes + stage_bytes + cell);
                    scale = there && act ? mx_scale(scales[stage_bytes + cell_scale]) : 0.f;
                }
#pragma unroll
                for (int r = 0; r < R; ++r) {
                    const float pe = fast_exp2(pr[r] - m[r]);
                    l[r] += pe;
                    const uint64_t pp = pack_f32x2(pe * scale, pe * scale);
#pragma unroll
                    for (int i = 0; i < E / 2; ++i) o[r][i] = fma_f32x2(val[i], pp, o[r][i]);
                }
            }
            __syncwarp();
            slot = (slot + 1) % kRing;
        }
        cp_async_wait_all();
        // key groups of the warp, then the warps
#pragma unroll
        for (int r = 0; r < R; ++r) {
            float mt = m[r];
#pragma unroll
            for (int b = P; b < 32; b <<= 1) mt = fmaxf(mt, __shfl_xor_sync(0xffffffffu, mt, b));
            const float f = fast_exp2(m[r] - mt);
            float lt = l[r] * f;
#pragma unroll
            for (int b = P; b < 32; b <<= 1) lt += __shfl_xor_sync(0xffffffffu, lt, b);
            float *to = sums + (warp * R + r) * d2;
#pragma unroll
            for (int i = 0; i < E / 2; ++i) {
                float x, y;
                unpack_f32x2(o[r][i], x, y);
                x *= f, y *= f;
#pragma unroll
                for (int b = P; b < 32; b <<= 1) x += __shfl_xor_sync(0xffffffffu, x, b), y += __shfl_xor_sync(0xffffffffu, y, b);
                if (sub == 0 && act) to[part * E + 2 * i] = x, to[part * E + 2 * i + 1] = y;
            }
            if (lane == 0) to[d] = mt, to[d + 1] = lt;
        }
        __syncthreads();
        const bool begins = cur.block == 0, ends = cur.block + take == cur.blocks;
        float *rec = a.records + (size_t)(2 * cta + (begins ? 1 : 0)) * R * d2;
        for (int x = tid; x < rows * d; x += kRowThreads) {
            const int r = x / d, col = x - r * d;
            float mt = -FLT_MAX, sum = 0.f, weight = 0.f;
#pragma unroll
            for (int w = 0; w < kRowWarps; ++w) mt = fmaxf(mt, sums[(w * R + r) * d2 + d]);
#pragma unroll
            for (int w = 0; w < kRowWarps; ++w) {
                const float *from = sums + (w * R + r) * d2;
                const float f = fast_exp2(from[d] - mt);
                sum += from[col] * f, weight += from[d + 1] * f;
            }
            if (begins && ends) {
                T *dst = static_cast<T *>(a.out) + row_at(a, e.row0, head, r0 + r, a.out_stride, d) + col;
                // (no keys: a zero row; a bad sequence: no number)
                *dst = (T)(e.length < 0 ? NAN : groups == 0 ? 0.f : sum / weight);
            } else {
                rec[r * d + col] = sum;
                if (col == 0) rec[R * d + 2 * r] = mt, rec[R * d + 2 * r + 1] = weight;
            }
        }
        if (ends && !begins && tid == 0) {
            int s = cta;
            while (s > 0 && cut(total, ctas, s) > tile_u0) --s;
            PieceHeader h{};
            h.row0 = e.row0, h.first_cta = s, h.head = head, h.r0 = r0, h.rows = rows;
            a.headers[cta] = h;
        }
        if (e.length < 0 && tid == 0) atomicOr(c.status, AIF_STATUS_BAD_ID);
        u += take;
        if (u < u1) plan_next(a, cur);
        __syncthreads();   // the warps' sums are read: the next tile may write them
    }
    if (bad_page) atomicOr(c.status, AIF_STATUS_BAD_ID);
}

// Tiles that were cut, one per CTA of the attention kernel at most: sums of the pieces, brought to one offset, over their weights.  Block (c, y) has eight
// rows of the tile that ended in CTA c, a warp to a row; where a tile has fewer rows, several warps share the pieces of one.
constexpr int kJoinPieces = 448;   // most CTAs of an attention kernel, so most pieces of a tile
template <typename T>
__global__ void __launch_bounds__(256) k_att4_join(const AttCall a, int permuted)
{
    grid_dep_wait();
    grid_dep_launch();
    const PieceHeader h = a.headers[blockIdx.x];
    const int first_row = blockIdx.y * 8;
    if (h.first_cta < 0 || first_row >= h.rows) return;
    __shared__ float factor[8][kJoinPieces];
    __shared__ float4 part_sum[8][32];
    const int d = a.c.d, pieces = (int)blockIdx.x - h.first_cta + 1, warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
    const int rows = min(8, h.rows - first_row);
    int share = 1;   // warps to a row
    while (share * 2 * rows <= 8) share *= 2;
    const int r = first_row + warp / share, part = warp % share;
    const bool work = warp < rows * share;
    const size_t record = (size_t)a.tile_rows * (d + 2);
    // the piece of CTA first_cta is the beginning of a tile, the others are continuations
    auto piece = [&](int p) { return a.records + (size_t)(2 * (h.first_cta + p) + (p == 0)) * record; };
    float weight = 0.f;
    if (work) {
        float mt = -FLT_MAX;
        for (int p = lane; p < pieces; p += 32) mt = fmaxf(mt, piece(p)[(size_t)a.tile_rows * d + 2 * r]);
#pragma unroll
        for (int b = 16; b > 0; b >>= 1) mt = fmaxf(mt, __shfl_xor_sync(0xffffffffu, mt, b));
        for (int p = lane; p < pieces; p += 32) {
            const float *st = piece(p) + (size_t)a.tile_rows * d + 2 * r;
            const float f = fast_exp2(st[0] - mt);
            factor[warp][p] = f, weight += st[1] * f;
        }
#pragma unroll
        for (int b = 16; b > 0; b >>= 1) weight += __shfl_xor_sync(0xffffffffu, weight, b);
    }
    __syncwarp();
#pragma unroll 1
    for (int col0 = 0; col0 < d; col0 += 128) {
        const int col = col0 + lane * 4;   // of the records: the tensor-core kernels' sums stand in the order of the unpacked codes
        float4 sum = make_float4(0.f, 0.f, 0.f, 0.f);
        if (work && col < d) {
#pragma unroll 4
            for (int p = part; p < pieces; p += share) {
                const float2 x = *reinterpret_cast<const float2 *>(piece(p) + (size_t)r * d + col), y = *reinterpret_cast<const float2 *>(piece(p) + (size_t)r * d + col + 2);
                const float f = factor[warp][p];
                sum.x += x.x * f, sum.y += x.y * f, sum.z += y.x * f, sum.w += y.y * f;
            }
        }
        if (share > 1) {
            part_sum[warp][lane] = sum;
            __syncthreads();
            if (work && part == 0) {
                for (int w = 1; w < share; ++w) {
                    const float4 o = part_sum[warp + w][lane];
                    sum.x += o.x, sum.y += o.y, sum.z += o.z, sum.w += o.w;
                }
            }
            __syncthreads();
        }
        if (work && part == 0 && col < d) {
            T *dst = static_cast<T *>(a.out) + row_at(a, h.row0, h.head, h.r0 + r, a.out_stride, d);
            const float v[4] = {sum.x, sum.y, sum.z, sum.w};
#pragma unroll
            for (int i = 0; i < 4; ++i) {
                const int at = col + i, to = permuted ? (at & ~7) | ((at & 1) << 2) | ((at >> 1) & 3) : at;   // 0, 4, 1, 5, 2, 6, 3, 7
                dst[to] = (T)(v[i] / weight);
            }
        }
    }
}

bool at16(const void *p) { return (reinterpret_cast<uintptr_t>(p) & 15) == 0; }

template <typename T, int R, int P, bool SHARED>
cudaError_t run_rows_at(const AttCall &a, int grid, cudaStream_t st)
{
    const size_t smem = (size_t)kRowWarps * kRing * (SHARED ? 1 : 2) * RowsCfg<R, P>::kKeys * (a.c.d / 2 + a.c.d / 32) + (size_t)kRowWarps * R * (a.c.d + 2) * 4;
    if (smem > 48 * 1024) {
        const cudaError_t e = allow_smem<k_att4_rows<T, R, P, SHARED>>(200 * 1024);
        if (e != cudaSuccess) return e;
    }
    count_launch();
    return launch_pdl(k_att4_rows<T, R, P, SHARED>, dim3(grid), dim3(kRowThreads), smem, st, a);
}
template <typename T, int R, bool SHARED>
cudaError_t run_rows(const AttCall &a, int grid, cudaStream_t st)
{
    constexpr int kF = R == 1 ? 1 : 2;   // lanes to a block of 32 elements
    const int blocks = a.c.d / 32;
    if (blocks <= 1) return run_rows_at<T, R, kF, SHARED>(a, grid, st);
    if (blocks <= 2) return run_rows_at<T, R, 2 * kF, SHARED>(a, grid, st);
    if (blocks <= 4) return run_rows_at<T, R, 4 * kF, SHARED>(a, grid, st);
    return run_rows_at<T, R, 8 * kF, SHARED>(a, grid, st);
}

// How a call is run: which kernel, and how far it may be cut.
struct AttForm {
    enum { kRows, kFew, kPair, kTensor } kernel;
    int tile_rows, block_keys;   // powers of two; block_keys < 0: that many groups of 16 rows
    int grid, min_units;
    bool cut;   // a tile may have several units, and so be cut between CTAs
};
// The tensor-core kernels: pieces of a cut tile have eight blocks (of some 1.2 us) on average at least, since a piece costs its queries, its record and its part of the join: 16
// sequences of 1000 rows with 1000 keys (d = 128) 35 us against 45 with pieces of four, 64 of 128 rows with 1000 keys (d = 256) 37 us against 60; one of 256 rows with 1000
// keys 28 us against 25.
// Few or many rows, at 32 (the lengths are on the device): where the border would be best depends on what the call fills.  us of the kernel of few rows and of the one of many, on one box:
//   rows per sequence          16          32          64
//   16 x 1000 keys, d = 128    12.4  20.2  14.3  20.2  19.9  21.0
//   16 x 10^4, d = 128         26.7  32.4  36.4  32.9  58.6  34.5
//   148 x 10^4, d = 128        112   149   209   149   405   148
//   148 x 10^4, d = 64         72    121   134   121   259   121
//   148 x 10^4, d = 256        195   207   384   208   759   210
//   148 x 10^4, d = 128, own   180   171   340   171   664   172
//   1 x 1000, d = 128          10.7  19.5  10.8  19.8  10.8  20.2
AttForm kernel_of(const aif_cache4 *c, const aif_cache4_query *q)
{
    const int64_t group = q->n_heads / c->heads, per_seq = (q->rows + q->n - 1) / q->n * group;   // query rows of a sequence and a head of the cache, on average
    const bool bf = q->dtype == AIF_BF16;
    if (bf && per_seq > 32 && (c->d == 64 || c->d == 128)) return {AttForm::kPair, 256, 64, 148, 8};
    if (bf && per_seq > 32 && c->d == 256) return {AttForm::kTensor, 128, 64, 148, 8};
    if (bf && (c->d == 32 || c->d == 64 || c->d == 128 || c->d == 256)) return {AttForm::kFew, 8, -16, c->d == 256 ? 296 : 444, 1};
    return {AttForm::kRows, per_seq <= 2 ? 1 : 4, -kRowGroups, 444, 1};
}
AttForm form_of(const aif_cache4 *c, const aif_cache4_query *q)
{
    AttForm f = kernel_of(c, q);
    // most rows that a sequence can show: what its pages hold, or the window and the first rows (which may begin inside a group of 16)
    int64_t most = (int64_t)c->max_pages * c->page_rows;
    if (q->window > 0) most = std::min<int64_t>(most, (int64_t)q->window + q->sinks + 32);
    f.cut = most > (f.block_keys > 0 ? f.block_keys : -16 * f.block_keys);
    return f;
}
int64_t workspace_of(const AttForm &f, const aif_cache4 *c)
{
    return f.cut ? (int64_t)f.grid * (int64_t)sizeof(PieceHeader) + 2ll * f.grid * f.tile_rows * (c->d + 2) * 4 : 0;
}

int check_query(const aif_cache4 *c, const aif_cache4_query *q)
{
    const int rc = cache4_check(c);
    if (rc != AIF_OK) return rc;
    if (!q || q->struct_size != sizeof(aif_cache4_query)) return AIF_ERR_ARG;
    if (q->dtype != AIF_F32 && q->dtype != AIF_BF16) return AIF_ERR_ARG;
    if (q->n < 0 || q->rows < 0 || q->n_heads < 1 || q->n_heads % c->heads != 0 || q->n_heads / c->heads > 64) return AIF_ERR_SHAPE;
    if (!q->offsets && q->rows != q->n) return AIF_ERR_SHAPE;
    if (!q->seq_ids && q->n > c->n_seqs) return AIF_ERR_SHAPE;
    if (q->rows > INT_MAX / 64) return AIF_ERR_SHAPE;
    const int64_t width = (int64_t)q->n_heads * c->d, el = q->dtype == AIF_BF16 ? 2 : 4;
    if (q->q_stride < width || q->out_stride < width || q->q_stride * el % 16 != 0 || q->out_stride * el % 16 != 0) return AIF_ERR_SHAPE;
    if (q->window < 0 || q->sinks < 0) return AIF_ERR_SHAPE;
    if (!(q->scale >= 0.f) || q->scale - q->scale != 0.f) return AIF_ERR_ARG;   // (NaN, infinite)
    return AIF_OK;
}

}  // namespace
}  // namespace aif

using namespace aif;

extern "C" {

int64_t aif_cache4_attention_workspace(const aif_cache4 *c, const aif_cache4_query *q)
{
    const int rc = check_query(c, q);
    if (rc != AIF_OK) return rc;
    return q->n == 0 || q->rows == 0 ? 0 : workspace_of(form_of(c, q), c);
}

int aif_cache4_attention(const aif_cache4 *c, const aif_cache4_query *q, aif_stream stream)
{
    StageRange range("aif_cache4_attention");
    const int rc = check_query(c, q);
    if (rc != AIF_OK) return rc;
    if (q->n == 0 || q->rows == 0) return AIF_OK;
    if (!q->q || !q->out || !at16(q->q) || !at16(q->out)) return AIF_ERR_ARG;
    const AttForm f = form_of(c, q);
    if (f.cut && (!q->workspace || !at16(q->workspace) || q->workspace_bytes < workspace_of(f, c))) return AIF_ERR_ARG;
    cudaStream_t st = reinterpret_cast<cudaStream_t>(stream);
    AttCall a{};
    a.c = cache4_of(c), a.n = q->n, a.n_heads = q->n_heads, a.group = q->n_heads / c->heads, a.by_group = FastDiv::of((uint32_t)a.group), a.seq_ids = q->seq_ids, a.offsets = q->offsets;
    a.rows = q->rows, a.q = q->q, a.out = q->out, a.q_stride = q->q_stride, a.out_stride = q->out_stride;
    a.scale_log2 = 1.4426950408889634f * (q->scale == 0.f ? 1.0f / sqrtf((float)c->d) : q->scale);
    a.window = q->window, a.sinks = q->sinks, a.tile_rows = f.tile_rows, a.min_units = f.min_units;
    a.in_groups = f.block_keys < 0, a.tile_shift = __builtin_ctz((unsigned)f.tile_rows), a.block_shift = __builtin_ctz((unsigned)std::abs(f.block_keys));
    if (f.cut) a.headers = static_cast<PieceHeader *>(q->workspace), a.records = reinterpret_cast<float *>(a.headers + f.grid);
    const bool bf = q->dtype == AIF_BF16, shared = c->shared != 0;
    cudaError_t e;
    if (f.kernel == AttForm::kPair) e = launch_att4_pair(a, f.grid, st);
    else if (f.kernel == AttForm::kTensor) e = launch_att4_tc(a, f.grid, st);
    else if (f.kernel == AttForm::kFew) e = launch_att4_few(a, f.grid, st);
    else if (f.tile_rows == 1)
        e = bf ? (shared ? run_rows<__nv_bfloat16, 1, true>(a, f.grid, st) : run_rows<__nv_bfloat16, 1, false>(a, f.grid, st))
               : (shared ? run_rows<float, 1, true>(a, f.grid, st) : run_rows<float, 1, false>(a, f.grid, st));
    else
        e = bf ? (shared ? run_rows<__nv_bfloat16, 4, true>(a, f.grid, st) : run_rows<__nv_bfloat16, 4, false>(a, f.grid, st))
               : (shared ? run_rows<float, 4, true>(a, f.grid, st) : run_rows<float, 4, false>(a, f.grid, st));
    if (e == cudaSuccess && f.cut) {
        const bool tensor = f.kernel == AttForm::kPair || f.kernel == AttForm::kTensor;
        const dim3 grid(f.grid, (f.tile_rows + 7) / 8);
        e = bf ? launch_pdl(k_att4_join<__nv_bfloat16>, grid, dim3(256), 0, st, a, tensor ? 1 : 0) : launch_pdl(k_att4_join<float>, grid, dim3(256), 0, st, a, 0);
        count_launch();
    }
    return cache4_failed(e, "aif_cache4_attention");
}

}  // extern "C"
