// Attention of query rows over sequences in the 4-bit cache: the CUDA-core kernel (fp32 models, and few rows per sequence, where the
// work is to read the cache once), the kernel that joins pieces, and the entry points.
//
// k_att4_rows: R query rows of a sequence against all its visible keys.  A key row is spread over P lanes (32 of its elements, one block, to a lane for one
// query row; 16 elements where R rows share the decoding), 32 / P keys to a warp step, each key group of lanes with a running maximum, weight and sum of its
// own, so a step needs no exchange but the score's sum over P lanes.  Codes are decoded once for score and sum where values are the keys;
// sums are fp32 throughout (f32x2 fused multiply-adds).  Codes and scales of a warp's next steps are in flight in registers while one is at work.
// Bound: HBM (17/32 byte per element) or issue slots (2.5 instructions per element and row).
#include <algorithm>
#include <cfloat>
#include <cstdio>

#include "aif_cache4_plan.cuh"
#include "aif_tc_ptx.cuh"

namespace aif {
namespace {

constexpr int kRowThreads = 256;
constexpr int kRowWarps = kRowThreads / 32;
constexpr int kSteps = 4;          // steps whose codes a warp loads at a time
constexpr int kRowBlock = 256;     // visible keys of a unit

template <typename T>
__device__ __forceinline__ float to_f32(T x) { return (float)x; }

template <typename T, int R, int P, bool SHARED>
__global__ void __launch_bounds__(kRowThreads, R == 1 ? 2 : 1) k_att4_rows(const AttCall a)
{
    constexpr int E = R == 1 ? 32 : 16;   // elements of a lane
    constexpr int KS = 32 / P;            // keys of a step
    constexpr int W = E / 8;              // code words of a lane
    const Cache4 &c = a.c;
    const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5;
    const int part = lane % P, sub = lane / P;
    const bool act = part * E < c.d;
    extern __shared__ float smem[];   // [warps][R][d + 2]
    __shared__ PlanShared<kRowThreads> plan;

    grid_dep_wait();
    grid_dep_launch();
    const int64_t total = plan_total(a, plan);
    const int ctas = (int)min((int64_t)gridDim.x, max((int64_t)1, total / a.min_units));
    const int cta = blockIdx.x;
    if (tid == 0) a.headers[cta].first_cta = -1;
    if (total == 0 || cta >= ctas) return;
    const int64_t u1 = cut(total, ctas, cta + 1);
    int64_t u = cut(total, ctas, cta);
    Cursor cur = plan_find(a, plan, u);
    const int d2 = c.d + 2;
    bool bad_page = false;
    while (u < u1) {
        const Entry &e = cur.e;
        const int row_tiles = cur.tiles / c.heads, head = cur.tile / row_tiles, r0 = (cur.tile - head * row_tiles) * R, rows = min(R, e.rows - r0);
        const int64_t tile_u0 = u - cur.block;
        const int take = (int)min(u1 - u, (int64_t)(cur.blocks - cur.block));
        const int keys = e.keys(), k0 = cur.block * kRowBlock, k1 = min(keys, (cur.block + take) * kRowBlock);

        float2 q[R][E / 2], o[R][E / 2];
        float m[R], l[R];
#pragma unroll
        for (int r = 0; r < R; ++r) {
            m[r] = -FLT_MAX, l[r] = 0.f;
            const int rr = min(r, rows - 1) + r0, query = rr / a.group;
            const T *src = static_cast<const T *>(a.q) + (e.row0 + query) * a.q_stride + (head * a.group + rr - query * a.group) * c.d + part * E;
#pragma unroll
            for (int w = 0; w < W; ++w) {
                float v[8] = {};
                if (act) load8<T, true>(src + w * 8, v);
#pragma unroll
                for (int i = 0; i < 4; ++i) {
                    q[r][w * 4 + i] = make_float2(v[2 * i] * a.scale_log2, v[2 * i + 1] * a.scale_log2);
                    o[r][w * 4 + i] = make_float2(0.f, 0.f);
                }
            }
        }
        const int32_t *table = c.table + (size_t)max(e.seq, 0) * c.max_pages;
        constexpr int kChunk = kSteps * KS;

        uint32_t kc[kSteps][W], vc[SHARED ? 1 : kSteps][W];
        float ks[kSteps], vs[SHARED ? 1 : kSteps];
        auto fetch = [&](int v0) {   // codes and scales of the chunk at visible key v0 (zero weight and zero codes behind the end)
#pragma unroll
            for (int s = 0; s < kSteps; ++s) {
                const int v = v0 + s * KS + sub;
#pragma unroll
                for (int w = 0; w < W; ++w) kc[s][w] = 0u;
                ks[s] = 0.f;
                if (!SHARED) {
#pragma unroll
                    for (int w = 0; w < W; ++w) vc[s][w] = 0u;
                    vs[s] = 0.f;
                }
                if (v >= k1 || !act) continue;
                const int key = e.key(v), page = __ldg(table + (key >> c.page_shift));
                if (!c.holds(page)) {
                    bad_page = true, ks[s] = NAN;
                    continue;
                }
                const size_t row = c.row(page, head, key & (c.page_rows() - 1));
                auto load = [&](int which, uint32_t (&to)[W], float &scale) {
                    const uint8_t *p = c.codes[which] + row * (c.d / 2) + part * (E / 2);
                    if constexpr (W == 4) {
                        const uint4 x = __ldg(reinterpret_cast<const uint4 *>(p));
                        to[0] = x.x, to[1] = x.y, to[2] = x.z, to[3] = x.w;
                    } else {
                        const uint2 x = __ldg(reinterpret_cast<const uint2 *>(p));
                        to[0] = x.x, to[1] = x.y;
                    }
                    scale = mx_scale(__ldg(c.scales[which] + row * (c.d / 32) + part * E / 32));
                };
                load(0, kc[s], ks[s]);
                if constexpr (!SHARED) load(1, vc[s], vs[s]);
            }
        };
        int v0 = k0 + warp * kChunk;
        if (v0 < k1) fetch(v0);
        for (; v0 < k1; v0 += kRowWarps * kChunk) {
            uint32_t kn[kSteps][W], vn[SHARED ? 1 : kSteps][W];
            float kns[kSteps], vns[SHARED ? 1 : kSteps];
#pragma unroll
            for (int s = 0; s < kSteps; ++s) {
                kns[s] = ks[s];
#pragma unroll
                for (int w = 0; w < W; ++w) kn[s][w] = kc[s][w];
                if constexpr (!SHARED) {
                    vns[s] = vs[s];
#pragma unroll
                    for (int w = 0; w < W; ++w) vn[s][w] = vc[s][w];
                }
            }
            if (v0 + kRowWarps * kChunk < k1) fetch(v0 + kRowWarps * kChunk);
#pragma unroll
            for (int s = 0; s < kSteps; ++s) {
                uint64_t val[E / 2];
                auto decode = [&](const uint32_t (&codes)[W]) {
#pragma unroll
                    for (int w = 0; w < W; ++w) {
                        uint32_t h[4];
                        mx_decode8_f16(codes[w], h);
#pragma unroll
                        for (int i = 0; i < 4; ++i) {
                            const float2 f = half2_to_float2(h[i]);
                            val[w * 4 + i] = pack_f32x2(f.x, f.y);
                        }
                    }
                };
                decode(kn[s]);
                const bool there = v0 + s * KS + sub < k1;
                float pr[R];
                bool raise = false;
#pragma unroll
                for (int r = 0; r < R; ++r) {
                    uint64_t acc = 0ull;
#pragma unroll
                    for (int i = 0; i < E / 2; ++i) acc = fma_f32x2(val[i], pack_f32x2(q[r][i].x, q[r][i].y), acc);
                    float x, y;
                    unpack_f32x2(acc, x, y);
                    float sc = (x + y) * kns[s];   // (a block of zero codes behind d: 0 x 0)
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
#pragma unroll
                        for (int i = 0; i < E / 2; ++i) o[r][i].x *= f, o[r][i].y *= f;
                    }
                }
                if constexpr (!SHARED) decode(vn[s]);
                const float scale = SHARED ? kns[s] : vns[SHARED ? 0 : s];
#pragma unroll
                for (int r = 0; r < R; ++r) {
                    const float pe = fast_exp2(pr[r] - m[r]);
                    l[r] += pe;
                    const float pv = there ? pe * scale : 0.f;
                    const uint64_t pp = pack_f32x2(pv, pv);
#pragma unroll
                    for (int i = 0; i < E / 2; ++i) {
                        const uint64_t t = fma_f32x2(val[i], pp, pack_f32x2(o[r][i].x, o[r][i].y));
                        unpack_f32x2(t, o[r][i].x, o[r][i].y);
                    }
                }
            }
        }
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
            float *to = smem + (warp * R + r) * d2;
#pragma unroll
            for (int i = 0; i < E / 2; ++i) {
                float x = o[r][i].x * f, y = o[r][i].y * f;
#pragma unroll
                for (int b = P; b < 32; b <<= 1) x += __shfl_xor_sync(0xffffffffu, x, b), y += __shfl_xor_sync(0xffffffffu, y, b);
                if (sub == 0 && act) to[part * E + 2 * i] = x, to[part * E + 2 * i + 1] = y;
            }
            if (lane == 0) to[c.d] = mt, to[c.d + 1] = lt;
        }
        __syncthreads();
        const bool begins = cur.block == 0, ends = cur.block + take == cur.blocks;
        const int slot = 2 * cta + (begins ? 1 : 0);
        float *rec = a.records + (size_t)slot * R * d2;
        for (int x = tid; x < rows * c.d; x += kRowThreads) {
            const int r = x / c.d, col = x - r * c.d;
            float mt = -FLT_MAX, sum = 0.f, weight = 0.f;
#pragma unroll
            for (int w = 0; w < kRowWarps; ++w) mt = fmaxf(mt, smem[(w * R + r) * d2 + c.d]);
#pragma unroll
            for (int w = 0; w < kRowWarps; ++w) {
                const float *from = smem + (w * R + r) * d2;
                const float f = fast_exp2(from[c.d] - mt);
                sum += from[col] * f, weight += from[c.d + 1] * f;
            }
            if (begins && ends) {
                const int rr = r0 + r, query = rr / a.group;
                T *dst = static_cast<T *>(a.out) + (e.row0 + query) * a.out_stride + (head * a.group + rr - query * a.group) * c.d + col;
                // (no keys: a zero row; a bad sequence: no number)
                *dst = (T)(e.length < 0 ? NAN : keys == 0 ? 0.f : sum / weight);
            } else {
                rec[r * c.d + col] = sum;
                if (col == 0) rec[R * c.d + 2 * r] = mt, rec[R * c.d + 2 * r + 1] = weight;
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

// Tiles that were cut, one per CTA of the attention kernel at most: sums of the pieces, brought to one offset, over their weights.
// The rows of a tile are spread over gridDim.y CTAs.
template <typename T>
__global__ void __launch_bounds__(256) k_att4_join(const AttCall a, int permuted)
{
    grid_dep_wait();
    grid_dep_launch();
    const PieceHeader h = a.headers[blockIdx.x];
    if (h.first_cta < 0) return;
    const int d = a.c.d, last = blockIdx.x;
    const size_t record = (size_t)a.tile_rows * (d + 2);
    for (int x = blockIdx.y * 256 + threadIdx.x; x < h.rows * d; x += gridDim.y * 256) {
        const int r = x / d, col = x - r * d;
        float mt = -FLT_MAX;
        for (int p = h.first_cta; p <= last; ++p) mt = fmaxf(mt, a.records[(2 * p + (p == h.first_cta)) * record + (size_t)a.tile_rows * d + 2 * r]);
        float sum = 0.f, weight = 0.f;
        for (int p = h.first_cta; p <= last; ++p) {
            const float *rec = a.records + (2 * p + (p == h.first_cta)) * record;
            const float f = fast_exp2(rec[(size_t)a.tile_rows * d + 2 * r] - mt);
            // the tensor-core kernel's sums stand in the order of the unpacked codes: 0, 4, 1, 5, 2, 6, 3, 7
            const int at = permuted ? (col & ~7) | ((col & 3) << 1) | ((col >> 2) & 1) : col;
            sum += rec[r * d + at] * f, weight += rec[(size_t)a.tile_rows * d + 2 * r + 1] * f;
        }
        const int rr = h.r0 + r, query = rr / a.group;
        static_cast<T *>(a.out)[(h.row0 + query) * a.out_stride + (h.head * a.group + rr - query * a.group) * d + col] = (T)(sum / weight);
    }
}

bool at16(const void *p) { return (reinterpret_cast<uintptr_t>(p) & 15) == 0; }

template <typename T, int R, bool SHARED>
cudaError_t run_rows(const AttCall &a, int grid, cudaStream_t st)
{
    const size_t smem = (size_t)kRowWarps * R * (a.c.d + 2) * 4;   // 33 KB at most
    const int lanes = (a.c.d + (R == 1 ? 31 : 15)) / (R == 1 ? 32 : 16);
    auto go = [&](auto kernel) { return launch_pdl(kernel, dim3(grid), dim3(kRowThreads), smem, st, a); };
    count_launch();
    constexpr int kF = R == 1 ? 1 : 2;
    if (lanes <= kF) return go(k_att4_rows<T, R, kF, SHARED>);
    if (lanes <= 2 * kF) return go(k_att4_rows<T, R, 2 * kF, SHARED>);
    if (lanes <= 4 * kF) return go(k_att4_rows<T, R, 4 * kF, SHARED>);
    return go(k_att4_rows<T, R, 8 * kF, SHARED>);
}

// How a call is run: which kernel, and how far it may be cut.
struct AttForm {
    bool tensor;      // the tensor-core kernel: tiles of 128 rows
    int tile_rows, block_keys, grid, min_units;
};
AttForm form_of(const aif_cache4 *c, const aif_cache4_query *q)
{
    AttForm f{};
    const int64_t group = q->n_heads / c->heads, per_seq = (q->rows + q->n - 1) / q->n * group;
    f.tensor = q->dtype == AIF_BF16 && att4_tc_block_keys(c->d) > 0 && per_seq > 8;
    if (f.tensor) {
        f.tile_rows = 128, f.block_keys = att4_tc_block_keys(c->d), f.grid = 148, f.min_units = 4;
    } else {
        f.tile_rows = per_seq <= 1 ? 1 : 4, f.block_keys = kRowBlock, f.grid = per_seq <= 1 ? 296 : 148, f.min_units = 1;
    }
    return f;
}
int64_t workspace_of(const AttForm &f, const aif_cache4 *c)
{
    return (int64_t)f.grid * (int64_t)sizeof(PieceHeader) + 2ll * f.grid * f.tile_rows * (c->d + 2) * 4;
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
    if (!(q->scale == q->scale) || q->scale - q->scale != 0.f) return AIF_ERR_ARG;   // NaN, infinite
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
    if (!q->workspace || !at16(q->workspace) || q->workspace_bytes < workspace_of(f, c)) return AIF_ERR_ARG;
    cudaStream_t st = reinterpret_cast<cudaStream_t>(stream);
    AttCall a{};
    a.c = cache4_of(c), a.n = q->n, a.n_heads = q->n_heads, a.group = q->n_heads / c->heads, a.seq_ids = q->seq_ids, a.offsets = q->offsets;
    a.rows = q->rows, a.q = q->q, a.out = q->out, a.q_stride = q->q_stride, a.out_stride = q->out_stride;
    a.scale_log2 = 1.4426950408889634f * (q->scale == 0.f ? 1.0f / sqrtf((float)c->d) : q->scale);
    a.window = q->window, a.sinks = q->sinks, a.tile_rows = f.tile_rows, a.block_keys = f.block_keys, a.min_units = f.min_units;
    a.headers = static_cast<PieceHeader *>(q->workspace);
    a.records = reinterpret_cast<float *>(a.headers + f.grid);
    const bool bf = q->dtype == AIF_BF16, shared = c->shared != 0;
    cudaError_t e;
    if (f.tensor) e = launch_att4_tc(a, f.grid, st);
    else if (f.tile_rows == 1)
        e = bf ? (shared ? run_rows<__nv_bfloat16, 1, true>(a, f.grid, st) : run_rows<__nv_bfloat16, 1, false>(a, f.grid, st))
               : (shared ? run_rows<float, 1, true>(a, f.grid, st) : run_rows<float, 1, false>(a, f.grid, st));
    else
        e = bf ? (shared ? run_rows<__nv_bfloat16, 4, true>(a, f.grid, st) : run_rows<__nv_bfloat16, 4, false>(a, f.grid, st))
               : (shared ? run_rows<float, 4, true>(a, f.grid, st) : run_rows<float, 4, false>(a, f.grid, st));
    if (e == cudaSuccess) {
        const dim3 grid(f.grid, f.tensor ? 16 : 1);
        e = bf ? launch_pdl(k_att4_join<__nv_bfloat16>, grid, dim3(256), 0, st, a, f.tensor ? 1 : 0) : launch_pdl(k_att4_join<float>, grid, dim3(256), 0, st, a, 0);
        count_launch();
    }
    return cache4_failed(e, "aif_cache4_attention");
}

}  // extern "C"
