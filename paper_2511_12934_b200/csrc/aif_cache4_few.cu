// Attention of up to eight query rows (queries x heads of a group) of a sequence in the 4-bit cache, bf16, d = 32, 64, 128, 256, where the work is to read
// the cache once: warp-level tensor-core products, bf16 operands, fp32 sums.
//
// A warp takes 16 keys at a time, one group of 16 rows of a page.  Lane (g, t) = (lane / 4, lane % 4) reads a quarter of the rows g and g + 8 and unpacks it to
// bf16, which holds every 4-bit value exactly.  Those registers are the A operand of scores^T [16 keys x 8 rows] = K Q^T (the order of the columns is the lanes' own, the same
// for keys and queries) and, transposed 8 x 8 by movmatrix, of O^T [d x 8 rows] += V^T P^T, so a row is read and unpacked once where values are the keys.
// Roundings: scores and sums are fp32 sums of exact products; a weight goes in as two bf16 numbers, together within 2^-16 of it.  (fp16 operands relative to a row's largest scale, that scale in the
// row's weight, need fewer instructions: 256 x 10^4 keys 87 us against 99 at d = 128, 140 against 177 at d = 256, 119 against 157 with values of their own; but fp16 then spans all columns
// of a row and all rows of a sequence at once, and columns or rows 2^24 below the largest were lost.)
// Bound: the instructions that unpack (at d = 128 issue slots 59 %, ALU 47 %), not HBM (22 %) and not the products (31 %).  256 sequences of 10^4 rows, one query row each: d = 32 64 us, d = 64 65 us, d = 128
// 99 us, d = 256 177 us; values of their own d = 64 91 us, d = 128 157 us; one sequence of 200 rows 5.9 us.  A warp has a ring of stages in shared memory, filled by
// asynchronous copies of whole groups.
#include <cfloat>

#include "aif_cache4_plan.cuh"
#include "aif_tc_ptx.cuh"

namespace aif {
namespace {

constexpr int kFewThreads = 128, kFewWarps = kFewThreads / 32;
constexpr int kFewRows = 8;
constexpr int kFewGroups = 16;    // groups of 16 rows of a unit

__device__ __forceinline__ uint32_t transpose8(uint32_t x)
{
    uint32_t o;
    asm volatile("movmatrix.sync.aligned.m8n8.trans.b16 %0, %1;" : "=r"(o) : "r"(x));
    return o;
}
__device__ __forceinline__ uint32_t pack_bf16x2(float lo, float hi)
{
    uint32_t o;
    asm("cvt.rn.bf16x2.f32 %0, %1, %2;" : "=r"(o) : "f"(hi), "f"(lo));
    return o;
}

// Codes of a lane's quarter of a row, and the scale bytes of the whole row.
template <int NB>
struct RowCodes {
    uint32_t w[NB];
    uint32_t sc[(NB + 3) / 4];
};

template <int NB>
__device__ __forceinline__ void load_row(RowCodes<NB> &r, const uint8_t *codes, const uint8_t *scales, int t)
{
    if constexpr (NB == 1) r.w[0] = reinterpret_cast<const uint32_t *>(codes)[t], r.sc[0] = *scales;
    if constexpr (NB == 2) {
        const uint2 x = reinterpret_cast<const uint2 *>(codes)[t];
        r.w[0] = x.x, r.w[1] = x.y, r.sc[0] = *reinterpret_cast<const uint16_t *>(scales);
    }
    if constexpr (NB >= 4) {
#pragma unroll
        for (int i = 0; i < NB / 4; ++i) {
            const uint4 x = reinterpret_cast<const uint4 *>(codes)[t * (NB / 4) + i];
            r.w[4 * i] = x.x, r.w[4 * i + 1] = x.y, r.w[4 * i + 2] = x.z, r.w[4 * i + 3] = x.w;
            r.sc[i] = reinterpret_cast<const uint32_t *>(scales)[i];
        }
    }
}
// The values of two quarter rows: words 4 i .. 4 i + 3 of a row's o are the pairs (0,4) (1,5) (2,6) (3,7) of code word i.  The lane's words t NB .. t NB + NB - 1 of the 4 NB of a row lie
// in one block of four words, or (NB = 8) in two.  Large scales have a second factor (see UnpackScale): a branch of the whole warp.
template <int NB>
__device__ __forceinline__ void unpack_rows(const RowCodes<NB> *r, int t, uint32_t (*o)[4 * NB])
{
    constexpr int kScales = NB == 8 ? 2 : 1;
    uint32_t byte[2][kScales];
    bool two = false;
#pragma unroll
    for (int x = 0; x < 2; ++x) {
        if constexpr (NB == 8) {
            const uint32_t sc = (t & 2 ? r[x].sc[1] : r[x].sc[0]) >> (16 * (t & 1));
            byte[x][0] = sc & 255u, byte[x][1] = (sc >> 8) & 255u;
        } else {
            byte[x][0] = (r[x].sc[0] >> (8 * (t * NB / 4))) & 255u;
        }
#pragma unroll
        for (int i = 0; i < kScales; ++i) {
            const UnpackScale s(byte[x][i]);
            two |= s.two;
#pragma unroll
            for (int w = i * NB / kScales; w < (i + 1) * NB / kScales; ++w) {
                const uint4 v = unpack8_first(r[x].w[w], s.first);
                o[x][4 * w] = v.x, o[x][4 * w + 1] = v.y, o[x][4 * w + 2] = v.z, o[x][4 * w + 3] = v.w;
            }
        }
    }
    if (__any_sync(0xffffffffu, two)) {
#pragma unroll
        for (int x = 0; x < 2; ++x)
#pragma unroll
            for (int i = 0; i < kScales; ++i) {
                const UnpackScale s(byte[x][i]);
                const uint32_t factor = s.two ? s.second : 0x3f803f80u;
#pragma unroll
                for (int w = 4 * i * NB / kScales; w < 4 * (i + 1) * NB / kScales; ++w) o[x][w] = mul_bf16x2(o[x][w], factor);
            }
    }
}

template <int NB, bool SHARED>
struct FewCfg {
    static constexpr int kGroups = NB == 8 ? 1 : 2;   // groups of 16 rows at a time: their products and exponentials overlap (one at d = 256, for want of registers)
    static constexpr int kKinds = SHARED ? 1 : 2;
    static constexpr int kRing = SHARED ? 6 : 4;      // stages of a warp's ring
    static constexpr int kCodes = 16 * 16 * NB, kScales = 16 * NB;   // bytes of a group
    static constexpr int kStage = kKinds * kGroups * (kCodes + kScales);
    static constexpr int kBlocks = NB == 8 ? 2 : 3;   // blocks of a multiprocessor
    static constexpr size_t kSmem = (size_t)kFewWarps * (kRing * kStage + kFewRows * (32 * NB + 2) * 4);
};

template <int NB, bool SHARED>
__global__ void __launch_bounds__(kFewThreads, (FewCfg<NB, SHARED>::kBlocks)) k_att4_few(const AttCall a)
{
    constexpr int D = 32 * NB, KS = 2 * NB;   // steps of 16 columns
    const Cache4 &c = a.c;
    const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5, g = lane >> 2, t = lane & 3;
    using F = FewCfg<NB, SHARED>;
    extern __shared__ __align__(16) unsigned char smem_dyn[];   // rings [warps][kRing][kinds][groups]: codes, then scales; sums [warps][rows][D + 2]
    unsigned char *ring = smem_dyn + warp * F::kRing * F::kStage;
    float *smem = reinterpret_cast<float *>(smem_dyn + kFewWarps * F::kRing * F::kStage);
    __shared__ PlanShared<kFewThreads> plan;

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
    bool bad_page = false;
    while (u < u1) {
        const Entry &e = cur.e;
        const int head = cur.head, r0 = cur.row_tile * kFewRows, rows = min(kFewRows, e.rows - r0);
        const int64_t tile_u0 = u - cur.block;
        const int take = (int)min(u1 - u, (int64_t)(cur.blocks - cur.block));
        const int groups = e.groups(), g0 = cur.block * kFewGroups, g1 = min(groups, (cur.block + take) * kFewGroups);
        const int sink_groups = e.sink_groups(), rest_group = (e.rest >> 4) - sink_groups;
        const int32_t *table = c.table + (size_t)max(e.seq, 0) * c.max_pages;

        // Queries as B operand: lane (g, t) holds its quarter of the columns of row g, in the order of the unpacked codes.
        uint32_t q[2 * KS];
        {
            const bool there = g < rows;
            const __nv_bfloat16 *src = static_cast<const __nv_bfloat16 *>(a.q) + row_at(a, e.row0, head, r0 + (there ? g : 0), a.q_stride, D) + t * (D / 4);
#pragma unroll
            for (int i = 0; i < NB; ++i) {
                const uint4 x = there ? __ldg(reinterpret_cast<const uint4 *>(src) + i) : make_uint4(0u, 0u, 0u, 0u);
                q[4 * i] = __byte_perm(x.x, x.z, 0x5410), q[4 * i + 1] = __byte_perm(x.x, x.z, 0x7632);
                q[4 * i + 2] = __byte_perm(x.y, x.w, 0x5410), q[4 * i + 3] = __byte_perm(x.y, x.w, 0x7632);
            }
        }
        // Stage n of this warp: groups first + n kStride and, if two, the one behind.  Where they lie and what of them is visible is worked out for 32 groups at a time, one to
        // a lane, a batch ahead; codes and scales come kRing - 1 stages ahead, by asynchronous copies: a group is one piece of each.
        constexpr int G = F::kGroups, kStride = kFewWarps * G;
        const int first = g0 + warp * G, stages = first < g1 ? (g1 - first + kStride - 1) / kStride : 0;
        struct Batch {
            int32_t page;            // of this lane's group
            uint32_t in_pages, span; // groups before it in a page (all heads), its visible rows: [span & 255, span >> 8)
        };
        auto load_batch = [&](int n) {
            const int gi = min(first + (n + lane / G) * kStride + lane % G, g1 - 1);   // (behind the last group: that one again, of which nothing is visible)
            const bool sink = gi < sink_groups, there = gi == first + (n + lane / G) * kStride + lane % G;
            const int row = (sink ? gi : gi + rest_group) << 4;
            const int lo = sink ? 0 : max(e.rest - row, 0), hi = there ? min(16, (sink ? e.first : e.length) - row) : 0;
            return Batch{__ldg(table + (row >> c.page_shift)), (uint32_t)((head << c.page_shift) + (row & (c.page_rows() - 1))) >> 4, (uint32_t)lo | (uint32_t)hi << 8};
        };
        const uint32_t page_groups = (uint32_t)(c.heads << c.page_shift) >> 4;
        // the groups' places in the pool, in groups; those of pages that do not exist are marked in the span and read page 0
        uint32_t place = 0, span = 0;
        Batch ahead{};
        auto settle = [&](const Batch &b) {
            const bool ok = c.holds(b.page);
            bad_page |= !ok;
            place = (ok ? (uint32_t)b.page : 0u) * page_groups + b.in_pages, span = b.span | (ok ? 0u : 1u << 16);
        };
        if (stages > 0) settle(load_batch(0));
        if (stages > 32 / G) ahead = load_batch(32 / G);
        const uint32_t ring_at = smem_u32(ring) + lane * 16;
        const uint8_t *codes_at[F::kKinds], *scales_at[F::kKinds];
#pragma unroll
        for (int k = 0; k < F::kKinds; ++k) codes_at[k] = c.codes[k] + lane * 16, scales_at[k] = c.scales[k] + lane * 16;
        int slot_in = 0;
        uint32_t span_now = span, span_next = 0;   // spans of the batch that is at work (copies may be in the next one already)
        auto bring = [&](int n) {
            if (n < stages) {
                if (n > 0 && n % (32 / G) == 0) {
                    settle(ahead);
                    span_next = span;
                    if (n + 32 / G < stages) ahead = load_batch(n + 32 / G);
                }
                const uint32_t to0 = ring_at + (uint32_t)(slot_in * F::kStage);
#pragma unroll
                for (int x = 0; x < G; ++x) {
                    const uint32_t at = __shfl_sync(0xffffffffu, place, (n * G + x) & 31);
#pragma unroll
                    for (int k = 0; k < F::kKinds; ++k) {
                        const uint32_t to = to0 + (uint32_t)((k * G + x) * (F::kCodes + F::kScales));
                        const uint8_t *codes = codes_at[k] + (size_t)at * F::kCodes;
#pragma unroll
                        for (int y = 0; y < (NB + 1) / 2; ++y)
                            if (NB > 1 || lane < 16) cp_async16(to + y * 512, codes + y * 512, 16u);
                        if (lane < NB) cp_async16(to + F::kCodes, scales_at[k] + (size_t)at * F::kScales, 16u);
                    }
                }
                slot_in = slot_in + 1 == F::kRing ? 0 : slot_in + 1;
            }
            cp_async_commit();
        };
#pragma unroll 1
        for (int n = 0; n < F::kRing - 1; ++n) bring(n);
        float o[KS][4];
#pragma unroll
        for (int s = 0; s < KS; ++s) o[s][0] = o[s][1] = o[s][2] = o[s][3] = 0.f;
        float m[2] = {-FLT_MAX, -FLT_MAX}, l[2] = {0.f, 0.f};   // of the rows 2 t and 2 t + 1, as the scores come to a lane

        int slot = 0;
        for (int n = 0; n < stages; ++n) {
            if (n > 0 && n % (32 / G) == 0) span_now = span_next;
            bring(n + F::kRing - 1);   // (into the slot that was read a stage ago)
            cp_async_wait<F::kRing - 1>();
            __syncwarp();
            const unsigned char *stage = ring + slot * F::kStage + g * (D / 2), *stage_sc = ring + slot * F::kStage + F::kCodes + g * NB;
            slot = slot + 1 == F::kRing ? 0 : slot + 1;
            uint32_t kf[2 * G][4 * NB];                      // keys (then values) as bf16 pairs: rows g and g + 8 of each group
            RowCodes<NB> kr[2 * G], vc[SHARED ? 1 : 2 * G];
            float s[G][4];
            bool see[G][2];
#pragma unroll
            for (int x = 0; x < G; ++x) {
                const uint32_t sp = __shfl_sync(0xffffffffu, span_now, (n * G + x) & 31), lo = sp & 255u, hi = (sp >> 8) & 255u;
#pragma unroll
                for (int h = 0; h < 2; ++h) {
                    load_row<NB>(kr[2 * x + h], stage + x * (F::kCodes + F::kScales) + 8 * h * (D / 2), stage_sc + x * (F::kCodes + F::kScales) + 8 * h * NB, t);
                    if constexpr (!SHARED)
                        load_row<NB>(vc[2 * x + h], stage + (G + x) * (F::kCodes + F::kScales) + 8 * h * (D / 2), stage_sc + (G + x) * (F::kCodes + F::kScales) + 8 * h * NB, t);
                    see[x][h] = g + 8 * h >= lo && g + 8 * h < hi;
                }
                if (sp != 16u << 8) {
                    // rows that are not visible have no scale, whatever stands there (codes are finite); those of a page that does not exist are no numbers
#pragma unroll
                    for (int h = 0; h < 2; ++h)
#pragma unroll
                        for (int i = 0; i < (NB + 3) / 4; ++i) {
                            const uint32_t bad = NB == 1 ? 0xffu : NB == 2 ? 0xffffu : 0xffffffffu;
                            kr[2 * x + h].sc[i] = !see[x][h] ? 0u : sp >> 16 ? bad : kr[2 * x + h].sc[i];
                            if constexpr (!SHARED) vc[2 * x + h].sc[i] = !see[x][h] ? 0u : vc[2 * x + h].sc[i];
                        }
                }
            }
#pragma unroll
            for (int x = 0; x < G; ++x) unpack_rows<NB>(kr + 2 * x, t, kf + 2 * x);
            bool raise = false;
#pragma unroll
            for (int x = 0; x < G; ++x) {
                float s2[2][4] = {};   // two chains of products
#pragma unroll
                for (int i = 0; i < KS; ++i) mma_bf16(s2[i & 1], kf[2 * x][2 * i], kf[2 * x + 1][2 * i], kf[2 * x][2 * i + 1], kf[2 * x + 1][2 * i + 1], q[2 * i], q[2 * i + 1]);
                // s[0], s[1]: key g, rows 2 t, 2 t + 1; s[2], s[3]: key g + 8
#pragma unroll
                for (int i = 0; i < 4; ++i) {
                    s[x][i] = see[x][i >> 1] ? (s2[0][i] + s2[1][i]) * a.scale_log2 : -INFINITY;
                    raise |= s[x][i] > m[i & 1] + 8.f;
                }
            }
            // the offset follows the maximum only when that has grown by a factor of 2^8
            if (__any_sync(0xffffffffu, raise)) {
#pragma unroll
                for (int r = 0; r < 2; ++r) {
                    float ms = -FLT_MAX;
#pragma unroll
                    for (int x = 0; x < G; ++x) ms = fmaxf(ms, fmaxf(s[x][r], s[x][r + 2]));
#pragma unroll
                    for (int b = 4; b < 32; b <<= 1) ms = fmaxf(ms, __shfl_xor_sync(0xffffffffu, ms, b));
                    ms = ms > m[r] + 8.f ? ms : m[r];
                    const float f = fast_exp2(m[r] - ms);
                    l[r] *= f, m[r] = ms;
#pragma unroll
                    for (int i = 0; i < KS; ++i) o[i][r] *= f, o[i][r + 2] *= f;
                }
            }
#pragma unroll
            for (int x = 0; x < G; ++x) {
                uint32_t p[2][2];   // [upper, lower half of the weights][keys g, keys g + 8], as B operand
#pragma unroll
                for (int h = 0; h < 2; ++h) {
                    const float w0 = fast_exp2(s[x][2 * h] - m[0]), w1 = fast_exp2(s[x][2 * h + 1] - m[1]);
                    l[0] += w0, l[1] += w1;
                    const uint32_t hi = pack_bf16x2(w0, w1);
                    p[0][h] = transpose8(hi), p[1][h] = transpose8(pack_bf16x2(w0 - __uint_as_float(hi << 16), w1 - __uint_as_float(hi & 0xffff0000u)));
                }
                if constexpr (!SHARED) unpack_rows<NB>(vc + 2 * x, t, kf + 2 * x);
#pragma unroll
                for (int i = 0; i < KS; ++i) {
                    const uint32_t v0 = transpose8(kf[2 * x][2 * i]), v1 = transpose8(kf[2 * x][2 * i + 1]), v2 = transpose8(kf[2 * x + 1][2 * i]), v3 = transpose8(kf[2 * x + 1][2 * i + 1]);
                    mma_bf16(o[i], v0, v1, v2, v3, p[0][0], p[0][1]);
                    mma_bf16(o[i], v0, v1, v2, v3, p[1][0], p[1][1]);
                }
            }
        }
        cp_async_wait_all();
        // O^T: o[i][0], [1]: rows 2 t, 2 t + 1 of the column that lane quarter g / 2 has as element g % 2 of its pair 2 i (columns c and c + 4 of a code word's eight);
        // o[i][2], [3]: of its pair 2 i + 1
#pragma unroll
        for (int r = 0; r < 2; ++r) {
            float lt = l[r];
#pragma unroll
            for (int b = 4; b < 32; b <<= 1) lt += __shfl_xor_sync(0xffffffffu, lt, b);
            float *to = smem + (warp * kFewRows + 2 * t + r) * (D + 2);
#pragma unroll
            for (int i = 0; i < KS; ++i) {
                const int col = (g >> 1) * (D / 4) + (i >> 1) * 8 + (i & 1) * 2 + (g & 1) * 4;
                to[col] = o[i][r], to[col + 1] = o[i][r + 2];
            }
            if (g == 0) to[D] = m[r], to[D + 1] = lt;
        }
        __syncthreads();
        const bool begins = cur.block == 0, ends = cur.block + take == cur.blocks;
        float *rec = a.records + (size_t)(2 * cta + (begins ? 1 : 0)) * kFewRows * (D + 2);
        for (int x = tid; x < rows * D; x += kFewThreads) {
            const int r = x / D, col = x - r * D;
            float mt = -FLT_MAX, sum = 0.f, weight = 0.f;
#pragma unroll
            for (int w = 0; w < kFewWarps; ++w) mt = fmaxf(mt, smem[(w * kFewRows + r) * (D + 2) + D]);
#pragma unroll
            for (int w = 0; w < kFewWarps; ++w) {
                const float *from = smem + (w * kFewRows + r) * (D + 2);
                if (g0 + w * G < g1) {   // (a warp without keys has nothing to say)
                    const float f = fast_exp2(from[D] - mt);
                    sum += from[col] * f, weight += from[D + 1] * f;
                }
            }
            if (begins && ends) {
                __nv_bfloat16 *dst = static_cast<__nv_bfloat16 *>(a.out) + row_at(a, e.row0, head, r0 + r, a.out_stride, D) + col;
                // (no keys: a zero row; a bad sequence: no number)
                *dst = (__nv_bfloat16)(e.length < 0 ? NAN : groups == 0 ? 0.f : sum / weight);
            } else {
                rec[r * D + col] = sum;
                if (col == 0) rec[kFewRows * D + 2 * r] = mt, rec[kFewRows * D + 2 * r + 1] = weight;
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

template <int NB, bool SHARED>
cudaError_t run_few(const AttCall &a, int grid, cudaStream_t st)
{
    const size_t smem = FewCfg<NB, SHARED>::kSmem;
    const cudaError_t e = allow_smem<k_att4_few<NB, SHARED>>(smem);
    if (e != cudaSuccess) return e;
    count_launch();
    return launch_pdl(k_att4_few<NB, SHARED>, dim3(grid), dim3(kFewThreads), smem, st, a);
}

}  // namespace

cudaError_t launch_att4_few(const AttCall &a, int grid, cudaStream_t st)
{
    const bool shared = a.c.codes[0] == a.c.codes[1];
    switch (a.c.d) {
        case 32: return shared ? run_few<1, true>(a, grid, st) : run_few<1, false>(a, grid, st);
        case 64: return shared ? run_few<2, true>(a, grid, st) : run_few<2, false>(a, grid, st);
        case 128: return shared ? run_few<4, true>(a, grid, st) : run_few<4, false>(a, grid, st);
        default: return shared ? run_few<8, true>(a, grid, st) : run_few<8, false>(a, grid, st);
    }
}

}  // namespace aif
