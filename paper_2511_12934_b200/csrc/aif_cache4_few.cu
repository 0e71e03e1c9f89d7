// Attention of up to eight query rows (queries x heads of a group) of a sequence in the 4-bit cache, bf16, d = 32, 64, 128, 256, where the work is to read
// the cache once: warp-level tensor-core products, fp16 operands, fp32 sums.
//
// A warp takes 16 keys at a time, one group of 16 rows of a page.  Lane (g, t) = (lane / 4, lane % 4) reads a quarter of the rows g and g + 8 and unpacks it to
// fp16 relative to the row's largest scale (exact down to 2^-23 of it).  Those registers are the A operand of scores^T [16 keys x 8 rows] = K Q^T (the
// order of the columns is the lanes' own, the same for keys and queries) and, transposed 8 x 8 by movmatrix, of O^T [d x 8 rows] += V^T P^T, so a row is
// read and unpacked once where values are the keys.  The row's scale 2^E_j goes into its weight: weights are exp2(s_j + E_j - m'), with m' following
// the largest s_j + E_j, beside the softmax's own exp2(s_j - m): fp16 weights lie in (2^-24, 2^15], and what falls below is less than 2^-31 of the largest term.  Queries are
// held in fp16 relative to a power of two per row.  Roundings: weights to fp16 (2^-11), queries' and keys' elements below 2^-14 of their row's largest.
// Bound: HBM, 17/32 byte per element; the products (two of 8 cycles per 256 elements and scheduler) stay below that.  Codes of the next 32 keys of a warp are in flight meanwhile.
#include <cfloat>

#include "aif_cache4_plan.cuh"
#include "aif_tc_ptx.cuh"

namespace aif {
namespace {

constexpr int kFewThreads = 128, kFewWarps = kFewThreads / 32;
constexpr int kFewRows = 8;
constexpr int kFewGroups = 16;    // groups of 16 rows of a unit
constexpr float kWeightBias = 7.f;   // weights are 2^7 at the offset and may grow by 2^8

__device__ __forceinline__ void mma_f16(float (&c)[4], uint32_t a0, uint32_t a1, uint32_t a2, uint32_t a3, uint32_t b0, uint32_t b1)
{
    asm volatile("mma.sync.aligned.m16n8k16.row.col.f32.f16.f16.f32 {%0, %1, %2, %3}, {%4, %5, %6, %7}, {%8, %9}, {%0, %1, %2, %3};"
                 : "+f"(c[0]), "+f"(c[1]), "+f"(c[2]), "+f"(c[3])
                 : "r"(a0), "r"(a1), "r"(a2), "r"(a3), "r"(b0), "r"(b1));
}
__device__ __forceinline__ uint32_t transpose8(uint32_t x)
{
    uint32_t o;
    asm volatile("movmatrix.sync.aligned.m8n8.trans.b16 %0, %1;" : "=r"(o) : "r"(x));
    return o;
}
__device__ __forceinline__ uint32_t mul_f16x2(uint32_t a, uint32_t b)
{
    uint32_t o;
    asm("mul.rn.f16x2 %0, %1, %2;" : "=r"(o) : "r"(a), "r"(b));
    return o;
}
__device__ __forceinline__ uint32_t pack_f16x2(float lo, float hi)
{
    uint32_t o;
    asm("cvt.rn.f16x2.f32 %0, %1, %2;" : "=r"(o) : "f"(hi), "f"(lo));
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
    if constexpr (NB == 1) r.w[0] = __ldg(reinterpret_cast<const uint32_t *>(codes) + t), r.sc[0] = __ldg(scales);
    if constexpr (NB == 2) {
        const uint2 x = __ldg(reinterpret_cast<const uint2 *>(codes) + t);
        r.w[0] = x.x, r.w[1] = x.y, r.sc[0] = __ldg(reinterpret_cast<const uint16_t *>(scales));
    }
    if constexpr (NB >= 4) {
#pragma unroll
        for (int i = 0; i < NB / 4; ++i) {
            const uint4 x = __ldg(reinterpret_cast<const uint4 *>(codes) + t * (NB / 4) + i);
            r.w[4 * i] = x.x, r.w[4 * i + 1] = x.y, r.w[4 * i + 2] = x.z, r.w[4 * i + 3] = x.w;
            r.sc[i] = __ldg(reinterpret_cast<const uint32_t *>(scales) + i);
        }
    }
}
// Largest scale byte of the row.
template <int NB>
__device__ __forceinline__ uint32_t top_scale(const RowCodes<NB> &r)
{
    auto of_word = [](uint32_t x) { return max(max(x & 255u, (x >> 8) & 255u), max((x >> 16) & 255u, x >> 24)); };
    if constexpr (NB == 1) return r.sc[0];
    if constexpr (NB == 2) return max(r.sc[0] & 255u, r.sc[0] >> 8);
    if constexpr (NB == 4) return of_word(r.sc[0]);
    if constexpr (NB == 8) return max(of_word(r.sc[0]), of_word(r.sc[1]));
}
// fp16 pair of 2^(byte - top): 0 below 2^-24, NaN for the byte that says so.
__device__ __forceinline__ uint32_t relative_scale(uint32_t byte, uint32_t top)
{
    const uint32_t down = top - byte;
    uint32_t h = down <= 14u ? (15u - down) << 10 : (1u << 24) >> min(down, 31u);
    h = byte == kMxNan ? 0x7fffu : h;
    return h | (h << 16);
}
// The quarter row's values over 2^(top - 127): words 4 i .. 4 i + 3 of o are the pairs of code word i.  The lane's words t NB .. t NB + NB - 1 of the 4 NB of a row lie in
// one block of four words, or (NB = 8) in two.
template <int NB>
__device__ __forceinline__ void unpack_row(const RowCodes<NB> &r, uint32_t top, int t, uint32_t (&o)[4 * NB])
{
    uint32_t f[NB == 8 ? 2 : 1];
    if constexpr (NB == 8) {
        const uint32_t sc = (t & 2 ? r.sc[1] : r.sc[0]) >> (16 * (t & 1));
        f[0] = relative_scale(sc & 255u, top), f[1] = relative_scale((sc >> 8) & 255u, top);
    } else {
        f[0] = relative_scale((r.sc[0] >> (8 * (t * NB / 4))) & 255u, top);
    }
#pragma unroll
    for (int i = 0; i < NB; ++i) {
        uint32_t h[4];
        mx_decode8_f16(r.w[i], h);
#pragma unroll
        for (int k = 0; k < 4; ++k) o[4 * i + k] = mul_f16x2(h[k], f[NB == 8 ? i / 4 : 0]);
    }
}

template <int NB, bool SHARED>
__global__ void __launch_bounds__(kFewThreads, NB == 8 ? 2 : 3) k_att4_few(const AttCall a)
{
    constexpr int D = 32 * NB, KS = 2 * NB;   // steps of 16 columns
    const Cache4 &c = a.c;
    const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5, g = lane >> 2, t = lane & 3;
    extern __shared__ float smem[];   // [warps][rows][D + 2]
    __shared__ PlanShared<kFewThreads> plan;

    grid_dep_wait();
    grid_dep_launch();
    const int64_t total = plan_total(a, plan);
    const int ctas = (int)min((int64_t)gridDim.x, max((int64_t)1, total / a.min_units));
    const int cta = blockIdx.x;
    if (tid == 0 && a.headers) a.headers[cta].first_cta = -1;
    if (total == 0 || cta >= ctas) return;
    const int64_t u1 = cut(total, ctas, cta + 1);
    int64_t u = cut(total, ctas, cta);
    Cursor cur = plan_find(a, plan, u);
    bool bad_page = false;
    while (u < u1) {
        const Entry &e = cur.e;
        const int row_tiles = cur.tiles / c.heads, head = cur.tile / row_tiles, r0 = (cur.tile - head * row_tiles) * kFewRows, rows = min(kFewRows, e.rows - r0);
        const int64_t tile_u0 = u - cur.block;
        const int take = (int)min(u1 - u, (int64_t)(cur.blocks - cur.block));
        const int groups = e.groups(), g0 = cur.block * kFewGroups, g1 = min(groups, (cur.block + take) * kFewGroups);
        const int sink_groups = e.sink_groups(), rest_group = (e.rest >> 4) - sink_groups;
        const int32_t *table = c.table + (size_t)max(e.seq, 0) * c.max_pages;

        // Queries as B operand: lane (g, t) holds its quarter of the columns of row g.
        uint32_t q[2 * KS];
        float q_scale = 0.f;   // of row g: scale x log2(e) x the power of two that its fp16 values are relative to
        {
            uint32_t raw[2 * KS], top = 0;
            const bool there = g < rows;
            const int rr = r0 + (there ? g : 0), query = rr / a.group;
            const __nv_bfloat16 *src = static_cast<const __nv_bfloat16 *>(a.q) + (e.row0 + query) * a.q_stride + (head * a.group + rr - query * a.group) * D + t * (D / 4);
#pragma unroll
            for (int i = 0; i < NB; ++i) {
                const uint4 x = there ? __ldg(reinterpret_cast<const uint4 *>(src) + i) : make_uint4(0u, 0u, 0u, 0u);
                raw[4 * i] = x.x, raw[4 * i + 1] = x.y, raw[4 * i + 2] = x.z, raw[4 * i + 3] = x.w;
            }
#pragma unroll
            for (int i = 0; i < 2 * KS; ++i) top = max(top, max(raw[i] & 0x7fffu, (raw[i] >> 16) & 0x7fffu));
            top = max(top, __shfl_xor_sync(0xffffffffu, top, 1));
            top = max(top, __shfl_xor_sync(0xffffffffu, top, 2));
            const uint32_t field = min(max(top >> 7, 1u), 253u);            // exponent field of the largest (253: its inverse is still a number)
            const float inv = __uint_as_float((254u - field) << 23);
            q_scale = a.scale_log2 * __uint_as_float(field << 23);
#pragma unroll
            for (int i = 0; i < 2 * KS; ++i) q[i] = pack_f16x2(__uint_as_float(raw[i] << 16) * inv, __uint_as_float(raw[i] & 0xffff0000u) * inv);
        }
        // scores come with the rows 2 t and 2 t + 1 to a lane
        const float k2[2] = {__shfl_sync(0xffffffffu, q_scale, 8 * t), __shfl_sync(0xffffffffu, q_scale, 8 * t + 4)};

        float o[KS][4];
#pragma unroll
        for (int s = 0; s < KS; ++s) o[s][0] = o[s][1] = o[s][2] = o[s][3] = 0.f;
        float m[2] = {-FLT_MAX, -FLT_MAX}, mw[2] = {-FLT_MAX, -FLT_MAX}, l[2] = {0.f, 0.f};   // offsets of the weights' sum and of the values', per row

        RowCodes<NB> kn[2][2], vn[SHARED ? 1 : 2][2];   // [group][key g, key g + 8]
        // a lane's piece of row g of a page's group: from here, page strides and rows further
        const uint32_t page_codes = (uint32_t)(c.heads << c.page_shift) * (D / 2), page_scales = (uint32_t)(c.heads << c.page_shift) * NB;
        const size_t head_row = ((size_t)head << c.page_shift) + g;
        auto fetch = [&](int grp) {   // codes of the groups grp and grp + 1
#pragma unroll
            for (int x = 0; x < 2; ++x) {
                const int gi = min(grp + x, g1 - 1);   // (an odd last one is read twice and used once)
                const int row = (gi < sink_groups ? gi : gi + rest_group) << 4;
                int page = __ldg(table + (row >> c.page_shift));
                const bool ok = c.holds(page);
                bad_page |= !ok;
                page = ok ? page : 0;
                const size_t at = head_row + (row & (c.page_rows() - 1));
                const size_t codes = (size_t)(uint32_t)page * page_codes + at * (D / 2), scales = (size_t)(uint32_t)page * page_scales + at * NB;
#pragma unroll
                for (int h = 0; h < 2; ++h) {
                    load_row<NB>(kn[x][h], c.codes[0] + codes + h * 8 * (D / 2), c.scales[0] + scales + h * 8 * NB, t);
                    if constexpr (!SHARED) load_row<NB>(vn[x][h], c.codes[1] + codes + h * 8 * (D / 2), c.scales[1] + scales + h * 8 * NB, t);
                    if (!ok) {   // no such page: no number
#pragma unroll
                        for (int i = 0; i < (NB + 3) / 4; ++i) kn[x][h].sc[i] = NB == 1 ? 0xffu : NB == 2 ? 0xffffu : 0xffffffffu;
                    }
                }
            }
        };
        int grp = g0 + warp * 2;
        if (grp < g1) fetch(grp);
        for (; grp < g1; grp += kFewWarps * 2) {
            RowCodes<NB> kc[2][2], vc[SHARED ? 1 : 2][2];
#pragma unroll
            for (int x = 0; x < 2; ++x)
#pragma unroll
                for (int h = 0; h < 2; ++h) {
                    kc[x][h] = kn[x][h];
                    if constexpr (!SHARED) vc[x][h] = vn[x][h];
                }
            if (grp + kFewWarps * 2 < g1) fetch(grp + kFewWarps * 2);
#pragma unroll
            for (int x = 0; x < 2; ++x) {
                if (grp + x >= g1) break;
                const int gi = grp + x;
                const bool sink = gi < sink_groups;
                const int row = (sink ? gi : gi + rest_group) << 4;
                const int lo = sink ? 0 : e.rest, hi = sink ? e.first : e.length;   // visible rows of the group: [lo, hi)
                const bool see[2] = {row + g >= lo && row + g < hi, row + g + 8 >= lo && row + g + 8 < hi};
                if (row < lo || row + 16 > hi) {
                    // rows that are not visible have no scale, whatever stands there (codes are finite)
#pragma unroll
                    for (int h = 0; h < 2; ++h)
                        if (!see[h]) {
#pragma unroll
                            for (int i = 0; i < (NB + 3) / 4; ++i) {
                                kc[x][h].sc[i] = 0u;
                                if constexpr (!SHARED) vc[x][h].sc[i] = 0u;
                            }
                        }
                }
                uint32_t top[2] = {top_scale<NB>(kc[x][0]), top_scale<NB>(kc[x][1])};
                uint32_t ka[4 * NB], kb[4 * NB];
                unpack_row<NB>(kc[x][0], top[0], t, ka);
                unpack_row<NB>(kc[x][1], top[1], t, kb);
                float s[4] = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
                for (int i = 0; i < KS; ++i) mma_f16(s, ka[2 * i], kb[2 * i], ka[2 * i + 1], kb[2 * i + 1], q[2 * i], q[2 * i + 1]);
                // s[0], s[1]: key g, rows 2 t, 2 t + 1; s[2], s[3]: key g + 8
                const float scale[2] = {mx_scale(top[0]), mx_scale(top[1])};
                uint32_t vtop[2] = {top[0], top[1]};
                if constexpr (!SHARED) vtop[0] = top_scale<NB>(vc[x][0]), vtop[1] = top_scale<NB>(vc[x][1]);
                float w[4];
                bool raise = false;
#pragma unroll
                for (int i = 0; i < 4; ++i) {
                    s[i] = see[i >> 1] ? s[i] * (k2[i & 1] * scale[i >> 1]) : -INFINITY;
                    w[i] = s[i] + (float)((int)vtop[i >> 1] - 127);
                    raise |= s[i] > m[i & 1] + 8.f || w[i] > mw[i & 1] + 8.f;
                }
                // the offsets follow the maxima only when those have grown by a factor of 2^8
                if (__any_sync(0xffffffffu, raise)) {
#pragma unroll
                    for (int r = 0; r < 2; ++r) {
                        float ms = fmaxf(s[r], s[r + 2]), mv = fmaxf(w[r], w[r + 2]);
#pragma unroll
                        for (int b = 4; b < 32; b <<= 1) ms = fmaxf(ms, __shfl_xor_sync(0xffffffffu, ms, b)), mv = fmaxf(mv, __shfl_xor_sync(0xffffffffu, mv, b));
                        ms = ms > m[r] + 8.f ? ms : m[r], mv = mv > mw[r] + 8.f ? mv : mw[r];
                        const float f = fast_exp2(mw[r] - mv);
                        l[r] *= fast_exp2(m[r] - ms);
                        m[r] = ms, mw[r] = mv;
#pragma unroll
                        for (int i = 0; i < KS; ++i) o[i][r] *= f, o[i][r + 2] *= f;
                    }
                }
#pragma unroll
                for (int i = 0; i < 4; ++i) {
                    l[i & 1] += fast_exp2(s[i] - m[i & 1]);
                    w[i] = fast_exp2(w[i] - mw[i & 1] + kWeightBias);
                }
                const uint32_t p0 = transpose8(pack_f16x2(w[0], w[1])), p1 = transpose8(pack_f16x2(w[2], w[3]));
                if constexpr (!SHARED) {
                    unpack_row<NB>(vc[x][0], vtop[0], t, ka);
                    unpack_row<NB>(vc[x][1], vtop[1], t, kb);
                }
#pragma unroll
                for (int i = 0; i < KS; ++i)
                    mma_f16(o[i], transpose8(ka[2 * i]), transpose8(ka[2 * i + 1]), transpose8(kb[2 * i]), transpose8(kb[2 * i + 1]), p0, p1);
            }
        }
        // O^T: o[i][0], [1]: rows 2 t, 2 t + 1 of the column that lane quarter g / 2 has as element g % 2 of its pair 2 i; o[i][2], [3]: of its pair 2 i + 1
#pragma unroll
        for (int r = 0; r < 2; ++r) {
            float lt = l[r];
#pragma unroll
            for (int b = 4; b < 32; b <<= 1) lt += __shfl_xor_sync(0xffffffffu, lt, b);
            float *to = smem + (warp * kFewRows + 2 * t + r) * (D + 2);
            const float f = fast_exp2(mw[r] - kWeightBias - m[r]);   // sums relative to the offset of the weights' sum
#pragma unroll
            for (int i = 0; i < KS; ++i) {
                const int col = (g >> 1) * (D / 4) + (g & 1) + 4 * i;
                to[col] = o[i][r] * f, to[col + 2] = o[i][r + 2] * f;
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
                if (g0 + w * 2 < g1) {   // (a warp without keys has nothing to say)
                    const float f = fast_exp2(from[D] - mt);
                    sum += from[col] * f, weight += from[D + 1] * f;
                }
            }
            if (begins && ends) {
                const int rr = r0 + r, query = rr / a.group;
                __nv_bfloat16 *dst = static_cast<__nv_bfloat16 *>(a.out) + (e.row0 + query) * a.out_stride + (head * a.group + rr - query * a.group) * D + col;
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
    const size_t smem = (size_t)kFewWarps * kFewRows * (32 * NB + 2) * 4;   // up to 65 KB
    if (smem > 48 * 1024) {
        const cudaError_t e = allow_smem<k_att4_few<NB, SHARED>>(smem);
        if (e != cudaSuccess) return e;
    }
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
