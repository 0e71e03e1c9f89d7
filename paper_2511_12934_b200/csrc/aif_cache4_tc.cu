// Attention of many query rows over sequences in the 4-bit cache on the tensor cores (sm_100a), bf16, d = 256:
//   out_i = softmax_j(scale q_i k_j) v   for tiles of 128 query rows (queries x heads of a group) of one sequence.
//
// The 4-bit codes are unpacked to bf16 on their way into shared memory (exact: two significant bits and a power of two), once per tile and
// block of keys, and both products run as bf16 tcgen05 products with fp32 accumulators in tensor memory.  One CTA per SM takes
// an even share of the launch's units (aif_cache4_plan.cuh).  Warps:
//   0-7    softmax: a thread owns a query row, two warps share a quarter of the rows, each with half of a block's keys; scores from tensor memory,
//          exponentials in fp32, probabilities back to tensor memory as bf16 pairs; at the end of a tile they normalise and store its rows
//   8, 9   one lane issues scores = Q K^T up to two blocks ahead, one lane O += P V with V read MN-major from the tile K was read from
//   10, 11 bring the query rows of the next tile
//   12-15  unpack keys and values: a thread takes half of a key row; its codes for the next block are in flight in registers
//          meanwhile, and the page numbers for the one after that
// Eight codes of a word come apart as the pairs (0,4) (1,5) (2,6) (3,7) with two shifts, two masks and a multiplication each; queries are put
// into the same order as they are brought, and sums are taken out of it as they are stored.
// Bound: no unit by itself (issue slots 55 %, ALU 43 %, products 41 % of the cycles, exponentials 21 %): one tile of 128 rows is at work, and its softmax, its products and the
// unpacking of 64 keys x 256 wait for one another.  148 tiles x 8192 keys 180 us (880 TFLOP/s; values of their own 326 us), 16 x 10^4 rows x 10^4 keys 1.96 ms (832 TFLOP/s), one
// tile of two blocks 16 us.
// Rounding: probabilities are rounded to bf16 for the product (relative 2^-8 each), and their sum is of the rounded ones, everything else is fp32.
#include <cfloat>

#include "aif_cache4_plan.cuh"
#include "aif_tc_ptx.cuh"

namespace aif {
namespace {

constexpr int D = 256;   // (sums of two halves of 256 rows, as for smaller d, would fill all of tensor memory)

template <bool SHARED>
struct Att4Cfg {
    static constexpr int kBN = 64;                        // keys of a block: two score buffers, two of probabilities and O fill 512 columns
    static constexpr int kChunks = D / 64;                // 64-column (128-byte) chunks of a row
    static constexpr int kQBytes = kChunks * 128 * 128;
    static constexpr int kQBufs = 1;
    static constexpr int kChunkBytes = kBN * 128;
    static constexpr int kTileBytes = kChunks * kChunkBytes;
    static constexpr int kKinds = SHARED ? 1 : 2;
    static constexpr int kStages = SHARED ? 3 : 2;
    static constexpr int kStageBytes = kKinds * kTileBytes;
    static constexpr int kSoftWarps = 8, kQkWarp = 8, kPvWarp = 9, kQWarp = 10, kUnpackWarp = 12;
    static constexpr int kThreads = 512;
    static constexpr int kTmemP = 2 * kBN, kTmemO = 3 * kBN;
    static constexpr int kOutBytes = 8 * 2048;            // 32 rows x 64 bytes for each softmax warp
    static constexpr int kMisc = 512 + 2 * 2 * 128 * 4 + 2 * 128 * 4;   // barriers; block maxima [2][2][128]; weights [2][128]
    static constexpr size_t kSmem = 1024 + kQBufs * kQBytes + kStages * kStageBytes + kOutBytes + kMisc;
};

template <bool SHARED>
__global__ void __launch_bounds__(512, 1) k_att4_tc(const AttCall a)
{
    using C = Att4Cfg<SHARED>;
    constexpr int BN = C::kBN, kS = C::kStages, kQB = C::kQBufs;
    extern __shared__ unsigned char smem_dyn[];
    unsigned char *base = reinterpret_cast<unsigned char *>(((uintptr_t)smem_dyn + 1023) & ~(uintptr_t)1023);
    unsigned char *smQ = base, *smKV = smQ + kQB * C::kQBytes, *smOut = smKV + kS * C::kStageBytes;
    uint64_t *bars = reinterpret_cast<uint64_t *>(smOut + C::kOutBytes);
    uint64_t *k_full = bars, *v_full = bars + kS, *kv_empty = bars + 2 * kS, *s_full = bars + 3 * kS, *s_free = s_full + 2, *p_full = s_free + 2;
    uint64_t *pv_done = p_full + 2, *q_full = pv_done + 2, *q_empty = q_full + 2, *q_first = q_empty + 2, *o_final = q_first + 1, *o_free = o_final + 1;
    uint32_t *tmem_slot = reinterpret_cast<uint32_t *>(o_free + 1);
    volatile uint32_t *abort_flag = tmem_slot + 1;
    float *mx_s = reinterpret_cast<float *>(smOut + C::kOutBytes + 512);   // [2 blocks][2 halves][128]
    float *l_s = mx_s + 512;                                               // [2 halves][128]
    __shared__ PlanShared<C::kThreads> plan;

    const Cache4 &c = a.c;
    const int tid = threadIdx.x, warp = tid >> 5, lane = tid & 31;
    if (tid == 0) {
        for (int s = 0; s < kS; ++s) mbar_init(smem_u32(k_full + s), 128), mbar_init(smem_u32(v_full + s), 128), mbar_init(smem_u32(kv_empty + s), 1);
        for (int b = 0; b < 2; ++b) {
            mbar_init(smem_u32(s_full + b), 1), mbar_init(smem_u32(s_free + b), C::kSoftWarps), mbar_init(smem_u32(p_full + b), C::kSoftWarps * 32);
            mbar_init(smem_u32(pv_done + b), 1), mbar_init(smem_u32(q_full + b), 64), mbar_init(smem_u32(q_empty + b), 1);
        }
        mbar_init(smem_u32(q_first), C::kSoftWarps * 32), mbar_init(smem_u32(o_final), 1), mbar_init(smem_u32(o_free), C::kSoftWarps);
        *abort_flag = 0u;
        asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
    }
    if (warp == C::kQkWarp) tmem_alloc(smem_u32(tmem_slot), 512);
    tc_fence_before();
    __syncthreads();
    tc_fence_after();
    const uint32_t tmem = *tmem_slot;
    grid_dep_wait();
    grid_dep_launch();

    const int cta = blockIdx.x;
    if (tid == 0 && a.headers) a.headers[cta].first_cta = -1;
    const Share share = plan_share(a, plan);
    const int64_t total = share.total, u0 = share.u0, u1 = share.u1;
    const int ctas = share.ctas;
    const bool work = u0 < u1;
    Cursor cur = share.cur;
    int64_t u = u0;

    // One query row of the tile that `at` stands on, 16 bytes (piece p of D / 8) into a query buffer, in the order of the unpacked codes.
    auto query_piece = [&](const Cursor &at, int r, int p) -> uint4 {
        const int rr = at.row_tile * 128 + r;
        if (rr >= at.e.rows) return make_uint4(0u, 0u, 0u, 0u);
        return __ldg(reinterpret_cast<const uint4 *>(static_cast<const __nv_bfloat16 *>(a.q) + row_at(a, at.e.row0, at.head, rr, a.q_stride, D) + p * 8));
    };
    auto put_query = [&](unsigned char *q, int r, int p, uint4 w) {
        const uint4 o = make_uint4(__byte_perm(w.x, w.z, 0x5410), __byte_perm(w.x, w.z, 0x7632), __byte_perm(w.y, w.w, 0x5410), __byte_perm(w.y, w.w, 0x7632));
        *reinterpret_cast<uint4 *>(q + (p >> 3) * 16384 + r * 128 + (((p & 7) ^ (r & 7)) << 4)) = o;
    };

    if (warp < C::kSoftWarps) {
        // ===================== softmax, output =====================
        constexpr int CW = BN / 2;
        const int wq = warp & 3, half = warp >> 2, row = wq * 32 + lane;
        const uint32_t lane_base = tmem + ((uint32_t)(wq * 32) << 16);
        const float k2 = a.scale_log2;
        if (work) {
            constexpr int kPer = D / 8;   // pieces of a row
#pragma unroll 8
            for (int x = tid; x < 128 * kPer; x += 256) put_query(smQ, x / kPer, x % kPer, query_piece(cur, x / kPer, x % kPer));
            fence_proxy_async();
            mbar_arrive(smem_u32(q_first));
        }
        uint32_t gb = 0;
        int t = 0;
        bool ok = true;
        while (ok && u < u1) {
            const int take = (int)min(u1 - u, (int64_t)(cur.blocks - cur.block)), keys = cur.e.keys();
            float m_used = -FLT_MAX, l_sum = 0.f;
            for (int j = 0; j < take; ++j, ++gb) {
                const int b = (int)(gb & 1u);
                const int vc = min(CW, keys - (cur.block + j) * BN - half * CW);   // this warp's keys of the block that exist (may be <= 0)
                const bool got = __all_sync(0xffffffffu, mbar_wait(smem_u32(s_full + b), (gb >> 1) & 1u, abort_flag));
                uint32_t sc[CW];
                if (got) {
                    tc_fence_after();
#pragma unroll
                    for (int c0 = 0; c0 < CW; c0 += 32) tmem_ld32(lane_base + (uint32_t)(b * BN + half * CW + c0), *reinterpret_cast<uint32_t(*)[32]>(&sc[c0]));
                }
                const bool p_free = gb < 2 || __all_sync(0xffffffffu, mbar_wait(smem_u32(pv_done + b), ((gb - 2) >> 1) & 1u, abort_flag));
                float mt = -INFINITY;
                if (got) {
                    tmem_ld_wait();
                    tc_fence_before();
                    __syncwarp();
                    if (lane == 0) mbar_arrive(smem_u32(s_free + b));   // the scores are in registers
                    float mx[4] = {-INFINITY, -INFINITY, -INFINITY, -INFINITY};
                    if (vc == CW) {
#pragma unroll
                        for (int i = 0; i < CW; i += 8) {
#pragma unroll
                            for (int q = 0; q < 4; ++q) mx[q] = fmax3(mx[q], __uint_as_float(sc[i + 2 * q]), __uint_as_float(sc[i + 2 * q + 1]));
                        }
                    } else {
#pragma unroll
                        for (int i = 0; i < CW; ++i)
                            if (i < vc) mx[i & 3] = fmaxf(mx[i & 3], __uint_as_float(sc[i]));
                    }
                    mt = fmaxf(fmaxf(mx[0], mx[1]), fmaxf(mx[2], mx[3])) * k2;
                }
                // the two warps of a quarter agree on the block's maximum (two buffers: the partner may still read the block before)
                float *mx = mx_s + (gb & 1u) * 256;
                mx[half * 128 + row] = mt;
                tc_fence_before();
                const bool bad = named_bar_or(1 + wq, 64, !got || !p_free);
                tc_fence_after();
                if (bad) {
                    ok = false;
                    break;
                }
                mt = fmaxf(mt, mx[(half ^ 1) * 128 + row]);
                bool lost = false;
                if (j == 0) {
                    m_used = fmaxf(mt, -FLT_MAX);   // finite even where no score is
                } else {
                    const bool need = mt > m_used + 8.0f;
                    if (__any_sync(0xffffffffu, need)) {
                        // the exponent's offset follows the maximum only when that has grown by 2^8; this warp's half of its rows of O then
                        const float m_new = need ? mt : m_used, f = fast_exp2(m_used - m_new);
                        l_sum *= f, m_used = m_new;
                        lost = !__all_sync(0xffffffffu, mbar_wait(smem_u32(pv_done + ((gb - 1) & 1u)), ((gb - 1) >> 1) & 1u, abort_flag));
                        if (!lost) {
                            tc_fence_after();
#pragma unroll 1
                            for (int c0 = half * (D / 2); c0 < (half + 1) * (D / 2); c0 += 32) {
                                uint32_t r[32];
                                tmem_ld32(lane_base + (uint32_t)(C::kTmemO + c0), r);
                                tmem_ld_wait();
#pragma unroll
                                for (int i = 0; i < 32; ++i) r[i] = __float_as_uint(__uint_as_float(r[i]) * f);
                                tmem_st32(lane_base + (uint32_t)(C::kTmemO + c0), r);
                            }
                            tmem_st_wait();
                        }
                    }
                }
                (void)lost;   // the abort flag is up: the next meeting point sees a wait that gives up
                const uint64_t k2p = pack_f32x2(k2, k2), mneg = pack_f32x2(-m_used, -m_used);
                uint64_t ls2[2] = {0ull, 0ull};
                auto probabilities = [&](auto masked) {
#pragma unroll
                    for (int c0 = 0; c0 < CW; c0 += 32) {
                        uint32_t packed[16];
#pragma unroll
                        for (int i = 0; i < 16; ++i) {
                            float p0, p1;
                            unpack_f32x2(fma_f32x2(pack_f32x2(__uint_as_float(sc[c0 + 2 * i]), __uint_as_float(sc[c0 + 2 * i + 1])), k2p, mneg), p0, p1);
                            p0 = fast_exp2(p0), p1 = fast_exp2(p1);
                            if (decltype(masked)::value) {
                                if (c0 + 2 * i >= vc) p0 = 0.f;
                                if (c0 + 2 * i + 1 >= vc) p1 = 0.f;
                            }
                            const __nv_bfloat162 h = __floats2bfloat162_rn(p0, p1);
                            packed[i] = *reinterpret_cast<const uint32_t *>(&h);
                            // the sum is of the rounded weights, those that the values get: a row with one heavy key is then as exact as its value
                            ls2[i & 1] = add_f32x2(ls2[i & 1], pack_f32x2(__uint_as_float(packed[i] << 16), __uint_as_float(packed[i] & 0xffff0000u)));
                        }
                        tmem_st16(lane_base + (uint32_t)(C::kTmemP + b * (BN / 2) + ((half * CW + c0) >> 1)), packed);
                    }
                };
                if (vc == CW) probabilities(std::false_type{});
                else probabilities(std::true_type{});
                tmem_st_wait();
                float x0, x1, y0, y1;
                unpack_f32x2(ls2[0], x0, x1), unpack_f32x2(ls2[1], y0, y1);
                l_sum += (x0 + x1) + (y0 + y1);
                tc_fence_before();
                mbar_arrive(smem_u32(p_full + b));
            }
            if (!ok) break;
            // the piece is done: weights of the two halves, then this warp's half of the columns of its rows
            const bool fin = __all_sync(0xffffffffu, mbar_wait(smem_u32(o_final), (uint32_t)(t & 1), abort_flag));
            l_s[half * 128 + row] = l_sum;
            if (named_bar_or(1 + wq, 64, !fin)) {
                ok = false;
                break;
            }
            tc_fence_after();
            const float weight = l_sum + l_s[(half ^ 1) * 128 + row];
            const int head = cur.head, r0 = cur.row_tile * 128, rows = min(128, cur.e.rows - r0);
            const bool begins = cur.block == 0, ends = cur.block + take == cur.blocks;
            const float inv = cur.e.length < 0 ? NAN : keys == 0 ? 0.f : 1.0f / weight;
            float *rec = a.records + (size_t)(2 * cta + (begins ? 1 : 0)) * 128 * (D + 2);
            unsigned char *slab = smOut + warp * 2048;
            int64_t dst[4];   // where the rows that this lane stores begin
#pragma unroll
            for (int i = 0; i < 4; ++i) dst[i] = row_at(a, cur.e.row0, head, r0 + wq * 32 + i * 8 + (lane >> 2), a.out_stride, D) + (lane & 3) * 8;
#pragma unroll 1
            for (int c0 = half * (D / 2); c0 < (half + 1) * (D / 2); c0 += 32) {
                uint32_t r[32];
                tmem_ld32(lane_base + (uint32_t)(C::kTmemO + c0), r);
                tmem_ld_wait();
                if (begins && ends) {
                    // out of the unpacked order, 16 bytes at a time, through shared memory: four lanes then store 64 bytes of a row
#pragma unroll
                    for (int q = 0; q < 4; ++q) {
                        uint32_t pk[4];
                        constexpr int kFrom[8] = {0, 2, 4, 6, 1, 3, 5, 7};   // place of column i in the unpacked order
#pragma unroll
                        for (int i = 0; i < 4; ++i) {
                            const __nv_bfloat162 h =
                                __floats2bfloat162_rn(__uint_as_float(r[8 * q + kFrom[2 * i]]) * inv, __uint_as_float(r[8 * q + kFrom[2 * i + 1]]) * inv);
                            pk[i] = *reinterpret_cast<const uint32_t *>(&h);
                        }
                        *reinterpret_cast<uint4 *>(slab + lane * 64 + ((q ^ ((lane >> 1) & 3)) << 4)) = make_uint4(pk[0], pk[1], pk[2], pk[3]);
                    }
                    __syncwarp();
#pragma unroll
                    for (int i = 0; i < 4; ++i) {
                        const int rl = i * 8 + (lane >> 2), q = lane & 3;
                        const uint4 o = *reinterpret_cast<const uint4 *>(slab + rl * 64 + ((q ^ ((rl >> 1) & 3)) << 4));
                        if (wq * 32 + rl < rows) *reinterpret_cast<uint4 *>(static_cast<__nv_bfloat16 *>(a.out) + dst[i] + c0) = o;
                    }
                    __syncwarp();
                } else if (row < rows) {
#pragma unroll
                    for (int i = 0; i < 8; ++i)
                        *reinterpret_cast<uint4 *>(rec + row * D + c0 + 4 * i) = make_uint4(r[4 * i], r[4 * i + 1], r[4 * i + 2], r[4 * i + 3]);
                }
            }
            tc_fence_before();
            __syncwarp();
            if (lane == 0) mbar_arrive(smem_u32(o_free));
            if (!(begins && ends) && half == 0 && row < rows) rec[128 * D + 2 * row] = m_used, rec[128 * D + 2 * row + 1] = weight;
            if (ends && !begins && tid == 0) {
                const int64_t tile_u0 = u - cur.block;
                int s = cta;
                while (s > 0 && cut(total, ctas, s) > tile_u0) --s;
                PieceHeader h{};
                h.row0 = cur.e.row0, h.first_cta = s, h.head = head, h.r0 = r0, h.rows = rows;
                a.headers[cta] = h;
            }
            if (cur.e.length < 0 && tid == 0) atomicOr(c.status, AIF_STATUS_BAD_ID);
            u += take, ++t;
            if (u < u1) plan_next(a, cur);
        }
    } else if (warp == C::kQkWarp) {
        // ===================== scores = Q K^T =====================
        if (lane == 0) {
            constexpr uint32_t idesc = umma_idesc_bf16(128, BN);
            uint32_t gb = 0;
            int t = 0;
            bool ok = true;
            while (ok && u < u1) {
                const int take = (int)min(u1 - u, (int64_t)(cur.blocks - cur.block)), qb = t % kQB;
                ok = t == 0 ? mbar_wait(smem_u32(q_first), 0u, abort_flag) : mbar_wait(smem_u32(q_full + qb), (uint32_t)(((t - 1) / kQB) & 1), abort_flag);
                const uint64_t qd = umma_desc_sw128(smem_u32(smQ + qb * C::kQBytes));
                for (int j = 0; ok && j < take; ++j, ++gb) {
                    const int s = (int)(gb % kS);
                    if (!mbar_wait(smem_u32(k_full + s), (gb / kS) & 1u, abort_flag) ||
                        (gb >= 2 && !mbar_wait(smem_u32(s_free + (gb & 1u)), ((gb - 2) >> 1) & 1u, abort_flag))) {
                        ok = false;
                        break;
                    }
                    tc_fence_after();
                    const uint64_t kd = umma_desc_sw128(smem_u32(smKV + s * C::kStageBytes));
#pragma unroll
                    for (int kk = 0; kk < D / 16; ++kk)
                        umma_bf16(tmem + (gb & 1u) * BN, qd + (uint64_t)((kk >> 2) * (16384 >> 4) + 2 * (kk & 3)),
                                  kd + (uint64_t)((kk >> 2) * (C::kChunkBytes >> 4) + 2 * (kk & 3)), idesc, kk > 0 ? 1u : 0u);
                    umma_commit(smem_u32(s_full + (gb & 1u)));
                    if (j == take - 1) umma_commit(smem_u32(q_empty + qb));
                }
                u += take, ++t;
                if (u < u1) plan_next(a, cur);
            }
        }
        __syncwarp();
    } else if (warp == C::kPvWarp) {
        // ===================== O += P V =====================
        if (lane == 0) {
            constexpr uint32_t idesc = umma_idesc_bf16_bmn(128, D);
            uint32_t gb = 0;
            int t = 0;
            bool ok = true;
            while (ok && u < u1) {
                const int take = (int)min(u1 - u, (int64_t)(cur.blocks - cur.block));
                for (int j = 0; j < take; ++j, ++gb) {
                    const int s = (int)(gb % kS);
                    if (!mbar_wait(smem_u32(p_full + (gb & 1u)), (gb >> 1) & 1u, abort_flag) ||
                        (!SHARED && !mbar_wait(smem_u32(v_full + s), (gb / kS) & 1u, abort_flag)) ||
                        (j == 0 && t > 0 && !mbar_wait(smem_u32(o_free), (uint32_t)((t - 1) & 1), abort_flag))) {
                        ok = false;
                        break;
                    }
                    tc_fence_after();
                    const uint64_t vd = umma_desc_mn_sw128(smem_u32(smKV + s * C::kStageBytes + (SHARED ? 0 : C::kTileBytes)), C::kChunkBytes);
                    const uint32_t p_tmem = tmem + (uint32_t)(C::kTmemP + (gb & 1u) * (BN / 2));
#pragma unroll
                    for (int kk = 0; kk < BN / 16; ++kk)
                        umma_bf16_ts(tmem + C::kTmemO, p_tmem + (uint32_t)(kk * 8), vd + (uint64_t)(kk * (2048 >> 4)), idesc, (j > 0 || kk > 0) ? 1u : 0u);
                    umma_commit(smem_u32(pv_done + (gb & 1u)));
                    umma_commit(smem_u32(kv_empty + s));   // (Q K^T of the block, the stage's other reader, was done before there were probabilities)
                    if (j == take - 1) umma_commit(smem_u32(o_final));
                }
                u += take, ++t;
                if (u < u1) plan_next(a, cur);
            }
        }
        __syncwarp();
    } else if (warp < C::kUnpackWarp) {
        // ===================== query rows of the next tiles (64 threads) =====================
        const int x0 = tid - C::kQWarp * 32;
        int t = 0;
        while (u < u1) {
            u += min(u1 - u, (int64_t)(cur.blocks - cur.block)), ++t;
            if (u >= u1) break;
            plan_next(a, cur);
            const int qb = t % kQB;
            if (t >= kQB && !mbar_wait(smem_u32(q_empty + qb), (uint32_t)(((t - kQB) / kQB) & 1), abort_flag)) break;
            unsigned char *q = smQ + qb * C::kQBytes;
            constexpr int kPer = D / 8;
#pragma unroll 8
            for (int x = x0; x < 128 * kPer; x += 64) put_query(q, x / kPer, x % kPer, query_piece(cur, x / kPer, x % kPer));
            fence_proxy_async();
            mbar_arrive(smem_u32(q_full + qb));
        }
    } else {
        // ===================== keys and values (128 threads) =====================
        constexpr int kSplit = 128 / BN;                // threads to a key
        constexpr int kBlk = D / 32 / kSplit;           // blocks of 32 elements of a thread
        const int x = tid - C::kUnpackWarp * 32, r = x % BN, b0 = x / BN * kBlk;
        struct Codes {
            uint4 w[kBlk];
            uint32_t sc[(kBlk + 3) / 4];
        };
        Codes next[C::kKinds];
        bool bad_page = false;
        // the walk over blocks runs two ahead for page numbers, one ahead for codes
        struct Walk {
            int64_t u;
            Cursor at;
        } ahead{u0, cur};
        auto step = [&](Walk &w) {
            if (++w.u >= u1) return;
            if (++w.at.block >= w.at.blocks) plan_next(a, w.at);
        };
        // page and row of this thread's key of the block that the walk stands on; page -1: no such key, -2: no such page
        auto place = [&](const Walk &w, int &page, int &in_page, int &head) {
            page = -1, in_page = 0, head = 0;
            if (w.u >= u1) return;
            const int v = w.at.block * BN + r;
            if (v >= w.at.e.keys()) return;
            const int key = w.at.e.key(v);
            head = w.at.head, in_page = key & (c.page_rows() - 1);
            page = __ldg(c.table + (size_t)w.at.e.seq * c.max_pages + (key >> c.page_shift));
            if (!c.holds(page)) page = -2;
        };
        auto fetch = [&](int page, int in_page, int head) {
#pragma unroll
            for (int k = 0; k < C::kKinds; ++k) {
#pragma unroll
                for (int b = 0; b < kBlk; ++b) next[k].w[b] = make_uint4(0u, 0u, 0u, 0u);
                next[k].sc[0] = page == -2 ? 0xffffffffu : 0u;
                if (page < 0) {
                    bad_page |= page == -2;
                    continue;
                }
                const size_t row = c.row(page, head, in_page);
                const uint4 *p = reinterpret_cast<const uint4 *>(c.codes[k] + row * (D / 2)) + b0;
#pragma unroll
                for (int b = 0; b < kBlk; ++b) next[k].w[b] = __ldg(p + b);
                const uint8_t *ps = c.scales[k] + row * (D / 32) + b0;
                next[k].sc[0] = __ldg(reinterpret_cast<const uint32_t *>(ps));
            }
        };
        int page = -1, in_page = 0, head = 0;
        if (work) {
            place(ahead, page, in_page, head);
            fetch(page, in_page, head);
            step(ahead);
            place(ahead, page, in_page, head);
        }
        uint32_t gb = 0;
        for (int64_t i = u0; i < u1; ++i, ++gb) {
            Codes now[C::kKinds];
#pragma unroll
            for (int k = 0; k < C::kKinds; ++k) now[k] = next[k];
            if (i + 1 < u1) {
                fetch(page, in_page, head);
                step(ahead);
                place(ahead, page, in_page, head);
            }
            const int s = (int)(gb % kS);
            if (!mbar_wait(smem_u32(kv_empty + s), ((gb / kS) & 1u) ^ 1u, abort_flag)) break;
#pragma unroll
            for (int k = 0; k < C::kKinds; ++k) {
                unsigned char *tile = smKV + s * C::kStageBytes + k * C::kTileBytes + r * 128;
#pragma unroll
                for (int b = 0; b < kBlk; ++b) {
                    const UnpackScale us((now[k].sc[0] >> (8 * b)) & 255u);
                    unsigned char *chunk = tile + ((b0 + b) >> 1) * C::kChunkBytes;
                    const uint32_t w[4] = {now[k].w[b].x, now[k].w[b].y, now[k].w[b].z, now[k].w[b].w};
#pragma unroll
                    for (int i4 = 0; i4 < 4; ++i4)
                        *reinterpret_cast<uint4 *>(chunk + (((((b0 + b) & 1) * 4 + i4) ^ (r & 7)) << 4)) = unpack8(w[i4], us);
                }
                fence_proxy_async();
                mbar_arrive(smem_u32((k == 0 ? k_full : v_full) + s));
            }
        }
        if (bad_page) atomicOr(c.status, AIF_STATUS_BAD_ID);
    }

    if (*abort_flag) {
        if (tid == 0) atomicOr(c.status, AIF_STATUS_TIMEOUT);
        const long long t0 = clock64();
        while (clock64() - t0 < 2000000ll) __nanosleep(1000);   // products in flight end before their memory is given up
    }
    tc_fence_before();
    __syncthreads();
    if (warp == C::kQkWarp) tmem_dealloc(tmem, 512);
}

template <bool SHARED>
cudaError_t run_tc(const AttCall &a, int grid, cudaStream_t st)
{
    using C = Att4Cfg<SHARED>;
    cudaError_t e = allow_smem<k_att4_tc<SHARED>>(C::kSmem);
    if (e != cudaSuccess) return e;
    count_launch();
    return launch_pdl(k_att4_tc<SHARED>, dim3(grid), dim3(C::kThreads), C::kSmem, st, a);
}

}  // namespace

cudaError_t launch_att4_tc(const AttCall &a, int grid, cudaStream_t st)
{
    return a.c.codes[0] == a.c.codes[1] ? run_tc<true>(a, grid, st) : run_tc<false>(a, grid, st);
}

}  // namespace aif
