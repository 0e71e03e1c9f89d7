// Attention of many query rows over sequences in the 4-bit cache on the tensor cores (sm_100a), bf16, d = 64 and 128:
//   out_i = softmax_j(scale q_i k_j) v   for tiles of 256 query rows (queries x heads of a group) of one sequence.
//
// The 4-bit codes are unpacked to bf16 on their way into shared memory (exact: two significant bits and a power of two), once for 256 rows, and
// both products run as bf16 tcgen05 products with fp32 accumulators in tensor memory.  A tile's two halves of 128 rows take turns: while the
// tensor cores work for one, the exponentials of the other are formed.  One CTA per SM takes an even share of the launch's units
// (aif_cache4_plan.cuh).  Warps:
//   0-3, 4-7  queries, softmax and output of the first and the second half: a thread owns a row; scores from tensor memory, exponentials in fp32,
//             probabilities back over the scores as bf16 pairs; at the end of a tile they bring the next one's query rows, normalise and store
//   8, 9      issue scores = Q K^T, up to two blocks ahead of the softmax (two buffers of scores per half), and O += P V with V read MN-major from
//             the tile K was read from
//   10-15     unpack keys and values, 32 rows of a block at a time in turn (two to a block): a thread takes a key row; the codes of its next one are
//             in flight in registers meanwhile, and the page number of the one after that
// The maximum costs the softmax a third of its time, so it is left out where it cannot matter: |q| (formed as the queries are brought) times a bound of |k| (from the
// scales of a block's keys, as they are unpacked) bounds every score; up to 2^+-82 the exponentials need no offset, since neither fp32 sums nor bf16
// probabilities lose precision with magnitude.
// Eight codes of a word come apart as the pairs (0,4) (1,5) (2,6) (3,7) with two shifts, two masks and a multiplication each; queries are put
// into the same order as they are brought, and sums are taken out of it as they are stored.
// Bound: what the softmax warps issue and wait for, not one unit: issue slots 59 %, exponentials 51 %, products 50 % of the cycles, ALU 43 %; a scheduler's warps wait longest for
// scores and probabilities on their way from and to tensor memory.  (A polynomial on other units in place of a quarter or half of the exponentials gained nothing, half of the products left out
// 1 %.)  k_att_tc does the same sizes with bf16 keys in 672 us: it has no unpacking warps, and its Q K^T of block j + 2 does not wait for P V of block j, whose probabilities lie
// in the columns of the scores here.  Instruction fetch: five kinds of code share a multiprocessor, so parts stand once and cold ones aside.
// 16 x 10^4 rows x 10^4 keys, d = 128: 782 us, 1050 TFLOP/s; 148 x 256 x 8192: 161 us, d = 64 136 us, values of their own 180 us; one tile of two blocks 17 us, of which 3
// plan, 2.5 queries, 2.3 the output.
// Rounding: probabilities are rounded to bf16 for the product (relative 2^-8 each), and their sum is of the rounded ones, everything else is fp32.
#include <cfloat>
#include <type_traits>

#include "aif_cache4_plan.cuh"
#include "aif_tc_ptx.cuh"

namespace aif {
namespace {

template <int D, bool SHARED>
struct PairCfg {
    static constexpr int kBN = 64;                         // keys of a block
    static constexpr int kChunks = D / 64;                // 64-column (128-byte) chunks of a row
    static constexpr int kHalfBytes = kChunks * 128 * 128;   // query rows of one half
    static constexpr int kQBytes = 2 * kHalfBytes;
    static constexpr int kChunkBytes = kBN * 128;
    static constexpr int kTileBytes = kChunks * kChunkBytes;
    static constexpr int kKinds = SHARED ? 1 : 2;
    static constexpr int kStages = SHARED ? 6 : 4;
    static constexpr int kStageBytes = kKinds * kTileBytes;
    static constexpr int kThreads = 512;
    static constexpr int kTmemS = 0, kTmemO = 256;        // scores (then probabilities) of the halves at 0 and 128, two buffers of 64 columns each; sums at 256 and 256 + D
    static constexpr int kOutBytes = 8 * 2048;            // 32 rows x 64 bytes for each softmax warp
    static constexpr size_t kSmem = 1024 + kQBytes + kStages * kStageBytes + kOutBytes + 512 + 256 * 4 + kStages * 2 * 2 * 4;
};

// Where no maximum is taken, exponents of weights lie within +-kFreeScore, the offset within +-kFreeOffset, scales of values between 2^-36 and 2^8: a weight is at most
// 2^86, a value 6 x 2^8 < 2^10.6, a sequence 2^30 rows, so sums stay below 2^126.6, those of a tile's joined pieces among them; and the product of a weight of
// 2^-86 or more with a value of 2^-37 or more is no subnormal.  (Scales of 2^-127 do not count: their values are zero or within 2^-124 of it.)
constexpr float kFreeScore = 82.f, kFreeOffset = 4.f;
constexpr uint32_t kFreeLow = 127u - 36u, kFreeTop = 127u + 8u;   // scale bytes

template <int D, bool SHARED>
__global__ void __launch_bounds__(512, 1) k_att4_pair(const AttCall a)
{
    using C = PairCfg<D, SHARED>;
    constexpr int BN = C::kBN, kS = C::kStages;
    extern __shared__ unsigned char smem_dyn[];
    unsigned char *base = reinterpret_cast<unsigned char *>(((uintptr_t)smem_dyn + 1023) & ~(uintptr_t)1023);
    unsigned char *smQ = base, *smKV = smQ + C::kQBytes, *smOut = smKV + kS * C::kStageBytes;
    uint64_t *bars = reinterpret_cast<uint64_t *>(smOut + C::kOutBytes);
    uint64_t *k_full = bars, *v_full = bars + kS, *kv_empty = bars + 2 * kS;
    uint64_t *s_full = bars + 3 * kS, *p_full = s_full + 4, *pv_done = p_full + 4, *q_full = pv_done + 4;   // [half][buffer]; [half]
    uint32_t *tmem_slot = reinterpret_cast<uint32_t *>(q_full + 2);
    volatile uint32_t *abort_flag = tmem_slot + 1;
    float *q_norm = reinterpret_cast<float *>(smOut + C::kOutBytes + 512);   // [256], squared
    float2 *k_bound = reinterpret_cast<float2 *>(q_norm + 256);        // [stage][32 rows each]: largest sum of a row's squared scales; 0 where the values' scales allow weights of any size
    __shared__ PlanShared<C::kThreads> plan;

    const Cache4 &c = a.c;
    const int tid = threadIdx.x, warp = tid >> 5, lane = tid & 31;
    if (tid == 0) {
        for (int s = 0; s < kS; ++s) mbar_init(smem_u32(k_full + s), BN), mbar_init(smem_u32(v_full + s), BN), mbar_init(smem_u32(kv_empty + s), 1);
        for (int b = 0; b < 4; ++b) mbar_init(smem_u32(s_full + b), 1), mbar_init(smem_u32(p_full + b), 128), mbar_init(smem_u32(pv_done + b), 1);
        for (int b = 0; b < 2; ++b) mbar_init(smem_u32(q_full + b), 128);
        *abort_flag = 0u;
        asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
    }
    if (warp == 8) tmem_alloc(smem_u32(tmem_slot), 512);
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
    Cursor cur = share.cur;
    int64_t u = u0;
    auto tile_of = [&](const Cursor &at, int &head, int &r0, int &rows) {
        head = at.head, r0 = at.row_tile * 256, rows = min(256, at.e.rows - r0);
    };

    if (warp < 8) {
        // ===================== queries, softmax, output =====================
        const int x = warp >> 2, wq = warp & 3, row = wq * 32 + lane;   // half of the tile, quarter of its rows
        // This half's query rows of the tile that `cur` stands on, in the order of the unpacked codes, and their norms.  The half's last scores have arrived
        // by then, so nothing reads the rows before.
        auto bring_queries = [&]() {
            int head, r0, rows;
            tile_of(cur, head, r0, rows);
            if (rows <= x * 128) return;
            constexpr int kPer = D / 8;   // pieces of 16 bytes of a row
            const int piece = lane % kPer, first = wq * 32 + lane / kPer;   // a warp brings the rows it owns
            unsigned char *q = smQ + x * C::kHalfBytes;
            uint4 w[kPer];
#pragma unroll
            for (int i = 0; i < kPer; ++i) {
                const int r = x * 128 + first + i * (32 / kPer);
                w[i] = make_uint4(0u, 0u, 0u, 0u);
                if (r < rows) w[i] = __ldg(reinterpret_cast<const uint4 *>(static_cast<const __nv_bfloat16 *>(a.q) + row_at(a, cur.e.row0, head, r0 + r, a.q_stride, D) + piece * 8));
            }
            float n2[kPer];   // sums of squares of this lane's pieces
#pragma unroll
            for (int i = 0; i < kPer; ++i) {
                const int r = first + i * (32 / kPer);
                const uint4 o = make_uint4(__byte_perm(w[i].x, w[i].z, 0x5410), __byte_perm(w[i].x, w[i].z, 0x7632), __byte_perm(w[i].y, w[i].w, 0x5410), __byte_perm(w[i].y, w[i].w, 0x7632));
                *reinterpret_cast<uint4 *>(q + (piece >> 3) * 16384 + r * 128 + (((piece & 7) ^ (r & 7)) << 4)) = o;
                const uint32_t ww[4] = {w[i].x, w[i].y, w[i].z, w[i].w};
                n2[i] = 0.f;
#pragma unroll
                for (int y = 0; y < 4; ++y) {
                    const float lo = __uint_as_float(ww[y] << 16), hi = __uint_as_float(ww[y] & 0xffff0000u);
                    n2[i] = fmaf(lo, lo, fmaf(hi, hi, n2[i]));
                }
            }
            // kPer neighbouring lanes have kPer rows: each step hands half of a lane's sums over, and the lane of piece i ends with row i
#pragma unroll
            for (int y = kPer / 2; y > 0; y >>= 1) {
                const bool upper = (lane & y) != 0;
#pragma unroll
                for (int i = 0; i < y; ++i) {
                    const float give = upper ? n2[i] : n2[i + y], keep = upper ? n2[i + y] : n2[i];
                    n2[i] = keep + __shfl_xor_sync(0xffffffffu, give, y);
                }
            }
            q_norm[x * 128 + first + piece * (32 / kPer)] = n2[0];
            fence_proxy_async();
            __syncwarp();   // (the norms are read by the lanes that own the rows)
            mbar_arrive(smem_u32(q_full + x));
        };
        const uint32_t ts0 = tmem + ((uint32_t)(wq * 32) << 16) + (uint32_t)(C::kTmemS + x * 128), to = tmem + ((uint32_t)(wq * 32) << 16) + (uint32_t)(C::kTmemO + x * D);
        const float k2 = a.scale_log2;
        uint32_t gb = 0, cb = 0;   // blocks of this half; of the CTA, up to the tile's first
        bool ok = true, pending = false;   // pending: the tile `done` has its weights and waits for its last products
        Cursor done = cur;
        int done_take = 0;
        float m_used = 0.f, l_sum = 0.f;
        // (one round more than there are tiles: the code of every part stands once, instructions are what these warps wait for most)
        while (ok) {
            if (u < u1) bring_queries();   // while the last products of the tile before run
            if (pending) {
                const int take = done_take, keys = done.e.keys();
                int head, r0, rows;
                tile_of(done, head, r0, rows);
                if (!__all_sync(0xffffffffu, mbar_wait(smem_u32(pv_done + 2 * x + ((gb - 1) & 1u)), ((gb - 1) >> 1) & 1u, abort_flag))) break;
                tc_fence_after();
                const bool begins = done.block == 0, ends = done.block + take == done.blocks;
                const float inv = done.e.length < 0 ? NAN : keys == 0 ? 0.f : 1.0f / l_sum;
                const int r = x * 128 + row;
                float *rec = a.records + (size_t)(2 * cta + (begins ? 1 : 0)) * 256 * (D + 2);
                unsigned char *slab = smOut + warp * 2048;
                int64_t dst[4];   // where the rows that this lane stores begin
#pragma unroll
                for (int i = 0; i < 4; ++i) dst[i] = row_at(a, done.e.row0, head, r0 + x * 128 + wq * 32 + i * 8 + (lane >> 2), a.out_stride, D) + (lane & 3) * 8;
#pragma unroll 1
                for (int c0 = 0; c0 < D; c0 += 32) {
                    uint32_t v[32];
                    tmem_ld32(to + (uint32_t)c0, v);
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
                                    __floats2bfloat162_rn(__uint_as_float(v[8 * q + kFrom[2 * i]]) * inv, __uint_as_float(v[8 * q + kFrom[2 * i + 1]]) * inv);
                                pk[i] = *reinterpret_cast<const uint32_t *>(&h);
                            }
                            *reinterpret_cast<uint4 *>(slab + lane * 64 + ((q ^ ((lane >> 1) & 3)) << 4)) = make_uint4(pk[0], pk[1], pk[2], pk[3]);
                        }
                        __syncwarp();
#pragma unroll
                        for (int i = 0; i < 4; ++i) {
                            const int rl = i * 8 + (lane >> 2), q = lane & 3;
                            const uint4 o = *reinterpret_cast<const uint4 *>(slab + rl * 64 + ((q ^ ((rl >> 1) & 3)) << 4));
                            if (x * 128 + wq * 32 + rl < rows) *reinterpret_cast<uint4 *>(static_cast<__nv_bfloat16 *>(a.out) + dst[i] + c0) = o;
                        }
                        __syncwarp();
                    } else if (r < rows) {
#pragma unroll
                        for (int i = 0; i < 8; ++i) *reinterpret_cast<uint4 *>(rec + (size_t)r * D + c0 + 4 * i) = make_uint4(v[4 * i], v[4 * i + 1], v[4 * i + 2], v[4 * i + 3]);
                    }
                }
                tc_fence_before();
                if (!(begins && ends) && r < rows) rec[256 * D + 2 * r] = m_used, rec[256 * D + 2 * r + 1] = l_sum;
                if (ends && !begins && tid == 0) {
                    const int64_t tile_u0 = u - take - done.block;
                    int s = cta;
                    while (s > 0 && cut(total, ctas, s) > tile_u0) --s;
                    PieceHeader h{};
                    h.row0 = done.e.row0, h.first_cta = s, h.head = head, h.r0 = r0, h.rows = rows;
                    a.headers[cta] = h;
                }
                if (done.e.length < 0 && tid == 0) atomicOr(c.status, AIF_STATUS_BAD_ID);
            }
            if (u >= u1) break;
            const int take = (int)min(u1 - u, (int64_t)(cur.blocks - cur.block)), keys = cur.e.keys();
            int head, r0, rows;
            tile_of(cur, head, r0, rows);
            pending = rows > x * 128;
            if (pending) {
                m_used = 0.f, l_sum = 0.f;
                const float reach = sqrtf(q_norm[x * 128 + row]) * k2;   // times a bound of |k|: a bound of the row's scores
                uint32_t sc[BN];
                auto bring_scores = [&](uint32_t n) {
                    if (!__all_sync(0xffffffffu, mbar_wait(smem_u32(s_full + 2 * x + (n & 1u)), (n >> 1) & 1u, abort_flag))) return false;
                    tc_fence_after();
                    tmem_ld32(ts0 + (n & 1u) * BN, *reinterpret_cast<uint32_t(*)[32]>(&sc[0]));
                    return true;
                };
                for (int j = 0; j < take; ++j, ++gb) {
                    const int vc = min(BN, keys - (cur.block + j) * BN);   // keys of the block that exist (none: an empty sequence)
                    const uint32_t b = gb & 1u, ts = ts0 + b * BN;
                    // the first half of the block's scores was asked for with the block before; the second comes while the first is at work
                    if (!(ok = bring_scores(gb))) break;
                    const float4 kb = *reinterpret_cast<const float4 *>(k_bound + (cb + (uint32_t)j) % kS * 2);
                    // a code is at most 6: |k|^2 <= 36 x 32 x the sum of its blocks' squared scales
                    bool free = reach * 33.9411255f * sqrtf(fmaxf(kb.x, kb.z)) <= kFreeScore && fabsf(m_used) <= kFreeOffset && kb.y + kb.w == 0.f;
                    free = __all_sync(0xffffffffu, free);   // (NaN: not)
                    tmem_ld_wait();
                    tmem_ld32(ts + 32, *reinterpret_cast<uint32_t(*)[32]>(&sc[32]));
                    if (__builtin_expect(!free || vc < BN, 0)) {
                        tmem_ld_wait();
                        if (vc < BN) {
#pragma unroll
                            for (int i = 0; i < BN; ++i)
                                if (i >= vc) sc[i] = 0xff800000u;   // no key, no weight
                        }
                        if (!free) {
                            float mx[4] = {-INFINITY, -INFINITY, -INFINITY, -INFINITY};
#pragma unroll
                            for (int i = 0; i < BN; i += 8)
#pragma unroll
                                for (int q = 0; q < 4; ++q) mx[q] = fmax3(mx[q], __uint_as_float(sc[i + 2 * q]), __uint_as_float(sc[i + 2 * q + 1]));
                            const float mt = fmaxf(fmaxf(mx[0], mx[1]), fmaxf(mx[2], mx[3])) * k2;
                            if (j == 0) {
                                m_used = fmaxf(mt, -FLT_MAX);   // finite even where no score is
                            } else {
                                const bool need = mt > m_used + 8.0f;
                                if (__any_sync(0xffffffffu, need)) {
                                    // the exponent's offset follows the maximum only when that has grown by 2^8; this warp's rows of O then
                                    const float m_new = need ? mt : m_used, f = fast_exp2(m_used - m_new);
                                    l_sum *= f, m_used = m_new;
                                    if (!__all_sync(0xffffffffu, mbar_wait(smem_u32(pv_done + 2 * x + (b ^ 1u)), ((gb - 1) >> 1) & 1u, abort_flag))) {
                                        ok = false;
                                        break;
                                    }
                                    tc_fence_after();
#pragma unroll 1
                                    for (int c0 = 0; c0 < D; c0 += 16) {
                                        uint32_t r[16];
                                        tmem_ld16(to + (uint32_t)c0, r);
                                        tmem_ld_wait();
#pragma unroll
                                        for (int i = 0; i < 16; ++i) r[i] = __float_as_uint(__uint_as_float(r[i]) * f);
                                        tmem_st16(to + (uint32_t)c0, r);
                                    }
                                }
                            }
                        }
                    }
                    const uint64_t k2p = pack_f32x2(k2, k2), mneg = pack_f32x2(-m_used, -m_used);
                    uint64_t ls2[2] = {0ull, 0ull};
                    // probabilities over the scores, as bf16 pairs
#pragma unroll
                    for (int c0 = 0; c0 < BN; c0 += 32) {
                        if (c0 == 32) tmem_ld_wait();
                        uint32_t packed[16];
#pragma unroll
                        for (int i = 0; i < 16; ++i) {
                            float p0, p1;
                            unpack_f32x2(fma_f32x2(pack_f32x2(__uint_as_float(sc[c0 + 2 * i]), __uint_as_float(sc[c0 + 2 * i + 1])), k2p, mneg), p0, p1);
                            const __nv_bfloat162 h = __floats2bfloat162_rn(fast_exp2(p0), fast_exp2(p1));
                            packed[i] = *reinterpret_cast<const uint32_t *>(&h);
                            // the sum is of the rounded weights, those that the values get: a row with one heavy key is then as exact as its value
                            ls2[i & 1] = add_f32x2(ls2[i & 1], pack_f32x2(__uint_as_float(packed[i] << 16), __uint_as_float(packed[i] & 0xffff0000u)));
                        }
                        tmem_st16(ts + (uint32_t)(c0 / 2), packed);
                    }
                    tmem_st_wait();
                    float x0, x1, y0, y1;
                    unpack_f32x2(ls2[0], x0, x1), unpack_f32x2(ls2[1], y0, y1);
                    l_sum += (x0 + x1) + (y0 + y1);
                    tc_fence_before();
                    mbar_arrive(smem_u32(p_full + 2 * x + b));
                }
                if (!ok) break;
            }
            done = cur, done_take = take;
            u += take, cb += (uint32_t)take;
            if (u < u1) plan_next(a, cur);
        }
    } else if (warp < 10) {
        // ===================== products =====================
        // The whole warp walks (descriptors and addresses then live in uniform registers); one lane issues.
        const uint32_t one = elect_one();
        constexpr uint32_t idesc_qk = umma_idesc_bf16(128, BN), idesc_pv = umma_idesc_bf16_bmn(128, D);
        uint32_t gb = 0, hb[2] = {0u, 0u}, qbits = 0;   // blocks of the CTA; of each half; bit x: parity of the half's tiles
        bool ok = true;
        using First = std::integral_constant<int, 0>;
        using Second = std::integral_constant<int, 1>;
        if (warp == 8) {
            const uint64_t qd0 = umma_desc_sw128(smem_u32(smQ)), kd0 = umma_desc_sw128(smem_u32(smKV));
            auto scores = [&](auto half) {
                constexpr int x = decltype(half)::value;
                const uint32_t n = hb[x]++, b = n & 1u;
                // the buffer's probabilities, two blocks ago, have been used
                if (n >= 2 && !mbar_wait(smem_u32(pv_done + 2 * x + b), ((n - 2) >> 1) & 1u, abort_flag)) return false;
                tc_fence_after();
                const uint64_t q = qd0 + (uint64_t)(x * (C::kHalfBytes >> 4)), k = kd0 + (uint64_t)(gb % kS * (uint32_t)(C::kStageBytes >> 4));
                const uint32_t d_tmem = tmem + (uint32_t)(C::kTmemS + x * 128) + b * BN;
#pragma unroll
                for (int kk = 0; kk < D / 16; ++kk)
                    umma_bf16_if(one, d_tmem, q + (uint64_t)((kk >> 2) * (16384 >> 4) + 2 * (kk & 3)), k + (uint64_t)((kk >> 2) * (C::kChunkBytes >> 4) + 2 * (kk & 3)), idesc_qk, kk > 0 ? 1u : 0u);
                umma_commit_if(one, smem_u32(s_full + 2 * x + b));
                return true;
            };
            while (ok && u < u1) {
                const int take = (int)min(u1 - u, (int64_t)(cur.blocks - cur.block));
                int head, r0, rows;
                tile_of(cur, head, r0, rows);
                const bool two = rows > 128;
                for (int x = 0; ok && x < (two ? 2 : 1); ++x) {
                    ok = mbar_wait(smem_u32(q_full + x), (qbits >> x) & 1u, abort_flag);
                    qbits ^= 1u << x;
                }
                for (int j = 0; ok && j < take; ++j, ++gb) {
                    ok = mbar_wait(smem_u32(k_full + gb % kS), (gb / kS) & 1u, abort_flag);
                    ok = ok && scores(First{}) && (!two || scores(Second{}));
                }
                u += take;
                if (u < u1) plan_next(a, cur);
            }
        } else {
            const uint64_t vd0 = umma_desc_mn_sw128(smem_u32(smKV + (SHARED ? 0 : C::kTileBytes)), C::kChunkBytes);
            auto values = [&](auto half, bool first) {
                constexpr int x = decltype(half)::value;
                const uint32_t n = hb[x]++, b = n & 1u;
                if (!mbar_wait(smem_u32(p_full + 2 * x + b), (n >> 1) & 1u, abort_flag)) return false;
                tc_fence_after();
                const uint64_t v = vd0 + (uint64_t)(gb % kS * (uint32_t)(C::kStageBytes >> 4));
                const uint32_t o_tmem = tmem + (uint32_t)(C::kTmemO + x * D), p_tmem = tmem + (uint32_t)(C::kTmemS + x * 128) + b * BN;
#pragma unroll
                for (int kk = 0; kk < BN / 16; ++kk)
                    umma_bf16_ts_if(one, o_tmem, p_tmem + (uint32_t)(kk * 8), v + (uint64_t)(kk * (2048 >> 4)), idesc_pv, first && kk == 0 ? 0u : 1u);
                umma_commit_if(one, smem_u32(pv_done + 2 * x + b));
                return true;
            };
            while (ok && u < u1) {
                const int take = (int)min(u1 - u, (int64_t)(cur.blocks - cur.block));
                int head, r0, rows;
                tile_of(cur, head, r0, rows);
                const bool two = rows > 128;
                for (int j = 0; ok && j < take; ++j, ++gb) {
                    if (!SHARED) ok = mbar_wait(smem_u32(v_full + gb % kS), (gb / kS) & 1u, abort_flag);
                    ok = ok && values(First{}, j == 0) && (!two || values(Second{}, j == 0));
                    umma_commit_if(one, smem_u32(kv_empty + gb % kS));   // (Q K^T of the block, the stage's other reader, was done before there were probabilities)
                }
                u += take;
                if (u < u1) plan_next(a, cur);
            }
        }
    } else {
        // ===================== keys and values (six warps) =====================
        constexpr int kBlk = D / 32;   // blocks of 32 elements of a row
        constexpr int kUnpackers = 6;
        // item i: rows 32 (i % 2) .. of the CTA's block i / 2
        const int64_t items = 2 * (u1 - u0);
        struct Codes {
            uint4 w[kBlk];
            uint32_t sc;
        };
        Codes next[C::kKinds] = {};
        bool bad_page = false;
        // The walk runs two of this warp's items ahead for page numbers, one ahead for codes.
        int64_t ahead = u0;
        // page and row of this thread's key of an item; no page where there is no such key
        constexpr int kNoKey = -0x40000000;
        int page = kNoKey, in_page = 0, head = 0;
        auto place = [&](int64_t item) {
            page = kNoKey;
            if (item >= items) return;
            while (ahead < u0 + (item >> 1)) {
                ++ahead;
                if (++cur.block >= cur.blocks) plan_next(a, cur);
            }
            const int v = cur.block * BN + (int)(item & 1) * 32 + lane;
            if (v >= cur.e.keys()) return;
            const int key = cur.e.key(v);
            head = cur.head, in_page = key & (c.page_rows() - 1);
            page = __ldg(c.table + (size_t)cur.e.seq * c.max_pages + (key >> c.page_shift));
        };
        auto fetch = [&]() {
            const bool ok = c.holds(page), missing = !ok && page != kNoKey;
            const size_t at = ok ? c.row(page, head, in_page) : 0;
            bad_page |= missing;
#pragma unroll
            for (int k = 0; k < C::kKinds; ++k) {
#pragma unroll
                for (int b = 0; b < kBlk; ++b) next[k].w[b] = make_uint4(0u, 0u, 0u, 0u);
                next[k].sc = missing ? 0xffffffffu : 0u;
                if (!ok) continue;
                const uint4 *p = reinterpret_cast<const uint4 *>(c.codes[k] + at * (D / 2));
#pragma unroll
                for (int b = 0; b < kBlk; ++b) next[k].w[b] = __ldg(p + b);
                const uint8_t *ps = c.scales[k] + at * (D / 32);
                next[k].sc = kBlk == 2 ? (uint32_t)__ldg(reinterpret_cast<const uint16_t *>(ps)) : __ldg(reinterpret_cast<const uint32_t *>(ps));
            }
        };
        // (two rounds before the first item: the code of every part stands once)
        for (int64_t item = warp - 10 - 2 * kUnpackers; item < items; item += kUnpackers) {
            const bool begun = item >= 0;
            const uint32_t gb = (uint32_t)(item >> 1);
            const int s = (int)(gb % kS), r = (int)(item & 1) * 32 + lane;
            if (begun && !__all_sync(0xffffffffu, mbar_wait(smem_u32(kv_empty + s), ((gb / kS) & 1u) ^ 1u, abort_flag))) break;
#pragma unroll
            for (int k = 0; k < C::kKinds; ++k) {
                if (begun) {
                    if (k == 0) {
                        // bounds of the rows
                        float sum = 0.f;
                        uint32_t top = 0u, low = ~0u;   // largest scale byte of the values, least that is not 0, less 1
#pragma unroll
                        for (int b = 0; b < kBlk; ++b) {
                            const float f = mx_scale((next[0].sc >> (8 * b)) & 255u);
                            const uint32_t vb = (next[C::kKinds - 1].sc >> (8 * b)) & 255u;
                            sum = fmaf(f, f, sum), top = max(top, vb), low = min(low, vb - 1u);
                        }
                        // (as integers: NaN stays the largest)
                        const uint32_t st = __reduce_max_sync(0xffffffffu, __float_as_uint(sum));
                        const bool fit = __all_sync(0xffffffffu, top <= kFreeTop && low >= kFreeLow - 1u);
                        if (lane == 0) k_bound[s * 2 + (item & 1)] = make_float2(__uint_as_float(st), fit ? 0.f : 1.f);
                    }
                    // A block of 32 at a time, its codes moved to the front: a loop of a quarter of the instructions, since the warps of a multiprocessor's quarter run different
                    // code and wait for it (16 x 10^4 x 10^4, d = 128: 784 us against 916; with values of their own, 148 x 256 x 8192: 181 us against 213)
                    unsigned char *tile = smKV + s * C::kStageBytes + k * C::kTileBytes + r * 128;
#pragma unroll 1
                    for (int b = 0; b < kBlk; ++b) {
                        const UnpackScale us(next[k].sc & 255u);
                        unsigned char *chunk = tile + (b >> 1) * C::kChunkBytes;
                        const uint32_t w[4] = {next[k].w[0].x, next[k].w[0].y, next[k].w[0].z, next[k].w[0].w};
#pragma unroll
                        for (int i4 = 0; i4 < 4; ++i4) *reinterpret_cast<uint4 *>(chunk + ((((b & 1) * 4 + i4) ^ (r & 7)) << 4)) = unpack8(w[i4], us);
#pragma unroll
                        for (int i = 1; i < kBlk; ++i) next[k].w[i - 1] = next[k].w[i];
                        next[k].sc >>= 8;
                    }
                }
                if (k == C::kKinds - 1) fetch();   // the codes have been used: the next item's may come
                if (begun) {
                    fence_proxy_async();
                    mbar_arrive(smem_u32((k == 0 ? k_full : v_full) + s));
                }
            }
            place(item + 2 * kUnpackers);
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
    if (warp == 8) tmem_dealloc(tmem, 512);
}

template <int D, bool SHARED>
cudaError_t run_pair(const AttCall &a, int grid, cudaStream_t st)
{
    using C = PairCfg<D, SHARED>;
    cudaError_t e = allow_smem<k_att4_pair<D, SHARED>>(C::kSmem);
    if (e != cudaSuccess) return e;
    count_launch();
    return launch_pdl(k_att4_pair<D, SHARED>, dim3(grid), dim3(C::kThreads), C::kSmem, st, a);
}

}  // namespace

cudaError_t launch_att4_pair(const AttCall &a, int grid, cudaStream_t st)
{
    const bool shared = a.c.codes[0] == a.c.codes[1];
    if (a.c.d == 64) return shared ? run_pair<64, true>(a, grid, st) : run_pair<64, false>(a, grid, st);
    return shared ? run_pair<128, true>(a, grid, st) : run_pair<128, false>(a, grid, st);
}

}  // namespace aif
