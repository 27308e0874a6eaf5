// Attention of a tree of drafted tokens over the paged cache on the 5th-generation tensor cores (del_tree_attention, many query rows).
//
// One CTA = up to two tiles of 128 query rows (node x query head of the group) of one kv head of one sequence, and a contiguous part
// of its keys; a cluster of CTAs covers all keys and joins its parts through distributed shared memory: one launch, no workspace.
// Keys and values stream once through shared memory in blocks of 64 positions (four pages), whatever the number of rows: the key
// pages [16][hd] and the value pages [hd][16] are the K-major operand tiles tcgen05.mma wants, so TMA copies them as they lie (5-d maps
// of the cache, 128-byte swizzle for keys, 32-byte swizzle for values).  Per block and tile:
//   S = Q K^T      M 128, N 64, into one of two 64-column accumulators in tensor memory;
//   softmax        one thread per query row: tcgen05.ld of its 64 scores, p = 2^(s - m) against a lazily raised reference m (the output in
//                  tensor memory is rescaled only when the row maximum has grown by more than 2^8), p as bf16 into shared memory;
//   O += P V       M 128, N hd, K 16 per page.
// Roles: warp 0 issues the copies, warp 1 the MMAs (the scores of block j + 1 before the probabilities of block j are waited for),
// four warps per tile do the softmax; quarters of a tile without rows do nothing.  Every mbarrier wait is bounded and gives up as soon as
// another role has: the rows then become NaN and the caller's error word, if there is one, is set.
//
// What is masked never enters a sum: scores by selection; values of drafted or never written slots are looked at, and where one is not
// finite its token's column is zeroed in shared memory and added at the end to those rows that see it.
#include <cooperative_groups.h>
#include <cuda.h>

#include <cstring>

#include "tc_common.cuh"
#include "tree_attn.cuh"

namespace cg = cooperative_groups;

namespace {

using namespace tc;

constexpr int BQ = 128, BKEY = 64;
constexpr float RESCALE_STEP = 8.f;              // log2 units

template <int HD, int TILES>
struct Cfg {
    static constexpr int KB = HD / 64;                             // 64-dim k-blocks of a key or query row
    static constexpr int Q_PART = BQ * 128;                        // [128 rows][128 B]
    static constexpr int Q_BYTES = TILES * KB * Q_PART;
    static constexpr int P_BYTES = TILES * BQ * 128;               // [128 rows][64 keys] bf16 each
    static constexpr int K_BYTES = KB * BKEY * 128, V_BYTES = 4 * HD * 32, STAGE = K_BYTES + V_BYTES;
    static constexpr int STAGES = HD == 128 ? (TILES == 2 ? 4 : 5) : 8;
    static constexpr int O_BYTES = TILES * BQ * HD * 4;            // the parts' outputs, where the stages were
    static constexpr int SMEM = Q_BYTES + P_BYTES + STAGES * STAGE + 1024;
    static constexpr int THREADS = 64 + TILES * 128;
    static constexpr uint32_t O_COL = TILES * 2 * BKEY;            // S buffers first, then the outputs
    static constexpr uint32_t TMEM = O_COL + TILES * HD <= 256 ? 256 : 512;
    static_assert(O_BYTES <= STAGES * STAGE, "outputs do not fit where the stages were");
    static_assert(SMEM <= 232448 - 512, "too much shared memory");
};

struct Maps { CUtensorMap k, v; };

__device__ __forceinline__ bool wait_or_err(uint64_t *b, uint32_t parity, volatile int *err) {
    for (uint32_t i = 0; i < WAIT_LIMIT; ++i) {
        if (mbar_try(b, parity)) return true;
        if ((i & 255u) == 255u && *err) return false;
    }
    return false;
}
__device__ __forceinline__ void tma_load_5d(void *dst, const CUtensorMap *map, int c0, int c1, int c2, int c3, int c4, uint64_t *bar) {
    asm volatile("cp.async.bulk.tensor.5d.shared::cluster.global.mbarrier::complete_tx::bytes [%0], [%1, {%2, %3, %4, %5, %6}], [%7];"
                 ::"r"(smem_u32(dst)), "l"(map), "r"(c0), "r"(c1), "r"(c2), "r"(c3), "r"(c4), "r"(smem_u32(bar)) : "memory");
}
// K-major operand tile with 32-byte swizzle: rows of 32 bytes, 8-row groups 256 bytes apart
__device__ __forceinline__ uint64_t umma_desc_sw32(uint32_t smem_addr) {
    uint64_t lo = ((smem_addr & 0x3FFFFu) >> 4) | (1u << 16);
    uint64_t hi = (256u >> 4) | (1u << 14) | (6u << 29);
    return lo | (hi << 32);
}
__device__ __forceinline__ void tmem_st32(uint32_t taddr, const uint32_t (&r)[32]) {
    asm volatile("tcgen05.st.sync.aligned.32x32b.x32.b32 [%0], "
                 "{%1, %2, %3, %4, %5, %6, %7, %8, %9, %10, %11, %12, %13, %14, %15, %16, "
                 "%17, %18, %19, %20, %21, %22, %23, %24, %25, %26, %27, %28, %29, %30, %31, %32};"
                 ::"r"(taddr), "r"(r[0]), "r"(r[1]), "r"(r[2]), "r"(r[3]), "r"(r[4]), "r"(r[5]), "r"(r[6]), "r"(r[7]),
                   "r"(r[8]), "r"(r[9]), "r"(r[10]), "r"(r[11]), "r"(r[12]), "r"(r[13]), "r"(r[14]), "r"(r[15]),
                   "r"(r[16]), "r"(r[17]), "r"(r[18]), "r"(r[19]), "r"(r[20]), "r"(r[21]), "r"(r[22]), "r"(r[23]),
                   "r"(r[24]), "r"(r[25]), "r"(r[26]), "r"(r[27]), "r"(r[28]), "r"(r[29]), "r"(r[30]), "r"(r[31])
                 : "memory");
}
__device__ __forceinline__ float ex2f(float x) {
    float y;
    asm("ex2.approx.ftz.f32 %0, %1;" : "=f"(y) : "f"(x));
    return y;
}
__device__ __forceinline__ bool odd_pair(uint32_t x) {             // either bf16 of the word is an infinity or no number
    return (x & 0x7f800000u) == 0x7f800000u || (x & 0x7f80u) == 0x7f80u;
}

// which of the block's 64 positions a row sees: bit e = position key0 + e
__device__ __forceinline__ uint64_t visible(uint64_t bits, int key0, int len, int n_keys) {
    const int c = len - key0;                                       // committed positions of the block and beyond it
    uint64_t vm = c >= 64 ? ~0ull : c > 0 ? ((1ull << c) - 1) | (bits << c) : c > -64 ? bits >> -c : 0;
    const int left = n_keys - key0;
    if (left < 64) vm &= left > 0 ? (1ull << left) - 1 : 0;
    return vm;
}

template <int HD, int TILES>
__global__ void __launch_bounds__(Cfg<HD, TILES>::THREADS, 1) tree_attention_tc_kernel(const __grid_constant__ Maps maps, const __grid_constant__ TreeArgs a) {
    using C = Cfg<HD, TILES>;
    extern __shared__ unsigned char smem_dyn[];
    __shared__ __align__(8) uint64_t q_full, kv_full[C::STAGES], kv_empty[C::STAGES], s_full[TILES][2], s_empty[TILES][2], p_full[TILES], o_done[TILES], tile_bar, all_bar;
    __shared__ uint32_t tmem_base_s;
    __shared__ volatile int s_err;
    __shared__ int s_bad_page, s_odd[2];
    __shared__ unsigned long long s_odd_tokens;                     // drafted tokens whose values were zeroed
    unsigned char *base = reinterpret_cast<unsigned char *>((reinterpret_cast<uintptr_t>(smem_dyn) + 1023) & ~(uintptr_t)1023);
    unsigned char *q_sm = base, *p_sm = base + C::Q_BYTES, *kv_sm = p_sm + C::P_BYTES;

    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
    const int n_splits = gridDim.x, split = blockIdx.x, b = blockIdx.z;
    const int group = a.nh / a.kv.nkv;
    const int n_rt = (a.max_nodes * group + TILES * BQ - 1) / (TILES * BQ);
    const int kvh = blockIdx.y / n_rt, row0 = (blockIdx.y - kvh * n_rt) * TILES * BQ;
    const tree::Seq s = tree::load_seq(a, b);
    const int R = s.n * group;
    if (row0 >= R) return;                                          // (the whole cluster)

    // this CTA's blocks of 64 positions
    const int nb = (s.n_keys + BKEY - 1) / BKEY, per = (nb + n_splits - 1) / n_splits;
    const int kb0 = min(split * per, nb), n_kb = min(per, nb - kb0);
    const int n_pages = (s.n_keys + 15) >> 4;

    auto quarters = [&](int t) { return min(4, max(0, (R - row0 - t * BQ + 31) >> 5)); };      // of tile t, that have rows
    const int n_tiles = TILES == 2 && quarters(1) > 0 ? 2 : 1;
    const int n_warps = quarters(0) + (TILES == 2 ? quarters(TILES - 1) : 0);                  // softmax warps at work
    auto part_ml = [&](unsigned char *p, int x) { return reinterpret_cast<float2 *>(p + (x >> 7) * BQ * 128 + (x & 127) * 8); };   // where the probabilities were
    if (threadIdx.x == 0) {
        mbar_init(&q_full, n_warps);
        mbar_init(&all_bar, n_warps);
        mbar_init(&tile_bar, max(1, quarters(0)));
        for (int i = 0; i < C::STAGES; ++i) { mbar_init(&kv_full[i], 1); mbar_init(&kv_empty[i], 1); }
        for (int t = 0; t < TILES; ++t) {
            const int nq = max(1, quarters(t));
            for (int i = 0; i < 2; ++i) { mbar_init(&s_full[t][i], 1); mbar_init(&s_empty[t][i], nq); }
            mbar_init(&p_full[t], nq);
            mbar_init(&o_done[t], 1);
        }
        s_err = 0;
        s_bad_page = s_odd[0] = s_odd[1] = 0;
        s_odd_tokens = 0;
        asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
    }
    if (warp == 1) {
        asm volatile("tcgen05.alloc.cta_group::1.sync.aligned.shared::cta.b32 [%0], %1;" ::"r"(smem_u32(&tmem_base_s)), "r"(C::TMEM) : "memory");
        asm volatile("tcgen05.relinquish_alloc_permit.cta_group::1.sync.aligned;" ::: "memory");
    }
    asm volatile("tcgen05.fence::before_thread_sync;" ::: "memory");
    __syncthreads();
    asm volatile("tcgen05.fence::after_thread_sync;" ::: "memory");
    const uint32_t tmem_base = tmem_base_s;

    if (warp == 0) {
        // Page ids: lane i holds page i of the current eight blocks, the next eight are requested one round ahead.  A position
        // behind the last, or an id that names no page, is copied from coordinate -1: zeros.
        auto page_of = [&](int pi) {
            const int pg = pi < n_pages ? s.pt[pi] : -1;
            return a.kv.holds(pg) ? pg : -1;
        };
        int cur = page_of(4 * kb0 + lane), nxt = page_of(4 * kb0 + 32 + lane);
        int j = 0;
        for (; j < n_kb; ++j) {
            const int st = j % C::STAGES, first = (4 * j) & 31;
            if (first == 0 && j > 0) { cur = nxt; nxt = page_of(4 * (kb0 + j) + 32 + lane); }
            int pages[4];
#pragma unroll
            for (int pg = 0; pg < 4; ++pg) pages[pg] = __shfl_sync(0xffffffffu, cur, first + pg);
            bool ok = true;
            if (lane == 0) {
                if (j >= C::STAGES && !wait_or_err(&kv_empty[st], ((j / C::STAGES) & 1) ^ 1, &s_err)) {
                    if (!s_err) s_err = 1;
                    ok = false;
                } else {
                    mbar_expect_tx(&kv_full[st], C::STAGE);
                    unsigned char *kst = kv_sm + (size_t)st * C::STAGE, *vst = kst + C::K_BYTES;
#pragma unroll
                    for (int pg = 0; pg < 4; ++pg) {
#pragma unroll
                        for (int kb = 0; kb < C::KB; ++kb)
                            tma_load_5d(kst + kb * BKEY * 128 + pg * 2048, &maps.k, kb * 64, 0, kvh, a.layer - 1, pages[pg], &kv_full[st]);
                        tma_load_5d(vst + pg * HD * 32, &maps.v, 0, 0, kvh, a.layer - 1, pages[pg], &kv_full[st]);
                    }
                }
            }
            if (!__shfl_sync(0xffffffffu, (int)ok, 0)) break;
        }
        if (s_err && lane == 0) drain(kv_full, C::STAGES, j % C::STAGES, (uint32_t)(j / C::STAGES) & 1);
    } else if (warp == 1) {
        if (lane == 0 && n_kb > 0) {
            // instruction descriptors: fp32 accumulate, bf16 x bf16, both operands K-major, M = 128, N = 64 / HD
            const uint32_t idesc_s = (1u << 4) | (1u << 7) | (1u << 10) | ((uint32_t)(BKEY >> 3) << 17) | ((uint32_t)(BQ >> 4) << 24);
            const uint32_t idesc_o = (1u << 4) | (1u << 7) | (1u << 10) | ((uint32_t)(HD >> 3) << 17) | ((uint32_t)(BQ >> 4) << 24);
            const uint32_t q_addr = smem_u32(q_sm), p_addr = smem_u32(p_sm);
            int n_s[TILES] = {}, n_o = 0;            // blocks whose scores of tile t, whose products with the values have been issued
            bool ok = wait_or_err(&q_full, 0, &s_err);
            if (!ok && !s_err) s_err = 2;
            auto issue_scores = [&](int j) -> bool {
                const int st = j % C::STAGES, buf = j & 1;
                if (!wait_or_err(&kv_full[st], (j / C::STAGES) & 1, &s_err)) { if (!s_err) s_err = 3; return false; }
                const uint32_t k_addr = smem_u32(kv_sm + (size_t)st * C::STAGE);
#pragma unroll
                for (int t = 0; t < TILES; ++t) {
                    if (t >= n_tiles) break;
                    if (j >= 2 && !wait_or_err(&s_empty[t][buf], ((j >> 1) & 1) ^ 1, &s_err)) { if (!s_err) s_err = 4; return false; }
                    asm volatile("tcgen05.fence::after_thread_sync;" ::: "memory");
                    const uint32_t d_tmem = tmem_base + (uint32_t)((t * 2 + buf) * BKEY);
#pragma unroll
                    for (int kb = 0; kb < C::KB; ++kb) {
                        const uint64_t da = umma_desc(q_addr + (t * C::KB + kb) * C::Q_PART), db = umma_desc(k_addr + kb * BKEY * 128);
#pragma unroll
                        for (int k = 0; k < 4; ++k) umma_bf16(d_tmem, da + 2 * k, db + 2 * k, idesc_s, (kb | k) != 0);
                    }
                    umma_commit(&s_full[t][buf]);
                    n_s[t] = j + 1;
                }
                return true;
            };
            if (ok) ok = issue_scores(0);
            for (int j = 0; ok && j < n_kb; ++j) {
                if (j + 1 < n_kb) ok = issue_scores(j + 1);
                if (!ok) break;
                const uint32_t v_addr = smem_u32(kv_sm + (size_t)(j % C::STAGES) * C::STAGE + C::K_BYTES);
#pragma unroll
                for (int t = 0; t < TILES; ++t) {
                    if (t >= n_tiles) break;
                    if (!wait_or_err(&p_full[t], j & 1, &s_err)) { if (!s_err) s_err = 5; ok = false; break; }
                    asm volatile("tcgen05.fence::after_thread_sync;" ::: "memory");
                    const uint64_t da = umma_desc(p_addr + t * BQ * 128);
#pragma unroll
                    for (int kk = 0; kk < 4; ++kk)
                        umma_bf16(tmem_base + C::O_COL + (uint32_t)(t * HD), da + 2 * kk, umma_desc_sw32(v_addr + kk * HD * 32), idesc_o, (j | kk) != 0);
                    umma_commit(&o_done[t]);         // the output holds blocks 0..j; the probabilities may be overwritten
                }
                if (!ok) break;
                umma_commit(&kv_empty[j % C::STAGES]);
                n_o = j + 1;
            }
            if (s_err) {
                for (int t = 0; t < TILES; ++t) drain(s_full[t], 2, n_s[t] & 1, (uint32_t)(n_s[t] >> 1) & 1);
                drain(kv_empty, C::STAGES, n_o % C::STAGES, (uint32_t)(n_o / C::STAGES) & 1);
                for (int t = 0; t < TILES; ++t) drain(&o_done[t], 1, 0, (uint32_t)n_o & 1);
            }
        }
    } else {
        const int t = (warp - 2) >> 2, q = warp & 3;             // tile, TMEM lane quarter this warp may access
        const int trow = q * 32 + lane, rr = row0 + t * BQ + trow, nq = quarters(t);
        const bool row_ok = rr < R;
        if (q < nq) {
            // queries: row of 128-byte k-blocks with the 128-byte swizzle; rows behind the last are zero
            const int i = row_ok ? rr / group : 0, hq = row_ok ? rr - i * group : 0;
            const uint64_t bits = row_ok ? tree::node_bits(a, b, i) : 0;
            const bf16 *qp = a.q + b * a.q_seq + i * a.q_node + (size_t)(kvh * group + hq) * HD;
            unsigned char *qrow = q_sm + t * C::KB * C::Q_PART + trow * 128;
#pragma unroll
            for (int c = 0; c < HD / 8; ++c) {
                const uint4 v = row_ok ? *reinterpret_cast<const uint4 *>(qp + 8 * c) : make_uint4(0, 0, 0, 0);
                *reinterpret_cast<uint4 *>(qrow + (c >> 3) * C::Q_PART + (((c & 7) ^ (trow & 7)) << 4)) = v;
            }
            asm volatile("fence.proxy.async.shared::cta;" ::: "memory");
            __syncwarp();
            if (lane == 0) mbar_arrive(&q_full);
            // does the table name pages that are none?  (then every block's ids are looked at again)
            bool bad = false;
            for (int p = 4 * kb0 + trow; p < min(n_pages, 4 * (kb0 + n_kb)); p += nq * 32) bad |= !a.kv.holds(s.pt[p]);
            if (__any_sync(0xffffffffu, bad) && lane == 0) s_bad_page = 1;
            // barriers among softmax warps, bounded like every wait
            auto meet = [&](uint64_t *bar, uint32_t parity) -> bool {
                __syncwarp();
                if (lane == 0) mbar_arrive(bar);
                return wait_or_err(bar, parity, &s_err);
            };
            uint32_t tile_phase = 0;
            bool ok = meet(&all_bar, 0);
            if (!ok && !s_err) s_err = 10;
            const bool bad_pages = s_bad_page != 0;

            const uint32_t lane_addr = tmem_base + ((uint32_t)(q * 32) << 16);
            const uint32_t o_addr = lane_addr + C::O_COL + (uint32_t)(t * HD);
            unsigned char *prow = p_sm + t * BQ * 128 + trow * 128;
            float m_ref = -INFINITY, l = 0.f;
            for (int j = 0; ok && j < n_kb; ++j) {
                const int buf = j & 1, key0 = (kb0 + j) * BKEY;
                if (!wait_or_err(&s_full[t][buf], (j >> 1) & 1, &s_err)) { if (!s_err) s_err = 6; ok = false; break; }
                asm volatile("tcgen05.fence::after_thread_sync;" ::: "memory");
                uint32_t r0[32], r1[32];
                tmem_ld32(lane_addr + (uint32_t)((t * 2 + buf) * BKEY), r0);
                tmem_ld32(lane_addr + (uint32_t)((t * 2 + buf) * BKEY + 32), r1);
                asm volatile("tcgen05.wait::ld.sync.aligned;" ::: "memory");
                asm volatile("tcgen05.fence::before_thread_sync;" ::: "memory");
                __syncwarp();
                if (lane == 0) mbar_arrive(&s_empty[t][buf]);
                float sv[64], mx = -INFINITY;
#pragma unroll
                for (int e = 0; e < 32; ++e) {
                    sv[e] = __uint_as_float(r0[e]) * a.scale;
                    sv[32 + e] = __uint_as_float(r1[e]) * a.scale;
                }
                const bool tail = key0 + BKEY > s.len;
                if (tail || bad_pages) {
                    uint64_t vm = visible(bits, key0, s.len, s.n_keys);
                    if (bad_pages)
                        for (int pg = 0; pg < 4; ++pg) {
                            const int pi = (key0 >> 4) + pg;
                            if (pi >= n_pages || !a.kv.holds(s.pt[pi])) vm &= ~(0xffffull << (16 * pg));
                        }
                    const uint32_t v0 = (uint32_t)vm, v1 = (uint32_t)(vm >> 32);
#pragma unroll
                    for (int e = 0; e < 32; ++e) {
                        if (!((v0 >> e) & 1)) sv[e] = -INFINITY;
                        if (!((v1 >> e) & 1)) sv[32 + e] = -INFINITY;
                    }
                }
#pragma unroll
                for (int e = 0; e < 64; ++e) mx = fmaxf(mx, sv[e]);
                // reference maximum: raised only when the row maximum has outgrown it by RESCALE_STEP
                float alpha = 1.f;
                if (m_ref == -INFINITY) {
                    m_ref = mx;                                   // (nothing but zeros has been added so far)
                } else if (mx > m_ref + RESCALE_STEP) {
                    alpha = ex2f(m_ref - mx);
                    m_ref = mx;
                    l *= alpha;
                }
                const float m_use = m_ref == -INFINITY ? 0.f : m_ref;
                float psum = 0.f;
#pragma unroll
                for (int e = 0; e < 64; ++e) { sv[e] = ex2f(sv[e] - m_use); psum += sv[e]; }
                l += psum;
                // the previous block's P*V has read the probabilities and updated the output
                if (j > 0 && !wait_or_err(&o_done[t], (j - 1) & 1, &s_err)) { if (!s_err) s_err = 7; ok = false; break; }
                if (__any_sync(0xffffffffu, alpha != 1.f)) {
                    asm volatile("tcgen05.fence::after_thread_sync;" ::: "memory");
                    for (int c0 = 0; c0 < HD; c0 += 32) {
                        uint32_t o[32];
                        tmem_ld32(o_addr + (uint32_t)c0, o);
                        asm volatile("tcgen05.wait::ld.sync.aligned;" ::: "memory");
#pragma unroll
                        for (int e = 0; e < 32; ++e) o[e] = __float_as_uint(__uint_as_float(o[e]) * alpha);
                        tmem_st32(o_addr + (uint32_t)c0, o);
                    }
                    asm volatile("tcgen05.wait::st.sync.aligned;" ::: "memory");
                }
#pragma unroll
                for (int c = 0; c < 8; ++c) {
                    uint4 v;
                    v.x = pack_bf16(sv[8 * c + 0], sv[8 * c + 1]);
                    v.y = pack_bf16(sv[8 * c + 2], sv[8 * c + 3]);
                    v.z = pack_bf16(sv[8 * c + 4], sv[8 * c + 5]);
                    v.w = pack_bf16(sv[8 * c + 6], sv[8 * c + 7]);
                    *reinterpret_cast<uint4 *>(prow + ((c ^ (trow & 7)) << 4)) = v;
                }
                if (tail && t == 0) {
                    // Values of drafted and of never written slots must not meet a probability of zero as infinity or NaN.  The
                    // first tile's warps look; what they find they zero, by whole tokens, and remember the drafted ones.
                    unsigned char *vst = kv_sm + (size_t)(j % C::STAGES) * C::STAGE + C::K_BYTES;
                    if (!wait_or_err(&kv_full[j % C::STAGES], (j / C::STAGES) & 1, &s_err)) { if (!s_err) s_err = 8; ok = false; break; }
                    bool odd = false;
                    for (int u = trow; u < 4 * HD * 2; u += nq * 32) {
                        const uint4 v = *reinterpret_cast<const uint4 *>(vst + u * 16);
                        odd |= odd_pair(v.x) | odd_pair(v.y) | odd_pair(v.z) | odd_pair(v.w);
                    }
                    if (__any_sync(0xffffffffu, odd) && lane == 0) s_odd[j & 1] = 1;      // (never cleared: two blocks later it only costs time)
                    if (!meet(&tile_bar, tile_phase)) { if (!s_err) s_err = 11; ok = false; break; }
                    tile_phase ^= 1;
                    for (int e = q; s_odd[j & 1] && e < BKEY; e += nq) {
                        if (key0 + e < s.len) continue;           // committed: every row sees it
                        const int tk = e & 15;
                        unsigned char *col = vst + (e >> 4) * HD * 32 + (tk & 7) * 2;
                        bool mine = false;
                        for (int d = lane; d < HD; d += 32)
                            mine |= (*reinterpret_cast<const uint16_t *>(col + d * 32 + (((tk >> 3) ^ ((d >> 2) & 1)) << 4)) & 0x7f80u) == 0x7f80u;
                        if (!__any_sync(0xffffffffu, mine)) continue;
                        for (int d = lane; d < HD; d += 32) *reinterpret_cast<uint16_t *>(col + d * 32 + (((tk >> 3) ^ ((d >> 2) & 1)) << 4)) = 0;
                        if (lane == 0 && key0 + e < s.n_keys) atomicOr(&s_odd_tokens, 1ull << (key0 + e - s.len));
                    }
                }
                asm volatile("fence.proxy.async.shared::cta;" ::: "memory");      // visible to the tensor core's reads
                asm volatile("tcgen05.fence::before_thread_sync;" ::: "memory");
                __syncwarp();
                if (lane == 0) mbar_arrive(&p_full[t]);
            }
            if (ok && n_kb > 0 && !wait_or_err(&o_done[t], (n_kb - 1) & 1, &s_err)) { if (!s_err) s_err = 9; ok = false; }
            if (!meet(&all_bar, 1)) { if (!s_err) s_err = 12; ok = false; }       // both tiles are done with the stages, s_odd_tokens is complete
            asm volatile("tcgen05.fence::after_thread_sync;" ::: "memory");
            const uint64_t odd_seen = s_odd_tokens & bits;
            const float m_use = m_ref == -INFINITY ? 0.f : m_ref;
            const size_t head = ((size_t)(a.layer - 1) * a.kv.nkv + kvh) * a.kv.head_elems();
            const float inv = l == 0.f ? 0.f : 1.f / l;            // (l = 0: nothing is visible, the result is zero)
            const size_t out = b * a.o_seq + i * a.o_node + (size_t)(kvh * group + hq) * HD;
            if (n_splits > 1) *part_ml(p_sm, t * BQ + trow) = make_float2(m_ref, l);
            float *po = reinterpret_cast<float *>(kv_sm) + (size_t)(t * BQ + trow) * HD;
            for (int c0 = 0; c0 < HD && n_kb > 0; c0 += 32) {
                uint32_t o[32];
                if (ok) tmem_ld32(o_addr + (uint32_t)c0, o);
                asm volatile("tcgen05.wait::ld.sync.aligned;" ::: "memory");
                for (uint64_t left = odd_seen; left; left &= left - 1) {
                    // a drafted token that this row sees and whose values are not finite: added here, in fp32
                    const int pos = s.len + __ffsll((long long)left) - 1;
                    const size_t at = (size_t)s.pt[pos >> 4] * a.kv.page_elems() + head;
                    float dot = 0.f;
                    for (int d = 0; d < HD; ++d) dot += bf16_to_f(qp[d]) * bf16_to_f(a.kv.k[at + (pos & 15) * HD + d]);
                    const float w = ex2f(dot * a.scale - m_use);
#pragma unroll
                    for (int e = 0; e < 32; ++e) o[e] = __float_as_uint(__uint_as_float(o[e]) + w * bf16_to_f(a.kv.v[at + (c0 + e) * 16 + (pos & 15)]));
                }
                if (n_splits > 1) {
#pragma unroll
                    for (int e = 0; e < 32; e += 4)                 // 16-byte pieces, spread over the banks by the row
                        *reinterpret_cast<uint4 *>(po + ((((c0 + e) >> 2) ^ (trow & 15)) << 2)) = make_uint4(o[e], o[e + 1], o[e + 2], o[e + 3]);
                } else if (row_ok && ok) {
#pragma unroll
                    for (int e = 0; e < 32; e += 8) {
                        uint4 hi, lo;
                        split_bf16x2(__uint_as_float(o[e + 0]) * inv, __uint_as_float(o[e + 1]) * inv, hi.x, lo.x);
                        split_bf16x2(__uint_as_float(o[e + 2]) * inv, __uint_as_float(o[e + 3]) * inv, hi.y, lo.y);
                        split_bf16x2(__uint_as_float(o[e + 4]) * inv, __uint_as_float(o[e + 5]) * inv, hi.z, lo.z);
                        split_bf16x2(__uint_as_float(o[e + 6]) * inv, __uint_as_float(o[e + 7]) * inv, hi.w, lo.w);
                        *reinterpret_cast<uint4 *>(a.out + out + c0 + e) = hi;
                        if (a.out_lo) *reinterpret_cast<uint4 *>(a.out_lo + out + c0 + e) = lo;
                    }
                }
            }
            if (n_splits == 1 && n_kb == 0 && row_ok) {             // a table of no page at all
                for (int e = 0; e < HD; e += 8) {
                    *reinterpret_cast<uint4 *>(a.out + out + e) = make_uint4(0, 0, 0, 0);
                    if (a.out_lo) *reinterpret_cast<uint4 *>(a.out_lo + out + e) = make_uint4(0, 0, 0, 0);
                }
            }
            asm volatile("tcgen05.fence::before_thread_sync;" ::: "memory");
        }
    }
    __syncthreads();
    if (warp == 1) {
        asm volatile("tcgen05.fence::after_thread_sync;" ::: "memory");
        asm volatile("tcgen05.dealloc.cta_group::1.sync.aligned.b32 %0, %1;" ::"r"(tmem_base), "r"(C::TMEM) : "memory");
    }
    if (threadIdx.x == 0 && s_err && a.err) atomicMax(a.err, (int)s_err);
    const int rows = min(R - row0, TILES * BQ);
    if (n_splits > 1) {
        cg::cluster_group cl = cg::this_cluster();
        cl.sync();
        // the parts' states of one row each: a warp takes a row of the cluster's rows, every lane four columns
        bool failed = false;
        for (int k = 0; k < n_splits; ++k) failed |= *cl.map_shared_rank(const_cast<int *>(&s_err), k) != 0;
        constexpr int LPR = HD / 4;                                 // lanes per row
        for (int x = (split * C::THREADS + threadIdx.x) / LPR; x < rows; x += n_splits * C::THREADS / LPR) {
            const int c = threadIdx.x % LPR;
            float M = -INFINITY;
            for (int k = 0; k < n_splits; ++k) M = fmaxf(M, part_ml(cl.map_shared_rank(p_sm, k), x)->x);
            const float mu = M == -INFINITY ? 0.f : M;
            float L = 0.f;
            float4 o = make_float4(0.f, 0.f, 0.f, 0.f);
            for (int k = 0; k < n_splits; ++k) {
                const float2 ml = *part_ml(cl.map_shared_rank(p_sm, k), x);
                if (k * per >= nb) break;                           // (this part and the later ones have no block)
                const float w = ex2f(ml.x - mu);
                const float4 v = *reinterpret_cast<const float4 *>(cl.map_shared_rank(reinterpret_cast<float *>(kv_sm), k) + (size_t)x * HD + ((c ^ (x & 15)) << 2));
                L += ml.y * w;
                o.x += v.x * w; o.y += v.y * w; o.z += v.z * w; o.w += v.w * w;
            }
            const float inv = failed ? NAN : L == 0.f ? 0.f : 1.f / L;
            const int rr = row0 + x, i = rr / group, hq = rr - i * group;
            const size_t at = b * a.o_seq + i * a.o_node + (size_t)(kvh * group + hq) * HD + 4 * c;
            uint2 hi, lo;
            split_bf16x2(o.x * inv, o.y * inv, hi.x, lo.x);
            split_bf16x2(o.z * inv, o.w * inv, hi.y, lo.y);
            *reinterpret_cast<uint2 *>(a.out + at) = hi;
            if (a.out_lo) *reinterpret_cast<uint2 *>(a.out_lo + at) = lo;
        }
        cl.sync();                                                  // nobody leaves while its shared memory is read
    } else if (s_err) {
        for (int e = threadIdx.x; e < rows * HD; e += C::THREADS) {
            const int rr = row0 + e / HD, i = rr / group, hq = rr - i * group;
            a.out[b * a.o_seq + i * a.o_node + (size_t)(kvh * group + hq) * HD + e % HD] = __float2bfloat16_rn(NAN);
        }
    }
}

typedef CUresult (*EncodeTiledFn)(CUtensorMap *, CUtensorMapDataType, cuuint32_t, void *, const cuuint64_t *, const cuuint64_t *,
                                  const cuuint32_t *, const cuuint32_t *, CUtensorMapInterleave, CUtensorMapSwizzle,
                                  CUtensorMapL2promotion, CUtensorMapFloatOOBfill);
EncodeTiledFn encode_fn() {
    static EncodeTiledFn fn = [] {
        void *q = nullptr;
        cudaDriverEntryPointQueryResult qr;
        return cudaGetDriverEntryPoint("cuTensorMapEncodeTiled", &q, cudaEnableDefault, &qr) == cudaSuccess && qr == cudaDriverEntryPointSuccess
                   ? reinterpret_cast<EncodeTiledFn>(q) : nullptr;
    }();
    return fn;
}

// 5-d maps of the cache: keys in boxes of 16 tokens x 64 dims (128-byte swizzle), values in boxes of hd dims x 16 tokens (32-byte swizzle)
bool make_maps(const PageView &kv, Maps *m) {
    EncodeTiledFn fn = encode_fn();
    if (!fn) return false;
    const cuuint64_t hd = kv.hd, nkv = kv.nkv, L = kv.L, head = 16 * hd * 2;
    const cuuint64_t strides_k[4] = {hd * 2, head, head * nkv, head * nkv * L}, strides_v[4] = {32, head, head * nkv, head * nkv * L};
    const cuuint64_t dims_k[5] = {hd, 16, nkv, L, (cuuint64_t)kv.n_pages}, dims_v[5] = {16, hd, nkv, L, (cuuint64_t)kv.n_pages};
    const cuuint32_t box_k[5] = {64, 16, 1, 1, 1}, box_v[5] = {16, (cuuint32_t)hd, 1, 1, 1}, one[5] = {1, 1, 1, 1, 1};
    return fn(&m->k, CU_TENSOR_MAP_DATA_TYPE_BFLOAT16, 5, kv.k, dims_k, strides_k, box_k, one, CU_TENSOR_MAP_INTERLEAVE_NONE,
              CU_TENSOR_MAP_SWIZZLE_128B, CU_TENSOR_MAP_L2_PROMOTION_L2_256B, CU_TENSOR_MAP_FLOAT_OOB_FILL_NONE) == CUDA_SUCCESS &&
           fn(&m->v, CU_TENSOR_MAP_DATA_TYPE_BFLOAT16, 5, kv.v, dims_v, strides_v, box_v, one, CU_TENSOR_MAP_INTERLEAVE_NONE,
              CU_TENSOR_MAP_SWIZZLE_32B, CU_TENSOR_MAP_L2_PROMOTION_L2_256B, CU_TENSOR_MAP_FLOAT_OOB_FILL_NONE) == CUDA_SUCCESS;
}

template <int HD, int TILES>
cudaError_t launch(const Maps &m, const TreeArgs &a, int batch, int max_len, int n_sms, cudaStream_t st) {
    auto kern = tree_attention_tc_kernel<HD, TILES>;
    static SmemAttrOnce attr;
    cudaError_t e = attr.set(kern, Cfg<HD, TILES>::SMEM);
    if (e != cudaSuccess) return e;
    const int group = a.nh / a.kv.nkv, n_rt = (a.max_nodes * group + TILES * BQ - 1) / (TILES * BQ);
    // one CTA per SM: as many parts of the keys as one wave holds, of at least two blocks each
    const int64_t units = (int64_t)a.kv.nkv * n_rt * batch;
    const int blocks = (max_len + a.max_nodes + BKEY - 1) / BKEY;
    int splits = (int)(n_sms / units < 8 ? n_sms / units : 8);
    if (splits > blocks / 2) splits = blocks / 2;
    if (splits < 1) splits = 1;
    return launch_cluster(kern, dim3(splits, a.kv.nkv * n_rt, batch), Cfg<HD, TILES>::THREADS, Cfg<HD, TILES>::SMEM, splits, st, m, a);
}

}  // namespace

cudaError_t launch_tree_attention_tc(const TreeArgs &a, int batch, int max_len, int n_sms, cudaStream_t st) {
    Maps m;
    if (!make_maps(a.kv, &m)) return cudaErrorInvalidValue;
    const bool one = a.max_nodes * (a.nh / a.kv.nkv) <= BQ;
    if (a.kv.hd == 128) return one ? launch<128, 1>(m, a, batch, max_len, n_sms, st) : launch<128, 2>(m, a, batch, max_len, n_sms, st);
    return one ? launch<64, 1>(m, a, batch, max_len, n_sms, st) : launch<64, 2>(m, a, batch, max_len, n_sms, st);
}
