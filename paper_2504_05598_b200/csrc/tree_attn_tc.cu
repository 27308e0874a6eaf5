// Attention of a tree of drafted tokens over the paged cache on the 5th-generation tensor cores (del_tree_attention, many query rows).
//
// One CTA = up to two tiles of 128 query rows (node x query head of the group) of one kv head of one sequence, and a contiguous part
// of its keys; a cluster of CTAs covers all keys and joins its parts through distributed shared memory: one launch, no workspace.
// Keys and values stream once through shared memory in blocks of 128 positions (eight pages), whatever the number of rows: the key
// pages [16][hd] and the value pages [hd][16] are the K-major operand tiles tcgen05.mma wants, so TMA copies them as they lie (5-d maps
// of the cache, 128-byte swizzle for keys, 32-byte swizzle for values).  Per block and tile:
//   S = Q K^T      M 128, N 128, into tensor memory;
//   softmax        two threads per query row, in two warps, 64 scores each: two sweeps of tcgen05.ld, first their maximum, exchanged through
//                  shared memory; then p = 2^(s - m) against a lazily raised reference m (the output in tensor memory is rescaled
//                  only when the row maximum has grown by more than 2^8), written as bf16 over the scores;
//   O += P V       M 128, N hd, K 16 per page, P read from tensor memory.
// Shared memory's 128 bytes per clock are what the MMAs compete for: with N = 64 and P in shared memory, scores and products of a
// block of 64 keys read 80 KB per tile (640 cycles, 256 of arithmetic); with N = 128 and P in tensor memory 48 KB.
// Roles: warp 0 issues the copies, warp 1 the MMAs, eight warps per tile do the softmax; quarters of a tile without rows do nothing.
// With two tiles each has one score buffer and one tile's softmax runs beside the other's MMAs; a single tile has two buffers.  (Two buffers of
// 128 keys for each of two tiles would take 2 x 2 x 128 + 2 x 128 = 768 columns of tensor memory at head dimension 128; of 64 keys 512, all there are.)
// Registers: the 18 warps of two tiles count as 20, which leaves 96 a thread, and the softmax spills (68 bytes stored, 92 loaded at head
// dimension 128, 228 and 248 at 64); with one tile 144 and 167 a thread, no spills.
// What bounds it (8B shape): 8 x 64 nodes over 32.7k positions 302 to 314 us, 3250 GB/s and 840 TFLOP/s, half of either rate: a tile's
// softmax waits for its scores and its products for the softmax, and the two tiles' chains (2.3 us per block) overlap in part.
// One sweep by the reference maximum so far, repeated where it did not hold, scores 16 at a time with the next on their way, was
// slower (349 us).  Called in a row the clock falls to the power limit (350 us).  With one tile a call takes 8.6 us for start, join
// and end, and 1.5 us per block, 64 KB at an SM's share of HBM (13B shape, 26 nodes, 3100 positions: 21.6 us).
// Every mbarrier wait is bounded and gives up as soon as another role has: the rows then become NaN and the caller's error word, if
// there is one, is set.
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

constexpr int BQ = 128, BKEY = 128, PAGES = BKEY / 16;
constexpr float RESCALE_STEP = 8.f;              // log2 units

template <int HD, int TILES>
struct Cfg {
    static constexpr int KB = HD / 64;                             // 64-dim k-blocks of a key or query row
    static constexpr int Q_PART = BQ * 128;                        // [128 rows][128 B]
    static constexpr int Q_BYTES = TILES * KB * Q_PART;
    static constexpr int K_BYTES = KB * BKEY * 128, V_BYTES = PAGES * HD * 32;
    static constexpr int KS = HD == 128 ? (TILES == 2 ? 2 : 3) : 5, VS = HD == 128 ? 2 : 5;      // blocks in the rings
    static constexpr int RING = KS * K_BYTES + VS * V_BYTES;
    static constexpr int O_BYTES = TILES * BQ * HD * 4;            // the parts' outputs, where the rings were
    static constexpr int SMEM = Q_BYTES + RING + 1024;
    static constexpr int THREADS = 64 + TILES * 256;
    static constexpr int BUFS = 2;                                 // score buffers: one per tile, or two of the only tile
    static constexpr uint32_t O_COL = BUFS * BKEY;                 // score buffers first, then the outputs
    static constexpr uint32_t TMEM = 512;
    static_assert(O_BYTES <= RING, "outputs do not fit where the rings were");
    static_assert(O_COL + TILES * HD <= TMEM, "too much tensor memory");
    static_assert(SMEM <= 232448 - 4096, "too much shared memory");        // (beside the barriers and block maxima)
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
__device__ __forceinline__ void tmem_st16(uint32_t taddr, const uint32_t (&r)[16]) {
    asm volatile("tcgen05.st.sync.aligned.32x32b.x16.b32 [%0], {%1, %2, %3, %4, %5, %6, %7, %8, %9, %10, %11, %12, %13, %14, %15, %16};"
                 ::"r"(taddr), "r"(r[0]), "r"(r[1]), "r"(r[2]), "r"(r[3]), "r"(r[4]), "r"(r[5]), "r"(r[6]), "r"(r[7]),
                   "r"(r[8]), "r"(r[9]), "r"(r[10]), "r"(r[11]), "r"(r[12]), "r"(r[13]), "r"(r[14]), "r"(r[15]) : "memory");
}
// the same product with A in tensor memory: lane = row, a 32-bit column holds two consecutive bf16 of k
__device__ __forceinline__ void umma_bf16_ts(uint32_t tmem_d, uint32_t tmem_a, uint64_t db, uint32_t idesc, uint32_t accumulate) {
    asm volatile("{\n\t.reg .pred p;\n\tsetp.ne.b32 p, %4, 0;\n\t"
                 "tcgen05.mma.cta_group::1.kind::f16 [%0], [%1], %2, %3, {%5, %5, %5, %5}, p;\n\t}"
                 ::"r"(tmem_d), "r"(tmem_a), "l"(db), "r"(idesc), "r"(accumulate), "r"(0u) : "memory");
}
__device__ __forceinline__ void tmem_ld_wait() { asm volatile("tcgen05.wait::ld.sync.aligned;" ::: "memory"); }
__device__ __forceinline__ float ex2f(float x) {
    float y;
    asm("ex2.approx.ftz.f32 %0, %1;" : "=f"(y) : "f"(x));
    return y;
}
// two lanes of fp32 arithmetic in one instruction
__device__ __forceinline__ void fma2(float &x0, float &x1, float b, float c) {          // x = x * b + c
    asm("{\n\t.reg .b64 x, y, z;\n\tmov.b64 x, {%0, %1};\n\tmov.b64 y, {%2, %2};\n\tmov.b64 z, {%3, %3};\n\t"
        "fma.rn.f32x2 x, x, y, z;\n\tmov.b64 {%0, %1}, x;\n\t}" : "+f"(x0), "+f"(x1) : "f"(b), "f"(c));
}
__device__ __forceinline__ void add2(float &x0, float &x1, float b0, float b1) {        // x += b
    asm("{\n\t.reg .b64 x, y;\n\tmov.b64 x, {%0, %1};\n\tmov.b64 y, {%2, %3};\n\tadd.rn.f32x2 x, x, y;\n\tmov.b64 {%0, %1}, x;\n\t}"
        : "+f"(x0), "+f"(x1) : "f"(b0), "f"(b1));
}
__device__ __forceinline__ bool odd_pair(uint32_t x) {             // either bf16 of the word is an infinity or no number
    return (x & 0x7f800000u) == 0x7f800000u || (x & 0x7f80u) == 0x7f80u;
}

// which of 64 positions from key0 on a row sees: bit e = position key0 + e
__device__ __forceinline__ uint64_t visible(uint64_t bits, int key0, int len, int n_keys) {
    const int c = len - key0;                                       // committed positions from key0 on
    uint64_t vm = c >= 64 ? ~0ull : c > 0 ? ((1ull << c) - 1) | (bits << c) : c > -64 ? bits >> -c : 0;
    const int left = n_keys - key0;
    if (left < 64) vm &= left > 0 ? (1ull << left) - 1 : 0;
    return vm;
}

template <int HD, int TILES>
__global__ void __launch_bounds__(Cfg<HD, TILES>::THREADS, 1) tree_attention_tc_kernel(const __grid_constant__ Maps maps, const __grid_constant__ TreeArgs a) {
    using C = Cfg<HD, TILES>;
    extern __shared__ unsigned char smem_dyn[];
    __shared__ __align__(8) uint64_t q_full, k_full[C::KS], k_empty[C::KS], v_full[C::VS], v_empty[C::VS], s_full[2], p_full[2], o_done[TILES], o_all[TILES], tile_bar, all_bar, pair_bar[TILES][4];
    __shared__ uint32_t tmem_base_s;
    __shared__ volatile int s_err;
    __shared__ int s_bad_page, s_odd[2];
    __shared__ float s_max[2][2][BQ], s_sum[TILES][BQ];             // [tile, or buffer of the only one][half][row] block maxima; the second halves' sums
    __shared__ unsigned long long s_odd_tokens;                     // drafted tokens whose values were zeroed
    unsigned char *base = reinterpret_cast<unsigned char *>((reinterpret_cast<uintptr_t>(smem_dyn) + 1023) & ~(uintptr_t)1023);
    unsigned char *q_sm = base, *k_sm = base + C::Q_BYTES, *v_sm = k_sm + C::KS * C::K_BYTES;

    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
    const int n_splits = gridDim.x, split = blockIdx.x, b = blockIdx.z;
    const int group = a.nh / a.kv.nkv;
    if (threadIdx.x == 0) {
        asm volatile("prefetch.tensormap [%0];" ::"l"(&maps.k) : "memory");
        asm volatile("prefetch.tensormap [%0];" ::"l"(&maps.v) : "memory");
    }
    pdl_wait();                                                     // (before tensor memory is taken: the kernel before this one may still want some)
    const int n_rt = (a.max_nodes * group + TILES * BQ - 1) / (TILES * BQ);
    const int kvh = blockIdx.y / n_rt, row0 = (blockIdx.y - kvh * n_rt) * TILES * BQ;
    const float inv_group = 1.f / (float)group;
    auto node_of = [&](int rr) { return (int)(((float)rr + 0.5f) * inv_group); };              // rr / group: rr < 2^16, off by less than 1/2 / group
    auto q_row = [&](int rr) {                                      // query row rr (node x head of the group), which exists whatever nodes[b] is
        const int i = node_of(rr);
        return a.q + b * a.q_seq + i * a.q_node + (size_t)(kvh * group + rr - i * group) * HD;
    };
    // The queries are the first thing requested, before it is known how many nodes there are: 16-byte pieces, a thread every 256th
    // of its tile.  (Each thread its own row, after the lengths: the first scores came 2.6 us into the kernel, now 1.4.)
    constexpr int PPR = HD / 8, QP = BQ * PPR / 256;                // pieces per row, per thread
    const int t_of = warp < 2 ? 0 : (warp - 2) >> 3, t_tid = threadIdx.x - 64 - t_of * 256;
    uint4 q_pre[QP];
    if (warp >= 2) {
#pragma unroll
        for (int e = 0; e < QP; ++e) {
            const int u = e * 256 + t_tid, rr = row0 + t_of * BQ + u / PPR;
            q_pre[e] = rr < a.max_nodes * group ? *reinterpret_cast<const uint4 *>(q_row(rr) + u % PPR * 8) : make_uint4(0, 0, 0, 0);
        }
    }
    const tree::Seq s = tree::load_seq(a, b);
    const int R = s.n * group;
    if (row0 >= R) return;                                          // (the whole cluster)

    // this CTA's blocks of positions
    const int nb = (s.n_keys + BKEY - 1) / BKEY, per = (nb + n_splits - 1) / n_splits;
    const int kb0 = min(split * per, nb), n_kb = min(per, nb - kb0);
    const int n_pages = (s.n_keys + 15) >> 4;

    auto quarters = [&](int t) { return min(4, max(0, (R - row0 - t * BQ + 31) >> 5)); };      // of tile t, that have rows
    const int n_tiles = TILES == 2 && quarters(1) > 0 ? 2 : 1;
    const int n_warps = 2 * (quarters(0) + (TILES == 2 ? quarters(TILES - 1) : 0));            // softmax warps at work
    auto part_ml = [&](unsigned char *p, int x) { return reinterpret_cast<float2 *>(p + x * 8); };       // where the queries were
    if (threadIdx.x == 0) {
        mbar_init(&q_full, 8 * TILES);
        mbar_init(&all_bar, n_warps);
        mbar_init(&tile_bar, 2 * quarters(0));
        for (int t = 0; t < TILES; ++t)
            for (int i = 0; i < 4; ++i) mbar_init(&pair_bar[t][i], 2);
        for (int i = 0; i < C::KS; ++i) { mbar_init(&k_full[i], 1); mbar_init(&k_empty[i], 1); }
        for (int i = 0; i < C::VS; ++i) { mbar_init(&v_full[i], 1); mbar_init(&v_empty[i], 1); }
        for (int i = 0; i < 2; ++i) {
            mbar_init(&s_full[i], 1);
            mbar_init(&p_full[i], 2 * (TILES == 2 ? max(1, quarters(i)) : quarters(0)));
        }
        for (int t = 0; t < TILES; ++t) { mbar_init(&o_done[t], 1); mbar_init(&o_all[t], 1); }
        s_err = 0;
        s_bad_page = s_odd[0] = s_odd[1] = 0;
        s_odd_tokens = 0;
        asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
    }
    if (warp == 1) {
        asm volatile("tcgen05.alloc.cta_group::1.sync.aligned.shared::cta.b32 [%0], %1;" ::"r"(smem_u32(&tmem_base_s)), "r"(C::TMEM) : "memory");
        asm volatile("tcgen05.relinquish_alloc_permit.cta_group::1.sync.aligned;" ::: "memory");
    }
    // Page ids (warp 0): lane i holds page i of the current four blocks, the next four are requested one round ahead.  A position
    // behind the last, or an id that names no page, is copied from coordinate -1: zeros.
    auto page_of = [&](int pi) {
        const int pg = pi < n_pages ? s.pt[pi] : -1;
        return a.kv.holds(pg) ? pg : -1;
    };
    int cur = warp == 0 ? page_of(PAGES * kb0 + lane) : -1, nxt = warp == 0 ? page_of(PAGES * kb0 + 32 + lane) : -1;
    asm volatile("tcgen05.fence::before_thread_sync;" ::: "memory");
    __syncthreads();
    asm volatile("tcgen05.fence::after_thread_sync;" ::: "memory");
    const uint32_t tmem_base = tmem_base_s;
    pdl_launch();

    if (warp == 0) {
        int n_k = 0, n_v = 0;                        // blocks whose keys, whose values are on their way
        for (int j = 0; j < n_kb; ++j) {
            const int ks = j % C::KS, vs = j % C::VS, first = (PAGES * j) & 31;
            if (first == 0 && j > 0) { cur = nxt; nxt = page_of(PAGES * (kb0 + j) + 32 + lane); }
            int pages[PAGES];
#pragma unroll
            for (int pg = 0; pg < PAGES; ++pg) pages[pg] = __shfl_sync(0xffffffffu, cur, first + pg);
            bool ok = true;
            if (lane == 0) {
                if (j >= C::KS && !wait_or_err(&k_empty[ks], ((j / C::KS) & 1) ^ 1, &s_err)) {
                    if (!s_err) s_err = 1;
                    ok = false;
                } else {
                    mbar_expect_tx(&k_full[ks], C::K_BYTES);
#pragma unroll
                    for (int pg = 0; pg < PAGES; ++pg)
#pragma unroll
                        for (int kb = 0; kb < C::KB; ++kb)
                            tma_load_5d(k_sm + ks * C::K_BYTES + kb * BKEY * 128 + pg * 2048, &maps.k, kb * 64, 0, kvh, a.layer - 1, pages[pg], &k_full[ks]);
                    n_k = j + 1;
                }
                if (ok && j >= C::VS && !wait_or_err(&v_empty[vs], ((j / C::VS) & 1) ^ 1, &s_err)) {
                    if (!s_err) s_err = 2;
                    ok = false;
                } else if (ok) {
                    mbar_expect_tx(&v_full[vs], C::V_BYTES);
#pragma unroll
                    for (int pg = 0; pg < PAGES; ++pg)
                        tma_load_5d(v_sm + vs * C::V_BYTES + pg * HD * 32, &maps.v, 0, 0, kvh, a.layer - 1, pages[pg], &v_full[vs]);
                    n_v = j + 1;
                }
            }
            if (!__shfl_sync(0xffffffffu, (int)ok, 0)) break;
        }
        if (s_err && lane == 0) {
            drain(k_full, C::KS, n_k % C::KS, (uint32_t)(n_k / C::KS) & 1);
            drain(v_full, C::VS, n_v % C::VS, (uint32_t)(n_v / C::VS) & 1);
        }
    } else if (warp == 1) {
        if (lane == 0 && n_kb > 0) {
            // instruction descriptors: fp32 accumulate, bf16 x bf16, both operands K-major, M = 128, N = 128 / HD
            const uint32_t idesc_s = (1u << 4) | (1u << 7) | (1u << 10) | ((uint32_t)(BKEY >> 3) << 17) | ((uint32_t)(BQ >> 4) << 24);
            const uint32_t idesc_o = (1u << 4) | (1u << 7) | (1u << 10) | ((uint32_t)(HD >> 3) << 17) | ((uint32_t)(BQ >> 4) << 24);
            const uint32_t q_addr = smem_u32(q_sm), k_addr = smem_u32(k_sm), v_addr = smem_u32(v_sm);
            int n_s[2] = {0, 0}, n_p[2] = {0, 0}, n_v = 0, n_k = 0;   // scores issued into each buffer, products of each tile, blocks whose values, whose keys were given back
            bool ok = wait_or_err(&q_full, 0, &s_err);
            if (!ok && !s_err) s_err = 3;
            // scores of block j, tile t, into buffer buf: whatever used the buffer before was issued earlier, and MMAs run in order
            auto scores = [&](int j, int t, int buf) -> bool {
                if (!wait_or_err(&k_full[j % C::KS], (j / C::KS) & 1, &s_err)) { if (!s_err) s_err = 4; return false; }
                asm volatile("tcgen05.fence::after_thread_sync;" ::: "memory");
#pragma unroll
                for (int kb = 0; kb < C::KB; ++kb) {
                    const uint64_t da = umma_desc(q_addr + (t * C::KB + kb) * C::Q_PART), db = umma_desc(k_addr + (j % C::KS) * C::K_BYTES + kb * BKEY * 128);
#pragma unroll
                    for (int k = 0; k < 4; ++k) umma_bf16(tmem_base + (uint32_t)(buf * BKEY), da + 2 * k, db + 2 * k, idesc_s, (kb | k) != 0);
                }
                umma_commit(&s_full[buf]);
                ++n_s[buf];
                if (t == n_tiles - 1) { umma_commit(&k_empty[j % C::KS]); n_k = j + 1; }
                return true;
            };
            auto products = [&](int j, int t, int buf) -> bool {
                if (!wait_or_err(&p_full[buf], (TILES == 2 ? j : j >> 1) & 1, &s_err)) { if (!s_err) s_err = 5; return false; }
                if (t == 0 && !wait_or_err(&v_full[j % C::VS], (j / C::VS) & 1, &s_err)) { if (!s_err) s_err = 6; return false; }
                asm volatile("tcgen05.fence::after_thread_sync;" ::: "memory");
#pragma unroll
                for (int kk = 0; kk < PAGES; ++kk)
                    umma_bf16_ts(tmem_base + C::O_COL + (uint32_t)(t * HD), tmem_base + (uint32_t)(buf * BKEY + (kk >> 2) * 64 + (kk & 3) * 8),
                                 umma_desc_sw32(v_addr + (j % C::VS) * C::V_BYTES + kk * HD * 32), idesc_o, (j | kk) != 0);
                umma_commit(&o_done[t]);
                ++n_p[t];
                if (t == n_tiles - 1) { umma_commit(&v_empty[j % C::VS]); n_v = j + 1; }
                if (j == n_kb - 1) umma_commit(&o_all[t]);         // (last: nothing of this thread's arrives behind it)
                return true;
            };
            for (int t = 0; ok && t < n_tiles; ++t) ok = scores(0, t, t);
            for (int j = 0; ok && j < n_kb; ++j) {
                if (TILES == 1) {
                    if (j + 1 < n_kb) ok = scores(j + 1, 0, (j + 1) & 1);
                    if (ok) ok = products(j, 0, j & 1);
                } else {
                    for (int t = 0; ok && t < n_tiles; ++t) {
                        ok = products(j, t, t);
                        if (ok && j + 1 < n_kb) ok = scores(j + 1, t, t);
                    }
                }
            }
            if (s_err) {
                for (int i = 0; i < 2; ++i)
                    if (n_s[i]) drain(&s_full[i], 1, 0, (uint32_t)n_s[i] & 1);
                for (int t = 0; t < TILES; ++t)
                    if (n_p[t]) {
                        drain(&o_done[t], 1, 0, (uint32_t)n_p[t] & 1);
                        if (n_p[t] == n_kb) drain(&o_all[t], 1, 0, 1);
                    }
                drain(k_empty, C::KS, n_k % C::KS, (uint32_t)(n_k / C::KS) & 1);
                drain(v_empty, C::VS, n_v % C::VS, (uint32_t)(n_v / C::VS) & 1);
            }
        }
    } else {
        const int t = t_of, half = ((warp - 2) >> 2) & 1, q = warp & 3;      // tile, which 64 of a block's keys, TMEM lane quarter this warp may access
        const int trow = q * 32 + lane, rr = row0 + t * BQ + trow, nq = quarters(t);
        const bool row_ok = rr < R;
        // queries: rows of 128-byte k-blocks with the 128-byte swizzle
#pragma unroll
        for (int e = 0; e < QP; ++e) {
            const int u = e * 256 + t_tid, r = u / PPR, c = u % PPR;
            *reinterpret_cast<uint4 *>(q_sm + t * C::KB * C::Q_PART + (c >> 3) * C::Q_PART + r * 128 + (((c & 7) ^ (r & 7)) << 4)) = q_pre[e];
        }
        asm volatile("fence.proxy.async.shared::cta;" ::: "memory");
        __syncwarp();
        if (lane == 0) mbar_arrive(&q_full);
        if (q < nq) {
            const int i = row_ok ? node_of(rr) : 0, hq = row_ok ? rr - i * group : 0;
            const uint64_t bits = row_ok ? tree::node_bits(a, b, i) : 0;
            const bf16 *qp = a.q + b * a.q_seq + i * a.q_node + (size_t)(kvh * group + hq) * HD;
            // does the table name pages that are none?  (then every block's ids are looked at again)
            bool bad = false;
            for (int p = PAGES * kb0 + half * nq * 32 + trow; p < min(n_pages, PAGES * (kb0 + n_kb)); p += 2 * nq * 32) bad |= !a.kv.holds(s.pt[p]);
            if (__any_sync(0xffffffffu, bad) && lane == 0) s_bad_page = 1;
            // barriers among softmax warps, bounded like every wait
            auto meet = [&](uint64_t *bar, uint32_t parity) -> bool {
                __syncwarp();
                if (lane == 0) mbar_arrive(bar);
                return wait_or_err(bar, parity, &s_err);
            };
            uint32_t tile_phase = 0;
            bool ok = meet(&all_bar, 0);
            if (!ok && !s_err) s_err = 7;
            const bool bad_pages = s_bad_page != 0;

            const uint32_t lane_addr = tmem_base + ((uint32_t)(q * 32) << 16);
            const uint32_t o_addr = lane_addr + C::O_COL + (uint32_t)(t * HD);
            float m_ref = -INFINITY, l = 0.f;
            for (int j = 0; ok && j < n_kb; ++j) {
                const int buf = TILES == 2 ? t : j & 1, key0 = (kb0 + j) * BKEY, key1 = key0 + 64 * half;
                const uint32_t s_addr = lane_addr + (uint32_t)(buf * BKEY + 64 * half);
                const bool tail = key0 + BKEY > s.len, masked = tail || bad_pages;
                uint64_t vm = ~0ull;
                if (masked) {
                    vm = visible(bits, key1, s.len, s.n_keys);
                    for (int pg = 0; bad_pages && pg < 4; ++pg) {
                        const int pi = (key1 >> 4) + pg;
                        if (pi >= n_pages || !a.kv.holds(s.pt[pi])) vm &= ~(0xffffull << (16 * pg));
                    }
                }
                if (!wait_or_err(&s_full[buf], (TILES == 2 ? j : j >> 1) & 1, &s_err)) { if (!s_err) s_err = 8; ok = false; break; }
                asm volatile("tcgen05.fence::after_thread_sync;" ::: "memory");
                uint32_t x[32];
                auto mask_chunk = [&](int c) {
                    const uint32_t v = (uint32_t)(vm >> (32 * c));
#pragma unroll
                    for (int e = 0; e < 32; ++e)
                        if (!((v >> e) & 1)) x[e] = 0xff800000u;
                };
                // first sweep: the maximum, of both halves
                float m4[4] = {-INFINITY, -INFINITY, -INFINITY, -INFINITY};
#pragma unroll
                for (int c = 1; c >= 0; --c) {                    // (the first chunk last: the second sweep begins with it)
                    tmem_ld32(s_addr + 32 * c, x);
                    tmem_ld_wait();
                    if (masked) mask_chunk(c);
#pragma unroll
                    for (int e = 0; e < 32; ++e) m4[e & 3] = fmaxf(m4[e & 3], __uint_as_float(x[e]));
                }
                float mx = fmaxf(fmaxf(m4[0], m4[1]), fmaxf(m4[2], m4[3]));
                s_max[buf][half][trow] = mx;
                if (!meet(&pair_bar[t][q], j & 1)) { if (!s_err) s_err = 14; ok = false; break; }
                mx = fmaxf(mx, s_max[buf][half ^ 1][trow]) * a.scale;
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
                // second sweep: probabilities, as bf16 over the scores of this half that have been read
                float ps[4] = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
                for (int c = 0; c < 2; ++c) {
                    if (c == 1) {
                        tmem_ld32(s_addr + 32, x);
                        tmem_ld_wait();
                        if (masked) mask_chunk(1);
                    }
                    uint32_t pk[16];
#pragma unroll
                    for (int e = 0; e < 32; e += 4) {
                        float f[4];
#pragma unroll
                        for (int i = 0; i < 4; ++i) f[i] = __uint_as_float(x[e + i]);
                        fma2(f[0], f[1], a.scale, -m_use);
                        fma2(f[2], f[3], a.scale, -m_use);
#pragma unroll
                        for (int i = 0; i < 4; ++i) f[i] = ex2f(f[i]);
                        add2(ps[0], ps[1], f[0], f[1]);
                        add2(ps[2], ps[3], f[2], f[3]);
                        pk[e / 2] = pack_bf16(f[0], f[1]);
                        pk[e / 2 + 1] = pack_bf16(f[2], f[3]);
                    }
                    tmem_st16(s_addr + 16 * c, pk);
                }
                l += (ps[0] + ps[1]) + (ps[2] + ps[3]);
                if (__any_sync(0xffffffffu, alpha != 1.f)) {
                    // (The previous block's products are part of the output; with one tile they may still be running.  Those before them are done,
                    // as this block's scores were issued after them, and this block's wait for this warp: the phase is the one meant.)
                    if (TILES == 1 && !wait_or_err(&o_done[t], (j - 1) & 1, &s_err)) { if (!s_err) s_err = 9; ok = false; break; }
                    asm volatile("tcgen05.fence::after_thread_sync;" ::: "memory");
                    for (int c0 = half * (HD / 2); c0 < (half + 1) * (HD / 2); c0 += 32) {
                        tmem_ld32(o_addr + (uint32_t)c0, x);
                        tmem_ld_wait();
#pragma unroll
                        for (int e = 0; e < 32; ++e) x[e] = __float_as_uint(__uint_as_float(x[e]) * alpha);
                        tmem_st32(o_addr + (uint32_t)c0, x);
                    }
                }
                if (tail && t == 0) {
                    // Values of drafted and of never written slots must not meet a probability of zero as infinity or NaN.  The
                    // first tile's warps look; what they find they zero, by whole tokens, and remember the drafted ones.
                    unsigned char *vst = v_sm + (j % C::VS) * C::V_BYTES;
                    if (!wait_or_err(&v_full[j % C::VS], (j / C::VS) & 1, &s_err)) { if (!s_err) s_err = 10; ok = false; break; }
                    bool odd = false;
                    const int u0 = max(0, (s.len - key0) >> 4) * HD * 2, u1 = min(PAGES, n_pages - (key0 >> 4)) * HD * 2;     // (pages behind the last are zeros)
                    for (int u = u0 + half * nq * 32 + trow; u < u1; u += 2 * nq * 32) {
                        const uint4 v = *reinterpret_cast<const uint4 *>(vst + u * 16);
                        odd |= odd_pair(v.x) | odd_pair(v.y) | odd_pair(v.z) | odd_pair(v.w);
                    }
                    if (__any_sync(0xffffffffu, odd) && lane == 0) s_odd[j & 1] = 1;      // (never cleared: two blocks later it only costs time)
                    if (!meet(&tile_bar, tile_phase)) { if (!s_err) s_err = 11; ok = false; break; }
                    tile_phase ^= 1;
                    for (int e = 2 * q + half; s_odd[j & 1] && e < BKEY; e += 2 * nq) {
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
                    asm volatile("fence.proxy.async.shared::cta;" ::: "memory");      // visible to the tensor core's reads
                }
                asm volatile("tcgen05.wait::st.sync.aligned;" ::: "memory");
                asm volatile("tcgen05.fence::before_thread_sync;" ::: "memory");
                __syncwarp();
                if (lane == 0) mbar_arrive(&p_full[buf]);
            }
            // The output is complete: a barrier of its own, used once.  A wait names a phase of o_done by its parity alone, and here either of
            // its last two phases may be open, or none: with one tile scores(j + 1) are issued before products(j), so the last
            // scores say nothing about the products of the block before.
            if (ok && n_kb > 0 && !wait_or_err(&o_all[t], 0, &s_err)) { if (!s_err) s_err = 12; ok = false; }
            if (half) s_sum[t][trow] = l;
            if (!meet(&all_bar, 1)) { if (!s_err) s_err = 13; ok = false; }       // both tiles are done with the rings, s_odd_tokens and the sums are complete
            l = half ? l : l + s_sum[t][trow];                   // (the first half's threads go on with the sum)
            asm volatile("tcgen05.fence::after_thread_sync;" ::: "memory");
            const uint64_t odd_seen = s_odd_tokens & bits;
            const float m_use = m_ref == -INFINITY ? 0.f : m_ref;
            const size_t head = ((size_t)(a.layer - 1) * a.kv.nkv + kvh) * a.kv.head_elems();
            if (n_splits == 1) {                                   // (then the second half's need it as well)
                if (!half) s_sum[t][trow] = l;
                if (!meet(&pair_bar[t][q], n_kb & 1)) { if (!s_err) s_err = 15; ok = false; }
                l = s_sum[t][trow];
            }
            const float inv = l == 0.f ? 0.f : 1.f / l;            // (l = 0: nothing is visible, the result is zero)
            const size_t out = b * a.o_seq + i * a.o_node + (size_t)(kvh * group + hq) * HD;
            if (n_splits > 1 && !half) *part_ml(q_sm, t * BQ + trow) = make_float2(m_ref, ok && !s_err ? l : NAN);
            float *po = reinterpret_cast<float *>(k_sm) + (size_t)(t * BQ + trow) * HD;
            for (int c0 = half * (HD / 2); c0 < (half + 1) * (HD / 2) && n_kb > 0; c0 += 32) {
                uint32_t o[32];
                if (ok) tmem_ld32(o_addr + (uint32_t)c0, o);
                tmem_ld_wait();
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
                        tree::split_out(__uint_as_float(o[e + 0]) * inv, __uint_as_float(o[e + 1]) * inv, hi.x, lo.x);
                        tree::split_out(__uint_as_float(o[e + 2]) * inv, __uint_as_float(o[e + 3]) * inv, hi.y, lo.y);
                        tree::split_out(__uint_as_float(o[e + 4]) * inv, __uint_as_float(o[e + 5]) * inv, hi.z, lo.z);
                        tree::split_out(__uint_as_float(o[e + 6]) * inv, __uint_as_float(o[e + 7]) * inv, hi.w, lo.w);
                        *reinterpret_cast<uint4 *>(a.out + out + c0 + e) = hi;
                        if (a.out_lo) *reinterpret_cast<uint4 *>(a.out_lo + out + c0 + e) = lo;
                    }
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
        // Each CTA finishes a share of the rows, four columns per thread, states and outputs of four parts on their way together (the
        // states first and the weights through shared memory took a round trip more).
        constexpr int LPR = HD / 4;
        const int parts = (nb + per - 1) / per, mine0 = rows * split / n_splits, mine1 = rows * (split + 1) / n_splits;     // (parts with blocks, this CTA's rows)
        for (int e = mine0 * LPR + threadIdx.x; e < mine1 * LPR; e += C::THREADS) {
            const int x = e / LPR, c = e % LPR;
            const size_t off = (size_t)x * HD + ((c ^ (x & 15)) << 2);
            float M = -INFINITY, L = 0.f;
            float4 o = make_float4(0.f, 0.f, 0.f, 0.f);
#pragma unroll 1
            for (int k0 = 0; k0 < parts; k0 += 4) {
                float2 ml[4];
                float4 v[4];
#pragma unroll
                for (int k = 0; k < 4; ++k) {
                    ml[k] = make_float2(-INFINITY, 0.f);
                    if (k0 + k < parts) {
                        ml[k] = *part_ml(cl.map_shared_rank(q_sm, k0 + k), x);
                        v[k] = *reinterpret_cast<const float4 *>(cl.map_shared_rank(reinterpret_cast<float *>(k_sm), k0 + k) + off);
                    }
                }
                const float m_new = fmaxf(fmaxf(M, fmaxf(ml[0].x, ml[1].x)), fmaxf(ml[2].x, ml[3].x)), mu = m_new == -INFINITY ? 0.f : m_new;
                const float f = ex2f(M - mu);
                M = m_new;
                L *= f; o.x *= f; o.y *= f; o.z *= f; o.w *= f;
#pragma unroll
                for (int k = 0; k < 4; ++k)
                    if (k0 + k < parts) {
                        const float w = ex2f(ml[k].x - mu);
                        L += ml[k].y * w;
                        o.x += v[k].x * w; o.y += v[k].y * w; o.z += v[k].z * w; o.w += v[k].w * w;
                    }
            }
            const float inv = L == 0.f ? 0.f : 1.f / L;             // (no number if a part gave up)
            o.x *= inv; o.y *= inv; o.z *= inv; o.w *= inv;
            const int rr = row0 + x, i = node_of(rr), hq = rr - i * group;
            const size_t at = b * a.o_seq + i * a.o_node + (size_t)(kvh * group + hq) * HD + 4 * c;
            uint2 hi, lo;
            tree::split_out(o.x, o.y, hi.x, lo.x);
            tree::split_out(o.z, o.w, hi.y, lo.y);
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

// how a call's blocks of keys are spread
struct Plan {
    int splits;          // CTAs of a cluster; 0: an error
    int64_t steps;       // blocks that a CTA takes, times the waves of CTAs
};

template <int HD, int TILES>
Plan plan(const TreeArgs &a, int batch, int max_len) {
    auto kern = tree_attention_tc_kernel<HD, TILES>;
    static SmemAttrOnce attr;
    static ClusterRoom room;
    const int n_sms = current_sms();
    if (!n_sms || attr.set(kern, Cfg<HD, TILES>::SMEM) != cudaSuccess) return Plan{0, 0};
    // as many parts of the keys as are resident together, none for three blocks and less: joining parts costs as much as two blocks
    const int n_rt = (a.max_nodes * (a.nh / a.kv.nkv) + TILES * BQ - 1) / (TILES * BQ), blocks = (max_len + a.max_nodes + BKEY - 1) / BKEY;
    const int64_t units = (int64_t)a.kv.nkv * n_rt * batch;
    const int splits = blocks <= 3 ? 1 : room.best(kern, Cfg<HD, TILES>::THREADS, Cfg<HD, TILES>::SMEM, units, blocks);
    return Plan{splits, (blocks + splits - 1) / splits * ((units * splits + n_sms - 1) / n_sms)};
}

template <int HD, int TILES>
cudaError_t launch(const Maps &m, const TreeArgs &a, int batch, int splits, cudaStream_t st) {
    const int n_rt = (a.max_nodes * (a.nh / a.kv.nkv) + TILES * BQ - 1) / (TILES * BQ);
    return launch_cluster(tree_attention_tc_kernel<HD, TILES>, dim3(splits, a.kv.nkv * n_rt, batch), Cfg<HD, TILES>::THREADS, Cfg<HD, TILES>::SMEM, splits, st, m, a);
}

template <int HD>
cudaError_t launch_form(const TreeArgs &a, int batch, int max_len, cudaStream_t st) {
    Maps m;
    if (!make_maps(a.kv, &m)) return cudaErrorInvalidValue;
    const Plan one = plan<HD, 1>(a, batch, max_len);
    if (!one.splits) return cudaErrorInvalidDevice;
    if (a.max_nodes * (a.nh / a.kv.nkv) > BQ) {
        // Two tiles per CTA read the keys once for both, one's softmax beside the other's MMAs; with one per CTA (the second reads
        // the keys from L2) there are twice the CTAs, with two score buffers each.  us, one / two tiles:
        //   8B shape, 1 x 64 nodes   100 positions 10.4 / 17.8,  2000: 13.3 / 20.8,  16000:  41.9 /  49.6
        //   8B shape, 4 x 64 nodes   500           13.8 / 19.2,  4000: 35.5 / 36.9,  16000: 106   /  90
        //   8B shape, 8 x 64 nodes   1300          25.4 / 31.9,  4000: 58.0 / 57.2,  16000: 203   / 161
        //   1B shape, 4 x 40 nodes   500           11.3 / 13.3,  4000: 27.3 / 26.4,  16000:  81   /  72
        // That is 8.6 + 1.6 steps against 15.6 + 2.4 steps at head dimension 128, 8.4 + 1.15 against 10.5 + 2.0 at 64.
        const Plan two = plan<HD, 2>(a, batch, max_len);
        if (!two.splits) return cudaErrorInvalidDevice;
        if (HD == 128 ? 3 * two.steps + 9 < 2 * one.steps : 7 * two.steps + 7 < 4 * one.steps) return launch<HD, 2>(m, a, batch, two.splits, st);
    }
    return launch<HD, 1>(m, a, batch, one.splits, st);
}

}  // namespace

cudaError_t launch_tree_attention_tc(const TreeArgs &a, int batch, int max_len, cudaStream_t st) {
    return a.kv.hd == 128 ? launch_form<128>(a, batch, max_len, st) : launch_form<64>(a, batch, max_len, st);
}
