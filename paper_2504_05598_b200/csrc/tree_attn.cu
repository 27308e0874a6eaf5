// Attention of a tree of drafted tokens over the paged cache (del_tree_attention).
//
// For every sequence, kv head and tile of 16 query rows (node x query head of the group) one cluster of CTAs walks the pages of
// the keys, each warp of it every so manyth page (so that the first page ids can be requested before the lengths are known).  A warp
// keeps the online-softmax state of the tile in registers: S = Q K^T and O += P V are bf16 m16n8k16 MMAs with fp32 sums, the running
// maximum and sum are fp32; the probabilities are rounded to bf16, which the MMA takes (off by 2^-8 of their value at most, as the
// output's own rounding), their sum is of the unrounded ones.  The warps join through shared memory, the CTAs of the cluster through
// distributed shared memory: one launch, no workspace, a fixed order of sums.
//
// Long calls are bound by HBM (single tokens, 8B shape, 16 rows of 4000 positions: 44 us, 5600 GB/s; 1B shape, 64 rows of 3000: 67 us,
// 5480 GB/s), short ones by latency (8B shape, 8 nodes behind 200 positions: 7.0 us, of which an empty launch is some 2.5 and the walk
// lengths -> page ids -> keys -> join three round trips).
//
// Fragments: the MMA sums over its k index, so a permutation of k that both operands share is free.  For Q K^T a thread takes 16
// contiguous bytes of a key row and of the query row; for P V the page holds V^T rows of 16 tokens, and the score columns are
// assigned to tokens such that a thread's four probabilities belong to tokens 4t .. 4t + 3, 8 contiguous bytes of a V^T row.
//
// What is masked never enters a sum: scores by selection, values of slots that nobody may see by zeroing them in registers (a slot that
// was never written may hold anything), and where a drafted token's values are not finite, the page's P V is summed element by
// element over the visible tokens.
#include <cooperative_groups.h>
#include <cstring>

#include "tree_attn.cuh"
#include "tree_form.h"

namespace cg = cooperative_groups;

namespace {

using namespace tree;

constexpr int NW = 8, THREADS = NW * 32;
static_assert(NW == 8, "the join of the warps adds four pairs");
constexpr float LOG2E = 1.4426950408889634f;

template <int HD>
__global__ void __launch_bounds__(THREADS, HD == 64 ? 2 : 1) tree_attention_kernel(const TreeArgs a) {
    constexpr int KS = HD / 32, NJ = HD / 8, LD = HD + 8;
    __shared__ float so[NW / 2][16][LD];
    __shared__ float2 sml[NW][16];
    __shared__ float2 tile_ml[16];
    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31, g = lane >> 2, t = lane & 3;
    const int n_splits = gridDim.x, split = blockIdx.x;
    pdl_wait();
    pdl_launch();
    const int group = a.nh / a.kv.nkv, n_mt = (a.max_nodes * group + 15) >> 4;
    const int kvh = blockIdx.y / n_mt, mt = blockIdx.y - kvh * n_mt, b = blockIdx.z;
    // page ids: lane i holds the id of the warp's i-th page of the current 32
    const int p_first = split * NW + warp, p_step = n_splits * NW;
    const int32_t *pt = a.table + (size_t)b * a.stride;
    auto ids = [&](int i0) {
        const int64_t p = p_first + (int64_t)p_step * (i0 + lane);
        return p < a.cols ? pt[p] : -1;
    };
    int id32 = ids(0);
    const Seq s = load_seq(a, b);
    const int R = s.n * group;
    if (mt * 16 >= R) return;                                   // (the whole cluster)

    // this thread's two rows of the tile: node and query head, what the node sees, its query fragments
    uint4 qf[2][KS];
    uint64_t bits[2];
    bool rv[2];
#pragma unroll
    for (int h = 0; h < 2; ++h) {
        const int rr = mt * 16 + g + 8 * h;
        rv[h] = rr < R;
        const int i = rv[h] ? rr / group : 0, hq = rv[h] ? rr - i * group : 0;
        bits[h] = rv[h] ? node_bits(a, b, i) : 0;
        const bf16 *qp = a.q + b * a.q_seq + i * a.q_node + (size_t)(kvh * group + hq) * HD + 8 * t;
#pragma unroll
        for (int ks = 0; ks < KS; ++ks) qf[h][ks] = rv[h] ? *reinterpret_cast<const uint4 *>(qp + 32 * ks) : make_uint4(0, 0, 0, 0);
    }
    float m_run[2] = {-INFINITY, -INFINITY}, l_run[2] = {0.f, 0.f}, O[NJ][4];
#pragma unroll
    for (int j = 0; j < NJ; ++j) O[j][0] = O[j][1] = O[j][2] = O[j][3] = 0.f;

    const int n_pages = (s.n_keys + 15) >> 4;
    const size_t page_stride = a.kv.page_elems(), head_off = ((size_t)(a.layer - 1) * a.kv.nkv + kvh) * a.kv.head_elems();
    const int key0 = 4 * (g >> 1) + (g & 1);                    // token of column g of score tile 0; tile 1: +2
    // With one CTA per SM the warps' own loads do not cover the latency: the next page is requested into L2 (8B shape, 16 single tokens of 4000
    // positions: 48.1 -> 44.0 us; of one row of 3000, three pages a warp, 8.5 -> 9.0, hence the bound.  With two CTAs per SM, hd 64, it costs 8 %.)
    const bool ahead = HD == 128 && n_pages > 4 * p_step;
    for (int p = p_first, it = 0; p < n_pages; p += p_step, ++it) {
        if (it > 0 && (it & 31) == 0) id32 = ids(it);
        const int pg = __shfl_sync(0xffffffffu, id32, it & 31);
        if (ahead) {
            const int next = __shfl_sync(0xffffffffu, id32, (it + 1) & 31);
            if (lane == 0 && ((it + 1) & 31) != 0 && p + p_step < n_pages && a.kv.holds(next)) {
                l2_prefetch_bulk(a.kv.k + (size_t)next * page_stride + head_off, 16 * HD * 2);
                l2_prefetch_bulk(a.kv.v + (size_t)next * page_stride + head_off, 16 * HD * 2);
            }
        }
        if (!a.kv.holds(pg)) continue;                          // (the same in every lane)
        const bf16 *kp = a.kv.k + (size_t)pg * page_stride + head_off, *vp = a.kv.v + (size_t)pg * page_stride + head_off;
        uint4 kf[2][KS];
        uint2 vf[NJ];
#pragma unroll
        for (int ks = 0; ks < KS; ++ks) {
            kf[0][ks] = ldg_act16(kp + key0 * HD + 32 * ks + 8 * t);
            kf[1][ks] = ldg_act16(kp + (key0 + 2) * HD + 32 * ks + 8 * t);
        }
#pragma unroll
        for (int j = 0; j < NJ; ++j) vf[j] = ldg_act8(vp + (8 * j + g) * 16 + 4 * t);
        float s0[4] = {0.f, 0.f, 0.f, 0.f}, s1[4] = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
        for (int ks = 0; ks < KS; ++ks) {
            mma_bf16_16816(s0, qf[0][ks].x, qf[1][ks].x, qf[0][ks].y, qf[1][ks].y, kf[0][ks].x, kf[0][ks].y);
            mma_bf16_16816(s0, qf[0][ks].z, qf[1][ks].z, qf[0][ks].w, qf[1][ks].w, kf[0][ks].z, kf[0][ks].w);
            mma_bf16_16816(s1, qf[0][ks].x, qf[1][ks].x, qf[0][ks].y, qf[1][ks].y, kf[1][ks].x, kf[1][ks].y);
            mma_bf16_16816(s1, qf[0][ks].z, qf[1][ks].z, qf[0][ks].w, qf[1][ks].w, kf[1][ks].z, kf[1][ks].w);
        }
        const int tok0 = p * 16 + 4 * t;                        // tokens tok0 .. tok0 + 3: s0[0], s0[1], s1[0], s1[1] of row g
        const bool tail = p * 16 + 16 > s.len;
        bool odd_values = false;                                // a drafted token's values are not finite
        if (tail) {
            // slots behind the last node: zero; drafted tokens: looked at
#pragma unroll
            for (int j = 0; j < NJ; ++j) {
                if (tok0 + 0 >= s.n_keys) vf[j].x &= 0xffff0000u;
                if (tok0 + 1 >= s.n_keys) vf[j].x &= 0x0000ffffu;
                if (tok0 + 2 >= s.n_keys) vf[j].y &= 0xffff0000u;
                if (tok0 + 3 >= s.n_keys) vf[j].y &= 0x0000ffffu;
                const uint32_t e = 0x7f807f80u;
                const uint32_t x = vf[j].x & e, y = vf[j].y & e;
                odd_values |= (x & 0xffff0000u) == 0x7f800000u || (x & 0xffffu) == 0x7f80u || (y & 0xffff0000u) == 0x7f800000u || (y & 0xffffu) == 0x7f80u;
            }
            odd_values = __any_sync(0xffffffffu, odd_values);
        }
        float pr[2][4];
#pragma unroll
        for (int h = 0; h < 2; ++h) {
            float v[4] = {s0[2 * h] * a.scale, s0[2 * h + 1] * a.scale, s1[2 * h] * a.scale, s1[2 * h + 1] * a.scale};
            if (tail) {
#pragma unroll
                for (int e = 0; e < 4; ++e)
                    if (!sees(bits[h], tok0 + e, s.len, s.n_keys)) v[e] = -INFINITY;
            }
            float mx = fmaxf(fmaxf(v[0], v[1]), fmaxf(v[2], v[3]));
            mx = fmaxf(mx, __shfl_xor_sync(0xffffffffu, mx, 1));
            mx = fmaxf(mx, __shfl_xor_sync(0xffffffffu, mx, 2));
            const float m_new = fmaxf(m_run[h], mx), base = m_new == -INFINITY ? 0.f : m_new;
            const float alpha = exp2f(m_run[h] - base);
            m_run[h] = m_new;
            float psum = 0.f;
#pragma unroll
            for (int e = 0; e < 4; ++e) { pr[h][e] = exp2f(v[e] - base); psum += pr[h][e]; }
            l_run[h] = l_run[h] * alpha + psum;
#pragma unroll
            for (int j = 0; j < NJ; ++j) { O[j][2 * h] *= alpha; O[j][2 * h + 1] *= alpha; }
        }
        if (!odd_values) {
            const uint32_t pa0 = pack_bf16(pr[0][0], pr[0][1]), pa1 = pack_bf16(pr[1][0], pr[1][1]);
            const uint32_t pa2 = pack_bf16(pr[0][2], pr[0][3]), pa3 = pack_bf16(pr[1][2], pr[1][3]);
#pragma unroll
            for (int j = 0; j < NJ; ++j) mma_bf16_16816(O[j], pa0, pa1, pa2, pa3, vf[j].x, vf[j].y);
        } else {
#pragma unroll
            for (int k = 0; k < 16; ++k) {
                const int src = (lane & ~3) | (k >> 2);
                const float p0 = __shfl_sync(0xffffffffu, pr[0][k & 3], src), p1 = __shfl_sync(0xffffffffu, pr[1][k & 3], src);
                const bool see0 = sees(bits[0], p * 16 + k, s.len, s.n_keys), see1 = sees(bits[1], p * 16 + k, s.len, s.n_keys);
                for (int j = 0; j < NJ; ++j) {
                    const float v0 = bf16_to_f(vp[(8 * j + 2 * t) * 16 + k]), v1 = bf16_to_f(vp[(8 * j + 2 * t + 1) * 16 + k]);
#pragma unroll
                    for (int jj = 0; jj < NJ; ++jj)
                        if (jj == j) {
                            if (see0) { O[jj][0] += p0 * v0; O[jj][1] += p0 * v1; }
                            if (see1) { O[jj][2] += p1 * v0; O[jj][3] += p1 * v1; }
                        }
                }
            }
        }
    }

    // the warps' states: the upper four leave theirs in shared memory, the lower four add theirs; then one sum over four
#pragma unroll
    for (int h = 0; h < 2; ++h) {
        l_run[h] += __shfl_xor_sync(0xffffffffu, l_run[h], 1);
        l_run[h] += __shfl_xor_sync(0xffffffffu, l_run[h], 2);
        if (t == 0) sml[warp][g + 8 * h] = make_float2(m_run[h], l_run[h]);
    }
    __syncthreads();
    float M[2], f[2];
#pragma unroll
    for (int h = 0; h < 2; ++h) {
        M[h] = -INFINITY;
#pragma unroll
        for (int w = 0; w < NW; ++w) M[h] = fmaxf(M[h], sml[w][g + 8 * h].x);
        f[h] = exp2f(m_run[h] - (M[h] == -INFINITY ? 0.f : M[h]));
    }
    if (warp >= NW / 2) {
#pragma unroll
        for (int h = 0; h < 2; ++h)
#pragma unroll
            for (int j = 0; j < NJ; ++j)
                *reinterpret_cast<float2 *>(&so[warp - NW / 2][g + 8 * h][8 * j + 2 * t]) = make_float2(O[j][2 * h] * f[h], O[j][2 * h + 1] * f[h]);
    }
    __syncthreads();
    if (warp < NW / 2) {
#pragma unroll
        for (int h = 0; h < 2; ++h)
#pragma unroll
            for (int j = 0; j < NJ; ++j) {
                float2 *dst = reinterpret_cast<float2 *>(&so[warp][g + 8 * h][8 * j + 2 * t]);
                const float2 v = *dst;
                *dst = make_float2(v.x + O[j][2 * h] * f[h], v.y + O[j][2 * h + 1] * f[h]);
            }
    }
    if (threadIdx.x < 16) {
        float m = -INFINITY, l = 0.f;
        for (int w = 0; w < NW; ++w) m = fmaxf(m, sml[w][threadIdx.x].x);
        const float base = m == -INFINITY ? 0.f : m;
        for (int w = 0; w < NW; ++w) l += sml[w][threadIdx.x].y * exp2f(sml[w][threadIdx.x].x - base);
        tile_ml[threadIdx.x] = make_float2(m, l);
    }
    __syncthreads();
    for (int e = threadIdx.x; e < 16 * HD; e += THREADS) {
        const int r = e / HD, c = e - r * HD;
        so[0][r][c] = (so[0][r][c] + so[1][r][c]) + (so[2][r][c] + so[3][r][c]);
    }
    cg::cluster_group cl = cg::this_cluster();
    if (n_splits > 1) cl.sync();
    else __syncthreads();

    // the tile's result: every CTA of the cluster finishes its share of the elements
    for (int e = split * THREADS + threadIdx.x; e < 16 * (HD / 2); e += n_splits * THREADS) {
        const int r = e / (HD / 2), c = (e - r * (HD / 2)) * 2, rr = mt * 16 + r;
        if (rr >= R) break;
        float m = -INFINITY, l = 0.f, o0 = 0.f, o1 = 0.f;
        if (n_splits == 1) {
            const float2 v = *reinterpret_cast<const float2 *>(&so[0][r][c]);
            l = tile_ml[r].y;
            o0 = v.x;
            o1 = v.y;
        }
#pragma unroll 1
        for (int k0 = 0; n_splits > 1 && k0 < n_splits; k0 += 4) {            // states and outputs of four CTAs on their way together
            float2 ml[4], v[4];
#pragma unroll
            for (int k = 0; k < 4; ++k) {
                ml[k] = make_float2(-INFINITY, 0.f);
                if (k0 + k < n_splits) {
                    ml[k] = cl.map_shared_rank(tile_ml, k0 + k)[r];
                    v[k] = *reinterpret_cast<const float2 *>(cl.map_shared_rank(&so[0][0][0], k0 + k) + r * LD + c);
                }
            }
            const float m_new = fmaxf(fmaxf(m, fmaxf(ml[0].x, ml[1].x)), fmaxf(ml[2].x, ml[3].x)), base = m_new == -INFINITY ? 0.f : m_new;
            const float f = exp2f(m - base);
            m = m_new;
            l *= f; o0 *= f; o1 *= f;
#pragma unroll
            for (int k = 0; k < 4; ++k)
                if (k0 + k < n_splits) {
                    const float w = exp2f(ml[k].x - base);
                    l += ml[k].y * w;
                    o0 += v[k].x * w;
                    o1 += v[k].y * w;
                }
        }
        const float inv = l == 0.f ? 0.f : 1.f / l;             // nothing visible: zeros
        const int i = rr / group, hq = rr - i * group;
        const size_t at = b * a.o_seq + i * a.o_node + (size_t)(kvh * group + hq) * HD + c;
        uint32_t hi, lo;
        split_out(o0 * inv, o1 * inv, hi, lo);
        *reinterpret_cast<uint32_t *>(a.out + at) = hi;
        if (a.out_lo) *reinterpret_cast<uint32_t *>(a.out_lo + at) = lo;
    }
    if (n_splits > 1) cl.sync();                                // nobody leaves while its shared memory is read
}

template <int HD>
cudaError_t launch(const TreeArgs &a, int batch, int pages, cudaStream_t st) {
    static ClusterRoom room;
    const int group = a.nh / a.kv.nkv, n_mt = (a.max_nodes * group + 15) / 16;
    const int64_t units = (int64_t)a.kv.nkv * n_mt * batch;
    const int splits = room.best(tree_attention_kernel<HD>, THREADS, 0, units, (pages + NW - 1) / NW);      // (a page per warp at least)
    return launch_cluster(tree_attention_kernel<HD>, dim3(splits, a.kv.nkv * n_mt, batch), THREADS, 0, splits, st, a);
}

}  // namespace

cudaError_t launch_tree_attention(const TreeArgs &a, int batch, int max_len, cudaStream_t st, bool streaming) {
    const int pages = (max_len + a.max_nodes + 15) / 16, n_sms = current_sms();
    if (!n_sms) return cudaErrorInvalidDevice;
    if (tree::takes_tcgen05(a.kv.hd, a.kv.nkv, a.nh / a.kv.nkv, a.max_nodes, batch, pages, n_sms, streaming)) return launch_tree_attention_tc(a, batch, max_len, st);
    return a.kv.hd == 128 ? launch<128>(a, batch, pages, st) : launch<64>(a, batch, pages, st);
}

extern "C" int del_tree_attention(const del_pages *kv, const del_tree_attn *x, void *cuda_stream) {
    TreeArgs a;
    memset(&a, 0, sizeof(a));
    if (!x || !page_view(kv, &a.kv)) return DEL_EINVAL;
    if (!x->q || !x->out || !x->page_table || !x->lens) return DEL_EINVAL;
    if (((uintptr_t)x->q | (uintptr_t)x->out | (uintptr_t)x->out_lo) & 15) return DEL_EINVAL;
    if (((uintptr_t)x->page_table | (uintptr_t)x->lens | (uintptr_t)x->nodes | (uintptr_t)x->error) & 3 || (uintptr_t)x->mask & 7) return DEL_EINVAL;
    if ((x->q_seq_stride | x->q_node_stride | x->out_seq_stride | x->out_node_stride) & 7) return DEL_EINVAL;
    if (x->batch < 1 || x->batch > 65535 || x->max_nodes < 1 || x->max_nodes > 64) return DEL_EINVAL;
    if (x->n_heads < 1 || x->n_heads % a.kv.nkv || x->n_heads / a.kv.nkv > 1024 || x->layer < 1 || x->layer > a.kv.L) return DEL_EINVAL;
    if (x->table_cols < 1 || x->table_cols > (INT32_MAX - 1024) / 16 || x->table_stride < 0 || x->max_len < 0) return DEL_EINVAL;
    if (!(x->scale >= 0.f && x->scale * LOG2E < INFINITY)) return DEL_EINVAL;      // (the scores are powers of two)
    const int64_t group = x->n_heads / a.kv.nkv, tiles = (x->max_nodes * group + 15) / 16;
    if (tiles * a.kv.nkv > 65535) return DEL_EINVAL;
    a.q = (const bf16 *)x->q; a.out = (bf16 *)x->out; a.out_lo = (bf16 *)x->out_lo;
    a.table = x->page_table; a.lens = x->lens; a.nodes = x->nodes; a.mask = x->mask;
    a.q_seq = x->q_seq_stride; a.q_node = x->q_node_stride; a.o_seq = x->out_seq_stride; a.o_node = x->out_node_stride;
    a.max_nodes = x->max_nodes; a.nh = x->n_heads; a.layer = x->layer; a.cols = x->table_cols; a.stride = x->table_stride;
    a.scale = (x->scale > 0.f ? x->scale : 1.f / sqrtf((float)a.kv.hd)) * LOG2E;
    a.err = x->error;
    const int len = x->max_len ? (x->max_len < x->table_cols * 16 ? x->max_len : x->table_cols * 16) : x->table_cols * 16;
    return launch_tree_attention(a, x->batch, len, (cudaStream_t)cuda_stream, false) == cudaSuccess ? DEL_OK : DEL_ECUDA;
}
