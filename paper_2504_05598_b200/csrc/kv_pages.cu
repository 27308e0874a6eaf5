// Pages of the cache moved about: positions compacted (del_kv_compact), rows that share pages forked, reordered and given up
// (del_kv_fork).  Nothing is computed: both are bound by the bytes they read and write once.
#include <cstring>

#include "pages.cuh"

namespace {

// ---------------------------------------------------------------- compaction
//
// One CTA moves all positions of one (row, layer, kv head), a warp a destination page at a time, in rounds: every warp reads what its
// page gets into registers, barrier, then out.  With src_pos ascending and never behind its destination, a page written in this round
// holds no source of a later page, and the sources that earlier pages had in it have been read: in-place moves need no second buffer.
// Moves between two tables have no order: there a row's pages are spread over further CTAs (about six per SM, which evens out what
// two or three large ones per SM leave idle, and fills the GPU at all where layers x kv heads x rows are few).
//
// A key is a row of hd values: 16-byte copies.  Values lie transposed, 16 tokens in 32 bytes: the source pages' blocks are copied whole
// into shared memory, a lane picks the tokens of its dimensions in the order of their destinations and writes 32-byte rows (two bytes at a
// time where a destination page is only partly written).  So values are read by whole source pages: of contexts kept by halves, 5
// bytes move where 4 would do.  The copies are asynchronous and one round ahead, page ids two rounds, positions three: a round would
// otherwise wait for three to five round trips to memory in turn (2 x 4 003 of 8 001 positions, 1B shape: 165 us that way, 126 now:
// 3900 GB/s of moved bytes, 4900 with the rest of the value pages).
constexpr int CP_WARPS = 4, CP_RUNS = 2, CP_SPARSE = 4;      // source pages of a destination page that are staged, the next ones are loaded directly; with
                                                             // more than CP_SPARSE, each token's values are loaded by themselves

struct CompactArgs {
    PageView kv;
    del_compact c;
};

// 16-bit element `slot` of a 32-byte row
__device__ __forceinline__ uint32_t pick(const uint4 (&r)[2], int slot) {
    const bool h = slot & 8, w2 = slot & 4, w1 = slot & 2;
    const uint32_t a = h ? r[1].x : r[0].x, b = h ? r[1].y : r[0].y, c = h ? r[1].z : r[0].z, d = h ? r[1].w : r[0].w;
    const uint32_t e = w2 ? c : a, f = w2 ? d : b, g = w1 ? f : e;
    return slot & 1 ? g >> 16 : g & 0xffffu;
}

template <int HD> struct Compact {
    static constexpr int K_BYTES = 16 * HD * 2, V_BYTES = HD * 32, STAGE = K_BYTES + CP_RUNS * V_BYTES, WARP = 2 * STAGE;      // a warp's page of a round; two rounds
};

template <int HD>
__global__ void __launch_bounds__(CP_WARPS * 32, 4) compact_kernel(const CompactArgs a) {
    using C = Compact<HD>;
    extern __shared__ __align__(16) unsigned char smem[];
    constexpr int DPL = HD / 32;                                // dimensions per lane
    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31, n_warps = blockDim.x >> 5, b = blockIdx.y;
    pdl_wait();
    const int n = min(max(a.c.counts[b], 0), a.c.max_count);
    const int64_t start = a.c.dst_start[b], first_page = start >= 0 ? start >> 4 : -((-start + 15) >> 4);
    const int64_t all_pages = n > 0 ? ((start + n - 1) >> 4) - first_page + 1 : 0;
    const int64_t per_part = (all_pages + gridDim.z - 1) / gridDim.z, p_first = per_part * blockIdx.z, n_pages = min(all_pages, p_first + per_part);
    const size_t head = (size_t)blockIdx.x * a.kv.head_elems(), page_elems = a.kv.page_elems();
    // lane j < 16 looks after slot j of the warp's destination page
    auto position = [&](int64_t p0) -> int {                     // source position of the lane's slot, -1: none
        const int64_t dp = first_page + p0 + warp, i = dp * 16 + lane - start;
        return p0 + warp < n_pages && dp >= 0 && dp < a.c.dst_cols && lane < 16 && i >= 0 && i < n ? a.c.src_pos[(size_t)b * a.c.pos_stride + i] : -1;
    };
    struct From { int src, dst, slot; uint32_t moved, runs; };   // source page of the lane's slot, destination page; slots that are written, that begin a source page
    auto ids = [&](int64_t p0, int sp, From &f) {
        const int64_t dp = first_page + p0 + warp;
        f.dst = p0 + warp < n_pages && dp >= 0 && dp < a.c.dst_cols ? a.c.dst_table[(size_t)b * a.c.dst_stride + dp] : -1;
        f.src = sp >= 0 && sp < (int64_t)a.c.src_cols * 16 ? a.c.src_table[(size_t)b * a.c.src_stride + (sp >> 4)] : -1;
        f.slot = sp & 15;
    };
    unsigned char *mine = smem + warp * C::WARP;
    auto fetch = [&](From &f, int stage) {                       // requests the round's keys and values
        if (!a.kv.holds(f.dst)) f.dst = -1;
        if (f.dst < 0 || !a.kv.holds(f.src)) f.src = -1;
        f.moved = __ballot_sync(0xffffffffu, f.src >= 0);
        const int before = __shfl_up_sync(0xffffffffu, f.src, 1);
        f.runs = __ballot_sync(0xffffffffu, lane < 16 && f.src >= 0 && (lane == 0 || f.src != before));
        unsigned char *ks = mine + stage * C::STAGE, *vs = ks + C::K_BYTES;
        if (f.moved) {
#pragma unroll
            for (int v = 0; v < C::K_BYTES / 512; ++v) {
                const int piece = v * 32 + lane, j = piece / (HD / 8), c = piece % (HD / 8) * 8;
                const int pg = __shfl_sync(0xffffffffu, f.src, j), sl = __shfl_sync(0xffffffffu, f.slot, j);
                if (pg >= 0) cp_async16(ks + piece * 16, a.kv.k + (size_t)pg * page_elems + head + sl * HD + c, true);
            }
            uint32_t left = f.runs;
            for (int r = 0; r < CP_RUNS && left && __popc(f.runs) <= CP_SPARSE; ++r, left &= left - 1) {
                const int pg = __shfl_sync(0xffffffffu, f.src, __ffs(left) - 1);
                const bf16 *v = a.kv.v + (size_t)pg * page_elems + head;
#pragma unroll
                for (int i = 0; i < C::V_BYTES / 512; ++i) cp_async16(vs + r * C::V_BYTES + (i * 32 + lane) * 16, v + (i * 32 + lane) * 8, true);
            }
        }
        cp_async_commit();
    };
    From cur, nxt;
    int pos1 = position(p_first), pos2 = position(p_first + n_warps);
    ids(p_first, pos1, nxt);
    pos1 = pos2;
    pos2 = position(p_first + 2 * n_warps);
    fetch(nxt, 0);
    cur = nxt;
    ids(p_first + n_warps, pos1, nxt);
    int stage = 0;
    for (int64_t p0 = p_first; p0 < n_pages; p0 += n_warps, stage ^= 1) {
        fetch(nxt, stage ^ 1);                                    // (behind the last round: nothing)
        From later;
        ids(p0 + 2 * n_warps, pos2, later);
        pos2 = position(p0 + 3 * n_warps);
        cp_async_wait<1>();
        __syncwarp();
        const unsigned char *ks = mine + stage * C::STAGE, *vs = ks + C::K_BYTES;
        uint32_t vals[DPL][8];
        if (__popc(cur.runs) > CP_SPARSE) {
            const uint16_t *v = reinterpret_cast<const uint16_t *>(a.kv.v) + head + (size_t)lane * 16;
#pragma unroll
            for (int j = 0; j < 16; ++j) {
                const int pg = __shfl_sync(0xffffffffu, cur.src, j), sl = __shfl_sync(0xffffffffu, cur.slot, j);
#pragma unroll
                for (int d = 0; d < DPL; ++d) {
                    const uint32_t x = pg >= 0 ? v[(size_t)pg * page_elems + d * 512 + sl] : 0u;
                    vals[d][j >> 1] = j & 1 ? vals[d][j >> 1] | (x << 16) : x;
                }
            }
        } else if (cur.moved) {
            uint4 rows[DPL][2];
            int run = -1;
#pragma unroll
            for (int j = 0; j < 16; ++j) {
                if ((cur.runs >> j) & 1) {
                    ++run;
                    if (run < CP_RUNS) {
#pragma unroll
                        for (int d = 0; d < DPL; ++d) {
                            const uint4 *r = reinterpret_cast<const uint4 *>(vs + run * C::V_BYTES + (lane + d * 32) * 32);
                            rows[d][0] = r[0];
                            rows[d][1] = r[1];
                        }
                    } else {
                        const bf16 *v = a.kv.v + (size_t)__shfl_sync(0xffffffffu, cur.src, j) * page_elems + head + (size_t)lane * 16;
#pragma unroll
                        for (int d = 0; d < DPL; ++d) {
                            rows[d][0] = *reinterpret_cast<const uint4 *>(v + d * 512);
                            rows[d][1] = *reinterpret_cast<const uint4 *>(v + d * 512 + 8);
                        }
                    }
                }
                const int sl = __shfl_sync(0xffffffffu, cur.slot, j);
#pragma unroll
                for (int d = 0; d < DPL; ++d) {
                    const uint32_t x = pick(rows[d], sl);         // (of a slot that stays: never written)
                    vals[d][j >> 1] = j & 1 ? vals[d][j >> 1] | (x << 16) : x;
                }
            }
        }
        __syncthreads();                                          // every page of the round has been read
        if (cur.moved) {
            bf16 *kd = a.kv.k + (size_t)cur.dst * page_elems + head, *vd = a.kv.v + (size_t)cur.dst * page_elems + head + (size_t)lane * 16;
#pragma unroll
            for (int v = 0; v < C::K_BYTES / 512; ++v) {
                const int piece = v * 32 + lane;
                if ((cur.moved >> (piece / (HD / 8))) & 1) *reinterpret_cast<uint4 *>(kd + piece * 8) = *reinterpret_cast<const uint4 *>(ks + piece * 16);
            }
            if (cur.moved == 0xffffu) {
#pragma unroll
                for (int d = 0; d < DPL; ++d) {
                    // a lane pair swaps halves, so that each store writes whole 32-byte rows: first the even lane's, then the odd one's
                    uint32_t *v = vals[d];
#pragma unroll
                    for (int i = 0; i < 4; ++i) {
                        const uint32_t give = lane & 1 ? v[i] : v[4 + i], got = __shfl_xor_sync(0xffffffffu, give, 1);
                        if (lane & 1) v[i] = got;
                        else v[4 + i] = got;
                    }
                    bf16 *even = vd - (lane & 1) * 16 + (lane & 1) * 8 + d * 512;
                    *reinterpret_cast<uint4 *>(even) = make_uint4(v[0], v[1], v[2], v[3]);
                    *reinterpret_cast<uint4 *>(even + 16) = make_uint4(v[4], v[5], v[6], v[7]);
                }
            } else {
#pragma unroll
                for (int j = 0; j < 16; ++j)
                    if ((cur.moved >> j) & 1)
#pragma unroll
                        for (int d = 0; d < DPL; ++d)
                            reinterpret_cast<uint16_t *>(vd + d * 512)[j] = (uint16_t)(j & 1 ? vals[d][j >> 1] >> 16 : vals[d][j >> 1]);
            }
        }
        // (The next rounds' sources, some of them read already, lie behind this round's destinations, or in pages that are not
        // written: no second barrier.)
        __syncwarp();                                             // the stage may be filled again
        cur = nxt;
        nxt = later;
    }
}

// The same for a few pages, one round of one part (accepted paths): nothing to pipeline, and the tokens of a page come from several
// others.  A lane loads its dimensions' values of each token by themselves, all on their way together (4 paths of 5, 8B shape:
// 6.5 to 7.3 us; through staged pages 14.6).
template <int HD>
__global__ void __launch_bounds__(CP_WARPS * 32, 4) compact_few_kernel(const CompactArgs a) {
    constexpr int KV = HD / 16, DPL = HD / 32;                  // 16-byte pieces of 16 keys, dimensions, per lane
    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31, b = blockIdx.y;
    pdl_wait();
    const int n = min(max(a.c.counts[b], 0), a.c.max_count);
    const int64_t start = a.c.dst_start[b], dp = (start >= 0 ? start >> 4 : -((-start + 15) >> 4)) + warp, i = dp * 16 + lane - start;
    const size_t head = (size_t)blockIdx.x * a.kv.head_elems(), page_elems = a.kv.page_elems();
    int dst = -1, src = -1, slot = 0;
    if (dp >= 0 && dp < a.c.dst_cols && dp * 16 < start + n) {
        const int sp = lane < 16 && i >= 0 && i < n ? a.c.src_pos[(size_t)b * a.c.pos_stride + i] : -1;
        dst = a.c.dst_table[(size_t)b * a.c.dst_stride + dp];
        if (sp >= 0 && sp < (int64_t)a.c.src_cols * 16) {
            src = a.c.src_table[(size_t)b * a.c.src_stride + (sp >> 4)];
            slot = sp & 15;
        }
        if (!a.kv.holds(dst) || !a.kv.holds(src)) src = -1;
    }
    const uint32_t moved = __ballot_sync(0xffffffffu, src >= 0);
    uint4 keys[KV];
    uint16_t vals[16][DPL];
    if (moved) {
#pragma unroll
        for (int v = 0; v < KV; ++v) {
            const int piece = v * 32 + lane, j = piece / (HD / 8), c = piece % (HD / 8) * 8;
            const int pg = __shfl_sync(0xffffffffu, src, j), sl = __shfl_sync(0xffffffffu, slot, j);
            if (pg >= 0) keys[v] = *reinterpret_cast<const uint4 *>(a.kv.k + (size_t)pg * page_elems + head + sl * HD + c);
        }
#pragma unroll
        for (int j = 0; j < 16; ++j) {
            const int pg = __shfl_sync(0xffffffffu, src, j), sl = __shfl_sync(0xffffffffu, slot, j);
            const uint16_t *v = reinterpret_cast<const uint16_t *>(a.kv.v) + (size_t)max(pg, 0) * page_elems + head + (size_t)lane * 16 + sl;
            if (pg >= 0)
#pragma unroll
                for (int d = 0; d < DPL; ++d) vals[j][d] = v[d * 512];
        }
    }
    __syncthreads();                                              // every page has been read
    if (!moved) return;
    bf16 *kd = a.kv.k + (size_t)dst * page_elems + head;
    uint16_t *vd = reinterpret_cast<uint16_t *>(a.kv.v) + (size_t)dst * page_elems + head + (size_t)lane * 16;
#pragma unroll
    for (int v = 0; v < KV; ++v) {
        const int piece = v * 32 + lane;
        if ((moved >> (piece / (HD / 8))) & 1) *reinterpret_cast<uint4 *>(kd + piece * 8) = keys[v];
    }
#pragma unroll
    for (int j = 0; j < 16; ++j)
        if ((moved >> j) & 1)
#pragma unroll
            for (int d = 0; d < DPL; ++d) vd[d * 512 + j] = vals[j][d];
}

// ---------------------------------------------------------------- forks
//
// One launch.  Which row gets which pages is a few hundred integers: every CTA works it out for itself in shared memory, and no CTA
// waits for another.  Then the CTAs share the tables' rows and the pieces of the pages to copy; the last one lists the free pages.
// 16 x 4 rows of the 8B shape: 15.9 us, 5000 GB/s; 1 x 4 rows of the 1B shape: 4.9 us, all latency.
constexpr int FK_THREADS = 1024, FK_ROWS = 1024;
constexpr int FK_MAX_FREE = 1 << 20;          // pages of which the used ones are marked in shared memory (128 KB of bits)
constexpr int PIECE = 16384;                  // bytes of a page that a CTA copies at a time

struct ForkArgs {
    PageView kv;
    del_fork_args f;
};

__device__ __forceinline__ int block_scan(int v, int *warp_sums, int &total) {       // exclusive, over all threads
    const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
    int x = v;
#pragma unroll
    for (int o = 1; o < 32; o <<= 1) {
        const int y = __shfl_up_sync(0xffffffffu, x, o);
        if (lane >= o) x += y;
    }
    __syncthreads();
    if (lane == 31) warp_sums[warp] = x;
    __syncthreads();
    if (warp == 0) {
        int w = warp_sums[lane];
#pragma unroll
        for (int o = 1; o < 32; o <<= 1) {
            const int y = __shfl_up_sync(0xffffffffu, w, o);
            if (lane >= o) w += y;
        }
        warp_sums[lane] = w;
    }
    __syncthreads();
    total = warp_sums[31];
    return x - v + (warp ? warp_sums[warp - 1] : 0);
}

__global__ void __launch_bounds__(FK_THREADS) fork_kernel(const ForkArgs a) {
    extern __shared__ uint32_t used_bits[];
    __shared__ int first[FK_ROWS], base[FK_ROWS], copy_src[FK_ROWS], copy_dst[FK_ROWS], warp_sums[32];
    const del_fork_args &f = a.f;
    const int r = threadIdx.x, n_cta = gridDim.x;
    first[r] = INT32_MAX;
    __syncthreads();
    pdl_wait();
    int parent = -1, len = 0;
    if (r < f.n_new) {
        parent = f.parents[r];
        if (parent < 0 || parent >= f.n_old) parent = -1;
        else {
            len = min(max(f.lens[parent], 0), (int)min((int64_t)f.old_cols, (int64_t)f.new_cols) * 16);
            atomicMin(&first[parent], r);
        }
    }
    __syncthreads();
    const int full = len >> 4, part = (len & 15) != 0;
    const bool copies = parent >= 0 && part && first[parent] != r;
    const int held = full + part;
    const int wanted = parent < 0 ? 0 : max(held, (int)min((int64_t)f.new_cols, ((int64_t)len + f.room + 15) >> 4));
    const int fresh = (copies ? 1 : 0) + wanted - held;
    const int n_spare = min(max(f.n_spare[0], 0), f.spare_cap);
    int total, n_copies;
    const int b0 = block_scan(fresh, warp_sums, total);
    base[r] = b0;
    int src = -1, dst = -1, missing = 0;
    if (copies) {
        src = f.table[(size_t)parent * f.old_stride + full];
        dst = b0 < n_spare ? f.spare[b0] : -1;
        if (!a.kv.holds(src) || !a.kv.holds(dst)) dst = -1;
    }
    const int slot = block_scan(dst >= 0 ? 1 : 0, warp_sums, n_copies);
    if (dst >= 0) { copy_src[slot] = src; copy_dst[slot] = dst; }
    // a row per CTA and turn: its table
    __shared__ int row_parent[FK_ROWS], row_len[FK_ROWS], row_wanted[FK_ROWS], row_copy[FK_ROWS];     // row_copy: page, -1 missing, -2 none
    row_parent[r] = parent;
    row_len[r] = len;
    row_wanted[r] = wanted;
    row_copy[r] = copies ? dst : -2;
    __syncthreads();
    auto entry = [&](int b, int p) -> int {                    // page p of new row b
        const int ln = row_len[b], fl = ln >> 4, pt = (ln & 15) != 0;
        if (p < fl || (p == fl && pt && row_copy[b] == -2)) return f.table[(size_t)row_parent[b] * f.old_stride + p];
        if (p == fl && pt) return row_copy[b];
        const int at = base[b] + p - (fl + pt) + (row_copy[b] != -2 ? 1 : 0);
        const int pg = at < n_spare ? f.spare[at] : -1;
        return a.kv.holds(pg) ? pg : -1;
    };
    for (int b = blockIdx.x; b < f.n_new; b += n_cta) {
        for (int p = threadIdx.x; p < row_wanted[b]; p += FK_THREADS) f.new_table[(size_t)b * f.new_stride + p] = entry(b, p);
        if (threadIdx.x == 0) f.new_lens[b] = row_len[b];
    }
    if (blockIdx.x == n_cta - 1) {
        // how many entries are missing, and which pages nobody holds
        for (int p = held; p < wanted; ++p) missing += entry(r, p) < 0;
        missing += copies && dst < 0;
        int n_missing, before = 0;
        block_scan(missing, warp_sums, n_missing);
        if (f.free_pages) {
            const int words = (a.kv.n_pages + 31) >> 5;
            for (int w = threadIdx.x; w < words; w += FK_THREADS) used_bits[w] = 0;
            __syncthreads();
            for (int b = threadIdx.x >> 5; b < f.n_new; b += FK_THREADS / 32)       // a row per warp
                for (int p = threadIdx.x & 31; p < row_wanted[b]; p += 32) {
                    const int pg = entry(b, p);
                    if (a.kv.holds(pg)) atomicOr(&used_bits[pg >> 5], 1u << (pg & 31));
                }
            __syncthreads();
            for (int w0 = 0; w0 < words; w0 += FK_THREADS) {
                const int w = w0 + threadIdx.x;
                uint32_t bits = w < words ? ~used_bits[w] : 0u;
                if (w == words - 1 && (a.kv.n_pages & 31)) bits &= (1u << (a.kv.n_pages & 31)) - 1;
                int n;
                int at = before + block_scan(__popc(bits), warp_sums, n);
                before += n;
                while (bits) {
                    f.free_pages[at++] = w * 32 + __ffs(bits) - 1;
                    bits &= bits - 1;
                }
            }
        }
        if (threadIdx.x == 0) { f.counts[0] = before; f.counts[1] = n_missing; }
    }
    // pieces of the pages to copy, keys and values: large ones, four loads of a thread in flight, where there are enough of them
    const size_t page_bytes = a.kv.page_elems() * sizeof(bf16);
    const bool large = (int64_t)n_copies * 2 * (int64_t)(page_bytes / (4 * PIECE)) >= n_cta;
    const size_t piece = large ? 4 * PIECE : PIECE;
    const int per_page = (int)((page_bytes + piece - 1) / piece);
    const int64_t items = (int64_t)n_copies * per_page * 2;
    for (int64_t it = blockIdx.x; it < items; it += n_cta) {
        const int c = (int)(it / (per_page * 2)), q = (int)(it % (per_page * 2));
        char *pool = reinterpret_cast<char *>(q < per_page ? a.kv.k : a.kv.v);
        const size_t off = (size_t)(q < per_page ? q : q - per_page) * piece;
        const uint4 *s = reinterpret_cast<const uint4 *>(pool + copy_src[c] * page_bytes + off);
        uint4 *d = reinterpret_cast<uint4 *>(pool + copy_dst[c] * page_bytes + off);
        const int n = (int)(min(piece, page_bytes - off) / 16);
        if (n == 4 * FK_THREADS) {
            uint4 v[4];
#pragma unroll
            for (int e = 0; e < 4; ++e) v[e] = __ldcs(s + e * FK_THREADS + threadIdx.x);
#pragma unroll
            for (int e = 0; e < 4; ++e) __stcs(d + e * FK_THREADS + threadIdx.x, v[e]);
        } else {
            for (int e = threadIdx.x; e < n; e += FK_THREADS) d[e] = s[e];
        }
    }
}

bool overlap(const void *a, size_t na, const void *b, size_t nb) {
    const uintptr_t x = (uintptr_t)a, y = (uintptr_t)b;
    return x < y + nb && y < x + na;
}

}  // namespace

cudaError_t launch_kv_compact(const PageView &kv, const del_compact &x, cudaStream_t st) {
    CompactArgs a{kv, x};
    // a warp for each destination page of a round; positions of up to max_count / 16 + 2 pages
    const int n_sms = current_sms(), pages = (x.max_count + 14) / 16 + 1, warps = pages < CP_WARPS ? pages : CP_WARPS;
    if (!n_sms) return cudaErrorInvalidDevice;
    const int64_t units = (int64_t)a.kv.L * a.kv.nkv * x.batch, rounds = (pages + warps - 1) / warps;
    int64_t parts = 1;
    if (x.src_table != x.dst_table) {
        parts = (6 * n_sms + units - 1) / units;
        parts = parts < rounds ? parts : rounds;
    }
    const dim3 grid(a.kv.L * a.kv.nkv, x.batch, (unsigned)parts);
    if (pages <= warps) {
        return a.kv.hd == 128 ? launch_cluster(compact_few_kernel<128>, grid, warps * 32, 0, 1, st, a) : launch_cluster(compact_few_kernel<64>, grid, warps * 32, 0, 1, st, a);
    }
    static SmemAttrOnce attr128, attr64;
    const cudaError_t e = a.kv.hd == 128 ? attr128.set(compact_kernel<128>, CP_WARPS * Compact<128>::WARP) : attr64.set(compact_kernel<64>, CP_WARPS * Compact<64>::WARP);
    if (e != cudaSuccess) return e;
    return a.kv.hd == 128 ? launch_cluster(compact_kernel<128>, grid, CP_WARPS * 32, CP_WARPS * Compact<128>::WARP, 1, st, a)
                          : launch_cluster(compact_kernel<64>, grid, CP_WARPS * 32, CP_WARPS * Compact<64>::WARP, 1, st, a);
}

extern "C" int del_kv_compact(const del_pages *kv, const del_compact *x, void *cuda_stream) {
    PageView view;
    if (!x || !page_view(kv, &view)) return DEL_EINVAL;
    if (!x->src_table || !x->dst_table || !x->src_pos || !x->counts || !x->dst_start) return DEL_EINVAL;
    if (((uintptr_t)x->src_table | (uintptr_t)x->dst_table | (uintptr_t)x->src_pos | (uintptr_t)x->counts | (uintptr_t)x->dst_start) & 3) return DEL_EINVAL;
    if (x->batch < 1 || x->batch > 65535 || x->max_count < 1 || x->max_count > (1 << 30) || x->src_cols < 1 || x->dst_cols < 1) return DEL_EINVAL;
    if (x->src_stride < 0 || x->dst_stride < 0 || x->pos_stride < 0) return DEL_EINVAL;
    return launch_kv_compact(view, *x, (cudaStream_t)cuda_stream) == cudaSuccess ? DEL_OK : DEL_ECUDA;
}

extern "C" int del_kv_fork(const del_pages *kv, const del_fork_args *x, void *cuda_stream) {
    ForkArgs a;
    if (!x || !page_view(kv, &a.kv)) return DEL_EINVAL;
    if (!x->table || !x->lens || !x->parents || (!x->spare && x->spare_cap) || !x->n_spare || !x->new_table || !x->new_lens || !x->counts) return DEL_EINVAL;
    if (((uintptr_t)x->table | (uintptr_t)x->lens | (uintptr_t)x->parents | (uintptr_t)x->spare | (uintptr_t)x->n_spare | (uintptr_t)x->new_table |
         (uintptr_t)x->new_lens | (uintptr_t)x->free_pages | (uintptr_t)x->counts) & 3)
        return DEL_EINVAL;
    if (x->n_old < 1 || x->n_old > FK_ROWS || x->n_new < 1 || x->n_new > FK_ROWS) return DEL_EINVAL;
    if (x->old_cols < 1 || x->new_cols < 1 || x->old_cols > INT32_MAX / 16 || x->new_cols > INT32_MAX / 16) return DEL_EINVAL;
    if ((int64_t)x->n_new * x->new_cols > INT32_MAX) return DEL_EINVAL;               // spare pages are counted in 32 bits
    if (x->old_stride < x->old_cols || x->new_stride < x->new_cols || x->spare_cap < 0 || x->room < 0) return DEL_EINVAL;
    if (x->free_pages && a.kv.n_pages > FK_MAX_FREE) return DEL_EINVAL;
    const size_t old_bytes = 4 * ((size_t)(x->n_old - 1) * x->old_stride + x->old_cols), new_bytes = 4 * ((size_t)(x->n_new - 1) * x->new_stride + x->new_cols);
    // nothing is written that is read, or written twice: CTAs may start after others are done
    struct Range { const void *p; size_t n; };
    const Range in[] = {{x->table, old_bytes}, {x->lens, 4 * (size_t)x->n_old}, {x->parents, 4 * (size_t)x->n_new}, {x->spare, 4 * (size_t)x->spare_cap}, {x->n_spare, 4}};
    const Range out[] = {{x->new_table, new_bytes}, {x->new_lens, 4 * (size_t)x->n_new}, {x->counts, 8}, {x->free_pages, x->free_pages ? 4 * (size_t)a.kv.n_pages : 0}};
    for (int i = 0; i < 4; ++i) {
        for (const Range &r : in)
            if (overlap(out[i].p, out[i].n, r.p, r.n)) return DEL_EINVAL;
        for (int j = 0; j < i; ++j)
            if (overlap(out[i].p, out[i].n, out[j].p, out[j].n)) return DEL_EINVAL;
    }
    const int n_sms = current_sms();
    if (!n_sms) return DEL_ECUDA;
    a.f = *x;
    static SmemAttrOnce attr;
    const size_t bits = x->free_pages ? ((size_t)a.kv.n_pages + 31) / 32 * 4 : 0;
    if (attr.set(fork_kernel, FK_MAX_FREE / 8) != cudaSuccess) return DEL_ECUDA;
    return launch_cluster(fork_kernel, dim3(n_sms), FK_THREADS, bits, 1, (cudaStream_t)cuda_stream, a) == cudaSuccess ? DEL_OK : DEL_ECUDA;
}
