// Pages of the cache moved about: positions compacted (del_kv_compact), rows that share pages forked, reordered and given up
// (del_kv_fork).  Nothing is computed: both are bound by the bytes they read and write once.
#include <cstring>

#include "pages.cuh"

namespace {

// ---------------------------------------------------------------- compaction
//
// One CTA moves all positions of one (row, layer, kv head), CHUNK of them at a time in ascending order: sources into shared
// memory, barrier, then out.  A chunk's sources are read before anything of it is written, and with src_pos ascending and never
// behind its destination, no earlier chunk has written what a later one reads: in-place moves need no second buffer.
constexpr int CP_THREADS = 256, CHUNK = 32;

struct CompactArgs {
    PageView kv;
    del_compact c;
};

template <int HD>
__global__ void __launch_bounds__(CP_THREADS) compact_kernel(const CompactArgs a) {
    __shared__ __align__(16) bf16 sk[CHUNK][HD];
    __shared__ bf16 sv[HD][CHUNK + 2];
    __shared__ int64_t src_page[CHUNK], dst_page[CHUNK];      // element offset of the (page, layer, head) block, -1: not moved
    __shared__ int src_slot[CHUNK], dst_slot[CHUNK];
    const int b = blockIdx.y;
    const int n = min(max(a.c.counts[b], 0), a.c.max_count);
    const int start = a.c.dst_start[b];
    const size_t head = (size_t)blockIdx.x * a.kv.head_elems(), page_elems = a.kv.page_elems();
    for (int i0 = 0; i0 < n; i0 += CHUNK) {
        if (threadIdx.x < CHUNK) {
            const int i = i0 + threadIdx.x;
            int64_t s = -1, d = -1;
            if (i < n) {
                const int64_t sp = a.c.src_pos[(size_t)b * a.c.pos_stride + i], dp = (int64_t)start + i;
                if (sp >= 0 && sp < (int64_t)a.c.src_cols * 16 && dp >= 0 && dp < (int64_t)a.c.dst_cols * 16) {
                    const int spg = a.c.src_table[(size_t)b * a.c.src_stride + (sp >> 4)], dpg = a.c.dst_table[(size_t)b * a.c.dst_stride + (dp >> 4)];
                    if (a.kv.holds(spg) && a.kv.holds(dpg)) {
                        s = (int64_t)((size_t)spg * page_elems + head);
                        d = (int64_t)((size_t)dpg * page_elems + head);
                        src_slot[threadIdx.x] = (int)(sp & 15);
                        dst_slot[threadIdx.x] = (int)(dp & 15);
                    }
                }
            }
            src_page[threadIdx.x] = s;
            dst_page[threadIdx.x] = d;
        }
        __syncthreads();
        for (int e = threadIdx.x; e < CHUNK * (HD / 8); e += CP_THREADS) {
            const int i = e / (HD / 8), c = e % (HD / 8) * 8;
            if (src_page[i] >= 0) *reinterpret_cast<uint4 *>(&sk[i][c]) = *reinterpret_cast<const uint4 *>(a.kv.k + src_page[i] + src_slot[i] * HD + c);
        }
        for (int e = threadIdx.x; e < CHUNK * HD; e += CP_THREADS) {
            const int i = e % CHUNK, c = e / CHUNK;
            if (src_page[i] >= 0) sv[c][i] = a.kv.v[src_page[i] + c * 16 + src_slot[i]];
        }
        __syncthreads();
        for (int e = threadIdx.x; e < CHUNK * (HD / 8); e += CP_THREADS) {
            const int i = e / (HD / 8), c = e % (HD / 8) * 8;
            if (dst_page[i] >= 0) *reinterpret_cast<uint4 *>(a.kv.k + dst_page[i] + dst_slot[i] * HD + c) = *reinterpret_cast<const uint4 *>(&sk[i][c]);
        }
        for (int e = threadIdx.x; e < CHUNK * HD; e += CP_THREADS) {
            const int i = e % CHUNK, c = e / CHUNK;
            if (dst_page[i] >= 0) a.kv.v[dst_page[i] + c * 16 + dst_slot[i]] = sv[c][i];
        }
        __syncthreads();
    }
}

// ---------------------------------------------------------------- forks
//
// One launch.  Which row gets which pages is a few hundred integers: every CTA works it out for itself in shared memory, and no CTA
// waits for another.  Then the CTAs share the tables' rows and the pieces of the pages to copy; the last one lists the free pages.
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
            for (int b = 0; b < f.n_new; ++b)
                for (int p = threadIdx.x; p < row_wanted[b]; p += FK_THREADS) {
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
    // pieces of the pages to copy, keys and values
    const size_t page_bytes = a.kv.page_elems() * sizeof(bf16);
    const int per_page = (int)((page_bytes + PIECE - 1) / PIECE);
    const int64_t items = (int64_t)n_copies * per_page * 2;
    for (int64_t it = blockIdx.x; it < items; it += n_cta) {
        const int c = (int)(it / (per_page * 2)), q = (int)(it % (per_page * 2));
        char *pool = reinterpret_cast<char *>(q < per_page ? a.kv.k : a.kv.v);
        const size_t off = (size_t)(q < per_page ? q : q - per_page) * PIECE;
        const uint4 *s = reinterpret_cast<const uint4 *>(pool + copy_src[c] * page_bytes + off);
        uint4 *d = reinterpret_cast<uint4 *>(pool + copy_dst[c] * page_bytes + off);
        const int n = (int)(min((size_t)PIECE, page_bytes - off) / 16);
        for (int e = threadIdx.x; e < n; e += FK_THREADS) d[e] = s[e];
    }
}

bool overlap(const void *a, size_t na, const void *b, size_t nb) {
    const uintptr_t x = (uintptr_t)a, y = (uintptr_t)b;
    return x < y + nb && y < x + na;
}

}  // namespace

extern "C" int del_kv_compact(const del_pages *kv, const del_compact *x, void *cuda_stream) {
    CompactArgs a;
    if (!x || !page_view(kv, &a.kv)) return DEL_EINVAL;
    if (!x->src_table || !x->dst_table || !x->src_pos || !x->counts || !x->dst_start) return DEL_EINVAL;
    if (((uintptr_t)x->src_table | (uintptr_t)x->dst_table | (uintptr_t)x->src_pos | (uintptr_t)x->counts | (uintptr_t)x->dst_start) & 3) return DEL_EINVAL;
    if (x->batch < 1 || x->batch > 65535 || x->max_count < 1 || x->src_cols < 1 || x->dst_cols < 1) return DEL_EINVAL;
    if (x->src_stride < 0 || x->dst_stride < 0 || x->pos_stride < 0) return DEL_EINVAL;
    a.c = *x;
    const dim3 grid(a.kv.L * a.kv.nkv, x->batch);
    cudaStream_t st = (cudaStream_t)cuda_stream;
    if (a.kv.hd == 128) compact_kernel<128><<<grid, CP_THREADS, 0, st>>>(a);
    else compact_kernel<64><<<grid, CP_THREADS, 0, st>>>(a);
    return cudaGetLastError() == cudaSuccess ? DEL_OK : DEL_ECUDA;
}

extern "C" int del_kv_fork(const del_pages *kv, const del_fork_args *x, void *cuda_stream) {
    ForkArgs a;
    if (!x || !page_view(kv, &a.kv)) return DEL_EINVAL;
    if (!x->table || !x->lens || !x->parents || !x->spare || !x->n_spare || !x->new_table || !x->new_lens || !x->counts) return DEL_EINVAL;
    if (((uintptr_t)x->table | (uintptr_t)x->lens | (uintptr_t)x->parents | (uintptr_t)x->spare | (uintptr_t)x->n_spare | (uintptr_t)x->new_table |
         (uintptr_t)x->new_lens | (uintptr_t)x->free_pages | (uintptr_t)x->counts) & 3)
        return DEL_EINVAL;
    if (x->n_old < 1 || x->n_old > FK_ROWS || x->n_new < 1 || x->n_new > FK_ROWS) return DEL_EINVAL;
    if (x->old_cols < 1 || x->new_cols < 1 || x->old_cols > INT32_MAX / 16 || x->new_cols > INT32_MAX / 16) return DEL_EINVAL;
    if (x->old_stride < x->old_cols || x->new_stride < x->new_cols || x->spare_cap < 0 || x->room < 0) return DEL_EINVAL;
    if (x->free_pages && a.kv.n_pages > FK_MAX_FREE) return DEL_EINVAL;
    const size_t old_bytes = 4 * ((size_t)(x->n_old - 1) * x->old_stride + x->old_cols), new_bytes = 4 * ((size_t)(x->n_new - 1) * x->new_stride + x->new_cols);
    if (overlap(x->table, old_bytes, x->new_table, new_bytes) || overlap(x->lens, 4 * (size_t)x->n_old, x->new_lens, 4 * (size_t)x->n_new)) return DEL_EINVAL;
    if (x->free_pages && overlap(x->free_pages, 4 * (size_t)a.kv.n_pages, x->spare, 4 * (size_t)x->spare_cap)) return DEL_EINVAL;
    if (overlap(x->counts, 8, x->n_spare, 4)) return DEL_EINVAL;        // the count is read by CTAs that may start after the last one is done
    const int n_sms = current_sms();
    if (!n_sms) return DEL_ECUDA;
    a.f = *x;
    static SmemAttrOnce attr;
    const size_t bits = x->free_pages ? ((size_t)a.kv.n_pages + 31) / 32 * 4 : 0;
    if (attr.set(fork_kernel, FK_MAX_FREE / 8) != cudaSuccess) return DEL_ECUDA;
    fork_kernel<<<n_sms, FK_THREADS, bits, (cudaStream_t)cuda_stream>>>(a);
    return cudaGetLastError() == cudaSuccess ? DEL_OK : DEL_ECUDA;
}
