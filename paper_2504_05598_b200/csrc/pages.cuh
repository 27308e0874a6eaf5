// Device view of a paged cache handed to the context-free operators (del_pages), and the launch helper they share.
#pragma once

#include <atomic>

#include "../../include/del.h"
#include "kernels.h"

// keys [page][layer][kv head][16 tokens][hd], values [page][layer][kv head][hd][16 tokens]
struct PageView {
    bf16 *k, *v;
    int32_t n_pages, L, nkv, hd;
    __host__ __device__ size_t head_elems() const { return (size_t)16 * hd; }                 // of one (page, layer, head)
    __host__ __device__ size_t page_elems() const { return (size_t)L * nkv * 16 * hd; }
    __host__ __device__ bool holds(int page) const { return (unsigned)page < (unsigned)n_pages; }
};

// false: not a cache these operators take
inline bool page_view(const del_pages *kv, PageView *v) {
    if (!kv || !kv->k_pages || !kv->v_pages) return false;
    if (((uintptr_t)kv->k_pages | (uintptr_t)kv->v_pages) & 15) return false;
    if (kv->n_pages < 1 || kv->n_layers < 1 || kv->n_kv_heads < 1 || (kv->head_dim != 64 && kv->head_dim != 128)) return false;
    if ((int64_t)kv->n_layers * kv->n_kv_heads > (1 << 20)) return false;
    *v = PageView{(bf16 *)kv->k_pages, (bf16 *)kv->v_pages, kv->n_pages, kv->n_layers, kv->n_kv_heads, kv->head_dim};
    return true;
}

// del_kv_compact behind its checks (kv_pages.cu)
cudaError_t launch_kv_compact(const PageView &kv, const del_compact &x, cudaStream_t st);

// SMs of the current device (0: the query failed)
inline int current_sms() {
    static std::atomic<int> n[DEL_MAX_DEVICES] = {};
    int dev = 0;
    if (cudaGetDevice(&dev) != cudaSuccess) return 0;
    int sms = dev >= 0 && dev < DEL_MAX_DEVICES ? n[dev].load(std::memory_order_relaxed) : 0;
    if (sms) return sms;
    if (cudaDeviceGetAttribute(&sms, cudaDevAttrMultiProcessorCount, dev) != cudaSuccess) return 0;
    if (dev >= 0 && dev < DEL_MAX_DEVICES) n[dev].store(sms, std::memory_order_relaxed);
    return sms;
}

// A launch of these operators: clusters of cluster_x CTAs, and programmatic dependent launch, so that the launch itself runs beside
// the kernel before it (0.3 to 0.6 us of a small call, 1 to 2 us of a large one).  Every kernel waits (pdl_wait) before it touches
// global memory, and lets the next one start (pdl_launch) only after that, so that a kernel that runs beside this one finds the work of
// all kernels before this one done.  A kernel that writes pages never lets the next one start before its end: the decode attention reads
// committed pages before it waits.
template <typename K, typename... A>
inline cudaError_t launch_cluster(K kern, dim3 grid, int threads, size_t smem, int cluster_x, cudaStream_t st, const A &...args) {
    cudaLaunchConfig_t cfg = {};
    cfg.gridDim = grid;
    cfg.blockDim = dim3(threads);
    cfg.dynamicSmemBytes = smem;
    cfg.stream = st;
    cudaLaunchAttribute at[2];
    at[0].id = cudaLaunchAttributeProgrammaticStreamSerialization;
    at[0].val.programmaticStreamSerializationAllowed = 1;
    at[1].id = cudaLaunchAttributeClusterDimension;
    at[1].val.clusterDim.x = cluster_x;
    at[1].val.clusterDim.y = at[1].val.clusterDim.z = 1;
    cfg.attrs = at;
    cfg.numAttrs = cluster_x > 1 ? 2 : 1;
    return cudaLaunchKernelEx(&cfg, kern, args...);
}

// How many clusters of `cluster_x` CTAs (1..16) of a kernel a device keeps resident, asked once per device and size; one object per
// kernel.  A launch of more runs in waves: of clusters of 8 with one CTA per SM, B200 holds 15.  (Several threads may ask at once, and
// write the same values.)
struct ClusterRoom {
    std::atomic<int> n[DEL_MAX_DEVICES][17] = {};
    std::atomic<bool> wide[DEL_MAX_DEVICES] = {};       // clusters of more than 8 are allowed for the kernel
    template <typename K> int of(K kern, int threads, size_t smem, int cluster_x, int dev) {
        int got = n[dev][cluster_x].load(std::memory_order_acquire);
        if (got) return got;
        if (cluster_x > 8 && !wide[dev].load(std::memory_order_acquire)) {
            if (cudaFuncSetAttribute(kern, cudaFuncAttributeNonPortableClusterSizeAllowed, 1) != cudaSuccess) {
                cudaGetLastError();
                return 0;
            }
            wide[dev].store(true, std::memory_order_release);
        }
        cudaLaunchConfig_t cfg = {};
        cfg.gridDim = dim3(cluster_x);
        cfg.blockDim = dim3(threads);
        cfg.dynamicSmemBytes = smem;
        cudaLaunchAttribute at[1];
        at[0].id = cudaLaunchAttributeClusterDimension;
        at[0].val.clusterDim.x = cluster_x;
        at[0].val.clusterDim.y = at[0].val.clusterDim.z = 1;
        cfg.attrs = at;
        cfg.numAttrs = 1;
        if (cudaOccupancyMaxActiveClusters(&got, kern, &cfg) != cudaSuccess) {
            cudaGetLastError();
            return 0;
        }
        n[dev][cluster_x].store(got, std::memory_order_release);
        return got;
    }
    // Cluster size (1: none) for `units` clusters with `steps` steps of work each: of those sizes whose clusters are all resident
    // together the one with the fewest steps per CTA, of equal ones the smallest.  Beyond 8 it pays where steps are many (one sequence of 30 000
    // positions, 8B shape: 10 CTAs per kv head 36.8 us, 8 CTAs 42.4; 1B shape 16 CTAs 22.9, 8 CTAs 35.3).
    template <typename K> int best(K kern, int threads, size_t smem, int64_t units, int steps) {
        int dev = 0;
        if (cudaGetDevice(&dev) != cudaSuccess || dev < 0 || dev >= DEL_MAX_DEVICES) return 1;
        for (int c = steps < 16 ? steps : 16; c > 1; --c)
            if (units <= of(kern, threads, smem, c, dev)) {
                const int each = (steps + c - 1) / c, least = (steps + each - 1) / each;
                // (3 are slower than 4 or as fast: 8B shape, 16 nodes behind 500 positions 8.2 / 7.5 us, behind 700 8.3 / 8.0, 2 x 8 nodes
                // behind 700 8.2 / 7.9, 3 x 4 nodes 7.9 / 7.4; 120 other calls of both forms, 300 to 4000 positions, within 3 %)
                return least == 3 && c > 3 ? 4 : least;
            }
        return 1;
    }
};
