// Beam search's selection (del_beam_select): log softmax, scores and the k best of beams x vocabulary in one pass over the logits.
//
// One cluster of CTAs works on one batch item; CTA r owns the same slice of columns of every beam.  Within a beam the score rises
// with the logit, so each CTA keeps, per beam, the k largest logits of its slice (equal ones: the lower token) beside the running
// maximum and sum of exponentials.  Then the CTAs share out the beams: the slices' lists are merged, the log-sum-exp turns logits
// into scores (64 bits: near candidates of different beams are ordered by it); CTA 0 merges the beams' lists.
//
// The k largest of a block of CHUNK logits, which lie in registers: every warp takes the r-th largest of its threads' maxima,
// r = ceil(k / warps); the smallest of these over the warps has at least k logits at or above it and, for logits in no special
// order, few more.  Those are appended to a list and ranked by counting.  Where the list would overflow (sorted logits, say), the
// k largest are taken one by one instead.
#include <cooperative_groups.h>
#include <cuda_fp16.h>
#include <cstring>

#include "pages.cuh"

namespace cg = cooperative_groups;

namespace {

typedef unsigned long long u64;

constexpr int THREADS = 512, NW = THREADS / 32, EPT = 16, CHUNK = THREADS * EPT, MAX_K = 64, MAX_BEAMS = 64, MAX_CLUSTER = 16;
constexpr int LIST = 1024;                 // candidates of a chunk that are ranked by counting
constexpr float LOG2E = 1.4426950408889634f;

struct BeamArgs {
    del_beam b;
    int32_t slice;                         // columns per CTA, a multiple of 8
    int32_t aligned;                       // rows start on 16-byte boundaries
};

// Logits in the order of their value as unsigned numbers; the key of a token puts equal logits in the order of their ids.
// A key is never 0: that stands for no token.
__device__ __forceinline__ uint32_t ordered(float x) {
    const uint32_t b = __float_as_uint(x + 0.f);                  // (-0 becomes +0)
    return b & 0x80000000u ? ~b : b | 0x80000000u;
}
__device__ __forceinline__ float unordered(uint32_t o) { return __uint_as_float(o & 0x80000000u ? o & 0x7fffffffu : ~o); }
__device__ __forceinline__ u64 make_key(float x, int token) { return ((u64)ordered(x) << 32) | (0xffffffffu - (uint32_t)token); }
__device__ __forceinline__ int key_token(u64 key) { return (int)(0xffffffffu - (uint32_t)key); }
__device__ __forceinline__ float key_value(u64 key) { return unordered((uint32_t)(key >> 32)); }

template <typename T> __device__ __forceinline__ float to_f(T v);
template <> __device__ __forceinline__ float to_f<float>(float v) { return v; }
template <> __device__ __forceinline__ float to_f<bf16>(bf16 v) { return __bfloat162float(v); }
template <> __device__ __forceinline__ float to_f<__half>(__half v) { return __half2float(v); }

__device__ __forceinline__ u64 warp_max_u64(u64 v) {
#pragma unroll
    for (int o = 16; o > 0; o >>= 1) {
        const u64 w = __shfl_xor_sync(0xffffffffu, v, o);
        if (w > v) v = w;
    }
    return v;
}

struct Shared {
    u64 list[LIST + MAX_K];
    u64 warp_key[NW];
    float warp_m[NW];
    double warp_s[NW];
    int count;
    float m[MAX_BEAMS];                    // per beam: maximum and sum of exponentials of this CTA's slice
    double s[MAX_BEAMS];
    double fin_score[MAX_BEAMS * MAX_K];   // rank 0: the beams' merged lists
    int32_t fin_token[MAX_BEAMS * MAX_K];
    u64 cand[MAX_BEAMS * MAX_K];           // per beam: this CTA's k largest, descending, 0 behind the last
    u64 gather[MAX_CLUSTER * MAX_K];
};

// the column of element e of this thread in a chunk: vectors of VEC elements, threads side by side
template <int VEC> __device__ __forceinline__ int column(int e) { return ((e / VEC) * THREADS + threadIdx.x) * VEC + e % VEC; }

template <typename T>
__global__ void __launch_bounds__(THREADS) beam_kernel(const BeamArgs a) {
    constexpr int VEC = 16 / sizeof(T);
    extern __shared__ __align__(16) unsigned char smem[];
    Shared &sm = *reinterpret_cast<Shared *>(smem);
    cg::cluster_group cl = cg::this_cluster();
    const int rank = cl.block_rank(), n_ranks = cl.num_blocks();
    const int item = blockIdx.x / n_ranks, beams = a.b.beams, V = a.b.vocab, k = a.b.k;
    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
    const int lo = min((int64_t)rank * a.slice, (int64_t)V), hi = min((int64_t)lo + a.slice, (int64_t)V);

    for (int e = threadIdx.x; e < beams * k; e += THREADS) sm.cand[e] = 0;
    for (int e = threadIdx.x; e < beams; e += THREADS) { sm.m[e] = -INFINITY; sm.s[e] = 0.0; }
    __syncthreads();
    for (int beam = 0; beam < beams; ++beam) {
        const int row = item * beams + beam;
        if (a.b.finished && a.b.finished[row]) continue;
        const T *logits = reinterpret_cast<const T *>(a.b.logits) + row * a.b.row_stride;
        for (int c0 = lo; c0 < hi; c0 += CHUNK) {
            const int n = min(CHUNK, hi - c0);
            float x[EPT];
            if (a.aligned) {
#pragma unroll
                for (int v = 0; v < EPT / VEC; ++v) {
                    const int c = column<VEC>(v * VEC);
                    if (c + VEC <= n) {
                        const uint4 q = ldg_stream16(logits + c0 + c);
                        T t[VEC];
                        memcpy(t, &q, 16);
#pragma unroll
                        for (int e = 0; e < VEC; ++e) x[v * VEC + e] = to_f<T>(t[e]);
                    } else {
#pragma unroll
                        for (int e = 0; e < VEC; ++e) x[v * VEC + e] = c + e < n ? to_f<T>(logits[c0 + c + e]) : -INFINITY;
                    }
                }
            } else {
#pragma unroll
                for (int e = 0; e < EPT; ++e) x[e] = column<VEC>(e) < n ? to_f<T>(logits[c0 + column<VEC>(e)]) : -INFINITY;
            }
            // maximum, sum of exponentials, this thread's best key
            float m = -INFINITY;
            u64 best = 0;
#pragma unroll
            for (int e = 0; e < EPT; ++e) {
                m = fmaxf(m, x[e]);
                if (column<VEC>(e) < n) {
                    const u64 key = make_key(x[e], c0 + column<VEC>(e));
                    if (key > best) best = key;
                }
            }
            const float base = m == -INFINITY ? 0.f : m;
            float s = 0.f;
#pragma unroll
            for (int e = 0; e < EPT; ++e) s += exp2f((x[e] - base) * LOG2E);
            float wm = m;
#pragma unroll
            for (int o = 16; o > 0; o >>= 1) wm = fmaxf(wm, __shfl_xor_sync(0xffffffffu, wm, o));
            double ws = m == -INFINITY ? (double)s : (double)s * (double)exp2f((m - wm) * LOG2E);      // (m = -inf: 0, or no number)
#pragma unroll
            for (int o = 16; o > 0; o >>= 1) ws += __shfl_xor_sync(0xffffffffu, ws, o);
            // the r-th largest thread maximum of the warp, of those warps whose threads all have logits
            const int n_full = min(NW, n / (32 * VEC));
            const int r_th = n_full ? (k + n_full - 1) / n_full : 0;
            u64 mine = best, w = 0;
            for (int r = 0; r < r_th; ++r) {
                w = warp_max_u64(mine);
                if (mine == w) mine = 0;
            }
            if (lane == 0) { sm.warp_key[warp] = w; sm.warp_m[warp] = wm; sm.warp_s[warp] = ws; }
            if (threadIdx.x == 0) sm.count = 0;
            __syncthreads();
            u64 least = 0;                                        // (r_th > 32: fewer than 64 threads' logits, all of them are listed)
            if (n_full && r_th <= 32) {
                least = ~0ull;
                for (int i = 0; i < n_full; ++i) least = min(least, sm.warp_key[i]);
            }
            const u64 kth = sm.cand[beam * k + k - 1];
            if (kth > least) least = kth;
#pragma unroll
            for (int e = 0; e < EPT; ++e)
                if (column<VEC>(e) < n) {
                    const u64 key = make_key(x[e], c0 + column<VEC>(e));
                    if (key >= least) {
                        const int at = atomicAdd(&sm.count, 1);
                        if (at < LIST) sm.list[at] = key;
                    }
                }
            __syncthreads();
            int count = sm.count;
            if (count > LIST) {                                   // (the same in every thread)
                u64 last = ~0ull;
                count = 0;
                for (int i = 0; i < k; ++i) {
                    u64 next = 0;
#pragma unroll
                    for (int e = 0; e < EPT; ++e)
                        if (column<VEC>(e) < n) {
                            const u64 key = make_key(x[e], c0 + column<VEC>(e));
                            if (key < last && key > next) next = key;
                        }
                    next = warp_max_u64(next);
                    __syncthreads();
                    if (lane == 0) sm.warp_key[warp] = next;
                    __syncthreads();
                    for (int j = 0; j < NW; ++j) next = max(next, sm.warp_key[j]);
                    if (next == 0) break;
                    if (threadIdx.x == 0) sm.list[i] = next;
                    last = next;
                    ++count;
                }
                __syncthreads();
            }
            // with what the beam had already; ranked by counting
            for (int i = threadIdx.x; i < k; i += THREADS) sm.list[count + i] = sm.cand[beam * k + i];
            if (threadIdx.x == 0) {
                float M = sm.m[beam];
                for (int i = 0; i < NW; ++i) M = fmaxf(M, sm.warp_m[i]);
                const float b0 = M == -INFINITY ? 0.f : M;
                double S = sm.m[beam] == -INFINITY ? sm.s[beam] : sm.s[beam] * (double)exp2f((sm.m[beam] - b0) * LOG2E);
                for (int i = 0; i < NW; ++i) S += sm.warp_m[i] == -INFINITY ? sm.warp_s[i] : sm.warp_s[i] * (double)exp2f((sm.warp_m[i] - b0) * LOG2E);
                sm.m[beam] = M;
                sm.s[beam] = S;
            }
            __syncthreads();
            const int total = count + k;
            for (int i = threadIdx.x; i < total; i += THREADS) {
                const u64 key = sm.list[i];
                if (key == 0) continue;
                int above = 0;
                for (int j = 0; j < total; ++j) above += sm.list[j] > key;
                if (above < k) sm.cand[beam * k + above] = key;
            }
            __syncthreads();
        }
    }
    cl.sync();
    // beams shared out: the slices' lists become one list of scores in CTA 0
    double *fin_score = cl.map_shared_rank(sm.fin_score, 0);
    int32_t *fin_token = cl.map_shared_rank(sm.fin_token, 0);
    for (int beam = rank; beam < beams; beam += n_ranks) {
        const int row = item * beams + beam;
        const double cum = a.b.scores[row];
        const bool done = a.b.finished && a.b.finished[row];
        float M = -INFINITY;
        for (int r = 0; r < n_ranks; ++r) M = fmaxf(M, cl.map_shared_rank(sm.m, r)[beam]);
        double S = 0.0;
        for (int r = 0; r < n_ranks; ++r) {
            const float m = cl.map_shared_rank(sm.m, r)[beam];
            S += cl.map_shared_rank(sm.s, r)[beam] * (m == -INFINITY ? 1.0 : exp((double)m - (double)M));
        }
        const double lse = (double)M + log(S);
        const bool dead = !(cum > -INFINITY && cum < INFINITY) || !(lse > -INFINITY && lse < INFINITY);
        if (done || dead) {
            // one continuation at most; behind it the lowest tokens at -inf
            const bool has = done && cum > -INFINITY && cum < INFINITY;
            for (int i = threadIdx.x; i < k; i += THREADS) {
                const int t = has ? (i == 0 ? a.b.eos : i - 1 + (i - 1 >= a.b.eos)) : i;
                fin_score[beam * k + i] = has && i == 0 ? cum : -INFINITY;
                fin_token[beam * k + i] = t < V ? t : -1;
            }
            continue;                                             // (the whole CTA)
        }
        __syncthreads();
        for (int e = threadIdx.x; e < n_ranks * k; e += THREADS) sm.gather[e] = cl.map_shared_rank(sm.cand, e / k)[beam * k + e % k];
        __syncthreads();
        if (threadIdx.x < k && V < k && (int)threadIdx.x >= V) fin_token[beam * k + threadIdx.x] = -1;       // (a live row lists min(k, V))
        for (int e = threadIdx.x; e < n_ranks * k; e += THREADS) {
            const u64 key = sm.gather[e];
            if (key == 0) continue;
            int above = 0;
            for (int j = 0; j < n_ranks * k; ++j) above += sm.gather[j] > key;
            if (above < k) {
                fin_score[beam * k + above] = cum + ((double)key_value(key) - lse);
                fin_token[beam * k + above] = key_token(key);
            }
        }
    }
    cl.sync();
    if (rank != 0) return;
    // the beams' lists descend: a candidate's rank is its place plus what the others have before it
    for (int e = threadIdx.x; e < beams * k; e += THREADS) {
        if (sm.fin_token[e] < 0) continue;
        const int beam = e / k;
        const double s = sm.fin_score[e];
        int above = e % k;
        for (int o = 0; o < beams && above < k; ++o) {
            if (o == beam) continue;
            int n = 0;
            while (n < k && sm.fin_token[o * k + n] >= 0 && (sm.fin_score[o * k + n] > s || (sm.fin_score[o * k + n] == s && o < beam))) ++n;
            above += n;
        }
        if (above < k) {
            const size_t at = (size_t)item * k + above;
            a.b.out_scores[at] = (float)s;
            a.b.out_tokens[at] = sm.fin_token[e];
            a.b.out_rows[at] = item * beams + beam;
        }
    }
}

template <typename T>
cudaError_t launch(const BeamArgs &a, int ranks, cudaStream_t st) {
    auto kern = beam_kernel<T>;
    static SmemAttrOnce attr;
    static bool big[DEL_MAX_DEVICES] = {};
    cudaError_t e = attr.set(kern, (int)sizeof(Shared));
    int dev = 0;
    if (e == cudaSuccess) e = cudaGetDevice(&dev);
    if (e != cudaSuccess) return e;
    if (!(dev < DEL_MAX_DEVICES && big[dev])) {
        e = cudaFuncSetAttribute(kern, cudaFuncAttributeNonPortableClusterSizeAllowed, 1);
        if (e != cudaSuccess) return e;
        if (dev < DEL_MAX_DEVICES) big[dev] = true;
    }
    return launch_cluster(kern, dim3(a.b.batch * ranks), THREADS, sizeof(Shared), ranks, st, a);
}

}  // namespace

extern "C" int del_beam_select(const del_beam *x, void *cuda_stream) {
    if (!x || !x->logits || !x->scores || !x->out_scores || !x->out_tokens || !x->out_rows) return DEL_EINVAL;
    if (x->dtype != DEL_F32 && x->dtype != DEL_BF16 && x->dtype != DEL_F16) return DEL_EINVAL;
    const int size = x->dtype == DEL_F32 ? 4 : 2;
    if (((uintptr_t)x->scores | (uintptr_t)x->out_scores | (uintptr_t)x->out_tokens | (uintptr_t)x->out_rows) & 3 || (uintptr_t)x->logits % size) return DEL_EINVAL;
    if (x->batch < 1 || x->batch > (1 << 20) || x->beams < 1 || x->beams > MAX_BEAMS || x->vocab < 1 || x->vocab > (1 << 30)) return DEL_EINVAL;
    if (x->k < 1 || x->k > MAX_K || (int64_t)x->beams * x->vocab < x->k || x->row_stride < x->vocab) return DEL_EINVAL;
    if ((int64_t)x->batch * x->beams > INT32_MAX) return DEL_EINVAL;
    if (x->finished && (x->eos < 0 || x->eos >= x->vocab)) return DEL_EINVAL;
    const int n_sms = current_sms();
    if (!n_sms) return DEL_ECUDA;
    BeamArgs a;
    memset(&a, 0, sizeof(a));
    a.b = *x;
    a.aligned = ((uintptr_t)x->logits & 15) == 0 && (x->row_stride * size) % 16 == 0;
    int ranks = 1;
    while (ranks < MAX_CLUSTER && ranks * 2 * x->batch <= 2 * n_sms && ranks * 1024 < x->vocab) ranks *= 2;
    a.slice = ((x->vocab + ranks - 1) / ranks + 7) / 8 * 8;
    cudaStream_t st = (cudaStream_t)cuda_stream;
    const cudaError_t e = x->dtype == DEL_F32 ? launch<float>(a, ranks, st) : x->dtype == DEL_BF16 ? launch<bf16>(a, ranks, st) : launch<__half>(a, ranks, st);
    return e == cudaSuccess ? DEL_OK : DEL_ECUDA;
}
