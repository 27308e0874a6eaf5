// Beam search's selection (del_beam_select): log softmax, scores and the k best of beams x vocabulary in one pass over the logits.
//
// One cluster of CTAs works on one batch item, a CTA on a slice of one beam's row (or on whole rows in turn, with more beams than
// CTAs).  Within a beam the score rises with the logit, so a CTA keeps the k largest logits of its slice (equal ones: the lower
// token) beside the running maximum and sum of exponentials.  The slices' lists of a beam are then merged, the log-sum-exp turns
// logits into scores (64 bits: near candidates of different beams are ordered by it), and CTA 0 merges the beams' lists.
//
// The k largest of a slice that streams through registers in chunks of 8192: of the first chunk every warp takes the r-th largest of
// its threads' maxima, r = ceil(k / warps); the smallest of these over the warps has at least k logits at or above it and, for
// logits in no special order, few more.  Those go to a list, ranked by counting; the k-th of them is the bar for the next chunks,
// where hardly any logit passes it.  Where the list would overflow (rising logits, say) the chunk's k largest are taken one by one.
// What is left per logit is its load, a maximum, a multiply-add, an exponential and a sum.
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
    int32_t slices, slice;                 // CTAs per row, columns per CTA (a multiple of 8)
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
    int count[3];                          // logits listed of chunk i: count[i % 3] (cleared while no thread can still read it)
    float m[MAX_BEAMS];                    // per row of this CTA: maximum and sum of exponentials of its slice
    double s[MAX_BEAMS];
    double fin_score[MAX_BEAMS * MAX_K];   // CTA 0: the beams' merged lists
    int32_t fin_token[MAX_BEAMS * MAX_K];
    u64 cand[MAX_BEAMS * MAX_K];           // per row: its k largest, descending, 0 behind the last
    u64 gather[MAX_CLUSTER * MAX_K];
};

// the column of element e of this thread in a chunk: vectors of VEC elements, threads side by side
template <int VEC> __device__ __forceinline__ int column(int e) { return ((e / VEC) * THREADS + threadIdx.x) * VEC + e % VEC; }

__device__ __forceinline__ float ex2f(float x) {
    float y;
    asm("ex2.approx.ftz.f32 %0, %1;" : "=f"(y) : "f"(x));
    return y;
}

// elements [c0, c0 + n) of a row into registers; -inf behind the end
template <typename T>
__device__ __forceinline__ void load_chunk(float (&x)[EPT], const T *p, int n, bool aligned) {
    constexpr int VEC = 16 / sizeof(T);
    if (aligned) {
#pragma unroll
        for (int v = 0; v < EPT / VEC; ++v) {
            const int c = column<VEC>(v * VEC);
            if (c + VEC <= n) {
                const uint4 q = ldg_stream16(p + c);
                T t[VEC];
                memcpy(t, &q, 16);
#pragma unroll
                for (int e = 0; e < VEC; ++e) x[v * VEC + e] = to_f<T>(t[e]);
            } else {
#pragma unroll
                for (int e = 0; e < VEC; ++e) x[v * VEC + e] = c + e < n ? to_f<T>(p[c + e]) : -INFINITY;
            }
        }
    } else {
#pragma unroll
        for (int e = 0; e < EPT; ++e) x[e] = column<VEC>(e) < n ? to_f<T>(p[column<VEC>(e)]) : -INFINITY;
    }
}

// The list's k largest, descending, to list[0 .. k) (0 behind the last); returns how many it has.  All threads call.
__device__ __forceinline__ int prune(Shared &sm, int count, int k) {
    u64 mine[(LIST + MAX_K + THREADS - 1) / THREADS];
    int at[(LIST + MAX_K + THREADS - 1) / THREADS];
#pragma unroll
    for (int r = 0; r < (LIST + MAX_K + THREADS - 1) / THREADS; ++r) {
        const int i = threadIdx.x + r * THREADS;
        at[r] = k;
        if (i < count) {
            mine[r] = sm.list[i];
            int above = 0;
#pragma unroll 8
            for (int j = 0; j < count; ++j) above += sm.list[j] > mine[r];
            at[r] = above;
        }
    }
    __syncthreads();
#pragma unroll
    for (int r = 0; r < (LIST + MAX_K + THREADS - 1) / THREADS; ++r)
        if (at[r] < k) sm.list[at[r]] = mine[r];
    for (int i = count + threadIdx.x; i < k; i += THREADS) sm.list[i] = 0;
    __syncthreads();
    return min(count, k);
}

// k largest keys and (maximum, sum of exponentials) of columns [lo, hi) of a row -> cand, m, s of this CTA's row `local`
template <typename T>
__device__ void slice_best(Shared &sm, const T *row, int lo, int hi, int k, bool aligned, int local) {
    constexpr int VEC = 16 / sizeof(T);
    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
    float m = -INFINITY, s = 0.f;
    u64 bar = 0;                                                  // only keys at or above it count
    float bar_x = -INFINITY;
    int count = 0;                                                // entries of the list (the same in every thread)
    float nx[EPT];
    load_chunk<T>(nx, row + lo, min(CHUNK, hi - lo), aligned);
    int ci = 0;                                                   // chunk number modulo 3
    for (int c0 = lo; c0 < hi; c0 += CHUNK, ci = ci == 2 ? 0 : ci + 1) {
        const int n = min(CHUNK, hi - c0);
        float x[EPT];
#pragma unroll
        for (int e = 0; e < EPT; ++e) x[e] = nx[e];
        if (c0 + CHUNK < hi) load_chunk<T>(nx, row + c0 + CHUNK, min(CHUNK, hi - c0 - CHUNK), aligned);
        float cm = x[0];
#pragma unroll
        for (int e = 1; e < EPT; ++e) cm = fmaxf(cm, x[e]);
        // (x - m before the factor: far from zero, the product x * log2 e has lost what the difference needs)
        const float m_new = fmaxf(m, cm), base = m_new == -INFINITY ? 0.f : m_new;
        if (m != -INFINITY) s *= ex2f((m - base) * LOG2E);
        m = m_new;
        float p0 = 0.f, p1 = 0.f;
#pragma unroll
        for (int e = 0; e < EPT; e += 2) {
            p0 += ex2f((x[e] - base) * LOG2E);
            p1 += ex2f((x[e + 1] - base) * LOG2E);
        }
        s += p0 + p1;
        if (c0 == lo) {
            // the bar of the first chunk, from the warps whose threads all have logits
            const int n_full = min(NW, n / (32 * VEC)), r_th = n_full ? (k + n_full - 1) / n_full : 0;
            u64 best = 0;
#pragma unroll
            for (int e = 0; e < EPT; ++e)
                if (column<VEC>(e) < n && (best == 0 || x[e] > key_value(best))) best = make_key(x[e], c0 + column<VEC>(e));
            u64 w = 0;
            for (int r = 0; r < r_th; ++r) {
                w = warp_max_u64(best);
                if (best == w) best = 0;
            }
            if (lane == 0) sm.warp_key[warp] = w;
            if (threadIdx.x < 3) sm.count[threadIdx.x] = 0;
            __syncthreads();
            if (n_full && r_th <= 32) {                           // (r_th > 32: fewer than 64 threads' logits, all of them are listed)
                bar = ~0ull;
                for (int i = 0; i < n_full; ++i) bar = min(bar, sm.warp_key[i]);
                bar_x = bar ? key_value(bar) : -INFINITY;
            }
        }
        if (!(cm < bar_x)) {                                      // (a NaN passes on to the key's comparison)
#pragma unroll
            for (int e = 0; e < EPT; ++e)
                if (!(x[e] < bar_x) && column<VEC>(e) < n) {
                    const u64 key = make_key(x[e], c0 + column<VEC>(e));
                    if (key >= bar) {
                        const int at = count + atomicAdd(&sm.count[ci], 1);
                        if (at < LIST) sm.list[at] = key;
                    }
                }
        }
        if (threadIdx.x == 0) sm.count[ci == 2 ? 0 : ci + 1] = 0;
        __syncthreads();
        int now = count + sm.count[ci];
        if (now > LIST) {
            // too many: the chunk's k largest one by one, behind what was there
            u64 last = ~0ull;
            now = count;
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
                if (threadIdx.x == 0) sm.list[now] = next;
                last = next;
                ++now;
            }
            __syncthreads();
        }
        count = now;
        if (c0 + CHUNK >= hi || c0 == lo || count > LIST / 4) {
            count = prune(sm, count, k);
            if (count == k) {
                bar = sm.list[k - 1];
                bar_x = key_value(bar);
            }
        }
    }
    // sums of the threads, in double
    float wm = m;
#pragma unroll
    for (int o = 16; o > 0; o >>= 1) wm = fmaxf(wm, __shfl_xor_sync(0xffffffffu, wm, o));
    double ws = m == -INFINITY ? (double)s : (double)(s * ex2f((m - wm) * LOG2E));       // (m = -inf: 0, or no number)
#pragma unroll
    for (int o = 16; o > 0; o >>= 1) ws += __shfl_xor_sync(0xffffffffu, ws, o);
    if (lane == 0) { sm.warp_m[warp] = wm; sm.warp_s[warp] = ws; }
    for (int i = threadIdx.x; i < k; i += THREADS) sm.cand[local * k + i] = i < count ? sm.list[i] : 0;
    __syncthreads();
    if (warp == 0) {
        const float tm = lane < NW ? sm.warp_m[lane] : -INFINITY;
        const double ts = lane < NW ? sm.warp_s[lane] : 0.0;
        float M = tm;
#pragma unroll
        for (int o = 16; o > 0; o >>= 1) M = fmaxf(M, __shfl_xor_sync(0xffffffffu, M, o));
        double S = tm == -INFINITY ? ts : ts * (double)ex2f((tm - M) * LOG2E);
#pragma unroll
        for (int o = 16; o > 0; o >>= 1) S += __shfl_xor_sync(0xffffffffu, S, o);
        if (lane == 0) { sm.m[local] = M; sm.s[local] = S; }
    }
    __syncthreads();
}

template <typename T>
__global__ void __launch_bounds__(THREADS, 2) beam_kernel(const BeamArgs a) {
    extern __shared__ __align__(16) unsigned char smem[];
    Shared &sm = *reinterpret_cast<Shared *>(smem);
    cg::cluster_group cl = cg::this_cluster();
    const int rank = cl.block_rank(), n_ranks = cl.num_blocks();
    const int item = blockIdx.x / n_ranks, beams = a.b.beams, V = a.b.vocab, k = a.b.k, slices = a.slices;
    // rank = beam * slices + slice; with more beams than CTAs (slices = 1) beams rank, rank + n_ranks, ...
    for (int e = threadIdx.x; e < MAX_BEAMS; e += THREADS) { sm.m[e] = -INFINITY; sm.s[e] = 0.0; }
    const int lo = (int)min((int64_t)(rank % slices) * a.slice, (int64_t)V), hi = (int)min((int64_t)lo + a.slice, (int64_t)V);
    int local = 0;
    for (int beam = rank / slices; beam < beams; beam += n_ranks, ++local) {
        const int row = item * beams + beam;
        if (a.b.finished && a.b.finished[row]) continue;
        if (lo < hi) slice_best<T>(sm, reinterpret_cast<const T *>(a.b.logits) + row * a.b.row_stride, lo, hi, k, a.aligned, local);
        else
            for (int i = threadIdx.x; i < k; i += THREADS) sm.cand[local * k + i] = 0;
    }
    cl.sync();
    // each beam's first CTA: the slices' lists become one list of scores in CTA 0
    double *fin_score = cl.map_shared_rank(sm.fin_score, 0);
    int32_t *fin_token = cl.map_shared_rank(sm.fin_token, 0);
    local = 0;
    for (int beam = rank / slices; beam < beams && rank % slices == 0; beam += n_ranks, ++local) {
        const int row = item * beams + beam;
        const double cum = a.b.scores[row];
        const bool done = a.b.finished && a.b.finished[row];
        double lse = 0.0;
        if (!done) {
            float M = -INFINITY;
            for (int r = 0; r < slices; ++r) M = fmaxf(M, cl.map_shared_rank(sm.m, rank + r)[local]);
            double S = 0.0;
            for (int r = 0; r < slices; ++r) {
                const float m = cl.map_shared_rank(sm.m, rank + r)[local];
                S += cl.map_shared_rank(sm.s, rank + r)[local] * (m == -INFINITY ? 1.0 : (double)ex2f((m - M) * LOG2E));
            }
            lse = (double)M + log(S);
        }
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
        for (int e = threadIdx.x; e < slices * k; e += THREADS) sm.gather[e] = cl.map_shared_rank(sm.cand, rank + e / k)[local * k + e % k];
        __syncthreads();
        if (threadIdx.x < k && (int)threadIdx.x >= V) fin_token[beam * k + threadIdx.x] = -1;       // (a live row lists min(k, V))
        for (int e = threadIdx.x; e < slices * k; e += THREADS) {
            const u64 key = sm.gather[e];
            if (key == 0) continue;
            int above = e % k;                                    // its place in its own list; the others descend as well
            for (int r = 0; r < slices && above < k; ++r) {
                if (r == e / k) continue;
                int n = 0;
                while (n < k && sm.gather[r * k + n] > key) ++n;
                above += n;
            }
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
    // CTAs per item: two per SM over all items, at most 16 (a cluster), none with less than 2048 columns (a smaller slice is all
    // latency); whole rows per CTA where there are more beams than CTAs
    int64_t ranks = 2 * (int64_t)n_sms / x->batch, most = (int64_t)x->beams * ((x->vocab + 2047) / 2048);
    if (ranks > MAX_CLUSTER) ranks = MAX_CLUSTER;
    if (ranks > most) ranks = most;
    if (ranks < 1) ranks = 1;
    a.slices = ranks >= x->beams ? (int)(ranks / x->beams) : 1;
    if (ranks >= x->beams) ranks = (int64_t)a.slices * x->beams;
    a.slice = ((x->vocab + a.slices - 1) / a.slices + 7) / 8 * 8;
    cudaStream_t st = (cudaStream_t)cuda_stream;
    const cudaError_t e = x->dtype == DEL_F32 ? launch<float>(a, (int)ranks, st) : x->dtype == DEL_BF16 ? launch<bf16>(a, (int)ranks, st) : launch<__half>(a, (int)ranks, st);
    return e == cudaSuccess ? DEL_OK : DEL_ECUDA;
}
