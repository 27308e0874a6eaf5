// Beam search's selection (del_beam_select): log softmax, scores and the k best of beams x vocabulary in one pass over the logits.
//
// One cluster of CTAs works on one batch item, a CTA on a slice of one beam's row (or on whole rows in turn, with more beams than
// CTAs).  Within a beam the score rises with the logit, so a CTA keeps the k largest logits of its slice (equal ones: the lower
// token) beside the running maximum and sum of exponentials, and leaves them in the shared memory of the cluster's first CTA.  That
// one turns logits into scores (64 bits: near candidates of different beams are ordered by them) and merges the lists.
//
// The k largest of a slice that streams through registers in chunks: of the first chunk every warp lists the largest of its threads'
// maxima, r = k / 4 of them; the k-th of all listed is a bar that at least k logits reach and, for logits in no special order, hardly
// more.  What reaches the bar goes to a list; every four chunks the list is ranked by counting where it has grown, and its k-th
// becomes the bar.  A logit that passes costs a warp some 250 cycles, so the bar has to be good: with the smallest of the warps'
// maxima as the first bar (54 logits of 8192 pass instead of k) 16 x 8 x 128256 took 84 us, 45 of them for what passed.  Where the list would
// overflow (rising logits, say) the k largest of the four chunks are taken one by one.  What is left per logit is its load, a
// maximum, a comparison, an exponential and a sum.
//
// The smallest calls are all latency, much of it instruction fetch: what runs rarely reads the logits again in rolled loops instead of
// unrolling over the registers that hold them.
#include <cooperative_groups.h>
#include <cuda_fp16.h>
#include <cstring>
#include <utility>

#include "pages.cuh"

namespace cg = cooperative_groups;

namespace {

typedef unsigned long long u64;

constexpr int THREADS = 512, NW = THREADS / 32, NV = 2, MAX_K = 64, MAX_BEAMS = 64, MAX_CLUSTER = 16;
constexpr int GROUP = 4;                   // chunks between two looks at the list's length
constexpr int LIST = 1024;                 // candidates of a slice that are ranked by counting
constexpr int LISTS = MAX_BEAMS;           // most lists of an item: beams x slices <= MAX_CLUSTER, or one per beam
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
    u64 warp_key[NW * 32], bar;
    float warp_m[NW];
    double warp_s[NW];
    int count[3];                          // logits listed of group i: count[i % 3] (cleared while no thread can still read it)
    // the cluster's first CTA: list i belongs to beam i / slices
    u64 key[LISTS * MAX_K];                // k each, descending, 0 behind the last
    float m[LISTS];                        // maximum and sum of exponentials of the slice
    double s[LISTS];
    double score[LISTS * MAX_K];
    double lse[MAX_BEAMS];
};

// a chunk: NV vectors of 16 bytes per thread, threads side by side
template <typename T> struct Chunk {
    static constexpr int VEC = 16 / sizeof(T), EPT = NV * VEC, SIZE = THREADS * EPT;
    static __device__ __forceinline__ int column(int e) { return ((e / VEC) * THREADS + threadIdx.x) * VEC + e % VEC; }
};

__device__ __forceinline__ float ex2f(float x) {
    float y;
    asm("ex2.approx.ftz.f32 %0, %1;" : "=f"(y) : "f"(x));
    return y;
}

// elements [0, n) of p into registers; what lies behind the end is left as it is
template <typename T>
__device__ __forceinline__ void load_chunk(uint4 (&q)[NV], const T *p, int n, bool aligned) {
    using C = Chunk<T>;
#pragma unroll
    for (int v = 0; v < NV; ++v) {
        const int c = C::column(v * C::VEC);
        if (aligned && c + C::VEC <= n) q[v] = ldg_stream16(p + c);
        else if (c < n) {
            T t[C::VEC];
#pragma unroll
            for (int e = 0; e < C::VEC; ++e) t[e] = p[min(c + e, n - 1)];
            memcpy(&q[v], t, 16);
        }
    }
}

// The list's k largest, descending, to list[0 .. k) (0 behind the last); returns how many it has.  All threads call.
__device__ __noinline__ int prune(Shared &sm, int count, int k) {
    constexpr int N = (LIST + MAX_K + THREADS - 1) / THREADS;
    u64 mine[N];
    int at[N];
#pragma unroll
    for (int r = 0; r < N; ++r) {
        const int i = threadIdx.x + r * THREADS;
        mine[r] = i < count ? sm.list[i] : 0;
        at[r] = i < count ? 0 : k;
    }
    if ((int)(threadIdx.x & ~31u) < count) {
#pragma unroll 4
        for (int j = 0; j < count; ++j) {
            const u64 o = sm.list[j];
#pragma unroll
            for (int r = 0; r < N; ++r) at[r] += o > mine[r];
        }
    }
    __syncthreads();
#pragma unroll
    for (int r = 0; r < N; ++r)
        if (at[r] < k) sm.list[at[r]] = mine[r];
    for (int i = count + threadIdx.x; i < k; i += THREADS) sm.list[i] = 0;
    __syncthreads();
    return min(count, k);
}

// the k largest of p[0, n) one by one, behind the list's first `count` entries; returns the new count.  All threads call.
template <typename T>
__device__ __noinline__ int take_largest(Shared &sm, const T *p, int first_token, int n, int count, int k) {
    u64 last = ~0ull;
    for (int i = 0; i < k; ++i) {
        u64 next = 0;
        for (int c = threadIdx.x; c < n; c += THREADS) {
            const u64 key = make_key(to_f<T>(p[c]), first_token + c);
            if (key < last && key > next) next = key;
        }
        next = warp_max_u64(next);
        __syncthreads();
        if ((threadIdx.x & 31) == 0) sm.warp_key[threadIdx.x >> 5] = next;
        __syncthreads();
        for (int j = 0; j < NW; ++j) next = max(next, sm.warp_key[j]);
        if (next == 0) break;
        if (threadIdx.x == 0) sm.list[count] = next;
        last = next;
        ++count;
    }
    __syncthreads();
    return count;
}

// k largest keys and (maximum, sum of exponentials) of columns [lo, hi) of a row -> list, (m, s) in every thread of warp 0
template <typename T>
__device__ __forceinline__ int slice_best(Shared &sm, const T *row, int lo, int hi, int k, bool aligned, float &m_out, double &s_out) {
    using C = Chunk<T>;
    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
    float m = -INFINITY, s = 0.f;
    u64 bar = 0;                                                  // only keys at or above it count
    float bar_x = -INFINITY;
    int count = 0;                                                // entries of the list (the same in every thread)
    int gi = 0;                                                   // group number modulo 3

    auto load = [&](uint4 (&q)[NV], int c0) {
        if (c0 < hi) load_chunk<T>(q, row + c0, min(C::SIZE, hi - c0), aligned);
    };
    auto work = [&](uint4 (&q)[NV], int c0) {
        const int n = min(C::SIZE, hi - c0);
        float x[C::EPT];
#pragma unroll
        for (int v = 0; v < NV; ++v) {
            T t[C::VEC];
            memcpy(t, &q[v], 16);
#pragma unroll
            for (int e = 0; e < C::VEC; ++e) x[v * C::VEC + e] = n == C::SIZE || C::column(v * C::VEC + e) < n ? to_f<T>(t[e]) : -INFINITY;
        }
        load(q, c0 + 2 * C::SIZE);
        float cm = x[0];
#pragma unroll
        for (int e = 1; e < C::EPT; ++e) cm = fmaxf(cm, x[e]);
        // (x - m before the factor: far from zero, the product x * log2 e has lost what the difference needs)
        const float m_new = fmaxf(m, cm), base = m_new == -INFINITY ? 0.f : m_new;
        if (m != -INFINITY) s *= ex2f((m - base) * LOG2E);
        m = m_new;
        float p0 = 0.f, p1 = 0.f;
#pragma unroll
        for (int e = 0; e < C::EPT; e += 2) {
            p0 += ex2f((x[e] - base) * LOG2E);
            p1 += ex2f((x[e + 1] - base) * LOG2E);
        }
        s += p0 + p1;
        if (c0 == lo) {
            // the first bar, from the warps' lists of their threads' maxima (f: warps whose threads all have logits)
            const int f = min(NW, n / (32 * C::VEC)), r_th = f ? max((k + 3) / 4, (k + f - 1) / f) : 33;
            if (threadIdx.x < 3) sm.count[threadIdx.x] = 0;
            if (threadIdx.x == 0) sm.bar = 0;
            if (r_th <= 32) {                                     // (else fewer than 64 threads' logits: all of them are listed)
                uint32_t hi32 = 0, lo32 = 0;
                if (C::column(0) < n) {
                    int at = 0;
#pragma unroll
                    for (int e = C::EPT - 1; e >= 0; --e)
                        if (x[e] == cm && C::column(e) < n) at = e;
                    const u64 best = make_key(cm, c0 + C::column(at));
                    hi32 = (uint32_t)(best >> 32);
                    lo32 = (uint32_t)best;
                }
                for (int r = 0; r < r_th; ++r) {
                    const uint32_t top = __reduce_max_sync(0xffffffffu, hi32), low = __reduce_max_sync(0xffffffffu, hi32 == top ? lo32 : 0u);
                    if (lane == 0) sm.warp_key[warp * r_th + r] = ((u64)top << 32) | low;
                    if (hi32 == top && lo32 == low) hi32 = lo32 = 0;
                }
                __syncthreads();
                if (threadIdx.x < NW * r_th) {
                    const u64 mine = sm.warp_key[threadIdx.x];
                    int above = 0;
#pragma unroll 8
                    for (int i = 0; i < NW * r_th; ++i) above += sm.warp_key[i] > mine;
                    if (mine && above == k - 1) sm.bar = mine;
                }
            }
            __syncthreads();
            bar = sm.bar;
            bar_x = bar ? key_value(bar) : -INFINITY;
        }
        if (!(cm < bar_x)) {                                      // (a NaN passes on to the key's comparison)
            uint32_t pass = 0;
#pragma unroll
            for (int e = 0; e < C::EPT; ++e) pass |= !(x[e] < bar_x) && (n == C::SIZE || C::column(e) < n) ? 1u << e : 0u;
            for (; pass; pass &= pass - 1) {
                const int e0 = __ffs(pass) - 1;
                float v = x[0];
#pragma unroll
                for (int e = 1; e < C::EPT; ++e) v = e == e0 ? x[e] : v;
                const u64 key = make_key(v, c0 + C::column(e0));
                if (key >= bar) {
                    const int at = count + atomicAdd(&sm.count[gi], 1);
                    if (at < LIST) sm.list[at] = key;
                }
            }
        }
    };
    // after a group of chunks: did the list hold, and can the bar be raised?
    auto look = [&](int g0) {
        const int n = min(GROUP * C::SIZE, hi - g0);
        if (threadIdx.x == 0) sm.count[gi == 2 ? 0 : gi + 1] = 0;
        __syncthreads();
        const int now = count + sm.count[gi];
        count = now <= LIST ? now : take_largest<T>(sm, row + g0, g0, n, count, k);
        if (g0 + GROUP * C::SIZE >= hi || count > 2 * k + 16) {
            count = prune(sm, count, k);
            if (count == k) {
                bar = sm.list[k - 1];
                bar_x = key_value(bar);
            }
            // (prune's last barrier lies between these reads and the next writes to the list: they go behind its k entries)
        }
        gi = gi == 2 ? 0 : gi + 1;
    };

    // two chunks in flight: a buffer is filled again as soon as it has been read
    uint4 qa[NV], qb[NV];
#pragma unroll
    for (int v = 0; v < NV; ++v) qa[v] = qb[v] = make_uint4(0, 0, 0, 0);
    load(qa, lo);
    load(qb, lo + C::SIZE);
    for (int g0 = lo; g0 < hi; g0 += GROUP * C::SIZE) {
        for (int c0 = g0; c0 < min(hi, g0 + GROUP * C::SIZE); c0 += 2 * C::SIZE) {
            work(qa, c0);
            if (c0 + C::SIZE < hi) work(qb, c0 + C::SIZE);
        }
        look(g0);
    }
    // sums of the threads, in double
    float wm = m;
#pragma unroll
    for (int o = 16; o > 0; o >>= 1) wm = fmaxf(wm, __shfl_xor_sync(0xffffffffu, wm, o));
    double ws = m == -INFINITY ? (double)s : (double)(s * ex2f((m - wm) * LOG2E));       // (m = -inf: 0, or no number)
#pragma unroll
    for (int o = 16; o > 0; o >>= 1) ws += __shfl_xor_sync(0xffffffffu, ws, o);
    if (lane == 0) { sm.warp_m[warp] = wm; sm.warp_s[warp] = ws; }
    __syncthreads();
    const float tm = lane < NW ? sm.warp_m[lane] : -INFINITY;
    const double ts = lane < NW ? sm.warp_s[lane] : 0.0;
    float M = tm;
#pragma unroll
    for (int o = 16; o > 0; o >>= 1) M = fmaxf(M, __shfl_xor_sync(0xffffffffu, M, o));
    double S = tm == -INFINITY ? ts : ts * (double)ex2f((tm - M) * LOG2E);
#pragma unroll
    for (int o = 16; o > 0; o >>= 1) S += __shfl_xor_sync(0xffffffffu, S, o);
    m_out = M;
    s_out = S;
    return count;
}

template <typename T>
__global__ void __launch_bounds__(THREADS, 2) beam_kernel(const BeamArgs a) {
    extern __shared__ __align__(16) unsigned char smem[];
    Shared &sm = *reinterpret_cast<Shared *>(smem);
    cg::cluster_group cl = cg::this_cluster();
    const int rank = cl.block_rank(), n_ranks = cl.num_blocks();
    const int item = blockIdx.x / n_ranks, beams = a.b.beams, V = a.b.vocab, k = a.b.k, slices = a.slices, n_lists = beams * slices;
    auto started = cl.barrier_arrive();
    Shared &first = *cl.map_shared_rank(&sm, 0);
    // list = beam * slices + slice; with more beams than CTAs (slices = 1) lists rank, rank + n_ranks, ...
    const int lo = (int)min((int64_t)(rank % slices) * a.slice, (int64_t)V), hi = (int)min((int64_t)lo + a.slice, (int64_t)V);
    for (int list = rank; list < n_lists; list += n_ranks) {       // (every rank has one)
        const int row = item * beams + list / slices;
        float m = -INFINITY;
        double s = 0.0;
        int count = 0;
        if (lo < hi && !(a.b.finished && a.b.finished[row]))
            count = slice_best<T>(sm, reinterpret_cast<const T *>(a.b.logits) + row * a.b.row_stride, lo, hi, k, a.aligned, m, s);
        if (list == rank) cl.barrier_wait(std::move(started));    // the first CTA runs: its shared memory may be written
        for (int i = threadIdx.x; i < k; i += THREADS) first.key[list * k + i] = i < count ? sm.list[i] : 0;
        if (threadIdx.x == 0) { first.m[list] = m; first.s[list] = s; }
        __syncthreads();
    }
    if (n_ranks > 1) cl.sync();
    if (rank != 0) return;
    // a beam's log-sum-exp; then its lists' scores
    for (int beam = threadIdx.x; beam < beams; beam += THREADS) {
        const int row = item * beams + beam;
        const double cum = a.b.scores[row];
        const bool number = cum > -INFINITY && cum < INFINITY;
        double lse = INFINITY;                                    // no candidates but those at -inf; -inf: finished
        if (a.b.finished && a.b.finished[row]) lse = number ? -INFINITY : INFINITY;
        else if (number) {
            float M = -INFINITY;
            for (int r = 0; r < slices; ++r) M = fmaxf(M, sm.m[beam * slices + r]);
            double S = 0.0;
            for (int r = 0; r < slices; ++r) {
                const float m = sm.m[beam * slices + r];
                S += sm.s[beam * slices + r] * (m == -INFINITY ? 1.0 : (double)ex2f((m - M) * LOG2E));
            }
            lse = (double)M + log(S);
            if (!(lse > -INFINITY && lse < INFINITY)) lse = INFINITY;
        }
        sm.lse[beam] = lse;
    }
    __syncthreads();
    for (int e = threadIdx.x; e < n_lists * k; e += THREADS) {
        const int list = e / k, i = e - list * k, beam = list / slices;
        const double cum = a.b.scores[item * beams + beam], lse = sm.lse[beam];
        u64 key = sm.key[e];
        double score = -INFINITY;
        if (lse == INFINITY || lse == -INFINITY) {
            // one continuation (finished) or none; behind it the lowest tokens at -inf, in the beam's first list
            const int eos = a.b.eos, t = lse == INFINITY ? i : i == 0 ? eos : i - 1 + (i - 1 >= eos);
            if (lse == -INFINITY && i == 0) score = cum;
            key = list % slices == 0 && t < V ? make_key(0.f, t) : 0;
        } else if (key) {
            score = cum + ((double)key_value(key) - lse);
        }
        sm.key[e] = key;
        sm.score[e] = score;
    }
    __syncthreads();
    // the lists descend: a candidate's rank is its place plus what the others have before it
    for (int e = threadIdx.x; e < n_lists * k; e += THREADS) {
        const u64 key = sm.key[e];
        if (key == 0) continue;
        const int list = e / k, beam = list / slices;
        const double s = sm.score[e];
        int above = e - list * k;
        for (int o = 0; o < n_lists && above < k; ++o) {
            if (o == list) continue;
            const int ob = o / slices;
            int n = 0;
            while (n < k) {
                const u64 ok = sm.key[o * k + n];
                const double os = sm.score[o * k + n];
                if (ok == 0 || !(ob == beam ? ok > key : os > s || (os == s && ob < beam))) break;
                ++n;
            }
            above += n;
        }
        if (above < k) {
            const size_t at = (size_t)item * k + above;
            a.b.out_scores[at] = (float)s;
            a.b.out_tokens[at] = key_token(key);
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
    if (ranks > (x->batch <= 6 ? MAX_CLUSTER : 8)) ranks = x->batch <= 6 ? MAX_CLUSTER : 8;
    if (ranks > most) ranks = most;
    if (ranks < 1) ranks = 1;
    a.slices = ranks >= x->beams ? (int)(ranks / x->beams) : 1;
    if (ranks >= x->beams) ranks = (int64_t)a.slices * x->beams;
    a.slice = ((x->vocab + a.slices - 1) / a.slices + 7) / 8 * 8;
    cudaStream_t st = (cudaStream_t)cuda_stream;
    const cudaError_t e = x->dtype == DEL_F32 ? launch<float>(a, (int)ranks, st) : x->dtype == DEL_BF16 ? launch<bf16>(a, (int)ranks, st) : launch<__half>(a, (int)ranks, st);
    return e == cudaSuccess ? DEL_OK : DEL_ECUDA;
}
