// Beam search's selection (del_beam_select): log softmax, scores and the k best of beams x vocabulary in one pass over the logits.
//
// A CTA takes a slice of one row.  Within a row the score rises with the logit, so the CTA keeps the k largest logits of its slice
// (equal ones: the lower token) beside the running maximum and sum of exponentials, and leaves them in the workspace.  One CTA per
// item then turns the slices' logits into scores (64 bits: near candidates of different rows are ordered by them) and takes the k best.
// Small calls do both in one launch, an item's CTAs being a cluster; the others in two, the second starting while the first
// drains.  B200 keeps 15 clusters of 8 or 7 of 16 resident with one CTA per SM: 16 x 8 x 128256 takes 59 us in clusters of 8 (two
// waves), 25 us as 128 free CTAs, but a second launch costs the host 4 us (1 x 4 x 32000: 10 us a call in one launch, 13 in two).
//
// The k largest of a slice that streams through registers in chunks: of the first chunk every warp lists the largest of its threads'
// maxima, r = k / 4 of them; the k-th of all listed is a bar that at least k logits reach and, for logits in no special order, hardly
// more.  What reaches the bar goes to a list; every four chunks the list is ranked by counting where it has grown, and its k-th
// becomes the bar.  A logit that passes costs a warp some 250 cycles, so the bar has to be good: with the smallest of the warps'
// maxima as the first bar (54 logits of 8192 pass instead of k) 16 x 8 x 128256 took 84 us, 45 of them for what passed.  Behind the first
// chunk a logit has to lie above the bar, as an equal one has a higher token.  Where the list would
// overflow (rising logits, say) the k largest of the four chunks are taken one by one.  What is left per logit is its load, a
// maximum, a comparison, an exponential and a sum.
//
// Equal logits cost more in a slice's first chunk, where all of them pass to the comparison of keys: with all but 10 tokens of each row at
// -inf, 16 x 8 x 128256 takes 36 us instead of 24 (87 when equal ones passed in every chunk), 4 x 4 of 128256 in bf16 47 instead of 15,
// 1 x 4 x 32000 24 instead of 7.7; rows of one value 43, 57 and 29.  With more allowed tokens in a chunk than k nothing changes.
//
// The smallest calls are all latency, much of it instruction fetch: what runs rarely reads the logits again in rolled loops instead of
// unrolling over the registers that hold them.
#include <cooperative_groups.h>
#include <cuda_fp16.h>
#include <cstring>

#include "pages.cuh"

namespace {

typedef unsigned long long u64;

constexpr int THREADS = 512, NW = THREADS / 32, NV = 4, MAX_K = 64, MAX_BEAMS = 64, MAX_CAND = 4096, MAX_CLUSTER = 16;
constexpr int GROUP = 4;                   // chunks between two looks at the list's length
constexpr int LIST = 1024;                 // candidates of a slice that are ranked by counting
constexpr float LOG2E = 1.4426950408889634f;

struct BeamArgs {
    del_beam b;
    int32_t slices, slice;                 // CTAs per row, columns per CTA (a multiple of 8)
    int32_t aligned;                       // rows start on 16-byte boundaries
    int32_t fused;                         // one launch, an item's CTAs a cluster
    // workspace: list = row * slices + slice
    u64 *key;                              // [lists][k], descending, 0 behind the last
    double *s;                             // [lists] sums of exponentials
    float *m;                              // [lists] maxima
};

// Logits in the order of their value as unsigned numbers; the key of a token puts equal logits in the order of their ids.
// A key is never 0: that stands for no token.
__device__ __forceinline__ uint32_t ordered(float x) {
    const uint32_t b = __float_as_uint(x + 0.f);                  // (-0 becomes +0)
    return b & 0x80000000u ? ~b : b | 0x80000000u;
}
__device__ __forceinline__ float unordered(uint32_t o) { return __uint_as_float(o & 0x80000000u ? o & 0x7fffffffu : ~o); }
// the next number above (of +inf: none, nothing is below it)
__device__ __forceinline__ float above(float x) { return unordered(ordered(x) + 1); }
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
};

// (each function names the array itself: through a pointer the accesses would be generic ones)
__device__ __forceinline__ Shared &shared() {
    extern __shared__ __align__(16) unsigned char smem[];
    return *reinterpret_cast<Shared *>(smem);
}

// Of one number per thread (0: none): the k-th largest of those listed, r per warp; 0 if fewer are.  At least k of the numbers reach it.
// All threads call; ends with a barrier.
__device__ __forceinline__ u64 kth_of_threads(Shared &sm, u64 mine, int k, int r) {
    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
    uint32_t hi = (uint32_t)(mine >> 32), lo = (uint32_t)mine;
    for (int i = 0; i < r; ++i) {
        const uint32_t top = __reduce_max_sync(0xffffffffu, hi), low = __reduce_max_sync(0xffffffffu, hi == top ? lo : 0u);
        const uint32_t who = __ballot_sync(0xffffffffu, hi == top && lo == low);
        if (lane == 0) sm.warp_key[warp * r + i] = ((u64)top << 32) | low;
        if (lane == __ffs(who) - 1) hi = lo = 0;
    }
    if (threadIdx.x == 0) sm.bar = 0;
    __syncthreads();
    if ((int)threadIdx.x < NW * r) {
        const u64 key = sm.warp_key[threadIdx.x];
        int above = 0, before = 0;                                // equal numbers: in the order of the list
#pragma unroll 8
        for (int i = 0; i < NW * r; ++i) {
            const u64 o = sm.warp_key[i];
            above += o > key;
            before += o == key && i < (int)threadIdx.x;
        }
        if (key && above + before == k - 1) sm.bar = key;
    }
    __syncthreads();
    return sm.bar;
}

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

// two lanes of fp32 arithmetic in one instruction: (x - a) * b, and x += b
__device__ __forceinline__ void sub_mul2(float &x0, float &x1, float a, float b) {
    asm("{\n\t.reg .b64 x, y, z;\n\tmov.b64 x, {%0, %1};\n\tmov.b64 y, {%2, %2};\n\tmov.b64 z, {%3, %3};\n\t"
        "add.rn.f32x2 x, x, y;\n\tmul.rn.f32x2 x, x, z;\n\tmov.b64 {%0, %1}, x;\n\t}" : "+f"(x0), "+f"(x1) : "f"(-a), "f"(b));
}
__device__ __forceinline__ void add2(float &x0, float &x1, float b0, float b1) {
    asm("{\n\t.reg .b64 x, y;\n\tmov.b64 x, {%0, %1};\n\tmov.b64 y, {%2, %3};\n\tadd.rn.f32x2 x, x, y;\n\tmov.b64 {%0, %1}, x;\n\t}"
        : "+f"(x0), "+f"(x1) : "f"(b0), "f"(b1));
}

template <typename T> __device__ __forceinline__ T minus_infinity() { return T(-INFINITY); }
template <> __device__ __forceinline__ bf16 minus_infinity<bf16>() { return __ushort_as_bfloat16(0xff80); }
template <> __device__ __forceinline__ __half minus_infinity<__half>() { return __ushort_as_half(0xfc00); }

// elements [0, n) of p into registers, -inf behind the end
template <typename T>
__device__ __forceinline__ void load_chunk(uint4 (&q)[NV], const T *p, int n, bool aligned) {
    using C = Chunk<T>;
    if (aligned && n >= C::SIZE) {
#pragma unroll
        for (int v = 0; v < NV; ++v) q[v] = ldg_stream16(p + C::column(v * C::VEC));
    } else {
#pragma unroll
        for (int v = 0; v < NV; ++v) {
            const int c = C::column(v * C::VEC);
            if (aligned && c + C::VEC <= n) q[v] = ldg_stream16(p + c);
            else {
                T t[C::VEC];
#pragma unroll
                for (int e = 0; e < C::VEC; ++e) t[e] = c + e < n ? p[c + e] : minus_infinity<T>();
                memcpy(&q[v], t, 16);
            }
        }
    }
}

// The list's k largest, descending, to list[0 .. k) (0 behind the last); returns how many it has.  All threads call.
__device__ __noinline__ int prune(int count, int k) {
    Shared &sm = shared();
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
__device__ __noinline__ int take_largest(const T *p, int first_token, int n, int count, int k) {
    Shared &sm = shared();
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
    float m = -INFINITY, s0 = 0.f, s1 = 0.f;
    u64 bar = 0;                                                  // only keys at or above it count
    float bar_x = -INFINITY;
    int count = 0;                                                // entries of the list (the same in every thread)
    int gi = 0;                                                   // group number modulo 3

    auto load = [&](uint4 (&q)[NV], int c0) __attribute__((always_inline)) {
        if (c0 < hi) load_chunk<T>(q, row + c0, min(C::SIZE, hi - c0), aligned);
    };
    auto work = [&](uint4 (&q)[NV], int c0) __attribute__((always_inline)) {
        const int n = min(C::SIZE, hi - c0);
        float x[C::EPT];
#pragma unroll
        for (int v = 0; v < NV; ++v) {
            T t[C::VEC];
            memcpy(t, &q[v], 16);
#pragma unroll
            for (int e = 0; e < C::VEC; ++e) x[v * C::VEC + e] = to_f<T>(t[e]);
        }
        load(q, c0 + 2 * C::SIZE);
        float c2[2] = {x[0], x[1]};
#pragma unroll
        for (int e = 2; e < C::EPT; ++e) c2[e & 1] = fmaxf(c2[e & 1], x[e]);
        const float cm = fmaxf(c2[0], c2[1]);
        // (x - m before the factor: far from zero, the product x * log2 e has lost what the difference needs)
        if (cm > m) {
            const float f = m == -INFINITY ? 1.f : ex2f((m - cm) * LOG2E);      // (before the first number: sums of 0, or no number)
            s0 *= f;
            s1 *= f;
            m = cm;
        }
        const float base = m == -INFINITY ? 0.f : m;
#pragma unroll
        for (int e = 0; e < C::EPT; e += 2) {
            float d0 = x[e], d1 = x[e + 1];
            sub_mul2(d0, d1, base, LOG2E);
            add2(s0, s1, ex2f(d0), ex2f(d1));
        }
        if (c0 == lo) {
            // the first bar, from the warps' lists of their threads' maxima (f: warps whose threads all have logits)
            const int f = min(NW, n / (32 * C::VEC)), r_th = f ? max((k + 3) / 4, (k + f - 1) / f) : 33;
            if (threadIdx.x < 3) sm.count[threadIdx.x] = 0;
            if (r_th <= 32) {                                     // (else fewer than 64 threads' logits: all of them are listed)
                u64 best = 0;
                if (C::column(0) < n) {
                    int at = 0;
#pragma unroll
                    for (int e = C::EPT - 1; e >= 0; --e)
                        if (x[e] == cm && C::column(e) < n) at = e;
                    best = make_key(cm, c0 + C::column(at));
                }
                bar = kth_of_threads(sm, best, k, r_th);
            } else {
                __syncthreads();
            }
            bar_x = bar ? key_value(bar) : -INFINITY;
        }
        if (!(cm < bar_x)) {                                      // (a NaN passes on to the key's comparison)
            uint32_t pass = 0;
#pragma unroll
            for (int e = 0; e < C::EPT; ++e) pass |= !(x[e] < bar_x) ? 1u << e : 0u;
            for (; pass; pass &= pass - 1) {
                const int e0 = __ffs(pass) - 1;
                if (C::column(e0) >= n) break;                    // (columns rise with e: nothing but padding is left)
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
        if (c0 == lo && bar) bar_x = above(bar_x);                // (from here on a logit that equals the bar has a higher token)
    };
    // after a group of chunks: did the list hold, and can the bar be raised?
    auto look = [&](int g0) __attribute__((always_inline)) {
        const int n = min(GROUP * C::SIZE, hi - g0);
        if (threadIdx.x == 0) sm.count[gi == 2 ? 0 : gi + 1] = 0;
        __syncthreads();
        const int now = count + sm.count[gi];
        count = now <= LIST ? now : take_largest<T>(row + g0, g0, n, count, k);
        if (g0 + GROUP * C::SIZE >= hi || count > 2 * k + 16) {
            count = prune(count, k);
            if (count == k) {
                bar = sm.list[k - 1];
                bar_x = above(key_value(bar));
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
    const float s = s0 + s1;
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

// the candidates of an item: k of each of its lists
struct Cand {
    u64 *key, *order;                      // order: the scores as numbers in the same order, 0: no candidate
    double *score, *lse, *cum;             // lse, cum: per beam
    int32_t *index;                        // of the candidates in the list
    __device__ Cand(unsigned char *at, int n)
        : key(reinterpret_cast<u64 *>(at)), order(key + n), score(reinterpret_cast<double *>(order + n)), lse(score + n), cum(lse + MAX_BEAMS),
          index(reinterpret_cast<int32_t *>(cum + MAX_BEAMS)) {}
    static constexpr size_t bytes(int n) { return 24 * (size_t)n + 16 * MAX_BEAMS + 4 * LIST; }
};

// one CTA merges the lists of an item; `wait`: for the kernel that wrote them
__device__ __forceinline__ void merge(const BeamArgs &a, int item, bool wait) {
    Shared &sm = shared();
    const int beams = a.b.beams, V = a.b.vocab, k = a.b.k, slices = a.slices, n_lists = beams * slices, n_cand = n_lists * k;
    const Cand cd(reinterpret_cast<unsigned char *>(&sm) + (sizeof(Shared) + 15) / 16 * 16, n_cand);
    if (wait) {                            // (before the scores too: this kernel starts while the first one runs)
        pdl_wait();
        pdl_launch();
    }
    double cum = 0.0;
    bool done = false;
    if ((int)threadIdx.x < beams) {
        cum = a.b.scores[item * beams + threadIdx.x];
        done = a.b.finished && a.b.finished[item * beams + threadIdx.x];
    }
    if (threadIdx.x == 0) sm.count[0] = 0;
    const size_t list0 = (size_t)item * n_lists;
    for (int e = threadIdx.x; e < n_cand; e += THREADS) cd.key[e] = __ldcg(a.key + list0 * k + e);
    if ((int)threadIdx.x < beams) {
        // the row's log-sum-exp
        const bool number = cum > -INFINITY && cum < INFINITY;
        double lse = INFINITY;                                    // no candidates but those at -inf; -inf: finished
        if (done) lse = number ? -INFINITY : INFINITY;
        else if (number) {
            const size_t l0 = list0 + threadIdx.x * slices;
            float M = -INFINITY;
            for (int r = 0; r < slices; ++r) M = fmaxf(M, __ldcg(a.m + l0 + r));
            double S = 0.0;
            for (int r = 0; r < slices; ++r) {
                const float m = __ldcg(a.m + l0 + r);
                S += __ldcg(a.s + l0 + r) * (m == -INFINITY ? 1.0 : (double)ex2f((m - M) * LOG2E));
            }
            lse = (double)M + log(S);
            if (!(lse > -INFINITY && lse < INFINITY)) lse = INFINITY;
        }
        cd.lse[threadIdx.x] = lse;
        cd.cum[threadIdx.x] = cum;
    }
    __syncthreads();
    u64 best = 0;
    for (int e = threadIdx.x; e < n_cand; e += THREADS) {
        const int list = e / k, i = e - list * k, beam = list / slices;
        const double c = cd.cum[beam], lse = cd.lse[beam];
        u64 key = cd.key[e];
        double score = -INFINITY;
        if (lse == INFINITY || lse == -INFINITY) {
            // one continuation (finished) or none; behind it the lowest tokens at -inf, in the beam's first list
            const int eos = a.b.eos, t = lse == INFINITY ? i : i == 0 ? eos : i - 1 + (i - 1 >= eos);
            if (lse == -INFINITY && i == 0) score = c;
            key = list == beam * slices && t < V ? make_key(0.f, t) : 0;
        } else if (key) {
            score = c + ((double)key_value(key) - lse);
        }
        const u64 bits = (u64)__double_as_longlong(score + 0.0), order = key ? (bits >> 63 ? ~bits : bits | (1ull << 63)) : 0;
        cd.key[e] = key;
        cd.score[e] = score;
        cd.order[e] = order;
        best = max(best, order);
    }
    // A score that at least k candidates reach, from the threads' best (0, when the threads have fewer than k), thins out many
    // candidates; a few are ranked as they are (128 of them: 1 us less).
    const bool thin = n_cand > THREADS / 2;
    if (thin) {
        const u64 bar = kth_of_threads(sm, best, k, min(32, (k + 3) / 4));
        for (int e = threadIdx.x; e < n_cand; e += THREADS)
            if (cd.order[e] && cd.order[e] >= bar) {
                const int at = atomicAdd(&sm.count[0], 1);
                if (at < LIST) { sm.list[at] = cd.order[e]; cd.index[at] = e; }
            }
    }
    __syncthreads();
    // those are ranked by counting; where they are too many (equal scores), all are
    const bool listed = thin && sm.count[0] <= LIST;
    const int total = listed ? sm.count[0] : n_cand;
    const u64 *order = listed ? sm.list : cd.order;
    for (int c = threadIdx.x; c < total; c += THREADS) {
        const u64 mine = order[c];
        if (!mine) continue;
        int above = 0, equal = 0;
#pragma unroll 8
        for (int o = 0; o < total; ++o) {
            above += order[o] > mine;
            equal += order[o] == mine;
        }
        if (above >= k) continue;
        const int e = listed ? cd.index[c] : c, beam = e / k / slices;
        const u64 key = cd.key[e];
        for (int o = 0; equal > 1 && o < total; ++o) {
            if (order[o] != mine || o == c) continue;
            const int e2 = listed ? cd.index[o] : o, b2 = e2 / k / slices;
            above += b2 < beam || (b2 == beam && cd.key[e2] > key);
        }
        if (above < k) {
            const size_t at = (size_t)item * k + above;
            a.b.out_scores[at] = (float)cd.score[e];
            a.b.out_tokens[at] = key_token(key);
            a.b.out_rows[at] = item * beams + beam;
        }
    }
}

template <typename T, bool FUSED>
__global__ void __launch_bounds__(THREADS, 1) beam_slice_kernel(const BeamArgs a) {
    Shared &sm = shared();
    const int row = blockIdx.y, k = a.b.k, list = row * a.slices + blockIdx.x;
    const int lo = (int)min((int64_t)blockIdx.x * a.slice, (int64_t)a.b.vocab), hi = (int)min((int64_t)lo + a.slice, (int64_t)a.b.vocab);
    pdl_wait();
    pdl_launch();
    float m = -INFINITY;
    double s = 0.0;
    int count = 0;
    if (lo < hi && !(a.b.finished && a.b.finished[row]))
        count = slice_best<T>(sm, reinterpret_cast<const T *>(a.b.logits) + row * a.b.row_stride, lo, hi, k, a.aligned, m, s);
    for (int i = threadIdx.x; i < k; i += THREADS) a.key[(size_t)list * k + i] = i < count ? sm.list[i] : 0;
    if (threadIdx.x == 0) { a.m[list] = m; a.s[list] = s; }
    if (FUSED) {
        cooperative_groups::this_cluster().sync();                // the item's lists are written
        if (blockIdx.x == 0 && row % a.b.beams == 0) merge(a, row / a.b.beams, false);
    }
}

__global__ void __launch_bounds__(THREADS) beam_merge_kernel(const BeamArgs a) { merge(a, blockIdx.x, true); }

template <typename T>
cudaError_t launch(const BeamArgs &a, cudaStream_t st) {
    constexpr size_t fixed = (sizeof(Shared) + 15) / 16 * 16;
    const size_t merge_bytes = fixed + Cand::bytes(a.b.beams * a.slices * a.b.k);
    cudaLaunchConfig_t cfg = {};
    cudaLaunchAttribute at[2];
    at[0].id = cudaLaunchAttributeProgrammaticStreamSerialization;
    at[0].val.programmaticStreamSerializationAllowed = 1;
    cfg.blockDim = dim3(THREADS);
    cfg.stream = st;
    cfg.attrs = at;
    cfg.numAttrs = 1;
    cfg.gridDim = dim3(a.slices, a.b.batch * a.b.beams);
    if (a.fused) {
        static SmemAttrOnce attr;
        static std::atomic<bool> big[DEL_MAX_DEVICES] = {};
        auto kern = beam_slice_kernel<T, true>;
        cudaError_t e = attr.set(kern, (int)(fixed + Cand::bytes(MAX_CLUSTER * MAX_K)));
        int dev = 0;
        if (e == cudaSuccess) e = cudaGetDevice(&dev);
        if (e != cudaSuccess) return e;
        if (a.slices * a.b.beams > 8 && !(dev < DEL_MAX_DEVICES && big[dev].load(std::memory_order_acquire))) {
            e = cudaFuncSetAttribute(kern, cudaFuncAttributeNonPortableClusterSizeAllowed, 1);
            if (e != cudaSuccess) return e;
            if (dev < DEL_MAX_DEVICES) big[dev].store(true, std::memory_order_release);
        }
        at[1].id = cudaLaunchAttributeClusterDimension;
        at[1].val.clusterDim.x = a.slices;
        at[1].val.clusterDim.y = a.b.beams;
        at[1].val.clusterDim.z = 1;
        cfg.numAttrs = 2;
        cfg.dynamicSmemBytes = merge_bytes;
        return cudaLaunchKernelEx(&cfg, kern, a);
    }
    cfg.dynamicSmemBytes = sizeof(Shared);
    cudaError_t e = cudaLaunchKernelEx(&cfg, beam_slice_kernel<T, false>, a);
    if (e != cudaSuccess) return e;
    static SmemAttrOnce attr;
    e = attr.set(beam_merge_kernel, (int)(fixed + Cand::bytes(MAX_CAND)));
    if (e != cudaSuccess) return e;
    // (the second kernel's CTAs are few and short: they start while the first drains, and wait for its end before they read)
    cfg.gridDim = dim3(a.b.batch);
    cfg.dynamicSmemBytes = merge_bytes;
    return cudaLaunchKernelEx(&cfg, beam_merge_kernel, a);
}

// CTAs per row: as many over all rows as the device has SMs, none with less than 2048 columns (a smaller slice is all latency),
// and no more candidates of an item than the merge holds
int slices_of(const del_beam &x, int n_sms) {
    int64_t n = n_sms / ((int64_t)x.batch * x.beams);
    const int64_t most = (x.vocab + 2047) / 2048, held = MAX_CAND / ((int64_t)x.beams * x.k);
    n = n < most ? n : most;
    n = n < held ? n : held;
    return n < 1 ? 1 : (int)n;
}

// The one-launch form: slices per row such that an item is a cluster, all of which are resident (B200: 15 of 8, 7 of 16), and no slice is
// longer than 32768 columns; 0: two launches, which spread the rows over more CTAs.  us on the device, one launch / two:
//                    1 x 4 fp32    1 x 4 bf16    2 x 4 fp32    2 x 4 bf16    4 x 4 fp32    4 x 4 bf16    7 x 4 fp32    7 x 4 bf16    1 x 8 fp32    4 x 8 bf16
//   vocab  32000      8.4 / 10.2    9.5 / 11.0    8.8 /  9.7   11.5 / 10.9    8.8 /  9.5   14.7 / 11.6    9.0 /  9.9   14.8 / 17.2   12.8 / 12.0   22.2 / 12.1
//          64128      9.4 / 11.6    9.3 / 12.5    9.7 / 11.5   13.1 / 13.2    9.9 /  9.6   13.1 / 11.5   10.0 / 10.8   14.8 / 17.4   14.7 / 14.3   24.0 / 12.2
//         128256     11.3 / 13.3   12.4 / 14.7   11.5 / 11.6   16.1 / 13.3   11.8 / 10.5   14.5 / 11.0   12.0 / 12.7   16.4 / 18.2   18.7 / 14.4   27.1 / 14.0
//         262144     14.2 / 13.3   15.0 / 14.6   14.7 / 12.8   16.5 / 13.0   14.8 / 12.7   18.5 / 13.1   15.6 / 16.5   19.0 / 21.1   24.1 / 15.6   32.2 / 17.8
// A second launch costs the host up to 4 us more where nothing else runs (1 x 4 x 8000: 8.6 us a call / 12.6).  The line is right for one
// to four beams of few items and errs to one launch where 4 items of 4 beams or any of 8 would have more CTAs in two (in 16 bits by 3 to 12 us).
int fused_slices(const del_beam &x) {
    if (x.beams > MAX_CLUSTER) return 0;
    const int most = (x.vocab + 2047) / 2048, n = MAX_CLUSTER / x.beams < most ? MAX_CLUSTER / x.beams : most;
    return x.batch <= (n * x.beams <= 8 ? 15 : 7) && x.vocab / n <= 32768 ? n : 0;
}

bool valid(const del_beam *x) {
    if (!x || (x->dtype != DEL_F32 && x->dtype != DEL_BF16 && x->dtype != DEL_F16)) return false;
    if (x->batch < 1 || x->batch > 65535 || x->beams < 1 || x->beams > MAX_BEAMS || x->vocab < 1 || x->vocab > (1 << 30)) return false;
    return x->k >= 1 && x->k <= MAX_K && (int64_t)x->beams * x->vocab >= x->k && (int64_t)x->batch * x->beams <= 65535;
}

// slices_of gives at most n_sms lists, or one per row, fused_slices at most 120: enough for any device of up to 1024 SMs
size_t workspace_bytes(const del_beam &x) {
    const size_t rows = (size_t)x.batch * x.beams, lists = rows > 1024 ? rows : 1024;
    return lists * (8 * (size_t)x.k + 16);
}

}  // namespace

extern "C" size_t del_beam_workspace_bytes(const del_beam *x) {
    return valid(x) ? workspace_bytes(*x) : 0;
}

extern "C" int del_beam_select(const del_beam *x, void *cuda_stream) {
    if (!valid(x) || !x->logits || !x->scores || !x->out_scores || !x->out_tokens || !x->out_rows || !x->workspace) return DEL_EINVAL;
    const int size = x->dtype == DEL_F32 ? 4 : 2;
    if (((uintptr_t)x->scores | (uintptr_t)x->out_scores | (uintptr_t)x->out_tokens | (uintptr_t)x->out_rows) & 3 || (uintptr_t)x->logits % size) return DEL_EINVAL;
    if ((uintptr_t)x->workspace & 15 || x->row_stride < x->vocab) return DEL_EINVAL;
    if (x->finished && (x->eos < 0 || x->eos >= x->vocab)) return DEL_EINVAL;
    const int n_sms = current_sms();
    if (!n_sms || n_sms > 1024) return DEL_ECUDA;
    BeamArgs a;
    memset(&a, 0, sizeof(a));
    a.b = *x;
    a.aligned = ((uintptr_t)x->logits & 15) == 0 && (x->row_stride * size) % 16 == 0;
    a.slices = fused_slices(*x);
    a.fused = a.slices > 0;
    if (!a.fused) a.slices = slices_of(*x, n_sms);
    a.slice = ((x->vocab + a.slices - 1) / a.slices + 7) / 8 * 8;
    if (x->workspace_bytes < workspace_bytes(*x)) return DEL_ENOSPC;
    const size_t lists = (size_t)x->batch * x->beams * a.slices;
    a.key = (u64 *)x->workspace;
    a.s = (double *)(a.key + lists * x->k);
    a.m = (float *)(a.s + lists);
    cudaStream_t st = (cudaStream_t)cuda_stream;
    const cudaError_t e = x->dtype == DEL_F32 ? launch<float>(a, st) : x->dtype == DEL_BF16 ? launch<bf16>(a, st) : launch<__half>(a, st);
    return e == cudaSuccess ? DEL_OK : DEL_ECUDA;
}
