// Beam search's selection (the step between two decode steps of a beam decoder, Section 4.1: beam
// 4; Figure 5: beams 4 to 20).  For every sentence the `beam` best continuations are taken from the
// candidates of all of its hypotheses:
//     a live hypothesis b offers every token v with       score_b + log Softmax(logits_b)[v],
//     a finished one offers itself, unchanged, with       score_b,
// ranked by score / ((5 + length) / 6)^alpha, ties to the lowest (slot, token).
//
// The logits are read once and that is what bounds the call; everything else is a few KB:
//   select_rows_kernel   CTA = (hypothesis, part of the vocabulary), in steps of 8 or 16 KB, the next step's logits on their way
//     into registers while a step is worked on.  A thread keeps the maximum and the sum of 2^(x log2(e) - M) of
//     its logits (float32 within a step, double across steps and threads).  The part's best `beam` logits come out without sorting it: the beam-th largest of the 256
//     threads' maxima in the first step is a lower bound T of the beam-th best logit, which hardly more than
//     `beam` logits of a step reach; those go to a list in shared memory, T is raised when the list fills up, and
//     at the end each key finds its own place by counting the ones above it.
//   select_merge_kernel  CTA = sentence.  Joins the parts' maxima and sums to the log-sum-exp of each row
//     (double: scores of different hypotheses are compared with one another), ranks the beam x parts
//     x beam candidates, 1024 at a time, the best of every part first, until the parts' next ones cannot matter, and carries
//     scores, lengths and token histories over.  It is launched with programmatic stream serialisation: its
//     CTAs are in place, and the histories in shared memory, when the last logits arrive.
//     Part after part in place of the best first took every pass: one sentence of 32 rows of 128000 float32 86 us, 29 so (24 with the longer steps that it has now).
//     Both in one launch, a sentence's CTAs as a cluster whose first CTA went on behind the cluster's barrier, was slower
//     (device time: 4 rows of 32000 float32 10.3 us against 8.8, 256 of bf16 16.0 against 14.9, 512 of 128000 47.6 against 42.4).
// Measured (device time of the whole call): 512 rows of 128000 bf16 logits 41.2 us, issue slots and the
// units of the exponentials half full each (ten thread instructions a logit, of which the sum and the maximum need some four; what the
// others do has not been measured part by part); 740 rows of 50257 float32 ones off 16-byte boundaries 47.2 (twenty-two a logit:
// single loads, short steps, more listing), of bf16 ones 59.8 (two-byte loads, 104 bytes of registers spilled); 4 rows of
// 32000 7.6, the chain of one sentence.  The first
// version, which sorted a key per thread and held 32 logits in float32, took 162, 133 and 12.3.  A ring of cp.async stages in
// shared memory in place of the registers measured the same: loads are not what is waited for.
// Where more candidates reach the bound than the list holds (rows that are alike nearly everywhere: a mask of
// the type's lowest value) the best ones are taken one by one, each the largest below the one before.
// A finished hypothesis, or one without a score, has its logits skipped.
#pragma once

#include <cfloat>

#include "san_kernels.cuh"

namespace san {

constexpr int kSelThreads = 256;
constexpr int kSelWarps = kSelThreads / 32;
// 32-bit words of logits per thread and step (W), and the CTAs of the rows' kernel that an SM holds with so many (registers are
// limited for that).  Steps of 16 words are the faster ones but where one wave of CTAs with 8 takes rows that need two with 16.
// Measured for float32, time with 8 words over time with 16, rows of 32000 to 50257 (beam 1): 200 rows 1.05 to 1.12,
// 400 1.21 to 1.26, 592 1.08 to 1.12, 600 0.96 to 0.99, 740 0.92 to 0.94, 741 1.07 to 1.17, 888 1.09 to 1.23, 1184 1.13 to 1.15,
// 1480 0.99 to 1.01, 2220 1.04 to 1.05; 740 rows of beam 20 47.3 us against 53.3.  bf16: 512 rows of 128000 48.5 us with 8 words, 42.4
// with 16 (before the merge took what it takes now).
constexpr int kSelWordsLong = 16, kSelWordsShort = 8;
constexpr int select_ctas(int words) { return words == kSelWordsLong ? 4 : 5; }
constexpr int kSelList = 1024;                 // keys that may reach the bound between two checks; more: one by one
constexpr int kSelLong = 96;                   // list length at which the bound is raised
constexpr int kSelTight = 64;                  // what the list is cut down to (equal logits aside)
constexpr int kSelMaxTokens = 0x7fff0000;      // of a history: a window of the merge behind it is still within 32 bits
constexpr int TAG_SELECT = 8;

struct SelectParams {
    const void* logits; long long ld;          // elements between rows
    int vocab, n_sent, beam, chunks, steps, eos;     // steps of a chunk (a part of a row)
    double alpha;
    const float* score; const int* len; const int* done;
    const int* tokens; long long ld_tokens;
    float* score_out; int* len_out; int* done_out; int* tokens_out; int* parent; int* next;
    char* ws;                                  // per (row, chunk): max, sum, best keys
    int* status;
};
__host__ __device__ inline size_t select_part_bytes(int beam) { return 16 + 8 * (size_t)beam; }

// A hypothesis that offers nothing: no score (a beam slot not in use yet).
__device__ __forceinline__ bool select_dead(float score) { return !(score > -INFINITY && score < INFINITY); }

__device__ __forceinline__ void select_error(int* status, int item, int value, int limit) {
    if (status) record_error(status, TAG_SELECT, item, value, limit);
}

// Order-preserving map of a float to an unsigned number; -0 and +0 are one value.
__device__ __forceinline__ unsigned order_f32(float x) {
    const unsigned u = __float_as_uint(x + 0.0f);
    return u & 0x80000000u ? ~u : u | 0x80000000u;
}
__device__ __forceinline__ float unorder_f32(unsigned u) {
    return __uint_as_float(u & 0x80000000u ? u & 0x7fffffffu : ~u);
}
__device__ __forceinline__ double unorder_f64(unsigned long long u) {
    return __longlong_as_double((long long)(u >> 63 ? u & ~(1ull << 63) : ~u));
}
__device__ __forceinline__ unsigned long long order_f64(double x) {
    const unsigned long long u = (unsigned long long)__double_as_longlong(x + 0.0);
    return u >> 63 ? ~u : u | (1ull << 63);
}

// Keys, largest first.  Zero stands for "none".
struct Key64 {
    unsigned long long a;
    __device__ __forceinline__ bool over(const Key64& o) const { return a > o.a; }
    __device__ __forceinline__ Key64 swapped(int mask) const { return {__shfl_xor_sync(0xffffffffu, a, mask)}; }
};
struct Key128 {
    unsigned long long a, b;
    __device__ __forceinline__ bool over(const Key128& o) const { return (a > o.a) | ((a == o.a) & (b > o.b)); }
    __device__ __forceinline__ Key128 swapped(int mask) const {
        return {__shfl_xor_sync(0xffffffffu, a, mask), __shfl_xor_sync(0xffffffffu, b, mask)};
    }
};
template <typename K> __device__ __forceinline__ K larger(const K& x, const K& y) { return y.over(x) ? y : x; }

// The CTA's largest key, in all threads.  `slots`: kSelWarps keys of shared memory, free again after the next barrier.
template <typename K> __device__ __forceinline__ K block_largest(K k, K* slots) {
#pragma unroll
    for (int o = 16; o > 0; o >>= 1) k = larger(k, k.swapped(o));
    __syncthreads();
    if ((threadIdx.x & 31) == 0) slots[threadIdx.x >> 5] = k;
    __syncthreads();
    k = slots[0];
#pragma unroll
    for (int w = 1; w < kSelWarps; ++w) k = larger(k, slots[w]);
    return k;
}

// From one value per thread, the thread's largest: its warp's largest, and what the warp adds to a lower bound of the
// CTA's n-th largest value.  Up to n = 8 each warp has at least n groups of lanes of its own, and the largest of the
// warps' least maxima serves; beyond that all warps together have 16 or 32 groups and the least maximum serves.
template <typename V> __device__ __forceinline__ void group_bounds(V top, int n, V* warp_top, V* warp_least) {
    const int groups = n <= 1 ? 1 : n <= 2 ? 2 : n <= 4 ? 4 : n <= 8 ? 8 : n <= 16 ? 2 : 4;     // of this warp
    const int width = 32 / groups;
    V least = top;
#pragma unroll
    for (int o = 1; o < 32; o <<= 1) {
        const V other = __shfl_xor_sync(0xffffffffu, top, o);
        const V other_least = __shfl_xor_sync(0xffffffffu, least, o);
        top = other > top ? other : top;
        least = o < width ? top : other_least < least ? other_least : least;
    }
    *warp_top = top; *warp_least = least;
}
template <typename V> __device__ __forceinline__ V join_bounds(const V* warp_least, int n) {
    V t = warp_least[0];
#pragma unroll
    for (int w = 1; w < kSelWarps; ++w) t = (warp_least[w] > t) == (n <= 8) ? warp_least[w] : t;
    return t;
}

// Gives the n largest of `count` different keys to out(place, key); the list is in shared memory.  Up to 32 threads
// count the keys above one, as many as there are for each.
template <typename K, typename F> __device__ __forceinline__ void rank_list(const K* list, int count, int n, F out) {
    int per = kSelThreads;
    while (per > 1 && (per > 32 || per * count > kSelThreads)) per >>= 1;
    const int part = threadIdx.x & (per - 1);
    for (int first = 0; first < count; first += kSelThreads / per) {
        const int i = first + (int)threadIdx.x / per;
        const K mine = list[min(i, count - 1)];
        int above = 0;
#pragma unroll 4
        for (int j = part; j < count; j += per) above += list[j].over(mine) ? 1 : 0;
        for (int o = 1; o < per; o <<= 1) above += __shfl_xor_sync(0xffffffffu, above, o);
        if (i < count && above < n && part == 0) out(above, mine);
    }
}
// The same for longer lists: eight threads count for four keys at a time, so that a key read serves four.  (144 keys: 8000
// clocks with a thread a key.)
template <typename K, typename F> __device__ __forceinline__ void rank_long_list(const K* list, int count, int n, F out) {
    const int part = threadIdx.x & 7, group = threadIdx.x >> 3, groups = kSelThreads / 8;
    for (int first = 0; first < count; first += 4 * groups) {
        K mine[4];
        int above[4] = {0, 0, 0, 0};
#pragma unroll
        for (int e = 0; e < 4; ++e) mine[e] = list[min(first + group + e * groups, count - 1)];
#pragma unroll 2
        for (int j = part; j < count; j += 8) {
            const K other = list[j];
#pragma unroll
            for (int e = 0; e < 4; ++e) above[e] += other.over(mine[e]) ? 1 : 0;
        }
#pragma unroll
        for (int e = 0; e < 4; ++e) {
            for (int o = 1; o < 8; o <<= 1) above[e] += __shfl_xor_sync(0xffffffffu, above[e], o);
            if (part == e && first + group + e * groups < count && above[e] < n) out(above[e], mine[e]);
        }
    }
}

template <typename T> __device__ __forceinline__ float as_f32(T x);
template <> __device__ __forceinline__ float as_f32<float>(float x) { return x; }
template <> __device__ __forceinline__ float as_f32<__nv_bfloat16>(__nv_bfloat16 x) { return __bfloat162float(x); }

// The logits of a thread in one step: W registers, eight logits at a time.
template <typename T, int W> struct SelectHeld;
template <int W> struct SelectHeld<float, W> {
    static constexpr int kWords = W, N = kWords;
    float x[kWords];
    __device__ __forceinline__ void set(int i, float v) { x[i] = v; }
    __device__ __forceinline__ void set16(int j, const uint4& v) {
        x[4 * j] = __uint_as_float(v.x); x[4 * j + 1] = __uint_as_float(v.y);
        x[4 * j + 2] = __uint_as_float(v.z); x[4 * j + 3] = __uint_as_float(v.w);
    }
    __device__ __forceinline__ float get(int i) const { return x[i]; }
    __device__ __forceinline__ void mask_nan() {
#pragma unroll
        for (int i = 0; i < kWords; ++i) x[i] = fmaxf(x[i], -INFINITY);
    }
    __device__ __forceinline__ float pick8(int g, int e) const {      // logit 8 g + e
        const float a = e & 1 ? x[8 * g + 1] : x[8 * g], b = e & 1 ? x[8 * g + 3] : x[8 * g + 2];
        const float c = e & 1 ? x[8 * g + 5] : x[8 * g + 4], d = e & 1 ? x[8 * g + 7] : x[8 * g + 6];
        return e & 4 ? (e & 2 ? d : c) : (e & 2 ? b : a);
    }
    // The largest of logits 8 g .. 8 g + 7, NaN if one of them is.
    __device__ __forceinline__ float top8(int g) const {
        float t = x[8 * g];
#pragma unroll
        for (int i = 1; i < 8; ++i) asm("max.NaN.f32 %0, %0, %1;" : "+f"(t) : "f"(x[8 * g + i]));
        return t;
    }
};
template <int W> struct SelectHeld<__nv_bfloat16, W> {
    static constexpr int kWords = W, N = 2 * kWords;
    uint32_t x[kWords];                                            // logit 2 i low, 2 i + 1 high
    __device__ __forceinline__ void set(int i, float v) {
        const uint32_t b = __float_as_uint(v) >> 16;                  // v is a bf16 number
        x[i >> 1] = i & 1 ? (x[i >> 1] & 0xffffu) | b << 16 : b;
    }
    __device__ __forceinline__ void set16(int j, const uint4& v) { x[4 * j] = v.x; x[4 * j + 1] = v.y; x[4 * j + 2] = v.z; x[4 * j + 3] = v.w; }
    __device__ __forceinline__ float get(int i) const { return __uint_as_float(i & 1 ? x[i >> 1] & 0xffff0000u : x[i >> 1] << 16); }
    __device__ __forceinline__ static __nv_bfloat162 two(uint32_t w) { return *reinterpret_cast<__nv_bfloat162*>(&w); }
    __device__ __forceinline__ void mask_nan() {
#pragma unroll
        for (int i = 0; i < kWords; ++i) {
            const __nv_bfloat162 v = __hmax2(two(x[i]), two(0xff80ff80u));
            x[i] = *reinterpret_cast<const uint32_t*>(&v);
        }
    }
    __device__ __forceinline__ float pick8(int g, int e) const {
        const uint32_t a = e & 2 ? x[4 * g + 1] : x[4 * g], b = e & 2 ? x[4 * g + 3] : x[4 * g + 2], w = e & 4 ? b : a;
        return __uint_as_float(e & 1 ? w & 0xffff0000u : w << 16);
    }
    __device__ __forceinline__ float top8(int g) const {
        const __nv_bfloat162 t = __hmax2_nan(__hmax2_nan(two(x[4 * g]), two(x[4 * g + 1])), __hmax2_nan(two(x[4 * g + 2]), two(x[4 * g + 3])));
        float r = __low2float(t);
        asm("max.NaN.f32 %0, %0, %1;" : "+f"(r) : "f"(__high2float(t)));
        return r;
    }
};

// Two float32 numbers in one instruction.
__device__ __forceinline__ unsigned long long pair_f32(float x, float y) {
    unsigned long long r;
    asm("mov.b64 %0, {%1, %2};" : "=l"(r) : "f"(x), "f"(y));
    return r;
}
__device__ __forceinline__ void unpair_f32(unsigned long long r, float& x, float& y) { asm("mov.b64 {%0, %1}, %2;" : "=f"(x), "=f"(y) : "l"(r)); }
__device__ __forceinline__ unsigned long long fma_f32x2(unsigned long long a, unsigned long long b, unsigned long long c) {
    unsigned long long d;
    asm("fma.rn.f32x2 %0, %1, %2, %3;" : "=l"(d) : "l"(a), "l"(b), "l"(c));
    return d;
}
__device__ __forceinline__ unsigned long long add_f32x2(unsigned long long a, unsigned long long b) {
    unsigned long long d;
    asm("add.rn.f32x2 %0, %1, %2;" : "=l"(d) : "l"(a), "l"(b));
    return d;
}
__device__ __forceinline__ float exp2_fast(float x) {
    float y;
    asm("ex2.approx.ftz.f32 %0, %1;" : "=f"(y) : "f"(x));
    return y;
}
__device__ __forceinline__ unsigned long long select_key(float x, int index) {       // x > -inf
    return ((unsigned long long)order_f32(x) << 32) | (unsigned)~index;
}

// One warp: of the `count` keys of the list keeps those that reach a bound raised, from `lo` on, until at most
// kSelTight do (never fewer than n).  Returns the bound; *left: keys left, packed together.
__device__ __forceinline__ uint32_t tighten(Key64* list, int count, int n, uint32_t lo, int* left, int lane) {
    uint32_t hi = 0;
    for (int j = lane; j < count; j += 32) hi = max(hi, (uint32_t)(list[j].a >> 32));
    hi = __reduce_max_sync(0xffffffffu, hi);
    int have = count;
    while (have > kSelTight && hi > lo) {
        const uint32_t mid = lo + (hi - lo + 1) / 2;
        int k = 0;
        for (int j = lane; j < count; j += 32) k += (uint32_t)(list[j].a >> 32) >= mid ? 1 : 0;
        k = __reduce_add_sync(0xffffffffu, k);
        if (k >= n) { lo = mid; have = k; } else hi = mid - 1;
    }
    int at = 0;
    for (int j = 0; j < count; j += 32) {
        const Key64 k = list[min(j + lane, count - 1)];
        const unsigned keeps = __ballot_sync(0xffffffffu, j + lane < count && (uint32_t)(k.a >> 32) >= lo);
        if (keeps >> lane & 1) list[at + __popc(keeps & ((1u << lane) - 1))] = k;      // at or before what was just read
        at += __popc(keeps);
        __syncwarp();
    }
    *left = at;
    return lo;
}

// grid = rows * chunks, then select_merge_kernel.  VECTOR: every row starts on a 16-byte boundary and a thread holds runs
// of 16 bytes, else single logits 256 apart (one mapping for all rows of a call, so that equal rows get equal sums
// whatever their addresses).
template <typename T, bool VECTOR, int W>
__global__ void __launch_bounds__(kSelThreads, select_ctas(W)) select_rows_kernel(const SelectParams p) {
    asm volatile("griddepcontrol.launch_dependents;");
    using Held = SelectHeld<T, W>;
    constexpr int N = Held::N, VEC = VECTOR ? 16 / (int)sizeof(T) : 1, STEP = N * kSelThreads;
    __shared__ Key64 s_list[kSelList];
    __shared__ Key64 s_slots[kSelWarps];
    __shared__ float s_max[kSelWarps], s_least[kSelWarps];
    __shared__ double s_sum[kSelWarps];
    __shared__ int s_count;
    __shared__ uint32_t s_bound;
    const int row = (int)(blockIdx.x / (unsigned)p.chunks), chunk = (int)(blockIdx.x % (unsigned)p.chunks);
    if (select_dead(p.score[row]) || p.done[row] != 0) return;        // uniform over the CTA
    const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
    const T* x = static_cast<const T*>(p.logits) + (long long)row * p.ld;
    const int begin = min(chunk * p.steps * STEP, p.vocab), end = (int)min((long long)begin + (long long)p.steps * STEP, (long long)p.vocab);

    auto load = [&](Held& v, int base) {
        if (base + STEP <= end) {                                     // a whole step: no bounds
            const T* at = x + base + (int)threadIdx.x * VEC;
#pragma unroll
            for (int j = 0; j < N / VEC; ++j) {
                if constexpr (VECTOR) v.set16(j, ld16_stream(at + j * kSelThreads * VEC));
                else v.set(j, as_f32<T>(at[j * kSelThreads]));
            }
            return;
        }
#pragma unroll
        for (int j = 0; j < N / VEC; ++j) {
            const int at = base + (j * kSelThreads + (int)threadIdx.x) * VEC;
            if constexpr (VECTOR) {
                if (at + VEC <= end) {
                    v.set16(j, ld16_stream(x + at));
                } else {
#pragma unroll
                    for (int e = 0; e < VEC; ++e) v.set(j * VEC + e, at + e < end ? as_f32<T>(x[at + e]) : -INFINITY);
                }
            } else {
                v.set(j, at < end ? as_f32<T>(x[at]) : -INFINITY);
            }
        }
    };
    // Sum of e^(x - top): the terms of a step in float32 (8 to 32 of them, four partial sums), the steps in double, so that
    // the additions' roundings do not grow with the row (in float32 throughout: 512 rows of 128000 bf16 logits off by up
    // to 7e-6, 592 of 2^20 by 5e-5, but 1.3 us less
    // for either measured case).  Terms are 2^(c x - M), c = fl(log2 e): the arguments are rounded once,
    // relative to themselves (the product is exact inside the FMA), and 2^(M - c top) is put right at the end.  M is the
    // rounded c top of some step before and moves when the maximum has grown by 2^4 since, so that what a
    // rescaling is off by shrinks faster than rescalings come.  A maximum so large that c x could be infinite, or infinite
    // itself: only logits equal to it count.
    constexpr float c = 1.4426950408889634f;
    float top = -INFINITY, m = 0.f;
    double part = 0.0;
    float bound = -INFINITY;
    if (threadIdx.x == 0) s_count = 0;
    int step = 0;
    Held next;
    load(next, begin);
    for (int base = begin; base < end; base += STEP) {
        Held v = next;
        if (base + STEP < end) load(next, base + STEP);
        float t8[N / 8], t = -INFINITY;
        auto largest = [&]() {
            t = -INFINITY;
#pragma unroll
            for (int g = 0; g < N / 8; ++g) { t8[g] = v.top8(g); asm("max.NaN.f32 %0, %0, %1;" : "+f"(t) : "f"(t8[g])); }
        };
        largest();
        if (t != t) {                                                 // masked tokens among them: -inf from here on
            v.mask_nan();
            largest();
        }
        if (t > top) {
            if (!(fabsf(top) < 1e30f && fabsf(t) < 1e30f)) {
                part = 0.0;
                m = t * c;
            } else if (fmaf(t, c, -m) > 4.f) {
                const float m_new = t * c;
                part *= (double)exp2_fast(m - m_new);
                m = m_new;
            }
            top = t;
        }
        if (fabsf(top) < 1e30f) {
            unsigned long long sum[2] = {0ull, 0ull};
            const unsigned long long c2 = pair_f32(c, c), m2 = pair_f32(-m, -m);
#pragma unroll
            for (int i = 0; i < N; i += 2) {
                float y, z;
                unpair_f32(fma_f32x2(pair_f32(v.get(i), v.get(i + 1)), c2, m2), y, z);
                sum[(i >> 1) & 1] = add_f32x2(sum[(i >> 1) & 1], pair_f32(exp2_fast(y), exp2_fast(z)));
            }
            float y, z;
            unpair_f32(add_f32x2(sum[0], sum[1]), y, z);
            part += (double)(y + z);
        } else if (top > -INFINITY) {
            float equal = 0.f;
#pragma unroll
            for (int i = 0; i < N; ++i) equal += v.get(i) == top ? 1.f : 0.f;
            part += (double)equal;
        }
        if (base == begin) {
            // The first bound: the beam-th largest of the threads' maxima, or a little below it, found by halving the
            // way from the groups' bound to the largest; some `beam` to 2 beam + 8 logits of the step reach it.
            float wtop, least;
            group_bounds(t, p.beam, &wtop, &least);
            if (lane == 0) { s_least[warp] = least; s_max[warp] = wtop; }
            __syncthreads();
            float most = s_max[0];
#pragma unroll
            for (int w = 1; w < kSelWarps; ++w) most = fmaxf(most, s_max[w]);
            const uint32_t mine = order_f32(t);
            uint32_t lo = order_f32(join_bounds(s_least, p.beam)), hi = order_f32(most);
            for (int count = kSelThreads; count > 2 * p.beam + 8 && hi > lo; ) {
                const uint32_t mid = lo + (hi - lo + 1) / 2;
                const int n = __syncthreads_count(mine >= mid);
                if (n >= p.beam) { lo = mid; count = n; } else hi = mid - 1;
            }
            bound = unorder_f32(lo);
        }
        const float least = fmaxf(bound, -FLT_MAX);                   // -inf offers nothing
        if (t >= least) {
#pragma unroll
            for (int g = 0; g < N / 8; ++g) {
                if (!(t8[g] >= least)) continue;
                // A warp's lanes list their hits together, one each in turn: a branch per logit would take the hits of
                // different places one after another.
                unsigned hits = 0;
#pragma unroll
                for (int i = 0; i < 8; ++i) hits |= v.get(8 * g + i) >= least ? 1u << i : 0u;
                for (; hits; hits &= hits - 1) {
                    const int e = __ffs((int)hits) - 1, i = 8 * g + e, at = atomicAdd(&s_count, 1);
                    if (at < kSelList) s_list[at].a = select_key(v.pick8(g, e), base + ((i / VEC) * kSelThreads + (int)threadIdx.x) * VEC + i % VEC);
                }
            }
        }
        // The list is looked at every fourth step: some hundred keys come in between.
        if ((++step & 3) != 0 || base + STEP >= end) continue;
        __syncthreads();
        const int count = s_count;
        __syncthreads();
        if (count > kSelList) {                                       // keys were lost: only the sums go on
            bound = INFINITY;
        } else if (count > kSelLong) {
            if (warp == 0) {
                int left;
                const uint32_t b = tighten(s_list, count, p.beam, order_f32(bound), &left, lane);
                if (lane == 0) { s_count = left; s_bound = b; }
            }
            __syncthreads();
            bound = unorder_f32(s_bound);
        }
    }
    __syncthreads();
    // 2^(M - c top).  The maximum's own term alone counts as 1 whatever it was rounded to (a row of one token has the sum 1), and
    // rounding to float32 once lets the two exponentials' errors cancel where they are one another's reverse: rows with the same
    // terms under another maximum mostly have the same sum.  (A division by that term: 3 to 15 us more for the cases above.)
    if (fabsf(top) < 1e30f) {
        const float rest = fmaf(top, c, -m);
        part = part == (double)exp2_fast(rest) ? 1.0 : (double)((float)part * exp2_fast(-rest));
    }
    const float wtop = warp_max(top);
    double wsum = part == 0.0 || top == wtop ? part : part * (double)exp2_fast((top - wtop) * c);
#pragma unroll
    for (int o = 16; o > 0; o >>= 1) wsum += __shfl_xor_sync(0xffffffffu, wsum, o);
    if (lane == 0) { s_max[warp] = wtop; s_sum[warp] = wsum; }
    int count = s_count;
    if (count > kSelTight && count <= kSelList && warp == 0) {
        int left;
        tighten(s_list, count, p.beam, order_f32(bound), &left, lane);
        if (lane == 0) s_count = left;
    }
    __syncthreads();
    char* out = p.ws + (size_t)blockIdx.x * select_part_bytes(p.beam);
    if (warp == kSelWarps - 1) {
        float t = lane < kSelWarps ? s_max[lane] : -INFINITY;
        double s = lane < kSelWarps ? s_sum[lane] : 0.0;
        const float all = warp_max(t);
        s = s == 0.0 || t == all ? s : s * (double)exp2_fast((t - all) * c);
#pragma unroll
        for (int o = kSelWarps / 2; o > 0; o >>= 1) s += __shfl_xor_sync(0xffffffffu, s, o);
        if (lane == 0) {
            *reinterpret_cast<float*>(out) = all;
            *reinterpret_cast<double*>(out + 8) = s;
        }
    }
    Key64* best = reinterpret_cast<Key64*>(out + 16);
    if (count <= kSelList) {
        count = s_count;
        rank_list(s_list, count, p.beam, [&](int place, const Key64& k) { best[place] = k; });
        for (int i = count + (int)threadIdx.x; i < p.beam; i += kSelThreads) best[i] = Key64{0};
        return;
    }
    Key64 last{~0ull};
    for (int k = 0; k < p.beam; ++k) {                                // read once more for every place (from L2)
        Key64 mine{0};
#pragma unroll 8
        for (int at = begin + (int)threadIdx.x; at < end; at += kSelThreads) {
            const float f = as_f32<T>(x[at]);
            const Key64 y{f > -INFINITY ? select_key(f, at) : 0ull};
            if (last.over(y)) mine = larger(mine, y);
        }
        last = block_largest(mine, s_slots);
        if (threadIdx.x == 0) best[k] = last;
    }
}

constexpr int kMergeHeld = 4;                  // candidates per thread and pass
constexpr int kMergeShort = 64;                // candidates up to which a few threads count for each
constexpr int kMergeHistory = 4096;            // tokens of the histories in shared memory at once

__device__ __forceinline__ void copy4_async(int* dst, const int* src) {
    asm volatile("cp.async.ca.shared.global [%0], [%1], 4;" ::"r"((unsigned)__cvta_generic_to_shared(dst)), "l"(src) : "memory");
}

// grid = sentences.
static __global__ void __launch_bounds__(kSelThreads) select_merge_kernel(const SelectParams p) {
    __shared__ Key128 s_list[kSelThreads * kMergeHeld];
    __shared__ int s_history[kMergeHistory];
    __shared__ Key128 s_best[2][SAN_MAX_BEAM];
    __shared__ unsigned long long s_least[kSelWarps], s_most[kSelWarps], s_rank[SAN_MAX_BEAM];
    __shared__ int s_counts[2][kSelWarps];
    __shared__ Key128 s_slots[kSelWarps];
    __shared__ float s_score[SAN_MAX_BEAM], s_top[SAN_MAX_BEAM];
    __shared__ double s_logsum[SAN_MAX_BEAM], s_norm[SAN_MAX_BEAM], s_inverse[SAN_MAX_BEAM];
    __shared__ int s_len[SAN_MAX_BEAM], s_done[SAN_MAX_BEAM], s_parent[SAN_MAX_BEAM], s_token[SAN_MAX_BEAM];
    __shared__ int s_count, s_bad, s_longest;
    const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
    const int sent = blockIdx.x, beam = p.beam;
    if (threadIdx.x == 0) { s_count = 0; s_bad = 0; s_longest = 0; }
    __syncthreads();
    if (threadIdx.x < beam) {
        const int b = threadIdx.x, row = sent * beam + b;
        const float score = p.score[row];
        const int len = p.len[row], done = p.done[row] != 0;
        const bool dead = select_dead(score);
        s_score[b] = dead ? -INFINITY : score; s_len[b] = len; s_done[b] = done;
        s_norm[b] = p.alpha == 0.0 ? 1.0 : pow((5.0 + (double)(len + (done ? 0 : 1))) / 6.0, p.alpha);
        s_inverse[b] = 1.0 / s_norm[b];
        s_parent[b] = b; s_token[b] = -1;
        const long long limit = p.tokens ? p.ld_tokens : 0x7ffffffe;
        // Scores come back out of ranks by a product with the norm: neither a float32 score over it nor one of its ranks may
        // leave the normal numbers (2^-149 / 10^250 = 10^-295; 2^128 * 10^250 = 10^289).
        const bool scale = dead || (s_norm[b] >= 1e-250 && s_norm[b] <= 1e250);
        if (len < 0 || len > limit || (len == limit && !done && !dead) || !scale) {
            s_bad = 1;
            select_error(p.status, row, len, (int)limit);
        }
        atomicMax(&s_longest, len);
    }
    __syncthreads();
    // Histories, `span` positions at a time; the first ones are on their way while the rows are worked on.
    const int span = kMergeHistory / beam & ~31, longest = p.tokens ? (int)min((long long)s_longest + 1, p.ld_tokens) : 0;
    auto fetch = [&](int first) {
        for (int b = warp; b < beam; b += kSelWarps) {
            const int* from = p.tokens + ((long long)sent * beam + b) * p.ld_tokens;
            for (int pos = first + lane; pos < min(first + span, s_len[b]); pos += 32) copy4_async(s_history + b * span + pos - first, from + pos);
        }
    };
    if (longest > 0 && !s_bad) fetch(0);
    asm volatile("griddepcontrol.wait;" ::: "memory");
    if (s_bad) return;                                                // the sentence keeps its old state
    const size_t part_bytes = select_part_bytes(beam);
    const char* parts = p.ws + (size_t)sent * beam * p.chunks * part_bytes;
    // candidate i of the sentence: (place, slot, chunk), so that the best ones of every part come first; a finished
    // hypothesis stands at its first one
    const int n_parts = p.chunks * beam, total = beam * n_parts;
    auto slot_of = [&](int i) { return (int)((unsigned)i % (unsigned)n_parts / (unsigned)p.chunks); };
    unsigned long long held[kMergeHeld];
    auto load = [&](int first) {
#pragma unroll
        for (int j = 0; j < kMergeHeld; ++j) {
            const int i = first + j * kSelThreads + (int)threadIdx.x;
            held[j] = 0;
            if (i >= total) continue;
            const int place = (unsigned)i / (unsigned)n_parts, part = i - place * n_parts, b = (unsigned)part / (unsigned)p.chunks;
            if (s_score[b] == -INFINITY) continue;
            if (s_done[b]) held[j] = i == b * p.chunks ? 1 : 0;       // itself
            else held[j] = *reinterpret_cast<const unsigned long long*>(parts + (size_t)part * part_bytes + 16 + 8 * (size_t)place);
        }
    };
    load(0);
    // log of each row's sum of exponentials: as many lanes for a row as it has parts (32 at most)
    int width = 1;
    while (width < 32 && width < p.chunks) width <<= 1;
    for (int b0 = warp * (32 / width); b0 < beam; b0 += kSelWarps * (32 / width)) {
        const int b = b0 + lane / width, c = lane & (width - 1);
        const bool row = b < beam && !s_done[min(b, beam - 1)] && s_score[min(b, beam - 1)] > -INFINITY;
        const char* part = parts + (size_t)min(b, beam - 1) * p.chunks * part_bytes;
        float m = -INFINITY;
        double s = 0.0;
        for (int c0 = 0; c0 < p.chunks; c0 += width) {
            const bool have = row && c0 + c < p.chunks;
            const float mc = have ? *reinterpret_cast<const float*>(part + (c0 + c) * part_bytes) : -INFINITY;
            const double sc = have ? *reinterpret_cast<const double*>(part + (c0 + c) * part_bytes + 8) : 0.0;
            float m_new = mc;
            for (int o = 1; o < width; o <<= 1) m_new = fmaxf(m_new, __shfl_xor_sync(0xffffffffu, m_new, o));
            m_new = fmaxf(m, m_new);
            double t = mc == -INFINITY ? 0.0 : mc == m_new ? sc : sc * (double)exp2_fast((mc - m_new) * 1.4426950408889634f);
            for (int o = 1; o < width; o <<= 1) t += __shfl_xor_sync(0xffffffffu, t, o);
            s = (m == -INFINITY ? 0.0 : m == m_new ? s : s * (double)exp2_fast((m - m_new) * 1.4426950408889634f)) + t;
            m = m_new;
        }
        if (row && c == 0) { s_top[b] = m; s_logsum[b] = log(s); }
    }
    __syncthreads();
    auto score_of = [&](int b, float x) {
        const double d = x == s_top[b] ? 0.0 : (double)x - (double)s_top[b];
        return (double)s_score[b] + (d - s_logsum[b]);
    };
    int kept = 0;                                                     // candidates kept from the passes before
    int idle = 0;                                                     // candidates in a row, the last ones, that are below the ones kept
    for (int first = 0, turn = 0; first < total; first += kSelThreads * kMergeHeld, turn ^= 1) {
        if (first > 0) load(first);
        auto score_at = [&](int b, unsigned long long h) { return s_done[b] ? (double)s_score[b] : score_of(b, unorder_f32((unsigned)(h >> 32))); };
        auto exact = [&](int b, unsigned long long h) {                   // the key that orders the sentence's candidates
            const double rank = score_at(b, h) / s_norm[b];
            const int token = s_done[b] ? max(p.eos, 0) : (int)~(unsigned)h;
            return Key128{rank > -INFINITY ? order_f64(rank) : 0, ~(((unsigned long long)(unsigned)b << 32) | (unsigned)token)};
        };
        auto list = [&](bool in, const Key128& k) {
            const unsigned all = __ballot_sync(0xffffffffu, in);
            int at = 0;
            if (lane == 0 && all) at = atomicAdd(&s_count, __popc(all));
            at = __shfl_sync(0xffffffffu, at, 0) + __popc(all & ((1u << lane) - 1));
            if (in) s_list[at] = k;
        };
        unsigned long long key[kMergeHeld];
        if (total <= kSelThreads) {                                   // one a thread
            Key128 k{0, 0};
            if (held[0] != 0) k = exact(slot_of((int)threadIdx.x), held[0]);
            // Only the best ones are listed, found by the upper halves of their ranks: 87 sentences x 12
            // rows of 1549, 144 candidates each, take 22.9 us so and 26.9 with all of them ordered.
            const unsigned upper = (unsigned)(k.a >> 32);
            unsigned bound = 1;
            int have = __syncthreads_count(upper >= bound);
            if (have > kMergeShort) {
                unsigned warp_top, least;
                group_bounds(upper, beam, &warp_top, &least);
                if (lane == 0) { s_least[warp] = least; s_most[warp] = warp_top; }
                __syncthreads();
                unsigned long long most = s_most[0];
#pragma unroll
                for (int w = 1; w < kSelWarps; ++w) most = s_most[w] > most ? s_most[w] : most;
                bound = max((unsigned)join_bounds(s_least, beam), 1u);
                have = __syncthreads_count(upper >= bound);
                for (unsigned hi = (unsigned)most; have > kMergeShort && hi > bound; ) {
                    const unsigned mid = bound + (hi - bound + 1) / 2;
                    const int n = __syncthreads_count(upper >= mid);
                    if (n >= beam) { bound = mid; have = n; } else hi = mid - 1;
                }
            }
            list(upper >= bound, k);
        } else {
            // ranks by a multiplication, within 2^-51 of the ones by the division: good enough for a bound
            unsigned long long top = 0;
#pragma unroll
            for (int j = 0; j < kMergeHeld; ++j) {
                key[j] = 0;
                if (first + j * kSelThreads >= total || held[j] == 0) continue;
                const int b = slot_of(first + j * kSelThreads + (int)threadIdx.x);
                const double rank = score_at(b, held[j]) * s_inverse[b];
                if (rank > -INFINITY) key[j] = order_f64(rank);
                top = key[j] > top ? key[j] : top;
            }
            unsigned long long warp_top, least;
            group_bounds(top, beam, &warp_top, &least);
            if (lane == 0) { s_least[warp] = least; s_most[warp] = warp_top; }
            __syncthreads();
            unsigned long long most = s_most[0], bound = join_bounds(s_least, beam);
#pragma unroll
            for (int w = 1; w < kSelWarps; ++w) most = s_most[w] > most ? s_most[w] : most;
            if (kept == beam && s_best[turn][beam - 1].a > bound) bound = s_best[turn][beam - 1].a - 16;     // an exact rank
            if (bound == 0) bound = 1;
            // Candidates are not mixed over the threads as logits are (hypotheses differ in score, places in rank), so the
            // bound may be low: halve the way to the largest until at most kMergeShort reach it, never fewer than `beam` of this pass
            // unless the bound is that of the passes before.
            for (int step = 0, count = 0; step < 64; ++step) {
                const unsigned long long mid = step == 0 ? bound : bound + (most - bound + 1) / 2;
                int n = 0;
#pragma unroll
                for (int j = 0; j < kMergeHeld; ++j) n += key[j] >= mid ? 1 : 0;
                n = __reduce_add_sync(0xffffffffu, n);
                if (lane == 0) s_counts[step & 1][warp] = n;
                __syncthreads();
                n = 0;
#pragma unroll
                for (int w = 0; w < kSelWarps; ++w) n += s_counts[step & 1][w];
                if (step == 0 || n >= beam) { bound = mid; count = n; }
                else most = mid - 1;                                  // fewer than `beam` reach mid
                if (count <= kMergeShort || most <= bound) break;
            }
            bound = bound > 16 ? bound - 16 : 1;                      // further down than the two ranks can differ
#pragma unroll
            for (int j = 0; j < kMergeHeld; ++j)
                list(key[j] >= bound, Key128{held[j], (unsigned long long)slot_of(first + j * kSelThreads + (int)threadIdx.x)});
            __syncthreads();
            for (int i = threadIdx.x; i < s_count; i += kSelThreads) s_list[i] = exact((int)s_list[i].b, s_list[i].a);
        }
        __syncthreads();
        int count = s_count;
        const bool long_list = count > 256;                           // counting would take longer than picking them out
        if (!long_list && (int)threadIdx.x < kept) s_list[count + threadIdx.x] = s_best[turn][threadIdx.x];
        __syncthreads();
        if (threadIdx.x == 0) s_count = 0;
        if (!long_list) {
            count += kept;
            auto out = [&](int place, const Key128& k) { s_best[turn ^ 1][place] = k; };
            if (count <= kMergeShort) rank_list(s_list, count, beam, out);
            else rank_long_list(s_list, count, beam, out);
            kept = min(count, beam);
        } else {
            Key128 last{~0ull, ~0ull};
            for (int k = 0; k < beam; ++k) {
                Key128 mine{0, 0};
                for (int i = threadIdx.x; i < count; i += kSelThreads)
                    if (last.over(s_list[i])) mine = larger(mine, s_list[i]);
                if ((int)threadIdx.x < kept && last.over(s_best[turn][threadIdx.x])) mine = larger(mine, s_best[turn][threadIdx.x]);
                last = block_largest(mine, s_slots);
                if (threadIdx.x == 0) s_best[turn ^ 1][k] = last;    // more than 256 candidates: there are `beam`
            }
            kept = beam;
        }
        __syncthreads();
        if ((int)threadIdx.x < kept && s_best[turn ^ 1][threadIdx.x].a != 0) {
            const unsigned long long id = ~s_best[turn ^ 1][threadIdx.x].b;
            s_parent[threadIdx.x] = (int)(id >> 32);
            s_token[threadIdx.x] = (int)(unsigned)id;
            s_rank[threadIdx.x] = s_best[turn ^ 1][threadIdx.x].a;
        }
        // A part's candidates are in order, and so are their ranks: once as many candidates in a row as there are parts are
        // below the ones kept, all that come after are.
        const int end = first + kSelThreads * kMergeHeld, from = max(first, end - n_parts);
        if (end >= total) break;
        const unsigned long long least = s_best[turn ^ 1][beam - 1].a;
        bool over = kept < beam || least <= 16;
#pragma unroll
        for (int j = 0; j < kMergeHeld; ++j) over |= first + j * kSelThreads + (int)threadIdx.x >= from && key[j] >= least - 16;
        idle = __syncthreads_or(over) ? 0 : idle + (end - from);
        if (idle >= n_parts) break;
    }
    __syncthreads();
    if (threadIdx.x < beam) {
        const int s = threadIdx.x, b = s_parent[s], row = sent * beam + s;
        const bool none = s_token[s] < 0, keeps = none || s_done[b];
        const int token = none ? max(p.eos, 0) : s_token[s];
        float score = none ? -INFINITY : s_score[b];
        if (!keeps) score = (float)(unorder_f64(s_rank[s]) * s_norm[b]);     // the candidate's score again, within 2^-53
        p.score_out[row] = score;
        p.len_out[row] = s_len[b] + (keeps ? 0 : 1);
        p.done_out[row] = keeps || token == p.eos;
        p.parent[row] = b;
        p.next[row] = token;
        s_token[s] = keeps ? -1 : token;                              // the token that joins the history
    }
    // Histories: each position is read in every hypothesis before it is written, so that the new histories may take
    // the old ones' place.
    for (int first = 0; first < longest; first += span) {
        if (first > 0) {
            __syncthreads();                                          // the positions before have been written
            fetch(first);
        }
        asm volatile("cp.async.wait_all;" ::: "memory");
        __syncthreads();
        for (int s = warp; s < beam; s += kSelWarps) {
            const int b = s_parent[s], len = s_len[b], token = s_token[s], end = min(first + span, token < 0 ? len : len + 1);
            int* to = p.tokens_out + ((long long)sent * beam + s) * p.ld_tokens;
            for (int pos = first + lane; pos < end; pos += 32) to[pos] = pos < len ? s_history[b * span + pos - first] : token;
        }
    }
}

}  // namespace san
