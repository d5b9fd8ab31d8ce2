// Beam search's selection (the step between two decode steps of a beam decoder, Section 4.1: beam
// 4; Figure 5: beams 4 to 20).  For every sentence the `beam` best continuations are taken from the
// candidates of all of its hypotheses:
//     a live hypothesis b offers every token v with       score_b + log Softmax(logits_b)[v],
//     a finished one offers itself, unchanged, with       score_b,
// ranked by score / ((5 + length) / 6)^alpha, ties to the lowest (slot, token).
//
// The logits are read once and that is what bounds the call; everything else is a few KB:
//   select_rows_kernel   CTA = (hypothesis, chunk of the vocabulary).  A thread loads its 8 or 32 logits
//     into registers (all loads in flight at once), keeps their maximum, and adds exp(x - max) over
//     them in float32 (32 terms at most), the threads' sums in double.  The chunk's best `beam` logits come out without sorting it:
//     the beam-th largest of the 256 threads' maxima is a lower bound T that at most 32 x beam logits
//     reach and about beam do; those go to a list in shared memory, and each finds its own place in it
//     by counting the ones above it.  Keys are (logit, index) pairs and therefore all different, so ties
//     cost nothing and fall to the lowest index.
//   select_merge_kernel  CTA = sentence.  Joins the chunks' maxima and sums to the log-sum-exp of each row
//     (double: scores of different hypotheses are compared with one another), ranks the beam x chunks
//     x beam candidates the same way, and carries scores, lengths and token histories over.  It is launched
//     with programmatic stream serialisation: its CTAs are in place when the last logits arrive.
// A finished hypothesis, or one without a score, has its logits skipped.
#pragma once

#include "san_kernels.cuh"

namespace san {

constexpr int kSelThreads = 256;
constexpr int kSelWarps = kSelThreads / 32;
constexpr int kSelList = 2048;                 // most candidates that can pass the bound (see below)
constexpr int TAG_SELECT = 8;

struct SelectParams {
    const void* logits; long long ld;          // elements between rows
    int vocab, n_sent, beam, chunks, eos;
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
__device__ __forceinline__ unsigned long long order_f64(double x) {
    const unsigned long long u = (unsigned long long)__double_as_longlong(x + 0.0);
    return u >> 63 ? ~u : u | (1ull << 63);
}

// Keys, largest first.  Zero stands for "none".
struct Key64 {
    unsigned long long a;
    __device__ __forceinline__ bool over(const Key64& o) const { return a > o.a; }
    __device__ __forceinline__ bool any() const { return a != 0; }
    __device__ __forceinline__ Key64 swapped(int mask) const { return {__shfl_xor_sync(0xffffffffu, a, mask)}; }
    __device__ __forceinline__ Key64 from(int lane) const { return {__shfl_sync(0xffffffffu, a, lane)}; }
};
struct Key128 {
    unsigned long long a, b;
    __device__ __forceinline__ bool over(const Key128& o) const { return a > o.a || (a == o.a && b > o.b); }
    __device__ __forceinline__ bool any() const { return a != 0; }
    __device__ __forceinline__ Key128 swapped(int mask) const {
        return {__shfl_xor_sync(0xffffffffu, a, mask), __shfl_xor_sync(0xffffffffu, b, mask)};
    }
    __device__ __forceinline__ Key128 from(int lane) const {
        return {__shfl_sync(0xffffffffu, a, lane), __shfl_sync(0xffffffffu, b, lane)};
    }
};

template <typename K> __device__ __forceinline__ K keep(const K& mine, const K& other, bool larger) {
    return other.over(mine) == larger ? other : mine;
}
// The warp's 32 keys in descending order over the lanes (bitonic network).
template <typename K> __device__ __forceinline__ K warp_sort(K k, int lane) {
#pragma unroll
    for (int size = 2; size <= 32; size <<= 1)
#pragma unroll
        for (int step = size >> 1; step > 0; step >>= 1)
            k = keep(k, k.swapped(step), ((lane & step) == 0) == ((lane & size) == 0));
    return k;
}
// The 32 largest of two descending runs of 32, descending.
template <typename K> __device__ __forceinline__ K warp_merge(K k, const K& other, int lane) {
    k = keep(k, other.from(31 - lane), true);
#pragma unroll
    for (int step = 16; step > 0; step >>= 1) k = keep(k, k.swapped(step), (lane & step) == 0);
    return k;
}

// A lower bound of the CTA's n-th largest key (n <= 32) from one key per thread, the thread's largest; a key
// that n threads reach.  Up to eight wanted keys the warps' own n-th largest serve: the largest of them is
// reached by at most n threads of each warp (n * 8 * 32 <= kSelList keys); beyond that the warps' runs
// are merged and exactly n threads reach the bound.  `runs`: kSelWarps * 32 keys of shared memory.
template <typename K> __device__ __forceinline__ K nth_bound(K mine, int n, K* runs) {
    const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
    mine = warp_sort(mine, lane);
    if (n <= 8) {
        if (lane == n - 1) runs[warp] = mine;
        __syncthreads();
        K best = runs[0];
#pragma unroll
        for (int w = 1; w < kSelWarps; ++w) best = keep(best, runs[w], true);
        return best;
    }
    runs[threadIdx.x] = mine;
    for (int half = kSelWarps / 2; half > 0; half >>= 1) {
        __syncthreads();
        if (warp < half) {
            mine = warp_merge(mine, runs[(warp + half) * 32 + lane], lane);
            runs[threadIdx.x] = mine;
        }
    }
    __syncthreads();
    return runs[n - 1];
}

// Writes the n largest of `count` different keys to out(place, key); the list is in shared memory.
template <typename K, typename F> __device__ __forceinline__ void rank_list(const K* list, int count, int n, F out) {
    for (int i = threadIdx.x; i < count; i += kSelThreads) {
        const K mine = list[i];
        int above = 0;
        for (int j = 0; j < count; ++j) above += list[j].over(mine) ? 1 : 0;
        if (above < n) out(above, mine);
    }
}

// 32-bit view of the logits a thread holds.
template <typename T> __device__ __forceinline__ float as_f32(T x);
template <> __device__ __forceinline__ float as_f32<float>(float x) { return x; }
template <> __device__ __forceinline__ float as_f32<__nv_bfloat16>(__nv_bfloat16 x) { return __bfloat162float(x); }

// grid = rows * chunks.  PER logits per thread; VECTOR: every row starts on a 16-byte boundary and a thread
// holds runs of 16 bytes, else single logits 256 apart (one mapping for all rows of a call, so that equal
// rows get equal sums whatever their addresses).
template <typename T, int PER, bool VECTOR>
__global__ void __launch_bounds__(kSelThreads) select_rows_kernel(const SelectParams p) {
    asm volatile("griddepcontrol.launch_dependents;");
    constexpr int VEC = VECTOR ? 16 / (int)sizeof(T) : 1;
    constexpr int NV = PER / VEC;
    __shared__ unsigned long long s_list[kSelList];
    __shared__ Key64 s_runs[kSelWarps * 32];
    __shared__ float s_max[kSelWarps];
    __shared__ double s_sum[kSelWarps];
    __shared__ int s_count;
    const int row = (int)(blockIdx.x / (unsigned)p.chunks), chunk = (int)(blockIdx.x % (unsigned)p.chunks);
    if (select_dead(p.score[row]) || p.done[row] != 0) return;        // uniform over the CTA
    const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
    const T* x = static_cast<const T*>(p.logits) + (long long)row * p.ld;
    const int base = chunk * (PER * kSelThreads);

    float v[PER];
#pragma unroll
    for (int j = 0; j < NV; ++j) {
        const int at = base + (j * kSelThreads + (int)threadIdx.x) * VEC;
        if constexpr (VECTOR) {
            if (at + VEC <= p.vocab) {
                unpack16<T>(ld16_stream(x + at), v + j * VEC);
            } else {
#pragma unroll
                for (int e = 0; e < VEC; ++e) v[j * VEC + e] = at + e < p.vocab ? as_f32<T>(x[at + e]) : -INFINITY;
            }
        } else {
            v[j] = at < p.vocab ? as_f32<T>(x[at]) : -INFINITY;
        }
    }
    if (threadIdx.x == 0) s_count = 0;
    auto index_of = [&](int i) { return base + ((i / VEC) * kSelThreads + (int)threadIdx.x) * VEC + i % VEC; };
    float top = -INFINITY;
    int top_i = 0;
#pragma unroll
    for (int i = 0; i < PER; ++i) {
        v[i] = v[i] == v[i] ? v[i] : -INFINITY;                       // NaN: masked
        if (v[i] > top) { top = v[i]; top_i = i; }
    }
    // exp2 of differences to the thread's own maximum; equal values (two infinities too) differ by nothing
    float sum = 0.f;
#pragma unroll
    for (int i = 0; i < PER; ++i) sum += v[i] == top ? 1.0f : exp2f((v[i] - top) * 1.4426950408889634f);
    if (top == -INFINITY) sum = 0.f;

    const float wtop = warp_max(top);
    double wsum = top == wtop ? (double)sum : (double)sum * (double)exp2f((top - wtop) * 1.4426950408889634f);
    if (wtop == -INFINITY) wsum = 0.0;
#pragma unroll
    for (int o = 16; o > 0; o >>= 1) wsum += __shfl_xor_sync(0xffffffffu, wsum, o);
    if (lane == 0) { s_max[warp] = wtop; s_sum[warp] = wsum; }

    auto key_of = [](float f, int index) -> Key64 {
        return {f == -INFINITY ? 0ull : ((unsigned long long)order_f32(f) << 32) | (unsigned)~index};
    };
    const Key64 mine = key_of(top, index_of(top_i));
    const Key64 bound = nth_bound<Key64>(mine, p.beam, s_runs);       // s_max, s_sum, s_count: behind its barrier
    if (mine.any() && !bound.over(mine)) {
#pragma unroll
        for (int i = 0; i < PER; ++i) {
            const Key64 k = key_of(v[i], index_of(i));
            if (k.any() && !bound.over(k)) s_list[atomicAdd(&s_count, 1)] = k.a;
        }
    }
    char* part = p.ws + (size_t)blockIdx.x * select_part_bytes(p.beam);
    if (threadIdx.x == 0) {
        float m = s_max[0];
        for (int w = 1; w < kSelWarps; ++w) m = fmaxf(m, s_max[w]);
        double s = 0.0;
        for (int w = 0; w < kSelWarps; ++w)
            if (s_max[w] > -INFINITY) s += s_max[w] == m ? s_sum[w] : s_sum[w] * (double)exp2f((s_max[w] - m) * 1.4426950408889634f);
        *reinterpret_cast<float*>(part) = m;
        *reinterpret_cast<double*>(part + 8) = s;
    }
    __syncthreads();
    const int count = s_count;
    unsigned long long* best = reinterpret_cast<unsigned long long*>(part + 16);
    rank_list(reinterpret_cast<const Key64*>(s_list), count, p.beam, [&](int place, const Key64& k) { best[place] = k.a; });
    for (int i = count + (int)threadIdx.x; i < p.beam; i += kSelThreads) best[i] = 0;
}

// grid = sentences.
template <typename T>
__global__ void __launch_bounds__(kSelThreads) select_merge_kernel(const SelectParams p) {
    __shared__ Key128 s_list[kSelList];        // 32 KB; the histories' columns after the ranking
    __shared__ Key128 s_runs[kSelWarps * 32];
    __shared__ float s_score[SAN_MAX_BEAM], s_top[SAN_MAX_BEAM];
    __shared__ double s_logsum[SAN_MAX_BEAM], s_norm[SAN_MAX_BEAM];
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
        s_norm[b] = pow((5.0 + (double)(len + (done ? 0 : 1))) / 6.0, p.alpha);
        s_parent[b] = b; s_token[b] = -1;
        const long long limit = p.tokens ? p.ld_tokens : 0x7ffffffe;
        if (len < 0 || len > limit || (len == limit && !done && !dead)) {
            s_bad = 1;
            select_error(p.status, row, len, (int)limit);
        }
        atomicMax(&s_longest, len);
    }
    __syncthreads();
    if (s_bad) return;                                                // the sentence keeps its old state
    asm volatile("griddepcontrol.wait;" ::: "memory");
    const size_t part_bytes = select_part_bytes(beam);
    const char* parts = p.ws + (size_t)sent * beam * p.chunks * part_bytes;
    for (int b = warp; b < beam; b += kSelWarps) {                    // log of each row's sum of exponentials
        if (s_done[b] || s_score[b] == -INFINITY) continue;
        const char* part = parts + (size_t)b * p.chunks * part_bytes;
        float m = -INFINITY;
        for (int c = lane; c < p.chunks; c += 32) m = fmaxf(m, *reinterpret_cast<const float*>(part + c * part_bytes));
        m = warp_max(m);
        double s = 0.0;
        for (int c = lane; c < p.chunks; c += 32) {
            const float mc = *reinterpret_cast<const float*>(part + c * part_bytes);
            const double sc = *reinterpret_cast<const double*>(part + c * part_bytes + 8);
            if (mc > -INFINITY) s += mc == m ? sc : sc * exp((double)mc - (double)m);
        }
#pragma unroll
        for (int o = 16; o > 0; o >>= 1) s += __shfl_xor_sync(0xffffffffu, s, o);
        if (lane == 0) { s_top[b] = m; s_logsum[b] = log(s); }
    }
    __syncthreads();
    // candidate i of the sentence: (slot, chunk, place); a finished hypothesis stands at its first one
    const int per_row = p.chunks * beam, total = beam * per_row;
    auto score_of = [&](int b, float x) {
        const double d = x == s_top[b] ? 0.0 : (double)x - (double)s_top[b];
        return (double)s_score[b] + (d - s_logsum[b]);
    };
    auto key_at = [&](int i) -> Key128 {
        const int b = i / per_row, k = i - b * per_row;
        if (s_score[b] == -INFINITY) return {0, 0};
        double rank;
        int token;
        if (s_done[b]) {
            if (k != 0) return {0, 0};
            token = max(p.eos, 0);
            rank = (double)s_score[b] / s_norm[b];
        } else {
            const int c = k / beam;
            const unsigned long long key = *reinterpret_cast<const unsigned long long*>(parts + ((size_t)b * p.chunks + c) * part_bytes + 16 + 8 * (size_t)(k - c * beam));
            if (key == 0) return {0, 0};
            token = (int)~(unsigned)key;
            rank = score_of(b, unorder_f32((unsigned)(key >> 32))) / s_norm[b];
        }
        if (!(rank > -INFINITY)) return {0, 0};
        return {order_f64(rank), ~(((unsigned long long)(unsigned)b << 32) | (unsigned)token)};
    };
    int count;
    if (total <= kSelThreads) {                                       // all of them fit the list
        if ((int)threadIdx.x < total) {
            const Key128 k = key_at(threadIdx.x);
            if (k.any()) s_list[atomicAdd(&s_count, 1)] = k;
        }
    } else {
        Key128 mine{0, 0};
        for (int i = threadIdx.x; i < total; i += kSelThreads) mine = keep(mine, key_at(i), true);
        const Key128 bound = nth_bound<Key128>(mine, beam, s_runs);
        if (mine.any() && !bound.over(mine))
            for (int i = threadIdx.x; i < total; i += kSelThreads) {
                const Key128 k = key_at(i);
                if (k.any() && !bound.over(k)) {
                    const int at = atomicAdd(&s_count, 1);
                    if (at < kSelList) s_list[at] = k;
                }
            }
    }
    __syncthreads();
    count = s_count;
    if (count > kSelList) {
        // more candidates at or above the bound than the list holds (a few threads hold most of the best
        // ones): one after the other, the largest below the last
        Key128 last{~0ull, ~0ull};
        count = 0;
        for (int k = 0; k < beam; ++k) {
            Key128 mine{0, 0};
            for (int i = threadIdx.x; i < total; i += kSelThreads) {
                const Key128 c = key_at(i);
                if (last.over(c)) mine = keep(mine, c, true);
            }
            mine = warp_sort(mine, lane);
            __syncthreads();
            if (lane == 0) s_runs[warp] = mine;
            __syncthreads();
            last = s_runs[0];
            for (int w = 1; w < kSelWarps; ++w) last = keep(last, s_runs[w], true);
            if (!last.any()) break;
            if (threadIdx.x == 0) s_list[k] = last;
            count = k + 1;
        }
        __syncthreads();
    }
    rank_list(s_list, count, beam, [&](int place, const Key128& k) {
        const unsigned long long id = ~k.b;
        s_parent[place] = (int)(id >> 32);
        s_token[place] = (int)(unsigned)id;
    });
    __syncthreads();
    if (threadIdx.x < beam) {
        const int s = threadIdx.x, b = s_parent[s], row = sent * beam + s;
        const bool none = s_token[s] < 0, keeps = none || s_done[b];
        const int token = none ? max(p.eos, 0) : s_token[s];
        float score = none ? -INFINITY : s_score[b];
        if (!keeps) score = (float)score_of(b, as_f32<T>(static_cast<const T*>(p.logits)[(long long)(sent * beam + b) * p.ld + token]));
        p.score_out[row] = score;
        p.len_out[row] = s_len[b] + (keeps ? 0 : 1);
        p.done_out[row] = keeps || token == p.eos;
        p.parent[row] = b;
        p.next[row] = token;
        s_token[s] = keeps ? -1 : token;                              // the token that joins the history
    }
    if (!p.tokens) return;
    __syncthreads();
    // Histories: a thread owns positions, reads each of them in every hypothesis and then writes it, so
    // that the new histories may take the old ones' place.
    int* column = reinterpret_cast<int*>(s_list) + threadIdx.x;       // kSelThreads ints per hypothesis
    const int longest = min((long long)s_longest + 1, p.ld_tokens);
    for (int pos = threadIdx.x; pos < longest; pos += kSelThreads) {
        const long long first = (long long)sent * beam * p.ld_tokens + pos;
        for (int b = 0; b < beam; ++b) column[b * kSelThreads] = p.tokens[first + b * p.ld_tokens];
        for (int s = 0; s < beam; ++s) {
            const int b = s_parent[s], len = s_len[b], token = s_token[s];
            if (pos < len) p.tokens_out[first + s * p.ld_tokens] = column[b * kSelThreads];
            else if (pos == len && token >= 0) p.tokens_out[first + s * p.ld_tokens] = token;
        }
    }
}

}  // namespace san
