// What cached rows have received of the attention weights (san_weight_mass), and a cache cut back to the rows that received most
// (san_cache_evict).  A block of layers shares its weights, so that one mass and one choice serve all of its layers.
#pragma once

#include "san_attend.cuh"

namespace san {

constexpr int TAG_MASS = 15, TAG_EVICT = 16;

// ------------------------------------------------------------------------------------------- mass
struct MassParams {
    const float* S; long long item_stride, row_stride, head_stride;
    float* mass; long long ld;
    const int* rows; const int* ids; const int* lens; const int* begin;
    int n_rows, H, Hk, group, n_items, max_ids, max_len;
    float decay;
    int* status;
};

// Bound by reading S once.  A warp sums 32 U positions, U a lane, over every G-th of the (row, query head) pairs, several pairs' loads on
// their way at once; a CTA is 8 / G such groups of positions of one (key head, item), and the G sums of a position meet in
// shared memory in a fixed order.  Loads of a warp are 128 bytes on end whatever the strides, so that no alignment is asked for.
constexpr int kMassThreads = 256;
template <int G, int U> __host__ __device__ constexpr int mass_positions() { return kMassThreads / G * U; }       // of a CTA
template <int G, int U>
__global__ void __launch_bounds__(kMassThreads) mass_kernel(const __grid_constant__ MassParams p) {
    __shared__ float part[G > 1 ? kMassThreads * U : 1];
    const int item = blockIdx.z, hk = blockIdx.y, warp = threadIdx.x >> 5, lane = threadIdx.x & 31, grp = warp % G;
    const int id = p.ids[item], len = p.lens[item], rows = p.rows ? p.rows[item] : p.n_rows, begin = p.begin ? p.begin[item] : len;
    const bool by_id = id < 0 || id >= p.max_ids, by_len = len < 0 || len > p.max_len, by_rows = rows < 0 || rows > p.n_rows;
    if (by_id || by_len || by_rows || begin < 0 || begin > len) {
        if (blockIdx.x == 0 && hk == 0 && threadIdx.x == 0)
            attend_error(p.status, TAG_MASS, item, by_id ? id : by_len ? len : by_rows ? rows : begin,
                         by_id ? p.max_ids : by_len ? p.max_len : by_rows ? p.n_rows : len);
        return;
    }
    const int base = blockIdx.x * mass_positions<G, U>();
    if (base >= len) return;
    const int j0 = base + warp / G * 32 * U + lane;          // this lane's positions: j0 + 32 u
    float* to = p.mass + ((long long)id * p.Hk + hk) * p.ld + j0;
    float old[U], sum[U];
#pragma unroll
    for (int u = 0; u < U; ++u) {
        old[u] = grp == 0 && j0 + 32 * u < begin ? to[32 * u] : 0.f;
        sum[u] = 0.f;
    }
    const float* S = p.S + item * p.item_stride + (long long)hk * p.group * p.head_stride + j0;
    const int pairs = rows * p.group;
    // pair k is row k / group, head k % group: kept as an address and a head, which go on by G pairs at a time
    int head = grp % p.group;
    const float* src = S + grp / p.group * p.row_stride + head * p.head_stride;
    const int more = G % p.group;
    const long long step = G / p.group * p.row_stride + more * p.head_stride, wrap = p.row_stride - p.group * p.head_stride;
    constexpr int K = G > 1 ? 4 : 2;
    for (int k0 = grp; k0 < pairs; k0 += K * G) {
        float x[K][U];
#pragma unroll
        for (int k = 0; k < K; ++k) {
#pragma unroll
            for (int u = 0; u < U; ++u) x[k][u] = k0 + k * G < pairs && j0 + 32 * u < len ? __ldcs(src + 32 * u) : 0.f;
            src += step;
            head += more;
            if (head >= p.group) { head -= p.group; src += wrap; }
        }
#pragma unroll
        for (int k = 0; k < K; ++k)
#pragma unroll
            for (int u = 0; u < U; ++u) sum[u] += x[k][u];
    }
    if constexpr (G > 1) {
#pragma unroll
        for (int u = 0; u < U; ++u) part[(warp * U + u) * 32 + lane] = sum[u];
        __syncthreads();
        if (grp != 0) return;
        for (int k = 1; k < G; ++k)
#pragma unroll
            for (int u = 0; u < U; ++u) sum[u] += part[((warp + k) * U + u) * 32 + lane];
    }
#pragma unroll
    for (int u = 0; u < U; ++u)
        if (j0 + 32 * u < len) to[32 * u] = fmaf(p.decay, old[u], sum[u]);
}

// ------------------------------------------------------------------------------------------- eviction
struct EvictParams {
    char* k; char* v; long long v_stride;
    char* ks; char* vs; long long s_stride;
    const int* ids; const int* lens;
    float* mass; long long ld;
    int* kept; long long ld_kept;
    int* lens_out;
    int Hk, n_layers, max_ids, cap, n_items, max_len, keep, sink, recent;
    int cluster;                            // CTAs that move the rows of one plane together
    int* list;                              // [item][key head][keep]: rows that stay
    int2* plan;                             // [item][key head]: id and first entry of the list that moves (keep: none)
    int* status;
};
constexpr int kEvictThreads = 1024;

// Order of masses as unsigned numbers; NaN is the lowest, as -infinity is; -0 and 0 are equal.
__device__ __forceinline__ uint32_t evict_key(float x) {
    const uint32_t b = __float_as_uint(x == 0.f ? 0.f : x != x ? -INFINITY : x);
    return b & 0x80000000u ? ~b : b | 0x80000000u;
}

// What both ways to choose begin with: the item's id (-1: skipped and reported; nothing to do where its rows all stay).
__device__ __forceinline__ int evict_item(const EvictParams& p, int hk, int item, int* len) {
    const long long panel = (long long)item * p.Hk + hk;
    const int id = p.ids[item];
    *len = p.lens[item];
    const bool by_id = id < 0 || id >= p.max_ids;
    if (by_id || *len < 0 || *len > p.max_len) {
        if (threadIdx.x == 0) {
            if (hk == 0) attend_error(p.status, TAG_EVICT, item, by_id ? id : *len, by_id ? p.max_ids : p.max_len);
            p.plan[panel] = make_int2(-1, p.keep);
        }
        return -1;
    }
    if (*len <= p.keep) {
        for (int i = threadIdx.x; i < *len && p.kept; i += kEvictThreads) p.kept[panel * p.ld_kept + i] = i;
        if (threadIdx.x == 0) p.plan[panel] = make_int2(id, p.keep);
        return -1;
    }
    return id;
}

// The least key that stays, and how many rows above it, from counts of one digit of 8 bits after the other: four sets of counts, one for every
// fourth warp, which halves what atomics on the same count wait for one another (masses share their exponents).  Every thread of the CTA calls
// this; `each(f)` calls f with the thread's keys (0: not in question).  `want`: of them, 1 or more.
template <class Each>
__device__ __forceinline__ uint32_t evict_least(int want, int (&counts)[256][4], int* found, Each each) {
    const int tid = threadIdx.x, lane = tid & 31, set = tid >> 5 & 3;
    uint32_t prefix = 0, known = 0;
    for (int shift = 24; shift >= 0; shift -= 8) {
        for (int i = tid; i < 1024; i += kEvictThreads) (&counts[0][0])[i] = 0;
        __syncthreads();
        each([&](uint32_t key) { if (key != 0 && (key & known) == prefix) atomicAdd(&counts[key >> shift & 255][set], 1); });
        __syncthreads();
        if (tid < 32) {                                     // the digit at which the count from above reaches `want`
            int mine[8], sum = 0;
#pragma unroll
            for (int k = 0; k < 8; ++k) {
                const int4 c = *reinterpret_cast<const int4*>(counts[255 - (lane * 8 + k)]);
                mine[k] = c.x + c.y + c.z + c.w;
                sum += mine[k];
            }
            int before = sum;
#pragma unroll
            for (int o = 1; o < 32; o <<= 1) {
                const int y = __shfl_up_sync(0xffffffffu, before, o);
                if (lane >= o) before += y;
            }
            before -= sum;
#pragma unroll
            for (int k = 0; k < 8; ++k) {
                if (before < want && before + mine[k] >= want) { found[0] = 255 - (lane * 8 + k); found[1] = before; }
                before += mine[k];
            }
        }
        __syncthreads();
        prefix |= (uint32_t)found[0] << shift;
        known |= 255u << shift;
        want -= found[1];
    }
    return prefix;
}

// CTA = (key head, item), up to 32 R rows a warp, whose masses stay in registers (row 32 i + lane of the warp's run in register i; of R = 16, whose 1024
// threads have 64 registers each, 22 words a thread lie in local memory): read once, and places follow from the warps' counts alone.
// Instructions bound it, all of one SM: of a cache of 8 heads and 4096 rows 11 us cold (18 with the counts of every 1024 rows added up by every thread, 15
// with the key found by comparisons, two bits a turn).
template <int R>
__global__ void __launch_bounds__(kEvictThreads) evict_select_kernel(const __grid_constant__ EvictParams p) {
    __shared__ __align__(16) int digits[256][4];
    __shared__ int2 counts[32];
    __shared__ int found[2], first_gone[32];
    const int hk = blockIdx.x, item = blockIdx.y, tid = threadIdx.x, lane = tid & 31, warp = tid >> 5;
    int len;
    const int id = evict_item(p, hk, item, &len);
    asm volatile("griddepcontrol.launch_dependents;");
    if (id < 0) return;
    const long long panel = (long long)item * p.Hk + hk;
    float* mass = p.mass + ((long long)id * p.Hk + hk) * p.ld;
    const int lo = p.sink, hi = len - p.recent, want = p.keep - p.sink - p.recent;         // of rows lo .. hi - 1
    const int run = (len + 1023) / 1024 * 32, begin = warp * run + lane;                   // a warp's rows
    float x[R];
    uint32_t key[R];                                        // 0: not there, or not in question
#pragma unroll
    for (int i = 0; i < R; ++i) {
        const int j = begin + 32 * i;
        x[i] = 32 * i < run && j < len ? mass[j] : 0.f;
        key[i] = 32 * i < run && j >= lo && j < hi ? evict_key(x[i]) : 0u;
    }
    uint32_t least = 0xffffffffu;                           // nothing is above it
    if (want > 0)
        least = evict_least(want, digits, found, [&](auto f) {
#pragma unroll
            for (int i = 0; i < R; ++i) f(key[i]);
        });
    // rows that stay whatever the ties, and rows that tie
    int sure = 0, tied = 0;
#pragma unroll
    for (int i = 0; i < R; ++i) {
        const int j = begin + 32 * i;
        const bool forced = 32 * i < run && j < len && (j < lo || j >= hi);
        sure += __popc(__ballot_sync(0xffffffffu, forced || key[i] > least));
        tied += __popc(__ballot_sync(0xffffffffu, key[i] == least));
    }
    if (lane == 0) counts[warp] = make_int2(sure, tied);
    __syncthreads();
    const int2 mine = counts[lane];
    const int ties = p.keep - __reduce_add_sync(0xffffffffu, mine.x);                       // of them that stay, the lowest first
    int before = mine.y;
#pragma unroll
    for (int o = 1; o < 32; o <<= 1) {
        const int y = __shfl_up_sync(0xffffffffu, before, o);
        if (lane >= o) before += y;
    }
    before -= mine.y;
    const int stays = mine.x + max(0, min(mine.y, ties - before));                          // of warp `lane`
    int place = stays;
#pragma unroll
    for (int o = 1; o < 32; o <<= 1) {
        const int y = __shfl_up_sync(0xffffffffu, place, o);
        if (lane >= o) place += y;
    }
    int to = __shfl_sync(0xffffffffu, place - stays, warp), tie = __shfl_sync(0xffffffffu, before, warp);
    int* list = p.list + panel * p.keep;
    int* kept = p.kept ? p.kept + panel * p.ld_kept : nullptr;
    const unsigned below = (1u << lane) - 1;
    int gone = len;                                         // the first row that goes
#pragma unroll
    for (int i = 0; i < R; ++i) {
        if (32 * i >= run) break;
        const int j = begin + 32 * i;
        const bool forced = j < len && (j < lo || j >= hi), even = key[i] == least;
        const unsigned tb = __ballot_sync(0xffffffffu, even);
        const bool stay = forced || key[i] > least || (even && tie + __popc(tb & below) < ties);
        const unsigned sb = __ballot_sync(0xffffffffu, stay);
        if (stay) {
            const int at = to + __popc(sb & below);
            list[at] = j;
            if (kept) kept[at] = j;
            if (at != j) mass[at] = x[i];
        } else if (j < len) {
            gone = min(gone, j);
        }
        tie += __popc(tb);
        to += __popc(sb);
    }
    gone = __reduce_min_sync(0xffffffffu, gone);
    if (lane == 0) first_gone[warp] = gone;
    __syncthreads();
    if (warp == 0) {
        gone = __reduce_min_sync(0xffffffffu, first_gone[lane]);
        if (lane == 0) p.plan[panel] = make_int2(id, min(gone, p.keep));
    }
}

// Longer ones, read again for every digit of 8 bits and once in order, 1024 rows at a time.
static __global__ void __launch_bounds__(kEvictThreads) evict_select_long_kernel(const __grid_constant__ EvictParams p) {
    __shared__ __align__(16) int digits[256][4];
    __shared__ int found[2], warps[2][32];
    const int hk = blockIdx.x, item = blockIdx.y, tid = threadIdx.x, lane = tid & 31, warp = tid >> 5;
    int len;
    const int id = evict_item(p, hk, item, &len);
    asm volatile("griddepcontrol.launch_dependents;");
    if (id < 0) return;
    const long long panel = (long long)item * p.Hk + hk;
    int* list = p.list + panel * p.keep;
    int* kept = p.kept ? p.kept + panel * p.ld_kept : nullptr;
    float* mass = p.mass + ((long long)id * p.Hk + hk) * p.ld;
    const int lo = p.sink, hi = len - p.recent;
    const int want = p.keep - p.sink - p.recent;           // of rows lo .. hi - 1
    uint32_t prefix = 0xffffffffu;                          // the least key that stays
    int ties = 0;                                           // rows of that key that stay, the lowest first
    if (want > 0) {
        prefix = evict_least(want, digits, found, [&](auto f) {
            for (int j = lo + tid; j < hi; j += kEvictThreads) f(evict_key(mass[j]));
        });
        int above = 0;
        for (int j = lo + tid; j < hi; j += kEvictThreads) above += evict_key(mass[j]) > prefix;
        above = __reduce_add_sync(0xffffffffu, above);
        if (lane == 0) warps[0][warp] = above;
        __syncthreads();
        ties = want - __reduce_add_sync(0xffffffffu, warps[0][lane]);
        __syncthreads();
    }
    int n_kept = 0, n_ties = 0, first_moved = p.keep;
    for (int base = 0; base < len; base += kEvictThreads) {
        const int j = base + tid;
        const float x = j < len ? mass[j] : 0.f;
        const bool forced = j < len && (j < lo || j >= hi), open = j < len && !forced;
        const uint32_t key = evict_key(x);
        const bool tie = open && key == prefix;
        const unsigned tb = __ballot_sync(0xffffffffu, tie);
        if (lane == 0) warps[0][warp] = __popc(tb);
        __syncthreads();
        int before = n_ties, all = 0;
        for (int w = 0; w < 32; ++w) { before += w < warp ? warps[0][w] : 0; all += warps[0][w]; }
        n_ties += all;
        const bool stay = forced || (open && key > prefix) || (tie && before + __popc(tb & ((1u << lane) - 1)) < ties);
        const unsigned sb = __ballot_sync(0xffffffffu, stay);
        if (lane == 0) warps[1][warp] = __popc(sb);
        __syncthreads();                                    // (and every mass of this step has been read)
        int to = n_kept;
        all = 0;
        for (int w = 0; w < 32; ++w) { to += w < warp ? warps[1][w] : 0; all += warps[1][w]; }
        to += __popc(sb & ((1u << lane) - 1));
        if (stay) {
            list[to] = j;
            if (kept) kept[to] = j;
            if (to != j) mass[to] = x;
        }
        // rows before the first one that goes stay where they are
        if (first_moved == p.keep && all < min(kEvictThreads, len - base)) {
            int first = j < len && !stay ? j : 0x7fffffff;
#pragma unroll
            for (int o = 16; o > 0; o >>= 1) first = min(first, __shfl_xor_sync(0xffffffffu, first, o));
            if (lane == 0) warps[0][warp] = first;
            __syncthreads();
            for (int w = 0; w < 32; ++w) first = min(first, warps[0][w]);
            first_moved = min(first, p.keep);
        }
        n_kept += all;
        __syncthreads();
    }
    if (tid == 0) p.plan[panel] = make_int2(id, first_moved);
}

// Cluster of C CTAs = (plane, key head, item): rows in order, in steps of up to 1024 pieces of 16 bytes a CTA that are read by all of the
// cluster before any is written; the next step's reads are on their way meanwhile.  Entry i of the list is row i or a later one, so that a
// step never writes over what a later one reads.  PIECES: of a row.
constexpr int kMoveThreads = 512, kMoveU = 2;
__device__ __forceinline__ void evict_together(bool cluster) {
    if (cluster) {
        asm volatile("barrier.cluster.arrive.release.aligned;" ::: "memory");
        asm volatile("barrier.cluster.wait.acquire.aligned;" ::: "memory");
    } else {
        __syncthreads();
    }
}
template <int PIECES>
__global__ void __launch_bounds__(kMoveThreads) evict_move_kernel(const __grid_constant__ EvictParams p) {
    constexpr int U = kMoveU, T = kMoveThreads, SU = U / PIECES > 0 ? U / PIECES : 1;      // scales of a thread and step (rows of two pieces)
    const int C = p.cluster, plane = blockIdx.x / C, rank = blockIdx.x % C, hk = blockIdx.y, item = blockIdx.z;
    const long long panel = (long long)item * p.Hk + hk;
    asm volatile("griddepcontrol.wait;" ::: "memory");
    const int2 plan = p.plan[panel];
    if (blockIdx.x == 0 && hk == 0 && threadIdx.x == 0 && plan.x >= 0) p.lens_out[item] = min(p.lens[item], p.keep);
    if (plan.x < 0 || plan.y >= p.keep) return;             // the same for the whole cluster
    const int* list = p.list + panel * p.keep;
    const long long row0 = ((long long)plan.x * p.Hk + hk) * p.cap;
    char* rows = (plane == 0 ? p.k : p.v + (plane - 1) * p.v_stride) + row0 * (PIECES * 16);
    uint32_t* scales = PIECES == 2 ? reinterpret_cast<uint32_t*>((plane == 0 ? p.ks : p.vs + (plane - 1) * p.s_stride) + row0 * 4) : nullptr;
    const int step = C * T * U, n = (p.keep - plan.y) * PIECES, first = rank * T + threadIdx.x;      // pieces (2^26 rows at most)
    auto place = [&](int row, int c) { return reinterpret_cast<uint4*>(rows + (long long)row * (PIECES * 16) + (PIECES == 8 ? c ^ (row & 7) : c) * 16); };
    uint4 x[U], next[U];
    uint32_t sx[SU], snext[SU];
    auto read = [&](int base, uint4 (&to)[U], uint32_t (&sto)[SU]) {
#pragma unroll
        for (int u = 0; u < U; ++u) {
            const int i = base + u * C * T + first;
            if (i < n) to[u] = *place(list[plan.y + i / PIECES], i % PIECES);
        }
        if constexpr (PIECES == 2) {
#pragma unroll
            for (int u = 0; u < SU; ++u) {
                const int i = base / PIECES + u * C * T + first;
                if (i < n / PIECES) sto[u] = scales[list[plan.y + i]];
            }
        }
    };
    read(0, x, sx);
    for (int base = 0; base < n; base += step) {
        if (base + step < n) read(base + step, next, snext);
        evict_together(C > 1);
#pragma unroll
        for (int u = 0; u < U; ++u) {
            const int i = base + u * C * T + first;
            if (i < n) *place(plan.y + i / PIECES, i % PIECES) = x[u];
            x[u] = next[u];
        }
        if constexpr (PIECES == 2) {
#pragma unroll
            for (int u = 0; u < SU; ++u) {
                const int i = base / PIECES + u * C * T + first;
                if (i < n / PIECES) scales[plan.y + i] = sx[u];
                sx[u] = snext[u];
            }
        }
    }
}

}  // namespace san
