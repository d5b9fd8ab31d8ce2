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

// CTA = (256 / G positions, key head, item): thread = position and every G-th of the (row, head) pairs, whose sums meet in shared
// memory in a fixed order.
template <int G>
__global__ void __launch_bounds__(256) mass_kernel(const __grid_constant__ MassParams p) {
    constexpr int W = 256 / G;
    __shared__ float part[G > 1 ? 256 : 1];
    const int item = blockIdx.z, hk = blockIdx.y, x = threadIdx.x % W, grp = threadIdx.x / W;
    const int id = p.ids[item], len = p.lens[item], rows = p.rows ? p.rows[item] : p.n_rows, begin = p.begin ? p.begin[item] : len;
    const bool by_id = id < 0 || id >= p.max_ids, by_len = len < 0 || len > p.max_len, by_rows = rows < 0 || rows > p.n_rows;
    if (by_id || by_len || by_rows || begin < 0 || begin > len) {
        if (blockIdx.x == 0 && hk == 0 && threadIdx.x == 0)
            attend_error(p.status, TAG_MASS, item, by_id ? id : by_len ? len : by_rows ? rows : begin,
                         by_id ? p.max_ids : by_len ? p.max_len : by_rows ? p.n_rows : len);
        return;
    }
    const int j = blockIdx.x * W + x;
    if ((long long)blockIdx.x * W >= len) return;
    const bool mine = j < len;
    float sum = 0.f;
    if (mine) {
        const float* S = p.S + item * p.item_stride + (long long)hk * p.group * p.head_stride + j;
        for (int r = grp; r < rows; r += G)
            for (int h = 0; h < p.group; ++h) sum += S[r * p.row_stride + h * p.head_stride];
    }
    if constexpr (G > 1) {
        part[threadIdx.x] = sum;
        __syncthreads();
        if (grp != 0) return;
        for (int k = 1; k < G; ++k) sum += part[k * W + x];
    }
    if (!mine) return;
    float* to = p.mass + ((long long)id * p.Hk + hk) * p.ld + j;
    *to = (j < begin ? p.decay * *to : 0.f) + sum;
}

// ------------------------------------------------------------------------------------------- eviction
struct EvictParams {
    char* k; char* v; long long v_stride;
    char* ks; char* vs; long long s_stride;
    const int* ids; const int* lens;
    float* mass; long long ld;
    int* kept; long long ld_kept;
    int* lens_out;
    int Hk, n_layers, max_ids, cap, n_items, max_len, keep, sink, recent, row_bytes;
    bool permuted;
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

// CTA = (key head, item).  The least mass that stays is found digit by digit (8 bits) from counts; then one pass in order lists the rows
// and moves the mass.
static __global__ void __launch_bounds__(kEvictThreads) evict_select_kernel(const __grid_constant__ EvictParams p) {
    __shared__ int counts[256], warps[2][32];
    __shared__ int digit_s, above_s;
    const int hk = blockIdx.x, item = blockIdx.y, tid = threadIdx.x, lane = tid & 31, warp = tid >> 5;
    const int id = p.ids[item], len = p.lens[item];
    const long long panel = (long long)item * p.Hk + hk;
    if (id < 0 || id >= p.max_ids || len < 0 || len > p.max_len) {
        if (tid == 0) {
            const bool by_id = id < 0 || id >= p.max_ids;
            if (hk == 0) attend_error(p.status, TAG_EVICT, item, by_id ? id : len, by_id ? p.max_ids : p.max_len);
            p.plan[panel] = make_int2(-1, p.keep);
        }
        return;
    }
    int* list = p.list + panel * p.keep;
    int* kept = p.kept ? p.kept + panel * p.ld_kept : nullptr;
    if (len <= p.keep) {
        for (int i = tid; i < len && kept; i += kEvictThreads) kept[i] = i;
        if (tid == 0) p.plan[panel] = make_int2(id, p.keep);
        return;
    }
    float* mass = p.mass + ((long long)id * p.Hk + hk) * p.ld;
    const int lo = p.sink, hi = len - p.recent;
    int want = p.keep - p.sink - p.recent;                 // of rows lo .. hi - 1
    uint32_t prefix = 0, known = 0;                         // digits of the least key that stays
    int ties = 0;                                           // rows of that key that stay, the lowest first
    if (want > 0) {
        for (int shift = 24; shift >= 0; shift -= 8) {
            for (int i = tid; i < 256; i += kEvictThreads) counts[i] = 0;
            __syncthreads();
            for (int j = lo + tid; j < hi; j += kEvictThreads) {
                const uint32_t key = evict_key(mass[j]);
                if ((key & known) == prefix) atomicAdd(&counts[key >> shift & 255], 1);
            }
            __syncthreads();
            if (warp == 0) {                                // the digit at which the count from above reaches `want`
                int mine[8], sum = 0;
#pragma unroll
                for (int k = 0; k < 8; ++k) { mine[k] = counts[255 - (lane * 8 + k)]; sum += mine[k]; }
                int before = sum;
#pragma unroll
                for (int o = 1; o < 32; o <<= 1) {
                    const int y = __shfl_up_sync(0xffffffffu, before, o);
                    if (lane >= o) before += y;
                }
                before -= sum;
#pragma unroll
                for (int k = 0; k < 8; ++k) {
                    if (before < want && before + mine[k] >= want) { digit_s = 255 - (lane * 8 + k); above_s = before; }
                    before += mine[k];
                }
            }
            __syncthreads();
            prefix |= (uint32_t)digit_s << shift;
            known |= 255u << shift;
            want -= above_s;
        }
        ties = want;
    }
    int n_kept = 0, n_ties = 0, first_moved = p.keep;
    for (int base = 0; base < len; base += kEvictThreads) {
        const int j = base + tid;
        const float x = j < len ? mass[j] : 0.f;
        const bool forced = j < len && (j < lo || j >= hi), open = j < len && !forced && p.keep > p.sink + p.recent;
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

// CTA = (plane, key head, item): rows in order, a step of them read before any is written.  Entry i of the list is row i or a later one,
// so that a step never writes over what a later one reads.
static __global__ void __launch_bounds__(256) evict_move_kernel(const __grid_constant__ EvictParams p) {
    const int plane = blockIdx.x, hk = blockIdx.y, item = blockIdx.z;
    const long long panel = (long long)item * p.Hk + hk;
    const int2 plan = p.plan[panel];
    if (plane == 0 && hk == 0 && threadIdx.x == 0 && plan.x >= 0) p.lens_out[item] = min(p.lens[item], p.keep);
    if (plan.x < 0 || plan.y >= p.keep) return;
    const int* list = p.list + panel * p.keep;
    const long long row0 = ((long long)plan.x * p.Hk + hk) * p.cap;
    char* rows = (plane == 0 ? p.k : p.v + (plane - 1) * p.v_stride) + row0 * p.row_bytes;
    const int pieces = p.row_bytes / 16, n = (p.keep - plan.y) * pieces;        // (at most 2^28 rows of 16 pieces)
    constexpr int U = 4;
    for (int base = 0; base < n; base += 256 * U) {
        uint4 x[U];
#pragma unroll
        for (int u = 0; u < U; ++u) {
            const int i = base + u * 256 + threadIdx.x;
            if (i >= n) continue;
            const int to = plan.y + i / pieces, c = i % pieces, from = list[to];
            x[u] = *reinterpret_cast<const uint4*>(rows + (long long)from * p.row_bytes + (p.permuted ? c ^ (from & 7) : c) * 16);
        }
        __syncthreads();
#pragma unroll
        for (int u = 0; u < U; ++u) {
            const int i = base + u * 256 + threadIdx.x;
            if (i >= n) continue;
            const int to = plan.y + i / pieces, c = i % pieces;
            *reinterpret_cast<uint4*>(rows + (long long)to * p.row_bytes + (p.permuted ? c ^ (to & 7) : c) * 16) = x[u];
        }
    }
    if (!p.ks) return;
    uint32_t* scales = reinterpret_cast<uint32_t*>((plane == 0 ? p.ks : p.vs + (plane - 1) * p.s_stride) + row0 * 4);
    for (int base = plan.y; base < p.keep; base += 256 * U) {
        uint32_t x[U];
#pragma unroll
        for (int u = 0; u < U; ++u) {
            const int to = base + u * 256 + threadIdx.x;
            if (to < p.keep) x[u] = scales[list[to]];
        }
        __syncthreads();
#pragma unroll
        for (int u = 0; u < U; ++u) {
            const int to = base + u * 256 + threadIdx.x;
            if (to < p.keep) scales[to] = x[u];
        }
    }
}

}  // namespace san
