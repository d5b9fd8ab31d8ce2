// Whole sequences under a sliding window with sinks (san_window_block): query row a sees key row b <= a if
// b > a - window or b < n_sink; S = Softmax(q.K^T / 8) over those, computed once and applied to
// each layer of the block (Eq. 3, Eq. 4).
//
// window_block_kernel (mma.sync; sequences below 128 positions or windows of some 30, others go to the tiles of san_tile.cuh): CTA = 32 query
// rows of one (sequence, head, layer group), 8 per warp, which are the N side of both products as in attend_kernel: 16
// accumulator registers a layer, so that four CTAs fit an SM with three layers each.  The CTA walks the
// rows that any of its queries sees - the sinks, then the window of its first query up to its last query -
// in tiles of 64 through a ring of shared-memory slots that cp.async fills three slots ahead (keys, then each
// layer's values), with the running maximum and sum of the softmax; scores stay in registers.  Bound by the
// chain of one CTA (length, copies, products: some 4 us) and the number of CTAs: 64 sentences of up to 60 positions, 8 heads,
// 3 layers: 16.7 us with 16 queries per warp and layers in groups of two (each recomputing the scores), 14.6 in one
// group (236 registers, two CTAs per SM).
// A value that a row does not see has weight zero, and zero times an infinity or NaN is NaN: a row whose
// output came out as NaN is computed again over just the rows it sees (window_row_again: one position after the other, in few
// registers, and they are 128 at most; the tiles of san_tile.cuh, whose rows see more, do it their own way).
#pragma once

#include "san_attend.cuh"

namespace san {

struct WindowParams {
    const __nv_bfloat16* q; const __nv_bfloat16* k; const __nv_bfloat16* v; __nv_bfloat16* out;
    const int* lens;
    long long v_layer, out_layer;           // elements between layers
    int n_seq, cap, H, Hk, group, n_layers, lg, n_lg, max_len, window, n_sink;
    int pairs, whole;                       // tensor-core tiles: pairs of tiles of a sequence, CTAs that take a pair
    float scale_log2e;
};

constexpr int kWinQ = 32, kWinTile = 64, kWinSlots = 4;

// Row a of (sequence, head), one layer, by one warp: the definition, over the rows that are seen.  Leaves as soon as the
// row is known to be NaN, so that inputs full of NaN cost next to nothing.
__device__ __noinline__ void window_row_again(const WindowParams& p, int seq, int head, int layer, int a, int lane) {
    const long long kv = ((long long)seq * p.cap * p.Hk + head / p.group) * kDh + lane * 2;
    const long long at = (((long long)seq * p.cap + a) * p.H + head) * kDh + lane * 2;
    const long long step = (long long)p.Hk * kDh;
    auto two = [](const __nv_bfloat16* x) { return __bfloat1622float2(*reinterpret_cast<const __nv_bfloat162*>(x)); };
    const float2 q = two(p.q + at);
    const int lo = max(0, a - p.window + 1), ns = min(p.n_sink, lo), n = ns + a + 1 - lo;
    float m = -INFINITY, l = 0.f, ox = 0.f, oy = 0.f;
    for (int pass = 0; pass < 2; ++pass)
        for (int i = 0; i < n; ++i) {
            const long long b = i < ns ? i : lo + i - ns;
            const float2 k = two(p.k + kv + b * step);
            const float z = warp_sum(q.x * k.x + q.y * k.y) * p.scale_log2e;
            if (pass == 0) {
                m = fmaxf(m, z);
                if (z == z) continue;
                l = z;                       // a score that is seen is NaN: so is the row
                pass = 2;
                break;
            }
            const float w = exp2f(z - (m == -INFINITY ? 0.f : m));
            if (w == 0.f) continue;
            const float2 v = two(p.v + layer * p.v_layer + kv + b * step);
            l += w;
            ox = fmaf(w, v.x, ox); oy = fmaf(w, v.y, oy);
            if (__all_sync(0xffffffffu, ox != ox && oy != oy)) break;        // it cannot become anything else
        }
    const float inv = l == 0.f ? 0.f : 1.f / l;
    *reinterpret_cast<uint32_t*>(p.out + layer * p.out_layer + at) = pack_bf16(ox * inv, oy * inv);
}

template <int LG>
__global__ void __launch_bounds__(128) window_block_kernel(const __grid_constant__ WindowParams p) {
    __shared__ __align__(128) char ring[kWinSlots * kWinTile * 128];
    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
    const int head = blockIdx.y, seq = blockIdx.z / p.n_lg, layer0 = blockIdx.z % p.n_lg * p.lg;
    const int layers = min(p.lg, p.n_layers - layer0);
    const int len = max(0, min(p.lens[seq], p.max_len));
    const int a0 = ((int)gridDim.x - 1 - (int)blockIdx.x) * kWinQ;        // the longest rows first
    if (a0 >= len) return;
    const int a1 = min(a0 + kWinQ, len);
    const int lo = max(0, a0 - p.window + 1), ns = min(p.n_sink, lo), n = ns + a1 - lo;
    const uint32_t ring_addr = (uint32_t)__cvta_generic_to_shared(ring);
    const char* kbase = reinterpret_cast<const char*>(p.k + ((long long)seq * p.cap * p.Hk + head / p.group) * kDh);
    const char* vbase = reinterpret_cast<const char*>(p.v + layer0 * p.v_layer + ((long long)seq * p.cap * p.Hk + head / p.group) * kDh);
    const long long row_bytes = (long long)p.Hk * 128;

    int f_at = 0, f_plane = -1, f_slot = 0;
    auto fill = [&]() {
        if (f_at < n) {
            const char* src = f_plane < 0 ? kbase : vbase + f_plane * p.v_layer * 2;
            const uint32_t slot = ring_addr + f_slot * (kWinTile * 128);
#pragma unroll
            for (int j = 0; j < 4; ++j) {
                const int r = j * 16 + (threadIdx.x >> 3), c = threadIdx.x & 7, at = f_at + r;
                const bool full = at < n;
                const int pos = !full ? 0 : at < ns ? at : lo + at - ns;
                cp16(slot + r * 128 + ((c ^ (r & 7)) << 4), src + pos * row_bytes + (c << 4), full);
            }
            if (++f_plane == layers) { f_plane = -1; f_at += kWinTile; }
            f_slot = f_slot + 1 == kWinSlots ? 0 : f_slot + 1;
        }
        cp_commit();
    };
    for (int i = 0; i < kWinSlots - 1; ++i) fill();

    const int g = lane >> 2, t4 = lane & 3, r8 = lane & 7, mat = lane >> 3;
    const int qa0 = a0 + warp * 8;                                        // the warp's first query
    uint32_t qb[4][2];                                                    // B: query g, dims 16 c + 2 t4 .. and 8 further on
    {
        const int a = qa0 + g;
        const uint32_t* src = reinterpret_cast<const uint32_t*>(p.q + (((long long)seq * p.cap + a) * p.H + head) * kDh) + t4;
#pragma unroll
        for (int c = 0; c < 4; ++c) {
            qb[c][0] = a < a1 ? src[c * 8] : 0u;
            qb[c][1] = a < a1 ? src[c * 8 + 4] : 0u;
        }
    }
    float acc[LG][4][4];                                                  // [layer][16 dims]: dims g and g + 8, queries 2 t4 and 2 t4 + 1
#pragma unroll
    for (int y = 0; y < LG; ++y)
#pragma unroll
        for (int d = 0; d < 4; ++d)
#pragma unroll
            for (int e = 0; e < 4; ++e) acc[y][d][e] = 0.f;
    float m[2] = {-INFINITY, -INFINITY}, l[2] = {0.f, 0.f};
    const uint32_t k_row = ((mat & 1) * 8 + r8) * 128, v_row = ((mat >> 1) * 8 + r8) * 128;
    uint32_t k_chunk[4], v_chunk[4];
#pragma unroll
    for (int c = 0; c < 4; ++c) {
        k_chunk[c] = (uint32_t)((2 * c + (mat >> 1)) ^ r8) << 4;
        v_chunk[c] = (uint32_t)((2 * c + (mat & 1)) ^ r8) << 4;
    }

    int slot = 0;
    auto next = [&]() -> uint32_t {
        cp_wait<kWinSlots - 2>();
        __syncthreads();                                                  // arrived for all; the slot before it is free
        fill();
        const uint32_t s = ring_addr + slot * (kWinTile * 128);
        slot = slot + 1 == kWinSlots ? 0 : slot + 1;
        return s;
    };
    for (int at = 0; at < n; at += kWinTile) {
        const uint32_t ks = next() + k_row;
        const int b_first = at < ns ? 0 : lo + at - ns, b_last = lo + at + kWinTile - 1 - ns;
        // every one of the warp's queries sees the whole tile: nothing to mask
        const bool whole = at >= ns && at + kWinTile <= n && b_last <= qa0 && b_first > qa0 + 7 - p.window;
        const bool none = at >= ns && b_first > qa0 + 7;                  // behind the warp's last query
        uint32_t pb[4][2];
        if (!none) {
            float s[4][4];                                                // positions 16 c + g and + 8, queries 2 t4 and 2 t4 + 1
#pragma unroll
            for (int c = 0; c < 4; ++c) {
#pragma unroll
                for (int e = 0; e < 4; ++e) s[c][e] = 0.f;
#pragma unroll
                for (int k = 0; k < 4; ++k) {
                    uint32_t a[4];
                    ldsm4(a, ks + c * 16 * 128 + k_chunk[k]);
                    mma_bf16(s[c], a, qb[k][0], qb[k][1]);
                }
            }
            float top[2] = {-INFINITY, -INFINITY};
#pragma unroll
            for (int c = 0; c < 4; ++c)
#pragma unroll
                for (int e = 0; e < 4; ++e) {
                    bool seen = true;
                    if (!whole) {
                        const int at1 = at + c * 16 + (e >> 1) * 8 + g, a = qa0 + t4 * 2 + (e & 1);
                        const int b = at1 < ns ? at1 : lo + at1 - ns;
                        seen = at1 < n && b <= a && (b > a - p.window || b < p.n_sink);
                    }
                    s[c][e] = seen ? s[c][e] * p.scale_log2e : -INFINITY;
                    top[e & 1] = fmaxf(top[e & 1], s[c][e]);
                }
            float alpha[2];
#pragma unroll
            for (int j = 0; j < 2; ++j) {
#pragma unroll
                for (int o = 4; o < 32; o <<= 1) top[j] = fmaxf(top[j], __shfl_xor_sync(0xffffffffu, top[j], o));
                const float m_new = fmaxf(m[j], top[j]);
                const float base = m_new == -INFINITY ? 0.f : m_new;
                alpha[j] = m[j] == m_new ? 1.f : fast_exp2(m[j] - base);
                m[j] = m_new;
                float sum = 0.f;
#pragma unroll
                for (int c = 0; c < 4; ++c)
#pragma unroll
                    for (int e = 0; e < 2; ++e) {
                        s[c][2 * e + j] = fast_exp2(s[c][2 * e + j] - base);
                        sum += s[c][2 * e + j];
                    }
                l[j] = l[j] * alpha[j] + sum;
            }
#pragma unroll
            for (int c = 0; c < 4; ++c)
#pragma unroll
                for (int e = 0; e < 2; ++e)
                    asm volatile("movmatrix.sync.aligned.m8n8.trans.b16 %0, %1;" : "=r"(pb[c][e]) : "r"(pack_bf16(s[c][2 * e], s[c][2 * e + 1])));
            if (__any_sync(0xffffffffu, alpha[0] != 1.f || alpha[1] != 1.f)) {
#pragma unroll
                for (int y = 0; y < LG; ++y)
#pragma unroll
                    for (int d = 0; d < 4; ++d)
#pragma unroll
                        for (int e = 0; e < 4; ++e) acc[y][d][e] *= alpha[e & 1];
            }
        }
#pragma unroll
        for (int y = 0; y < LG; ++y) {
            if (y >= layers) break;
            const uint32_t vs = next() + v_row;
            if (none) continue;
#pragma unroll
            for (int c = 0; c < 4; ++c)
#pragma unroll
                for (int d = 0; d < 4; ++d) {
                    uint32_t a[4];
                    ldsm4t(a, vs + c * 16 * 128 + v_chunk[d]);
                    mma_bf16(acc[y][d], a, pb[c][0], pb[c][1]);
                }
        }
    }
    cp_wait<0>();
    __syncthreads();                                                      // the ring is free: outputs go through it, a warp's 8 rows at a time
    char* rows = ring + warp * (8 * 128);
    bool odd[2] = {false, false};
#pragma unroll
    for (int j = 0; j < 2; ++j) {
#pragma unroll
        for (int o = 4; o < 32; o <<= 1) l[j] += __shfl_xor_sync(0xffffffffu, l[j], o);
    }
    const float inv[2] = {l[0] == 0.f ? 0.f : 1.f / l[0], l[1] == 0.f ? 0.f : 1.f / l[1]};
#pragma unroll
    for (int y = 0; y < LG; ++y) {
        if (y >= layers) break;
#pragma unroll
        for (int j = 0; j < 2; ++j) {
            const int r = 2 * t4 + j;
#pragma unroll
            for (int d = 0; d < 4; ++d)
#pragma unroll
                for (int e = 0; e < 2; ++e) {
                    const float x = acc[y][d][2 * e + j] * inv[j];
                    odd[j] |= x != x;
                    *reinterpret_cast<__nv_bfloat16*>(rows + r * 128 + (((2 * d + e) ^ r) << 4) + 2 * g) = __float2bfloat16_rn(x);
                }
        }
        __syncwarp();
#pragma unroll
        for (int k = 0; k < 2; ++k) {
            const int r = k * 4 + (lane >> 3), c = lane & 7, a = qa0 + r;
            if (a < a1)
                *reinterpret_cast<uint4*>(p.out + (layer0 + y) * p.out_layer + (((long long)seq * p.cap + a) * p.H + head) * kDh + c * 8) =
                    *reinterpret_cast<const uint4*>(rows + r * 128 + ((c ^ r) << 4));
        }
        __syncwarp();
    }
    for (int r = 0; r < 8; ++r) {
        const bool again = __any_sync(0xffffffffu, (2 * t4 == r && odd[0]) || (2 * t4 + 1 == r && odd[1]));
        if (again && qa0 + r < a1)
            for (int y = 0; y < layers; ++y) window_row_again(p, seq, head, layer0 + y, qa0 + r, lane);
    }
}

}  // namespace san
