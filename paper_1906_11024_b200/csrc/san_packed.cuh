// Causal attention of whole prompts laid end to end (san_packed_block) on the fifth-generation tensor cores, for bounds of 128 tokens and
// more (shorter ones: window_block_kernel).  S = Softmax(q.K^T / 8) over a token's own and earlier tokens, once per block (Eq. 1,
// Eq. 3), O_l = S.V_l for each layer (Eq. 2, Eq. 4), in one pass with a running maximum.
//
// Work: items = (sequence, 256 query rows, head, up to kPackLayers layers), which cost as many chunks of 64 keys as lie before their
// last row.  One persistent CTA per SM takes items from a list sorted by cost (packed_list_kernel), forwards and backwards in turn,
// so that all SMs end together.  What an item needs before its first product (queries, keys, values, scores) is on its way while the one
// before it is still being finished: with a CTA per item nothing overlapped that, some 4 us of each.  Roles:
//   warps 0-3, 4-7  softmax of one tile each: thread = query row = tensor-memory lane, so maxima and sums need no shuffles.  Weights go
//                back to tensor memory in bf16, over the scores, as the A operand of the second product.  The maximum that
//                weights are taken against moves only when a row's own has grown by more than 2^8; then outputs are scaled.
//   warps 8, 9   copies: 16-byte cp.async into operand tiles (rows of 128 bytes, chunks XOR-swizzled by row & 7, what the matrix
//                descriptors name), keys up to four chunks ahead, values three, the next item's queries in a second buffer.
//   warps 10, 11 issue the MMAs of a tile each, one elected lane: scores of the next chunk (of the next item's first, behind the last), then
//                outputs of this one.  MMAs of a thread complete in order, so that scores never replace weights that have not been read.
//                The tiles share keys and values and nothing else, so that one may be at its exponentials while the other is not.
// Tensor memory: a tile of 128 rows has 256 columns: scores twice (64 each, weights over them) and up to two layers' outputs.
// What bounds it: the softmax warps.  A chunk (256 rows x 64 keys) takes some 1500 clocks, of which a warp is at its exponentials for 700 to 850 (two
// warps to an SM quarter, whose 16 exponentials a clock and SM they share), at maxima for 250, waiting for scores 200; an item's end takes 2500 to 4000.
// 48 prompts of 1 to 4096 tokens, 16 heads over 4 key heads: 234 us (296 with a CTA for an item, 16 softmax warps and two threads a row
// 345, since their meeting took 500 clocks a chunk); two of some 8000 tokens, 8 heads, 2 layers: 224 us = 835 TFLOP/s in calls one after the other, under the
// power limit, and 199 = 940 in a few of them (those before: 247, 296).
// Tried and not faster: no look for a chunk's maximum while sums stay small (273 and 235 us: the scores stay live), the second tile started
// later, weights stored in two halves, the next chunk's scores read and looked through between the halves of this one's exponentials (291 and 254).
// Every wait is bounded: one that runs out raises a flag that ends the CTA's other waits; the CTA frees its tensor memory, reports, and
// leaves what it has not written.
#pragma once

#include "san_tile.cuh"

namespace san {

constexpr int kPackWarps = 12, kPackThreads = kPackWarps * 32, kPackLoaders = 64, kPackLayers = 2;
constexpr int kPackQ = 2 * kTileQ * 128;                                // bytes of an item's queries
constexpr int kPackRows = 8 * 8192;                                     // outputs on their way out, 8 KB for 32 rows
static_assert(kAgainBytes <= 8192, "a row that is computed again");
__host__ __device__ constexpr int pack_smem_bytes(int layers) {
    return 1024 + 2 * kPackQ + (kTileKSlots + kTileVSlots * layers) * kTileK * 128 + kPackRows;
}

struct PackedParams {
    const __nv_bfloat16* q; const __nv_bfloat16* k; const __nv_bfloat16* v; __nv_bfloat16* out;
    long long q_ld, k_ld, v_ld, out_ld, v_layer, out_layer;             // elements between tokens, between layers
    const int* first; const int4* list;                                 // no list: one sequence
    int n_seq, n_tokens, max_len, pairs;                                // pairs: of tiles of all sequences, at most
    int H, group, n_layers, lg, n_lg;
    float scale_log2e;
    int* status;
};

__device__ __forceinline__ int packed_sequence(const PackedParams& p, int seq, int* len, bool report) {
    const int a = p.first[seq], b = p.first[seq + 1];
    const bool ok = a >= 0 && b >= a && b <= p.n_tokens && b - a <= p.max_len;
    if (!ok && report && p.status) {
        const bool order = a < 0 || b < a || b > p.n_tokens;
        record_error(p.status, TAG_PACKED, seq, order ? b : b - a, order ? p.n_tokens : p.max_len);
    }
    *len = ok ? b - a : 0;
    return a;
}

// The list of all sequences' pairs of tiles, those with the most keys first: entry i + 1 is (first token, length, pair, sequence), entry 0
// has their number.  One CTA: pairs are counted by their place in the sequence (all beyond 2047 together), the counts summed from
// above.  Sequences that are not in order have no pairs (and are reported).  A thread's sequences have no more pairs than the tokens and one each, unless
// they overlap: it counts no more, so that no sum passes 31 bits (2^28 tokens and sequences at most) and no call takes forever.
constexpr int kPackedBins = 2048;
static __global__ void __launch_bounds__(1024) packed_list_kernel(const __grid_constant__ PackedParams p, int4* list) {
    __shared__ int bins[kPackedBins], sums[32];
    const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5;
    asm volatile("griddepcontrol.launch_dependents;");                  // packed_kernel sets itself up meanwhile
    const int most = p.n_tokens / (2 * kTileQ) + (p.n_seq + 1023) / 1024;
    bins[tid] = bins[tid + 1024] = 0;
    __syncthreads();
    for (int s = tid, n = 0; s < p.n_seq; s += 1024) {
        int len;
        packed_sequence(p, s, &len, true);
        for (int i = 0; i * 2 * kTileQ < len && n < most; ++i, ++n) atomicAdd(&bins[min(i, kPackedBins - 1)], 1);
    }
    __syncthreads();
    const int hi = kPackedBins - 1 - 2 * tid, a = bins[hi], b = bins[hi - 1];
    int before = a + b;
#pragma unroll
    for (int o = 1; o < 32; o <<= 1) {
        const int y = __shfl_up_sync(0xffffffffu, before, o);
        if (lane >= o) before += y;
    }
    if (lane == 31) sums[warp] = before;
    __syncthreads();
    for (int w = 0; w < warp; ++w) before += sums[w];
    if (tid == 1023) list[0] = make_int4(min(before, p.pairs), 0, 0, 0);
    bins[hi] = before - a - b;
    bins[hi - 1] = before - b;
    __syncthreads();
    for (int s = tid, n = 0; s < p.n_seq; s += 1024) {
        int len;
        const int token0 = packed_sequence(p, s, &len, false);
        for (int i = 0; i * 2 * kTileQ < len; ++i, ++n) {
            const int at = n < most ? atomicAdd(&bins[min(i, kPackedBins - 1)], 1) : p.pairs;
            if (at < p.pairs) { list[1 + at] = make_int4(token0, len, i, s); continue; }
            if (p.status) record_error(p.status, TAG_PACKED, s, at, p.pairs);   // more than there can be: sequences that overlap
            if (n >= most) return;                                              // (no barrier follows)
        }
    }
}

// 2^x of two numbers on the FMA pipe: x = n + f with n the nearest whole number (the low bits of x + 1.5 2^23) and |f| <= 1/2, 2^f by a polynomial
// of third degree (1 at 0, fitted for the least relative error, 0.0001: a twentieth of what the rounding of a weight to bf16 is), n
// added to its exponent.  At -127 and below, -infinity among it, exactly 0.  Not for NaN.
__device__ __forceinline__ void pack_exp2(unsigned long long x, float& u, float& v) {
    tile_unpair(x, u, v);
    x = tile_pair(fmaxf(u, -127.f), fmaxf(v, -127.f));
    const unsigned long long r = tile_add2(x, tile_pair(12582912.f, 12582912.f)), n = tile_add2(r, tile_pair(-12582912.f, -12582912.f));
    const unsigned long long f = tile_fma2(n, tile_pair(-1.f, -1.f), x);
    unsigned long long y = tile_fma2(f, tile_pair(0.0550089329f, 0.0550089329f), tile_pair(0.242210954f, 0.242210954f));
    y = tile_fma2(y, f, tile_pair(0.693282902f, 0.693282902f));
    y = tile_fma2(y, f, tile_pair(1.f, 1.f));
    float a, b;
    tile_unpair(y, u, v);
    tile_unpair(r, a, b);
    u = __uint_as_float(__float_as_uint(a) * 0x800000u + __float_as_uint(u));
    v = __uint_as_float(__float_as_uint(b) * 0x800000u + __float_as_uint(v));
}
__device__ __forceinline__ float pack_max3(float a, float b, float c) {          // NaN if one is
    float d;
    asm("max.NaN.f32 %0, %1, %2, %3;" : "=f"(d) : "f"(a), "f"(b), "f"(c));
    return d;
}
// Of eight pairs of exponentials.  48 prompts of 1 to 4096 tokens and two of some 8000 (see the kernel): 250 and 218 us with none, 245 and 210 with
// one, 241 and 205 with two, 248 and 212 with three.
constexpr int kPackPoly = 2;

// What a CTA works on, and which comes next.
struct PackedItem {
    int token0, a0, rows, seq, head, layer0, layers;        // first token, first query row, query rows
    int chunks0, chunks1;                                   // of each tile; the second's are the item's if it has rows
    __device__ __forceinline__ int chunks(int x) const { return x ? chunks1 : chunks0; }
    __device__ __forceinline__ int all() const { return max(chunks0, chunks1); }
};
struct PackedWalk {
    const PackedParams& p;
    int count, each, len0, token0;
    unsigned at, turn;                                      // the next item's number
    int4 entry;                                             // of the list, read an item ahead
    __device__ __forceinline__ explicit PackedWalk(const PackedParams& params) : p(params), len0(0), token0(0), at(blockIdx.x), turn(0) {
        each = p.H * p.n_lg;
        if (p.list) {
            count = p.list[0].x;
            fetch();
        } else {
            token0 = packed_sequence(p, 0, &len0, blockIdx.x == 0 && threadIdx.x == 0);
            count = (len0 + 2 * kTileQ - 1) / (2 * kTileQ);
        }
    }
    __device__ __forceinline__ void fetch() {
        if (at < (unsigned)count * each) entry = p.list[1 + at / each];
    }
    // Item `at`, and on to the next turn's, which is dealt the other way round.
    __device__ __forceinline__ bool next(PackedItem* w) {
        if (at >= (unsigned)count * each) return false;     // (a later turn's are behind it)
        const int i = (int)(at / each), rest = (int)(at - (unsigned)i * each);
        int len, pair;
        if (p.list) {
            w->token0 = entry.x; len = entry.y; pair = entry.z; w->seq = entry.w;
        } else {
            w->token0 = token0; len = len0; pair = count - 1 - i; w->seq = 0;
        }
        at += turn++ & 1 ? 2 * blockIdx.x + 1 : 2 * (gridDim.x - 1 - blockIdx.x) + 1;
        if (p.list) fetch();
        w->head = rest / p.n_lg;
        w->layer0 = rest % p.n_lg * p.lg;
        w->layers = min(p.lg, p.n_layers - w->layer0);
        w->a0 = pair * 2 * kTileQ;
        w->rows = min(2 * kTileQ, len - w->a0);
        w->chunks0 = (w->a0 + min(kTileQ, w->rows) + kTileK - 1) / kTileK;
        w->chunks1 = w->rows > kTileQ ? (w->a0 + w->rows + kTileK - 1) / kTileK : 0;
        return true;
    }
};

// Row a of an item's head, its layers, by one warp: over the tokens that it sees, as a row of a decode step, kPackAgain of them at a time. A sum that
// is NaN ends it: nothing makes the row anything else.
constexpr int kPackAgain = 4096;
__device__ __forceinline__ void packed_row_again(const PackedParams& p, const PackedItem& w, int a, char* smem, int lane) {
    struct { const char* q; int H, group; float scale_log2e; } row;
    row.q = reinterpret_cast<const char*>(p.q + (long long)(w.token0 + a) * p.q_ld + w.head * kDh);
    row.H = 1; row.group = 1; row.scale_log2e = p.scale_log2e;
    AttendRun u;
    u.v = reinterpret_cast<const char*>(p.v + w.layer0 * p.v_layer + (long long)w.token0 * p.v_ld + w.head / p.group * kDh);
    u.k = reinterpret_cast<const char*>(p.k + (long long)w.token0 * p.k_ld + w.head / p.group * kDh);
    u.row_bytes = p.k_ld * 2; u.v_row_bytes = p.v_ld * 2; u.v_stride = p.v_layer * 2; u.permuted = false;
    u.lo = 0; u.n_sink = 0; u.n = a + 1;
    u.item0 = 0; u.row0 = 0; u.rows = 1; u.head0 = 0; u.layer0 = w.layer0; u.layers = w.layers; u.slot = 0;
    static_assert((kPackLayers - 1) * kAtRows * kAtOutLd * 4 + kDh * 4 <= kAtTile * 128, "the row's outputs, then (max, sum), in the ring's place");
    float2* ml = reinterpret_cast<float2*>(smem + kAtTile * 128);
    float m = -INFINITY, l = 0.f;
    float2 o[kPackLayers];
#pragma unroll
    for (int y = 0; y < kPackLayers; ++y) o[y] = make_float2(0.f, 0.f);
    for (u.begin = 0; u.begin <= a; u.begin += kPackAgain) {
        u.end = min(u.begin + kPackAgain, a + 1);
        __syncwarp();
        attend_warp_bf16<kPackLayers, 2>(row, u, u.begin, kAtTile, smem, ml, lane);
        __syncwarp();
        const float2 x = ml[0];
        const float m_new = fmaxf(m, x.x), f = m == m_new ? 1.f : exp2f(m - m_new), b = x.x == m_new ? 1.f : exp2f(x.x - m_new);
        l = l * f + x.y * b;
        m = m_new;
#pragma unroll
        for (int y = 0; y < kPackLayers; ++y) {
            if (y >= w.layers) break;
            const float2 v = *reinterpret_cast<const float2*>(smem + y * (kAtRows * kAtOutLd * 4) + lane * 8);
            o[y] = make_float2(o[y].x * f + v.x * b, o[y].y * f + v.y * b);
        }
        if (l != l) break;
    }
    const float inv = l == 0.f ? 0.f : 1.f / l;
#pragma unroll
    for (int y = 0; y < kPackLayers; ++y) {
        if (y >= w.layers) break;
        *reinterpret_cast<uint32_t*>(p.out + (w.layer0 + y) * p.out_layer + (long long)(w.token0 + a) * p.out_ld + w.head * kDh + lane * 2) = pack_bf16(o[y].x * inv, o[y].y * inv);
    }
}

// Rows of a warp's 32 in the tile x of an item that came out as NaN: computed again where a value that was multiplied by a weight of zero can be
// the cause, which only later tokens of the tile can hold.  The outputs, which this warp has written, are read for them.
__device__ __forceinline__ void packed_again(const PackedParams& p, const PackedItem& w, int x, int quarter, char* smem, int lane) {
    const int first = w.a0 + x * kTileQ, last = w.a0 + min((x + 1) * kTileQ, w.rows) - 1, row0 = first + 32 * quarter;
    uint32_t odd = 0;                                       // a bit for each
    for (int r = 0; r < 32 && row0 + r <= last; ++r) {
        bool nan = false;
        for (int y = 0; y < w.layers; ++y) {
            const uint32_t z = *reinterpret_cast<const uint32_t*>(p.out + (w.layer0 + y) * p.out_layer + (long long)(w.token0 + row0 + r) * p.out_ld + w.head * kDh + lane * 2);
            nan |= (z & 0x7fffu) > 0x7f80u || (z >> 16 & 0x7fffu) > 0x7f80u;
        }
        if (__any_sync(0xffffffffu, nan)) odd |= 1u << r;
    }
    if (odd == 0) return;
    int bad = 0;                                            // the last token of the tile with such a value
    for (int i = lane; i < w.layers * (last - first) * 8; i += 32) {
        const int b = first + 1 + (i >> 3) % (last - first), y = i / ((last - first) * 8);
        const uint4 v = *reinterpret_cast<const uint4*>(p.v + (w.layer0 + y) * p.v_layer + (long long)(w.token0 + b) * p.v_ld + w.head / p.group * kDh + (i & 7) * 8);
        const uint32_t e = 0x7f80u;                         // an exponent of all ones: no finite number
        for (const uint32_t z : {v.x, v.y, v.z, v.w})
            if ((z & e) == e || (z >> 16 & e) == e) bad = max(bad, b);
    }
    bad = __reduce_max_sync(0xffffffffu, bad);
    for (; odd; odd &= odd - 1) {
        const int a = row0 + __ffs(odd) - 1;
        if (a < bad) packed_row_again(p, w, a, smem, lane);  // later ones see it
    }
}

// The same for all items of the CTA, one after the other: 0.9 ms for 32 rows of a block of two layers and every 1000 tokens in front of them.
__device__ __noinline__ void packed_items_again(const PackedParams& p, int x, int quarter, char* smem, int lane) {
    PackedItem w;
    for (PackedWalk walk(p); walk.next(&w);)
        if (w.chunks(x) > 0) packed_again(p, w, x, quarter, smem, lane);
}

template <int LG>
__global__ void __launch_bounds__(kPackThreads, 1) packed_kernel(const __grid_constant__ PackedParams p) {
    constexpr uint32_t kCols = 512, kTileCols = 256, kOut = 128;
    static_assert(kOut + 64 * LG <= kTileCols, "tensor memory");
    extern __shared__ __align__(1024) char pack_smem[];
    __shared__ __align__(8) uint64_t q_full[2], q_free[2], k_full[kTileKSlots], k_free[kTileKSlots], v_full[kTileVSlots], v_free[kTileVSlots];
    __shared__ __align__(8) uint64_t s_full[2][2], p_full[2][2], pv_done[2][2], o_free[2];
    __shared__ uint32_t tmem_s;
    __shared__ int dead_s, again_s[2 * kTileQ / 32];                    // again: rows of a softmax warp came out as NaN
    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
    volatile int* dead = &dead_s;
    char* sQ = pack_smem + ((1024u - (tile_u32(pack_smem) & 1023u)) & 1023u);
    const uint32_t aQ = tile_u32(sQ), aK = aQ + 2 * kPackQ, aV = aK + kTileKSlots * kTileK * 128;
    char* sRows = sQ + 2 * kPackQ + (kTileKSlots + kTileVSlots * LG) * kTileK * 128;
    if (threadIdx.x == 0) {
        for (int i = 0; i < kTileKSlots; ++i) { tile_bar_init(&k_full[i], kPackLoaders); tile_bar_init(&k_free[i], 2); }
        for (int i = 0; i < kTileVSlots; ++i) { tile_bar_init(&v_full[i], kPackLoaders); tile_bar_init(&v_free[i], 2); }
        for (int i = 0; i < 2; ++i) {
            tile_bar_init(&q_full[i], kPackLoaders); tile_bar_init(&q_free[i], 2); tile_bar_init(&o_free[i], 4);
            for (int b = 0; b < 2; ++b) { tile_bar_init(&s_full[i][b], 1); tile_bar_init(&p_full[i][b], 4); tile_bar_init(&pv_done[i][b], 1); }
        }
        asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
        dead_s = 0;
    }
    if (warp == 10) {
        asm volatile("tcgen05.alloc.cta_group::1.sync.aligned.shared::cta.b32 [%0], %1;" :: "r"(tile_u32(&tmem_s)), "r"(kCols) : "memory");
        asm volatile("tcgen05.relinquish_alloc_permit.cta_group::1.sync.aligned;" ::: "memory");
    }
    tile_before_sync();
    __syncthreads();
    tile_after_sync();
    const uint32_t tmem = tmem_s;
    asm volatile("griddepcontrol.wait;" ::: "memory");                  // the list
    PackedWalk walk(p);
    PackedItem w;

    if (warp >= 10) {
        const int x = warp - 10;
        uint32_t elected;                                               // 1 in one lane
        asm volatile("{\n.reg .pred p;\nelect.sync _|p, 0xffffffff;\nselp.u32 %0, 1, 0, p;\n}" : "=r"(elected));
        const uint32_t id_s = tile_idesc(false, kTileK), base = tmem + (uint32_t)x * kTileCols;
        int scored = 0, applied = 0, tiles = 0;                         // chunks whose MMAs have been issued; items whose outputs have been begun
        int kc = 0, vc = 0, items = 0;                                  // chunks of all items
        // A slot is free when both tiles' MMAs are through with it.  A tile that has no rows before a chunk's keys waits for it all the same: its
        // arrival belongs to this filling of the slot.
        auto scores = [&](const PackedItem& it, int t, int item) -> bool {
            const int slot = kc % kTileKSlots;
            if (t == 0 && !tile_wait_warp(&q_full[item & 1], (uint32_t)(item >> 1) & 1u, dead)) return false;
            if (!tile_wait_warp(&k_full[slot], (uint32_t)(kc / kTileKSlots) & 1u, dead)) return false;
            if (t < it.chunks(x)) {
                tile_proxy_fence();                                     // the copies are writes of the generic proxy
                tile_after_sync();
                const uint64_t dK = tile_desc(aK + (uint32_t)slot * (kTileK * 128));
                const uint64_t dQ = tile_desc(aQ + (uint32_t)(item & 1) * kPackQ + (uint32_t)x * (kTileQ * 128));
                const int buf = scored & 1;                             // its weights of two chunks ago have been applied (in order)
                if (elected) {
#pragma unroll
                    for (int s = 0; s < 4; ++s) tile_mma(base + buf * kTileK, dQ + 2 * s, dK + 2 * s, id_s, s > 0);
                    tile_commit(&s_full[x][buf]);
                }
                ++scored;
            }
            if (elected) {
                tile_commit(&k_free[slot]);
                if (t + 1 == it.all()) tile_commit(&q_free[item & 1]);
            }
            ++kc;
            return true;
        };
        auto outputs = [&](const PackedItem& it, int t) -> bool {
            const int slot = vc % kTileVSlots;
            if (!tile_wait_warp(&v_full[slot], (uint32_t)(vc / kTileVSlots) & 1u, dead)) return false;
            if (t < it.chunks(x)) {
                tile_proxy_fence();
                if (t == 0) {                                           // the outputs of the tile's item before have been read
                    if (tiles > 0 && !tile_wait_warp(&o_free[x], (uint32_t)(tiles - 1) & 1u, dead)) return false;
                    ++tiles;
                }
                if (!tile_wait_warp(&p_full[x][applied & 1], (uint32_t)(applied >> 1) & 1u, dead)) return false;
                tile_after_sync();
                const uint64_t dV = tile_desc(aV + (uint32_t)(slot * LG) * (kTileK * 128), kTileK * 128);
                const uint32_t id_o = tile_idesc(true, it.layers * kDh);
                if (elected) {
#pragma unroll
                    for (int s = 0; s < kTileK / 16; ++s)
                        tile_mma_ta(base + kOut, base + (applied & 1) * kTileK + 8 * s, dV + 128 * s, id_o, t > 0 || s > 0);
                    tile_commit(&pv_done[x][applied & 1]);
                }
                ++applied;
            }
            if (elected) tile_commit(&v_free[slot]);
            ++vc;
            return true;
        };
        bool more = walk.next(&w), go = more && scores(w, 0, 0);
        while (go && more) {
            const int chunks = w.all();
            for (int t = 0; t + 1 < chunks && go; ++t) go = scores(w, t + 1, items) && outputs(w, t);
            PackedItem then;
            more = walk.next(&then);
            if (go && more) go = scores(then, 0, items + 1);
            if (go) go = outputs(w, chunks - 1);
            w = then;
            ++items;
        }
    } else if (warp >= 8) {
        // thread: 16-byte piece c of rows r0, r0 + 8, ..., whose chunks are swizzled alike
        static_assert(kPackLoaders == 64, "rows of a thread");
        const int r0 = (threadIdx.x - 2 * kTileQ) >> 3, c = threadIdx.x & 7;
        const uint32_t sw = (uint32_t)(r0 * 128 + ((c ^ r0) << 4));
        auto copy = [&](const __nv_bfloat16* src, long long ld, uint32_t dst, int rows, int of) {        // `rows` of `of` are there, the others zeros
            const char* at = reinterpret_cast<const char*>(src + r0 * ld + c * 8);
            const long long step = 16 * ld;
            dst += sw;
            if (rows >= of) {
#pragma unroll 8
                for (int r = 0; r < of; r += 8, at += step) cp16(dst + (uint32_t)(r * 128), at, true);
            } else {
                for (int r = 0; r < of; r += 8, at += step) cp16(dst + (uint32_t)(r * 128), r0 + r < rows ? at : reinterpret_cast<const char*>(src), r0 + r < rows);
            }
        };
        // the barrier hears of a thread's copies when they have landed; the thread does not wait for them
        auto landed = [](uint64_t* bar) {
            asm volatile("cp.async.mbarrier.arrive.noinc.shared::cta.b64 [%0];" ::"r"(tile_u32(bar)) : "memory");
        };
        bool go = true;
        int n = 0;                                                      // chunks of all items
        for (int item = 0; go && walk.next(&w); ++item) {
            const int b = item & 1, kv = w.head / p.group * kDh, len = w.a0 + w.rows;
            if (item >= 2 && !tile_wait(&q_free[b], (uint32_t)(item / 2 - 1) & 1u, dead)) break;
            copy(p.q + (long long)(w.token0 + w.a0) * p.q_ld + w.head * kDh, p.q_ld, aQ + (uint32_t)b * kPackQ, w.rows, w.rows > kTileQ ? 2 * kTileQ : kTileQ);
            landed(&q_full[b]);
            const __nv_bfloat16* k = p.k + (long long)w.token0 * p.k_ld + kv;
            const __nv_bfloat16* v = p.v + w.layer0 * p.v_layer + (long long)w.token0 * p.v_ld + kv;
            for (int t = 0; t < w.all(); ++t, ++n) {
                const int ks = n % kTileKSlots, vs = n % kTileVSlots, left = len - t * kTileK;
                go = n < kTileKSlots || tile_wait(&k_free[ks], (uint32_t)(n / kTileKSlots - 1) & 1u, dead);
                if (!go) break;
                copy(k + (long long)t * kTileK * p.k_ld, p.k_ld, aK + (uint32_t)ks * (kTileK * 128), left, kTileK);
                landed(&k_full[ks]);
                go = n < kTileVSlots || tile_wait(&v_free[vs], (uint32_t)(n / kTileVSlots - 1) & 1u, dead);
                if (!go) break;
                for (int y = 0; y < w.layers; ++y)
                    copy(v + y * p.v_layer + (long long)t * kTileK * p.v_ld, p.v_ld, aV + (uint32_t)(vs * LG + y) * (kTileK * 128), left, kTileK);
                landed(&v_full[vs]);
            }
        }
        asm volatile("cp.async.wait_all;" ::: "memory");
    } else {
        const int x = warp >> 2, quarter = warp & 3, row = quarter * 32 + lane;        // of the tile
        const uint32_t lanes = tmem + ((uint32_t)(quarter * 32) << 16) + (uint32_t)x * kTileCols;
        char* mine = sRows + warp * 8192;                               // 32 rows of 128 bytes
        const float sc = p.scale_log2e;
        const unsigned long long sc2 = tile_pair(sc, sc);
        int count = 0;                                                  // chunks of all items
        bool ok = true;
        if (lane == 0) again_s[warp] = 0;
        // The outputs of the tile's chunk n are complete.  Two barriers in turn, as for scores and weights, because a wait
        // names a phase by its parity: the outputs of chunk n - 2 were complete before the scores of chunk n.
        auto outputs = [&](int n) -> bool { return tile_wait_warp(&pv_done[x][n & 1], (uint32_t)(n >> 1) & 1u, dead); };
        while (ok && walk.next(&w)) {
            const int chunks = w.chunks(x), a = w.a0 + x * kTileQ;      // first row of the tile
            if (chunks == 0) continue;
            float m = -INFINITY, l = 0.f;
            for (int t = 0; t < chunks; ++t, ++count) {
                const uint32_t buf = lanes + (count & 1) * kTileK;
                ok = tile_wait_warp(&s_full[x][count & 1], (uint32_t)(count >> 1) & 1u, dead);
                if (!ok) break;
                tile_after_sync();
                float z[64];
                tile_ld32(buf, z);
                tile_ld32(buf + 32, z + 32);
                tile_wait_ld();
                if (t * kTileK + kTileK - 1 > a) {                      // not all of the tile's rows see the chunk
                    const int n = a + row - t * kTileK;                 // columns 0 .. n are seen
#pragma unroll
                    for (int j = 0; j < 64; ++j) z[j] = j <= n ? z[j] : -INFINITY;
                }
                float top[4] = {z[0], z[1], z[2], z[3]};
#pragma unroll
                for (int j = 4; j < 60; j += 8)
#pragma unroll
                    for (int e = 0; e < 4; ++e) top[e] = pack_max3(top[e], z[j + 2 * e], z[j + 2 * e + 1]);
#pragma unroll
                for (int e = 0; e < 4; e += 2) top[e] = pack_max3(top[e], z[60 + e], z[61 + e]);
                const float m_chunk = pack_max3(pack_max3(top[0], top[1], top[2]), top[3], top[3]) * sc;
                if (!(m_chunk < INFINITY)) l = NAN;                     // a score that is NaN or +infinity: so is the row
                // A row that has seen nothing yet has outputs and a sum of zero: its maximum starts here.
                const bool grown = m_chunk > m + 8.f && m > -INFINITY;
                if (m == -INFINITY) m = m_chunk;
                if (__any_sync(0xffffffffu, grown)) {                   // (t > 0)
                    ok = outputs(count - 1);                            // those of this chunk wait for its weights
                    if (!ok) break;
                    tile_after_sync();
                    const float f = grown ? fast_exp2(m - m_chunk) : 1.f;
                    if (grown) { m = m_chunk; l *= f; }
                    for (int y = 0; y < 4 * w.layers; ++y) {            // 16 columns at a time: the scores are still held
                        float o[16];
                        tile_ld16(lanes + kOut + y * 16, o);
                        tile_wait_ld();
#pragma unroll
                        for (int j = 0; j < 16; ++j) o[j] *= f;
                        tile_st16(lanes + kOut + y * 16, o);
                    }
                }
                const float base_m = m == -INFINITY ? 0.f : m;
                unsigned long long sum[2] = {0ull, 0ull};
                const unsigned long long m2 = tile_pair(-base_m, -base_m);
                float packed[32];
#pragma unroll
                for (int j = 0; j < 64; j += 2) {
                    float u, v;
                    const unsigned long long x2 = tile_fma2(tile_pair(z[j], z[j + 1]), sc2, m2);
                    if ((j >> 1) * kPackPoly % 8 < kPackPoly) {
                        pack_exp2(x2, u, v);
                    } else {
                        tile_unpair(x2, u, v);
                        u = fast_exp2(u);
                        v = fast_exp2(v);
                    }
                    sum[(j >> 1) & 1] = tile_add2(sum[(j >> 1) & 1], tile_pair(u, v));
                    packed[j >> 1] = __uint_as_float(pack_bf16(u, v));
                }
                tile_st16(buf, packed);                                 // over the scores, which have been read
                tile_st16(buf + 16, packed + 16);
                float sa, sb;
                tile_unpair(tile_add2(sum[0], sum[1]), sa, sb);
                l += sa + sb;
                tile_wait_st();
                tile_before_sync();
                __syncwarp();
                if (lane == 0) tile_arrive(&p_full[x][count & 1]);
            }
            if (!ok) break;
            ok = outputs(count - 1);
            if (!ok) break;
            tile_after_sync();
            // Loops that stay loops: this code runs once an item, and unrolled it took three times as long to fetch as to run.  A row's 128
            // bytes go by way of shared memory, so that eight lanes write them side by side.
            const float inv = l == 0.f ? 0.f : __fdividef(1.f, l);
            const int left = min(w.rows - x * kTileQ - quarter * 32, 32);          // of the warp's rows that are there
            bool odd = false;
            __nv_bfloat16* dst = p.out + w.layer0 * p.out_layer + (long long)(w.token0 + a + quarter * 32 + (lane >> 3)) * p.out_ld + w.head * kDh + (lane & 7) * 8;
#pragma unroll 1
            for (int y = 0; y < w.layers; ++y, dst += p.out_layer) {
#pragma unroll 1
                for (int h = 0; h < 4; ++h) {
                    float o[16];
                    tile_ld16(lanes + kOut + y * 64 + h * 16, o);
                    tile_wait_ld();
#pragma unroll
                    for (int c = 0; c < 16; ++c) { o[c] *= inv; odd |= o[c] != o[c]; }
#pragma unroll
                    for (int c = 0; c < 2; ++c)
                        *reinterpret_cast<uint4*>(mine + lane * 128 + (((2 * h + c) ^ (lane & 7)) << 4)) =
                            make_uint4(pack_bf16(o[8 * c], o[8 * c + 1]), pack_bf16(o[8 * c + 2], o[8 * c + 3]),
                                       pack_bf16(o[8 * c + 4], o[8 * c + 5]), pack_bf16(o[8 * c + 6], o[8 * c + 7]));
                }
                if (y + 1 == w.layers) tile_before_sync();
                __syncwarp();
                if (y + 1 == w.layers && lane == 0) tile_arrive(&o_free[x]);       // the next item's may take their place
#pragma unroll 2
                for (int r = lane >> 3; r < left; r += 4)
                    *reinterpret_cast<uint4*>(dst + (r - (lane >> 3)) * p.out_ld) = *reinterpret_cast<const uint4*>(mine + r * 128 + (((lane & 7) ^ (r & 7)) << 4));
                __syncwarp();
            }
            if (odd && lane < left) again_s[warp] = 1;
        }
        if (!ok && lane == 0 && p.status && atomicCAS(&p.status[0], 0, (int)SAN_ERR_TIMEOUT) == 0) { p.status[1] = TAG_PACKED; p.status[2] = w.seq; }
        // Behind all items, when no wait is under way any more: a row of a long sequence may take longer than a wait may last.
        __syncwarp();
        if (ok && again_s[warp]) packed_items_again(p, x, quarter, mine, lane);
    }
    tile_before_sync();
    __syncthreads();
    if (warp == 10) {
        __syncwarp();
        asm volatile("tcgen05.dealloc.cta_group::1.sync.aligned.b32 %0, %1;" :: "r"(tmem), "r"(kCols) : "memory");
    }
}

}  // namespace san
