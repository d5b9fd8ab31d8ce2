// One decode step of attention over cached rows, for one query position per sequence, in two forms:
//   san_window_attn   a row sees the last `window` rows of its cache and the first `n_sink` ones;
//   san_prefix_attn   a row sees all of its cache and, in front of it, a prefix that it shares with
//                     other rows of the batch.
// As everywhere in this library the weights of a block are computed once and applied to the values
// of each of its layers (Eq. 3, Eq. 4):
//     O_l = sum_j S_j V_l[j],   S = Softmax(q.K^T / 8) over the rows j that are seen.
//
// The call is bound by reading keys and values once: (1 + layers) * 128 bytes per position and
// key head (bf16) against 4 * 64 * (1 + layers) operations per query row.  What is laid out for that:
//   * A UNIT is (key head, up to 8 query rows that share its keys, layer group, a run of positions).  For a
//     sequence's own rows the query rows are the query heads of the key head's group; for a prefix they
//     are those of every sequence behind the prefix, so that the prefix is read once for all of them.
//   * A unit is streamed by 1 or 4 warps.  Each warp has a ring of slots of its own in shared memory (32 rows
//     of one plane each), filled by 16-byte cp.async all but one of the slots ahead: no barrier between warps until
//     their partial results meet at the end of the unit.
//   * One pass with the running maximum and sum of the softmax; scores never leave the registers.  bf16
//     rows go through mma.sync.m16n8k16 with the queries as N.  With one query row seven of eight columns are padding,
//     and it is still the cheapest form: about 5 warp instructions per position against 12 on the CUDA cores.  float32 rows (tolerance
//     1e-5) stay on the CUDA cores: a lane scores one position for up to 8 query rows, then owns two dims.
//   * Units of the same row (runs of a long row; its prefix and its own rows) leave (max, sum, unnormalised
//     outputs) in the workspace and attend_join_kernel adds them up, launched with programmatic stream
//     serialisation.  Nothing there has to be cleared between calls, no unit waits for another one, and
//     the order of the additions is fixed.  A row with a single unit is finished by it.
// Measured: 128 rows of 516 visible positions, 8 heads, 4 layers 53.0 us = 5.8 TB/s, 0.88 of the measured copy bandwidth
// (66 us with the queries as M: twice the accumulators, half the warps); 32 prefixes of 512 positions for 4 rows each with
// own rows of 1 to 255, 4 layers 36 us (50 before the runs were cut by a warp's share of the call).
// Positions that a row does not see are not read (their place in shared memory is filled with
// zeros), so what lies behind the end of a sequence or between the sinks and the window does not matter.
#pragma once

#include "san_kernels.cuh"

namespace san {

constexpr int TAG_ATTEND = 9, TAG_PREFIX = 10;
constexpr int kAtWarps = 4;                 // warps of a CTA
constexpr int kAtTile = 32;                 // positions per slot
constexpr int kAtMaxLayers = 4;             // layers whose outputs a warp accumulates at once

template <typename T> struct AttendGeom;
constexpr int kAtRows = 8;                  // query rows of a unit: one N of mma.sync
constexpr int kAtOutLd = 68;                // floats between the rows of outputs in shared memory (no bank conflicts)
template <> struct AttendGeom<__nv_bfloat16> { static constexpr int kRowBytes = 128; };
template <> struct AttendGeom<float>         { static constexpr int kRowBytes = 256; };
// N: slots of a warp's ring.
template <typename T, int N> __host__ __device__ constexpr int attend_warp_bytes() {       // ring; float32: query rows and weights behind it
    return N * kAtTile * AttendGeom<T>::kRowBytes +
           (sizeof(T) == 4 ? kAtRows * kDh * 4 + kAtTile * kAtRows * 4 : 0);
}
template <typename T, int N> __host__ __device__ constexpr int attend_smem_bytes() { return kAtWarps * (attend_warp_bytes<T, N>() + 2 * kAtRows * 4); }

struct AttendParams {
    const char* q; char* out;
    int H, Hk, group, n_layers, n_items;    // group = H / Hk query heads per key head
    // the sequences' own rows: planes [max_ids][Hk][cap][64] as the context keeps them
    const char* k; const char* v; long long v_stride;           // bytes between the layers' value planes
    int max_ids, cap, max_len, window, n_sink;                  // window 0: all rows are seen
    const int* ids; const int* lens;
    // shared prefixes: [n_prefix][pcap][Hk][64], rows in natural order
    const char* pk; const char* pv; long long pv_stride;
    int n_prefix, pcap, max_prefix, max_group;
    const int* plens; const int* first;
    // how the work is cut
    int lg, n_lg;                           // layers per unit
    int p_units, p_row_tiles, p_splits, p_span, p_wpu;          // units, runs of p_span tiles, warps per unit
    int o_units, o_row_tiles, o_splits, o_span, o_wpu;
    int p_ctas;                             // CTAs of the prefix units; those of the own rows follow
    int t_lg, t_n_lg;                       // layers per unit of the tensor-core tiles (0: the prefixes are not theirs)
    int slots;                              // partial results per row; 1: units write the outputs
    float* part_o;                          // [slot][layer][item * H + head][64]
    float2* part_ml;                        // [slot][item * H + head]
    int* status;
    float scale_log2e;
};

__device__ __forceinline__ void attend_error(int* status, int tag, int item, int value, int limit) {
    if (status) record_error(status, tag, item, value, limit);
}

// The prefix of an item: the g with first[g] <= item < first[g + 1], or -1.
__device__ __forceinline__ int prefix_of(const AttendParams& p, int item) {
    if (p.n_prefix == 0 || item < p.first[0] || item >= p.first[p.n_prefix]) return -1;
    int lo = 0, hi = p.n_prefix;            // first[lo] <= item < first[hi]
    while (hi - lo > 1) {
        const int mid = (lo + hi) >> 1;
        if (p.first[mid] <= item) lo = mid; else hi = mid;
    }
    return lo;
}
// A prefix whose description is in order.  An empty one (no rows behind it) is.
__device__ __forceinline__ bool prefix_ok(const AttendParams& p, int g) {
    const int a = p.first[g], b = p.first[g + 1], len = p.plens[g];
    return a >= 0 && b >= a && b <= p.n_items && b - a <= p.max_group && len >= 0 && len <= p.max_prefix;
}
__device__ __forceinline__ void prefix_report(const AttendParams& p, int g) {
    const int count = p.first[g + 1] - p.first[g];
    const bool by_len = p.plens[g] < 0 || p.plens[g] > p.max_prefix;
    attend_error(p.status, TAG_PREFIX, g, by_len ? p.plens[g] : count, by_len ? p.max_prefix : p.max_group);
}
__device__ __forceinline__ bool own_ok(const AttendParams& p, int item) {
    const int id = p.ids[item], len = p.lens[item];
    return id >= 0 && id < p.max_ids && len >= 0 && len <= p.max_len;
}

// What a unit reads: `n` positions, the first n_sink of them at 0.., the others from `lo` on.
struct AttendRun {
    const char* k; const char* v;
    long long row_bytes, v_stride;
    bool permuted;                          // chunk c of the row at pos sits at c ^ (pos & 7)
    int n_sink, lo, n;                      // visible rows (of the whole sequence)
    int begin, end;                         // this unit's part of them
    int item0, row0, rows, head0;           // query row i: item item0 + (row0 + i) / group, head head0 + (row0 + i) % group
    int layer0, layers, slot;
};

__device__ __forceinline__ void cp16(uint32_t dst, const void* src, bool full) {
    const int n = full ? 16 : 0;            // 0: the 16 bytes are filled with zeros and nothing is read
    asm volatile("cp.async.cg.shared.global [%0], [%1], 16, %2;" :: "r"(dst), "l"(src), "r"(n) : "memory");
}
__device__ __forceinline__ void cp_commit() { asm volatile("cp.async.commit_group;" ::: "memory"); }
template <int N> __device__ __forceinline__ void cp_wait() { asm volatile("cp.async.wait_group %0;" :: "n"(N) : "memory"); }

__device__ __forceinline__ void ldsm4(uint32_t* r, uint32_t addr) {
    asm volatile("ldmatrix.sync.aligned.m8n8.x4.shared.b16 {%0,%1,%2,%3}, [%4];"
                 : "=r"(r[0]), "=r"(r[1]), "=r"(r[2]), "=r"(r[3]) : "r"(addr) : "memory");
}
__device__ __forceinline__ void ldsm4t(uint32_t* r, uint32_t addr) {
    asm volatile("ldmatrix.sync.aligned.m8n8.x4.trans.shared.b16 {%0,%1,%2,%3}, [%4];"
                 : "=r"(r[0]), "=r"(r[1]), "=r"(r[2]), "=r"(r[3]) : "r"(addr) : "memory");
}
__device__ __forceinline__ void mma_bf16(float* d, const uint32_t* a, uint32_t b0, uint32_t b1) {
    asm volatile("mma.sync.aligned.m16n8k16.row.col.f32.bf16.bf16.f32 {%0,%1,%2,%3}, {%4,%5,%6,%7}, {%8,%9}, {%0,%1,%2,%3};"
                 : "+f"(d[0]), "+f"(d[1]), "+f"(d[2]), "+f"(d[3]) : "r"(a[0]), "r"(a[1]), "r"(a[2]), "r"(a[3]), "r"(b0), "r"(b1));
}
__device__ __forceinline__ uint32_t pack_bf16(float lo, float hi) {
    __nv_bfloat162 v = __floats2bfloat162_rn(lo, hi);
    return *reinterpret_cast<uint32_t*>(&v);
}
__device__ __forceinline__ float fast_exp2(float x) {
    float y;
    asm("ex2.approx.ftz.f32 %0, %1;" : "=f"(y) : "f"(x));
    return y;
}

// Fills one slot with rows [begin, begin + 32) of the visible ones, layer `plane` (-1: keys).
template <typename T>
__device__ __forceinline__ void attend_fill(const AttendRun& u, int begin, int end, int plane, uint32_t slot, int lane) {
    constexpr int RB = AttendGeom<T>::kRowBytes, CPR = RB / 16, RPI = 32 / CPR;     // chunks per row, rows per instruction
    const char* base = plane < 0 ? u.k : u.v + plane * u.v_stride;
    const int c_smem = lane % CPR, q = lane / CPR;
    const uint32_t dst = slot + q * RB + c_smem * 16;
    if (begin >= u.n_sink && begin + kAtTile <= end) {       // 32 rows on end
        const int pos = u.lo + begin - u.n_sink + q;
        const char* src = base + pos * u.row_bytes;
        const long long step = RPI * u.row_bytes;
        int off[8 / RPI];                                    // the chunk to fetch: row j * RPI + q has 8 / RPI swizzles
#pragma unroll
        for (int j = 0; j < 8 / RPI; ++j) {
            const int c = c_smem ^ ((j * RPI + q) & 7);
            off[j] = (u.permuted ? c ^ ((pos + j * RPI) & 7) : c) << 4;
        }
#pragma unroll
        for (int j = 0; j < kAtTile / RPI; ++j, src += step) cp16(dst + j * RPI * RB, src + off[j % (8 / RPI)], true);
    } else {
#pragma unroll
        for (int j = 0; j < kAtTile / RPI; ++j) {
            const int r = j * RPI + q, at = begin + r;
            const bool full = at < end;
            const int pos = !full ? 0 : at < u.n_sink ? at : u.lo + (at - u.n_sink);
            const int c = c_smem ^ (r & 7);
            const char* src = base + pos * u.row_bytes + ((u.permuted ? c ^ (pos & 7) : c) << 4);
            cp16(dst + j * RPI * RB, src, full);
        }
    }
    cp_commit();
}

// Where a unit's row goes, and the meeting of the warps of a unit.  Every warp of the CTA calls this (it
// holds CTA barriers).  In shared memory: per warp [layers][kAtRows] rows of 64 outputs, kAtOutLd floats
// apart, at the start of its part, (max, sum) per row at `ml`; warps of a unit are neighbours.
template <typename T, int N>
__device__ __forceinline__ void attend_finish(const AttendParams& p, const AttendRun& u, bool active, int wpu, char* smem,
                                              const float2* ml, int warp, int lane) {
    constexpr int R = kAtRows;
    __syncthreads();
    if (!active) return;
    const int w0 = warp / wpu * wpu;
    const long long n_rows = (long long)p.n_items * p.H;
    // a unit's warps share its rows: 16 lanes and float4 for a row's 64 outputs
    const int threads = wpu * 32, t = (warp - w0) * 32 + lane;
    for (int i = t >> 4; i < u.rows; i += threads >> 4) {
        float m = -INFINITY;
        for (int w = 0; w < wpu; ++w) m = fmaxf(m, ml[(w0 + w) * R + i].x);
        float l = 0.f, weight[kAtWarps];
#pragma unroll
        for (int w = 0; w < kAtWarps; ++w) {
            if (w >= wpu) { weight[w] = 0.f; continue; }
            const float2 x = ml[(w0 + w) * R + i];
            weight[w] = x.y > 0.f ? (x.x == m ? 1.f : exp2f(x.x - m)) : x.y;      // nothing seen: 0 (and NaN stays NaN)
            l += weight[w] * x.y;
        }
        const int row = u.row0 + i, item = u.item0 + row / p.group, head = u.head0 + row % p.group;
        const long long at = (long long)item * p.H + head;
        const bool direct = p.slots == 1;
        const float inv = direct ? (l == 0.f ? 0.f : 1.f / l) : 1.f;
        if (!direct && (t & 15) == 0 && u.layer0 == 0) p.part_ml[u.slot * n_rows + at] = make_float2(m, l);
        if (!direct && l == 0.f) continue;                                        // the join does not look at it
        for (int y = 0; y < u.layers; ++y) {
            float4 o = make_float4(0.f, 0.f, 0.f, 0.f);
#pragma unroll
            for (int w = 0; w < kAtWarps; ++w) {
                if (w >= wpu || weight[w] == 0.f) continue;
                const float4 x = *reinterpret_cast<const float4*>(smem + (w0 + w) * attend_warp_bytes<T, N>() + ((y * R + i) * kAtOutLd + (t & 15) * 4) * 4);
                o.x += weight[w] * x.x; o.y += weight[w] * x.y; o.z += weight[w] * x.z; o.w += weight[w] * x.w;
            }
            const int layer = u.layer0 + y;
            if (direct) {
                T* dst = reinterpret_cast<T*>(p.out) + ((long long)layer * n_rows + at) * kDh + (t & 15) * 4;
                if constexpr (sizeof(T) == 4) {
                    *reinterpret_cast<float4*>(dst) = make_float4(o.x * inv, o.y * inv, o.z * inv, o.w * inv);
                } else {
                    *reinterpret_cast<uint2*>(dst) = make_uint2(pack_bf16(o.x * inv, o.y * inv), pack_bf16(o.z * inv, o.w * inv));
                }
            } else {
                *reinterpret_cast<float4*>(p.part_o + (((long long)u.slot * p.n_layers + layer) * n_rows + at) * kDh + (t & 15) * 4) = o;
            }
        }
    }
}

// Walks a warp's tiles: fill() runs N - 1 slots ahead of use.  The slots of a tile are its keys and then the
// values of each layer.
template <typename T, int N> struct AttendRing {
    static constexpr int SB = kAtTile * AttendGeom<T>::kRowBytes;
    const AttendRun& u; uint32_t ring; int lane, step;      // step: positions between this warp's tiles
    int f_at, f_plane, f_slot, r_slot;
    __device__ __forceinline__ AttendRing(const AttendRun& run, uint32_t smem, int ln, int first, int stp)
        : u(run), ring(smem), lane(ln), step(stp), f_at(first), f_plane(-1), f_slot(0), r_slot(0) {
        for (int i = 0; i < N - 1; ++i) fill();
    }
    __device__ __forceinline__ void fill() {
        if (f_at < u.end) {
            attend_fill<T>(u, f_at, u.end, f_plane, ring + f_slot * SB, lane);
            if (++f_plane == u.layers) { f_plane = -1; f_at += step; }
            f_slot = f_slot + 1 == N ? 0 : f_slot + 1;
        } else {
            cp_commit();                                     // an empty group keeps the count
        }
    }
    // Offset of the next slot in order, arrived; every lane is done with the one before it, which is refilled.
    __device__ __forceinline__ uint32_t next() {
        cp_wait<N - 2>();
        __syncwarp();
        fill();
        const uint32_t s = r_slot * SB;
        r_slot = r_slot + 1 == N ? 0 : r_slot + 1;
        return s;
    }
};

// bf16, up to eight query rows, which are the N side of both products: scores D[16 positions x 8 queries] with
// the key rows as A, outputs D[16 dims x 8 queries] with the value rows, transposed by ldmatrix, as A.
template <int LG, int N, class Params>
__device__ __forceinline__ void attend_warp_bf16(const Params& p, const AttendRun& u, int first, int step, char* smem, float2* ml, int lane) {
    const uint32_t ring_addr = (uint32_t)__cvta_generic_to_shared(smem);
    AttendRing<__nv_bfloat16, N> ring(u, ring_addr, lane, first, step);
    const int g = lane >> 2, t4 = lane & 3;
    uint32_t qb[4][2];                                       // B: query g, dims 16 c + 2 t4 .. and 8 further on
    {
        const bool real = g < u.rows;
        const int row = u.row0 + (real ? g : 0), item = u.item0 + row / p.group, head = u.head0 + row % p.group;
        const uint32_t* src = reinterpret_cast<const uint32_t*>(p.q + ((long long)item * p.H + head) * 128) + t4;
#pragma unroll
        for (int c = 0; c < 4; ++c) {
            qb[c][0] = real ? src[c * 8] : 0u;
            qb[c][1] = real ? src[c * 8 + 4] : 0u;
        }
    }
    float acc[LG][4][4];                                     // [layer][16 dims]: dims g and g + 8, queries 2 t4 and 2 t4 + 1
#pragma unroll
    for (int y = 0; y < LG; ++y)
#pragma unroll
        for (int d = 0; d < 4; ++d)
#pragma unroll
            for (int e = 0; e < 4; ++e) acc[y][d][e] = 0.f;
    float m[2] = {-INFINITY, -INFINITY}, l[2] = {0.f, 0.f};

    const int r8 = lane & 7, mat = lane >> 3;
    const uint32_t k_row = ((mat & 1) * 8 + r8) * 128, v_row = ((mat >> 1) * 8 + r8) * 128;
    uint32_t k_chunk[4], v_chunk[4];
#pragma unroll
    for (int c = 0; c < 4; ++c) {
        k_chunk[c] = (uint32_t)((2 * c + (mat >> 1)) ^ r8) << 4;
        v_chunk[c] = (uint32_t)((2 * c + (mat & 1)) ^ r8) << 4;
    }
    for (int at = first; at < u.end; at += step) {
        const uint32_t ks = ring_addr + ring.next() + k_row;
        float s[2][4];                                       // positions 16 n + g and + 8, queries 2 t4 and 2 t4 + 1
#pragma unroll
        for (int n = 0; n < 2; ++n) {
#pragma unroll
            for (int e = 0; e < 4; ++e) s[n][e] = 0.f;
#pragma unroll
            for (int c = 0; c < 4; ++c) {
                uint32_t a[4];
                ldsm4(a, ks + n * 16 * 128 + k_chunk[c]);
                mma_bf16(s[n], a, qb[c][0], qb[c][1]);
            }
        }
        float top[2] = {-INFINITY, -INFINITY};
        const bool part = at + kAtTile > u.end;
#pragma unroll
        for (int n = 0; n < 2; ++n)
#pragma unroll
            for (int e = 0; e < 4; ++e) {
                s[n][e] = part && at + n * 16 + (e >> 1) * 8 + g >= u.end ? -INFINITY : s[n][e] * p.scale_log2e;
                top[e & 1] = fmaxf(top[e & 1], s[n][e]);
            }
        float alpha[2];
#pragma unroll
        for (int j = 0; j < 2; ++j) {
#pragma unroll
            for (int o = 4; o < 32; o <<= 1) top[j] = fmaxf(top[j], __shfl_xor_sync(0xffffffffu, top[j], o));
            const float m_new = fmaxf(m[j], top[j]);
            const float base = m_new == -INFINITY ? 0.f : m_new;         // all scores -inf so far: weights 0
            alpha[j] = m[j] == m_new ? 1.f : fast_exp2(m[j] - base);
            m[j] = m_new;
            float sum = 0.f;
#pragma unroll
            for (int n = 0; n < 2; ++n)
#pragma unroll
                for (int e = 0; e < 2; ++e) {
                    s[n][2 * e + j] = fast_exp2(s[n][2 * e + j] - base);
                    sum += s[n][2 * e + j];
                }
            l[j] = l[j] * alpha[j] + sum;
        }
        // The weights enter the second product in bf16 (at most half a step, 2^-8 relative, of independent sign); their
        // sum is that of the float32 ones.  As B they have to hold neighbouring positions: an 8 x 8 transpose.
        uint32_t pb[2][2];
#pragma unroll
        for (int n = 0; n < 2; ++n)
#pragma unroll
            for (int e = 0; e < 2; ++e)
                asm volatile("movmatrix.sync.aligned.m8n8.trans.b16 %0, %1;" : "=r"(pb[n][e]) : "r"(pack_bf16(s[n][2 * e], s[n][2 * e + 1])));
        if (__any_sync(0xffffffffu, alpha[0] != 1.f || alpha[1] != 1.f)) {
#pragma unroll
            for (int y = 0; y < LG; ++y)
#pragma unroll
                for (int d = 0; d < 4; ++d)
#pragma unroll
                    for (int e = 0; e < 4; ++e) acc[y][d][e] *= alpha[e & 1];
        }
#pragma unroll
        for (int y = 0; y < LG; ++y) {
            if (y >= u.layers) break;
            const uint32_t vs = ring_addr + ring.next() + v_row;
#pragma unroll
            for (int n = 0; n < 2; ++n)
#pragma unroll
                for (int d = 0; d < 4; ++d) {
                    uint32_t a[4];
                    ldsm4t(a, vs + n * 16 * 128 + v_chunk[d]);
                    mma_bf16(acc[y][d], a, pb[n][0], pb[n][1]);
                }
        }
    }
    cp_wait<0>();
    __syncwarp();
#pragma unroll
    for (int j = 0; j < 2; ++j) {
#pragma unroll
        for (int o = 4; o < 32; o <<= 1) l[j] += __shfl_xor_sync(0xffffffffu, l[j], o);
        const int row = 2 * t4 + j;
        if (g == 0) ml[row] = make_float2(m[j], l[j]);
        if (row < u.rows) {
            float* out = reinterpret_cast<float*>(smem) + row * kAtOutLd + g;
#pragma unroll
            for (int y = 0; y < LG; ++y)
#pragma unroll
                for (int d = 0; d < 4; ++d) {
                    out[y * kAtRows * kAtOutLd + d * 16] = acc[y][d][j];
                    out[y * kAtRows * kAtOutLd + d * 16 + 8] = acc[y][d][2 + j];
                }
        }
    }
}

// float32, up to R query rows on the CUDA cores.
template <int LG, int R, int N>
__device__ __forceinline__ void attend_warp_f32(const AttendParams& p, const AttendRun& u, int first, int step, char* smem, float2* ml, int lane) {
    constexpr int RMAX = kAtRows;
    AttendRing<float, N> ring(u, (uint32_t)__cvta_generic_to_shared(smem), lane, first, step);
    float* qs = reinterpret_cast<float*>(smem + N * kAtTile * 256);      // [R][64]
    float* ws = qs + RMAX * kDh;                                                                // [32][R] weights
    for (int i = 0; i < R; ++i) {
        const bool real = i < u.rows;
        const int row = u.row0 + (real ? i : 0), item = u.item0 + row / p.group, head = u.head0 + row % p.group;
        const float2* src = reinterpret_cast<const float2*>(p.q + ((long long)item * p.H + head) * 256);
        reinterpret_cast<float2*>(qs + i * kDh)[lane] = real ? src[lane] : make_float2(0.f, 0.f);
    }
    float acc[LG][R][2], m[R], l[R];
#pragma unroll
    for (int i = 0; i < R; ++i) {
        m[i] = -INFINITY; l[i] = 0.f;
#pragma unroll
        for (int y = 0; y < LG; ++y) acc[y][i][0] = acc[y][i][1] = 0.f;
    }
    __syncwarp();
    for (int at = first; at < u.end; at += step) {
        const uint32_t ks = ring.next();
        float s[R];
#pragma unroll
        for (int i = 0; i < R; ++i) s[i] = 0.f;
#pragma unroll
        for (int c = 0; c < 16; ++c) {
            const float4 k = *reinterpret_cast<const float4*>(smem + ks + lane * 256 + ((c ^ (lane & 7)) << 4));
#pragma unroll
            for (int i = 0; i < R; ++i) {
                const float4 q = *reinterpret_cast<const float4*>(qs + i * kDh + c * 4);
                s[i] = fmaf(q.x, k.x, fmaf(q.y, k.y, fmaf(q.z, k.z, fmaf(q.w, k.w, s[i]))));
            }
        }
        bool moved = false;
        float alpha[R];
#pragma unroll
        for (int i = 0; i < R; ++i) {
            s[i] = at + lane < u.end ? s[i] * p.scale_log2e : -INFINITY;
            const float m_new = fmaxf(m[i], warp_max(s[i]));
            const float b = m_new == -INFINITY ? 0.f : m_new;
            alpha[i] = m[i] == m_new ? 1.f : exp2f(m[i] - b);
            moved |= m[i] != m_new;
            m[i] = m_new;
            s[i] = exp2f(s[i] - b);
            l[i] = l[i] * alpha[i] + s[i];                    // this lane's positions; joined at the end
        }
        __syncwarp();
#pragma unroll
        for (int i = 0; i < R; ++i) ws[lane * R + i] = s[i];
        __syncwarp();
        if (moved)                                            // the same in all lanes
#pragma unroll
            for (int y = 0; y < LG; ++y)
#pragma unroll
                for (int i = 0; i < R; ++i) { acc[y][i][0] *= alpha[i]; acc[y][i][1] *= alpha[i]; }
#pragma unroll
        for (int y = 0; y < LG; ++y) {
            if (y >= u.layers) break;
            const uint32_t vs = ring.next();
#pragma unroll 8
            for (int j = 0; j < kAtTile; ++j) {
                const float2 v = *reinterpret_cast<const float2*>(smem + vs + j * 256 + ((((lane >> 1) ^ (j & 7)) << 4) | ((lane & 1) << 3)));
                float w[R];
                if constexpr (R % 4 == 0) {
#pragma unroll
                    for (int i = 0; i < R; i += 4) *reinterpret_cast<float4*>(w + i) = *reinterpret_cast<const float4*>(ws + j * R + i);
                } else {
#pragma unroll
                    for (int i = 0; i < R; ++i) w[i] = ws[j * R + i];
                }
#pragma unroll
                for (int i = 0; i < R; ++i) {
                    acc[y][i][0] = fmaf(w[i], v.x, acc[y][i][0]);
                    acc[y][i][1] = fmaf(w[i], v.y, acc[y][i][1]);
                }
            }
            }
    }
    cp_wait<0>();
    __syncwarp();
#pragma unroll
    for (int i = 0; i < R; ++i) {
        l[i] = warp_sum(l[i]);
        if (lane == 0) ml[i] = make_float2(m[i], l[i]);
#pragma unroll
        for (int y = 0; y < LG; ++y)
            *reinterpret_cast<float2*>(smem + ((y * RMAX + i) * kAtOutLd + lane * 2) * 4) = make_float2(acc[y][i][0], acc[y][i][1]);
    }
}

// Unit `index` of the prefix units or of the sequences' own rows.  False: nothing to do (reported where the input
// is at fault).
template <typename T>
__device__ __forceinline__ bool attend_unit(const AttendParams& p, bool prefix, int index, bool reporter, AttendRun* u) {
    constexpr int R = kAtRows, RB = AttendGeom<T>::kRowBytes;
    if (index >= (prefix ? p.p_units : p.o_units)) return false;
    const int lg = index % p.n_lg; index /= p.n_lg;
    const int splits = prefix ? p.p_splits : p.o_splits, span = (prefix ? p.p_span : p.o_span) * kAtTile;
    const int split = index % splits; index /= splits;
    const int hk = index % p.Hk; index /= p.Hk;
    u->head0 = hk * p.group;
    u->layer0 = lg * p.lg;
    u->layers = min(p.lg, p.n_layers - u->layer0);
    if (prefix) {
        const int tile = index % p.p_row_tiles, g = index / p.p_row_tiles;
        if (!prefix_ok(p, g)) {
            if (reporter && tile == 0 && split == 0 && hk == 0 && lg == 0) prefix_report(p, g);
            return false;
        }
        const int rows = (p.first[g + 1] - p.first[g]) * p.group;
        u->item0 = p.first[g];
        u->row0 = tile * R;
        u->rows = min(R, rows - u->row0);
        if (u->rows <= 0) return false;
        u->n = p.plens[g]; u->n_sink = 0; u->lo = 0;
        u->row_bytes = (long long)p.Hk * RB;
        const long long at = ((long long)g * p.pcap * p.Hk + hk) * RB;
        u->k = p.pk + at;
        u->v = p.pv + at + u->layer0 * p.pv_stride;
        u->v_stride = p.pv_stride;
        u->permuted = false;
        u->slot = split;
    } else {
        const int tile = index % p.o_row_tiles, item = index / p.o_row_tiles;
        if (!own_ok(p, item)) {
            if (reporter && tile == 0 && split == 0 && hk == 0 && lg == 0) {
                const int id = p.ids[item];
                const bool by_id = id < 0 || id >= p.max_ids;
                attend_error(p.status, TAG_ATTEND, item, by_id ? id : p.lens[item], by_id ? p.max_ids : p.max_len);
            }
            return false;
        }
        u->item0 = item; u->row0 = tile * R; u->rows = min(R, p.group - u->row0);
        const int len = p.lens[item];
        u->lo = p.window > 0 ? max(0, len - p.window) : 0;
        u->n_sink = min(p.n_sink, u->lo);
        u->n = u->n_sink + len - u->lo;
        u->row_bytes = RB;
        const long long at = ((long long)p.ids[item] * p.Hk + hk) * p.cap * RB;
        u->k = p.k + at;
        u->v = p.v + at + u->layer0 * p.v_stride;
        u->v_stride = p.v_stride;
        u->permuted = sizeof(T) == 2;
        u->slot = p.p_splits + split;
    }
    u->begin = min(split * span, u->n);
    u->end = min(u->begin + span, u->n);
    return true;
}

template <typename T, int LG, int N>
__global__ void __launch_bounds__(kAtWarps * 32) attend_kernel(const __grid_constant__ AttendParams p) {
    extern __shared__ __align__(128) char attend_smem[];
    if (p.slots > 1) asm volatile("griddepcontrol.launch_dependents;");       // the join may take its place (and wait there)
    constexpr int R = kAtRows;
    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
    const bool prefix = (int)blockIdx.x < p.p_ctas;
    const int wpu = prefix ? p.p_wpu : p.o_wpu;
    const int cta = prefix ? (int)blockIdx.x : (int)blockIdx.x - p.p_ctas;
    float2* ml = reinterpret_cast<float2*>(attend_smem + kAtWarps * attend_warp_bytes<T, N>());
    AttendRun u;
    const bool active = attend_unit<T>(p, prefix, cta * (kAtWarps / wpu) + warp / wpu, warp % wpu == 0 && lane == 0, &u);
    if (active) {
        char* smem = attend_smem + warp * attend_warp_bytes<T, N>();
        const int first = u.begin + (warp % wpu) * kAtTile, step = wpu * kAtTile;
        if constexpr (sizeof(T) == 2) {
            attend_warp_bf16<LG, N>(p, u, first, step, smem, ml + warp * R, lane);
        } else {
            if (u.rows <= 1) attend_warp_f32<LG, 1, N>(p, u, first, step, smem, ml + warp * R, lane);
            else if (u.rows <= 4) attend_warp_f32<LG, 4, N>(p, u, first, step, smem, ml + warp * R, lane);
            else attend_warp_f32<LG, 8, N>(p, u, first, step, smem, ml + warp * R, lane);
        }
    }
    attend_finish<T, N>(p, u, active, wpu, attend_smem, ml, warp, lane);
    // Beside the tensor-core tiles of the prefixes, launched before: this kernel is not over before they are, so that the
    // join, which waits for this kernel, finds both.
    if (p.t_lg > 0 && blockIdx.x == gridDim.x - 1) asm volatile("griddepcontrol.wait;" ::: "memory");
}

// Adds up the partial results of a row and layer: 16 threads for its outputs, four each, times G groups that
// take every G-th partial result (the loads of a row with many of them are a chain of G times fewer round
// trips).  grid = (rows / (16 / G), layers).
template <typename T, int G>
__global__ void __launch_bounds__(256) attend_join_kernel(const __grid_constant__ AttendParams p) {
    __shared__ float4 s_o[G > 1 ? 256 : 1];
    __shared__ float2 s_ml[G > 1 ? 256 : 1];
    const long long n_rows = (long long)p.n_items * p.H;
    const int c = threadIdx.x & 15, grp = threadIdx.x / 16 % G, layer = blockIdx.y;
    const long long at = (long long)blockIdx.x * (16 / G) + threadIdx.x / (16 * G);
    bool mine = at < n_rows;
    int begin = 0;
    if (mine) {
        const int item = (int)(at / p.H), g = prefix_of(p, item);
        mine = own_ok(p, item) && (g < 0 || prefix_ok(p, g));
        begin = g >= 0 ? 0 : p.p_splits;                // no prefix in front of this row: its own partial results only
    }
    asm volatile("griddepcontrol.wait;" ::: "memory");
    float m = -INFINITY, l = 0.f;
    float4 o = make_float4(0.f, 0.f, 0.f, 0.f);
    auto add = [&](float2 x, float4 v) {
        if (x.y == 0.f) return;                         // nothing seen there: its outputs were not written
        const float m_new = fmaxf(m, x.x);
        const float a = m == m_new ? 1.f : exp2f(m - m_new), b = x.x == m_new ? 1.f : exp2f(x.x - m_new);
        l = l * a + x.y * b;
        o.x = o.x * a + v.x * b; o.y = o.y * a + v.y * b; o.z = o.z * a + v.z * b; o.w = o.w * a + v.w * b;
        m = m_new;
    };
    if (mine) {
#pragma unroll 4
        for (int s = begin + grp; s < p.slots; s += G)
            add(__ldcg(p.part_ml + s * n_rows + at),
                __ldcg(reinterpret_cast<const float4*>(p.part_o + (((long long)s * p.n_layers + layer) * n_rows + at) * kDh + c * 4)));
    }
    if constexpr (G > 1) {
        s_o[threadIdx.x] = o;
        s_ml[threadIdx.x] = make_float2(m, l);
        __syncthreads();
        if (grp != 0) return;
        for (int k = 1; k < G; ++k) add(s_ml[threadIdx.x + k * 16], s_o[threadIdx.x + k * 16]);
    }
    if (!mine) return;
    const float inv = l == 0.f ? 0.f : 1.f / l;
    T* dst = reinterpret_cast<T*>(p.out) + ((long long)layer * n_rows + at) * kDh + c * 4;
    if constexpr (sizeof(T) == 4) *reinterpret_cast<float4*>(dst) = make_float4(o.x * inv, o.y * inv, o.z * inv, o.w * inv);
    else *reinterpret_cast<uint2*>(dst) = make_uint2(pack_bf16(o.x * inv, o.y * inv), pack_bf16(o.z * inv, o.w * inv));
}

}  // namespace san
