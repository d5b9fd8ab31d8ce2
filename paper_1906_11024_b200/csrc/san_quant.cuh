// A cache held in four bits a number: rows stored (san_quant_append), read back (san_quant_read), and one decode step of
// attention over them (san_quant_attn), whose weights serve every layer of a block (Eq. 3, Eq. 4).
//
// A row of 64 numbers x is 32 bytes of codes n (dim d in byte d / 2, the even one in the low half) and a pair of bf16 numbers:
//     low = min x, rounded down;   step = (max x - low) / 15, rounded up;   n = (x - low) / step, rounded half to even;
// it reads as low + step n.  Rounded that way low and step cover the row, so that no number is off by more than step / 2.
// Which code a number gets is decided as if in 64 bits: float32 where the quotient is clear of a border, doubles next to one.
//
// Attention.  Codes enter both products as whole numbers, which bf16 holds exactly, and a row's (step, low) is applied to its
// score and to its weight, once for 64 numbers:
//     q . x = step (q . n') + mid (sum of q),   sum_j S_j x_j = sum_j (S_j step_j) n'_j + sum_j S_j mid_j,
// with n' = n - 8 and mid = low + 8 step.  So a product loses nothing to the cache's format, and float32 queries (three bf16 numbers
// that add up to them, weights likewise) keep float32's accuracy on the tensor cores.
#pragma once

#include <type_traits>

#include "san_attend.cuh"

namespace san {

constexpr int TAG_QUANT = 13, TAG_QUANT_ROWS = 14;
constexpr int kQuantRow = 32;               // bytes of codes of a row
constexpr int kQuantTile = 64;              // positions per slot: 2 KB of codes, then their (step, low)
constexpr int kQuantSlot = kQuantTile * (kQuantRow + 4);

// ------------------------------------------------------------------------------------------- rows in and out
struct QuantRowsParams {
    char* k; char* v; char* ks; char* vs;
    long long v_stride, s_stride;           // bytes between the layers' planes of codes, of (step, low)
    const char* k_rows; const char* v_rows; // [n_items][rows][Hk][64], [layers] of those
    const int* ids; const int* pos; const int* nrows;
    int n_items, rows, Hk, n_layers, max_ids, cap;
    int* status;
};

__device__ __forceinline__ float bf16_down(float x) {       // of a finite x: the largest bf16 number not above it
    const int b = __float_as_int(x);
    return __int_as_float((b >= 0 ? b : b + 0xffff) & 0xffff0000);
}
__device__ __forceinline__ float bf16_up_positive(float x) { return __int_as_float((__float_as_int(x) + 0xffff) & 0xffff0000); }

// The place of a row of eight lanes (`row`: numbered layer, item, head, position, the last the fastest; layer 0: keys): false if it is
// none.  src: of the row's 64 numbers in elements, from the keys' or the layer's first.
struct QuantPlace { int layer; long long src, panel; int pos; };
__device__ __forceinline__ bool quant_place(const QuantRowsParams& p, long long row, bool reporter, QuantPlace* at) {
    if (row >= (long long)(1 + p.n_layers) * p.n_items * p.Hk * p.rows) return false;
    const int r = (int)(row % p.rows); row /= p.rows;
    const int h = (int)(row % p.Hk); row /= p.Hk;
    const int item = (int)(row % p.n_items);
    at->layer = (int)(row / p.n_items);
    const int id = p.ids[item], pos = p.pos ? p.pos[item] : 0, n = p.nrows ? p.nrows[item] : p.rows;
    const bool by_id = id < 0 || id >= p.max_ids, by_n = n < 0 || n > p.rows;
    if (by_id || by_n || pos < 0 || pos > p.cap - n) {
        if (reporter && at->layer == 0 && r == 0 && h == 0)
            attend_error(p.status, TAG_QUANT_ROWS, item, by_id ? id : by_n ? n : pos, by_id ? p.max_ids : by_n ? p.rows : p.cap);
        return false;
    }
    at->src = (((long long)item * p.rows + r) * p.Hk + h) * kDh;
    at->panel = (long long)id * p.Hk + h;
    at->pos = pos + r;
    return r < n;
}

template <typename T>
__global__ void __launch_bounds__(256) quant_append_kernel(const __grid_constant__ QuantRowsParams p) {
    const int c = threadIdx.x & 7;                          // numbers 8 c .. 8 c + 7 of the row
    QuantPlace at;
    const bool real = quant_place(p, (long long)blockIdx.x * 32 + (threadIdx.x >> 3), c == 0, &at);
    float x[8];
    if (real) {
        const T* src = reinterpret_cast<const T*>(at.layer == 0 ? p.k_rows : p.v_rows) + at.src + c * 8;
        if (at.layer > 0) src += (long long)(at.layer - 1) * p.n_items * p.rows * p.Hk * kDh;
        if constexpr (sizeof(T) == 2) {
            unpack16<__nv_bfloat16>(ld16_stream(src), x);
        } else {
            unpack16<float>(ld16_stream(src), x);
            unpack16<float>(ld16_stream(src + 4), x + 4);
        }
    } else {
#pragma unroll
        for (int i = 0; i < 8; ++i) x[i] = 0.f;
    }
    float lo = x[0], hi = x[0];
    bool finite = true;
#pragma unroll
    for (int i = 0; i < 8; ++i) {
        lo = fminf(lo, x[i]); hi = fmaxf(hi, x[i]);
        finite &= fabsf(x[i]) <= 3.4028234e38f;
    }
#pragma unroll
    for (int o = 1; o < 8; o <<= 1) {
        lo = fminf(lo, __shfl_xor_sync(0xffffffffu, lo, o));
        hi = fmaxf(hi, __shfl_xor_sync(0xffffffffu, hi, o));
    }
    const float low = bf16_down(lo);
    const double wide = ((double)hi - (double)low) / 15.0;
    const float step = bf16_up_positive(__double2float_ru(wide));
    const unsigned group = 0xffu << (threadIdx.x & 24);
    finite = (__ballot_sync(0xffffffffu, finite) & group) == group && fabsf(low) <= 3.4028234e38f && step <= 3.4028234e38f;
    uint32_t codes = 0;
    // Steps without a reciprocal: everything times 2^100, which is exact (and low is that small too, since float32 numbers have no
    // closer neighbours elsewhere).  A step of zero: codes of zero.
    const float up = step > 1e-30f ? 1.f : 1.2676506e30f;
    const float step1 = step * up, low1 = low * up, inv = step > 0.f ? 1.f / step1 : 0.f;
#pragma unroll
    for (int i = 0; i < 8; ++i) {
        const float x1 = x[i] * up, t = (x1 - low1) * inv;
        float n = rintf(t);
        if (fabsf(fabsf(t - n) - 0.5f) < 1e-4f) {           // t is within 2e-6 of the quotient; next to a border 64 bits decide
            const float k = floorf(t);
            const double d = (double)x1 - (double)low1, border = ((double)k + 0.5) * (double)step1;
            n = d > border || (d == border && ((int)k & 1)) ? k + 1.f : k;
        }
        codes |= (uint32_t)fminf(fmaxf(n, 0.f), 15.f) << (4 * i);
    }
    if (!real) return;
    char* to = (at.layer == 0 ? p.k : p.v + (at.layer - 1) * p.v_stride) + (at.panel * p.cap + at.pos) * kQuantRow;
    reinterpret_cast<uint32_t*>(to)[c] = finite ? codes : 0u;
    if (c == 0) {
        char* scale = (at.layer == 0 ? p.ks : p.vs + (at.layer - 1) * p.s_stride) + (at.panel * p.cap + at.pos) * 4;
        *reinterpret_cast<uint32_t*>(scale) = finite ? __float_as_uint(step) >> 16 | (__float_as_uint(low) & 0xffff0000u) : 0x7fc07fc0u;
    }
}

template <typename T>
__global__ void __launch_bounds__(256) quant_read_kernel(const __grid_constant__ QuantRowsParams p) {
    const int c = threadIdx.x & 7;
    QuantPlace at;
    if (!quant_place(p, (long long)blockIdx.x * 32 + (threadIdx.x >> 3), c == 0, &at)) return;
    const long long row = at.panel * p.cap + at.pos;
    const uint32_t codes = reinterpret_cast<const uint32_t*>((at.layer == 0 ? p.k : p.v + (at.layer - 1) * p.v_stride) + row * kQuantRow)[c];
    const uint32_t scale = *reinterpret_cast<const uint32_t*>((at.layer == 0 ? p.ks : p.vs + (at.layer - 1) * p.s_stride) + row * 4);
    const float step = __uint_as_float(scale << 16), low = __uint_as_float(scale & 0xffff0000u);
    float x[8];
#pragma unroll
    for (int i = 0; i < 8; ++i) x[i] = fmaf(step, (float)(codes >> (4 * i) & 15u), low);
    T* to = reinterpret_cast<T*>(const_cast<char*>(at.layer == 0 ? p.k_rows : p.v_rows)) + at.src + c * 8;
    if (at.layer > 0) to += (long long)(at.layer - 1) * p.n_items * p.rows * p.Hk * kDh;
    if constexpr (sizeof(T) == 2) {
        *reinterpret_cast<uint4*>(to) = pack16<__nv_bfloat16>(x);
    } else {
        *reinterpret_cast<uint4*>(to) = pack16<float>(x);
        *reinterpret_cast<uint4*>(to + 4) = pack16<float>(x + 4);
    }
}

// ------------------------------------------------------------------------------------------- attention
struct QuantParams {
    AttendParams a;                         // k, v: planes of codes
    const char* ks; const char* vs; long long s_stride;
    float* S; long long ld_s;               // scores, in powers of two, until quant_weights_kernel makes them weights
};
struct QuantRun {
    AttendRun r;
    const char* ks; const char* vs; long long s_stride;
    int item;
};

// N: slots of a warp's ring, later the place of its outputs (up to four layers of eight rows).
template <int N> __host__ __device__ constexpr int quant_warp_bytes() { return N * kQuantSlot; }
template <int N> __host__ __device__ constexpr int quant_smem_bytes() { return kAtWarps * (quant_warp_bytes<N>() + 2 * kAtRows * 4); }

__device__ __forceinline__ void cp4(uint32_t dst, const void* src, bool full) {
    const int n = full ? 4 : 0;
    asm volatile("cp.async.ca.shared.global [%0], [%1], 4, %2;" :: "r"(dst), "l"(src), "r"(n) : "memory");
}

// Fills one slot with positions [begin, begin + 64) of layer `plane` (-1: keys); what lies at or behind `end` becomes zeros.
// Value rows go to places where four lanes find rows 2 t of a block of eight in different banks: row r of eight to r / 2 + 4 (r % 2).
__device__ __forceinline__ void quant_fill(const QuantRun& u, int begin, int end, int plane, uint32_t slot, int lane) {
    const char* codes = plane < 0 ? u.r.k : u.r.v + plane * u.r.v_stride;
    const char* scales = plane < 0 ? u.ks : u.vs + plane * u.s_stride;
    const int half = lane & 1;
#pragma unroll
    for (int j = 0; j < kQuantTile / 16; ++j) {
        const int r = j * 16 + (lane >> 1), pos = begin + r;
        const int to = plane < 0 ? r : (r & ~7) | (r >> 1 & 3) | (r & 1) << 2;
        const bool full = pos < end;
        cp16(slot + to * kQuantRow + half * 16, codes + (long long)(full ? pos : 0) * kQuantRow + half * 16, full);
    }
#pragma unroll
    for (int j = 0; j < kQuantTile / 32; ++j) {
        const int r = j * 32 + lane, pos = begin + r;
        const bool full = pos < end;
        cp4(slot + kQuantTile * kQuantRow + r * 4, scales + (long long)(full ? pos : 0) * 4, full);
    }
    cp_commit();
}

template <int N> struct QuantRing {
    const QuantRun& u; uint32_t ring; int lane, step;
    int f_at, f_plane, f_slot, r_slot;
    __device__ __forceinline__ QuantRing(const QuantRun& run, uint32_t smem, int ln, int first, int stp)
        : u(run), ring(smem), lane(ln), step(stp), f_at(first), f_plane(-1), f_slot(0), r_slot(0) {
        for (int i = 0; i < N - 1; ++i) fill();
    }
    __device__ __forceinline__ void fill() {
        if (f_at < u.r.end) {
            quant_fill(u, f_at, u.r.end, f_plane, ring + f_slot * kQuantSlot, lane);
            if (++f_plane == u.r.layers) { f_plane = -1; f_at += step; }
            f_slot = f_slot + 1 == N ? 0 : f_slot + 1;
        } else {
            cp_commit();
        }
    }
    __device__ __forceinline__ uint32_t next() {
        cp_wait<N - 2>();
        __syncwarp();
        fill();
        const uint32_t s = r_slot * kQuantSlot;
        r_slot = r_slot + 1 == N ? 0 : r_slot + 1;
        return s;
    }
};

// Codes i and i + 4 of a word, less 8, as two bf16 numbers: 0x4300 | n is 128 + n.
__device__ __forceinline__ uint32_t quant_two(uint32_t w, int i) {
    const uint32_t x = (w >> (4 * i) & 0x000f000fu) | 0x43004300u;
    uint32_t y;
    asm("sub.rn.bf16x2 %0, %1, %2;" : "=r"(y) : "r"(x), "r"(0x43084308u));
    return y;
}
// x as P bf16 numbers that add up to it (P = 1: its rounding).
template <int P> __device__ __forceinline__ void quant_split(float x, float y, uint32_t* out) {
#pragma unroll
    for (int k = 0; k < P; ++k) {
        out[k] = pack_bf16(x, y);
        x -= __uint_as_float(out[k] << 16);
        y -= __uint_as_float(out[k] & 0xffff0000u);
    }
}

// Up to eight query rows, which are the N side of both products: scores D[16 positions x 8 queries] with the codes of key rows as
// A, outputs D[16 dims x 8 queries] with those of value rows.  P: 1 for bf16 queries, 3 for float32.
template <int LG, int N, int P>
__device__ __forceinline__ void attend_warp_quant(const QuantParams& p, const QuantRun& u, int first, int step, char* smem, float2* ml, int lane) {
    const uint32_t ring_addr = (uint32_t)__cvta_generic_to_shared(smem);
    QuantRing<N> ring(u, ring_addr, lane, first, step);
    const int g = lane >> 2, t4 = lane & 3;
    // B: query g, dims 16 t4 .. 16 t4 + 15 in the order of the codes' unpacking
    uint32_t qb[8][P];
    float qs[2];                                             // sum of queries 2 t4 and 2 t4 + 1, times the scores' scale
    {
        const bool real = g < u.r.rows;
        const int head = u.r.head0 + u.r.row0 + (real ? g : 0);
        float q[16];
#pragma unroll
        for (int i = 0; i < 16; ++i) q[i] = 0.f;
        const long long at = ((long long)u.item * p.a.H + head) * kDh + t4 * 16;
        if (real) {
            if constexpr (P == 1) {
                const uint4* src = reinterpret_cast<const uint4*>(p.a.q + at * 2);
                unpack16<__nv_bfloat16>(src[0], q);
                unpack16<__nv_bfloat16>(src[1], q + 8);
            } else {
                const uint4* src = reinterpret_cast<const uint4*>(p.a.q + at * 4);
#pragma unroll
                for (int i = 0; i < 4; ++i) unpack16<float>(src[i], q + 4 * i);
            }
        }
        float sum = 0.f;
#pragma unroll
        for (int i = 0; i < 16; ++i) sum = fabsf(q[i]) <= 3.4028234e38f ? sum + q[i] : NAN;
        sum += __shfl_xor_sync(0xffffffffu, sum, 1);
        sum += __shfl_xor_sync(0xffffffffu, sum, 2);
#pragma unroll
        for (int j = 0; j < 2; ++j) qs[j] = __shfl_sync(0xffffffffu, sum, 4 * (2 * t4 + j)) * p.a.scale_log2e;
#pragma unroll
        for (int h = 0; h < 2; ++h)
#pragma unroll
            for (int i = 0; i < 4; ++i) quant_split<P>(q[8 * h + i], q[8 * h + 4 + i], qb[4 * h + i]);
    }
    float acc[LG][4][4], mids[LG][2];        // [layer][d]: dims 8 g + d and 8 g + 4 + d of queries 2 t4, 2 t4 + 1; sums of S mid over rows g
#pragma unroll
    for (int y = 0; y < LG; ++y) {
        mids[y][0] = mids[y][1] = 0.f;
#pragma unroll
        for (int d = 0; d < 4; ++d)
#pragma unroll
            for (int e = 0; e < 4; ++e) acc[y][d][e] = 0.f;
    }
    float m[2] = {-INFINITY, -INFINITY}, l[2] = {0.f, 0.f};
    constexpr int kBlocks = kQuantTile / 16;
    for (int at = first; at < u.r.end; at += step) {
        const char* ks = smem + ring.next();
        float s[kBlocks][4];                                 // positions 16 n + g and + 8, queries 2 t4 and 2 t4 + 1
        float top[2] = {-INFINITY, -INFINITY};
        const bool part = at + kQuantTile > u.r.end;
#pragma unroll
        for (int n = 0; n < kBlocks; ++n) {
            const uint2 w0 = *reinterpret_cast<const uint2*>(ks + (n * 16 + g) * kQuantRow + t4 * 8);
            const uint2 w1 = *reinterpret_cast<const uint2*>(ks + (n * 16 + 8 + g) * kQuantRow + t4 * 8);
            float dot[4] = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
            for (int c = 0; c < 4; ++c) {
                const uint32_t x0 = c < 2 ? w0.x : w0.y, x1 = c < 2 ? w1.x : w1.y;
                const int i = 2 * (c & 1), b = 4 * (c >> 1) + i;
                const uint32_t a[4] = {quant_two(x0, i), quant_two(x1, i), quant_two(x0, i + 1), quant_two(x1, i + 1)};
#pragma unroll
                for (int k = 0; k < P; ++k) mma_bf16(dot, a, qb[b][k], qb[b + 1][k]);
            }
#pragma unroll
            for (int e = 0; e < 2; ++e) {
                const uint32_t scale = *reinterpret_cast<const uint32_t*>(ks + kQuantTile * kQuantRow + (n * 16 + e * 8 + g) * 4);
                const float st = __uint_as_float(scale << 16), mid = fmaf(8.f, st, __uint_as_float(scale & 0xffff0000u));
#pragma unroll
                for (int j = 0; j < 2; ++j) {
                    float z = fmaf(st * p.a.scale_log2e, dot[2 * e + j], mid * qs[j]);
                    if (part && at + n * 16 + e * 8 + g >= u.r.end) z = -INFINITY;
                    s[n][2 * e + j] = z;
                    top[j] = fmaxf(top[j], z);
                }
            }
        }
        if (p.S && u.r.layer0 == 0) {
#pragma unroll
            for (int j = 0; j < 2; ++j) {
                if (2 * t4 + j >= u.r.rows) continue;
                float* to = p.S + ((long long)u.item * p.a.H + u.r.head0 + u.r.row0 + 2 * t4 + j) * p.ld_s + at + g;
#pragma unroll
                for (int n = 0; n < kBlocks; ++n)
#pragma unroll
                    for (int e = 0; e < 2; ++e)
                        if (at + n * 16 + e * 8 + g < u.r.end) to[n * 16 + e * 8] = s[n][2 * e + j];
            }
        }
        float alpha[2];
#pragma unroll
        for (int j = 0; j < 2; ++j) {
#pragma unroll
            for (int o = 4; o < 32; o <<= 1) top[j] = fmaxf(top[j], __shfl_xor_sync(0xffffffffu, top[j], o));
            const float m_new = fmaxf(m[j], top[j]);
            const float base = m_new == -INFINITY ? 0.f : m_new;         // all scores -inf so far: weights 0
            alpha[j] = m[j] == m_new ? 1.f : P == 1 ? fast_exp2(m[j] - base) : exp2f(m[j] - base);
            m[j] = m_new;
            float sum = 0.f;
#pragma unroll
            for (int n = 0; n < kBlocks; ++n)
#pragma unroll
                for (int e = 0; e < 2; ++e) {
                    const float z = s[n][2 * e + j] - base;
                    s[n][2 * e + j] = P == 1 ? fast_exp2(z) : exp2f(z);
                    sum += s[n][2 * e + j];
                }
            l[j] = l[j] * alpha[j] + sum;
        }
        if (__any_sync(0xffffffffu, alpha[0] != 1.f || alpha[1] != 1.f)) {
#pragma unroll
            for (int y = 0; y < LG; ++y) {
                mids[y][0] *= alpha[0]; mids[y][1] *= alpha[1];
#pragma unroll
                for (int d = 0; d < 4; ++d)
#pragma unroll
                    for (int e = 0; e < 4; ++e) acc[y][d][e] *= alpha[e & 1];
            }
        }
#pragma unroll
        for (int y = 0; y < LG; ++y) {
            if (y >= u.r.layers) break;
            const char* vs = smem + ring.next();
#pragma unroll
            for (int n = 0; n < kBlocks; ++n) {
                // Weight times step, in P bf16 numbers.  One (bf16 outputs) is off by half a step, 2^-8 relative, of independent sign
                // over the positions.  As B they have to hold neighbouring positions: an 8 x 8 transpose.
                uint32_t pb[2][P];
#pragma unroll
                for (int e = 0; e < 2; ++e) {
                    const uint32_t scale = *reinterpret_cast<const uint32_t*>(vs + kQuantTile * kQuantRow + (n * 16 + e * 8 + g) * 4);
                    const float st = __uint_as_float(scale << 16), mid = fmaf(8.f, st, __uint_as_float(scale & 0xffff0000u));
                    mids[y][0] = fmaf(s[n][2 * e], mid, mids[y][0]);
                    mids[y][1] = fmaf(s[n][2 * e + 1], mid, mids[y][1]);
                    quant_split<P>(s[n][2 * e] * st, s[n][2 * e + 1] * st, pb[e]);
#pragma unroll
                    for (int k = 0; k < P; ++k)
                        asm volatile("movmatrix.sync.aligned.m8n8.trans.b16 %0, %0;" : "+r"(pb[e][k]));
                }
                // word g of positions 2 t4, 2 t4 + 1 and 8 further on, two positions to a register
                uint32_t lo[2], hi[2];
#pragma unroll
                for (int e = 0; e < 2; ++e) {
                    const char* at_row = vs + (n * 16 + e * 8 + t4) * kQuantRow + g * 4;
                    const uint32_t w0 = *reinterpret_cast<const uint32_t*>(at_row), w1 = *reinterpret_cast<const uint32_t*>(at_row + 4 * kQuantRow);
                    lo[e] = __byte_perm(w0, w1, 0x5410);
                    hi[e] = __byte_perm(w0, w1, 0x7632);
                }
#pragma unroll
                for (int d = 0; d < 4; ++d) {
                    const uint32_t a[4] = {quant_two(lo[0], d), quant_two(hi[0], d), quant_two(lo[1], d), quant_two(hi[1], d)};
#pragma unroll
                    for (int k = 0; k < P; ++k) mma_bf16(acc[y][d], a, pb[0][k], pb[1][k]);
                }
            }
        }
    }
    cp_wait<0>();
    __syncwarp();
#pragma unroll
    for (int j = 0; j < 2; ++j) {
#pragma unroll
        for (int o = 4; o < 32; o <<= 1) {
            l[j] += __shfl_xor_sync(0xffffffffu, l[j], o);
#pragma unroll
            for (int y = 0; y < LG; ++y) mids[y][j] += __shfl_xor_sync(0xffffffffu, mids[y][j], o);
        }
        const int row = 2 * t4 + j;
        if (g == 0) ml[row] = make_float2(m[j], l[j]);
        if (row < u.r.rows) {
            float* out = reinterpret_cast<float*>(smem) + row * kAtOutLd + g * 8;
#pragma unroll
            for (int y = 0; y < LG; ++y)
#pragma unroll
                for (int h = 0; h < 2; ++h)
                    *reinterpret_cast<float4*>(out + y * kAtRows * kAtOutLd + h * 4) =
                        make_float4(acc[y][0][2 * h + j] + mids[y][j], acc[y][1][2 * h + j] + mids[y][j],
                                    acc[y][2][2 * h + j] + mids[y][j], acc[y][3][2 * h + j] + mids[y][j]);
        }
    }
}

__device__ __forceinline__ bool quant_unit(const QuantParams& p, int index, bool reporter, QuantRun* u) {
    const AttendParams& a = p.a;
    if (index >= a.o_units) return false;
    const int lg = index % a.n_lg; index /= a.n_lg;
    const int split = index % a.o_splits; index /= a.o_splits;
    const int hk = index % a.Hk; index /= a.Hk;
    const int tile = index % a.o_row_tiles, item = index / a.o_row_tiles;
    if (!own_ok(a, item)) {
        if (reporter && tile == 0 && split == 0 && hk == 0 && lg == 0) {
            const int id = a.ids[item];
            const bool by_id = id < 0 || id >= a.max_ids;
            attend_error(a.status, TAG_QUANT, item, by_id ? id : a.lens[item], by_id ? a.max_ids : a.max_len);
        }
        return false;
    }
    AttendRun& r = u->r;
    u->item = r.item0 = item;
    r.head0 = hk * a.group; r.row0 = tile * kAtRows; r.rows = min(kAtRows, a.group - r.row0);
    r.layer0 = lg * a.lg; r.layers = min(a.lg, a.n_layers - r.layer0);
    r.n = a.lens[item]; r.n_sink = 0; r.lo = 0; r.permuted = false;
    r.row_bytes = r.v_row_bytes = kQuantRow;
    const long long panel = ((long long)a.ids[item] * a.Hk + hk) * a.cap;
    r.k = a.k + panel * kQuantRow;
    r.v = a.v + panel * kQuantRow + r.layer0 * a.v_stride;
    r.v_stride = a.v_stride;
    u->ks = p.ks + panel * 4;
    u->vs = p.vs + panel * 4 + r.layer0 * p.s_stride;
    u->s_stride = p.s_stride;
    r.slot = split;
    const int span = a.o_span * kQuantTile;
    r.begin = (int)min((long long)split * span, (long long)r.n);
    r.end = (int)min((long long)r.begin + span, (long long)r.n);
    return true;
}

template <int LG, int N, int P>
__global__ void __launch_bounds__(kAtWarps * 32) quant_attend_kernel(const __grid_constant__ QuantParams p) {
    static_assert(quant_warp_bytes<N>() >= LG * kAtRows * kAtOutLd * 4, "room for a warp's outputs");
    using T = typename std::conditional<P == 1, __nv_bfloat16, float>::type;
    extern __shared__ __align__(128) char attend_smem[];
    if (p.a.slots > 1 || p.S) asm volatile("griddepcontrol.launch_dependents;");
    constexpr int R = kAtRows, WB = quant_warp_bytes<N>();
    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31, wpu = p.a.o_wpu;
    float2* ml = reinterpret_cast<float2*>(attend_smem + kAtWarps * WB);
    QuantRun u;
    const bool active = quant_unit(p, (int)blockIdx.x * (kAtWarps / wpu) + warp / wpu, warp % wpu == 0 && lane == 0, &u);
    if (active)
        attend_warp_quant<LG, N, P>(p, u, u.r.begin + (warp % wpu) * kQuantTile, wpu * kQuantTile, attend_smem + warp * WB, ml + warp * R, lane);
    attend_finish<T, WB>(p.a, u.r, active, wpu, attend_smem, ml, warp, lane);
}

// Scores to weights, where the weights are wanted: grid = (rows, parts of 2048 positions).
constexpr int kQuantWeights = 2048;
static __global__ void __launch_bounds__(256) quant_weights_kernel(const __grid_constant__ QuantParams p) {
    const long long at = blockIdx.x, n_rows = (long long)p.a.n_items * p.a.H;
    const int item = (int)(at / p.a.H);
    asm volatile("griddepcontrol.wait;" ::: "memory");
    if (!own_ok(p.a, item)) return;
    const int begin = blockIdx.y * kQuantWeights, end = min(begin + kQuantWeights, p.a.lens[item]);
    if (begin >= end) return;
    float m = -INFINITY, l = 0.f;
    for (int s = 0; s < p.a.slots; ++s) {
        const float2 x = __ldcg(p.a.part_ml + s * n_rows + at);
        if (x.y == 0.f) continue;
        const float m_new = fmaxf(m, x.x);
        l = l * (m == m_new ? 1.f : exp2f(m - m_new)) + x.y * (x.x == m_new ? 1.f : exp2f(x.x - m_new));
        m = m_new;
    }
    const float inv = l == 0.f ? 0.f : 1.f / l, base = m == -INFINITY ? 0.f : m;
    float* S = p.S + at * p.ld_s;
    for (int j = begin + threadIdx.x; j < end; j += 256) S[j] = exp2f(S[j] - base) * inv;
}

}  // namespace san
