// A cache held in four bits a number: rows stored (san_quant_append), read back (san_quant_read), and one decode step of
// attention over them (san_quant_attn), whose weights serve every layer of a block (Eq. 3, Eq. 4).
//
// A row of 64 numbers x is 32 bytes of codes n (dim d in byte d / 2, the even one in the low half) and a pair of bf16 numbers:
//     low = min x, rounded down;   step = (max x - low) / 15, rounded up;   n = (x - low) / step, rounded half to even;
// it reads as low + step n.  Rounded that way low and step cover the row, so that no number is off by more than step / 2.
// A step is 0 or at least 2^-50; rows with a number of 2^40 or more are not held (they read as NaN, as rows with a NaN do).
// Which code a number gets is decided as if in 64 bits: float32 where the quotient is clear of a border, doubles next to one.
//
// Attention.  A row is read once and its 64 codes cost five instructions per eight, because they enter the products as they lie: as
// a bf16 number the bits 0-3 alone are n 2^-133 and the bits 4-7 alone 16 n 2^-133, exactly (subnormals and the binade above them have
// one distance), so that one shift and four ANDs make four operands of two numbers.  The other operand brings the magnitude back: queries
// are scaled to some 2^60 by a power of two of each row, weights are taken as 2^60 p.  A row's (step, low) is applied
// to its score and its weight, once for 64 numbers:
//     q . x = step (q . n) + low (sum of q),   sum_j p_j x_j = sum_j (p_j step_j) (n_j - 8) + sum_j p_j (low_j + 8 step_j),
// the -8 by a product with a constant, so that sums stay near zero, where an accumulator that cuts off does not drift.  Nothing is rounded for
// the cache's sake: bf16 rows round p step to bf16; float32 rows take queries and weights as three bf16 numbers that add up to
// them and keep float32's accuracy on the tensor cores.
#pragma once

#include <type_traits>

#include "san_attend.cuh"

namespace san {

constexpr int TAG_QUANT = 13, TAG_QUANT_ROWS = 14;
constexpr int kQuantRow = 32;               // bytes of codes of a row
constexpr int kQuantTile = 64;              // positions per slot: 2 KB of codes, then their (step, low)
constexpr int kQuantSlot = kQuantTile * (kQuantRow + 4);
constexpr float kQuantMost = 1.0995116e12f;             // 2^40
constexpr float kQuantLeastStep = 8.8817842e-16f;       // 2^-50

// ------------------------------------------------------------------------------------------- rows in and out
// Quotients by a number that the host knows, of numbers below 2^31 (a quotient of 64 bits takes some 80 instructions a thread, more
// than the row itself): with 2^shift >= d, times = ceil(2^(32 + shift) / d) - 2^32 makes (x + (x times) / 2^32) / 2^shift exact.
struct QuantDivide {
    uint32_t times, shift;
    __host__ void by(uint32_t d) {
        for (shift = 0; (1ull << shift) < d; ++shift) {}
        times = (uint32_t)((((1ull << shift) - d) << 32) / d + 1);
    }
    __device__ __forceinline__ uint32_t of(uint32_t x) const { return (__umulhi(x, times) + x) >> shift; }
};
constexpr int kQuantCtaRows = 64;           // of 256 threads, four lanes a row
struct QuantRowsParams {
    char* k; char* v; char* ks; char* vs;
    long long v_stride, s_stride;           // bytes between the layers' planes of codes, of (step, low)
    const char* k_rows; const char* v_rows; // [n_items][rows][Hk][64], [layers] of those
    const int* ids; const int* pos; const int* nrows;
    int n_items, rows, Hk, n_layers, max_ids, cap;
    uint32_t all_rows; long long layer_rows;                // of all layers; elements of a layer
    QuantDivide by_rows, by_heads, by_items;
    int* status;
};

__device__ __forceinline__ float bf16_down(float x) {       // of a finite x: the largest bf16 number not above it
    const int b = __float_as_int(x);
    return __int_as_float((b >= 0 ? b : b + 0xffff) & 0xffff0000);
}
__device__ __forceinline__ float quant_min3(float a, float b, float c) {        // NaN if one is
    float d;
    asm("min.NaN.f32 %0, %1, %2, %3;" : "=f"(d) : "f"(a), "f"(b), "f"(c));
    return d;
}
__device__ __forceinline__ float quant_max3(float a, float b, float c) {
    float d;
    asm("max.NaN.f32 %0, %1, %2, %3;" : "=f"(d) : "f"(a), "f"(b), "f"(c));
    return d;
}

// Two float32 numbers in one instruction.
__device__ __forceinline__ unsigned long long quant_pair(float x, float y) {
    unsigned long long r;
    asm("mov.b64 %0, {%1, %2};" : "=l"(r) : "f"(x), "f"(y));
    return r;
}
__device__ __forceinline__ void quant_unpair(unsigned long long r, float& x, float& y) { asm("mov.b64 {%0, %1}, %2;" : "=f"(x), "=f"(y) : "l"(r)); }
__device__ __forceinline__ unsigned long long quant_add2(unsigned long long a, unsigned long long b) {
    unsigned long long d;
    asm("add.rn.f32x2 %0, %1, %2;" : "=l"(d) : "l"(a), "l"(b));
    return d;
}
__device__ __forceinline__ unsigned long long quant_fma2(unsigned long long a, unsigned long long b, unsigned long long c) {
    unsigned long long d;
    asm("fma.rn.f32x2 %0, %1, %2, %3;" : "=l"(d) : "l"(a), "l"(b), "l"(c));
    return d;
}

// The place of a row (`row`: numbered layer, item, head, position, the last the fastest; layer 0: keys): false if it is
// none.  src: of the row's 64 numbers in elements, from the keys' or the layer's first.
struct QuantPlace { int layer; long long src, panel; int pos; };
__device__ __forceinline__ bool quant_place(const QuantRowsParams& p, uint32_t row, bool reporter, QuantPlace* at) {
    if (row >= p.all_rows) return false;
    uint32_t up = p.by_rows.of(row);
    const int r = (int)(row - up * p.rows);
    row = up; up = p.by_heads.of(row);
    const int h = (int)(row - up * p.Hk);
    at->layer = (int)p.by_items.of(up);
    const int item = (int)(up - at->layer * p.n_items);
    const int id = p.ids[item], pos = p.pos ? p.pos[item] : 0, n = p.nrows ? p.nrows[item] : p.rows;
    const bool by_id = id < 0 || id >= p.max_ids, by_n = n < 0 || n > p.rows;
    if (by_id || by_n || pos < 0 || pos > p.cap - n) {
        if (reporter && at->layer == 0 && r == 0 && h == 0)
            attend_error(p.status, TAG_QUANT_ROWS, item, by_id ? id : by_n ? n : pos, by_id ? p.max_ids : by_n ? p.rows : p.cap);
        return false;
    }
    at->src = ((long long)(item * p.rows + r) * p.Hk + h) * kDh + (at->layer > 0 ? (at->layer - 1) * p.layer_rows : 0);
    at->panel = (long long)id * p.Hk + h;
    at->pos = pos + r;
    return r < n;
}

// A row is four lanes of sixteen numbers; a CTA has 64 rows, those of one head on end where there are several. Bound by
// issue and latency: 5 x 4001 rows of 8 heads in 3 planes, float32, 32 us in (0.66 of the copy bandwidth) and 25 us back; with eight
// lanes a row, which find its place and step twice as often, 42 and 31.
template <typename T>
__global__ void __launch_bounds__(256, 5) quant_append_kernel(const __grid_constant__ QuantRowsParams p) {
    const int c = threadIdx.x & 3;                          // numbers 8 c .. 8 c + 7 of the row and of its second half
    QuantPlace at;
    const bool real = quant_place(p, blockIdx.x * kQuantCtaRows + (threadIdx.x >> 2), c == 0, &at);
    float x[16];
    if (real) {
        const T* src = reinterpret_cast<const T*>(at.layer == 0 ? p.k_rows : p.v_rows) + at.src + c * 8;
#pragma unroll
        for (int h = 0; h < 2; ++h) {
            if constexpr (sizeof(T) == 2) {
                unpack16<__nv_bfloat16>(ld16_stream(src + 32 * h), x + 8 * h);
            } else {
                unpack16<float>(ld16_stream(src + 32 * h), x + 8 * h);
                unpack16<float>(ld16_stream(src + 32 * h + 4), x + 8 * h + 4);
            }
        }
    } else {
#pragma unroll
        for (int i = 0; i < 16; ++i) x[i] = 0.f;
    }
    float lo = x[0], hi = x[0];
#pragma unroll
    for (int i = 1; i < 15; i += 2) {
        lo = quant_min3(lo, x[i], x[i + 1]);
        hi = quant_max3(hi, x[i], x[i + 1]);
    }
    lo = quant_min3(lo, lo, x[15]);
    hi = quant_max3(hi, hi, x[15]);
#pragma unroll
    for (int o = 1; o < 4; o <<= 1) {
        lo = quant_min3(lo, lo, __shfl_xor_sync(0xffffffffu, lo, o));
        hi = quant_max3(hi, hi, __shfl_xor_sync(0xffffffffu, hi, o));
    }
    const bool held = -lo < kQuantMost && hi < kQuantMost;  // (false for NaN)
    // step: the least bf16 number b with 15 b >= hi - low.  The product is exact, and the difference may be rounded up, since 15 b is a
    // float32 number.  A product with a little less than 1 / 15, cut off, is that, the one below or two below.
    const float low = bf16_down(lo), wide = __fsub_ru(hi, low);
    float step = __int_as_float(__float_as_int(wide * 0.0666666627f) & 0xffff0000);
#pragma unroll
    for (int i = 0; i < 2; ++i)
        if (15.f * step < wide) step = __int_as_float(__float_as_int(step) + 0x10000);
    step = wide > 0.f ? fmaxf(step, kQuantLeastStep) : 0.f;
    const float inv = step > 0.f ? __fdividef(1.f, step) : 0.f;         // a step of zero: codes of zero
    constexpr float kWhole = 12582912.f;                    // 1.5 2^23
    const unsigned long long low2 = quant_pair(-low, -low), inv2 = quant_pair(inv, inv), zero2 = quant_pair(0.f, 0.f), most2 = quant_pair(kWhole, kWhole);
    uint32_t codes[2] = {0u, 0u};
    float off = 0.f;                                        // the furthest from a whole number
#pragma unroll
    for (int i = 14; i >= 0; i -= 2) {                      // two numbers in one instruction
        const unsigned long long t = quant_fma2(quant_add2(quant_pair(x[i], x[i + 1]), low2), inv2, zero2);
        const unsigned long long y = quant_add2(t, most2);               // the sums' low bits are t rounded half to even
        float a, b;
        quant_unpair(quant_fma2(quant_add2(y, quant_pair(-kWhole, -kWhole)), quant_pair(-1.f, -1.f), t), a, b);
        off = quant_max3(off, fabsf(a), fabsf(b));
        quant_unpair(y, a, b);
        codes[i >> 3] = (codes[i >> 3] * 16 + __float_as_uint(b)) * 16 + __float_as_uint(a);
    }
#pragma unroll
    for (int h = 0; h < 2; ++h) codes[h] -= 0x4b400000u * 0x11111111u;  // the bits of kWhole, eight times
    if (off > 0.4999f && held) {                            // t is within 1e-5 of the quotient; next to a border 64 bits decide
        codes[0] = codes[1] = 0u;
#pragma unroll
        for (int i = 15; i >= 0; --i) {
            const double d = (double)x[i] - (double)low;
            const float k = fminf(floorf((x[i] - low) * inv), 15.f);
            // k may be one too large or too small itself where the quotient is a whole number
            const double border = ((double)k + 0.5) * (double)step;
            const uint32_t n = (uint32_t)k + (d > border || (d == border && ((int)k & 1)));
            codes[i >> 3] = codes[i >> 3] << 4 | min(n, 15u);
        }
    }
    if (!real) return;
    const long long row = at.panel * p.cap + at.pos;
    char* to = (at.layer == 0 ? p.k : p.v + (at.layer - 1) * p.v_stride) + row * kQuantRow;
    reinterpret_cast<uint32_t*>(to)[c] = held ? codes[0] : 0u;
    reinterpret_cast<uint32_t*>(to)[c + 4] = held ? codes[1] : 0u;
    if (c == 0) {
        char* scale = (at.layer == 0 ? p.ks : p.vs + (at.layer - 1) * p.s_stride) + row * 4;
        *reinterpret_cast<uint32_t*>(scale) = held ? __float_as_uint(step) >> 16 | (__float_as_uint(low) & 0xffff0000u) : 0x7fc07fc0u;
    }
}

template <typename T>
__global__ void __launch_bounds__(256) quant_read_kernel(const __grid_constant__ QuantRowsParams p) {
    const int c = threadIdx.x & 3;
    QuantPlace at;
    if (!quant_place(p, blockIdx.x * kQuantCtaRows + (threadIdx.x >> 2), c == 0, &at)) return;
    const long long row = at.panel * p.cap + at.pos;
    const char* codes = (at.layer == 0 ? p.k : p.v + (at.layer - 1) * p.v_stride) + row * kQuantRow;
    const uint32_t scale = *reinterpret_cast<const uint32_t*>((at.layer == 0 ? p.ks : p.vs + (at.layer - 1) * p.s_stride) + row * 4);
    const float step = __uint_as_float(scale << 16), low = __uint_as_float(scale & 0xffff0000u);
    T* to = reinterpret_cast<T*>(const_cast<char*>(at.layer == 0 ? p.k_rows : p.v_rows)) + at.src;
    // 16 bytes at a time, four lanes side by side.
    constexpr int N = 16 / sizeof(T);                       // numbers
    uint32_t words[16 / N];
    if constexpr (N == 8) {
        for (int i = 0; i < 2; ++i) words[i] = reinterpret_cast<const uint32_t*>(codes)[c + 4 * i];
    } else {                                                // the lane's 16 bits of each of four pairs of words
#pragma unroll
        for (int i = 0; i < 2; ++i) {
            const uint4 half = reinterpret_cast<const uint4*>(codes)[i];
            words[2 * i] = (c < 2 ? half.x : half.y) >> 16 * (c & 1);
            words[2 * i + 1] = (c < 2 ? half.z : half.w) >> 16 * (c & 1);
        }
    }
#pragma unroll
    for (int w = 0; w < 16 / N; ++w) {
        float x[N];
#pragma unroll
        for (int i = 0; i < N; ++i) x[i] = fmaf(step, (float)(words[w] >> (4 * i) & 15u), low);
        *reinterpret_cast<uint4*>(to + (4 * w + c) * N) = pack16<T>(x);
    }
}

// ------------------------------------------------------------------------------------------- attention
struct QuantParams {
    AttendParams a;                         // k, v: planes of codes
    const char* ks; const char* vs; long long s_stride;
    float* S; long long ld_s;               // scores, in powers of two, until quant_finish_kernel makes them weights (by (max, sum) in the workspace)
    int join_ctas, parts;                   // of quant_finish_kernel: CTAs that join partial results, parts of a row of S
};
struct QuantRun {
    AttendRun r;
    const char* ks; const char* vs; long long s_stride;
    int item;
};

// A CTA takes one unit: a key head of an item, up to eight query rows, LG layers, a run of positions, in steps of one tile per warp.
// W: warps.  Where LG divides it, warp w applies layer w % LG to the LG tiles from w / LG * LG on; 3 layers are W = 3.
template <int LG> struct QuantWarps { static constexpr int W = LG == 3 ? 3 : 4; };
constexpr int kQuantSlots = 4;              // of a warp's ring, later the place of its outputs
constexpr int kQuantRing = kQuantSlots * kQuantSlot;
template <int LG, int J> __host__ __device__ constexpr int quant_weight_bytes() { return LG == 1 ? 0 : 8 * J * 128; }       // of a tile
template <int LG, int J> __host__ __device__ constexpr int quant_smem_bytes() { return QuantWarps<LG>::W * (kQuantRing + quant_weight_bytes<LG, J>() + 2 * kAtRows * 4); }
static_assert(kQuantRing >= kAtRows * kAtOutLd * 4, "room for a warp's outputs");

__device__ __forceinline__ void cp16_whole(uint32_t dst, const void* src) { asm volatile("cp.async.cg.shared.global [%0], [%1], 16;" :: "r"(dst), "l"(src) : "memory"); }
__device__ __forceinline__ void cp4_whole(uint32_t dst, const void* src) { asm volatile("cp.async.ca.shared.global [%0], [%1], 4;" :: "r"(dst), "l"(src) : "memory"); }
__device__ __forceinline__ void cp4(uint32_t dst, const void* src, bool full) {
    const int n = full ? 4 : 0;
    asm volatile("cp.async.ca.shared.global [%0], [%1], 4, %2;" :: "r"(dst), "l"(src), "r"(n) : "memory");
}

// Walks a warp's slots: of every step the tile of keys that it scores (item 0), then the tiles of values of its layer that it applies (items 1 ..
// LG), filled three ahead of use, into the place of the one used before.  Which comes when is known to the compiler, so that a fill is
// its copies and little else.  What lies at or behind `end` becomes zeros; tiles that begin there are not copied.  The halves of rows
// 4 .. 7 of eight change places, so that a half of eight rows is in different banks.
template <int W, int LG> struct QuantRing {
    static constexpr int kAhead = kQuantSlots - 1, kItems = LG + 1, kStep = W * kQuantTile;
    uint32_t ring, slot;                                    // slot: of the next item
    int lane, end, k_at, v_at;                              // positions of the warp's tiles of keys and of values in the step that is worked on
    bool values;                                            // its layer is there
    const char* k; const char* v; const char* ks; const char* vs;           // this lane's first bytes of them
    uint32_t v_to;                                          // where its first value row goes
    __device__ __forceinline__ QuantRing(const QuantRun& u, uint32_t smem, int ln, int warp) : ring(smem), slot(0), lane(ln), end(u.r.end) {
        const int y = warp % LG;
        values = y < u.r.layers;
        k_at = u.r.begin + warp * kQuantTile; v_at = u.r.begin + warp / LG * LG * kQuantTile;
        k = u.r.k + (long long)k_at * kQuantRow + lane * 16; ks = u.ks + (long long)k_at * 4 + lane * 4;
        v = u.r.v + (values ? y : 0) * u.r.v_stride + (long long)v_at * kQuantRow + lane * 16;
        vs = u.vs + (values ? y : 0) * u.s_stride + (long long)v_at * 4 + lane * 4;
        const int r = lane >> 1;
        v_to = r * kQuantRow + ((lane ^ r >> 2) & 1) * 16;
        fill<0>(0); fill<1>(kQuantSlot); fill<2>(2 * kQuantSlot);
    }
    // Item ITEM of this step (ITEM >= kItems: of a later one).
    template <int ITEM> __device__ __forceinline__ void fill(uint32_t to_slot) {
        constexpr int later = ITEM / kItems * kStep, item = ITEM % kItems, off = later + (item > 0 ? (item - 1) * kQuantTile : 0);
        const int at = (item == 0 ? k_at : v_at) + off;
        if (at < end && (item == 0 || values)) {
            const char* codes = (item == 0 ? k : v) + off * kQuantRow;
            const char* scales = (item == 0 ? ks : vs) + off * 4;
            const uint32_t to = ring + to_slot + (item == 0 ? lane * 16 : v_to), to_scale = ring + to_slot + kQuantTile * kQuantRow + lane * 4;
            if (at + kQuantTile <= end) {
#pragma unroll
                for (int j = 0; j < kQuantTile / 16; ++j) cp16_whole(to + j * 16 * kQuantRow, codes + j * 16 * kQuantRow);
#pragma unroll
                for (int j = 0; j < kQuantTile / 32; ++j) cp4_whole(to_scale + j * 128, scales + j * 128);
            } else {
#pragma unroll
                for (int j = 0; j < kQuantTile / 16; ++j) {
                    const bool full = at + j * 16 + (lane >> 1) < end;
                    cp16(to + j * 16 * kQuantRow, full ? codes + j * 16 * kQuantRow : v, full);
                }
#pragma unroll
                for (int j = 0; j < kQuantTile / 32; ++j) {
                    const bool full = at + j * 32 + lane < end;
                    cp4(to_scale + j * 128, full ? scales + j * 128 : vs, full);
                }
            }
        }
        cp_commit();                                        // where nothing was copied an empty group keeps the count
    }
    // Offset of item ITEM's slot, arrived; every lane is done with the one before it, which is refilled.
    template <int ITEM> __device__ __forceinline__ uint32_t next() {
        cp_wait<kAhead - 1>();
        __syncwarp();
        const uint32_t s = slot;
        fill<ITEM + kAhead>(s == 0 ? kAhead * kQuantSlot : s - kQuantSlot);
        slot = s == kAhead * kQuantSlot ? 0 : s + kQuantSlot;
        return s;
    }
    __device__ __forceinline__ void step() {
        k_at += kStep; v_at += kStep;
        k += kStep * kQuantRow; v += kStep * kQuantRow; ks += kStep * 4; vs += kStep * 4;
    }
};

// Four operands of two codes each from a word: bits 0-3, 4-7 (16 times as large), 8-11, 12-15 (16 times) of both halves.
__device__ __forceinline__ void quant_four(uint32_t w, uint32_t* out) {
    const uint32_t v = w >> 8;
    out[0] = w & 0x000f000fu; out[1] = w & 0x00f000f0u;
    out[2] = v & 0x000f000fu; out[3] = v & 0x00f000f0u;
}
// The same of value rows.  float32 rows (P = 3) take the codes less 8, as ordinary numbers (0x4300 | n is 128 + n): their sums stay small
// throughout, while sums of codes have the size of 8 times the weights until -8 has been added, and an accumulator that cuts off is off by
// 2^-24 of that at every step (6.8e-6 of the outputs in all; bf16 outputs are rounded by some hundred times that).
template <int P> __device__ __forceinline__ void quant_codes(uint32_t w, uint32_t* out) {
    if constexpr (P == 1) {
        quant_four(w, out);
    } else {
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            const uint32_t x = (w >> (4 * i) & 0x000f000fu) | 0x43004300u;
            asm("sub.rn.bf16x2 %0, %1, %2;" : "=r"(out[i]) : "r"(x), "r"(0x43084308u));
        }
    }
}
__device__ __forceinline__ void quant_mma(float* d, const uint32_t* a, uint32_t b0, uint32_t b1, const float* c) {
    asm("mma.sync.aligned.m16n8k16.row.col.f32.bf16.bf16.f32 {%0,%1,%2,%3}, {%4,%5,%6,%7}, {%8,%9}, {%10,%11,%12,%13};"
                 : "=f"(d[0]), "=f"(d[1]), "=f"(d[2]), "=f"(d[3])
                 : "r"(a[0]), "r"(a[1]), "r"(a[2]), "r"(a[3]), "r"(b0), "r"(b1), "f"(c[0]), "f"(c[1]), "f"(c[2]), "f"(c[3]));
}
// x as P bf16 numbers that add up to it (P = 1: its rounding).
template <int P> __device__ __forceinline__ void quant_split(float x, float y, uint32_t* out) {
#pragma unroll
    for (int k = 0; k < P; ++k) {
        out[k] = pack_bf16(x, y);
        if (k + 1 == P) break;
        x -= __uint_as_float(out[k] << 16);
        y -= __uint_as_float(out[k] & 0xffff0000u);
    }
}

// Query rows, which are the N side of both products: scores D[16 positions x 8 queries] with the codes of key rows as
// A, outputs D[16 dims x 8 queries] with those of value rows.  P: 1 for bf16 queries, 3 for float32.  J: a lane holds two neighbouring
// columns of D.  With J = 1 only the even one is a query (up to four rows), which halves what is done to scores and weights; with
// J = 2 both are (up to eight).
// Every warp of the CTA calls this.  Per step: scores of the warp's own tile, the largest of all tiles (a barrier), weights, which the
// warps share (a barrier), then the warp's layer.  So a warp holds one layer's outputs, 16 registers, and an SM holds 16 warps
// or more: with four layers a warp (64 registers, 12 warps) instructions waited for one another half of the time.
template <int LG, int P, int J>
__device__ __forceinline__ void attend_quant(const QuantParams& p, const QuantRun& u, char* smem, char* shared, float* tops, float2* ml, int warp, int lane) {
    constexpr int W = QuantWarps<LG>::W;
    const uint32_t ring_addr = (uint32_t)__cvta_generic_to_shared(smem);
    QuantRing<W, LG> ring(u, ring_addr, lane, warp);
    const int g = lane >> 2, t4 = lane & 3;
    // B: the query of column g, dims 16 t4 .. 16 t4 + 15 in the order of the codes' unpacking, scaled to at most 2^60 and odd ones of a byte by
    // another 1 / 16
    uint32_t qb[8][P];
    float qs[J], unit[J];                                    // of columns 2 t4 (+ 1): the query's sum times the scores' scale; what undoes the scaling, times it
    {
        const int row = J == 1 ? g >> 1 : g;
        const bool real = row < u.r.rows && (J == 2 || (g & 1) == 0);
        const int head = u.r.head0 + u.r.row0 + (real ? row : 0);
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
        float sum = 0.f, most = 0.f;
#pragma unroll
        for (int i = 0; i < 16; ++i) {
            sum = fabsf(q[i]) < kQuantMost ? sum + q[i] : NAN;           // a row with such a number gives NaN
            most = fmaxf(most, fabsf(q[i]));
        }
#pragma unroll
        for (int o = 1; o < 4; o <<= 1) {
            sum += __shfl_xor_sync(0xffffffffu, sum, o);
            most = fmaxf(most, __shfl_xor_sync(0xffffffffu, most, o));
        }
        // most = 2^e (1 + ..), e within -60 .. 40: times 2^(59 - e)
        const int e = max((int)(__float_as_uint(fminf(most, kQuantMost)) >> 23) - 127, -60);
        const float up = __uint_as_float((uint32_t)(59 - e + 127) << 23);
        const float down = __uint_as_float((uint32_t)(e + 74 + 127) << 23);      // 2^133 / up
#pragma unroll
        for (int j = 0; j < J; ++j) {
            qs[j] = __shfl_sync(0xffffffffu, sum, 4 * (2 * t4 + j)) * p.a.scale_log2e;
            unit[j] = __shfl_sync(0xffffffffu, down, 4 * (2 * t4 + j)) * p.a.scale_log2e;
        }
#pragma unroll
        for (int h = 0; h < 2; ++h)
#pragma unroll
            for (int i = 0; i < 4; ++i) {
                const float f = i & 1 ? up * 0.0625f : up;
                quant_split<P>(q[8 * h + i] * f, q[8 * h + 4 + i] * f, qb[4 * h + i]);
            }
    }
    // [d]: dims 4 g + d and 32 + 4 g + d of columns 2 t4, 2 t4 + 1: bf16 in units of 2^-73 (odd d: 16 times), float32 of 2^60; this lane's part of
    // the sums of p mid in units of 2^60
    float acc[4][4], mids[J], m[J], l[J];
#pragma unroll
    for (int j = 0; j < J; ++j) { mids[j] = 0.f; m[j] = -INFINITY; l[j] = 0.f; }
#pragma unroll
    for (int d = 0; d < 4; ++d)
#pragma unroll
        for (int e = 0; e < 4; ++e) acc[d][e] = 0.f;
    // the row's half that this lane names of 16 positions: eight lanes each for those of 0 .. 7, then of 8 .. 15
    const uint32_t row_at = ((lane >> 4) * 8 + (lane & 7)) * kQuantRow + ((lane >> 3 ^ lane >> 2) & 1) * 16;
    constexpr int kBlocks = kQuantTile / 16, kRegs = 2 * kBlocks * J;       // weights of a lane and tile
    const float none[4] = {0.f, 0.f, 0.f, 0.f};
    for (int at0 = u.r.begin; at0 < u.r.end; at0 += W * kQuantTile) {
        const int at = at0 + warp * kQuantTile;
        float s[kBlocks][2][J];                              // positions 16 n + g and + 8, columns 2 t4 (+ 1)
        const char* ks = smem + ring.template next<0>();
        if (at < u.r.end) {                                  // (the same in all lanes)
#pragma unroll
            for (int n = 0; n < kBlocks; ++n) {
                const uint2 w0 = *reinterpret_cast<const uint2*>(ks + (n * 16 + g) * kQuantRow + t4 * 8);
                const uint2 w1 = *reinterpret_cast<const uint2*>(ks + (n * 16 + 8 + g) * kQuantRow + t4 * 8);
                float dot[4];
                uint32_t x0[8], x1[8];
                quant_four(w0.x, x0); quant_four(w0.y, x0 + 4);
                quant_four(w1.x, x1); quant_four(w1.y, x1 + 4);
                // the smallest parts of the queries first: an accumulator cuts off what lies below its own last bit
#pragma unroll
                for (int k = P - 1; k >= 0; --k)
#pragma unroll
                    for (int c = 0; c < 8; c += 2) {
                        const uint32_t a[4] = {x0[c], x1[c], x0[c + 1], x1[c + 1]};
                        quant_mma(dot, a, qb[c][k], qb[c + 1][k], k == P - 1 && c == 0 ? none : dot);
                    }
#pragma unroll
                for (int e = 0; e < 2; ++e) {
                    const uint32_t scale = *reinterpret_cast<const uint32_t*>(ks + kQuantTile * kQuantRow + (n * 16 + e * 8 + g) * 4);
                    const float st = __uint_as_float(scale << 16), low = __uint_as_float(scale & 0xffff0000u);
#pragma unroll
                    for (int j = 0; j < J; ++j) s[n][e][j] = fmaf(st, dot[2 * e + j] * unit[j], low * qs[j]);
                }
            }
            if (at + kQuantTile > u.r.end) {
#pragma unroll
                for (int n = 0; n < kBlocks; ++n)
#pragma unroll
                    for (int e = 0; e < 2; ++e)
#pragma unroll
                        for (int j = 0; j < J; ++j)
                            if (at + n * 16 + e * 8 + g >= u.r.end) s[n][e][j] = -INFINITY;
            }
            if (p.S && u.r.layer0 == 0) {
#pragma unroll
                for (int j = 0; j < J; ++j) {
                    const int row = J * t4 + j;
                    if (row >= u.r.rows) continue;
                    float* to = p.S + ((long long)u.item * p.a.H + u.r.head0 + u.r.row0 + row) * p.ld_s + at + g;
#pragma unroll
                    for (int n = 0; n < kBlocks; ++n)
#pragma unroll
                        for (int e = 0; e < 2; ++e)
                            if (at + n * 16 + e * 8 + g < u.r.end) to[n * 16 + e * 8] = s[n][e][j];
                }
            }
        } else {
#pragma unroll
            for (int n = 0; n < kBlocks; ++n)
#pragma unroll
                for (int e = 0; e < 2; ++e)
#pragma unroll
                    for (int j = 0; j < J; ++j) s[n][e][j] = -INFINITY;
        }
        float top[J];
#pragma unroll
        for (int j = 0; j < J; ++j) {
            top[j] = fmaxf(s[0][0][j], s[0][1][j]);
#pragma unroll
            for (int n = 1; n < kBlocks; ++n) top[j] = fmaxf(top[j], fmaxf(s[n][0][j], s[n][1][j]));
#pragma unroll
            for (int o = 4; o < 32; o <<= 1) top[j] = fmaxf(top[j], __shfl_xor_sync(0xffffffffu, top[j], o));
            if (g == 0) tops[warp * kAtRows + J * t4 + j] = top[j];
        }
        __syncthreads();                                     // (and every warp is done with the weights of the step before)
        float alpha[J];
        bool moved = false;
#pragma unroll
        for (int j = 0; j < J; ++j) {
            float t = m[j];
#pragma unroll
            for (int w = 0; w < W; ++w) t = fmaxf(t, tops[w * kAtRows + J * t4 + j]);
            // times 2^60 by way of the argument (float32: after it, which costs the argument no bits); all scores -inf so far: weights 0
            const float base = (t == -INFINITY ? 0.f : t) - (P == 1 ? 60.f : 0.f);
            alpha[j] = m[j] == t ? 1.f : P == 1 ? fast_exp2(m[j] - t) : exp2f(m[j] - t);
            moved |= m[j] != t;
            m[j] = t;
            float sum = 0.f;
#pragma unroll
            for (int n = 0; n < kBlocks; ++n)
#pragma unroll
                for (int e = 0; e < 2; ++e) {
                    s[n][e][j] = P == 1 ? fast_exp2(s[n][e][j] - base) : exp2f(s[n][e][j] - base) * 1.152921504606846976e18f;
                    sum += s[n][e][j];
                }
            l[j] = l[j] * alpha[j] + sum;
        }
        float pw[kRegs];                                     // the tile's weights
#pragma unroll
        for (int n = 0; n < kBlocks; ++n)
#pragma unroll
            for (int e = 0; e < 2; ++e)
#pragma unroll
                for (int j = 0; j < J; ++j) pw[(2 * n + e) * J + j] = s[n][e][j];
        if constexpr (LG > 1) {
#pragma unroll
            for (int i = 0; i < kRegs / 4; ++i)
                *reinterpret_cast<float4*>(shared + ((warp * (kRegs / 4) + i) * 32 + lane) * 16) = make_float4(pw[4 * i], pw[4 * i + 1], pw[4 * i + 2], pw[4 * i + 3]);
        }
        if (__any_sync(0xffffffffu, moved)) {                // seldom, once a run is under way
#pragma unroll
            for (int j = 0; j < J; ++j) {
                mids[j] *= alpha[j];
#pragma unroll
                for (int d = 0; d < 4; ++d) { acc[d][j] *= alpha[j]; acc[d][2 + j] *= alpha[j]; }
            }
        }
        __syncthreads();                                     // (and the tops have been read)
        auto apply = [&](const char* vs, int tile) {
            if (!ring.values || at0 + tile * kQuantTile >= u.r.end) return;
            const char* scales = vs + kQuantTile * kQuantRow;
            const uint32_t rows = ring_addr + (uint32_t)(vs - smem) + row_at;
            if constexpr (LG > 1) {
#pragma unroll
                for (int i = 0; i < kRegs / 4; ++i) {
                    const float4 x = *reinterpret_cast<const float4*>(shared + ((tile * (kRegs / 4) + i) * 32 + lane) * 16);
                    pw[4 * i] = x.x; pw[4 * i + 1] = x.y; pw[4 * i + 2] = x.z; pw[4 * i + 3] = x.w;
                }
            }
            // Weights times steps, as B, which has to hold neighbouring positions (an 8 x 8 transpose): bf16 rows round them, by half a step
            // (2^-8 relative) at most, of independent sign; what they are taken with is within 8 steps of 0, not the number itself.
            uint32_t w[kBlocks][2][P];
#pragma unroll
            for (int n = 0; n < kBlocks; ++n)
#pragma unroll
                for (int e = 0; e < 2; ++e) {
                    const uint32_t scale = *reinterpret_cast<const uint32_t*>(scales + (n * 16 + e * 8 + g) * 4);
                    const float st = __uint_as_float(scale << 16), md = fmaf(8.f, st, __uint_as_float(scale & 0xffff0000u));
                    float x[2] = {0.f, 0.f};
#pragma unroll
                    for (int j = 0; j < J; ++j) {
                        x[j] = pw[(2 * n + e) * J + j];
                        mids[j] = fmaf(x[j], md, mids[j]);
                        x[j] *= st;
                    }
                    quant_split<P>(x[0], x[1], w[n][e]);
#pragma unroll
                    for (int k = 0; k < P; ++k) asm("movmatrix.sync.aligned.m8n8.trans.b16 %0, %0;" : "+r"(w[n][e][k]));
                }
            // -8 times the sum of the weights, in the units of the bits 0-3 (of the bits 4-7: 16 times)
            float start[4];
            if constexpr (P == 1) {
                const uint32_t eight[4] = {0x80088008u, 0x80088008u, 0x80088008u, 0x80088008u};
#pragma unroll
                for (int n = 0; n < kBlocks; ++n) quant_mma(start, eight, w[n][0][0], w[n][1][0], n == 0 ? none : start);
            }
            // float32 rows add a tile's sums to those of the run in float32, rounded: an accumulator would cut off at every product of a long run
            float part[4][4];
#pragma unroll
            for (int n = 0; n < kBlocks; ++n) {
                // four codes each of positions 2 t4 and 2 t4 + 1 (and 8 further on) in a register: dims 4 g .. and 32 + 4 g ..
                uint32_t lo[2][4], hi[2][4], x[4];
                asm volatile("ldmatrix.sync.aligned.m8n8.x4.trans.shared.b16 {%0,%1,%2,%3}, [%4];" : "=r"(x[0]), "=r"(x[1]), "=r"(x[2]), "=r"(x[3])
                             : "r"(rows + n * 16 * kQuantRow) : "memory");
#pragma unroll
                for (int e = 0; e < 2; ++e) {
                    quant_codes<P>(x[2 * e], lo[e]);
                    quant_codes<P>(x[2 * e + 1], hi[e]);
                }
#pragma unroll
                for (int c = 0; c < 4; ++c) {
                    const uint32_t a[4] = {lo[0][c], hi[0][c], lo[1][c], hi[1][c]};
                    if constexpr (P == 1) {
                        quant_mma(acc[c], a, w[n][0][0], w[n][1][0], acc[c]);
                    } else {
#pragma unroll
                        for (int k = P - 1; k >= 0; --k) quant_mma(part[c], a, w[n][0][k], w[n][1][k], n == 0 && k == P - 1 ? none : part[c]);
                    }
                }
            }
#pragma unroll
            for (int c = 0; c < 4; ++c)
#pragma unroll
                for (int e = 0; e < 2; ++e)
#pragma unroll
                    for (int j = 0; j < J; ++j) acc[c][2 * e + j] = P > 1 ? acc[c][2 * e + j] + part[c][2 * e + j] : fmaf(start[j], c & 1 ? 16.f : 1.f, acc[c][2 * e + j]);
        };
        const int tile0 = warp / LG * LG;
        apply(smem + ring.template next<1>(), tile0);
        if constexpr (LG > 1) apply(smem + ring.template next<2>(), tile0 + 1);
        if constexpr (LG > 2) apply(smem + ring.template next<3>(), tile0 + 2);
        if constexpr (LG > 3) apply(smem + ring.template next<4>(), tile0 + 3);
        ring.step();
    }
    cp_wait<0>();
    __syncwarp();
    constexpr float kDown = 8.67361737988403547e-19f, kUp = 9.44473296573929043e21f;      // 2^-60; 2^73
#pragma unroll
    for (int j = 0; j < J; ++j) {
#pragma unroll
        for (int o = 4; o < 32; o <<= 1) {
            l[j] += __shfl_xor_sync(0xffffffffu, l[j], o);
            mids[j] += __shfl_xor_sync(0xffffffffu, mids[j], o);
        }
        const int row = J * t4 + j;
        if (g == 0) ml[row] = make_float2(m[j], l[j] * kDown);
        float* out = reinterpret_cast<float*>(smem) + row * kAtOutLd + g * 4;
#pragma unroll
        for (int h = 0; h < 2; ++h) {
            float x[4];
#pragma unroll
            for (int c = 0; c < 4; ++c) x[c] = fmaf(acc[c][2 * h + j], P > 1 ? kDown : c & 1 ? kUp * 0.0625f : kUp, mids[j] * kDown);
            *reinterpret_cast<float4*>(out + h * 32) = make_float4(x[0], x[1], x[2], x[3]);
        }
    }
}

__device__ __forceinline__ bool quant_unit(const QuantParams& p, int index, bool reporter, QuantRun* u) {
    const AttendParams& a = p.a;
    if (index >= a.o_units) return false;
    // the first runs of all items first: those that only long items have come last, where short CTAs even out the end
    const int lg = index % a.n_lg; index /= a.n_lg;
    const int hk = index % a.Hk; index /= a.Hk;
    const int tile = index % a.o_row_tiles; index /= a.o_row_tiles;
    const int item = index % a.n_items, split = index / a.n_items;
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

// P, J: see attend_quant.  Registers leave room for 20 warps on an SM (bf16; 128 rows of up to 4096, 4 layers: 81.7 us; before transposed loads 90, with 16 warps some 4 more; six of the eight bf16 forms
// spill a word or two for it).
template <int LG, int P, int J>
__global__ void __launch_bounds__(QuantWarps<LG>::W * 32, P == 1 ? LG == 3 ? 6 : 5 : 3) quant_attend_kernel(const __grid_constant__ QuantParams p) {
    constexpr int W = QuantWarps<LG>::W, R = kAtRows;
    using T = typename std::conditional<P == 1, __nv_bfloat16, float>::type;
    extern __shared__ __align__(128) char attend_smem[];
    __shared__ float tops[W * R];
    if (p.a.slots > 1 || p.S) asm volatile("griddepcontrol.launch_dependents;");
    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
    char* shared = attend_smem + W * kQuantRing;
    float2* ml = reinterpret_cast<float2*>(shared + W * quant_weight_bytes<LG, J>());
    QuantRun u;
    if (!quant_unit(p, (int)blockIdx.x, threadIdx.x == 0, &u)) return;
    attend_quant<LG, P, J>(p, u, attend_smem + warp * kQuantRing, shared, tops, ml + warp * R, warp, lane);
    __syncthreads();
    // The warps' results: one maximum, sums of the tiles that each scored, outputs of the layer that each applied.  16 threads a row.
    const long long n_rows = (long long)p.a.n_items * p.a.H;
    const bool direct = p.a.slots == 1;
    for (int i = threadIdx.x >> 4; i < u.r.rows * LG; i += W * 2) {
        const int row = i / LG, y = i % LG, c = threadIdx.x & 15;
        if (y >= u.r.layers) continue;
        float l = 0.f;
#pragma unroll
        for (int w = 0; w < W; ++w) l += ml[w * R + row].y;
        const long long at = (long long)u.item * p.a.H + u.r.head0 + u.r.row0 + row;
        if ((!direct || p.S) && c == 0 && y == 0 && u.r.layer0 == 0) p.a.part_ml[u.r.slot * n_rows + at] = make_float2(ml[row].x, l);
        if (!direct && l == 0.f) continue;                   // the join does not look at it
        float4 o = make_float4(0.f, 0.f, 0.f, 0.f);
#pragma unroll
        for (int w = 0; w < W / LG; ++w) {
            const float4 x = *reinterpret_cast<const float4*>(attend_smem + (w * LG + y) * kQuantRing + (row * kAtOutLd + c * 4) * 4);
            o.x += x.x; o.y += x.y; o.z += x.z; o.w += x.w;
        }
        if (direct) {
            const float inv = l == 0.f ? 0.f : 1.f / l;
            T* dst = reinterpret_cast<T*>(p.a.out) + ((u.r.layer0 + y) * n_rows + at) * kDh + c * 4;
            if constexpr (P > 1) *reinterpret_cast<float4*>(dst) = make_float4(o.x * inv, o.y * inv, o.z * inv, o.w * inv);
            else *reinterpret_cast<uint2*>(dst) = make_uint2(pack_bf16(o.x * inv, o.y * inv), pack_bf16(o.z * inv, o.w * inv));
        } else {
            *reinterpret_cast<float4*>(p.a.part_o + (((long long)u.r.slot * p.a.n_layers + u.r.layer0 + y) * n_rows + at) * kDh + c * 4) = o;
        }
    }
}

// Behind the runs of all units: partial results of a row and layer added up (16 threads for its outputs, four each, times G groups
// that take every G-th result), and scores made weights where they are wanted (a CTA for 2048 positions of a row), side by side.
constexpr int kQuantWeights = 2048;
template <typename T, int G>
__global__ void __launch_bounds__(256) quant_finish_kernel(const __grid_constant__ QuantParams p) {
    __shared__ float4 s_o[G > 1 ? 256 : 1];
    __shared__ float2 s_ml[G > 1 ? 256 : 1];
    const AttendParams& a = p.a;
    const long long n_rows = (long long)a.n_items * a.H;
    if (blockIdx.x >= (unsigned)p.join_ctas) {
        const unsigned index = blockIdx.x - p.join_ctas;
        const long long at = index / p.parts;
        const int item = (int)(at / a.H), begin = (int)(index % p.parts) * kQuantWeights;
        const bool good = own_ok(a, item);
        const int end = good ? min(begin + kQuantWeights, a.lens[item]) : 0;
        asm volatile("griddepcontrol.wait;" ::: "memory");
        if (begin >= end) return;
        float m = -INFINITY, l = 0.f;
        for (int s = 0; s < a.slots; ++s) {
            const float2 x = __ldcg(a.part_ml + s * n_rows + at);
            if (x.y == 0.f) continue;
            const float m_new = fmaxf(m, x.x);
            l = l * (m == m_new ? 1.f : exp2f(m - m_new)) + x.y * (x.x == m_new ? 1.f : exp2f(x.x - m_new));
            m = m_new;
        }
        const float inv = l == 0.f ? 0.f : 1.f / l, base = m == -INFINITY ? 0.f : m;
        float* S = p.S + at * p.ld_s;
        constexpr int K = 4;
        for (int j0 = begin + threadIdx.x; j0 < end; j0 += K * 256) {
            float x[K];
#pragma unroll
            for (int k = 0; k < K; ++k) x[k] = j0 + k * 256 < end ? S[j0 + k * 256] : 0.f;
#pragma unroll
            for (int k = 0; k < K; ++k)
                if (j0 + k * 256 < end) S[j0 + k * 256] = exp2f(x[k] - base) * inv;
        }
        return;
    }
    const int per_layer = p.join_ctas / a.n_layers, layer = blockIdx.x / per_layer;
    const int c = threadIdx.x & 15, grp = threadIdx.x / 16 % G;
    const long long at = (long long)(blockIdx.x % per_layer) * (16 / G) + threadIdx.x / (16 * G);
    const bool mine = at < n_rows && own_ok(a, (int)(at / a.H));
    asm volatile("griddepcontrol.wait;" ::: "memory");
    float m = -INFINITY, l = 0.f;
    float4 o = make_float4(0.f, 0.f, 0.f, 0.f);
    auto add = [&](float2 x, float4 v) {
        if (x.y == 0.f) return;                              // nothing seen there: its outputs were not written
        const float m_new = fmaxf(m, x.x);
        const float f = m == m_new ? 1.f : exp2f(m - m_new), b = x.x == m_new ? 1.f : exp2f(x.x - m_new);
        l = l * f + x.y * b;
        o.x = o.x * f + v.x * b; o.y = o.y * f + v.y * b; o.z = o.z * f + v.z * b; o.w = o.w * f + v.w * b;
        m = m_new;
    };
    if (mine) {
#pragma unroll 4
        for (int s = grp; s < a.slots; s += G)
            add(__ldcg(a.part_ml + s * n_rows + at), __ldcg(reinterpret_cast<const float4*>(a.part_o + (((long long)s * a.n_layers + layer) * n_rows + at) * kDh + c * 4)));
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
    T* dst = reinterpret_cast<T*>(a.out) + ((long long)layer * n_rows + at) * kDh + c * 4;
    if constexpr (sizeof(T) == 4) *reinterpret_cast<float4*>(dst) = make_float4(o.x * inv, o.y * inv, o.z * inv, o.w * inv);
    else *reinterpret_cast<uint2*>(dst) = make_uint2(pack_bf16(o.x * inv, o.y * inv), pack_bf16(o.z * inv, o.w * inv));
}

}  // namespace san
