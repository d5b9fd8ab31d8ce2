// Attention of 128 query rows at a time on the fifth-generation tensor cores: long windowed prompts
// (san_window_block) and prefixes with many rows behind them (san_prefix_attn).  S = Softmax(q.K^T / 8) over the
// keys that a row sees, once per block (Eq. 1, Eq. 3), O_l = S.V_l for each layer (Eq. 2, Eq. 4), in one pass with a
// running maximum.
//
// CTA = two tiles of 128 query rows x (key head, up to kTileMaxLayers layers, a run of keys).  Keys come in chunks of 64 that
// both tiles use; per tile and chunk one tcgen05.mma chain writes the scores (M 128, N 64, K 64) into one of
// the tile's two score buffers in tensor memory, and one adds weights x values (N = 64 x layers, K 64) to the outputs,
// which stay there.  Roles:
//   warps 0-3, 4-7  softmax of one tile each: thread = query row = tensor-memory lane, so maxima and sums need no shuffles.
//              The weights go back to tensor memory in bf16, over the scores, as the A operand of the second
//              product.  The maximum that the weights are taken against moves only when a row's own has grown by
//              more than 2^8, since then the outputs have to be read, scaled and written back; the sum uses the
//              same one, so nothing is lost.
//   warps 8-10 copies: 16-byte cp.async into operand tiles (rows of 128 bytes, chunks XOR-swizzled by row & 7, what
//              the matrix descriptors name), keys up to four chunks ahead, values three; rows past the end are zeros.
//   warp 11    issues the MMAs: both tiles' scores of chunk t + 1, then their outputs of chunk t, so that scores
//              are there when a softmax warp comes for them.  MMAs of a thread complete in order: scores never
//              replace weights that have not been read.  All its lanes take the same path and one elected lane
//              issues, which leaves descriptors and addresses in uniform registers: with a single lane in a
//              branch the issue alone took 1700 clocks a chunk (now 1000) and bounded the kernel.
// What bounds it: the softmax warps, one of each tile per SM quarter: 1800 clocks per chunk measured, of which the
// exponentials of both tiles take 1170 (1024 at 16 per clock and SM), maxima 250, waiting for scores 220; the tensor cores
// are busy for a third of it.  Tried on top and not faster: taking turns with the exponentials (1690 to 1880),
// a quarter of them as polynomials on the FMA pipe (1770).  Two prompts of some 7800 positions, window 1024, 8
// heads, 2 layers (97.7 us now): 111 us with one tile per CTA (two CTAs per SM) and weights in shared memory, whose writes, operand reads and
// copies took 750 clocks of shared memory per chunk and tile; 117 us with 128-key chunks and one score buffer
// per tile, where a tile's next scores waited for its outputs.
// Every wait is bounded: one that runs out raises a flag that ends the CTA's other waits, the CTA frees its tensor
// memory and leaves its rows unwritten (reported where there is a status word).
#pragma once

#include "san_attend.cuh"
#include "san_window.cuh"

namespace san {

constexpr int kTileQ = 128, kTileK = 64, kTileThreads = 384, kTileLoaders = 96;
constexpr int kTileKSlots = 4, kTileVSlots = 3, kTileMaxLayers = 2;
constexpr int TAG_TILE = 11;
__host__ __device__ constexpr int tile_smem_bytes(int layers) {
    return 1024 + 2 * kTileQ * 128 + (kTileKSlots + kTileVSlots * layers) * kTileK * 128;
}

__device__ __forceinline__ uint32_t tile_u32(const void* p) { return (uint32_t)__cvta_generic_to_shared(p); }
__device__ __forceinline__ void tile_bar_init(uint64_t* bar, int count) {
    asm volatile("mbarrier.init.shared::cta.b64 [%0], %1;" ::"r"(tile_u32(bar)), "r"(count) : "memory");
}
__device__ __forceinline__ void tile_arrive(uint64_t* bar) {
    asm volatile("mbarrier.arrive.shared::cta.b64 _, [%0];" ::"r"(tile_u32(bar)) : "memory");
}
// Bounded wait for the phase of that parity: false once it has lasted about a second or another wait has given up.
__device__ __noinline__ bool tile_wait_slow(uint32_t addr, uint32_t parity, volatile int* dead) {
    uint32_t ok;
    const long long t0 = clock64();
    for (uint32_t turn = 0;; ++turn) {
        asm volatile("{\n.reg .pred p;\nmbarrier.try_wait.parity.shared::cta.b64 p, [%1], %2, %3;\nselp.u32 %0, 1, 0, p;\n}"
                     : "=r"(ok) : "r"(addr), "r"(parity), "r"(1000000u) : "memory");
        if (ok) return true;
        if ((turn & 63u) != 63u) continue;
        if (*dead) return false;
        if (clock64() - t0 > 2000000000LL) { *dead = 1; return false; }
    }
}
__device__ __forceinline__ bool tile_wait(uint64_t* bar, uint32_t parity, volatile int* dead) {
    const uint32_t addr = tile_u32(bar);
    uint32_t ok;
    asm volatile("{\n.reg .pred p;\nmbarrier.test_wait.parity.shared::cta.b64 p, [%1], %2;\nselp.u32 %0, 1, 0, p;\n}" : "=r"(ok) : "r"(addr), "r"(parity) : "memory");
    return ok ? true : tile_wait_slow(addr, parity, dead);
}
// The same for a whole warp, which goes on together: a lane left behind could meet the barrier two phases later, when
// the parity it waits for means another phase.
__device__ __forceinline__ bool tile_wait_warp(uint64_t* bar, uint32_t parity, volatile int* dead) {
    return __all_sync(0xffffffffu, tile_wait(bar, parity, dead));
}
// Shared-memory matrix descriptor: 128-byte swizzle, groups of 8 rows 1024 bytes apart; `lead`: bytes between the 64-element
// column blocks of an MN-major operand wider than 64.
__device__ __forceinline__ uint64_t tile_desc(uint32_t addr, uint32_t lead = 16) {
    return (uint64_t)((addr >> 4) & 0x3fffu) | ((uint64_t)((lead >> 4) & 0x3fffu) << 16) | ((uint64_t)(1024 >> 4) << 32) |
           ((uint64_t)1 << 46) | ((uint64_t)2 << 61);
}
// Instruction descriptor: float32 accumulator, bf16 operands, M 128, N n; b_mn: B is MN-major.
__device__ __forceinline__ uint32_t tile_idesc(bool b_mn, int n) {
    return (1u << 4) | (1u << 7) | (1u << 10) | (b_mn ? 1u << 16 : 0u) | ((uint32_t)(n >> 3) << 17) | ((uint32_t)(128 >> 4) << 24);
}
__device__ __forceinline__ void tile_mma(uint32_t d, uint64_t a, uint64_t b, uint32_t idesc, bool add) {
    asm volatile("{\n.reg .pred p;\nsetp.ne.b32 p, %4, 0;\ntcgen05.mma.cta_group::1.kind::f16 [%0], %1, %2, %3, p;\n}"
                 :: "r"(d), "l"(a), "l"(b), "r"(idesc), "r"(add ? 1u : 0u) : "memory");
}
// A in tensor memory: lane = row, a column holds two neighbouring elements of K.
__device__ __forceinline__ void tile_mma_ta(uint32_t d, uint32_t a, uint64_t b, uint32_t idesc, bool add) {
    asm volatile("{\n.reg .pred p;\nsetp.ne.b32 p, %4, 0;\ntcgen05.mma.cta_group::1.kind::f16 [%0], [%1], %2, %3, p;\n}"
                 :: "r"(d), "r"(a), "l"(b), "r"(idesc), "r"(add ? 1u : 0u) : "memory");
}
__device__ __forceinline__ void tile_commit(uint64_t* bar) {
    asm volatile("tcgen05.commit.cta_group::1.mbarrier::arrive::one.shared::cluster.b64 [%0];" ::"r"(tile_u32(bar)) : "memory");
}
__device__ __forceinline__ void tile_before_sync() { asm volatile("tcgen05.fence::before_thread_sync;" ::: "memory"); }
__device__ __forceinline__ void tile_after_sync() { asm volatile("tcgen05.fence::after_thread_sync;" ::: "memory"); }
__device__ __forceinline__ void tile_proxy_fence() { asm volatile("fence.proxy.async.shared::cta;" ::: "memory"); }
// 32 columns of this thread's lane, without the wait.
__device__ __forceinline__ void tile_ld32(uint32_t addr, float* v) {
    uint32_t* r = reinterpret_cast<uint32_t*>(v);
    asm volatile("tcgen05.ld.sync.aligned.32x32b.x32.b32 "
                 "{%0,%1,%2,%3,%4,%5,%6,%7,%8,%9,%10,%11,%12,%13,%14,%15,%16,%17,%18,%19,%20,%21,%22,%23,%24,%25,%26,%27,%28,%29,%30,%31}, [%32];"
                 : "=r"(r[0]), "=r"(r[1]), "=r"(r[2]), "=r"(r[3]), "=r"(r[4]), "=r"(r[5]), "=r"(r[6]), "=r"(r[7]),
                   "=r"(r[8]), "=r"(r[9]), "=r"(r[10]), "=r"(r[11]), "=r"(r[12]), "=r"(r[13]), "=r"(r[14]), "=r"(r[15]),
                   "=r"(r[16]), "=r"(r[17]), "=r"(r[18]), "=r"(r[19]), "=r"(r[20]), "=r"(r[21]), "=r"(r[22]), "=r"(r[23]),
                   "=r"(r[24]), "=r"(r[25]), "=r"(r[26]), "=r"(r[27]), "=r"(r[28]), "=r"(r[29]), "=r"(r[30]), "=r"(r[31])
                 : "r"(addr) : "memory");
}
__device__ __forceinline__ void tile_ld16(uint32_t addr, float* v) {
    uint32_t* r = reinterpret_cast<uint32_t*>(v);
    asm volatile("tcgen05.ld.sync.aligned.32x32b.x16.b32 {%0,%1,%2,%3,%4,%5,%6,%7,%8,%9,%10,%11,%12,%13,%14,%15}, [%16];"
                 : "=r"(r[0]), "=r"(r[1]), "=r"(r[2]), "=r"(r[3]), "=r"(r[4]), "=r"(r[5]), "=r"(r[6]), "=r"(r[7]),
                   "=r"(r[8]), "=r"(r[9]), "=r"(r[10]), "=r"(r[11]), "=r"(r[12]), "=r"(r[13]), "=r"(r[14]), "=r"(r[15])
                 : "r"(addr) : "memory");
}
__device__ __forceinline__ void tile_st16(uint32_t addr, const float* v) {
    const uint32_t* r = reinterpret_cast<const uint32_t*>(v);
    asm volatile("tcgen05.st.sync.aligned.32x32b.x16.b32 [%16], {%0,%1,%2,%3,%4,%5,%6,%7,%8,%9,%10,%11,%12,%13,%14,%15};"
                 :: "r"(r[0]), "r"(r[1]), "r"(r[2]), "r"(r[3]), "r"(r[4]), "r"(r[5]), "r"(r[6]), "r"(r[7]),
                    "r"(r[8]), "r"(r[9]), "r"(r[10]), "r"(r[11]), "r"(r[12]), "r"(r[13]), "r"(r[14]), "r"(r[15]), "r"(addr) : "memory");
}
__device__ __forceinline__ void tile_wait_ld() { asm volatile("tcgen05.wait::ld.sync.aligned;" ::: "memory"); }
__device__ __forceinline__ void tile_wait_st() { asm volatile("tcgen05.wait::st.sync.aligned;" ::: "memory"); }

// Two float32 numbers in one instruction, and the largest of three.
__device__ __forceinline__ unsigned long long tile_pair(float x, float y) {
    unsigned long long r;
    asm("mov.b64 %0, {%1, %2};" : "=l"(r) : "f"(x), "f"(y));
    return r;
}
__device__ __forceinline__ void tile_unpair(unsigned long long r, float& x, float& y) { asm("mov.b64 {%0, %1}, %2;" : "=f"(x), "=f"(y) : "l"(r)); }
__device__ __forceinline__ unsigned long long tile_fma2(unsigned long long a, unsigned long long b, unsigned long long c) {
    unsigned long long d;
    asm("fma.rn.f32x2 %0, %1, %2, %3;" : "=l"(d) : "l"(a), "l"(b), "l"(c));
    return d;
}
__device__ __forceinline__ unsigned long long tile_add2(unsigned long long a, unsigned long long b) {
    unsigned long long d;
    asm("add.rn.f32x2 %0, %1, %2;" : "=l"(d) : "l"(a), "l"(b));
    return d;
}
__device__ __forceinline__ float tile_max3(float a, float b, float c) {
    float d;
    asm("max.f32 %0, %1, %2, %3;" : "=f"(d) : "f"(a), "f"(b), "f"(c));
    return d;
}

// What a CTA works on.  Visible keys are numbered 0 .. end - 1: the first ns of them are rows 0.., the others rows lo...
struct TileWork {
    const char* k; const char* v;
    long long row_bytes, v_stride;          // bytes between rows, between layers
    int ns, lo, begin, end;
    int rows, layer0, layers;               // query rows, up to two tiles of them
};

// A warp writes 128 bytes of each of its lanes' rows (`piece`, to `dst`, if `mine`) by way of shared memory, so that eight lanes
// write a row's 128 bytes side by side.  `rows`: the warp's own 32 rows of 128 bytes.
__device__ __forceinline__ void tile_write_rows(char* rows, const uint4 (&piece)[8], char* dst, bool mine) {
    const int lane = threadIdx.x & 31;
    __syncwarp();
#pragma unroll
    for (int c = 0; c < 8; ++c) *reinterpret_cast<uint4*>(rows + lane * 128 + ((c ^ (lane & 7)) << 4)) = piece[c];
    __syncwarp();
    const unsigned long long to = mine ? reinterpret_cast<unsigned long long>(dst) : 0ull;
#pragma unroll
    for (int j = 0; j < 8; ++j) {
        const int r = j * 4 + (lane >> 3), c = lane & 7;
        const unsigned long long at = __shfl_sync(0xffffffffu, to, r);
        const uint4 v = *reinterpret_cast<const uint4*>(rows + r * 128 + ((c ^ (r & 7)) << 4));
        if (at) *reinterpret_cast<uint4*>(at + (c << 4)) = v;
    }
}

// Which chunks (numbers t of a CTA's run) a tile takes part in: t < sinks or first <= t < end; and from which to which all
// of its rows see all of the chunk.
struct TileRange {
    int sinks, first, end, whole_first, whole_end;
    __device__ __forceinline__ bool any(int t) const { return t < sinks || (t >= first && t < end); }
    __device__ __forceinline__ bool whole(int t) const { return t >= whole_first && t < whole_end; }
};

template <int WARPS> __device__ __noinline__ void tile_rows_again(const WindowParams& p, char* smem, const uint32_t* again_s);

// ---- windowed prompts: CTA = (query tiles, head, sequence, layer group), longest prompts' ends first; CTAs from
// `whole` on take one tile each of the pairs that are left (see launch_tiles of the host side)
struct TileWindow {
    static constexpr int kRegs = 168;
    const WindowParams& p;
    int seq, head, a0, len;
    __device__ __forceinline__ bool work(TileWork* w) {
        int index = blockIdx.x, half = -1;
        if (index >= p.whole) {
            half = (index - p.whole) & 1;
            index = p.whole + (index - p.whole) / 2;
        }
        const int layer_group = index % p.n_lg; index /= p.n_lg;
        head = index % p.H; index /= p.H;
        seq = index % p.n_seq;
        const int pair = p.pairs - 1 - index / p.n_seq;
        w->layer0 = layer_group * p.lg;
        w->layers = min(p.lg, p.n_layers - w->layer0);
        len = max(0, min(p.lens[seq], p.max_len));
        a0 = pair * 2 * kTileQ + (half > 0 ? kTileQ : 0);
        if (a0 >= len) return false;
        w->rows = min(half < 0 ? 2 * kTileQ : kTileQ, len - a0);
        w->lo = max(0, a0 - p.window + 1);
        w->ns = min(p.n_sink, w->lo);
        w->begin = 0;
        w->end = w->ns + a0 + w->rows - w->lo;
        const long long at = ((long long)seq * p.cap * p.Hk + head / p.group) * 128;
        w->row_bytes = (long long)p.Hk * 128;
        w->v_stride = p.v_layer * 2;
        w->k = reinterpret_cast<const char*>(p.k) + at;
        w->v = reinterpret_cast<const char*>(p.v) + at + w->layer0 * w->v_stride;
        return true;
    }
    __device__ __forceinline__ const uint4* query(int i) const {
        return reinterpret_cast<const uint4*>(p.q + (((long long)seq * p.cap + a0 + i) * p.H + head) * kDh);
    }
    __device__ __forceinline__ TileRange range(const TileWork& w, int x) const {
        const int first = a0 + x * kTileQ, last = min(first + kTileQ, a0 + w.rows) - 1;      // rows of the tile
        if (last < first) return {0, 0, 0, 0, 0};
        auto number = [&](int key) { return key - w.lo + w.ns; };
        TileRange r;
        r.end = number(last) / kTileK + 1;
        r.first = number(max(first - p.window + 1, w.lo)) / kTileK;
        r.sinks = min((number(max(p.n_sink, w.lo)) + kTileK - 1) / kTileK, r.end);           // numbers below it are sinks
        r.whole_first = (number(max(first + kTileQ - p.window, w.lo)) + kTileK - 1) / kTileK;
        r.whole_end = min(number(first) + 1, w.end) / kTileK;
        return r;
    }
    // Of columns 32 q .. 32 q + 31 of chunk [c0, c0 + 64) of the visible keys, those that row i sees.
    __device__ __forceinline__ uint32_t seen(const TileWork& w, int c0, int i, int q) const {
        auto below = [&](int n) { n -= c0 + 32 * q; return n <= 0 ? 0u : n >= 32 ? ~0u : (1u << n) - 1; };      // of numbers below n
        const int a = a0 + i, self = w.ns + a - w.lo;                   // the row's own number
        const uint32_t recent = ~below(w.ns + max(a - p.window + 1, w.lo) - w.lo);
        return (recent | below(w.ns + max(0, p.n_sink - w.lo))) & below(min(self + 1, w.end));
    }
    template <int LG> __device__ __forceinline__ void finish(const TileWork& w, uint32_t t_out, char* rows, uint32_t* again_s, int i, float m, float l) const {
        const bool mine = i < w.rows;
        const float inv = l == 0.f ? 0.f : 1.f / l;
        bool odd = false;
        __nv_bfloat16* dst = p.out + (((long long)seq * p.cap + a0 + i) * p.H + head) * kDh;
#pragma unroll
        for (int y = 0; y < LG; ++y) {
            if (y >= w.layers) break;
            uint4 piece[8];
#pragma unroll
            for (int h = 0; h < 2; ++h) {
                float o[32];
                __syncwarp();
                tile_ld32(t_out + y * 64 + h * 32, o);
                tile_wait_ld();
#pragma unroll
                for (int c = 0; c < 32; ++c) { o[c] *= inv; odd |= o[c] != o[c]; }
#pragma unroll
                for (int c = 0; c < 4; ++c)
                    piece[h * 4 + c] = make_uint4(pack_bf16(o[8 * c], o[8 * c + 1]), pack_bf16(o[8 * c + 2], o[8 * c + 3]),
                                                  pack_bf16(o[8 * c + 4], o[8 * c + 5]), pack_bf16(o[8 * c + 6], o[8 * c + 7]));
            }
            tile_write_rows(rows, piece, reinterpret_cast<char*>(dst + (w.layer0 + y) * p.out_layer), mine);
        }
        const unsigned rows_odd = __ballot_sync(0xffffffffu, odd && mine);
        if ((threadIdx.x & 31) == 0) again_s[threadIdx.x >> 5] = rows_odd;
    }
    template <int WARPS> __device__ __forceinline__ void again(char* smem, const uint32_t* again_s) const {
        uint32_t any = 0;
        for (int k = 0; k < 2 * kTileQ / 32; ++k) any |= again_s[k];
        if (any) tile_rows_again<WARPS>(p, smem, again_s);
    }
    __device__ __forceinline__ void failed() const {}
};

// Row a of (sequence, head), one layer, by one warp: over the rows that are seen and no others, as a row of a decode step.
constexpr int kAgainBytes = 2 * kAtTile * 128;                          // of shared memory for a warp
__device__ __forceinline__ void tile_row_again(const WindowParams& p, int seq, int head, int layer, int a, char* smem, int lane) {
    struct { const char* q; int H, group; float scale_log2e; } rows;
    rows.q = reinterpret_cast<const char*>(p.q + (long long)seq * p.cap * p.H * kDh);
    rows.H = p.H; rows.group = 1; rows.scale_log2e = p.scale_log2e;
    const long long kv = ((long long)seq * p.cap * p.Hk + head / p.group) * kDh;
    AttendRun u;
    u.k = reinterpret_cast<const char*>(p.k + kv);
    u.v = reinterpret_cast<const char*>(p.v + layer * p.v_layer + kv);
    u.row_bytes = u.v_row_bytes = (long long)p.Hk * 128; u.v_stride = 0; u.permuted = false;
    u.lo = max(0, a - p.window + 1);
    u.n_sink = min(p.n_sink, u.lo);
    u.n = u.n_sink + a + 1 - u.lo;
    u.begin = 0; u.end = u.n;
    u.item0 = a; u.row0 = 0; u.rows = 1; u.head0 = head;
    u.layer0 = layer; u.layers = 1; u.slot = 0;
    float2* ml = reinterpret_cast<float2*>(smem + kAtTile * 128);
    __syncwarp();                                                       // the row before has been written
    attend_warp_bf16<1, 2>(rows, u, 0, kAtTile, smem, ml, lane);
    __syncwarp();
    const float l = ml[0].y, inv = l == 0.f ? 0.f : 1.f / l;
    const float2 o = *reinterpret_cast<const float2*>(smem + lane * 8);
    *reinterpret_cast<uint32_t*>(p.out + layer * p.out_layer + (((long long)seq * p.cap + a) * p.H + head) * kDh + lane * 2) = pack_bf16(o.x * inv, o.y * inv);
}

// All threads of a CTA that is done: rows that came out as NaN (again_s, a bit for each) are computed again where a value that
// was multiplied by a weight of zero can be the cause, which chunks that not all of the tile's rows see may hold.  Rows that
// are NaN by what they see stay: with one NaN among the sinks those are all rows of a prompt.  2 x 8192 positions, window 1024, 8
// heads, 2 layers: 105 us; with a NaN value among the sinks 0.16 ms, in the middle 1.4, in every row 4.5 (one position
// after the other for every row that is NaN took 198, 52 and 198).
template <int WARPS> __device__ __noinline__ void tile_rows_again(const WindowParams& p, char* smem, const uint32_t* again_s) {
    static_assert(WARPS <= kTileThreads / 32, "warps");
    TileWindow mode{p};
    TileWork w;
    mode.work(&w);
    bool spoiled = false;
    for (int x = 0; x < 2; ++x) {
        if ((again_s[4 * x] | again_s[4 * x + 1] | again_s[4 * x + 2] | again_s[4 * x + 3]) == 0) continue;
        const TileRange r = mode.range(w, x);
        const int first = mode.a0 + x * kTileQ, last = min(first + kTileQ, mode.a0 + w.rows) - 1;      // rows of the tile
        for (int t = 0; t * kTileK < w.end; ++t) {
            if (!r.any(t) || r.whole(t)) continue;
            for (int i = threadIdx.x; i < w.layers * kTileK * 8; i += kTileThreads) {
                const int n = t * kTileK + (i >> 3) % kTileK, y = i / (kTileK * 8), b = n < w.ns ? n : w.lo + n - w.ns;
                if (n >= w.end || (b <= first && (b < p.n_sink || b > last - p.window))) continue;      // none, or seen by all
                const uint4 v = *reinterpret_cast<const uint4*>(w.v + y * w.v_stride + b * w.row_bytes + (i & 7) * 16);
                const uint32_t e = 0x7f80u;                             // an exponent of all ones: no finite number
                for (const uint32_t z : {v.x, v.y, v.z, v.w}) spoiled |= (z & e) == e || (z >> 16 & e) == e;
            }
        }
    }
    if (!__syncthreads_or(spoiled)) return;
    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
    int n = 0;
    for (int k = 0; k < 2 * kTileQ / 32; ++k)
        for (uint32_t rows = again_s[k]; rows; rows &= rows - 1, ++n)
            for (int y = 0; y < w.layers && n % WARPS == warp; ++y)
                tile_row_again(p, mode.seq, mode.head, w.layer0 + y, mode.a0 + 32 * k + __ffs(rows) - 1, smem + warp * kAgainBytes, lane);
}

// ---- shared prefixes: units as in attend_unit, 128 query rows and runs of p_span chunks
struct TilePrefix {
    static constexpr int kRegs = 136;       // leaves registers for a CTA of attend_kernel beside it on the SM
    const AttendParams& p;
    int g, hk, row0, slot;
    __device__ __forceinline__ bool work(TileWork* w) {
        asm volatile("griddepcontrol.launch_dependents;");              // the sequences' own rows may be worked on meanwhile
        int index = blockIdx.x;
        const int lg = index % p.t_n_lg; index /= p.t_n_lg;
        const int split = index % p.p_splits; index /= p.p_splits;
        hk = index % p.Hk; index /= p.Hk;
        const int tile = index % p.p_row_tiles;
        g = index / p.p_row_tiles;
        if (!prefix_ok(p, g)) {
            if (threadIdx.x == 0 && tile == 0 && split == 0 && hk == 0 && lg == 0) prefix_report(p, g);
            return false;
        }
        row0 = tile * 2 * kTileQ;
        w->rows = min(2 * kTileQ, (p.first[g + 1] - p.first[g]) * p.group - row0);
        if (w->rows <= 0) return false;
        w->layer0 = lg * p.t_lg;
        w->layers = min(p.t_lg, p.n_layers - w->layer0);
        w->ns = 0; w->lo = 0;
        w->begin = min(split * p.p_span * kTileK, p.plens[g]);
        w->end = min(w->begin + p.p_span * kTileK, p.plens[g]);
        const long long at = ((long long)g * p.pcap * p.Hk + hk) * 128;
        w->row_bytes = (long long)p.Hk * 128;
        w->v_stride = p.pv_stride;
        w->k = p.pk + at;
        w->v = p.pv + at + w->layer0 * p.pv_stride;
        slot = split;
        return true;
    }
    __device__ __forceinline__ long long place(int i) const {
        const int row = row0 + i;
        return (long long)(p.first[g] + row / p.group) * p.H + hk * p.group + row % p.group;
    }
    __device__ __forceinline__ const uint4* query(int i) const { return reinterpret_cast<const uint4*>(p.q + place(i) * 128); }
    __device__ __forceinline__ TileRange range(const TileWork& w, int x) const {
        if (x * kTileQ >= w.rows) return {0, 0, 0, 0, 0};
        return {0, 0, (w.end - w.begin + kTileK - 1) / kTileK, 0, (w.end - w.begin) / kTileK};
    }
    __device__ __forceinline__ uint32_t seen(const TileWork& w, int c0, int, int q) const {
        const int n = w.end - c0 - 32 * q;
        return n <= 0 ? 0u : n >= 32 ? ~0u : (1u << n) - 1;
    }
    template <int LG> __device__ __forceinline__ void finish(const TileWork& w, uint32_t t_out, char* rows, uint32_t*, int i, float m, float l) const {
        const long long n_rows = (long long)p.n_items * p.H, at = i < w.rows ? place(i) : 0;
        const bool mine = i < w.rows;
        if (mine && w.layer0 == 0) p.part_ml[slot * n_rows + at] = make_float2(m, l);
        if (w.begin == w.end) return;                                   // nothing there: the join does not look at the outputs
#pragma unroll
        for (int y = 0; y < LG; ++y) {
            if (y >= w.layers) break;
            float* dst = p.part_o + (((long long)slot * p.n_layers + w.layer0 + y) * n_rows + at) * kDh;
#pragma unroll
            for (int h = 0; h < 2; ++h) {
                uint4 piece[8];
                __syncwarp();
                tile_ld32(t_out + y * 64 + h * 32, reinterpret_cast<float*>(piece));
                tile_wait_ld();
                tile_write_rows(rows, piece, reinterpret_cast<char*>(dst + h * 32), mine);
            }
        }
    }
    template <int WARPS> __device__ __forceinline__ void again(char*, const uint32_t*) const {}      // all rows see all there is
    __device__ __forceinline__ void failed() const {
        if (p.status && atomicCAS(&p.status[0], 0, (int)SAN_ERR_TIMEOUT) == 0) { p.status[1] = TAG_TILE; p.status[2] = g; }
    }
};

template <class Mode, int LG, class Params>
__global__ void __maxnreg__(Mode::kRegs) tile_kernel(const __grid_constant__ Params params) {
    constexpr uint32_t kCols = 512, kTileCols = 256, kOut = 128;        // a tile's columns: scores twice (weights over them), outputs
    static_assert(kOut + 64 * LG <= kTileCols, "tensor memory");
    extern __shared__ __align__(1024) char tile_smem[];
    __shared__ __align__(8) uint64_t k_full[kTileKSlots], k_free[kTileKSlots], v_full[kTileVSlots], v_free[kTileVSlots], s_full[2][2], p_full[2][2], pv_done[2][2], q_full[2];
    __shared__ uint32_t tmem_s;
    __shared__ int dead_s;
    __shared__ uint32_t again_s[2 * kTileQ / 32];
    Mode mode{params};
    TileWork w;
    if (!mode.work(&w)) return;                                         // uniform over the CTA, before anything is allocated
    const int warp = threadIdx.x >> 5;
    volatile int* dead = &dead_s;
    char* sQ = tile_smem + ((1024u - (tile_u32(tile_smem) & 1023u)) & 1023u);
    const uint32_t aK = tile_u32(sQ) + 2 * kTileQ * 128;
    const uint32_t aV = aK + kTileKSlots * kTileK * 128;                // slots of LG value tiles
    if (threadIdx.x == 0) {
        for (int i = 0; i < kTileKSlots; ++i) { tile_bar_init(&k_full[i], kTileLoaders); tile_bar_init(&k_free[i], 1); }
        for (int i = 0; i < kTileVSlots; ++i) { tile_bar_init(&v_full[i], kTileLoaders); tile_bar_init(&v_free[i], 1); }
        for (int i = 0; i < 2; ++i) {
            tile_bar_init(&s_full[i][0], 1); tile_bar_init(&s_full[i][1], 1);
            tile_bar_init(&q_full[i], kTileQ);
            tile_bar_init(&p_full[i][0], kTileQ); tile_bar_init(&p_full[i][1], kTileQ); tile_bar_init(&pv_done[i][0], 1); tile_bar_init(&pv_done[i][1], 1);
        }
        asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
        dead_s = 0;
        for (int i = 0; i < 2 * kTileQ / 32; ++i) again_s[i] = 0;
    }
    if (warp == 11) {
        asm volatile("tcgen05.alloc.cta_group::1.sync.aligned.shared::cta.b32 [%0], %1;" :: "r"(tile_u32(&tmem_s)), "r"(kCols) : "memory");
        asm volatile("tcgen05.relinquish_alloc_permit.cta_group::1.sync.aligned;" ::: "memory");
    }
    tile_before_sync();
    __syncthreads();
    tile_after_sync();
    const uint32_t tmem = tmem_s;
    const int chunks = (w.end - w.begin + kTileK - 1) / kTileK;

    if (warp == 11) {
        uint32_t elected;                                           // 1 in one lane
        asm volatile("{\n.reg .pred p;\nelect.sync _|p, 0xffffffff;\nselp.u32 %0, 1, 0, p;\n}" : "=r"(elected));
        const uint32_t id_s = tile_idesc(false, kTileK), id_o = tile_idesc(true, w.layers * kDh);
        const TileRange range[2] = {mode.range(w, 0), mode.range(w, 1)};
        int scored[2] = {0, 0}, applied[2] = {0, 0};                // chunks of a tile whose MMAs have been issued
        auto scores = [&](int t) -> bool {
            const int slot = t % kTileKSlots;
            if (!tile_wait_warp(&k_full[slot], (uint32_t)(t / kTileKSlots) & 1u, dead)) return false;
            tile_proxy_fence();                                     // the copies are writes of the generic proxy
            tile_after_sync();
            const uint64_t dK = tile_desc(aK + (uint32_t)slot * (kTileK * 128));
#pragma unroll
            for (int x = 0; x < 2; ++x) {
                if (!range[x].any(t)) continue;
                const uint64_t dQ = tile_desc(tile_u32(sQ) + (uint32_t)x * (kTileQ * 128));
                const int buf = scored[x] & 1;                      // its weights of two chunks ago have been applied (in order)
                if (elected) {
#pragma unroll
                    for (int s = 0; s < 4; ++s) tile_mma(tmem + (uint32_t)x * kTileCols + buf * kTileK, dQ + 2 * s, dK + 2 * s, id_s, s > 0);
                    tile_commit(&s_full[x][buf]);
                }
                ++scored[x];
            }
            if (elected) tile_commit(&k_free[slot]);
            return true;
        };
        auto outputs = [&](int t) -> bool {
            const int slot = t % kTileVSlots;
            if (!tile_wait_warp(&v_full[slot], (uint32_t)(t / kTileVSlots) & 1u, dead)) return false;
            tile_proxy_fence();
            const uint64_t dV = tile_desc(aV + (uint32_t)(slot * LG) * (kTileK * 128), kTileK * 128);
#pragma unroll
            for (int x = 0; x < 2; ++x) {
                if (!range[x].any(t)) continue;
                if (!tile_wait_warp(&p_full[x][applied[x] & 1], (uint32_t)(applied[x] >> 1) & 1u, dead)) return false;
                tile_after_sync();
                const uint32_t base = tmem + (uint32_t)x * kTileCols;
                if (elected) {
#pragma unroll
                    for (int s = 0; s < kTileK / 16; ++s)
                        tile_mma_ta(base + kOut, base + (applied[x] & 1) * kTileK + 8 * s, dV + 128 * s, id_o, applied[x] > 0 || s > 0);
                    tile_commit(&pv_done[x][applied[x] & 1]);
                }
                ++applied[x];
            }
            if (elected) tile_commit(&v_free[slot]);
            return true;
        };
        bool go = tile_wait_warp(&q_full[0], 0u, dead) && tile_wait_warp(&q_full[1], 0u, dead) && (chunks == 0 || scores(0));
        for (int t = 0; t < chunks && go; ++t) go = (t + 1 >= chunks || scores(t + 1)) && outputs(t);
    } else if (warp >= 8) {
        // thread: 16-byte piece c of rows r0, r0 + 12, ...
        constexpr int kRows = (kTileK + 11) / 12;
        static_assert(kTileLoaders == 96, "rows of a thread");
        const int r0 = (threadIdx.x - 2 * kTileQ) >> 3, c = threadIdx.x & 7;
        const uint32_t sw0 = (uint32_t)(r0 * 128 + ((c ^ (r0 & 7)) << 4)), sw1 = (uint32_t)(r0 * 128 + ((c ^ ((r0 + 4) & 7)) << 4));
        const long long step = 12 * w.row_bytes;
        auto copy = [&](const char* src, uint32_t dst, int c0) {
            const int first = c0 + r0;
            if (c0 >= w.ns && c0 + kTileK <= w.end) {                   // rows on end
                const char* at = src + (long long)(w.lo + first - w.ns) * w.row_bytes + (c << 4);
#pragma unroll
                for (int j = 0; j < kRows; ++j, at += step)
                    if (r0 + 12 * j < kTileK) cp16(dst + (uint32_t)(j * 12 * 128) + (j & 1 ? sw1 : sw0), at, true);
            } else {
#pragma unroll
                for (int j = 0; j < kRows; ++j) {
                    const int n = first + j * 12;
                    const bool full = n < w.end;
                    const int pos = !full ? 0 : n < w.ns ? n : w.lo + n - w.ns;
                    if (r0 + 12 * j < kTileK) cp16(dst + (uint32_t)(j * 12 * 128) + (j & 1 ? sw1 : sw0), src + pos * w.row_bytes + (c << 4), full);
                }
            }
        };
        // the barrier hears of a thread's copies when they have landed; the thread does not wait for them
        auto landed = [](uint64_t* bar) {
            asm volatile("cp.async.mbarrier.arrive.noinc.shared::cta.b64 [%0];" ::"r"(tile_u32(bar)) : "memory");
        };
        for (int t = 0; t < chunks; ++t) {
            const int c0 = w.begin + t * kTileK, ks = t % kTileKSlots, vs = t % kTileVSlots;
            if (t >= kTileKSlots && !tile_wait(&k_free[ks], (uint32_t)(t / kTileKSlots - 1) & 1u, dead)) break;
            copy(w.k, aK + (uint32_t)ks * (kTileK * 128), c0);
            landed(&k_full[ks]);
            if (t >= kTileVSlots && !tile_wait(&v_free[vs], (uint32_t)(t / kTileVSlots - 1) & 1u, dead)) break;
            for (int y = 0; y < w.layers; ++y) copy(w.v + y * w.v_stride, aV + (uint32_t)(vs * LG + y) * (kTileK * 128), c0);
            landed(&v_full[vs]);
        }
        asm volatile("cp.async.wait_all;" ::: "memory");
    } else {
        const int x = warp >> 2, i = threadIdx.x;                       // tile; query row of the CTA
        const uint32_t lanes = tmem + ((uint32_t)((warp & 3) * 32) << 16) + (uint32_t)x * kTileCols;
        const float sc = params.scale_log2e;
        const unsigned long long sc2 = tile_pair(sc, sc);
        {
            const uint4* src = i < w.rows ? mode.query(i) : nullptr;
#pragma unroll
            for (int c = 0; c < 8; ++c)
                *reinterpret_cast<uint4*>(sQ + i * 128 + ((c ^ (i & 7)) << 4)) = src ? src[c] : make_uint4(0, 0, 0, 0);
            tile_proxy_fence();
            tile_arrive(&q_full[x]);
        }
        float m = -INFINITY, l = 0.f;
        bool ok = true;
        int count = 0;
        const TileRange range = mode.range(w, x);
        // The outputs of the tile's chunk n are complete.  Two barriers in turn, as for scores and weights, because a wait
        // names a phase by its parity: the outputs of chunk n - 2 were complete before the scores of chunk n.
        auto outputs = [&](int n) -> bool { return tile_wait_warp(&pv_done[x][n & 1], (uint32_t)(n >> 1) & 1u, dead); };
        for (int t = 0; t < chunks; ++t) {
            const int c0 = w.begin + t * kTileK;
            if (!range.any(t)) continue;
            const uint32_t buf = lanes + (count & 1) * kTileK;
            ok = tile_wait_warp(&s_full[x][count & 1], (uint32_t)(count >> 1) & 1u, dead);
            if (!ok) break;
            tile_after_sync();
            float z[64];
            tile_ld32(buf, z);
            tile_ld32(buf + 32, z + 32);
            tile_wait_ld();
            if (!range.whole(t)) {                                      // uniform over the tile's warps
                const uint32_t s0 = mode.seen(w, c0, i, 0), s1 = mode.seen(w, c0, i, 1);
#pragma unroll
                for (int j = 0; j < 32; ++j) {
                    z[j] = s0 >> j & 1u ? z[j] : -INFINITY;
                    z[32 + j] = s1 >> j & 1u ? z[32 + j] : -INFINITY;
                }
            }
            float top[4] = {z[0], z[1], z[2], z[3]};
#pragma unroll
            for (int j = 4; j < 60; j += 8)
#pragma unroll
                for (int e = 0; e < 4; ++e) top[e] = tile_max3(top[e], z[j + 2 * e], z[j + 2 * e + 1]);
#pragma unroll
            for (int e = 0; e < 4; ++e) top[e] = fmaxf(top[e], z[60 + e]);
            const float m_chunk = fmaxf(fmaxf(top[0], top[1]), fmaxf(top[2], top[3])) * sc;
            // A row that has seen nothing yet has outputs and a sum of zero: its maximum starts here.
            const bool grown = m_chunk > m + 8.f && m > -INFINITY;
            if (m == -INFINITY) m = m_chunk;
            if (__any_sync(0xffffffffu, grown)) {                       // (count > 0)
                ok = outputs(count - 1);                                // those of this chunk wait for its weights
                if (!ok) break;
                tile_after_sync();
                const float f = grown ? fast_exp2(m - m_chunk) : 1.f;
                if (grown) { m = m_chunk; l *= f; }
                for (int y = 0; y < 4 * w.layers; ++y) {                // 16 columns at a time: the scores are still held
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
                tile_unpair(tile_fma2(tile_pair(z[j], z[j + 1]), sc2, m2), u, v);
                u = fast_exp2(u);
                v = fast_exp2(v);
                sum[(j >> 1) & 1] = tile_add2(sum[(j >> 1) & 1], tile_pair(u, v));
                packed[j >> 1] = __uint_as_float(pack_bf16(u, v));
            }
            tile_st16(buf, packed);                                     // over the scores, which have been read
            tile_st16(buf + 16, packed + 16);
            float sa, sb;
            tile_unpair(tile_add2(sum[0], sum[1]), sa, sb);
            l += sa + sb;
            tile_wait_st();
            tile_before_sync();
            tile_arrive(&p_full[x][count & 1]);
            ++count;
        }
        if (ok && count > 0) ok = outputs(count - 1);
        tile_after_sync();
        if (ok) mode.template finish<LG>(w, lanes + kOut, sQ + (i & ~31) * 128, again_s, i, m, l);       // (the queries have been read)
    }
    tile_before_sync();
    __syncthreads();
    if (warp == 11) {
        __syncwarp();
        asm volatile("tcgen05.dealloc.cta_group::1.sync.aligned.b32 %0, %1;" :: "r"(tmem), "r"(kCols) : "memory");
    }
    // Whichever warp's wait ran out: the other tile may have finished by then.
    if (*dead != 0) {
        if (threadIdx.x == 0) mode.failed();
        return;
    }
    constexpr int kAgainWarps = (tile_smem_bytes(LG) - 1024) / kAgainBytes;      // as many as find room in the operands' place
    mode.template again<kAgainWarps < kTileThreads / 32 ? kAgainWarps : kTileThreads / 32>(sQ, again_s);
}

}  // namespace san
