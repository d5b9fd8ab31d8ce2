// Host side of the calls around the decode step of a beam decoder with long prompts: beam selection,
// step attention behind shared prefixes and over sliding windows, windowed prompts.  Argument checks
// and how the work is cut; the arithmetic is in san_select.cuh, san_attend.cuh and san_window.cuh.
#include <algorithm>
#include <cmath>
#include <cstring>

#include "san_ctx.h"
#include "san_kernels.cuh"
#include "san_select.cuh"
#include "san_attend.cuh"
#include "san_window.cuh"
#include "san_tile.cuh"

using namespace san;

namespace {

constexpr int kSms = 148;                   // the cuts are made for this GPU; any other number of SMs works
inline long long div_up(long long a, long long b) { return (a + b - 1) / b; }
inline int32_t cuda_status(cudaError_t e) { return e == cudaSuccess ? SAN_OK : SAN_ERR_CUDA; }
inline bool aligned(const void* p, uintptr_t n) { return ((uintptr_t)p & (n - 1)) == 0; }

// Opt-in to dynamic shared memory above 48 KB, an attribute of a kernel on a device: done once for each (`set`, one
// entry per device, belongs to the kernel).
int32_t opt_in(const void* fn, int bytes, bool* set) {
    int dev = 0;
    if (cudaGetDevice(&dev) != cudaSuccess) return SAN_ERR_CUDA;
    if (dev >= 0 && dev < 64 && set[dev]) return SAN_OK;
    if (cudaFuncSetAttribute(fn, cudaFuncAttributeMaxDynamicSharedMemorySize, bytes) != cudaSuccess) return SAN_ERR_CUDA;
    if (dev >= 0 && dev < 64) set[dev] = true;
    return SAN_OK;
}

// Launches `fn` so that its CTAs may be set up while the kernel before it on the stream still runs
// (it waits with griddepcontrol.wait before it reads what that one wrote).
template <typename P>
int32_t launch_after(void (*fn)(P), dim3 grid, unsigned block, cudaStream_t st, const P& p, size_t smem = 0) {
    cudaLaunchConfig_t cfg = {};
    cfg.gridDim = grid; cfg.blockDim = dim3(block); cfg.dynamicSmemBytes = smem; cfg.stream = st;
    cudaLaunchAttribute attr;
    attr.id = cudaLaunchAttributeProgrammaticStreamSerialization;
    attr.val.programmaticStreamSerializationAllowed = 1;
    cfg.attrs = &attr; cfg.numAttrs = 1;
    return cuda_status(cudaLaunchKernelEx(&cfg, fn, p));
}

// ------------------------------------------------------------------------------- beam selection
// Steps of 8 words where that makes one wave of two (see san_select.cuh).  Parts of a row, each of whole steps: the cut with the
// shortest estimate of (waves of CTAs) x (steps of a part + the 2.5 steps that the bound, the list and the hand-over of a part take).
struct SelectCut { int words, chunks, steps; };
constexpr int kSelectParts = 64;            // of a row at most
long long select_most_parts(int vocab) {    // with the shortest steps
    return std::min<long long>(kSelectParts, div_up(vocab, kSelWordsShort * kSelThreads));
}
SelectCut select_cut(int32_t dtype, long long rows, int vocab) {
    const bool f32 = dtype == SAN_F32;
    const int words = f32 && rows > kSms * select_ctas(kSelWordsLong) && rows <= kSms * select_ctas(kSelWordsShort) ? kSelWordsShort : kSelWordsLong;
    const int step = (f32 ? words : 2 * words) * kSelThreads, ctas = kSms * select_ctas(words);
    const long long all = div_up(vocab, step);
    SelectCut best{words, 1, (int)all};
    double least = 1e30;
    for (long long parts = 1; parts <= std::min<long long>(all, kSelectParts); ++parts) {
        const long long steps = div_up(all, parts), chunks = div_up(all, steps);
        const double cost = (double)std::max<long long>(1, div_up(rows * chunks, ctas)) * ((double)steps + 2.5);
        if (cost < least) { least = cost; best = {words, (int)chunks, (int)steps}; }
    }
    return best;
}

int32_t select_shape(int32_t n_sent, int32_t beam, int32_t vocab) {
    if (n_sent < 0 || beam < 1 || beam > SAN_MAX_BEAM || vocab < 1 || vocab > (1 << 28)) return SAN_ERR_SHAPE;
    if ((long long)n_sent * beam > (1 << 24)) return SAN_ERR_SHAPE;
    if ((long long)n_sent * beam * select_most_parts(vocab) > 0x7fffffffLL) return SAN_ERR_SHAPE;
    return SAN_OK;
}

template <typename T, bool VECTOR, int W>
int32_t launch_select_as(const SelectParams& p, cudaStream_t st) {
    const unsigned grid = (unsigned)((long long)p.n_sent * p.beam * p.chunks);
    select_rows_kernel<T, VECTOR, W><<<grid, kSelThreads, 0, st>>>(p);
    if (cudaGetLastError() != cudaSuccess) return SAN_ERR_CUDA;
    return launch_after(&select_merge_kernel, dim3((unsigned)p.n_sent), kSelThreads, st, p);
}
template <typename T, int W>
int32_t launch_select(const SelectParams& p, bool vector, cudaStream_t st) {
    return vector ? launch_select_as<T, true, W>(p, st) : launch_select_as<T, false, W>(p, st);
}

// ------------------------------------------------------------------------------- step attention
int32_t check_rows(const san_cached_rows* r) {
    if (!r) return SAN_ERR_NULL;
    if (r->dtype != SAN_F32 && r->dtype != SAN_BF16) return SAN_ERR_DTYPE;
    if (r->n_heads < 1 || r->n_heads > 1024 || r->n_kv_heads < 1 || r->n_heads % r->n_kv_heads != 0) return SAN_ERR_SHAPE;
    if (r->n_layers < 1 || r->n_layers > SAN_MAX_LAYERS) return SAN_ERR_SHAPE;
    if (r->max_ids < 1 || r->cap_len < 1 || r->cap_len > (1 << 28)) return SAN_ERR_SHAPE;
    if (r->n_items < 0 || r->n_items > (1 << 24)) return SAN_ERR_SHAPE;
    if (r->max_len < 0 || r->max_len > r->cap_len) return SAN_ERR_SHAPE;
    if (r->n_layers > 1 && (r->v_stride < 1 || r->v_stride % kDh != 0)) return SAN_ERR_SHAPE;
    return SAN_OK;
}
int32_t check_prefix(const san_cached_rows* r, const san_shared_prefix* x) {
    if (!x) return SAN_ERR_NULL;
    if (x->n_prefix < 0 || x->n_prefix > (1 << 24) || x->cap_len < 1 || x->cap_len > (1 << 28)) return SAN_ERR_SHAPE;
    if (x->max_len < 0 || x->max_len > x->cap_len || x->max_group < 0 || x->max_group > r->n_items) return SAN_ERR_SHAPE;
    if (r->n_layers > 1 && (x->v_stride < 1 || x->v_stride % kDh != 0)) return SAN_ERR_SHAPE;
    return SAN_OK;
}

constexpr int kOwnLeast = 4;                // tiles of own rows that are not cut
// How one kind of units (`units` runs of up to `tiles` tiles) is cut where a warp's share of the whole call is
// `share` tiles: warps per unit and runs of tiles.  A run of no more than 1.25 shares (or `least` tiles) is one warp's.  A longer
// one is cut into up to four runs for a warp each, so that the warps finish together; beyond that the four
// warps of a CTA take a run together, which leaves a quarter of the partial results.  Measured (device time): 32 prefixes of 16
// tiles beside 1024 rows of up to 8, share 10: 48.6 us uncut, 35.9 in two runs each; 1024 runs of 17 tiles, share 15: 53.4 us
// uncut, 58.7 by four warps each; 8 runs of 513 tiles: 13.0 us by four warps, 17.7 by one.
// `least`: tiles below which a cut costs more than it gives (a float32 tile of eight rows is several bf16 ones' work).
void cut_runs(int tiles, double share, int least, int* wpu, int* splits, int* span) {
    const int most = std::max(least, (int)std::ceil(1.25 * share));
    const int pieces = (int)div_up(tiles, most);
    *wpu = pieces > 4 ? kAtWarps : 1;
    *splits = pieces > 4 ? (int)div_up(pieces, kAtWarps) : pieces;
    *span = (int)div_up(tiles, *splits);
    *splits = (int)div_up(tiles, *span);
}

struct AttendPlan { AttendParams p; size_t ml_bytes, bytes; long long ctas, tiles, tiles_own; };

// Workspace of `rows` partial results: (max, sum) and the layers' outputs of each.
size_t partial_ml_bytes(size_t rows) { return (rows * sizeof(float2) + 255) / 256 * 256; }
size_t partial_bytes(size_t rows, int layers) { return partial_ml_bytes(rows) + rows * layers * kDh * sizeof(float); }

// Everything but the addresses.  Rows are cut into no more runs than find room in `room` bytes of workspace (a prefix's result and
// its row's own one always stay two): a workspace made for a larger batch, which needs fewer runs, serves a smaller one.
int32_t plan_attend(const san_cached_rows* r, const san_shared_prefix* x, int window, int n_sink, size_t room, AttendPlan* out) {
    std::memset(out, 0, sizeof(*out));
    AttendParams& p = out->p;
    const int R = kAtRows;
    const long long e = r->dtype == SAN_BF16 ? 2 : 4;
    p.H = r->n_heads; p.Hk = r->n_kv_heads; p.group = r->n_heads / r->n_kv_heads;
    p.n_layers = r->n_layers; p.n_items = r->n_items;
    p.max_ids = r->max_ids; p.cap = r->cap_len; p.max_len = r->max_len ? r->max_len : r->cap_len;
    p.window = window; p.n_sink = n_sink;
    p.v_stride = r->v_stride * e;
    p.n_lg = (int)div_up(r->n_layers, kAtMaxLayers);
    p.lg = (int)div_up(r->n_layers, p.n_lg);
    p.n_lg = (int)div_up(r->n_layers, p.lg);
    long long p_runs = 0, p_tiles = 0;          // runs of a prefix's rows before they are cut, and tiles (chunks of 64) of one
    if (x && x->n_prefix > 0) {
        p.n_prefix = x->n_prefix; p.pcap = x->cap_len; p.pv_stride = x->v_stride * e;
        p.max_prefix = x->max_len ? x->max_len : x->cap_len;
        p.max_group = x->max_group ? x->max_group : std::max(1, r->n_items);
        // Prefixes go to the tensor-core tiles where that is estimated to be faster.  Both measured: the streams of
        // eight query rows get through 2900 slots (32 positions of one plane) a microsecond, the tiles through
        // a chunk of 64 positions for 256 rows and up to two layers per SM and microsecond, after 9 us of set-up
        // and hand-over.
        const long long rows = (long long)p.max_group * p.group, tile_runs = (long long)p.n_prefix * p.Hk * div_up(rows, 2 * kTileQ) * div_up(r->n_layers, kTileMaxLayers);
        const double streams_us = (double)p.n_prefix * p.Hk * div_up(rows, R) * div_up(p.max_prefix, kAtTile) * (p.n_layers + p.n_lg) / 2900.0;
        const double tiles_us = (double)div_up(tile_runs * div_up(p.max_prefix, kTileK), kSms) + 9.0;
        if (r->dtype == SAN_BF16 && tiles_us < streams_us) {
            p.t_n_lg = (int)div_up(r->n_layers, kTileMaxLayers);
            p.t_lg = (int)div_up(r->n_layers, p.t_n_lg);
            p.t_n_lg = (int)div_up(r->n_layers, p.t_lg);
            p.p_row_tiles = (int)div_up(rows, 2 * kTileQ);
            // runs of chunks: as many as fill the SMs once, of four chunks or more
            const long long units = (long long)p.n_prefix * p.p_row_tiles * p.Hk * p.t_n_lg;
            p_tiles = div_up(p.max_prefix, kTileK);
            const long long want = std::max<long long>(1, std::min<long long>(kSms / std::max<long long>(units, 1), div_up(p_tiles, 4)));
            p.p_span = (int)div_up(p_tiles, want);
            p.p_splits = (int)div_up(p_tiles, p.p_span);
        }
    }
    p.o_row_tiles = (int)div_up(p.group, R);
    const long long bound = window > 0 ? std::min<long long>(p.max_len, (long long)window + n_sink) : p.max_len;
    const long long o_runs = (long long)r->n_items * p.o_row_tiles * p.Hk * p.n_lg, o_tiles = std::max<long long>(1, div_up(bound, kAtTile));
    if (p.n_prefix > 0 && p.t_lg == 0) {
        p.p_row_tiles = (int)div_up((long long)p.max_group * p.group, R);
        p_runs = (long long)p.n_prefix * p.p_row_tiles * p.Hk * p.n_lg;
        p_tiles = div_up(p.max_prefix, kAtTile);
    }
    out->tiles_own = o_tiles;
    const double share = ((double)o_runs * o_tiles + (double)p_runs * (p.t_lg ? 0 : p_tiles)) / ((double)kSms * 2 * kAtWarps);
    if (p_runs > 0) cut_runs((int)p_tiles, share, e == 4 ? 2 : 4, &p.p_wpu, &p.p_splits, &p.p_span);
    cut_runs((int)o_tiles, share, kOwnLeast, &p.o_wpu, &p.o_splits, &p.o_span);
    const size_t rows = (size_t)r->n_items * r->n_heads;
    if (rows > 0x7fffffff) return SAN_ERR_SHAPE;
    if (p.p_splits + p.o_splits > 1 && partial_bytes((p.p_splits + p.o_splits) * rows, r->n_layers) > room) {
        const int least = p.p_splits > 0 ? 2 : 1, all = p.p_splits + p.o_splits;
        int most = (int)std::max<size_t>(least, std::min<size_t>(all - 1, room / partial_bytes(rows, r->n_layers) + 1));
        while (most > least && partial_bytes(most * rows, r->n_layers) > room) --most;
        const int own = least == 1 ? most : std::max(1, (int)((long long)most * p.o_splits / all));
        p.o_span = (int)div_up(o_tiles, own);
        p.o_splits = (int)div_up(o_tiles, p.o_span);
        if (least > 1) {
            p.p_span = (int)div_up(p_tiles, most - own);
            p.p_splits = (int)div_up(p_tiles, p.p_span);
        }
    }
    if (p.t_lg > 0) {
        out->tiles = (long long)p.n_prefix * p.p_row_tiles * p.Hk * p.t_n_lg * p.p_splits;
        if (out->tiles > 0x7fffffffLL) return SAN_ERR_SHAPE;
    } else if (p_runs > 0) {
        if (p_runs * p.p_splits > 0x7fffffffLL) return SAN_ERR_SHAPE;
        p.p_units = (int)(p_runs * p.p_splits);
        p.p_ctas = (int)div_up(p.p_units, kAtWarps / p.p_wpu);
    }
    if (o_runs * p.o_splits > 0x7fffffffLL) return SAN_ERR_SHAPE;
    p.o_units = (int)(o_runs * p.o_splits);
    p.slots = p.p_splits + p.o_splits;
    if (p.slots > 1) {
        out->ml_bytes = partial_ml_bytes(p.slots * rows);
        out->bytes = partial_bytes(p.slots * rows, r->n_layers);
    }
    out->ctas = p.p_ctas + div_up(p.o_units, kAtWarps / p.o_wpu);
    if (out->ctas > 0x7fffffffLL) return SAN_ERR_SHAPE;
    p.scale_log2e = (float)(1.4426950408889634 / std::sqrt((double)kDh));
    return SAN_OK;
}

template <typename T, int LG, int N>
int32_t launch_attend_as(const AttendPlan& a, cudaStream_t st) {
    constexpr int smem = attend_smem_bytes<T, N>();
    static bool set[64] = {};
    const int32_t rc = opt_in((const void*)attend_kernel<T, LG, N>, smem, set);
    if (rc != SAN_OK) return rc;
    if (a.tiles > 0) {                              // beside the tiles, which it does not depend on
        const int32_t rc2 = launch_after(&attend_kernel<T, LG, N>, dim3((unsigned)a.ctas), kAtWarps * 32, st, a.p, smem);
        if (rc2 != SAN_OK) return rc2;
    } else {
        attend_kernel<T, LG, N><<<(unsigned)a.ctas, kAtWarps * 32, smem, st>>>(a.p);
        if (cudaGetLastError() != cudaSuccess) return SAN_ERR_CUDA;
    }
    if (a.p.slots == 1) return SAN_OK;
    const long long rows = (long long)a.p.n_items * a.p.H;
    const int groups = a.p.slots <= 6 ? 1 : a.p.slots <= 12 ? 4 : 16;
    const dim3 grid((unsigned)div_up(rows, 16 / groups), (unsigned)a.p.n_layers);
    return launch_after(groups == 1 ? &attend_join_kernel<T, 1> : groups == 4 ? &attend_join_kernel<T, 4> : &attend_join_kernel<T, 16>,
                        grid, 256, st, a.p);
}
// Slots of a warp's ring: what fits the shared memory of an SM (14 slots of a CTA's four warps) with the CTAs that it
// will hold; a warp's chain of slots is the faster the more of them are on their way.
template <typename T, int LG>
int32_t launch_attend_with(const AttendPlan& a, cudaStream_t st) {
    if constexpr (sizeof(T) == 4) return launch_attend_as<T, LG, 3>(a, st);
    else return a.ctas <= 2 * kSms ? launch_attend_as<T, LG, 6>(a, st) : a.ctas <= 3 * kSms ? launch_attend_as<T, LG, 4>(a, st) : launch_attend_as<T, LG, 3>(a, st);
}
template <class Mode, int LG, class P>
int32_t launch_tiles(const P& p, dim3 grid, cudaStream_t st) {
    constexpr int smem = tile_smem_bytes(LG);
    static bool set[64] = {};
    const int32_t rc = opt_in((const void*)tile_kernel<Mode, LG, P>, smem, set);
    if (rc != SAN_OK) return rc;
    tile_kernel<Mode, LG, P><<<grid, kTileThreads, smem, st>>>(p);
    return cuda_status(cudaGetLastError());
}

template <typename T>
int32_t launch_attend(const AttendPlan& a, cudaStream_t st) {
    if (a.tiles > 0) {
        const dim3 grid((unsigned)a.tiles);
        const int32_t rc = a.p.t_lg == 1 ? launch_tiles<TilePrefix, 1>(a.p, grid, st) : launch_tiles<TilePrefix, 2>(a.p, grid, st);
        if (rc != SAN_OK) return rc;
    }
    return a.p.lg == 1 ? launch_attend_with<T, 1>(a, st) : a.p.lg == 2 ? launch_attend_with<T, 2>(a, st) : launch_attend_with<T, 4>(a, st);
}

int32_t run_attend(const san_cached_rows* r, const san_shared_prefix* x, int window, int n_sink, void* ws, size_t ws_bytes, void* stream) {
    AttendPlan a;
    int32_t rc = plan_attend(r, x, window, n_sink, ws_bytes, &a);
    if (rc != SAN_OK) return rc;
    if (r->n_items == 0) return SAN_OK;
    if (!r->d_q || !r->d_k || !r->d_v || !r->d_ids || !r->d_lens || !r->d_out) return SAN_ERR_NULL;
    if (!aligned(r->d_q, 16) || !aligned(r->d_k, 16) || !aligned(r->d_v, 16) || !aligned(r->d_out, 16)) return SAN_ERR_SHAPE;
    if (x && x->n_prefix > 0) {
        if (!x->d_k || !x->d_v || !x->d_lens || !x->d_first) return SAN_ERR_NULL;
        if (!aligned(x->d_k, 16) || !aligned(x->d_v, 16)) return SAN_ERR_SHAPE;
        a.p.pk = static_cast<const char*>(x->d_k); a.p.pv = static_cast<const char*>(x->d_v);
        a.p.plens = x->d_lens; a.p.first = x->d_first;
    }
    if (a.bytes > 0) {
        if (!ws) return SAN_ERR_NULL;
        if (!aligned(ws, 256)) return SAN_ERR_SHAPE;
        if (ws_bytes < a.bytes) return SAN_ERR_CAPACITY;
    }
    a.p.q = static_cast<const char*>(r->d_q); a.p.out = static_cast<char*>(r->d_out);
    a.p.k = static_cast<const char*>(r->d_k); a.p.v = static_cast<const char*>(r->d_v);
    a.p.ids = r->d_ids; a.p.lens = r->d_lens; a.p.status = r->d_status;
    a.p.part_ml = static_cast<float2*>(ws);
    a.p.part_o = reinterpret_cast<float*>(static_cast<char*>(ws) + a.ml_bytes);
    cudaStream_t st = static_cast<cudaStream_t>(stream);
    return r->dtype == SAN_BF16 ? launch_attend<__nv_bfloat16>(a, st) : launch_attend<float>(a, st);
}

template <int LG>
int32_t launch_window(const WindowParams& p, dim3 grid, cudaStream_t st) {
    window_block_kernel<LG><<<grid, 128, 0, st>>>(p);
    return cuda_status(cudaGetLastError());
}

}  // namespace

extern "C" {

int32_t san_beam_select_bytes(int32_t n_sent, int32_t beam, int32_t vocab, size_t* workspace_bytes) {
    if (!workspace_bytes) return SAN_ERR_NULL;
    const int32_t rc = select_shape(n_sent, beam, vocab);
    if (rc != SAN_OK) return rc;
    // As many parts as a row can be cut into, not as many as this call's rows are: fewer sentences are cut into more.
    *workspace_bytes = (size_t)n_sent * beam * select_most_parts(vocab) * select_part_bytes(beam);
    return SAN_OK;
}

int32_t san_beam_select(const san_select_args* a, void* stream) {
    if (!a) return SAN_ERR_NULL;
    if (a->dtype != SAN_F32 && a->dtype != SAN_BF16) return SAN_ERR_DTYPE;
    const int32_t rc = select_shape(a->n_sent, a->beam, a->vocab);
    if (rc != SAN_OK) return rc;
    if (a->ld_logits < a->vocab || a->eos < -1 || a->eos >= a->vocab || !std::isfinite(a->alpha)) return SAN_ERR_SHAPE;
    if (a->n_sent == 0) return SAN_OK;
    if (!a->d_logits || !a->d_score || !a->d_len || !a->d_done || !a->d_score_out || !a->d_len_out || !a->d_done_out ||
        !a->d_parent || !a->d_next || !a->d_workspace) return SAN_ERR_NULL;
    if ((a->d_tokens == nullptr) != (a->d_tokens_out == nullptr)) return SAN_ERR_NULL;
    if (a->d_tokens && (a->ld_tokens < 1 || a->ld_tokens > kSelMaxTokens)) return SAN_ERR_SHAPE;
    const size_t e = a->dtype == SAN_F32 ? 4 : 2;
    if (!aligned(a->d_logits, e) || !aligned(a->d_workspace, 256)) return SAN_ERR_SHAPE;
    const long long rows = (long long)a->n_sent * a->beam;
    const SelectCut cut = select_cut(a->dtype, rows, a->vocab);
    if (a->workspace_bytes < (size_t)rows * cut.chunks * select_part_bytes(a->beam)) return SAN_ERR_CAPACITY;
    SelectParams p;
    std::memset(&p, 0, sizeof(p));
    p.logits = a->d_logits; p.ld = a->ld_logits; p.vocab = a->vocab; p.n_sent = a->n_sent; p.beam = a->beam;
    p.chunks = cut.chunks; p.steps = cut.steps;
    p.eos = a->eos; p.alpha = (double)a->alpha;
    p.score = a->d_score; p.len = a->d_len; p.done = a->d_done; p.tokens = a->d_tokens; p.ld_tokens = a->ld_tokens;
    p.score_out = a->d_score_out; p.len_out = a->d_len_out; p.done_out = a->d_done_out; p.tokens_out = a->d_tokens_out;
    p.parent = a->d_parent; p.next = a->d_next; p.ws = static_cast<char*>(a->d_workspace); p.status = a->d_status;
    const bool vector = aligned(a->d_logits, 16) && a->ld_logits * (int64_t)e % 16 == 0;
    cudaStream_t st = static_cast<cudaStream_t>(stream);
    if (a->dtype == SAN_BF16) return launch_select<__nv_bfloat16, kSelWordsLong>(p, vector, st);
    return cut.words == kSelWordsShort ? launch_select<float, kSelWordsShort>(p, vector, st) : launch_select<float, kSelWordsLong>(p, vector, st);
}

int32_t san_cache_planes(const san_ctx* ctx, int32_t kind, int32_t block, void** d_k, void** d_v, int64_t* v_stride) {
    if (!ctx || !d_k || !d_v || !v_stride) return SAN_ERR_NULL;
    if (kind != SAN_SELF && kind != SAN_ENCDEC) return SAN_ERR_RANGE;
    const bool self = kind == SAN_SELF;
    if (self && ctx->cfg.self_is_aan) return SAN_ERR_UNSUPPORTED;
    const Policy& pol = self ? ctx->self_pol : ctx->enc_pol;
    if (block < 0 || block >= pol.n_blocks) return SAN_ERR_RANGE;
    const size_t plane = self ? ctx->self_plane_bytes : ctx->mem_plane_bytes;
    const size_t v_plane = !self && ctx->cfg.encdec_shared_context ? (size_t)block : (size_t)pol.first_layer_of_block[block];
    *d_k = ctx->cache + (self ? ctx->off_self_k : ctx->off_mem_k) + (size_t)block * plane;
    *d_v = ctx->cache + (self ? ctx->off_self_v : ctx->off_mem_v) + v_plane * plane;
    // One plane for the whole block: no distance that a call over several layers would take.
    *v_stride = !self && ctx->cfg.encdec_shared_context ? 0 : (int64_t)(plane / (size_t)ctx->elem_bytes);
    return SAN_OK;
}

int32_t san_window_attn_bytes(const san_cached_rows* rows, int32_t window, int32_t n_sink, size_t* workspace_bytes) {
    if (!workspace_bytes) return SAN_ERR_NULL;
    int32_t rc = check_rows(rows);
    if (rc != SAN_OK) return rc;
    if (window < 1 || n_sink < 0) return SAN_ERR_SHAPE;
    AttendPlan a;
    if ((rc = plan_attend(rows, nullptr, window, n_sink, SIZE_MAX, &a)) != SAN_OK) return rc;
    // What any smaller batch or bound needs as well.  n items of c runs and t tiles each have a share of n c t / W tiles a warp (W
    // warps), so that a run is at most ceil(W / (1.25 n c)) pieces and all items together at most W / (1.25 c) + n.
    const long long pieces = div_up(a.tiles_own, kOwnLeast), n = rows->n_items, c = (long long)a.p.o_row_tiles * a.p.Hk * a.p.n_lg;
    const long long most = std::max(std::min<long long>(pieces, 4), div_up(pieces, kAtWarps));
    const long long partial = std::min(n * most, n + div_up(kSms * 2 * kAtWarps * 4 / 5 + 1, c));
    *workspace_bytes = most > 1 ? partial_bytes((size_t)partial * rows->n_heads, rows->n_layers) : 0;
    return SAN_OK;
}

int32_t san_window_attn(const san_cached_rows* rows, int32_t window, int32_t n_sink, void* d_workspace, size_t workspace_bytes,
                        void* stream) {
    const int32_t rc = check_rows(rows);
    if (rc != SAN_OK) return rc;
    if (window < 1 || n_sink < 0) return SAN_ERR_SHAPE;
    return run_attend(rows, nullptr, window, n_sink, d_workspace, workspace_bytes, stream);
}

int32_t san_prefix_attn_bytes(const san_cached_rows* rows, const san_shared_prefix* prefix, size_t* workspace_bytes) {
    if (!workspace_bytes) return SAN_ERR_NULL;
    int32_t rc = check_rows(rows);
    if (rc == SAN_OK) rc = check_prefix(rows, prefix);
    if (rc != SAN_OK) return rc;
    AttendPlan a;
    if ((rc = plan_attend(rows, prefix, 0, 0, SIZE_MAX, &a)) != SAN_OK) return rc;
    *workspace_bytes = a.bytes;
    return SAN_OK;
}

int32_t san_prefix_attn(const san_cached_rows* rows, const san_shared_prefix* prefix, void* d_workspace, size_t workspace_bytes,
                        void* stream) {
    int32_t rc = check_rows(rows);
    if (rc == SAN_OK) rc = check_prefix(rows, prefix);
    if (rc != SAN_OK) return rc;
    return run_attend(rows, prefix, 0, 0, d_workspace, workspace_bytes, stream);
}

int32_t san_window_block(int32_t dtype, int32_t n_heads, int32_t n_kv_heads, int32_t n_layers, int32_t window, int32_t n_sink,
                         const void* d_q, const void* d_k, const void* d_v, const int32_t* d_lens, int32_t n_seq, int32_t cap_len,
                         int32_t max_len, void* d_out, void* stream) {
    if (dtype != SAN_BF16) return dtype == SAN_F32 ? SAN_ERR_UNSUPPORTED : SAN_ERR_DTYPE;
    if (n_heads < 1 || n_heads > 65535 || n_kv_heads < 1 || n_heads % n_kv_heads != 0) return SAN_ERR_SHAPE;
    if (n_layers < 1 || n_layers > SAN_MAX_LAYERS || window < 1 || n_sink < 0) return SAN_ERR_SHAPE;
    if (n_seq < 0 || cap_len < 1 || cap_len > (1 << 28) || max_len < 0 || max_len > cap_len) return SAN_ERR_SHAPE;
    if (n_seq == 0) return SAN_OK;
    if (!d_q || !d_k || !d_v || !d_lens || !d_out) return SAN_ERR_NULL;
    if (!aligned(d_q, 16) || !aligned(d_k, 16) || !aligned(d_v, 16) || !aligned(d_out, 16)) return SAN_ERR_SHAPE;
    if (max_len == 0) max_len = cap_len;
    // No row has more rows before it than that: what "all of them" is written as (2^31 - 1, say) does not reach the index
    // arithmetic of the kernels, which adds to both.
    window = std::min(window, max_len);
    n_sink = std::min(n_sink, max_len);
    WindowParams p;
    std::memset(&p, 0, sizeof(p));
    p.q = static_cast<const __nv_bfloat16*>(d_q); p.k = static_cast<const __nv_bfloat16*>(d_k);
    p.v = static_cast<const __nv_bfloat16*>(d_v); p.out = static_cast<__nv_bfloat16*>(d_out);
    p.lens = d_lens; p.n_seq = n_seq; p.cap = cap_len; p.H = n_heads; p.Hk = n_kv_heads; p.group = n_heads / n_kv_heads;
    p.n_layers = n_layers; p.max_len = max_len; p.window = window; p.n_sink = n_sink;
    p.v_layer = (long long)n_seq * cap_len * n_kv_heads * kDh;
    p.out_layer = (long long)n_seq * cap_len * n_heads * kDh;
    // The tensor-core tiles take sequences of a tile and more, unless the rows that a CTA of window_block_kernel walks are
    // one slot of its ring.  Measured, tiles and window_block_kernel: 4 x 4096 positions, 8 heads, 4 sinks, window 4: 32.4 and
    // 24.4 us, 32: 32.2 and 31.8, 96: 35.9 and 43.3; 4 layers and window 4: 65.3 and 47.7.
    const bool use_tiles = max_len >= kTileQ && (long long)window + n_sink + kWinQ - 1 > kWinTile;
    const int at_once = use_tiles ? kTileMaxLayers : 4;
    p.n_lg = (int)div_up(n_layers, at_once);
    p.lg = (int)div_up(n_layers, p.n_lg);
    p.n_lg = (int)div_up(n_layers, p.lg);
    p.scale_log2e = (float)(1.4426950408889634 / std::sqrt((double)kDh));
    if ((long long)n_seq * p.n_lg > 65535) return SAN_ERR_SHAPE;
    if (use_tiles) {
        // A CTA takes a pair of tiles.  Where the last wave would hold less than half of the SMs' CTAs, its pairs are dealt as
        // single tiles, which take about two thirds of a pair's time: 7805 positions x 16 sequences and heads are 31 x 16 = 496
        // pairs, 3.35 waves, or three waves of pairs and 104 single tiles.
        const long long pairs = div_up(max_len, 2 * kTileQ), all = pairs * n_heads * n_seq * p.n_lg, rest = all % kSms;
        if (2 * all > 0x7fffffffLL) return SAN_ERR_SHAPE;
        p.pairs = (int)pairs;
        p.whole = (int)(2 * rest <= kSms ? all - rest : all);
        const dim3 tiles((unsigned)(2 * all - p.whole));
        cudaStream_t st = static_cast<cudaStream_t>(stream);
        return p.lg == 1 ? launch_tiles<TileWindow, 1>(p, tiles, st) : launch_tiles<TileWindow, 2>(p, tiles, st);
    }
    const dim3 grid((unsigned)div_up(max_len, kWinQ), (unsigned)n_heads, (unsigned)(n_seq * p.n_lg));
    cudaStream_t st = static_cast<cudaStream_t>(stream);
    return p.lg == 1 ? launch_window<1>(p, grid, st) : p.lg == 2 ? launch_window<2>(p, grid, st) : p.lg == 3 ? launch_window<3>(p, grid, st) : launch_window<4>(p, grid, st);
}

}  // extern "C"
