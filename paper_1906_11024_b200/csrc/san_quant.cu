// Host side of the calls for a cache that is kept small: rows in four bits, step attention over them, the mass of cached rows,
// eviction.  Argument checks and how the work is cut; the arithmetic is in san_quant.cuh and san_evict.cuh.
#include "san_launch.cuh"
#include "san_quant.cuh"
#include "san_evict.cuh"

using namespace san;

namespace {

int32_t check_planes(const san_planes* c, bool quant) {
    if (!c) return SAN_ERR_NULL;
    if (c->dtype != SAN_F32 && c->dtype != SAN_BF16 && c->dtype != SAN_Q4) return SAN_ERR_DTYPE;
    if (quant && c->dtype != SAN_Q4) return SAN_ERR_DTYPE;
    if (c->n_kv_heads < 1 || c->n_kv_heads > 1024 || c->n_layers < 1 || c->n_layers > SAN_MAX_LAYERS) return SAN_ERR_SHAPE;
    if (c->max_ids < 1 || c->cap_len < 1 || c->cap_len > (1 << 28)) return SAN_ERR_SHAPE;
    if (c->n_layers > 1 && (c->v_stride < 1 || c->v_stride % kDh != 0)) return SAN_ERR_SHAPE;
    return SAN_OK;
}
int32_t check_plane_pointers(const san_planes* c) {
    if (!c->d_k || !c->d_v) return SAN_ERR_NULL;
    if (!aligned(c->d_k, 16) || !aligned(c->d_v, 16)) return SAN_ERR_SHAPE;
    if (c->dtype != SAN_Q4) return SAN_OK;
    if (!c->d_k_scale || !c->d_v_scale) return SAN_ERR_NULL;
    return aligned(c->d_k_scale, 4) && aligned(c->d_v_scale, 4) ? SAN_OK : SAN_ERR_SHAPE;
}

int32_t quant_rows(bool append, const san_planes* c, int32_t dtype, const void* k, const void* v, const int32_t* ids, const int32_t* pos,
                   const int32_t* nrows, int32_t n_items, int32_t rows, int32_t* status, void* stream) {
    int32_t rc = check_planes(c, true);
    if (rc != SAN_OK) return rc;
    if (dtype != SAN_F32 && dtype != SAN_BF16) return SAN_ERR_DTYPE;
    if (n_items < 0 || rows < 1 || (!nrows && rows > c->cap_len)) return SAN_ERR_SHAPE;
    if (n_items == 0) return SAN_OK;
    if ((rc = check_plane_pointers(c)) != SAN_OK) return rc;
    if (!k || !v || !ids) return SAN_ERR_NULL;
    if (!aligned(k, 16) || !aligned(v, 16)) return SAN_ERR_SHAPE;
    const long long all = (long long)(1 + c->n_layers) * c->n_kv_heads * n_items;
    if (all > 0x7fffffffLL / rows) return SAN_ERR_SHAPE;
    QuantRowsParams p;
    std::memset(&p, 0, sizeof(p));
    p.k = static_cast<char*>(c->d_k); p.v = static_cast<char*>(c->d_v);
    p.ks = static_cast<char*>(c->d_k_scale); p.vs = static_cast<char*>(c->d_v_scale);
    p.v_stride = c->v_stride / kDh * kQuantRow; p.s_stride = c->v_stride / kDh * 4;
    p.k_rows = static_cast<const char*>(k); p.v_rows = static_cast<const char*>(v);
    p.ids = ids; p.pos = pos; p.nrows = nrows; p.n_items = n_items; p.rows = rows; p.Hk = c->n_kv_heads; p.n_layers = c->n_layers;
    p.max_ids = c->max_ids; p.cap = c->cap_len; p.status = status;
    p.all_rows = (uint32_t)(all * rows); p.layer_rows = (long long)n_items * rows * p.Hk * kDh;
    p.by_rows.by((uint32_t)rows); p.by_heads.by((uint32_t)p.Hk); p.by_items.by((uint32_t)n_items);
    const unsigned grid = (unsigned)div_up(all * rows, kQuantCtaRows);
    cudaStream_t st = static_cast<cudaStream_t>(stream);
    if (append) {
        if (dtype == SAN_BF16) quant_append_kernel<__nv_bfloat16><<<grid, 256, 0, st>>>(p);
        else quant_append_kernel<float><<<grid, 256, 0, st>>>(p);
    } else {
        if (dtype == SAN_BF16) quant_read_kernel<__nv_bfloat16><<<grid, 256, 0, st>>>(p);
        else quant_read_kernel<float><<<grid, 256, 0, st>>>(p);
    }
    return cuda_status(cudaGetLastError());
}

// ------------------------------------------------------------------------------- step attention
constexpr int kQuantCtas = kSms * 4;                 // on the GPU at once, or nearly
constexpr int kQuantStep = 4;                        // tiles of a step (four warps)
constexpr int kQuantFills = 6, kQuantSteps = 3;      // see plan_quant
struct QuantPlan { QuantParams p; size_t ml_bytes, bytes; long long ctas, tiles; };

// Everything but the addresses.  Rows are cut into no more runs than find room in `room` bytes of workspace: one made for a larger batch,
// which needs fewer runs, serves a smaller one.
int32_t plan_quant(const san_planes* c, const san_step_rows* r, size_t room, QuantPlan* out) {
    int32_t rc = check_planes(c, true);
    if (rc != SAN_OK) return rc;
    if (!r) return SAN_ERR_NULL;
    if (r->dtype != SAN_F32 && r->dtype != SAN_BF16) return SAN_ERR_DTYPE;
    if (r->n_heads < 1 || r->n_heads > 1024 || r->n_heads % c->n_kv_heads != 0) return SAN_ERR_SHAPE;
    if (r->n_items < 0 || r->n_items > (1 << 24) || r->max_len < 0 || r->max_len > c->cap_len) return SAN_ERR_SHAPE;
    std::memset(out, 0, sizeof(*out));
    AttendParams& p = out->p.a;
    p.H = r->n_heads; p.Hk = c->n_kv_heads; p.group = p.H / p.Hk;
    p.n_layers = c->n_layers; p.n_items = r->n_items;
    p.max_ids = c->max_ids; p.cap = c->cap_len; p.max_len = r->max_len ? r->max_len : c->cap_len;
    if (r->d_S && r->ld_s < p.max_len) return SAN_ERR_SHAPE;
    p.v_stride = c->v_stride / kDh * kQuantRow;
    out->p.s_stride = c->v_stride / kDh * 4;
    p.n_lg = (int)div_up(p.n_layers, kAtMaxLayers);
    p.lg = (int)div_up(p.n_layers, p.n_lg);
    p.n_lg = (int)div_up(p.n_layers, p.lg);
    p.o_row_tiles = (int)div_up(p.group, kAtRows);
    const long long runs = (long long)r->n_items * p.o_row_tiles * p.Hk * p.n_lg, tiles = std::max<long long>(1, div_up(p.max_len, kQuantTile));
    // Runs of equal length, of whole steps: as many as give every SM one, and where a run keeps three steps, as many as fill the GPU six
    // times, which evens out items of different lengths.  Measured: 4 units of 500 tiles 11.8 us in 125 runs each, 11.1 in 63, 10.4 in 32 (10.0
    // by now); 1024 units of up to 64 tiles 90.5 us in 3 runs each (81.7 by now), 92.2 in 4, and one run each takes a tenth more.
    const long long units = std::max<long long>(runs, 1), even = std::min<long long>(kQuantFills * kQuantCtas / units, tiles / (kQuantSteps * kQuantStep));
    const long long pieces = std::max<long long>(1, std::min<long long>(div_up(tiles, kQuantStep), std::max<long long>(kSms / units, even)));
    p.o_span = (int)(div_up(div_up(tiles, pieces), kQuantStep) * kQuantStep);
    p.o_splits = (int)div_up(tiles, p.o_span);
    out->tiles = tiles;
    const size_t rows = (size_t)r->n_items * r->n_heads;
    if (p.o_splits > 1 && partial_bytes(p.o_splits * rows, p.n_layers) > room) {
        int most = (int)std::max<size_t>(1, std::min<size_t>(p.o_splits - 1, room / partial_bytes(rows, p.n_layers) + 1));
        while (most > 1 && partial_bytes(most * rows, p.n_layers) > room) --most;
        p.o_span = (int)div_up(tiles, most);
        p.o_splits = (int)div_up(tiles, p.o_span);
    }
    if (rows > 0x7fffffff || runs * p.o_splits > 0x7fffffffLL) return SAN_ERR_SHAPE;
    if ((long long)rows * (p.n_layers + div_up(p.max_len, kQuantWeights)) > 0x7fffffffLL) return SAN_ERR_SHAPE;
    p.o_units = (int)(runs * p.o_splits);
    p.slots = p.o_splits;
    if (p.slots > 1 || r->d_S) out->ml_bytes = partial_ml_bytes(p.slots * rows);
    out->bytes = p.slots > 1 ? partial_bytes(p.slots * rows, p.n_layers) : out->ml_bytes;
    out->ctas = p.o_units;
    p.scale_log2e = (float)(1.4426950408889634 / std::sqrt((double)kDh));
    return SAN_OK;
}

template <int LG, int P, int J>
int32_t launch_quant(const QuantPlan& a, cudaStream_t st) {
    using T = typename std::conditional<P == 1, __nv_bfloat16, float>::type;
    constexpr int smem = quant_smem_bytes<LG, J>();
    static bool set[64] = {};
    int32_t rc = opt_in((const void*)quant_attend_kernel<LG, P, J>, smem, set);
    if (rc != SAN_OK) return rc;
    quant_attend_kernel<LG, P, J><<<(unsigned)a.ctas, QuantWarps<LG>::W * 32, smem, st>>>(a.p);
    if (cudaGetLastError() != cudaSuccess) return SAN_ERR_CUDA;
    if (a.p.a.slots == 1 && !a.p.S) return SAN_OK;
    const int slots = a.p.a.slots, groups = slots <= 6 ? 1 : slots <= 12 ? 4 : 16;
    QuantParams p = a.p;
    const long long rows = (long long)p.a.n_items * p.a.H;
    p.join_ctas = slots > 1 ? (int)(div_up(rows, 16 / groups) * p.a.n_layers) : 0;
    p.parts = p.S ? (int)div_up(p.a.max_len, kQuantWeights) : 0;
    const dim3 grid((unsigned)(p.join_ctas + rows * p.parts));
    return launch_after(groups == 1 ? &quant_finish_kernel<T, 1> : groups == 4 ? &quant_finish_kernel<T, 4> : &quant_finish_kernel<T, 16>, grid, 256, st, p);
}
template <int P, int J>
int32_t launch_quant_layers(const QuantPlan& a, cudaStream_t st) {
    return a.p.a.lg == 1 ? launch_quant<1, P, J>(a, st) : a.p.a.lg == 2 ? launch_quant<2, P, J>(a, st) :
           a.p.a.lg == 3 ? launch_quant<3, P, J>(a, st) : launch_quant<4, P, J>(a, st);
}
template <int P>
int32_t launch_quant_rows(const QuantPlan& a, cudaStream_t st) {
    return a.p.a.group <= 4 ? launch_quant_layers<P, 1>(a, st) : launch_quant_layers<P, 2>(a, st);
}

template <int G, int U>
int32_t launch_mass(const MassParams& p, cudaStream_t st) {
    mass_kernel<G, U><<<dim3((unsigned)div_up(p.max_len, mass_positions<G, U>()), (unsigned)p.Hk, (unsigned)p.n_items), kMassThreads, 0, st>>>(p);
    return cuda_status(cudaGetLastError());
}

int32_t check_evict(const san_planes* c, const san_evict_args* a) {
    const int32_t rc = check_planes(c, false);
    if (rc != SAN_OK) return rc;
    if (!a) return SAN_ERR_NULL;
    if (a->n_items < 0 || a->n_items > 65535 || a->max_len < 0 || a->max_len > c->cap_len) return SAN_ERR_SHAPE;
    if (a->n_keep < 1 || a->n_keep > (1 << 26) || a->n_sink < 0 || a->n_recent < 0 || (long long)a->n_sink + a->n_recent > a->n_keep) return SAN_ERR_SHAPE;
    if (a->ld_mass < (a->max_len ? a->max_len : c->cap_len) || (a->d_kept && a->ld_kept < a->n_keep)) return SAN_ERR_SHAPE;
    return SAN_OK;
}
template <int PIECES>
int32_t launch_move(const EvictParams& p, cudaStream_t st) {
    cudaLaunchConfig_t cfg = {};
    cfg.gridDim = dim3((unsigned)((1 + p.n_layers) * p.cluster), (unsigned)p.Hk, (unsigned)p.n_items);
    cfg.blockDim = dim3(kMoveThreads); cfg.stream = st;
    cudaLaunchAttribute attr[2];
    attr[0].id = cudaLaunchAttributeProgrammaticStreamSerialization;
    attr[0].val.programmaticStreamSerializationAllowed = 1;
    attr[1].id = cudaLaunchAttributeClusterDimension;
    attr[1].val.clusterDim.x = (unsigned)p.cluster; attr[1].val.clusterDim.y = attr[1].val.clusterDim.z = 1;
    cfg.attrs = attr; cfg.numAttrs = 2;
    return cuda_status(cudaLaunchKernelEx(&cfg, evict_move_kernel<PIECES>, p));
}
size_t evict_plan_bytes(const san_planes* c, const san_evict_args* a) {
    return ((size_t)a->n_items * c->n_kv_heads * sizeof(int2) + 255) / 256 * 256;
}
size_t evict_bytes(const san_planes* c, const san_evict_args* a) {
    return evict_plan_bytes(c, a) + (size_t)a->n_items * c->n_kv_heads * a->n_keep * sizeof(int);
}

}  // namespace

extern "C" {

int32_t san_quant_append(const san_planes* cache, int32_t dtype, const void* d_k_new, const void* d_v_new, const int32_t* d_ids,
                         const int32_t* d_pos, const int32_t* d_nrows, int32_t n_items, int32_t rows_per_item, int32_t* d_status, void* stream) {
    return quant_rows(true, cache, dtype, d_k_new, d_v_new, d_ids, d_pos, d_nrows, n_items, rows_per_item, d_status, stream);
}
int32_t san_quant_read(const san_planes* cache, int32_t dtype, void* d_k, void* d_v, const int32_t* d_ids, const int32_t* d_pos,
                       const int32_t* d_nrows, int32_t n_items, int32_t rows_per_item, int32_t* d_status, void* stream) {
    return quant_rows(false, cache, dtype, d_k, d_v, d_ids, d_pos, d_nrows, n_items, rows_per_item, d_status, stream);
}

int32_t san_quant_attn_bytes(const san_planes* cache, const san_step_rows* rows, size_t* workspace_bytes) {
    if (!workspace_bytes) return SAN_ERR_NULL;
    QuantPlan a;
    const int32_t rc = plan_quant(cache, rows, SIZE_MAX, &a);
    if (rc != SAN_OK) return rc;
    // What any smaller batch or bound needs as well: n items of c units each are cut into at most 6 C / (n c) pieces (C CTAs on the GPU), so
    // that all items together have at most 6 C / c, or one each.
    const AttendParams& p = a.p.a;
    const long long n = rows->n_items, c = (long long)p.o_row_tiles * p.Hk * p.n_lg, most = div_up(a.tiles, kQuantStep);
    const long long partial = std::min(n * most, std::max(n, kQuantFills * kQuantCtas / c));
    *workspace_bytes = most > 1 ? partial_bytes((size_t)partial * p.H, p.n_layers) : rows->d_S ? partial_ml_bytes((size_t)n * p.H) : 0;
    return SAN_OK;
}

int32_t san_quant_attn(const san_planes* cache, const san_step_rows* rows, void* d_workspace, size_t workspace_bytes, void* stream) {
    QuantPlan a;
    int32_t rc = plan_quant(cache, rows, workspace_bytes, &a);
    if (rc != SAN_OK) return rc;
    if (rows->n_items == 0) return SAN_OK;
    if ((rc = check_plane_pointers(cache)) != SAN_OK) return rc;
    if (!rows->d_q || !rows->d_ids || !rows->d_lens || !rows->d_out) return SAN_ERR_NULL;
    if (!aligned(rows->d_q, 16) || !aligned(rows->d_out, 16) || !aligned(rows->d_S, 4)) return SAN_ERR_SHAPE;
    if (a.bytes > 0) {
        if (!d_workspace) return SAN_ERR_NULL;
        if (!aligned(d_workspace, 256)) return SAN_ERR_SHAPE;
        if (workspace_bytes < a.bytes) return SAN_ERR_CAPACITY;
    }
    AttendParams& p = a.p.a;
    p.q = static_cast<const char*>(rows->d_q); p.out = static_cast<char*>(rows->d_out);
    p.k = static_cast<const char*>(cache->d_k); p.v = static_cast<const char*>(cache->d_v);
    a.p.ks = static_cast<const char*>(cache->d_k_scale); a.p.vs = static_cast<const char*>(cache->d_v_scale);
    p.ids = rows->d_ids; p.lens = rows->d_lens; p.status = rows->d_status;
    a.p.S = rows->d_S; a.p.ld_s = rows->ld_s;
    p.part_ml = static_cast<float2*>(d_workspace);
    p.part_o = reinterpret_cast<float*>(static_cast<char*>(d_workspace) + a.ml_bytes);
    cudaStream_t st = static_cast<cudaStream_t>(stream);
    return rows->dtype == SAN_BF16 ? launch_quant_rows<1>(a, st) : launch_quant_rows<3>(a, st);
}

int32_t san_weight_mass(const san_mass_args* a, void* stream) {
    if (!a) return SAN_ERR_NULL;
    if (a->n_heads < 1 || a->n_heads > 1024 || a->n_kv_heads < 1 || a->n_heads % a->n_kv_heads != 0) return SAN_ERR_SHAPE;
    if (a->n_rows < 0 || a->n_rows > (1 << 20) || a->n_items < 0 || a->n_items > 65535 || a->max_ids < 1 || a->max_len < 0 || a->max_len > (1 << 28)) return SAN_ERR_SHAPE;
    if (a->ld_mass < a->max_len || !std::isfinite(a->decay)) return SAN_ERR_SHAPE;
    if (a->max_len == 0 && a->ld_mass > (1 << 28)) return SAN_ERR_SHAPE;
    const int max_len = a->max_len ? a->max_len : (int)a->ld_mass;
    if (a->n_items == 0 || max_len == 0) return SAN_OK;
    if (!a->d_S || !a->d_ids || !a->d_lens || !a->d_mass) return SAN_ERR_NULL;
    if (!aligned(a->d_S, 4) || !aligned(a->d_mass, 4)) return SAN_ERR_SHAPE;
    MassParams p;
    std::memset(&p, 0, sizeof(p));
    p.S = a->d_S; p.item_stride = a->item_stride; p.row_stride = a->row_stride; p.head_stride = a->head_stride;
    p.mass = a->d_mass; p.ld = a->ld_mass; p.rows = a->d_rows; p.ids = a->d_ids; p.lens = a->d_lens; p.begin = a->d_begin;
    p.n_rows = a->n_rows; p.H = a->n_heads; p.Hk = a->n_kv_heads; p.group = p.H / p.Hk; p.n_items = a->n_items; p.max_ids = a->max_ids;
    p.max_len = max_len; p.decay = a->decay; p.status = a->d_status;
    cudaStream_t st = static_cast<cudaStream_t>(stream);
    // Eight warps share a position's pairs where there are many; short rows are cut into more CTAs where there would not be two an SM.
    if ((long long)a->n_rows * p.group < 16) return launch_mass<1, 8>(p, st);
    const long long wide = div_up(max_len, mass_positions<8, 4>()) * p.Hk * p.n_items;
    return wide >= 2 * kSms ? launch_mass<8, 4>(p, st) : launch_mass<8, 1>(p, st);
}

int32_t san_cache_evict_bytes(const san_planes* cache, const san_evict_args* a, size_t* workspace_bytes) {
    if (!workspace_bytes) return SAN_ERR_NULL;
    const int32_t rc = check_evict(cache, a);
    if (rc == SAN_OK) *workspace_bytes = evict_bytes(cache, a);
    return rc;
}

int32_t san_cache_evict(const san_planes* cache, const san_evict_args* a, void* d_workspace, size_t workspace_bytes, void* stream) {
    int32_t rc = check_evict(cache, a);
    if (rc != SAN_OK) return rc;
    if (a->n_items == 0) return SAN_OK;
    if ((rc = check_plane_pointers(cache)) != SAN_OK) return rc;
    if (!a->d_ids || !a->d_lens || !a->d_mass || !a->d_lens_out || !d_workspace) return SAN_ERR_NULL;
    if (!aligned(d_workspace, 256) || !aligned(a->d_mass, 4)) return SAN_ERR_SHAPE;
    if (workspace_bytes < evict_bytes(cache, a)) return SAN_ERR_CAPACITY;
    const bool q4 = cache->dtype == SAN_Q4;
    EvictParams p;
    std::memset(&p, 0, sizeof(p));
    const int row_bytes = q4 ? kQuantRow : kDh * (cache->dtype == SAN_BF16 ? 2 : 4);
    p.k = static_cast<char*>(cache->d_k); p.v = static_cast<char*>(cache->d_v); p.v_stride = cache->v_stride / kDh * row_bytes;
    if (q4) {
        p.ks = static_cast<char*>(cache->d_k_scale); p.vs = static_cast<char*>(cache->d_v_scale);
        p.s_stride = cache->v_stride / kDh * 4;
    }
    p.ids = a->d_ids; p.lens = a->d_lens; p.mass = a->d_mass; p.ld = a->ld_mass; p.kept = a->d_kept; p.ld_kept = a->ld_kept;
    p.lens_out = a->d_lens_out; p.Hk = cache->n_kv_heads; p.n_layers = cache->n_layers; p.max_ids = cache->max_ids; p.cap = cache->cap_len;
    p.n_items = a->n_items; p.max_len = a->max_len ? a->max_len : cache->cap_len; p.keep = a->n_keep; p.sink = a->n_sink; p.recent = a->n_recent;
    p.status = a->d_status;
    p.plan = static_cast<int2*>(d_workspace);
    p.list = reinterpret_cast<int*>(static_cast<char*>(d_workspace) + evict_plan_bytes(cache, a));
    cudaStream_t st = static_cast<cudaStream_t>(stream);
    const dim3 panels((unsigned)p.Hk, (unsigned)p.n_items);
    if (p.max_len <= 4 * 1024) evict_select_kernel<4><<<panels, kEvictThreads, 0, st>>>(p);
    else if (p.max_len <= 16 * 1024) evict_select_kernel<16><<<panels, kEvictThreads, 0, st>>>(p);
    else evict_select_long_kernel<<<panels, kEvictThreads, 0, st>>>(p);
    if (cudaGetLastError() != cudaSuccess) return SAN_ERR_CUDA;
    // A plane's rows are moved by as many CTAs as have something to do in a step, up to eight, where there are too few planes for the SMs.
    const long long pieces = (long long)p.keep * (row_bytes / 16), planes = (long long)(1 + p.n_layers) * p.Hk * p.n_items;
    p.cluster = 1;
    while (p.cluster < 8 && planes * p.cluster < 4 * kSms && (long long)p.cluster * kMoveThreads * 2 < pieces) p.cluster *= 2;
    return q4 ? launch_move<2>(p, st) : cache->dtype == SAN_BF16 ? launch_move<8>(p, st) : launch_move<16>(p, st);
}

}  // extern "C"
