// Host helpers of the calls that need no context: argument checks, opt-in to large shared memory, launches that overlap the
// kernel before them, workspaces of partial results.
#pragma once

#include <algorithm>
#include <cmath>
#include <cstring>

#include "san_attend.cuh"

namespace san {
namespace {

constexpr int kSms = 148;                   // the cuts are made for this GPU; any other number of SMs works
inline long long div_up(long long a, long long b) { return (a + b - 1) / b; }
inline int32_t cuda_status(cudaError_t e) { return e == cudaSuccess ? SAN_OK : SAN_ERR_CUDA; }
inline bool aligned(const void* p, uintptr_t n) { return ((uintptr_t)p & (n - 1)) == 0; }

// Opt-in to dynamic shared memory above 48 KB, an attribute of a kernel on a device: done once for each (`set`, one
// entry per device, belongs to the kernel).
inline int32_t opt_in(const void* fn, int bytes, bool* set) {
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

// Workspace of `rows` partial results: (max, sum) and the layers' outputs of each.
inline size_t partial_ml_bytes(size_t rows) { return (rows * sizeof(float2) + 255) / 256 * 256; }
inline size_t partial_bytes(size_t rows, int layers) { return partial_ml_bytes(rows) + rows * layers * kDh * sizeof(float); }

constexpr int kOwnLeast = 4;                // tiles of own rows that are not cut
// How one kind of units (`units` runs of up to `tiles` tiles) is cut where a warp's share of the whole call is
// `share` tiles: warps per unit and runs of tiles.  A run of no more than 1.25 shares (or `least` tiles) is one warp's.  A longer
// one is cut into up to four runs for a warp each, so that the warps finish together; beyond that the four
// warps of a CTA take a run together, which leaves a quarter of the partial results.  Measured (device time): 32 prefixes of 16
// tiles beside 1024 rows of up to 8, share 10: 48.6 us uncut, 35.9 in two runs each; 1024 runs of 17 tiles, share 15: 53.4 us
// uncut, 58.7 by four warps each; 8 runs of 513 tiles: 13.0 us by four warps, 17.7 by one.
// `least`: tiles below which a cut costs more than it gives (a float32 tile of eight rows is several bf16 ones' work).
inline void cut_runs(int tiles, double share, int least, int* wpu, int* splits, int* span) {
    const int most = std::max(least, (int)std::ceil(1.25 * share));
    const int pieces = (int)div_up(tiles, most);
    *wpu = pieces > 4 ? kAtWarps : 1;
    *splits = pieces > 4 ? (int)div_up(pieces, kAtWarps) : pieces;
    *span = (int)div_up(tiles, *splits);
    *splits = (int)div_up(tiles, *span);
}

}  // namespace
}  // namespace san
