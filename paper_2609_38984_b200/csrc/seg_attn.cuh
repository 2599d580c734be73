// Work decomposition shared by the segment-attention kernels (cross attention and shared-prefix attention).
//
// The rows of a block (one sample, or all samples of a group) that read one key/value head are flattened in the order
// (sample, query, head of the group) and cut into row tiles; the keys of the block are the tiles of segment 0 followed
// by the tiles of segment 1.  A work item is (block, key/value head, row tile, piece of the key tiles).  Lengths live
// on the device, so the pieces are cut there: the real key tiles of an item's block are shared out evenly.
#pragma once
#include <atomic>

#include "swam_internal.cuh"

namespace swam {

struct SegPass {
  int seg_lo, seg_hi;       // segments this pass walks over
  int block_samples;        // samples per block
  int blocks, row_tiles;    // blocks; row tiles per (block, key/value head)
  int splits, part0;        // pieces over the keys; index of the first piece's partial results
  int items;                // blocks * N_kv * row_tiles * splits
};

struct SegParams {
  SegArgs a;
  SegPass pass[2];
  int early;                // the second pass may start at once (it needs nothing from the first)
  int direct;               // 1: an item's result is final, 0: unnormalised partial results go to scratch
  int g;                    // query heads per key/value head
  float scale_log2;
  float* part_o;            // [parts][B * n_q * N_h][D]
  float2* part_ml;          // [parts][B * n_q * N_h] reference maximum (log2 domain) and sum
  int64_t rows;             // B * n_q * N_h
  int* status;
};

struct SegItem {
  int block, h_kv, row0, split;
};

__device__ __forceinline__ SegItem seg_item(const SegPass& ps, int N_kv, int tile_rows, int w) {
  SegItem it;
  it.row0 = (w % ps.row_tiles) * tile_rows;
  w /= ps.row_tiles;
  it.split = w % ps.splits;
  w /= ps.splits;
  it.h_kv = w % N_kv;
  it.block = w / N_kv;
  return it;
}

// real keys of segment s for group / sample idx; lengths out of range are clamped and flagged
__device__ __forceinline__ int seg_len(const SegParams& p, int s, int idx) {
  const int n = p.a.n[s];
  if (n == 0 || !p.a.len[s]) return n;
  const int l = __ldg(p.a.len[s] + idx);
  if (l < 0 || l > n) {
    if ((threadIdx.x & 31) == 0) atomicOr(p.status, ST_BAD_LEN);
    return l < 0 ? 0 : n;
  }
  return l;
}

// a flattened row of a block: its sample, query and head
struct SegRow {
  int b, t, h;
  bool real;
};
__device__ __forceinline__ SegRow seg_row(const SegParams& p, int block_samples, int b0, int h_kv, int row) {
  SegRow r;
  const int per_sample = p.a.n_q * p.g;
  r.real = row < block_samples * per_sample;
  const int rr = r.real ? row : 0;
  const int smp = block_samples > 1 ? rr / per_sample : 0;
  const int i = rr - smp * per_sample;
  r.b = b0 + smp;
  r.t = p.g == 1 ? i : i / p.g;
  r.h = h_kv * p.g + (i - r.t * p.g);
  return r;
}
__device__ __forceinline__ SegRow seg_row(const SegParams& p, const SegPass& ps, const SegItem& it, int row) {
  return seg_row(p, ps.block_samples, it.block * ps.block_samples, it.h_kv, row);
}
// keys of segment 1 that query t sees when the sample has `len` of them
__device__ __forceinline__ int seg_limit1(const SegArgs& a, int len, int t) {
  return a.causal ? max(0, len - a.n_q + t + 1) : len;
}

// An exponent is the scaled score minus the row's reference.  One fused multiply-add does not round the product as the reference was
// rounded: half a step of the reference, which outgrows the exponents of fp32 from 2^31 on (step 256), would stand in the
// exponent of the largest score itself.  From this magnitude on (half a step is 1 there) the product is rounded first.
constexpr float kSegBig = 16777216.f;      // 2^24

// What a row's sum of weights makes of its result: only a sum of exactly 0 is a row without keys.  A NaN sum (a NaN or +inf logit
// of a visible key) has to stay one.
__device__ __forceinline__ float seg_inverse(float sum) { return sum == 0.f ? 0.f : 1.f / sum; }
__device__ __forceinline__ float seg_lse(float m, float sum) { return sum == 0.f ? -INFINITY : (m + log2f(sum)) * 0.6931471805599453f; }

// the key tiles (KT keys each) of an item: [begin, end) of the concatenated tiles of segment 0 (len0 keys, n0 tiles)
// and segment 1 (len1 keys: no row of the tile sees more of them)
struct SegKeys {
  int len0, len1, n0, begin, end;
};
__device__ __forceinline__ SegKeys seg_keys(const SegParams& p, const SegPass& ps, const SegItem& it, int tile_rows, int KT) {
  SegKeys k;
  const int b0 = it.block * ps.block_samples;
  k.len0 = ps.seg_lo == 0 ? seg_len(p, 0, b0 / p.a.per_group) : 0;
  k.len1 = 0;
  if (ps.seg_hi == 1) {      // such a block is one sample
    const int last = min(it.row0 + tile_rows, p.a.n_q * p.g) - 1;
    k.len1 = seg_limit1(p.a, seg_len(p, 1, b0), last / p.g);
  }
  k.n0 = (k.len0 + KT - 1) / KT;
  const int total = k.n0 + (k.len1 + KT - 1) / KT;
  const int per = (total + ps.splits - 1) / ps.splits;
  k.begin = min(total, it.split * per);
  k.end = min(total, k.begin + per);
  return k;
}

// Kernels of one call follow each other without a gap: each lets the next one start (allow_next) once all its CTAs are past
// their last key tile, or, where that is a second pass, have started; and the next one's CTAs wait (griddepcontrol.wait) for the end of the one before: the merge before
// it reads, a second pass, which needs nothing from the first, before it ends, so that waiting for the second pass is
// waiting for both.
__device__ __forceinline__ void allow_next() { asm volatile("griddepcontrol.launch_dependents;" ::: "memory"); }
__device__ __forceinline__ void wait_previous() { asm volatile("griddepcontrol.wait;" ::: "memory"); }
// Opts a kernel in to its dynamic shared memory, once per device (every launch function has one of these).
struct SmemOptIn {
  std::atomic<uint64_t> done{0};
  cudaError_t operator()(const void* kernel, int bytes, int device) {
    const uint64_t bit = 1ull << (device & 63);
    if (device < 64 && (done.load(std::memory_order_acquire) & bit)) return cudaSuccess;
    const cudaError_t e = cudaFuncSetAttribute(kernel, cudaFuncAttributeMaxDynamicSharedMemorySize, bytes);
    if (e == cudaSuccess && device < 64) done.fetch_or(bit, std::memory_order_release);
    return e;
  }
};
template <typename... Params, typename... Args>
cudaError_t launch_after(void (*kernel)(Params...), dim3 grid, dim3 block, size_t smem, cudaStream_t st, Args... args) {
  cudaLaunchAttribute attr;
  attr.id = cudaLaunchAttributeProgrammaticStreamSerialization;
  attr.val.programmaticStreamSerializationAllowed = 1;
  cudaLaunchConfig_t cfg = {};
  cfg.gridDim = grid;
  cfg.blockDim = block;
  cfg.dynamicSmemBytes = smem;
  cfg.stream = st;
  cfg.attrs = &attr;
  cfg.numAttrs = 1;
  return cudaLaunchKernelEx(&cfg, kernel, args...);
}

// rows of a row tile of the warp-level and of the fp32 kernel for blocks of `rows` rows
inline int seg_mma_tile_rows(int64_t rows) { return rows <= 16 ? 16 : (rows <= 32 ? 32 : 64); }
// of the tcgen05 kernel: two query tiles, or one whose keys two streams take in turn
inline int seg_tc_tile_rows(int64_t rows) { return rows <= 128 ? 128 : 256; }
// of the fp32 kernel for `blocks` pairs of block and key/value head: 64 rows run at the best rate, 32 where there are not
// enough of them to fill the SMs evenly
inline int seg_f32_tile_rows(int64_t rows, int64_t blocks, int sms) {
  if (rows <= 16) return 16;
  return rows <= 32 || blocks * ((rows + 63) / 64) < 2 * sms ? 32 : 64;
}
// rows: rows of a block, per key/value head (they choose the row tile)
// wide: eight warps instead of four share the keys of a 16-row tile
cudaError_t launch_seg_mma(const SegParams& p, int pass, int tile_rows, bool wide, cudaStream_t st, int* launches);
// both: the items of pass 1 follow those of pass 0 in the same launch; alt: 128-row tiles whose keys two streams take in turn
cudaError_t launch_seg_tc(const SegParams& p, int pass, bool both, bool alt, cudaStream_t st, int* launches);
cudaError_t launch_seg_f32(const SegParams& p, int pass, int tile_rows, cudaStream_t st, int* launches);

}  // namespace swam
