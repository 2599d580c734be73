// Segment attention: how the work is cut, the merge of partial results, and the dispatch to the kernels.
//
// Partial results of the pieces i of a row are merged exactly: with reference maxima m_i, sums l_i and unnormalised
// outputs o_i, m = max m_i, out = sum_i 2^(m_i - m) o_i / sum_i 2^(m_i - m) l_i, lse = ln 2 (m + log2 sum).
#include "seg_attn.cuh"

namespace swam {
namespace {

constexpr int kMaxSplits = 64;
constexpr int64_t kMaxItemKeys = 1 << 26;

// One warp per row; lanes hold the pieces' weights and then D / 32 output columns each.  The first pieces' outputs are
// requested before the weights are known (an output of weight 0 may never have been written and is not used).
template <int D, typename T, int kMergeBatch>
__global__ void __launch_bounds__(128) seg_merge_kernel(const __grid_constant__ SegParams p, const int parts) {
  constexpr int CPL = D / 32;
  const int lane = threadIdx.x & 31;
  const uint32_t row = blockIdx.x * 4 + (threadIdx.x >> 5);           // (sample, query, head)
  const SegArgs& a = p.a;
  const uint32_t bt = row / (uint32_t)a.N_h, h = row - bt * a.N_h, b = bt / (uint32_t)a.n_q, t = bt - b * a.n_q;
  T* out = (T*)a.out + b * a.o_smp + t * a.o_tok + (int64_t)h * D + lane * CPL;
  const float* src = p.part_o + (int64_t)row * D + lane * CPL;
  const float2* ml = p.part_ml + row;
  wait_previous();                                                    // everything above ran beside the last pieces
  if (row >= p.rows) return;
  float v[kMergeBatch][CPL];
  auto load = [&](int i0) {
#pragma unroll
    for (int i = 0; i < kMergeBatch; ++i) {
      const float* x = src + (int64_t)min(i0 + i, parts - 1) * p.rows * D;
      if constexpr (CPL == 4) *reinterpret_cast<float4*>(v[i]) = *reinterpret_cast<const float4*>(x);
      else if constexpr (CPL == 2) *reinterpret_cast<float2*>(v[i]) = *reinterpret_cast<const float2*>(x);
      else v[i][0] = x[0];
    }
  };
  load(0);
  // up to 128 pieces: four per lane
  float mi[4], wi[4], m = -INFINITY, l = 0.f;
#pragma unroll
  for (int j = 0; j < 4; ++j) {
    const int i = j * 32 + lane;
    const float2 x = i < parts ? ml[(int64_t)i * p.rows] : make_float2(-INFINITY, 0.f);
    mi[j] = x.x;
    wi[j] = x.y;
    m = fmaxf(m, x.x);
  }
#pragma unroll
  for (int o = 16; o > 0; o >>= 1) m = fmaxf(m, __shfl_xor_sync(0xffffffffu, m, o));
#pragma unroll
  for (int j = 0; j < 4; ++j) {
    const float f = mi[j] == -INFINITY ? 0.f : exp2f(mi[j] - m);   // a piece without keys has weight 0
    l += f * wi[j];
    wi[j] = f;
  }
#pragma unroll
  for (int o = 16; o > 0; o >>= 1) l += __shfl_xor_sync(0xffffffffu, l, o);
  float acc[CPL];
#pragma unroll
  for (int c = 0; c < CPL; ++c) acc[c] = 0.f;
  for (int i0 = 0; i0 < parts; i0 += kMergeBatch) {
    if (i0 > 0) load(i0);
    const float w4 = i0 < 32 ? wi[0] : (i0 < 64 ? wi[1] : (i0 < 96 ? wi[2] : wi[3]));
#pragma unroll
    for (int i = 0; i < kMergeBatch; ++i) {
      const float f = i0 + i < parts ? __shfl_sync(0xffffffffu, w4, (i0 + i) & 31) : 0.f;
#pragma unroll
      for (int c = 0; c < CPL; ++c) acc[c] = f != 0.f ? fmaf(f, v[i][c], acc[c]) : acc[c];
    }
  }
  const float inv = seg_inverse(l);
  if constexpr (sizeof(T) == 4 && CPL == 4) {
    *reinterpret_cast<float4*>(out) = make_float4(acc[0] * inv, acc[1] * inv, acc[2] * inv, acc[3] * inv);
  } else if constexpr (sizeof(T) == 2 && CPL >= 2) {
#pragma unroll
    for (int c = 0; c < CPL; c += 2) *reinterpret_cast<__nv_bfloat162*>(out + c) = __floats2bfloat162_rn(acc[c] * inv, acc[c + 1] * inv);
  } else {
#pragma unroll
    for (int c = 0; c < CPL; ++c) out[c] = (T)(acc[c] * inv);
  }
  if (a.lse && lane == 0) a.lse[((int64_t)b * a.N_h + h) * a.n_q + t] = seg_lse(m, l);
}

template <int D, typename T>
cudaError_t launch_merge_d(const SegParams& p, int parts, cudaStream_t st, int* launches) {
  const dim3 grid((unsigned)((p.rows + 3) / 4)), block(128);
  ++*launches;
  // (loads beyond the last piece are repeats of it: two pieces, the usual number of a shared plan, want a batch of their own)
  if (parts <= 2) return launch_after(seg_merge_kernel<D, T, 2>, grid, block, 0, st, p, parts);
  return launch_after(seg_merge_kernel<D, T, 8>, grid, block, 0, st, p, parts);
}
template <typename T>
cudaError_t launch_merge(const SegParams& p, int parts, cudaStream_t st, int* launches) {
  switch (p.a.D) {
    case 32: return launch_merge_d<32, T>(p, parts, st, launches);
    case 64: return launch_merge_d<64, T>(p, parts, st, launches);
    default: return launch_merge_d<128, T>(p, parts, st, launches);
  }
}

// Lengths that belong to a tensor without rows: the other kernels have no reason to read them.
__global__ void seg_check_lengths_kernel(const int32_t* len, int n, int* status) {
  for (int i = threadIdx.x; i < n; i += blockDim.x)
    if (len[i] != 0) atomicOr(status, ST_BAD_LEN);
}

int64_t ceil_div(int64_t a, int64_t b) { return (a + b - 1) / b; }

// How a pass runs: `blocks` blocks with `rows` rows per key/value head each and up to `keys` keys.  pass: -1 = the only one.
enum Kind { kF32, kMma, kTc };
struct PassPlan {
  Kind kind;
  int tile_rows;
  bool wide;            // kMma: eight warps along the keys
  int splits;
};
PassPlan plan_pass(const SegArgs& a, int64_t blocks, int64_t rows, int64_t keys, bool warp_mma, int pass) {
  PassPlan p;
  const int sms = a.sms;
  // Few rows stream their keys through the warp-level kernel; from 33 rows on the tensor cores' tiles are filled well enough
  // (from 65 on with few keys, where the larger kernel's start costs more than its rate gains).
  p.kind = a.dtype == 0 ? kF32 : (a.D < 64 || warp_mma || rows <= 32 || (rows <= 64 && keys <= 512) ? kMma : kTc);
  p.tile_rows = p.kind == kF32 ? seg_f32_tile_rows(rows, blocks * a.N_kv, sms) : (p.kind == kMma ? seg_mma_tile_rows(rows) : seg_tc_tile_rows(rows));
  const int64_t items = blocks * a.N_kv * ceil_div(rows, p.tile_rows);
  // fewer items than two CTAs per SM: one CTA of eight warps streams an item twice as fast, and needs half the pieces
  p.wide = p.kind == kMma && p.tile_rows == 16 && items < 2 * sms;
  int64_t s, min_keys;
  if (p.kind == kTc || p.wide) {
    // one CTA per SM: as many pieces as one wave holds, or half a wave where a second pass with more keys fills the rest
    s = (pass == 0 && a.B * (int64_t)a.n[1] > blocks * keys ? sms / 2 : sms) / (items > 0 ? items : 1);
    min_keys = 512;
  } else {
    // Two CTAs per SM.  A merge costs some 10 us with its partial results, so that more pieces for the sake of even waves pay
    // only where there is one anyway (64 samples of 520 keys: 32 us in one piece each, 39 us in two).
    s = (pass >= 0 ? 4 : 2) * sms / (items > 0 ? items : 1);
    min_keys = p.kind == kF32 ? 96 : 256;
  }
  if (s > keys / min_keys) s = keys / min_keys;
  if (s > kMaxSplits) s = kMaxSplits;
  // Waits of the tensor-core kernel last as long as an item, at some 3110 clk a tile of 128 keys, and give up after kWaitCycles:
  // an item takes 1.6e9 of these 4e9 clk at most.  (2^30 keys, the most that a call may have, are 16 pieces.)
  if (p.kind == kTc && s < ceil_div(keys, kMaxItemKeys)) s = ceil_div(keys, kMaxItemKeys);
  p.splits = s < 1 ? 1 : (int)s;
  return p;
}
// the plan of pass i
PassPlan plan_of(const SegArgs& a, bool shared, int i, bool warp_mma) {
  const int64_t rows = (int64_t)a.n_q * (a.N_h / a.N_kv);
  if (!shared) return plan_pass(a, a.B, rows, (int64_t)a.n[0] + a.n[1], warp_mma, -1);
  if (i == 0) return plan_pass(a, a.B / a.per_group, rows * a.per_group, a.n[0], warp_mma, a.n[1] > 0 ? 0 : -1);
  return plan_pass(a, a.B, rows, a.n[1], warp_mma, 1);
}

}  // namespace

SegPlan seg_plan(const SegArgs& a, bool warp_mma) {
  SegPlan pl;
  const int64_t rows = (int64_t)a.n_q * (a.N_h / a.N_kv);       // of one sample
  // Samples share the row tiles of segment 0 when a tile (128 rows on the tensor cores, 64 otherwise) has room for two samples
  // at least: the shared keys are then read once for all of them and multiplied with full tiles (16 samples of 64 rows
  // behind 9216 keys: 168 us, each sample by itself 325 us).
  const int64_t tile = a.dtype == 0 || a.D < 64 || warp_mma ? 64 : 128;
  pl.shared = a.per_group > 1 && a.n[0] > 0 && 2 * rows <= tile;
  pl.splits[0] = plan_of(a, pl.shared, 0, warp_mma).splits;
  pl.splits[1] = pl.shared && a.n[1] > 0 ? plan_of(a, pl.shared, 1, warp_mma).splits : 0;
  return pl;
}

size_t seg_scratch_bytes(const SegArgs& a, const SegPlan& p) {
  if (!p.partial()) return 0;
  const size_t rows = (size_t)a.B * a.n_q * a.N_h;
  return (size_t)p.parts() * rows * ((size_t)a.D * sizeof(float) + sizeof(float2));
}

cudaError_t launch_seg_attn(const SegArgs& a, const SegPlan& pl, bool warp_mma, void* scratch, int* status, cudaStream_t st,
                            int* launches) {
  SegParams p;
  p.a = a;
  p.g = a.N_h / a.N_kv;
  p.scale_log2 = a.scale * 1.4426950408889634f;
  p.rows = (int64_t)a.B * a.n_q * a.N_h;
  p.direct = !pl.partial();
  p.part_o = (float*)scratch;
  p.part_ml = (float2*)((float*)scratch + (size_t)pl.parts() * p.rows * a.D);
  p.status = status;
  const int n_pass = pl.shared && pl.splits[1] > 0 ? 2 : 1;
  p.early = n_pass == 2;
  PassPlan pp[2];
  for (int i = 0; i < 2; ++i) {
    SegPass& ps = p.pass[i];
    const bool mixed = pl.shared && i == 0;
    pp[i] = plan_of(a, pl.shared, i, warp_mma);
    ps.seg_lo = pl.shared ? i : 0;
    ps.seg_hi = mixed ? 0 : 1;
    ps.block_samples = mixed ? a.per_group : 1;
    ps.blocks = a.B / ps.block_samples;
    ps.row_tiles = (int)ceil_div((int64_t)a.n_q * p.g * ps.block_samples, pp[i].tile_rows);
    ps.splits = i < n_pass ? pl.splits[i] : 0;
    ps.part0 = i == 0 ? 0 : pl.splits[0];
    const int64_t items = (int64_t)ps.blocks * a.N_kv * ps.row_tiles * ps.splits;
    if (items > 0x7fffffff) return cudaErrorInvalidConfiguration;
    ps.items = (int)items;
  }
  for (int i = 0; i < 2; ++i) {
    if (a.n[i] > 0 || !a.len[i]) continue;
    ++*launches;
    seg_check_lengths_kernel<<<1, 128, 0, st>>>(a.len[i], i == 0 ? a.B / a.per_group : a.B, status);
    const cudaError_t e = cudaGetLastError();
    if (e != cudaSuccess) return e;
  }
  const bool both = n_pass == 2 && pp[0].kind == kTc && pp[1].kind == kTc && pp[0].tile_rows == pp[1].tile_rows;
  if (both) p.early = 0;
  for (int i = 0; i < (both ? 1 : n_pass); ++i) {
    const cudaError_t e = pp[i].kind == kF32   ? launch_seg_f32(p, i, pp[i].tile_rows, st, launches)
                          : pp[i].kind == kMma ? launch_seg_mma(p, i, pp[i].tile_rows, pp[i].wide, st, launches)
                                               : launch_seg_tc(p, i, both, pp[i].tile_rows == 128, st, launches);
    if (e != cudaSuccess) return e;
  }
  if (p.direct) return cudaSuccess;
  return a.dtype == 0 ? launch_merge<float>(p, pl.parts(), st, launches) : launch_merge<__nv_bfloat16>(p, pl.parts(), st, launches);
}

}  // namespace swam
