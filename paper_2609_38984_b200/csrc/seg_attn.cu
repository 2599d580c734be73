// Segment attention: how the work is cut, the merge of partial results, and the dispatch to the kernels.
//
// Partial results of the pieces i of a row are merged exactly: with reference maxima m_i, sums l_i and unnormalised
// outputs o_i, m = max m_i, out = sum_i 2^(m_i - m) o_i / sum_i 2^(m_i - m) l_i, lse = ln 2 (m + log2 sum).
#include <string.h>

#include "seg_attn.cuh"

namespace swam {
namespace {

constexpr int kMaxSplits = 64;
constexpr int64_t kMaxItemKeys = 1 << 26;

// One warp per row; lanes hold the pieces' weights and then D / 32 output columns each.  The first pieces' outputs are
// requested before the weights are known (an output of weight 0 may never have been written and is not used).
// kPaged: only rows of samples that have pieces are joined; tokens in front of the first sample, behind the last one or of a sample that is
// left out have none.  (A plan with pieces has few samples, and looking the row's up runs beside the last pieces.)
template <int D, typename T, int kMergeBatch, bool kPaged>
__global__ void __launch_bounds__(128) seg_merge_kernel(const __grid_constant__ SegParams p, const int parts,
                                                        const __grid_constant__ CacheArg<kPaged> pc) {
  constexpr int CPL = D / 32;
  const int lane = threadIdx.x & 31;
  const uint32_t row = blockIdx.x * 4 + (threadIdx.x >> 5);           // (sample, query, head)
  const SegArgs& a = p.a;
  const uint32_t bt = row / (uint32_t)a.N_h, h = row - bt * a.N_h, b = bt / (uint32_t)a.n_q, t = bt - b * a.n_q;
  T* out = (T*)a.out + b * a.o_smp + t * a.o_tok + (int64_t)h * D + lane * CPL;
  const float* src = p.part_o + (int64_t)row * D + lane * CPL;
  const float2* ml = p.part_ml + row;
  bool owned = row < p.rows;
  if constexpr (kPaged) owned = owned && paged_owned(pc, a.n_q, (int)bt);
  wait_previous();                                                    // everything above ran beside the last pieces
  if (!owned) return;
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
  int used = parts;                                     // paged: pieces behind a sample's last key have weight 0
  if constexpr (kPaged) {
    used = 0;
#pragma unroll
    for (int j = 0; j < 4; ++j) {
      const uint32_t some = __ballot_sync(0xffffffffu, wi[j] != 0.f);
      if (some) used = j * 32 + 32 - __clz(some);
    }
  }
  for (int i0 = 0; i0 < used; i0 += kMergeBatch) {
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

template <int D, typename T, bool kPaged>
cudaError_t launch_merge_d(const SegParams& p, int parts, const CacheArg<kPaged>& c, cudaStream_t st, int* launches) {
  const dim3 grid((unsigned)((p.rows + 3) / 4)), block(128);
  ++*launches;
  // (loads beyond the last piece are repeats of it: two pieces, the usual number of a shared plan, want a batch of their own)
  if (parts <= 2) return launch_after(seg_merge_kernel<D, T, 2, kPaged>, grid, block, 0, st, p, parts, c);
  return launch_after(seg_merge_kernel<D, T, 8, kPaged>, grid, block, 0, st, p, parts, c);
}
template <typename T, bool kPaged>
cudaError_t launch_merge(const SegParams& p, int parts, const CacheArg<kPaged>& c, cudaStream_t st, int* launches) {
  switch (p.a.D) {
    case 32: return launch_merge_d<32, T, kPaged>(p, parts, c, st, launches);
    case 64: return launch_merge_d<64, T, kPaged>(p, parts, c, st, launches);
    default: return launch_merge_d<128, T, kPaged>(p, parts, c, st, launches);
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
  return a.dtype == 0 ? launch_merge<float, false>(p, pl.parts(), NoCache(), st, launches)
                      : launch_merge<__nv_bfloat16, false>(p, pl.parts(), NoCache(), st, launches);
}

// ---- paged keys: the same kernels where the pieces can be planned from sizes, and the warp-level one that shares the keys out on the device
namespace {
struct PagedPlan {
  Kind kind;
  int tile_rows, splits;     // kF32, kTc
  int blocks, row_tiles;     // kF32: samples and row tiles per sample and key/value head, or all samples' row tiles (at most) and 0
  int items;                 // at most
  int shares;                // kMma: CTAs
  bool cut;
};
// The kernel for paged keys, up to `rows` of a sample and key/value head and up to `keys` of them.  More than 64 rows fill a tile of the tensor
// cores, at every head dim; more than 32 do with more than 512 keys.  From 17 rows on it streams long histories faster than the warp-level
// kernel (24 heads of 128, 16 samples of 32 rows and up to 8704 keys: 160 us instead of 192; of 16 rows: 160 and 166), but starts later: head
// dim 128 with up to 1232 keys 52 and 57 us, with up to 432 keys 36 and 29; head dim 64, whose keys are half as many bytes,
// 96 and 112 with up to 8704 keys, 41 and 32 with up to 1232, 30 and 26 with 48 items of the SMs' 148.  At head dim 32 it is slower or even.
Kind paged_kind(const SegArgs& a, const PagedCache& c, int64_t rows, bool warp_mma) {
  if (a.dtype == 0) return kF32;
  if (warp_mma) return kMma;
  if (rows > 64) return kTc;
  if (a.D == 32 || rows <= 16) return kMma;
  if (rows > 32) return c.max_kv > 512 ? kTc : kMma;
  return a.D == 128 ? (c.max_kv > 1024 ? kTc : kMma) : (c.max_kv > 2048 && (int64_t)c.samples * a.N_kv >= 2 * a.sms ? kTc : kMma);
}
PagedPlan paged_plan(const SegArgs& a, const PagedCache& c, bool warp_mma) {
  PagedPlan pl;
  const int g = a.N_h / a.N_kv;
  const int64_t rows = (int64_t)c.max_q * g;
  pl.kind = paged_kind(a, c, rows, warp_mma);
  if (pl.kind == kTc) pl.tile_rows = seg_tc_tile_rows(rows);
  else if (pl.kind == kMma) pl.tile_rows = rows <= 8 ? 8 : seg_mma_tile_rows(rows);
  else pl.tile_rows = rows > 32 ? 64 : seg_f32_tile_rows(rows, c.samples * (int64_t)a.N_kv, a.sms);       // (30 us instead of 33 with 32)
  pl.blocks = c.samples;
  pl.row_tiles = (int)ceil_div(rows, pl.tile_rows);
  // A sample fills its tiles but for the last one; one without new tokens has none.  (A call has 2^30 rows at most, so that tiles * N_kv
  // stays below 2^30 + 2^26, and half as much again below 2^31.)
  const int64_t longest = (int64_t)c.samples * pl.row_tiles;       // if all samples had as many as the longest may have
  int64_t tiles = (int64_t)a.n_q * g / pl.tile_rows + (c.samples < a.n_q ? c.samples : a.n_q);
  if (tiles > longest) tiles = longest;
  int64_t s = 1;
  // Long histories, and row tiles for fewer than one or two rounds of the SMs: pieces for several blocks an SM, which load the SMs evenly
  // whatever the lengths (5 samples of some 290 tokens, 16 heads of 64 on 2, 17430 to 89139 keys: 544 us instead of 1154; 2 samples of 300 tokens,
  // 32 heads of 128 on 8, up to 60000 keys: 374 and 778; 144 tiles of 64 rows and 30000 keys each, where there is nothing to even out: 181 and
  // 172, the join; 240 such tiles, bound by memory on fewer SMs too, 289 and 277).
  const bool even = c.max_kv >= 16384 && tiles * a.N_kv < (pl.tile_rows == 128 ? 1 : 2) * a.sms;
  if (pl.kind == kTc) {
    // No more pieces than SMs.  Where samples differ in length, the longest may have more than its share, which the kernel decides (6 samples
    // of 3000 to 30000 keys: 76 us, 88 without).  256 rows of partial results cost more than that gains.
    s = a.sms / (tiles * a.N_kv);
    if (s > 1 && pl.tile_rows == 128) s *= 4;
    if (s > c.max_kv / 256) s = c.max_kv / 256;      // (148 tokens of 24 heads on 8 and 1281 keys: 23 us, 27 with pieces of 512)
    if (s > kMaxSplits) s = kMaxSplits;
    if (s < 8 && even) s = 8;
    if (s < ceil_div(c.max_kv, kMaxItemKeys)) s = ceil_div(c.max_kv, kMaxItemKeys);
    if (s < 1) s = 1;
  } else if (pl.kind == kF32) {
    // Many small pieces, of one size for all samples: those of short samples are empty, and the long ones are what takes time (6 samples
    // of 41 to 1521 keys, 90 row tiles: 56 us with 4 SMs' worth of CTAs, 30 with 12 or 16).
    // A block each for as many row tiles as the longest sample may have; where that is half as many again as there can be (a call that
    // does not say how many new tokens a sample has), the blocks look for theirs, which takes a pass over q_start.
    if (2 * longest > 3 * tiles) {
      pl.blocks = (int)tiles;
      pl.row_tiles = 0;
    } else {
      tiles = longest;
    }
    s = 16 * a.sms / (tiles * a.N_kv);
    if (s > c.max_kv / 96) s = c.max_kv / 96;
    if (s > kMaxSplits) s = kMaxSplits;
    if (s < 1) s = 1;
  }
  pl.splits = (int)s;
  int64_t items = tiles * a.N_kv * s;                              // (more than one piece only of few row tiles)
  if (pl.kind == kTc && s > 1 && items > (even ? 4 : 1) * a.sms) items = (even ? 4 : 1) * a.sms;      // blocks: each takes what is left in turn
  pl.items = (int)items;
  pl.shares = paged_mma_shares(a.sms);
  // A row tile's keys are cut only where they may be many: the second kernel costs more than 512 keys do.
  pl.cut = c.max_kv > 512;
  return pl;
}
}  // namespace

size_t paged_scratch_bytes(const SegArgs& a, const PagedCache& c, bool warp_mma) {
  if (a.n_q == 0 || c.samples == 0) return 0;
  const PagedPlan pl = paged_plan(a, c, warp_mma);
  if (pl.kind == kMma) return pl.cut ? paged_mma_scratch(pl.shares, pl.tile_rows, a.D) : 0;
  return pl.splits > 1 ? (size_t)pl.splits * a.n_q * a.N_h * ((size_t)a.D * sizeof(float) + sizeof(float2)) : 0;
}

cudaError_t launch_paged_attn(const SegArgs& a, const PagedCache& c, bool warp_mma, void* scratch, int* status, cudaStream_t st,
                              int* launches) {
  const PagedPlan pl = paged_plan(a, c, warp_mma);
  SegParams p;
  memset(&p, 0, sizeof(p));
  p.a = a;
  p.g = a.N_h / a.N_kv;
  p.scale_log2 = a.scale * 1.4426950408889634f;
  p.rows = (int64_t)a.n_q * a.N_h;
  p.status = status;
  p.part_o = (float*)scratch;
  if (pl.kind == kMma) return launch_paged_mma(p, c, pl.tile_rows, pl.shares, pl.cut, st, launches);
  p.direct = pl.splits == 1;
  p.part_ml = (float2*)((float*)scratch + (size_t)pl.splits * p.rows * a.D);
  SegPass& ps = p.pass[0];
  ps.seg_lo = ps.seg_hi = 1;
  ps.block_samples = 1;
  ps.blocks = pl.blocks;
  ps.row_tiles = pl.row_tiles;
  ps.splits = pl.splits;
  ps.items = pl.items;
  const cudaError_t e = pl.kind == kTc ? launch_paged_tc(p, c, pl.tile_rows == 128, st, launches)
                                       : launch_paged_f32(p, c, pl.tile_rows, st, launches);
  if (e != cudaSuccess || p.direct) return e;
  return a.dtype == 0 ? launch_merge<float, true>(p, pl.splits, c, st, launches) : launch_merge<__nv_bfloat16, true>(p, pl.splits, c, st, launches);
}

}  // namespace swam
