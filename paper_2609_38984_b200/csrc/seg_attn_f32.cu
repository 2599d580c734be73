// Segment attention for fp32 tensors, fp32 throughout on the FMA pipes.
//
// One CTA of 128 threads owns 16 * RPT query rows of one key/value head and walks over the keys in tiles of 32 that
// arrive by asynchronous copies into two stages.  Thread (ty, tx) of a 16 x 8 arrangement holds rows ty + 16 i and keys
// tx + 8 j of the score tile, then the same rows and output columns 4 tx + 32 c: every shared-memory load of four floats
// feeds RPT or 4 * RPT multiply-adds, so with RPT = 4 the FMA pipes and not the shared-memory port are the bound.
// RPT = 1 (16 rows) serves single tokens, RPT = 2 (32) calls too small to fill the SMs with 64 rows.  Keys beyond the real
// length are filled with zeros and masked.
// What bounds it: latency.  4 x 1000 rows, 8 heads of 64, 100 to 333 keys take 84 us (21 TFLOP/s of some 70 on the FMA pipes): three
// CTAs an SM leave 2.3 warps a scheduler, which issue every 2.2 clk.  Four CTAs with single K and V buffers took 86 us, 32-row
// tiles 92.  (Compiled to 128 registers, that instance, <64, 4>, spills 12 bytes a thread and loads 24; <128, 1> spills 4;
// for paged keys <64, 2> spills 48 and loads 40, which costs nothing that shows: 40 samples of 4 tokens 47 us with and without.)
// Paged single tokens have 15 of the 16 rows to no purpose and one tile in flight: 2 tokens, 32 heads of 128, 1500 and 1983 keys, 114 MB in 90
// us (1.3 TB/s).
#include "seg_attn.cuh"

namespace swam {
namespace {

constexpr int kKF = 32;        // keys per tile
constexpr int kThreadsF = 128;

__device__ __forceinline__ void cp16(void* dst, const void* src, uint32_t bytes) {
  asm volatile("cp.async.cg.shared.global [%0], [%1], 16, %2;"
               ::"r"((uint32_t)__cvta_generic_to_shared(dst)), "l"(src), "r"(bytes) : "memory");
}

// two multiply-adds in one instruction
__device__ __forceinline__ uint64_t pack2(float lo, float hi) {
  uint64_t r;
  asm("mov.b64 %0, {%1, %2};" : "=l"(r) : "f"(lo), "f"(hi));
  return r;
}
__device__ __forceinline__ void unpack2(uint64_t v, float& lo, float& hi) { asm("mov.b64 {%0, %1}, %2;" : "=f"(lo), "=f"(hi) : "l"(v)); }
__device__ __forceinline__ uint64_t fma2(uint64_t a, uint64_t b, uint64_t c) {
  uint64_t r;
  asm("fma.rn.f32x2 %0, %1, %2, %3;" : "=l"(r) : "l"(a), "l"(b), "l"(c));
  return r;
}

template <int D, int RPT>
struct F32Cfg {
  static constexpr int MR = 16 * RPT;
  static constexpr int QS = D + 4;                 // padded rows of Q and K: eight consecutive rows in different banks
  static constexpr int kQ = MR * QS, kK = kKF * QS, kV = kKF * D, kP = kKF * (MR + 4);
  static constexpr int kBytes = (kQ + 2 * (kK + kV) + kP) * 4;
};

// The sample of the tile-th of all samples' row tiles of MR rows, and its first row in the sample; false behind the last one.  (For the
// whole block: every thread adds up the tiles of a few neighbouring samples, and the one that has the tile among them looks for it.)
template <int MR>
__device__ __forceinline__ bool paged_find_tile(const PagedCache& c, int tokens, int g, int tile, int* sample, int* row0) {
  __shared__ int64_t warp_sum[kThreadsF / 32];
  __shared__ int2 found;
  const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
  const int per = (c.samples + kThreadsF - 1) / kThreadsF, b0 = min(c.samples, (int)threadIdx.x * per), b1 = min(c.samples, b0 + per);
  auto tiles = [&](int b) {
    const int q0 = __ldg(c.q_start + b), q1 = __ldg(c.q_start + b + 1);
    return paged_stretch(c, tokens, q0, q1) ? ((q1 - q0) * g + MR - 1) / MR : 0;
  };
  int64_t sum = 0;               // (stretches out of order may overlap)
  for (int b = b0; b < b1; ++b) sum += tiles(b);
  int64_t end = sum;
#pragma unroll
  for (int o = 1; o < 32; o <<= 1) {
    const int64_t y = __shfl_up_sync(0xffffffffu, end, o);
    if (lane >= o) end += y;
  }
  if (lane == 31) warp_sum[warp] = end;
  if (threadIdx.x == 0) found = make_int2(-1, 0);
  __syncthreads();
  for (int w = 0; w < warp; ++w) end += warp_sum[w];
  int64_t left = tile - (end - sum);
  if (left >= 0 && left < sum) {
    int b = b0;
    for (int n; left >= (n = tiles(b)); ++b) left -= n;
    found = make_int2(b, (int)left * MR);
  }
  __syncthreads();
  *sample = found.x;
  *row0 = found.y;
  return found.x >= 0;
}

// kPaged: an item is a row tile of one sample's new tokens, found from the block's number (and, where the plan counts the row tiles of all
// samples together, row_tiles = 0, from the samples' own lengths); its keys are found through the page table
template <int D, int RPT, bool kPaged>
__global__ void __launch_bounds__(kThreadsF) seg_f32_kernel(const __grid_constant__ SegParams p, const int pass,
                                                            const __grid_constant__ CacheArg<kPaged> pc) {
  using C = F32Cfg<D, RPT>;
  if (p.early && pass == 0) allow_next();
  constexpr int MR = C::MR, QS = C::QS, PS = MR + 4;
  extern __shared__ float sf[];
  float* sQ = sf;
  float* sK = sQ + C::kQ;        // [2][32][QS]
  float* sV = sK + 2 * C::kK;    // [2][32][D]
  float* sP = sV + 2 * C::kV;    // [32][MR + 4], row ty + 16 i at column ty * RPT + i
  const SegPass& ps = p.pass[pass];
  const SegArgs& a = p.a;
  SegItem it;
  if (kPaged && ps.row_tiles == 0) {
    const int w = blockIdx.x / ps.blocks;
    it.split = w % ps.splits;
    it.h_kv = w / ps.splits;
  } else {
    it = seg_item(ps, a.N_kv, MR, blockIdx.x);
  }
  SegKeys kk;
  PagedSample smp{0, 0, 0};
  int row_end = 0;               // kPaged: rows of the call in front of the end of the sample's
  if constexpr (kPaged) {
    if (ps.row_tiles == 0 && !paged_find_tile<MR>(pc, a.n_q, p.g, blockIdx.x % ps.blocks, &it.block, &it.row0)) {
      allow_next();
      return;
    }
    smp = paged_sample(pc, a.n_q, it.block, p.status);
    const int rows = smp.n * p.g;
    if (it.row0 >= rows) {       // (what the next kernel waits for is the end of all blocks)
      allow_next();
      return;
    }
    kk.len0 = kk.n0 = 0;
    kk.len1 = paged_limit(a.causal, smp, (min(it.row0 + MR, rows) - 1) / p.g);
    // pieces of one size for all samples, so that a short one has fewer: a share of the longest
    int longest = smp.len;
    if (ps.splits > 1) {
      __shared__ int most;
      if (threadIdx.x == 0) most = 0;
      __syncthreads();
      for (int b = threadIdx.x; b < pc.samples; b += kThreadsF) {
        const PagedSample s = paged_sample(pc, a.n_q, b, p.status);
        if (s.n > 0) atomicMax(&most, s.len);
      }
      __syncthreads();
      longest = most;
    }
    const int total = (kk.len1 + kKF - 1) / kKF, per = ((longest + kKF - 1) / kKF + ps.splits - 1) / ps.splits;
    kk.begin = min(total, it.split * per);
    kk.end = min(total, kk.begin + per);
    if (it.split > 0 && kk.begin == kk.end) {
      // a piece of weight 0
      for (int r = threadIdx.x; r < min(MR, rows - it.row0); r += kThreadsF) {
        const SegRow x = seg_row(p, 1, 0, it.h_kv, smp.q0 * p.g + it.row0 + r);
        p.part_ml[(int64_t)it.split * p.rows + (int64_t)x.t * a.N_h + x.h] = make_float2(-INFINITY, 0.f);
      }
      allow_next();
      return;
    }
    it.row0 += smp.q0 * p.g;
    row_end = smp.q0 * p.g + rows;
  } else {
    kk = seg_keys(p, ps, it, MR, kKF);
  }
  const int tx = threadIdx.x & 7, ty = threadIdx.x >> 3;
  const int b0 = it.block * ps.block_samples;
  auto row_of = [&](int r) {
    if constexpr (kPaged) {
      SegRow x = seg_row(p, 1, 0, it.h_kv, it.row0 + r);
      x.real = it.row0 + r < row_end;
      return x;
    } else {
      return seg_row(p, ps, it, it.row0 + r);
    }
  };

  for (int i = threadIdx.x; i < MR * (D / 4); i += kThreadsF) {
    const int r = i / (D / 4), c = (i % (D / 4)) * 4;
    const SegRow row = row_of(r);
    cp16(sQ + r * QS + c, (const float*)a.q + row.b * a.q_smp + row.t * a.q_tok + (int64_t)row.h * D + c, row.real ? 16u : 0u);
  }
  auto load_tile = [&](int t) {
    const int s = t >= kk.n0 ? 1 : 0;
    const int key0 = (s ? t - kk.n0 : t) * kKF;
    const int len = s ? kk.len1 : kk.len0;
    const int64_t idx = kPaged ? 0 : (s ? b0 : b0 / a.per_group);
    const float* kb = (const float*)a.k[s] + idx * a.k_smp[s] + (int64_t)it.h_kv * D;
    const float* vb = (const float*)a.v[s] + idx * a.v_smp[s] + (int64_t)it.h_kv * D;
    const int st = (t - kk.begin) & 1;
    for (int i = threadIdx.x; i < kKF * (D / 4); i += kThreadsF) {
      const int r = i / (D / 4), c = (i % (D / 4)) * 4;
      bool in = key0 + r < len;
      if constexpr (kPaged) {
        const int key = in ? key0 + r : 0;
        int page = in ? __ldg(pc.table + it.block * pc.table_stride + (key >> pc.page_shift)) : 0;
        if (in && (page < 0 || page >= pc.n_pages)) {
          atomicOr(p.status, ST_BAD_MAP);
          in = false;                // zeros
          page = 0;
        }
        const int64_t row = key & ((1 << pc.page_shift) - 1);
        cp16(sK + st * C::kK + r * QS + c, kb + page * pc.k_page + row * pc.k_tok + c, in ? 16u : 0u);
        cp16(sV + st * C::kV + r * D + c, vb + page * pc.v_page + row * pc.v_tok + c, in ? 16u : 0u);
      } else {
        const int64_t key = in ? key0 + r : 0;
        cp16(sK + st * C::kK + r * QS + c, kb + key * a.k_tok[s] + c, in ? 16u : 0u);
        cp16(sV + st * C::kV + r * D + c, vb + key * a.v_tok[s] + c, in ? 16u : 0u);
      }
    }
  };
  int lim1[RPT];
#pragma unroll
  for (int i = 0; i < RPT; ++i) {
    const SegRow row = row_of(ty + 16 * i);
    if constexpr (kPaged) lim1[i] = row.real ? paged_limit(a.causal, smp, row.t - smp.q0) : 0;
    else lim1[i] = seg_limit1(a, kk.end > kk.n0 ? seg_len(p, 1, row.b) : 0, row.t);
  }
  uint64_t o2[RPT][D / 16];                        // output columns 4 tx + 32 c + (0, 1) and (2, 3)
  float m[RPT], l[RPT];
#pragma unroll
  for (int i = 0; i < RPT; ++i) {
    m[i] = -INFINITY;
    l[i] = 0.f;
#pragma unroll
    for (int c = 0; c < D / 16; ++c) o2[i][c] = 0ull;
  }
  if (kk.begin < kk.end) load_tile(kk.begin);
  asm volatile("cp.async.commit_group;" ::: "memory");
  for (int t = kk.begin; t < kk.end; ++t) {
    __syncthreads();             // the stage about to be filled, and sP, have been read
    if (t + 1 < kk.end) load_tile(t + 1);
    asm volatile("cp.async.commit_group;" ::: "memory");
    asm volatile("cp.async.wait_group 1;" ::: "memory");
    __syncthreads();
    const int st = (t - kk.begin) & 1;
    const float* K = sK + st * C::kK;
    const float* V = sV + st * C::kV;
    // sums over even and odd elements side by side
    uint64_t sc2[RPT][4];
#pragma unroll
    for (int i = 0; i < RPT; ++i) sc2[i][0] = sc2[i][1] = sc2[i][2] = sc2[i][3] = 0ull;
#pragma unroll 4
    for (int d = 0; d < D; d += 4) {
      ulonglong2 q4[RPT], k4[4];
#pragma unroll
      for (int i = 0; i < RPT; ++i) q4[i] = *reinterpret_cast<const ulonglong2*>(sQ + (ty + 16 * i) * QS + d);
#pragma unroll
      for (int j = 0; j < 4; ++j) k4[j] = *reinterpret_cast<const ulonglong2*>(K + (tx + 8 * j) * QS + d);
#pragma unroll
      for (int i = 0; i < RPT; ++i) {
#pragma unroll
        for (int j = 0; j < 4; ++j) sc2[i][j] = fma2(q4[i].y, k4[j].y, fma2(q4[i].x, k4[j].x, sc2[i][j]));
      }
    }
    float sc[RPT][4];
#pragma unroll
    for (int i = 0; i < RPT; ++i) {
#pragma unroll
      for (int j = 0; j < 4; ++j) {
        float lo, hi;
        unpack2(sc2[i][j], lo, hi);
        sc[i][j] = lo + hi;
      }
    }
    const int seg = t >= kk.n0 ? 1 : 0;
    const int key0 = (seg ? t - kk.n0 : t) * kKF;
#pragma unroll
    for (int i = 0; i < RPT; ++i) {
      const int valid = (seg ? lim1[i] : kk.len0) - key0;
      float mx = -INFINITY;
#pragma unroll
      for (int j = 0; j < 4; ++j) {
        sc[i][j] = tx + 8 * j < valid ? sc[i][j] * p.scale_log2 : -INFINITY;
        mx = fmaxf(mx, sc[i][j]);
      }
#pragma unroll
      for (int s = 1; s < 8; s <<= 1) mx = fmaxf(mx, __shfl_xor_sync(0xffffffffu, mx, s));
      const float mn = fmaxf(m[i], mx);
      const float ref = mn == -INFINITY ? 0.f : mn;    // a row that has seen no key yet
      const float corr = exp2f(m[i] - ref);
      m[i] = mn;
      l[i] *= corr;
#pragma unroll
      for (int j = 0; j < 4; ++j) {
        const float e = exp2f(sc[i][j] - ref);
        l[i] += e;
        sP[(tx + 8 * j) * PS + ty * RPT + i] = e;
      }
      const uint64_t corr2 = pack2(corr, corr);
#pragma unroll
      for (int c = 0; c < D / 16; ++c) o2[i][c] = fma2(o2[i][c], corr2, 0ull);
    }
    __syncwarp();                // a warp reads only the P columns of its own rows
#pragma unroll 4
    for (int key = 0; key < kKF; ++key) {
      float pr[RPT];
      if constexpr (RPT == 4) {
        const float4 p4 = *reinterpret_cast<const float4*>(sP + key * PS + ty * 4);
        pr[0] = p4.x;
        pr[1] = p4.y;
        pr[2] = p4.z;
        pr[3] = p4.w;
      } else if constexpr (RPT == 2) {
        const float2 p2 = *reinterpret_cast<const float2*>(sP + key * PS + ty * 2);
        pr[0] = p2.x;
        pr[1] = p2.y;
      } else {
#pragma unroll
        for (int i = 0; i < RPT; ++i) pr[i] = sP[key * PS + ty * RPT + i];
      }
#pragma unroll
      for (int c = 0; c < D / 32; ++c) {
        const ulonglong2 v4 = *reinterpret_cast<const ulonglong2*>(V + key * D + c * 32 + tx * 4);
#pragma unroll
        for (int i = 0; i < RPT; ++i) {
          const uint64_t p2 = pack2(pr[i], pr[i]);
          o2[i][c * 2] = fma2(p2, v4.x, o2[i][c * 2]);
          o2[i][c * 2 + 1] = fma2(p2, v4.y, o2[i][c * 2 + 1]);
        }
      }
    }
  }
  asm volatile("cp.async.wait_all;" ::: "memory");
  allow_next();
#pragma unroll
  for (int i = 0; i < RPT; ++i) {
    float sum = l[i];
#pragma unroll
    for (int s = 1; s < 8; s <<= 1) sum += __shfl_xor_sync(0xffffffffu, sum, s);
    const SegRow row = row_of(ty + 16 * i);
    if (!row.real) continue;
    const int64_t gr = ((int64_t)row.b * a.n_q + row.t) * a.N_h + row.h;
    const int64_t pr = (int64_t)(ps.part0 + it.split) * p.rows + gr;
    float* dst = p.direct ? (float*)a.out + row.b * a.o_smp + row.t * a.o_tok + (int64_t)row.h * D : p.part_o + pr * D;
    const float inv = p.direct ? seg_inverse(sum) : 1.f;
#pragma unroll
    for (int c = 0; c < D / 32; ++c) {
      float4 w;
      unpack2(o2[i][c * 2], w.x, w.y);
      unpack2(o2[i][c * 2 + 1], w.z, w.w);
      *reinterpret_cast<float4*>(dst + c * 32 + tx * 4) = make_float4(w.x * inv, w.y * inv, w.z * inv, w.w * inv);
    }
    if (tx == 0) {
      if (!p.direct) p.part_ml[pr] = make_float2(m[i], sum);
      else if (a.lse) a.lse[((int64_t)row.b * a.N_h + row.h) * a.n_q + row.t] = seg_lse(m[i], sum);
    }
  }
  if (pass == 1) wait_previous();
}

template <int D, int RPT, bool kPaged>
cudaError_t launch_one(const SegParams& p, int pass, const CacheArg<kPaged>& c, cudaStream_t st, int* launches) {
  constexpr int smem = F32Cfg<D, RPT>::kBytes;
  static SmemOptIn opt_in;
  cudaError_t e = opt_in((const void*)seg_f32_kernel<D, RPT, kPaged>, smem, p.a.device);
  if (e != cudaSuccess) return e;
  ++*launches;
  if (pass == 1) return launch_after(seg_f32_kernel<D, RPT, kPaged>, dim3(p.pass[pass].items), dim3(kThreadsF), smem, st, p, pass, c);
  seg_f32_kernel<D, RPT, kPaged><<<p.pass[pass].items, kThreadsF, smem, st>>>(p, pass, c);
  return cudaGetLastError();
}
template <int D, bool kPaged>
cudaError_t launch_rows(const SegParams& p, int pass, const CacheArg<kPaged>& c, int tile_rows, cudaStream_t st, int* launches) {
  return tile_rows == 16 ? launch_one<D, 1, kPaged>(p, pass, c, st, launches)
                         : (tile_rows == 32 ? launch_one<D, 2, kPaged>(p, pass, c, st, launches) : launch_one<D, 4, kPaged>(p, pass, c, st, launches));
}
template <bool kPaged>
cudaError_t launch_dim(const SegParams& p, int pass, const CacheArg<kPaged>& c, int tile_rows, cudaStream_t st, int* launches) {
  switch (p.a.D) {
    case 32: return launch_rows<32, kPaged>(p, pass, c, tile_rows, st, launches);
    case 64: return launch_rows<64, kPaged>(p, pass, c, tile_rows, st, launches);
    case 128: return launch_rows<128, kPaged>(p, pass, c, tile_rows, st, launches);
    default: return cudaErrorInvalidConfiguration;
  }
}

}  // namespace

cudaError_t launch_seg_f32(const SegParams& p, int pass, int tile_rows, cudaStream_t st, int* launches) {
  return launch_dim<false>(p, pass, NoCache(), tile_rows, st, launches);
}
cudaError_t launch_paged_f32(const SegParams& p, const PagedCache& c, int tile_rows, cudaStream_t st, int* launches) {
  return launch_dim<true>(p, 0, c, tile_rows, st, launches);
}

}  // namespace swam
