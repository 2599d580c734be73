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
// tiles 92.  (Compiled to 128 registers, that instance, <64, 4>, spills 12 bytes a thread and loads 24; <128, 1> spills 4.)
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

template <int D, int RPT>
__global__ void __launch_bounds__(kThreadsF) seg_f32_kernel(const __grid_constant__ SegParams p, const int pass) {
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
  const SegItem it = seg_item(ps, a.N_kv, MR, blockIdx.x);
  const SegKeys kk = seg_keys(p, ps, it, MR, kKF);
  const int tx = threadIdx.x & 7, ty = threadIdx.x >> 3;
  const int b0 = it.block * ps.block_samples;

  for (int i = threadIdx.x; i < MR * (D / 4); i += kThreadsF) {
    const int r = i / (D / 4), c = (i % (D / 4)) * 4;
    const SegRow row = seg_row(p, ps, it, it.row0 + r);
    cp16(sQ + r * QS + c, (const float*)a.q + row.b * a.q_smp + row.t * a.q_tok + (int64_t)row.h * D + c, row.real ? 16u : 0u);
  }
  auto load_tile = [&](int t) {
    const int s = t >= kk.n0 ? 1 : 0;
    const int key0 = (s ? t - kk.n0 : t) * kKF;
    const int len = s ? kk.len1 : kk.len0;
    const int64_t idx = s ? b0 : b0 / a.per_group;
    const float* kb = (const float*)a.k[s] + idx * a.k_smp[s] + (int64_t)it.h_kv * D;
    const float* vb = (const float*)a.v[s] + idx * a.v_smp[s] + (int64_t)it.h_kv * D;
    const int st = (t - kk.begin) & 1;
    for (int i = threadIdx.x; i < kKF * (D / 4); i += kThreadsF) {
      const int r = i / (D / 4), c = (i % (D / 4)) * 4;
      const bool in = key0 + r < len;
      const int64_t key = in ? key0 + r : 0;
      cp16(sK + st * C::kK + r * QS + c, kb + key * a.k_tok[s] + c, in ? 16u : 0u);
      cp16(sV + st * C::kV + r * D + c, vb + key * a.v_tok[s] + c, in ? 16u : 0u);
    }
  };
  int lim1[RPT];
#pragma unroll
  for (int i = 0; i < RPT; ++i) {
    const SegRow row = seg_row(p, ps, it, it.row0 + ty + 16 * i);
    lim1[i] = seg_limit1(a, kk.end > kk.n0 ? seg_len(p, 1, row.b) : 0, row.t);
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
    const SegRow row = seg_row(p, ps, it, it.row0 + ty + 16 * i);
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

template <int D, int RPT>
cudaError_t launch_one(const SegParams& p, int pass, cudaStream_t st, int* launches) {
  constexpr int smem = F32Cfg<D, RPT>::kBytes;
  static SmemOptIn opt_in;
  cudaError_t e = opt_in((const void*)seg_f32_kernel<D, RPT>, smem, p.a.device);
  if (e != cudaSuccess) return e;
  ++*launches;
  if (pass == 1) return launch_after(seg_f32_kernel<D, RPT>, dim3(p.pass[pass].items), dim3(kThreadsF), smem, st, p, pass);
  seg_f32_kernel<D, RPT><<<p.pass[pass].items, kThreadsF, smem, st>>>(p, pass);
  return cudaGetLastError();
}
template <int D>
cudaError_t launch_rows(const SegParams& p, int pass, int tile_rows, cudaStream_t st, int* launches) {
  return tile_rows == 16 ? launch_one<D, 1>(p, pass, st, launches)
                         : (tile_rows == 32 ? launch_one<D, 2>(p, pass, st, launches) : launch_one<D, 4>(p, pass, st, launches));
}

}  // namespace

cudaError_t launch_seg_f32(const SegParams& p, int pass, int tile_rows, cudaStream_t st, int* launches) {
  switch (p.a.D) {
    case 32: return launch_rows<32>(p, pass, tile_rows, st, launches);
    case 64: return launch_rows<64>(p, pass, tile_rows, st, launches);
    case 128: return launch_rows<128>(p, pass, tile_rows, st, launches);
    default: return cudaErrorInvalidConfiguration;
  }
}

}  // namespace swam
