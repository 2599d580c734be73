// Segment attention for bf16 tensors on warp-level matrix instructions (mma.sync m16n8k16), keys streamed once through
// shared memory: the kernel for few query rows per key/value head (single tokens, short chunks), for head dim 32, and the
// independent second opinion on the tcgen05 kernel.
//
// One CTA of WR * WK warps owns a row tile of 16 * WR rows and a piece of the keys.  WR warps lie along the rows and WK
// along the keys: with 16 rows or fewer every warp holds all rows and 16 keys of each tile, so that no key is multiplied
// twice; every warp keeps its own running maximum and sum, and the warps of a row are merged once at the end.  Key and value
// tiles (64 keys, or 128 with eight warps) arrive by 16-byte asynchronous copies into a ring of three stages; keys beyond the
// real length are filled with zeros, so whatever the padding holds (NaN included) never meets a product.
// Scores, maxima, sums and outputs are fp32; the probabilities are rounded to bf16 for the second product.
#include "seg_attn.cuh"

namespace swam {
namespace {

constexpr int kStagesM = 3;

__device__ __forceinline__ uint32_t smem_u32(const void* p) { return (uint32_t)__cvta_generic_to_shared(p); }
__device__ __forceinline__ void cp16(uint32_t dst, const void* src, uint32_t bytes) {
  asm volatile("cp.async.cg.shared.global [%0], [%1], 16, %2;" ::"r"(dst), "l"(src), "r"(bytes) : "memory");
}
__device__ __forceinline__ void ldsm4(uint32_t (&r)[4], uint32_t addr) {
  asm volatile("ldmatrix.sync.aligned.m8n8.x4.shared.b16 {%0, %1, %2, %3}, [%4];"
               : "=r"(r[0]), "=r"(r[1]), "=r"(r[2]), "=r"(r[3]) : "r"(addr) : "memory");
}
__device__ __forceinline__ void ldsm4_t(uint32_t (&r)[4], uint32_t addr) {
  asm volatile("ldmatrix.sync.aligned.m8n8.x4.trans.shared.b16 {%0, %1, %2, %3}, [%4];"
               : "=r"(r[0]), "=r"(r[1]), "=r"(r[2]), "=r"(r[3]) : "r"(addr) : "memory");
}
__device__ __forceinline__ void mma_bf16(float (&c)[4], const uint32_t (&a)[4], uint32_t b0, uint32_t b1) {
  asm volatile("mma.sync.aligned.m16n8k16.row.col.f32.bf16.bf16.f32 {%0, %1, %2, %3}, {%4, %5, %6, %7}, {%8, %9}, {%0, %1, %2, %3};"
               : "+f"(c[0]), "+f"(c[1]), "+f"(c[2]), "+f"(c[3]) : "r"(a[0]), "r"(a[1]), "r"(a[2]), "r"(a[3]), "r"(b0), "r"(b1));
}
__device__ __forceinline__ uint32_t pack_pair(float lo, float hi) {
  uint32_t r;
  asm("cvt.rn.bf16x2.f32 %0, %1, %2;" : "=r"(r) : "f"(hi), "f"(lo));
  return r;
}

// byte offset of 16-byte chunk c of row r in a tile of D-element rows: rows of 128 bytes or more permute their chunks by
// r % 8, 64-byte rows (head dim 32) by (r / 2) % 4; both make eight consecutive rows of one chunk column conflict-free
template <int D>
__device__ __forceinline__ uint32_t tile_off(int r, int c) {
  return (uint32_t)(r * D * 2 + ((D >= 64 ? (c ^ (r & 7)) : (c ^ ((r >> 1) & 3))) << 4));
}

template <int D, int WR, int WK>
struct MmaCfg {
  static constexpr int kThreads = 32 * WR * WK, MR = 16 * WR;
  static constexpr int KT = WR == 1 ? 16 * WK : 64;      // keys per tile
  static constexpr int kRing = kStagesM * 2 * KT * D * 2, kMerge = WK * MR * (D + 4 + 2) * 4;
  static constexpr int kBytes = kRing > kMerge ? kRing : kMerge;
};

template <int D, int WR, int WK>
__global__ void __launch_bounds__(32 * WR * WK) seg_mma_kernel(const __grid_constant__ SegParams p, const int pass) {
  using C = MmaCfg<D, WR, WK>;
  constexpr int MR = C::MR, kKT = C::KT, KW = kKT / WK, kThreadsM = C::kThreads;
  constexpr int CPR = D / 8;                       // 16-byte chunks per row
  constexpr int kTileB = kKT * D * 2;              // bytes of a key or value tile
  extern __shared__ unsigned char smem_raw[];
  const uint32_t s0 = smem_u32(smem_raw);
  if (p.early && pass == 0) allow_next();
  const SegPass& ps = p.pass[pass];
  const SegArgs& a = p.a;
  const SegItem it = seg_item(ps, a.N_kv, MR, blockIdx.x);
  const SegKeys kk = seg_keys(p, ps, it, MR, kKT);
  const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
  const int wr = warp % WR, wk = warp / WR;
  const int b0 = it.block * ps.block_samples;

  // A thread copies the same 16-byte chunk of every RS-th row of a tile, so that one pointer per tensor and a fixed step
  // address all its copies.  lr0, lc: its first row and its chunk.
  constexpr int RS = kThreadsM / CPR, NL = kKT / RS;
  const int lr0 = threadIdx.x / CPR, lc = threadIdx.x % CPR;
  int next_seg = -1;                               // segment that the pointers stand in
  const __nv_bfloat16 *kp = nullptr, *vp = nullptr;
  int64_t k_step = 0, v_step = 0;
  int left = 0;                                    // real keys from the thread's first row of the tile on
  uint32_t stage_off = 0;
  auto load_tile = [&](int t) {
    const int sg = t >= kk.n0 ? 1 : 0;
    if (sg != next_seg) {
      next_seg = sg;
      const int key0 = (sg ? t - kk.n0 : t) * kKT + lr0;
      const int64_t idx = sg ? b0 : b0 / a.per_group;
      kp = (const __nv_bfloat16*)a.k[sg] + idx * a.k_smp[sg] + (int64_t)it.h_kv * D + key0 * a.k_tok[sg] + lc * 8;
      vp = (const __nv_bfloat16*)a.v[sg] + idx * a.v_smp[sg] + (int64_t)it.h_kv * D + key0 * a.v_tok[sg] + lc * 8;
      k_step = RS * a.k_tok[sg];
      v_step = RS * a.v_tok[sg];
      left = (sg ? kk.len1 : kk.len0) - key0;
    }
    const uint32_t ks = s0 + stage_off, vs = ks + kTileB;
    stage_off = stage_off + 2 * kTileB == kStagesM * 2 * kTileB ? 0 : stage_off + 2 * kTileB;
#pragma unroll
    for (int i = 0; i < NL; ++i) {
      const bool in = i * RS < left;
      const uint32_t off = tile_off<D>(lr0 + i * RS, lc);
      // (rows behind the real ones read nothing; the address stays inside the tensor)
      cp16(ks + off, in ? kp : (const __nv_bfloat16*)a.k[sg], in ? 16u : 0u);
      cp16(vs + off, in ? vp : (const __nv_bfloat16*)a.v[sg], in ? 16u : 0u);
      kp += k_step;
      vp += v_step;
    }
    left -= kKT;
  };

#pragma unroll
  for (int i = 0; i < kStagesM - 1; ++i) {
    if (kk.begin + i < kk.end) load_tile(kk.begin + i);
    asm volatile("cp.async.commit_group;" ::: "memory");
  }
  // this thread's two rows (accumulator rows lane / 4 and lane / 4 + 8 of the warp's 16), their queries as A fragments
  uint32_t qf[D / 16][4];
  int lim1[2];
#pragma unroll
  for (int i = 0; i < 2; ++i) {
    const SegRow r = seg_row(p, ps, it, it.row0 + wr * 16 + (lane >> 2) + 8 * i);
    lim1[i] = seg_limit1(a, kk.end > kk.n0 ? seg_len(p, 1, r.b) : 0, r.t);
    const uint32_t* src = reinterpret_cast<const uint32_t*>((const __nv_bfloat16*)a.q + r.b * a.q_smp + r.t * a.q_tok + (int64_t)r.h * D);
#pragma unroll
    for (int ks = 0; ks < D / 16; ++ks) {
      qf[ks][i] = r.real ? src[ks * 8 + (lane & 3)] : 0u;
      qf[ks][i + 2] = r.real ? src[ks * 8 + 4 + (lane & 3)] : 0u;
    }
  }

  float o[D / 8][4];
#pragma unroll
  for (int i = 0; i < D / 8; ++i) o[i][0] = o[i][1] = o[i][2] = o[i][3] = 0.f;
  float m[2] = {-INFINITY, -INFINITY}, l[2] = {0.f, 0.f};

  for (int t = kk.begin; t < kk.end; ++t) {
    asm volatile("cp.async.wait_group %0;" ::"n"(kStagesM - 2) : "memory");
    __syncthreads();
    if (t + kStagesM - 1 < kk.end) load_tile(t + kStagesM - 1);
    asm volatile("cp.async.commit_group;" ::: "memory");
    const int seg = t >= kk.n0 ? 1 : 0;
    const int key0 = (seg ? t - kk.n0 : t) * kKT + wk * KW;       // first key of this warp
    if (key0 >= (seg ? kk.len1 : kk.len0)) continue;              // none of them is real
    const uint32_t ks = s0 + (uint32_t)((t - kk.begin) % kStagesM) * 2 * kTileB, vs = ks + kTileB;

    float sc[KW / 8][4];
#pragma unroll
    for (int nb = 0; nb < KW / 16; ++nb) {
#pragma unroll
      for (int e = 0; e < 4; ++e) sc[2 * nb][e] = sc[2 * nb + 1][e] = 0.f;
#pragma unroll
      for (int kd = 0; kd < D / 16; ++kd) {
        uint32_t f[4];
        ldsm4(f, ks + tile_off<D>(wk * KW + nb * 16 + (lane & 7) + ((lane >> 4) << 3), kd * 2 + ((lane >> 3) & 1)));
        mma_bf16(sc[2 * nb], qf[kd], f[0], f[1]);
        mma_bf16(sc[2 * nb + 1], qf[kd], f[2], f[3]);
      }
    }
    const int v0 = (seg ? lim1[0] : kk.len0) - key0, v1 = (seg ? lim1[1] : kk.len0) - key0;   // keys of the warp's range the rows see
    if (min(v0, v1) < KW) {
#pragma unroll
      for (int nb = 0; nb < KW / 8; ++nb) {
        const int c = nb * 8 + (lane & 3) * 2;
        if (c >= v0) sc[nb][0] = -INFINITY;
        if (c + 1 >= v0) sc[nb][1] = -INFINITY;
        if (c >= v1) sc[nb][2] = -INFINITY;
        if (c + 1 >= v1) sc[nb][3] = -INFINITY;
      }
    }
    float corr[2], ref[2];
#pragma unroll
    for (int i = 0; i < 2; ++i) {
      float mx = -INFINITY;
#pragma unroll
      for (int nb = 0; nb < KW / 8; ++nb) mx = fmaxf(mx, fmaxf(sc[nb][2 * i], sc[nb][2 * i + 1]));
      mx = fmaxf(mx, __shfl_xor_sync(0xffffffffu, mx, 1));
      mx = fmaxf(mx, __shfl_xor_sync(0xffffffffu, mx, 2));
      const float mn = fmaxf(m[i], mx * p.scale_log2);
      ref[i] = mn == -INFINITY ? 0.f : mn;      // a row that has seen no key yet: every exponent stays -inf
      corr[i] = exp2f(m[i] - ref[i]);
      m[i] = mn;
      l[i] *= corr[i];
    }
#pragma unroll
    for (int nb = 0; nb < KW / 8; ++nb) {
#pragma unroll
      for (int e = 0; e < 4; ++e) {
        sc[nb][e] = exp2f(fmaf(sc[nb][e], p.scale_log2, -ref[e >> 1]));
        l[e >> 1] += sc[nb][e];
      }
    }
    if (__any_sync(0xffffffffu, corr[0] != 1.f || corr[1] != 1.f))   // rare after the first tiles
#pragma unroll
    for (int i = 0; i < D / 8; ++i) {
      o[i][0] *= corr[0];
      o[i][1] *= corr[0];
      o[i][2] *= corr[1];
      o[i][3] *= corr[1];
    }
#pragma unroll
    for (int nb = 0; nb < KW / 16; ++nb) {
      const uint32_t pf[4] = {pack_pair(sc[2 * nb][0], sc[2 * nb][1]), pack_pair(sc[2 * nb][2], sc[2 * nb][3]),
                              pack_pair(sc[2 * nb + 1][0], sc[2 * nb + 1][1]), pack_pair(sc[2 * nb + 1][2], sc[2 * nb + 1][3])};
#pragma unroll
      for (int dn = 0; dn < D / 16; ++dn) {
        uint32_t f[4];
        ldsm4_t(f, vs + tile_off<D>(wk * KW + nb * 16 + (lane & 7) + (((lane >> 3) & 1) << 3), dn * 2 + (lane >> 4)));
        mma_bf16(o[2 * dn], pf, f[0], f[1]);
        mma_bf16(o[2 * dn + 1], pf, f[2], f[3]);
      }
    }
  }
#pragma unroll
  for (int i = 0; i < 2; ++i) {
    l[i] += __shfl_xor_sync(0xffffffffu, l[i], 1);
    l[i] += __shfl_xor_sync(0xffffffffu, l[i], 2);
  }

  allow_next();
  // merge the WK warps of each row through shared memory (the ring is free by now), then write
  asm volatile("cp.async.wait_all;" ::: "memory");
  __syncthreads();
  constexpr int OS = D + 4;                        // padded row of partial outputs
  float* so = reinterpret_cast<float*>(smem_raw);  // [WK][MR][OS]
  float* sm = so + WK * MR * OS;                   // [WK][MR] maxima
  float* sl = sm + WK * MR;                        // [WK][MR] sums
#pragma unroll
  for (int i = 0; i < 2; ++i) {
    const int r = wk * MR + wr * 16 + (lane >> 2) + 8 * i;
    if ((lane & 3) == 0) {
      sm[r] = m[i];
      sl[r] = l[i];
    }
#pragma unroll
    for (int dn = 0; dn < D / 8; ++dn)
      *reinterpret_cast<float2*>(so + r * OS + dn * 8 + (lane & 3) * 2) = make_float2(o[dn][2 * i], o[dn][2 * i + 1]);
  }
  __syncthreads();
  constexpr int C8 = D / 8;                        // eight columns per thread and step
  for (int i = threadIdx.x; i < MR * C8; i += kThreadsM) {
    const int r = i / C8, c = (i % C8) * 8;
    const SegRow row = seg_row(p, ps, it, it.row0 + r);
    if (!row.real) continue;
    float mx = -INFINITY;
#pragma unroll
    for (int w = 0; w < WK; ++w) mx = fmaxf(mx, sm[w * MR + r]);
    float sum = 0.f, acc[8];
#pragma unroll
    for (int e = 0; e < 8; ++e) acc[e] = 0.f;
#pragma unroll
    for (int w = 0; w < WK; ++w) {
      const float f = mx == -INFINITY ? 0.f : exp2f(sm[w * MR + r] - mx);
      sum += f * sl[w * MR + r];
#pragma unroll
      for (int e = 0; e < 8; ++e) acc[e] += f * so[(w * MR + r) * OS + c + e];
    }
    const int64_t gr = ((int64_t)row.b * a.n_q + row.t) * a.N_h + row.h;
    if (p.direct) {
      const float inv = sum > 0.f ? 1.f / sum : 0.f;
      uint4 w;
      w.x = pack_pair(acc[0] * inv, acc[1] * inv);
      w.y = pack_pair(acc[2] * inv, acc[3] * inv);
      w.z = pack_pair(acc[4] * inv, acc[5] * inv);
      w.w = pack_pair(acc[6] * inv, acc[7] * inv);
      *reinterpret_cast<uint4*>((__nv_bfloat16*)a.out + row.b * a.o_smp + row.t * a.o_tok + (int64_t)row.h * D + c) = w;
      if (a.lse && c == 0)
        a.lse[((int64_t)row.b * a.N_h + row.h) * a.n_q + row.t] = sum > 0.f ? (mx + log2f(sum)) * 0.6931471805599453f : -INFINITY;
    } else {
      const int64_t pr = (int64_t)(ps.part0 + it.split) * p.rows + gr;
      float* dst = p.part_o + pr * D + c;
      *reinterpret_cast<float4*>(dst) = make_float4(acc[0], acc[1], acc[2], acc[3]);
      *reinterpret_cast<float4*>(dst + 4) = make_float4(acc[4], acc[5], acc[6], acc[7]);
      if (c == 0) p.part_ml[pr] = make_float2(mx, sum);
    }
  }
  if (pass == 1) wait_previous();
}

template <int D, int WR, int WK>
cudaError_t launch_one(const SegParams& p, int pass, cudaStream_t st, int* launches) {
  using C = MmaCfg<D, WR, WK>;
  cudaError_t e = cudaFuncSetAttribute(seg_mma_kernel<D, WR, WK>, cudaFuncAttributeMaxDynamicSharedMemorySize, C::kBytes);
  if (e != cudaSuccess) return e;
  ++*launches;
  if (pass == 1) return launch_after(seg_mma_kernel<D, WR, WK>, dim3(p.pass[pass].items), dim3(C::kThreads), C::kBytes, st, p, pass);
  seg_mma_kernel<D, WR, WK><<<p.pass[pass].items, C::kThreads, C::kBytes, st>>>(p, pass);
  return cudaGetLastError();
}
template <int D>
cudaError_t launch_rows(const SegParams& p, int pass, int rows, bool wide, cudaStream_t st, int* launches) {
  switch (rows) {
    case 16: return wide ? launch_one<D, 1, 8>(p, pass, st, launches) : launch_one<D, 1, 4>(p, pass, st, launches);
    case 32: return launch_one<D, 2, 2>(p, pass, st, launches);
    default: return launch_one<D, 4, 1>(p, pass, st, launches);
  }
}

}  // namespace

cudaError_t launch_seg_mma(const SegParams& p, int pass, int tile_rows, bool wide, cudaStream_t st, int* launches) {
  switch (p.a.D) {
    case 32: return launch_rows<32>(p, pass, tile_rows, wide, st, launches);
    case 64: return launch_rows<64>(p, pass, tile_rows, wide, st, launches);
    case 128: return launch_rows<128>(p, pass, tile_rows, wide, st, launches);
    default: return cudaErrorInvalidConfiguration;
  }
}

}  // namespace swam
