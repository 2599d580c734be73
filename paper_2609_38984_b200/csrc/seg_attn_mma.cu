// Segment attention for bf16 tensors on warp-level matrix instructions (mma.sync m16n8k16), keys streamed once through
// shared memory: the kernel for few query rows per key/value head (single tokens, short chunks), for head dim 32, and the
// independent second opinion on the tcgen05 kernel.
//
// One CTA of WR * WK warps owns a row tile of 16 * WR rows and a piece of the keys.  WR warps lie along the rows and WK
// along the keys: with 16 rows or fewer every warp holds all rows and 16 keys of each tile, so that no key is multiplied
// twice; every warp keeps its own running maximum and sum, and the warps of a row are merged once at the end.  Key and value
// tiles (64 keys, or 128 with eight warps) arrive by TMA in a ring of three stages.  (Copies by the threads themselves kept the
// load/store unit busy beside the products: 62 us instead of 57 for 64 single tokens behind 8192 shared and 16 to 1024 own keys,
// 32 query heads on 8 of 128.)
// Rows of V behind the real length become zeros in shared memory, so whatever the padding holds (NaN included) never meets a
// product.
// Scores, maxima, sums and outputs are fp32; the probabilities are rounded to bf16 for the second product (the operand type
// of the matrix instruction; half a step, 2^-8, of each weight).
// What bounds it: HBM.  64 single tokens (32 query heads on 8 of 128) with 4096 keys each stream at 6.9 TB/s, with 512 keys
// at 4.4 (some 10 us of every call are launch, first loads and the last CTAs).
#include <string.h>

#include "seg_maps.cuh"

namespace swam {
namespace {

constexpr int kStagesM = 3;

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
// byte offset of 16-byte chunk c of row r in a tile of KT rows, as the tensor maps lay it out: blocks of 64 columns whose
// 128-byte rows permute their chunks by r % 8, or (head dim 32) 64-byte rows that do so by (r / 2) % 4; both make eight
// consecutive rows of one chunk column conflict-free
template <int D, int KT>
__device__ __forceinline__ uint32_t tile_off(int r, int c) {
  if (D == 32) return (uint32_t)(r * 64 + ((c ^ ((r >> 1) & 3)) << 4));
  return (uint32_t)((c >> 3) * KT * 128 + r * 128 + (((c & 7) ^ (r & 7)) << 4));
}

template <int D, int WR, int WK>
struct MmaCfg {
  static constexpr int kThreads = 32 * WR * WK, MR = 16 * WR;
  static constexpr int KT = WR == 1 ? 16 * WK : 64;      // keys per tile
  static constexpr int kRing = kStagesM * 2 * KT * D * 2, kMerge = WK * MR * (D + 4 + 2) * 4;
  static constexpr int kBytes = (kRing > kMerge ? kRing : kMerge) + 1024 /*alignment*/ + 64 /*barriers*/;
};

template <int D, int WR, int WK>
__global__ void __launch_bounds__(32 * WR * WK) seg_mma_kernel(const __grid_constant__ CUtensorMap map_k0, const __grid_constant__ CUtensorMap map_v0,
                               const __grid_constant__ CUtensorMap map_k1, const __grid_constant__ CUtensorMap map_v1,
                               const __grid_constant__ SegParams p, const int pass) {
  using C = MmaCfg<D, WR, WK>;
  constexpr int MR = C::MR, kKT = C::KT, KW = kKT / WK, kThreadsM = C::kThreads;
  constexpr int CPR = D / 8;                       // 16-byte chunks per row
  constexpr int kTileB = kKT * D * 2;              // bytes of a key or value tile
  extern __shared__ unsigned char smem_raw[];
  const uint32_t s0 = (smem_addr(smem_raw) + 1023u) & ~1023u;
  unsigned char* base = smem_raw + (s0 - smem_addr(smem_raw));
  const uint32_t bars = s0 + (uint32_t)(C::kBytes - 1024 - 64);
  volatile int* abort_flag = reinterpret_cast<volatile int*>(base + C::kBytes - 1024 - 16);
  if (threadIdx.x == 0) {
    for (int i = 0; i < kStagesM; ++i) mbar_init(bars + 8 * i, 1);
    *abort_flag = 0;
    asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
  }
  if (p.early && pass == 0) allow_next();
  const SegPass& ps = p.pass[pass];
  const SegArgs& a = p.a;
  const SegItem it = seg_item(ps, a.N_kv, MR, blockIdx.x);
  const SegKeys kk = seg_keys(p, ps, it, MR, kKT);
  const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
  const int wr = warp % WR, wk = warp / WR;
  const int b0 = it.block * ps.block_samples;

  constexpr int DB = D == 32 ? 1 : D / 64, kCols = D == 32 ? 32 : 64;       // boxes per tile and their columns
  auto load_tile = [&](int t) {                    // one thread
    const bool s1 = t >= kk.n0;
    const int st = (t - kk.begin) % kStagesM, key0 = (s1 ? t - kk.n0 : t) * kKT, idx = s1 ? b0 : b0 / a.per_group;
    const uint32_t ks = s0 + (uint32_t)st * 2 * kTileB, bar = bars + 8 * st;
    mbar_expect_tx(bar, 2 * kTileB);
#pragma unroll
    for (int db = 0; db < DB; ++db) {
      tma_load_4d(ks + db * kKT * 128, s1 ? &map_k1 : &map_k0, bar, db * kCols, key0, it.h_kv, idx);
      tma_load_4d(ks + kTileB + db * kKT * 128, s1 ? &map_v1 : &map_v0, bar, db * kCols, key0, it.h_kv, idx);
    }
  };
  __syncthreads();                                 // the barriers are set up
  if (threadIdx.x == 0) {
    for (int i = 0; i < kStagesM - 1; ++i)
      if (kk.begin + i < kk.end) load_tile(kk.begin + i);
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
  bool big = false;                                // some row's reference is large: see kSegBig

  for (int t = kk.begin; t < kk.end; ++t) {
    const int st = (t - kk.begin) % kStagesM;
    const bool ok = mbar_wait(bars + 8 * st, ((t - kk.begin) / kStagesM) & 1, abort_flag);
    if (!__syncthreads_and(ok ? 1 : 0)) {          // (and every warp is through with the tile before)
      if (threadIdx.x == 0) atomicOr(p.status, ST_TIMEOUT);
      // the copies in flight write to memory that is used again below, and must not outlive the CTA
      drain_loads(bars, kStagesM, min(kk.end, t + kStagesM - 1) - kk.begin);
      break;
    }
    if (threadIdx.x == 0 && t + kStagesM - 1 < kk.end) load_tile(t + kStagesM - 1);
    const int seg = t >= kk.n0 ? 1 : 0;
    const int key0 = (seg ? t - kk.n0 : t) * kKT + wk * KW;       // first key of this warp
    const uint32_t ks = s0 + (uint32_t)st * 2 * kTileB, vs = ks + kTileB;
    const int len = seg ? kk.len1 : kk.len0, real = len - (seg ? t - kk.n0 : t) * kKT;       // real keys, and those of this tile
    if (real < kKT && len < a.n[seg]) {                           // the tile ends inside its tensor
      for (int i = threadIdx.x; i < (kKT - real) * CPR; i += kThreadsM)
        st_shared_16(vs + tile_off<D, kKT>(real + i / CPR, i % CPR), 0u, 0u, 0u, 0u);
      fence_proxy_async();                                        // the stage's next load comes through the other proxy
      __syncthreads();
    }
    if (key0 >= len) continue;                                    // none of this warp's keys is real

    float sc[KW / 8][4];
#pragma unroll
    for (int nb = 0; nb < KW / 16; ++nb) {
#pragma unroll
      for (int e = 0; e < 4; ++e) sc[2 * nb][e] = sc[2 * nb + 1][e] = 0.f;
#pragma unroll
      for (int kd = 0; kd < D / 16; ++kd) {
        uint32_t f[4];
        ldsm4(f, ks + tile_off<D, kKT>(wk * KW + nb * 16 + (lane & 7) + ((lane >> 4) << 3), kd * 2 + ((lane >> 3) & 1)));
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
      corr[i] = ex2(m[i] - ref[i]);
      m[i] = mn;
      l[i] *= corr[i];
    }
    const bool moved = __any_sync(0xffffffffu, corr[0] != 1.f || corr[1] != 1.f);       // rare after the first tiles
    if (moved) big = __any_sync(0xffffffffu, !(fmaxf(fabsf(ref[0]), fabsf(ref[1])) < kSegBig));
    float scale = p.scale_log2;
    if (big) {
      scale = 1.f;
#pragma unroll
      for (int nb = 0; nb < KW / 8; ++nb) {
#pragma unroll
        for (int e = 0; e < 4; ++e) sc[nb][e] *= p.scale_log2;
      }
    }
#pragma unroll
    for (int nb = 0; nb < KW / 8; ++nb) {
#pragma unroll
      for (int e = 0; e < 4; ++e) {
        sc[nb][e] = ex2(fmaf(sc[nb][e], scale, -ref[e >> 1]));
        l[e >> 1] += sc[nb][e];
      }
    }
    if (moved)
#pragma unroll
    for (int i = 0; i < D / 8; ++i) {
      o[i][0] *= corr[0];
      o[i][1] *= corr[0];
      o[i][2] *= corr[1];
      o[i][3] *= corr[1];
    }
#pragma unroll
    for (int nb = 0; nb < KW / 16; ++nb) {
      const uint32_t pf[4] = {pack_bf16x2(sc[2 * nb][0], sc[2 * nb][1]), pack_bf16x2(sc[2 * nb][2], sc[2 * nb][3]),
                              pack_bf16x2(sc[2 * nb + 1][0], sc[2 * nb + 1][1]), pack_bf16x2(sc[2 * nb + 1][2], sc[2 * nb + 1][3])};
#pragma unroll
      for (int dn = 0; dn < D / 16; ++dn) {
        uint32_t f[4];
        ldsm4_t(f, vs + tile_off<D, kKT>(wk * KW + nb * 16 + (lane & 7) + (((lane >> 3) & 1) << 3), dn * 2 + (lane >> 4)));
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
  __syncthreads();
  constexpr int OS = D + 4;                        // padded row of partial outputs
  float* so = reinterpret_cast<float*>(base);  // [WK][MR][OS]
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
      const float inv = seg_inverse(sum);
      uint4 w;
      w.x = pack_bf16x2(acc[0] * inv, acc[1] * inv);
      w.y = pack_bf16x2(acc[2] * inv, acc[3] * inv);
      w.z = pack_bf16x2(acc[4] * inv, acc[5] * inv);
      w.w = pack_bf16x2(acc[6] * inv, acc[7] * inv);
      *reinterpret_cast<uint4*>((__nv_bfloat16*)a.out + row.b * a.o_smp + row.t * a.o_tok + (int64_t)row.h * D + c) = w;
      if (a.lse && c == 0) a.lse[((int64_t)row.b * a.N_h + row.h) * a.n_q + row.t] = seg_lse(mx, sum);
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
  const SegArgs& a = p.a;
  CUtensorMap mk[2], mv[2];
  memset(mk, 0, sizeof(mk));       // a segment without keys: its maps are never used
  memset(mv, 0, sizeof(mv));
  for (int s = p.pass[pass].seg_lo; s <= p.pass[pass].seg_hi; ++s) {
    const int blocks = s == 0 ? a.B / a.per_group : a.B;
    if (a.n[s] > 0 && (!make_kv_map(&mk[s], a.k[s], blocks, a.n[s], a.N_kv, D, a.k_tok[s], a.k_smp[s], C::KT) ||
                       !make_kv_map(&mv[s], a.v[s], blocks, a.n[s], a.N_kv, D, a.v_tok[s], a.v_smp[s], C::KT)))
      return cudaErrorInvalidValue;
  }
  static SmemOptIn opt_in;
  cudaError_t e = opt_in((const void*)seg_mma_kernel<D, WR, WK>, C::kBytes, a.device);
  if (e != cudaSuccess) return e;
  const dim3 grid(p.pass[pass].items), block(C::kThreads);
  ++*launches;
  if (pass == 1) return launch_after(seg_mma_kernel<D, WR, WK>, grid, block, C::kBytes, st, mk[0], mv[0], mk[1], mv[1], p, pass);
  seg_mma_kernel<D, WR, WK><<<grid, block, C::kBytes, st>>>(mk[0], mv[0], mk[1], mv[1], p, pass);
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
