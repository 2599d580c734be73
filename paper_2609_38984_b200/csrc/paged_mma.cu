// Attention of few new tokens to paged keys, bf16, on warp-level matrix instructions: the kernel for single tokens and short chunks,
// and the independent second opinion on the tcgen05 kernel.
//
// The new tokens' rows of a sample and key/value head, in the order (token, head of the group), are cut into row tiles of 16 * WR
// rows.  A unit of work is a tile of 64 or 128 keys of a row tile, in the order (sample, key/value head, row tile, key tile); `shares` CTAs
// own equal stretches of that sequence, so that samples of any lengths load the SMs evenly.  Lengths are on the device: every
// CTA adds up the samples' units and finds its own first one.  A CTA keeps one pipeline of TMA loads running over the borders of its
// row tiles; keys arrive page by page through the table.
// A row tile that one CTA holds as a whole is finished there.  One that is cut leaves an unnormalised fp32 piece per CTA, which a second
// kernel joins: the block with the number of the CTA that holds the first piece.  A CTA has two pieces at most (it may end one row tile
// and begin another), so the scratch does not depend on the lengths.
// Inside a CTA a fifth warp issues the loads, a box for K and one for V per page, into a ring of stages; four warps multiply: WR along
// the rows and WK along the keys of a tile (WR * WK = 4), each with its own running maximum and sum.  They never wait for one another
// inside a row tile; its end merges them through the ring stage that was read last, which is given back only then.
// Rows of V behind the last key become zeros in shared memory (each warp's own ones), so whatever a page holds there (NaN included) never
// meets a product.
// Up to eight rows (WR = 0: single tokens of grouped heads) are the narrow side of the products: S^T = K Q^T and O^T = V^T P^T, 16 keys
// and 16 columns by 8 rows, half the instructions and exponentials of 16 rows; P^T becomes an operand by a transpose in registers.
// Scores, maxima, sums and outputs are fp32; the probabilities are rounded to bf16 for the second product (the operand type of
// the matrix instruction; half a step, 2^-8, of each weight).
// What bounds it: HBM.  64 single tokens, 32 heads on 8 of 128, 16 to 8192 keys (1.08 GB): 168 us of streaming at 6.4 TB/s, 177 with the
// join; two samples of 100001 and 131072 keys 155 us.  With 16 tokens a page the same call takes 177 us, 205 when the math warps issued
// the loads, two boxes for each of K and V.  Head dim 64 reaches 4.4 to 4.8 TB/s and 32 2.7 to 3.4: units go through a head's keys before the
// next head's, so that a CTA reads 128 or 64 bytes of a token's row at a time.  The narrow form
// changes nothing where memory bounds; it saves registers and a microsecond of the smallest calls (one sample of 501 keys: 11 us).  Short and
// ordinary histories are bound by the start, in which every CTA adds up the samples before its first load, and by the join: 51 samples of 62 to
// 153 keys 12 us, 30 of 900 to 1300 keys, 5 key/value heads of 128, 85 MB in 25 us.
// Two CTAs an SM leave 168 registers; instances with more rows a warp spill: <128, 4> 284 bytes a thread (236 loaded), <128, 2> 92 (96),
// <64, 4> 88 (92), the others nothing.
#include <string.h>

#include "seg_maps.cuh"
#include "seg_mma.cuh"

namespace swam {
namespace {

constexpr int kMathThreads = 128;      // of the warps that multiply
constexpr int kThreadsP = kMathThreads + 32;
constexpr int kCtasPerSm = 2;
constexpr int kMinUnits = 2;           // key tiles that a share has at least, where row tiles may be cut

template <int D, int WR>
struct PagedCfg {
  static constexpr int KT = D == 128 ? 64 : 128;                         // keys per tile: 16 KB of K (8 at head dim 32)
  static constexpr int WRows = WR == 0 ? 1 : WR;                         // warps along the rows
  static constexpr int WK = 4 / WRows, MR = WR == 0 ? 8 : 16 * WR, KW = KT / WK;
  static constexpr int kTileB = KT * D * 2;
  static constexpr int kStages = D == 32 ? 6 : 3;                        // 96 KB: two CTAs an SM
  static constexpr int kRing = kStages * 2 * kTileB;
  static constexpr int kBytes = kRing + 1024 /*alignment*/ + 16 * kStages + 64 * 8 /*maxima and sums of the warps*/;
};

// A stretch of the sequence of units.  [t, t_end) are the key tiles of the current row tile that belong to it.
struct Walk {
  int64_t left;            // units behind the current piece
  int b, h, r;             // sample, key/value head, row tile
  int rt;                  // row tiles of the sample and head
  int t, t_end, tiles;     // tiles: of the whole row tile
  PagedSample s;
};

struct Place {
  int64_t offset;          // units of the sample in front of the share's first one
  PagedSample s;
  int b;
};

// the math warps' own barrier
__device__ __forceinline__ void math_sync() { asm volatile("bar.sync 1, 128;" ::: "memory"); }

template <int MR>
__device__ __forceinline__ int row_tiles(const PagedSample& s, int g) { return (s.n * g + MR - 1) / MR; }
template <int MR, int KT>
__device__ __forceinline__ int key_tiles(const SegParams& p, const PagedSample& s, int r) {
  const int last = min((r + 1) * MR, s.n * p.g) - 1;
  return (paged_limit(p.a.causal, s, last / p.g) + KT - 1) / KT;
}
// units of one key/value head (a row tile without keys still has its zeros to write)
template <int MR, int KT>
__device__ __forceinline__ int64_t head_units(const SegParams& p, const PagedSample& s) {
  const int rt = row_tiles<MR>(s, p.g);
  if (!p.a.causal) return (int64_t)rt * max(1, (s.len + KT - 1) / KT);
  int64_t u = 0;
  for (int r = 0; r < rt; ++r) u += max(1, key_tiles<MR, KT>(p, s, r));
  return u;
}

// first unit of share c of `shares` equal ones of `total`; the share that holds unit u
__device__ __forceinline__ int64_t share_begin(int64_t total, int shares, int c) {
  const int64_t per = total / shares, more = total % shares;
  return c * per + min((int64_t)c, more);
}
__device__ __forceinline__ int share_of(int64_t total, int shares, int64_t u) {
  const int64_t per = total / shares, more = total % shares, big = more * (per + 1);
  return (int)(u < big ? u / (per + 1) : more + (u - big) / per);
}

template <int D, int WR>
__global__ void __launch_bounds__(kThreadsP, kCtasPerSm)
paged_mma_kernel(const __grid_constant__ CUtensorMap map_k, const __grid_constant__ CUtensorMap map_v, const __grid_constant__ SegParams p,
                 const __grid_constant__ PagedCache pc, const bool cut, int4* join) {
  using C = PagedCfg<D, WR>;
  constexpr int MR = C::MR, WK = C::WK, KT = C::KT, KW = C::KW, kStages = C::kStages, kTileB = C::kTileB;
  extern __shared__ unsigned char smem_raw[];
  __shared__ int64_t warp_sum[5];
  __shared__ Place place;
  __shared__ int abort_word;
  volatile int* abort_flag = &abort_word;
  const uint32_t s0 = (smem_addr(smem_raw) + 1023u) & ~1023u;
  unsigned char* base = smem_raw + (s0 - smem_addr(smem_raw));
  const uint32_t bars = s0 + C::kRing;
  auto bar_full = [&](int st) { return bars + 16 * st; };
  auto bar_empty = [&](int st) { return bars + 16 * st + 8; };
  float2* ml = reinterpret_cast<float2*>(base + C::kRing + 16 * kStages);      // [WK][MR]
  const SegArgs& a = p.a;
  const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
  if (threadIdx.x == 0) {
    for (int i = 0; i < kStages; ++i) {
      mbar_init(bar_full(i), 1);
      mbar_init(bar_empty(i), 4);
    }
    abort_word = 0;
    asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
    if (cut) join[blockIdx.x] = make_int4(0, 0, 0, 0);
  }
  if (warp == 4 && lane < 2) asm volatile("prefetch.tensormap [%0];" ::"l"(lane == 0 ? &map_k : &map_v) : "memory");

  // ---- the share of this CTA: add up the units, then find the sample of its first one
  int64_t mine0 = 0, sum = 0;
  PagedSample smp0{0, 0, 0};
  for (int b0 = 0; b0 < pc.samples; b0 += kThreadsP) {
    const int b = b0 + threadIdx.x;
    PagedSample smp{0, 0, 0};
    if (b < pc.samples) smp = paged_sample(pc, a.n_q, b, p.status);
    const int64_t u = head_units<MR, KT>(p, smp) * a.N_kv;
    if (b0 == 0) {
      mine0 = u;
      smp0 = smp;
    }
    sum += u;
  }
#pragma unroll
  for (int o = 16; o > 0; o >>= 1) sum += __shfl_xor_sync(0xffffffffu, sum, o);
  if (lane == 0) warp_sum[warp] = sum;
  __syncthreads();
  const int64_t total = warp_sum[0] + warp_sum[1] + warp_sum[2] + warp_sum[3] + warp_sum[4];
  const int64_t most = cut ? (total + kMinUnits - 1) / kMinUnits : total;
  const int shares = (int)min((int64_t)gridDim.x, most);
  if ((int)blockIdx.x >= shares) {
    allow_next();
    return;
  }
  const int64_t u0 = share_begin(total, shares, blockIdx.x), u1 = share_begin(total, shares, blockIdx.x + 1);
  int64_t before = 0;
  for (int b0 = 0; b0 < pc.samples && before <= u0; b0 += kThreadsP) {
    const int b = b0 + threadIdx.x;
    PagedSample smp = smp0;
    if (b0 > 0) {
      smp = PagedSample{0, 0, 0};
      if (b < pc.samples) smp = paged_sample(pc, a.n_q, b, p.status);
    }
    const int64_t u = b0 == 0 ? mine0 : head_units<MR, KT>(p, smp) * a.N_kv;
    int64_t end = u;
#pragma unroll
    for (int o = 1; o < 32; o <<= 1) {
      const int64_t y = __shfl_up_sync(0xffffffffu, end, o);
      if (lane >= o) end += y;
    }
    __syncthreads();
    if (lane == 31) warp_sum[warp] = end;
    __syncthreads();
    for (int w = 0; w < 5; ++w) {
      if (w < warp) end += warp_sum[w];
    }
    end += before;
    if (u0 >= end - u && u0 < end) place = Place{u0 - (end - u), smp, b};
    for (int w = 0; w < 5; ++w) before += warp_sum[w];
  }
  __syncthreads();

  // makes the current row tile's part of the stretch: from tile t on, as far as `left` reaches
  auto take = [&](Walk& w) {
    w.tiles = key_tiles<MR, KT>(p, w.s, w.r);
    const int units = max(1, w.tiles);
    const int64_t n = cut ? min((int64_t)(units - w.t), w.left) : units;
    w.left -= n;
    w.t_end = w.tiles == 0 ? 0 : w.t + (int)n;
  };
  // the next row tile; false at the end of the stretch
  auto next = [&](Walk& w) {
    if (w.left <= 0) return false;
    w.t = 0;
    if (++w.r == w.rt) {
      w.r = 0;
      if (++w.h == a.N_kv) {
        w.h = 0;
        do {
          if (++w.b >= pc.samples) return false;
          w.s = paged_sample(pc, a.n_q, w.b, p.status);
        } while (w.s.n == 0);
        w.rt = row_tiles<MR>(w.s, p.g);
      }
    }
    take(w);
    return true;
  };
  Walk w;
  bool more = true;
  {
    w.left = u1 - u0;
    w.b = place.b;
    w.s = place.s;
    w.rt = row_tiles<MR>(w.s, p.g);
    const int64_t units = head_units<MR, KT>(p, w.s);
    w.h = (int)(place.offset / units);
    int64_t off = place.offset - w.h * units;
    w.r = 0;
    if (!a.causal) {
      const int each = max(1, (w.s.len + KT - 1) / KT);
      w.r = (int)(off / each);
      off -= (int64_t)w.r * each;
    } else {
      for (int n; off >= (n = max(1, key_tiles<MR, KT>(p, w.s, w.r))); ++w.r) off -= n;
    }
    w.t = (int)off;
    if (!cut && w.t > 0) {
      // a row tile belongs to the share that holds its first unit
      w.left -= max(1, key_tiles<MR, KT>(p, w.s, w.r)) - w.t;
      more = next(w);
    } else {
      take(w);
    }
  }
  // A page's rows of a tile are [64-column block][row]: one box.  (A tile inside a page: that many rows of it.)
  const int sh = pc.page_shift, rows = min(KT, 1 << sh);

  if (warp == 4) {
    // ------------------------------------------------------------------ loads
    PageWindow pages;
    bool ok = true;
    int cnt = 0;
    for (; more && ok; more = next(w)) {
      const int keys_all = paged_limit(a.causal, w.s, (min((w.r + 1) * MR, w.s.n * p.g) - 1) / p.g);
      for (int t = w.t; t < w.t_end; ++t, ++cnt) {
        const int key0 = t * KT, keys = keys_all - key0;
        const int count = min(KT / rows, (keys + rows - 1) / rows);
        const int page = pages.get(pc, w.b, key0 >> sh, lane < count ? lane : 0);
        const int st = cnt % kStages;
        if (cnt >= kStages) ok = __all_sync(0xffffffffu, mbar_wait(bar_empty(st), ((cnt / kStages) & 1) ^ 1, abort_flag) ? 1 : 0) != 0;
        if (!ok) break;
        const uint32_t dst = s0 + (uint32_t)st * 2 * kTileB + lane * rows * D * 2, bar = bar_full(st);
        if (lane == 0) mbar_expect_tx(bar, 2 * count * rows * D * 2);
        __syncwarp();
        if (lane < count) {
          const int at = paged_page(pc, page, p.status), row = key0 & ((1 << sh) - 1);
          if constexpr (D == 32) {
            tma_load_4d(dst, &map_k, bar, 0, row, w.h, at);
            tma_load_4d(dst + kTileB, &map_v, bar, 0, row, w.h, at);
          } else {
            tma_load_5d(dst, &map_k, bar, 0, row, 0, w.h, at);
            tma_load_5d(dst + kTileB, &map_v, bar, 0, row, 0, w.h, at);
          }
        }
        __syncwarp();
      }
    }
    allow_next();
    if (!ok) {
      // copies in flight must not outlive the CTA
      for (int i = max(0, cnt - kStages); i < cnt; ++i) mbar_wait_bounded(bar_full(i % kStages), (i / kStages) & 1, kDrainCycles, nullptr);
    }
    return;
  }

  // ---------------------------------------------------------------------- products
  constexpr bool kNarrow = WR == 0;
  const int wr = warp % C::WRows, wk = warp / C::WRows;
  const int block_b = rows * (D == 32 ? 64 : 128);                   // bytes of a 64-column block of a page's rows
  // byte offset of the 16 keys from R on (they are in one page), and of a lane's row and chunk inside them
  auto group_off = [&](int R) { return (uint32_t)(R / rows * rows * D * 2 + (R & (rows - 1)) * (D == 32 ? 64 : 128)); };
  auto lane_off = [&](int r, int c) {
    if (D == 32) return (uint32_t)(r * 64 + ((c ^ ((r >> 1) & 3)) << 4));
    return (uint32_t)((c >> 3) * block_b + r * 128 + (((c & 7) ^ (r & 7)) << 4));
  };
  int cnt = 0;                                     // key tiles so far
  // When a wait has run out every warp still walks through its tiles, without products, so that all meet at the same barriers.
  bool ok = true;
  for (; more; more = next(w)) {
    const int row0 = (w.s.q0 * p.g) + w.r * MR;    // first row, counted from the call's first token
    const int row_end = (w.s.q0 + w.s.n) * p.g;
    const int t0 = w.t;
    const bool whole = t0 == 0 && w.t_end == w.tiles;
    const int len = paged_limit(a.causal, w.s, (min((w.r + 1) * MR, w.s.n * p.g) - 1) / p.g);
    // this thread's two rows: those of its accumulators, lane / 4 and lane / 4 + 8 of the warp's 16 (narrow: 2 (lane % 4) and the next),
    // and the queries as A fragments of the former (narrow: B fragments of row lane / 4)
    auto row_of = [&](int i) { return kNarrow ? (lane & 3) * 2 + i : wr * 16 + (lane >> 2) + 8 * i; };
    uint32_t qf[D / 16][kNarrow ? 2 : 4];
    int lim[2];
#pragma unroll
    for (int i = 0; i < 2; ++i) {
      const int row = row0 + row_of(i);
      lim[i] = row < row_end ? paged_limit(a.causal, w.s, row / p.g - w.s.q0) : 0;
    }
#pragma unroll
    for (int i = 0; i < (kNarrow ? 1 : 2); ++i) {
      const int row = row0 + wr * 16 + (lane >> 2) + 8 * i;
      const bool real = row < row_end;
      const int tok = real ? row / p.g : 0, h = w.h * p.g + (real ? row - tok * p.g : 0);
      const uint32_t* src = reinterpret_cast<const uint32_t*>((const __nv_bfloat16*)a.q + tok * a.q_tok + (int64_t)h * D);
#pragma unroll
      for (int ks = 0; ks < D / 16; ++ks) {
        qf[ks][i] = real ? src[ks * 8 + (lane & 3)] : 0u;
        qf[ks][i + (kNarrow ? 1 : 2)] = real ? src[ks * 8 + 4 + (lane & 3)] : 0u;
      }
    }
    constexpr int OB = kNarrow ? D / 16 : D / 8;   // blocks of accumulators
    float o[OB][4];
#pragma unroll
    for (int i = 0; i < OB; ++i) o[i][0] = o[i][1] = o[i][2] = o[i][3] = 0.f;
    float m[2] = {-INFINITY, -INFINITY}, l[2] = {0.f, 0.f};
    bool big = false;                              // some row's reference is large: see kSegBig

    for (int t = t0; t < w.t_end; ++t, ++cnt) {
      const int st = cnt % kStages;
      ok = ok && __all_sync(0xffffffffu, mbar_wait(bar_full(st), (cnt / kStages) & 1, abort_flag) ? 1 : 0) != 0;
      const int key0 = t * KT + wk * KW;           // first key of this warp
      if (ok && key0 < len) {                      // (some of this warp's keys are real)
        const uint32_t ks = s0 + (uint32_t)st * 2 * kTileB, vs = ks + kTileB;
        if (len - key0 < KW) {
          // this warp's rows of V behind the last key become zeros
          constexpr int CPR = D / 8;
          for (int i = lane; i < (KW - (len - key0)) * CPR; i += 32) {
            const int r = len - key0 + i / CPR;
            st_shared_16(vs + group_off(wk * KW + (r & ~15)) + lane_off(r & 15, i % CPR), 0u, 0u, 0u, 0u);
          }
          fence_proxy_async();                     // the stage's next load comes through the other proxy
          __syncwarp();
        }
        if constexpr (kNarrow) {
          // S^T: keys lane / 4 and lane / 4 + 8 of each 16, rows 2 (lane % 4) and the next
          float sc[KW / 16][4];
#pragma unroll
          for (int nb = 0; nb < KW / 16; ++nb) {
            const uint32_t at = ks + group_off(wk * KW + nb * 16);
            sc[nb][0] = sc[nb][1] = sc[nb][2] = sc[nb][3] = 0.f;
#pragma unroll
            for (int kd = 0; kd < D / 16; ++kd) {
              uint32_t f[4];
              ldsm4(f, at + lane_off((lane & 7) + (((lane >> 3) & 1) << 3), kd * 2 + (lane >> 4)));
              mma_bf16(sc[nb], f, qf[kd][0], qf[kd][1]);
            }
          }
          if (min(lim[0], lim[1]) - key0 < KW) {
#pragma unroll
            for (int nb = 0; nb < KW / 16; ++nb) {
#pragma unroll
              for (int e = 0; e < 4; ++e)
                if (key0 + nb * 16 + (lane >> 2) + (e & 2) * 4 >= lim[e & 1]) sc[nb][e] = -INFINITY;
            }
          }
          float corr[2], ref[2];
#pragma unroll
          for (int i = 0; i < 2; ++i) {
            float mx = -INFINITY;
#pragma unroll
            for (int nb = 0; nb < KW / 16; ++nb) mx = fmaxf(mx, fmaxf(sc[nb][i], sc[nb][i + 2]));
#pragma unroll
            for (int x = 4; x < 32; x <<= 1) mx = fmaxf(mx, __shfl_xor_sync(0xffffffffu, mx, x));
            const float mn = fmaxf(m[i], mx * p.scale_log2);
            ref[i] = mn == -INFINITY ? 0.f : mn;
            corr[i] = ex2(m[i] - ref[i]);
            m[i] = mn;
            l[i] *= corr[i];
          }
          const bool moved = __any_sync(0xffffffffu, corr[0] != 1.f || corr[1] != 1.f);
          if (moved) big = __any_sync(0xffffffffu, !(fmaxf(fabsf(ref[0]), fabsf(ref[1])) < kSegBig));
          float scale = p.scale_log2;
          if (big) {
            scale = 1.f;
#pragma unroll
            for (int nb = 0; nb < KW / 16; ++nb) {
#pragma unroll
              for (int e = 0; e < 4; ++e) sc[nb][e] *= p.scale_log2;
            }
          }
#pragma unroll
          for (int nb = 0; nb < KW / 16; ++nb) {
#pragma unroll
            for (int e = 0; e < 4; ++e) {
              sc[nb][e] = ex2(fmaf(sc[nb][e], scale, -ref[e & 1]));
              l[e & 1] += sc[nb][e];
            }
          }
          if (moved) {
#pragma unroll
            for (int i = 0; i < OB; ++i) {
              o[i][0] *= corr[0];
              o[i][1] *= corr[1];
              o[i][2] *= corr[0];
              o[i][3] *= corr[1];
            }
          }
#pragma unroll
          for (int nb = 0; nb < KW / 16; ++nb) {
            const uint32_t at = vs + group_off(wk * KW + nb * 16);
            const uint32_t p0 = transpose8(pack_bf16x2(sc[nb][0], sc[nb][1])), p1 = transpose8(pack_bf16x2(sc[nb][2], sc[nb][3]));
#pragma unroll
            for (int dn = 0; dn < D / 16; ++dn) {
              uint32_t f[4];
              ldsm4_t(f, at + lane_off((lane & 7) + ((lane >> 4) << 3), dn * 2 + ((lane >> 3) & 1)));
              mma_bf16(o[dn], f, p0, p1);
            }
          }
        } else {
          float sc[KW / 8][4];
#pragma unroll
          for (int nb = 0; nb < KW / 16; ++nb) {
            const uint32_t at = ks + group_off(wk * KW + nb * 16);
#pragma unroll
            for (int e = 0; e < 4; ++e) sc[2 * nb][e] = sc[2 * nb + 1][e] = 0.f;
#pragma unroll
            for (int kd = 0; kd < D / 16; ++kd) {
              uint32_t f[4];
              ldsm4(f, at + lane_off((lane & 7) + ((lane >> 4) << 3), kd * 2 + ((lane >> 3) & 1)));
              mma_bf16(sc[2 * nb], qf[kd], f[0], f[1]);
              mma_bf16(sc[2 * nb + 1], qf[kd], f[2], f[3]);
            }
          }
          const int v0 = lim[0] - key0, v1 = lim[1] - key0;       // keys of the warp's range that the rows see
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
            ref[i] = mn == -INFINITY ? 0.f : mn;       // a row that has seen no key yet: every exponent stays -inf
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
          if (moved) {
#pragma unroll
            for (int i = 0; i < OB; ++i) {
              o[i][0] *= corr[0];
              o[i][1] *= corr[0];
              o[i][2] *= corr[1];
              o[i][3] *= corr[1];
            }
          }
#pragma unroll
          for (int nb = 0; nb < KW / 16; ++nb) {
            const uint32_t at = vs + group_off(wk * KW + nb * 16);
            const uint32_t pf[4] = {pack_bf16x2(sc[2 * nb][0], sc[2 * nb][1]), pack_bf16x2(sc[2 * nb][2], sc[2 * nb][3]),
                                    pack_bf16x2(sc[2 * nb + 1][0], sc[2 * nb + 1][1]), pack_bf16x2(sc[2 * nb + 1][2], sc[2 * nb + 1][3])};
#pragma unroll
            for (int dn = 0; dn < D / 16; ++dn) {
              uint32_t f[4];
              ldsm4_t(f, at + lane_off((lane & 7) + (((lane >> 3) & 1) << 3), dn * 2 + (lane >> 4)));
              mma_bf16(o[2 * dn], pf, f[0], f[1]);
              mma_bf16(o[2 * dn + 1], pf, f[2], f[3]);
            }
          }
        }
      }
      // the stage is free, but for the row tile's last one, which serves the merge first
      if (WK == 1 || t + 1 < w.t_end) {
        __syncwarp();
        if (lane == 0) mbar_arrive(bar_empty(st));
      }
    }
#pragma unroll
    for (int i = 0; i < 2; ++i) {
#pragma unroll
      for (int x = kNarrow ? 4 : 1; x < (kNarrow ? 32 : 4); x <<= 1) l[i] += __shfl_xor_sync(0xffffffffu, l[i], x);
    }

    // ---- the row tile's result: every warp takes 1 / WK of the columns (narrow, head dim 32: two warps half of them each).  (A row tile
    // without keys has nothing to merge.)
    constexpr int NB = OB < WK ? 1 : OB / WK;      // blocks of a warp
    const bool mine = OB >= WK || wk < OB;
    float out[NB][4], mm[2], ll[2];
    if (WK > 1 && w.t_end > t0) {
      const int st = (cnt - 1) % kStages;
      float4* frag = reinterpret_cast<float4*>(base + (size_t)st * 2 * kTileB);       // [warp][block][lane]
      math_sync();                                 // all warps are through with the stage
#pragma unroll
      for (int i = 0; i < OB; ++i) frag[(warp * OB + i) * 32 + lane] = make_float4(o[i][0], o[i][1], o[i][2], o[i][3]);
      if (kNarrow ? lane < 4 : (lane & 3) == 0) {
        ml[wk * MR + row_of(0)] = make_float2(m[0], l[0]);
        ml[wk * MR + row_of(1)] = make_float2(m[1], l[1]);
      }
      math_sync();
      float f[WK][2];
#pragma unroll
      for (int i = 0; i < 2; ++i) {
        const int r = row_of(i);
        mm[i] = -INFINITY;
#pragma unroll
        for (int k = 0; k < WK; ++k) mm[i] = fmaxf(mm[i], ml[k * MR + r].x);
        ll[i] = 0.f;
#pragma unroll
        for (int k = 0; k < WK; ++k) {
          const float2 x = ml[k * MR + r];
          f[k][i] = mm[i] == -INFINITY ? 0.f : exp2f(x.x - mm[i]);
          ll[i] += f[k][i] * x.y;
        }
      }
#pragma unroll
      for (int i = 0; i < NB; ++i) {
        out[i][0] = out[i][1] = out[i][2] = out[i][3] = 0.f;
        if (mine) {
#pragma unroll
          for (int k = 0; k < WK; ++k) {
            const float4 x = frag[((k * C::WRows + wr) * OB + wk * NB + i) * 32 + lane];
            out[i][0] += f[k][0] * x.x;
            out[i][1] += f[k][kNarrow ? 1 : 0] * x.y;
            out[i][2] += f[k][kNarrow ? 0 : 1] * x.z;
            out[i][3] += f[k][1] * x.w;
          }
        }
      }
      fence_proxy_async();                         // the stage's next load comes through the other proxy
      math_sync();                                 // (the maxima and sums have been read too)
      if (lane == 0) mbar_arrive(bar_empty(st));
    } else {
#pragma unroll
      for (int i = 0; i < NB; ++i) {
#pragma unroll
        for (int e = 0; e < 4; ++e) out[i][e] = WK > 1 ? 0.f : o[i][e];      // (WK > 1: no keys)
      }
#pragma unroll
      for (int i = 0; i < 2; ++i) {
        mm[i] = m[i];
        ll[i] = l[i];
      }
    }
    const int slot = (int)blockIdx.x * 2 + (t0 == 0 ? 1 : 0);
    if constexpr (kNarrow) {
      // out[k]: columns 16 (wk NB + k) + lane / 4 and 8 further, rows 2 (lane % 4) and the next
      if (whole) {
        const float i0 = seg_inverse(ll[0]), i1 = seg_inverse(ll[1]);
        const int row = row0 + (lane >> 2), tok = row / p.g, h = w.h * p.g + row - tok * p.g;
        uint32_t* dst = reinterpret_cast<uint32_t*>((__nv_bfloat16*)a.out + tok * a.o_tok + (int64_t)h * D + wk * NB * 16 + (lane & 3) * 2);
#pragma unroll
        for (int k = 0; k < NB; ++k) {
          // (transposed: row lane / 4, two neighbouring columns)
          const uint32_t x0 = transpose8(pack_bf16x2(out[k][0] * i0, out[k][1] * i1)), x1 = transpose8(pack_bf16x2(out[k][2] * i0, out[k][3] * i1));
          if (mine && row < row_end) {
            dst[k * 8] = x0;
            dst[k * 8 + 4] = x1;
          }
        }
      }
#pragma unroll
      for (int i = 0; i < 2; ++i) {
        const int r = row_of(i), row = row0 + r;
        if (row >= row_end || !mine) continue;
        if (!whole) {
          float* dst = p.part_o + ((int64_t)slot * MR + r) * D + wk * NB * 16 + (lane >> 2);
#pragma unroll
          for (int k = 0; k < NB; ++k) {
            dst[k * 16] = out[k][i];
            dst[k * 16 + 8] = out[k][i + 2];
          }
          if (wk == 0 && lane < 4) p.part_ml[slot * MR + r] = make_float2(mm[i], ll[i]);
        } else if (a.lse && wk == 0 && lane < 4) {
          const int tok = row / p.g, h = w.h * p.g + row - tok * p.g;
          a.lse[(int64_t)h * a.n_q + tok] = seg_lse(mm[i], ll[i]);
        }
      }
    } else {
#pragma unroll
      for (int i = 0; i < 2; ++i) {
        const int r = row_of(i), row = row0 + r;
        if (row >= row_end) continue;
        const int tok = row / p.g, h = w.h * p.g + row - tok * p.g;
        const int c = wk * NB * 8 + (lane & 3) * 2;
        if (whole) {
          const float inv = seg_inverse(ll[i]);
          uint32_t* dst = reinterpret_cast<uint32_t*>((__nv_bfloat16*)a.out + tok * a.o_tok + (int64_t)h * D + c);
#pragma unroll
          for (int k = 0; k < NB; ++k) dst[k * 4] = pack_bf16x2(out[k][2 * i] * inv, out[k][2 * i + 1] * inv);
          if (a.lse && wk == 0 && (lane & 3) == 0) a.lse[(int64_t)h * a.n_q + tok] = seg_lse(mm[i], ll[i]);
        } else {
          float* dst = p.part_o + ((int64_t)slot * MR + r) * D + c;
#pragma unroll
          for (int k = 0; k < NB; ++k) *reinterpret_cast<float2*>(dst + k * 8) = make_float2(out[k][2 * i], out[k][2 * i + 1]);
          if (wk == 0 && (lane & 3) == 0) p.part_ml[slot * MR + r] = make_float2(mm[i], ll[i]);
        }
      }
    }
    if (!whole && t0 == 0 && threadIdx.x == 0) {
      // this is the first piece of a row tile that goes on in the next shares (left = 0: u1 is the unit behind this piece)
      const int pieces = share_of(total, shares, u1 + (w.tiles - w.t_end) - 1) - (int)blockIdx.x + 1;
      join[blockIdx.x] = make_int4(row0, min(row0 + MR, row_end), w.h, pieces);
    }
  }
  allow_next();
  if (!ok && lane == 0) atomicOr(p.status, ST_TIMEOUT);
}

// Joins the pieces of one row tile: out = sum_i 2^(m_i - m) o_i / sum_i 2^(m_i - m) l_i.  A thread takes four columns of a row and every
// groups-th piece, eight at a time with their maxima and sums (one trip to memory for up to 8 * groups pieces); the groups are then
// merged in order.
constexpr int kJoinThreads = 256;
struct Joined {
  float4 o;
  float m, l;
};
template <int D, int MR>
__global__ void __launch_bounds__(kJoinThreads) paged_join_kernel(const __grid_constant__ SegParams p, const int4* join) {
  __shared__ Joined part[kJoinThreads];
  constexpr int V = D / 4, kAhead = 8;
  const SegArgs& a = p.a;
  wait_previous();
  const int4 j = join[blockIdx.x];
  const int pieces = j.w, rows = j.y - j.x, items = rows * V;
  if (pieces <= 1) return;
  // piece 0 is in its share's second slot, piece i in the first slot of the i-th share behind it
  auto slot = [&](int i) { return i == 0 ? (int)blockIdx.x * 2 + 1 : ((int)blockIdx.x + i) * 2; };
  auto add = [](Joined& x, float m, float l, const float4& o) {
    const float mn = fmaxf(x.m, m);
    if (mn == -INFINITY) return;             // neither has keys
    const float f = exp2f(x.m - mn), g = exp2f(m - mn);
    x.l = x.l * f + l * g;
    x.o = make_float4(fmaf(o.x, g, x.o.x * f), fmaf(o.y, g, x.o.y * f), fmaf(o.z, g, x.o.z * f), fmaf(o.w, g, x.o.w * f));
    x.m = mn;
  };
  const int groups = items >= kJoinThreads ? 1 : kJoinThreads / items;
  for (int x0 = 0; x0 < items; x0 += kJoinThreads) {
    const int x = x0 + (int)threadIdx.x, grp = groups > 1 ? x / items : 0, item = x - grp * items;
    const int r = item / V, c = (item - r * V) * 4;
    const bool on = groups > 1 ? grp < groups : x < items;
    Joined sum{make_float4(0.f, 0.f, 0.f, 0.f), -INFINITY, 0.f};
    for (int i0 = grp; on && i0 < pieces; i0 += kAhead * groups) {
      float4 o[kAhead];
      float2 ml[kAhead];
#pragma unroll
      for (int k = 0; k < kAhead; ++k) {
        const int i = i0 + k * groups;
        if (i < pieces) {
          const int at = slot(i) * MR + r;
          ml[k] = p.part_ml[at];
          o[k] = *reinterpret_cast<const float4*>(p.part_o + (int64_t)at * D + c);
        } else {
          ml[k] = make_float2(-INFINITY, 0.f);
          o[k] = make_float4(0.f, 0.f, 0.f, 0.f);
        }
      }
#pragma unroll
      for (int k = 0; k < kAhead; ++k)
        add(sum, ml[k].x, ml[k].y, o[k]);
    }
    if (groups > 1) {
      part[threadIdx.x] = sum;
      __syncthreads();
      if ((int)threadIdx.x >= items) break;
      for (int k = 1; k < groups; ++k) {
        const Joined& y = part[threadIdx.x + k * items];
        add(sum, y.m, y.l, y.o);
      }
    }
    if (!on) continue;
    const int row = j.x + r, tok = row / p.g, h = j.z * p.g + row - tok * p.g;
    const float inv = seg_inverse(sum.l);
    *reinterpret_cast<uint2*>((__nv_bfloat16*)a.out + tok * a.o_tok + (int64_t)h * D + c) =
        make_uint2(pack_bf16x2(sum.o.x * inv, sum.o.y * inv), pack_bf16x2(sum.o.z * inv, sum.o.w * inv));
    if (a.lse && c == 0) a.lse[(int64_t)h * a.n_q + tok] = seg_lse(sum.m, sum.l);
  }
}

// Pages [n_pages, page, N_kv, D] with strides as (column of a 64-column block, row, block, head, page); box = `rows` rows of all columns
bool make_page_map(CUtensorMap* map, const void* ptr, int n_pages, int page, int N_kv, int D, int64_t tok, int64_t stride, int rows) {
  // L2 fetches what a row of one head has: the next head's keys would be gone before they are used (64 ragged single tokens, head dim 64:
  // 113 us, 126 with 256 bytes; head dim 32: 79 and 97)
  const CUtensorMapL2promotion fetch = D == 32 ? CU_TENSOR_MAP_L2_PROMOTION_L2_64B : (D == 64 ? CU_TENSOR_MAP_L2_PROMOTION_L2_128B : CU_TENSOR_MAP_L2_PROMOTION_L2_256B);
  if (D == 32) return make_kv_map(map, ptr, n_pages, page, N_kv, D, tok, stride, rows, fetch);
  const cuuint64_t dims[5] = {64, (cuuint64_t)page, (cuuint64_t)D / 64, (cuuint64_t)N_kv, (cuuint64_t)n_pages};
  const cuuint64_t strides[4] = {(cuuint64_t)tok * 2, 128, (cuuint64_t)D * 2, (cuuint64_t)stride * 2};
  const cuuint32_t box[5] = {64, (cuuint32_t)rows, (cuuint32_t)D / 64, 1, 1};
  return encode_bf16(map, ptr, 5, dims, strides, box, fetch);
}

template <int D, int WR>
cudaError_t launch_one(const SegParams& p0, const PagedCache& c, int shares, bool cut, cudaStream_t st, int* launches) {
  using C = PagedCfg<D, WR>;
  SegParams p = p0;
  const SegArgs& a = p.a;
  // scratch: outputs, maxima and sums of two pieces per share, and the join's description
  p.part_ml = (float2*)(p.part_o + (size_t)shares * 2 * C::MR * D);
  int4* join = (int4*)(p.part_ml + (size_t)shares * 2 * C::MR);
  CUtensorMap mk, mv;
  const int page = 1 << c.page_shift, rows = page < C::KT ? page : C::KT;
  if (!make_page_map(&mk, a.k[1], c.n_pages, page, a.N_kv, D, c.k_tok, c.k_page, rows) ||
      !make_page_map(&mv, a.v[1], c.n_pages, page, a.N_kv, D, c.v_tok, c.v_page, rows))
    return cudaErrorInvalidValue;
  static SmemOptIn opt_in;
  cudaError_t e = opt_in((const void*)paged_mma_kernel<D, WR>, C::kBytes, a.device);
  if (e != cudaSuccess) return e;
  ++*launches;
  paged_mma_kernel<D, WR><<<shares, kThreadsP, C::kBytes, st>>>(mk, mv, p, c, cut, join);
  e = cudaGetLastError();
  if (e != cudaSuccess || !cut) return e;
  ++*launches;
  return launch_after(paged_join_kernel<D, C::MR>, dim3(shares), dim3(kJoinThreads), 0, st, p, (const int4*)join);
}
template <int D>
cudaError_t launch_rows(const SegParams& p, const PagedCache& c, int rows, int shares, bool cut, cudaStream_t st, int* launches) {
  if (rows == 8) return launch_one<D, 0>(p, c, shares, cut, st, launches);
  return rows == 16 ? launch_one<D, 1>(p, c, shares, cut, st, launches)
                    : (rows == 32 ? launch_one<D, 2>(p, c, shares, cut, st, launches) : launch_one<D, 4>(p, c, shares, cut, st, launches));
}

}  // namespace

int paged_mma_shares(int sms) { return kCtasPerSm * sms; }
size_t paged_mma_scratch(int shares, int tile_rows, int D) {
  return (size_t)shares * (2 * tile_rows * ((size_t)D * sizeof(float) + sizeof(float2)) + sizeof(int4));
}
cudaError_t launch_paged_mma(const SegParams& p, const PagedCache& c, int tile_rows, int shares, bool cut, cudaStream_t st, int* launches) {
  switch (p.a.D) {
    case 32: return launch_rows<32>(p, c, tile_rows, shares, cut, st, launches);
    case 64: return launch_rows<64>(p, c, tile_rows, shares, cut, st, launches);
    case 128: return launch_rows<128>(p, c, tile_rows, shares, cut, st, launches);
    default: return cudaErrorInvalidConfiguration;
  }
}

}  // namespace swam
