// Segment attention for bf16 tensors on the 5th-generation tensor cores (tcgen05 + TMEM), keys and values fed by TMA:
// the kernel for many query rows per key/value head (head dim 64 and 128).
//
// A persistent CTA per SM walks through work items (seg_attn.cuh): a row tile and a range of 128-key tiles.
//   warp 11      scheduler: decodes the items ahead of everybody else (divisions, lengths from memory) into a small ring of
//                descriptors that all other warps read
//   warp 9       TMA producer: K and V tiles into one ring of shared-memory slots, in the order the tensor pipe uses them,
//                and the queries where a row tile is a box of the query tensor
//   warp 10      fetches the query rows one by one where it is not (a number of heads per key/value head that does not
//                divide the tile, samples that do not tile it), with 16-byte asynchronous copies into the same layout
//   warp 8       one elected thread issues every tcgen05.mma: S = Q K^T into TMEM, then O += P V with both operands in
//                shared memory; O stays in TMEM for the whole range of keys
//   warps 0-3    softmax of stream 0, one thread per row: S row from TMEM, exponentials against a running reference
//   warps 4-7    maximum (exp2 domain, raised only when a row outgrows it by 2^8: exact either way), P as bf16 into shared
//                memory; same for stream 1.  The streams' exponentials overlap each other's products.
// kAlt = false: a row tile has 256 rows; the streams are its two halves and share every key tile.
// kAlt = true: a row tile has at most 128 rows; both streams hold the same rows and take the key tiles in turn, each with
//   its own maximum, sum and output accumulator, and are merged in the epilogue.  The memory of the second query tile
//   goes to the ring.
// Rows of V behind a real length are overwritten with zeros in shared memory before the product (0 * NaN would poison the
// row); scores behind a row's limit become -inf.
// Every wait on an mbarrier is bounded; when one runs out the kernel raises the timeout bit of the status word and every
// role falls through to the exit.
#include <string.h>

#include "tc_ptx.cuh"
#include "seg_attn.cuh"

namespace swam {
namespace {

constexpr int kThreadsS = 384;
constexpr int kDesc = 4;            // descriptors in flight

// One work item as every warp sees it: tiles [0, na) are 128-key tiles of segment 0 (the first one starts at key base0), the
// rest of segment 1 (tile i starts at key base1 + 128 i; base1 may be negative).  n = 0: no key, n < 0: no more items.
struct __align__(16) SegDesc {
  int n, na, b0, h_kv;
  int row0, base0, base1, part;
  int len0, len1, own, kv0;         // real keys of segment 0, most that a row of the tile sees of segment 1, real keys of it; group
};

template <int D, bool kAlt>
struct SegCfg {
  static constexpr int DB = D / 64;                  // 64-column (128-byte) blocks per row
  static constexpr int kSub = kTile * 128;           // bytes of a [128 rows x 64 columns] block
  static constexpr int kTileBytes = DB * kSub;       // a 128 x D tile
  static constexpr int kPBytes = 2 * kSub;           // a 128 x 128 bf16 P tile
  static constexpr int NQ = kAlt ? 1 : 2;            // query tiles of an item
  static constexpr int kRows = NQ * kTile;
  // Query buffers: with two, an item's queries arrive while the previous item still multiplies (head dim 128 has no room
  // beside three key/value slots)
  static constexpr int QB = D == 64 ? 2 : 1;
  static constexpr int ST = (D == 128) ? (kAlt ? 4 : 3) : (kAlt ? 8 : 6);     // ring slots: what fits beside Q and P
  // Q K^T runs this many key tiles ahead of P V: in both forms one product of each stream is then in flight ahead
  static constexpr int LA = kAlt ? 2 : 1;
  static constexpr int kData = QB * NQ * kTileBytes + 2 * kPBytes + ST * kTileBytes;
  static constexpr int kBars = 8 * (2 * QB + 2 * ST + 2 * kDesc + 15);
  static constexpr int kDescOff = (kBars + 15) / 16 * 16;
  static constexpr int kTail = kDescOff + kDesc * (int)sizeof(SegDesc) + 16;
  static constexpr int kMlOff = kTail;
  static constexpr int kBytes = kData + 1024 /*alignment*/ + kTail + (kAlt ? kTile * 8 : 0) /*maxima and sums of stream 1*/;
  static_assert(kBytes <= 227 * 1024, "shared memory");
  static constexpr uint32_t kIdescQK = (1u << 4) | (1u << 7) | (1u << 10) | ((uint32_t)(kTile >> 3) << 17) | ((uint32_t)(kTile >> 4) << 24);
  static constexpr uint32_t kIdescPV = (1u << 4) | (1u << 7) | (1u << 10) | (1u << 16) | ((uint32_t)(D >> 3) << 17) | ((uint32_t)(kTile >> 4) << 24);
};

struct SegTcArgs {
  int box_q;        // queries come as boxes of map_q: box_tokens tokens of box_samples samples are the 128 rows of a tile
  int box_out;      // finished tiles leave as boxes of map_o
  int items;        // of both passes
};

__device__ __forceinline__ void tma_load_5d(uint32_t dst, const CUtensorMap* map, uint32_t bar, int c0, int c1, int c2, int c3, int c4) {
  asm volatile(
      "cp.async.bulk.tensor.5d.shared::cluster.global.mbarrier::complete_tx::bytes [%0], [%1, {%3, %4, %5, %6, %7}], [%2];"
      ::"r"(dst), "l"(map), "r"(bar), "r"(c0), "r"(c1), "r"(c2), "r"(c3), "r"(c4) : "memory");
}
__device__ __forceinline__ void tma_store_5d(const CUtensorMap* map, uint32_t src, int c0, int c1, int c2, int c3, int c4) {
  asm volatile("cp.async.bulk.tensor.5d.global.shared::cta.bulk_group [%0, {%2, %3, %4, %5, %6}], [%1];"
               ::"l"(map), "r"(src), "r"(c0), "r"(c1), "r"(c2), "r"(c3), "r"(c4) : "memory");
}

template <int D, bool kAlt>
__global__ void __launch_bounds__(kThreadsS, 1)
seg_tc_kernel(const __grid_constant__ CUtensorMap map_q, const __grid_constant__ CUtensorMap map_o,
              const __grid_constant__ CUtensorMap map_k0, const __grid_constant__ CUtensorMap map_v0,
              const __grid_constant__ CUtensorMap map_k1, const __grid_constant__ CUtensorMap map_v1,
              const __grid_constant__ SegParams p, const int pass0, const SegTcArgs x) {
  using C = SegCfg<D, kAlt>;
  constexpr int ST = C::ST, LA = C::LA, QB = C::QB;
  extern __shared__ unsigned char smem_raw[];
  const uint32_t base = (smem_addr(smem_raw) + 1023u) & ~1023u;
  unsigned char* base_ptr = smem_raw + (base - smem_addr(smem_raw));
  const uint32_t sQ = base, sP = sQ + QB * C::NQ * C::kTileBytes, sR = sP + 2 * C::kPBytes;
  const uint32_t bars = base + C::kData;
  auto bar_q = [&](int b) { return bars + 8 * b; };                          // queries have arrived
  auto bar_q_free = [&](int b) { return bars + 8 * (QB + b); };              // the item's last Q K^T has run
  auto bar_full = [&](int s) { return bars + 8 * (2 * QB + s); };
  auto bar_empty = [&](int s) { return bars + 8 * (2 * QB + ST + s); };
  auto bar_d_full = [&](int s) { return bars + 8 * (2 * QB + 2 * ST + s); };
  auto bar_d_empty = [&](int s) { return bars + 8 * (2 * QB + 2 * ST + kDesc + s); };
  constexpr int kB = 2 * QB + 2 * ST + 2 * kDesc;
  auto bar_s_full = [&](int s) { return bars + 8 * (kB + s); };
  auto bar_s_free = [&](int s) { return bars + 8 * (kB + 2 + s); };
  auto bar_p_full = [&](int s) { return bars + 8 * (kB + 4 + s); };
  auto bar_pv = [&](int s) { return bars + 8 * (kB + 6 + s); };
  auto bar_stage = [&](int s) { return bars + 8 * (kB + 8 + s); };           // the staged output has been read
  const uint32_t bar_o_final = bars + 8 * (kB + 10), bar_o_free = bars + 8 * (kB + 11);
  const uint32_t bar_x = bars + 8 * (kB + 12);                               // kAlt: stream 1 has left its maxima and sums
  auto bar_staged = [&](int s) { return bars + 8 * (kB + 13 + s); };         // every row of the output has been staged
  SegDesc* desc = reinterpret_cast<SegDesc*>(base_ptr + C::kData + C::kDescOff);
  uint32_t* tmem_slot = reinterpret_cast<uint32_t*>(base_ptr + C::kData + C::kTail - 16);
  volatile int* abort_flag = reinterpret_cast<volatile int*>(base_ptr + C::kData + C::kTail - 8);
  float2* ml_x = reinterpret_cast<float2*>(base_ptr + C::kData + C::kMlOff);

  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
  const SegArgs& a = p.a;

  if (threadIdx.x == 0) {
    for (int b = 0; b < QB; ++b) {
      mbar_init(bar_q(b), x.box_q ? 1 : 32);
      mbar_init(bar_q_free(b), 1);
    }
    for (int s = 0; s < ST; ++s) {
      mbar_init(bar_full(s), 1);
      mbar_init(bar_empty(s), 1);
    }
    for (int s = 0; s < kDesc; ++s) {
      mbar_init(bar_d_full(s), 1);
      mbar_init(bar_d_empty(s), 11);        // producer, query warp, issuer, eight softmax warps
    }
    for (int s = 0; s < 2; ++s) {
      mbar_init(bar_s_full(s), 1);
      mbar_init(bar_s_free(s), kTile);
      mbar_init(bar_p_full(s), kTile);
      mbar_init(bar_pv(s), 1);
      mbar_init(bar_stage(s), x.box_out ? 1 : kTile);
      mbar_init(bar_staged(s), kTile);
    }
    mbar_init(bar_o_final, 1);
    mbar_init(bar_o_free, 2 * kTile);
    mbar_init(bar_x, kTile);
    *abort_flag = 0;
    asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
  }
  if (warp == 8) {
    asm volatile("tcgen05.alloc.cta_group::1.sync.aligned.shared::cta.b32 [%0], 512;" ::"r"(smem_addr(tmem_slot)) : "memory");
    asm volatile("tcgen05.relinquish_alloc_permit.cta_group::1.sync.aligned;" ::: "memory");
  }
  tc_fence_before();
  __syncthreads();
  tc_fence_after();
  const uint32_t tmem = *tmem_slot;
  auto tm_S = [&](int s) { return tmem + (uint32_t)(s * kTile); };
  auto tm_O = [&](int s) { return tmem + (uint32_t)(2 * kTile + s * D); };
  // (a warp leaves its loops together: the TMEM instructions and shuffles need it converged)
  auto wait = [&](uint32_t bar, uint32_t parity) {
    return __all_sync(0xffffffffu, mbar_wait(bar, parity, abort_flag) ? 1 : 0) != 0;
  };
  // next descriptor: false at the end (or when a wait ran out).  di counts the descriptors read so far.
  auto next_desc = [&](int& di, SegDesc& d) {
    const int slot = di % kDesc;
    if (!wait(bar_d_full(slot), (di / kDesc) & 1)) return false;
    d = desc[slot];
    __syncwarp();
    if (lane == 0) mbar_arrive(bar_d_empty(slot));
    ++di;
    return d.n >= 0;
  };
  SegDesc d;
  int di = 0;

  // Every role walks through the same items; one whose rows see no key is only known to the softmax warps (they write
  // its zeros) and counts for nobody else, so all other barrier phases count the remaining items and their tiles.
  // (setmaxnreg: 384 threads start with 168 registers each; 56 for the third warpgroup frees exactly what 224 for the
  // other two takes)
  if (warp >= 8) {
    asm volatile("setmaxnreg.dec.sync.aligned.u32 56;");
    if (warp == 11) {
      // ------------------------------------------------------------------ scheduler
      for (int w = blockIdx.x, i = 0;; w += gridDim.x, ++i) {
        SegDesc o;
        o.n = -1;
        o.na = o.b0 = o.h_kv = o.row0 = o.base0 = o.base1 = o.part = o.len0 = o.len1 = o.own = o.kv0 = 0;
        if (w < x.items) {
          const int q = pass0 == 0 && w >= p.pass[0].items ? 1 : pass0;
          const SegPass& ps = p.pass[q];
          const SegItem it = seg_item(ps, a.N_kv, C::kRows, q != pass0 ? w - p.pass[0].items : w);
          const SegKeys kk = seg_keys(p, ps, it, C::kRows, kTile);
          o.n = kk.end - kk.begin;
          o.na = max(0, min(o.n, kk.n0 - kk.begin));
          o.b0 = it.block * ps.block_samples;
          o.h_kv = it.h_kv;
          o.row0 = it.row0 | (q << 30);                // rows of a block stay below 2^30
          o.base0 = kk.begin * kTile;
          o.base1 = (kk.begin - kk.n0) * kTile;
          o.part = ps.part0 + it.split;
          o.len0 = kk.len0;
          o.len1 = kk.len1;
          o.own = o.na < o.n ? seg_len(p, 1, o.b0) : 0;
          o.kv0 = o.b0 / a.per_group;
        }
        const int slot = i % kDesc;
        if (i >= kDesc && !wait(bar_d_empty(slot), ((i / kDesc) & 1) ^ 1)) break;
        if (lane == 0) {
          desc[slot] = o;
          mbar_arrive(bar_d_full(slot));
        }
        if (o.n < 0) break;
      }
    } else if (warp == 10) {
      // ------------------------------------------------------------------ query rows one by one
      constexpr int CPR = D / 8, RPI = 32 / CPR;     // 16-byte chunks per row, rows per warp instruction
      const int cc = lane % CPR, sub = lane / CPR;
      const __nv_bfloat16* q = (const __nv_bfloat16*)a.q + cc * 8;
      int iter = 0;
      while (next_desc(di, d)) {
        if (d.n == 0 || x.box_q) continue;
        const int qb = iter % QB;
        if (iter >= QB && !wait(bar_q_free(qb), ((iter / QB) & 1) ^ 1)) break;
        const int row0 = d.row0 & 0x3fffffff, block_samples = p.pass[d.row0 >> 30].block_samples;
        for (int blk = 0; blk < C::kRows / 32; ++blk) {
          // lane l knows row blk * 32 + l; the rows are then copied RPI at a time
          const SegRow r = seg_row(p, block_samples, d.b0, d.h_kv, row0 + blk * 32 + lane);
          const int64_t off = r.real ? r.b * a.q_smp + r.t * a.q_tok + (int64_t)r.h * D : -1;
          const uint32_t dst = sQ + (uint32_t)((qb * C::NQ + (blk >> 2)) * C::kTileBytes + (cc >> 3) * C::kSub + (blk & 3) * 32 * 128);
#pragma unroll 4
          for (int i = 0; i < 32 / RPI; ++i) {
            const int rl = i * RPI + sub;
            const int64_t o = __shfl_sync(0xffffffffu, off, rl);
            cp_async_16(dst + (uint32_t)(rl * 128 + (((cc & 7) ^ (rl & 7)) << 4)), q + (o < 0 ? 0 : o), o < 0 ? 0u : 16u);
          }
        }
        cp_async_arrive(bar_q(qb));
        ++iter;
      }
      cp_async_wait_all();
    } else if (warp == 9) {
      // ------------------------------------------------------------------ TMA producer
      int pos = 0, iter = 0;           // ring loads and items so far
      bool ok = true;
      while (ok && next_desc(di, d)) {
        if (d.n == 0) continue;
        const int n = d.n, qb = iter % QB;
        auto load = [&](bool is_v, int i) {
          const int st = pos % ST;
          if (!wait(bar_empty(st), ((pos / ST) & 1) ^ 1)) return false;
          if (lane == 0) {
            const bool s1 = i >= d.na;
            const CUtensorMap* m = s1 ? (is_v ? &map_v1 : &map_k1) : (is_v ? &map_v0 : &map_k0);
            mbar_expect_tx(bar_full(st), C::kTileBytes);
            for (int db = 0; db < C::DB; ++db)
              tma_load_4d(sR + st * C::kTileBytes + db * C::kSub, m, bar_full(st), db * 64, (s1 ? d.base1 : d.base0) + i * kTile, d.h_kv,
                          s1 ? d.b0 : d.kv0);
          }
          ++pos;
          return true;
        };
        auto load_q = [&]() {
          if (!x.box_q) return true;
          if (iter >= QB && !wait(bar_q_free(qb), ((iter / QB) & 1) ^ 1)) return false;
          if (lane == 0) {
            mbar_expect_tx(bar_q(qb), C::NQ * C::kTileBytes);
            const bool mixed = p.pass[d.row0 >> 30].block_samples > 1;
            for (int q = 0; q < C::NQ; ++q) {
              const int r = (d.row0 & 0x3fffffff) + q * kTile;
              const int smp = mixed ? r / (a.n_q * p.g) : 0, tok = mixed ? 0 : r / p.g;
              for (int db = 0; db < C::DB; ++db)
                tma_load_5d(sQ + (qb * C::NQ + q) * C::kTileBytes + db * C::kSub, &map_q, bar_q(qb), db * 64, 0, tok, d.h_kv, d.b0 + smp);
            }
          }
          return true;
        };
        // With one query buffer the queries must wait for the previous item's last Q K^T; the ring's free slots are filled
        // before that wait.
        const int q_after = iter < QB || QB > 1 ? -1 : min(ST, 2 * n) - 1;
        int m = 0;
        if (q_after < 0) ok = load_q();
        for (int i = 0; i < n + LA && ok; ++i) {
          if (i < n) {
            ok = load(false, i);
            if (ok && m++ == q_after) ok = load_q();
          }
          if (ok && i >= LA) {
            ok = load(true, i - LA);
            if (ok && m++ == q_after) ok = load_q();
          }
        }
        ++iter;
      }
    } else {
      // ------------------------------------------------------------------ MMA issuer (warp converged, one lane issues)
      const uint32_t el = elect_one();
      const uint32_t q_lo = desc_lo(sQ, 16), p_lo = desc_lo(sP, 16), k_lo = desc_lo(sR, 16), v_lo = desc_lo(sR, C::kSub);
      bool ok = true;
      int pos = 0, iter = 0;
      int qk_n0 = 0, qk_n1 = 0, pv_n0 = 0, pv_n1 = 0;   // products issued so far per stream
      while (ok && next_desc(di, d)) {
        const int n = d.n, qb = iter % QB;
        if (n == 0) continue;
        ok = wait(bar_q(qb), (iter / QB) & 1);
        if (!ok) break;
        if (!x.box_q) fence_proxy_async();
        auto qk = [&](int i) {
          const int st = pos % ST;
          if (!wait(bar_full(st), (pos / ST) & 1)) return false;
#pragma unroll
          for (int s = 0; s < 2; ++s) {
            if (kAlt && (i & 1) != s) continue;
            int& cnt = s ? qk_n1 : qk_n0;
            if (cnt > 0 && !wait(bar_s_free(s), (cnt - 1) & 1)) return false;
            ++cnt;
            tc_fence_after();
            const uint32_t a_lo = q_lo + ((uint32_t)((qb * C::NQ + (kAlt ? 0 : s)) * C::kTileBytes) >> 4);
            const uint32_t b_lo = k_lo + ((uint32_t)(st * C::kTileBytes) >> 4);
            mma_ss<false>(tm_S(s), a_lo, b_lo, kDescHi, C::kIdescQK, el);
#pragma unroll
            for (int ks = 1; ks < D / 16; ++ks) {
              constexpr int kSub16 = C::kSub >> 4;
              const uint32_t off = (uint32_t)((ks >> 2) * kSub16 + (ks & 3) * 2);
              mma_ss<true>(tm_S(s), a_lo + off, b_lo + off, kDescHi, C::kIdescQK, el);
            }
            tc_commit(bar_s_full(s), el);
          }
          tc_commit(bar_empty(st), el);
          if (i == n - 1) tc_commit(bar_q_free(qb), el);     // the queries have been read for the last time
          ++pos;
          return true;
        };
        auto pv = [&](int i) {
          const int st = pos % ST;
          if (!wait(bar_full(st), (pos / ST) & 1)) return false;
          // the first product of an item overwrites the accumulators: the previous item's epilogue must have read them
          if (i == 0 && iter > 0 && !wait(bar_o_free, (iter - 1) & 1)) return false;
#pragma unroll
          for (int s = 0; s < 2; ++s) {
            if (kAlt && (i & 1) != s) continue;
            int& cnt = s ? pv_n1 : pv_n0;
            if (!wait(bar_p_full(s), cnt & 1)) return false;
            ++cnt;
            tc_fence_after();
            const uint32_t a_lo = p_lo + ((uint32_t)(s * C::kPBytes) >> 4), b_lo = v_lo + ((uint32_t)(st * C::kTileBytes) >> 4);
            mma_ss_rt(tm_O(s), a_lo, b_lo, kDescHi, C::kIdescPV, (kAlt ? i > 1 : i > 0) ? 1u : 0u, el);
#pragma unroll
            for (int k = 1; k < kTile / 16; ++k) {
              constexpr int kSub16 = C::kSub >> 4;
              mma_ss_rt(tm_O(s), a_lo + (uint32_t)((k >> 2) * kSub16 + (k & 3) * 2), b_lo + k * (2048 >> 4), kDescHi, C::kIdescPV, 1u, el);
            }
            tc_commit(bar_pv(s), el);
          }
          tc_commit(bar_empty(st), el);
          ++pos;
          return true;
        };
        for (int i = 0; i < n + LA && ok; ++i) {
          if (i < n) ok = qk(i);
          if (ok && i >= LA) ok = pv(i - LA);
        }
        if (ok) tc_commit(bar_o_final, el);
        ++iter;
      }
    }
  } else {
    asm volatile("setmaxnreg.inc.sync.aligned.u32 224;");
    // ------------------------------------------------------------------ softmax: one thread per row and stream
    const int s = warp >> 2;                     // stream
    const int r = (warp & 3) * 32 + lane;        // row inside the tile == TMEM lane
    const uint32_t lane_off = (uint32_t)((warp & 3) * 32) << 16;
    const uint32_t tS = tm_S(s) + lane_off, tO = tm_O(s) + lane_off;
    const uint32_t p_row = sP + (uint32_t)(s * C::kPBytes + r * 128);
    bool ok = true;
    int iter = 0, cnt = 0, pos0 = 0;             // items; tiles of this stream; ring loads before the current item
    int staged = 0;                              // outputs staged in this stream's P tile so far
    while (ok && next_desc(di, d)) {
      const int n = d.n;
      const int row0 = (d.row0 & 0x3fffffff) + (kAlt ? 0 : s * kTile);       // of the stream's tile
      const SegRow row = seg_row(p, p.pass[d.row0 >> 30].block_samples, d.b0, d.h_kv, row0 + r);
      const bool warp_real = __any_sync(0xffffffffu, row.real);
      const int lim1 = seg_limit1(a, d.own, row.t);
      float m_used = -INFINITY, l_run = 0.f;
      bool any_key = false;
      for (int i = kAlt ? s : 0; i < n; i += kAlt ? 2 : 1, ++cnt) {
        ok = wait(bar_s_full(s), cnt & 1);
        if (!ok) break;
        const bool s1 = i >= d.na;
        const int key0 = (s1 ? d.base1 : d.base0) + i * kTile;
        const int real = (s1 ? d.len1 : d.len0) - key0;      // real keys of this tile
        tc_fence_after();
        if (!warp_real) {
          // rows behind the last one: nothing is computed, the barriers are kept in step (what their P rows hold only
          // reaches their own accumulator rows, which nobody reads)
          mbar_arrive(bar_s_free(s));
          if (cnt > 0) ok = wait(bar_pv(s), (cnt - 1) & 1);       // no warp runs a phase ahead of the others
          if (!ok) break;
        } else {
          float sv[kTile];
#pragma unroll
          for (int c = 0; c < 4; ++c) tmem_ld32(tS + c * 32, *reinterpret_cast<float(*)[32]>(&sv[c * 32]));
          tmem_ld_wait();
          tc_fence_before();
          mbar_arrive(bar_s_free(s));             // the scores are in registers
          const int valid = s1 ? lim1 - key0 : real;
          if (valid < kTile) {
#pragma unroll
            for (int c = 0; c < kTile; ++c)
              if (c >= valid) sv[c] = -INFINITY;
          }
          if (i == (kAlt ? s : 0)) {
            // the first tile fixes the row's reference maximum.  A row that sees none of its keys sees no later key
            // either (limits are a prefix of segment 1, and segment 0 has no limits below its length).
            any_key = valid > 0;
            float m8[8];
#pragma unroll
            for (int j = 0; j < 8; ++j) m8[j] = sv[j];
#pragma unroll
            for (int c = 8; c < kTile; c += 8) {
#pragma unroll
              for (int j = 0; j < 8; ++j) m8[j] = fmaxf(m8[j], sv[c + j]);
            }
            m_used = fmaxf(fmaxf(fmaxf(m8[0], m8[1]), fmaxf(m8[2], m8[3])), fmaxf(fmaxf(m8[4], m8[5]), fmaxf(m8[6], m8[7]))) * p.scale_log2;
            if (!any_key) m_used = 0.f;
          }
          if (cnt > 0) {
            // the P tile is free once the stream's previous product has read it, and the previous item's staged output
            // has left it
            ok = wait(bar_pv(s), (cnt - 1) & 1);
            if (ok && staged > 0 && i == (kAlt ? s : 0)) ok = wait(bar_stage(s), (staged - 1) & 1);
            if (!ok) break;
          }
          const uint64_t scale2 = pack2(p.scale_log2, p.scale_log2), negm2 = pack2(-m_used, -m_used);
          uint64_t acc2[4] = {0ull, 0ull, 0ull, 0ull};
          auto store_p16 = [&](int c, const uint32_t* v) {
#pragma unroll
            for (int q = 0; q < 4; ++q) {
              const int c16 = c * 4 + q;
              st_shared_16(p_row + (uint32_t)((c16 >> 3) * C::kSub + (((c16 & 7) ^ (r & 7)) << 4)), v[4 * q], v[4 * q + 1], v[4 * q + 2], v[4 * q + 3]);
            }
          };
          uint32_t pk[64];
#pragma unroll
          for (int j = 0; j < 64; ++j) {
            const uint64_t x2 = fma2(pack2(sv[2 * j], sv[2 * j + 1]), scale2, negm2);
            float p0, p1;
            if ((j & 7) == 0) {
              exp2_poly2(x2, p0, p1);             // one pair in eight on the FMA pipes, which the exp2 unit leaves idle
            } else {
              float t0, t1;
              unpack2(x2, t0, t1);
              p0 = ex2(t0);
              p1 = ex2(t1);
            }
            acc2[j & 3] = add2(acc2[j & 3], pack2(p0, p1));
            pk[j] = pack_bf16x2(p0, p1);
            if ((j & 15) == 15) store_p16(j >> 4, &pk[j - 15]);
          }
          float sum, a0, a1;
          unpack2(add2(add2(acc2[0], acc2[1]), add2(acc2[2], acc2[3])), a0, a1);
          sum = a0 + a1;
          const bool grew = !(sum <= 256.f * 128.f);           // some exponent above 2^8; also inf and NaN
          if (__any_sync(0xffffffffu, grew)) {
            // rare: raise the reference to the row's maximum, rescale O, repeat the pass
            float mraw = sv[0];
#pragma unroll
            for (int c = 1; c < kTile; ++c) mraw = fmaxf(mraw, sv[c]);
            const float delta = fmaxf(fmaf(mraw, p.scale_log2, -m_used), 0.f);
            const float f = ex2(-delta);
            m_used += delta;
            l_run *= f;
            if (i >= (kAlt ? 2 : 1)) {            // the previous product is complete (waited for above)
              tc_fence_after();
#pragma unroll
              for (int c = 0; c < D / 32; ++c) {
                float ov[32];
                tmem_ld32(tO + c * 32, ov);
                tmem_ld_wait();
                uint32_t ou[32];
#pragma unroll
                for (int j = 0; j < 32; ++j) ou[j] = __float_as_uint(ov[j] * f);
                tmem_st32(tO + c * 32, ou);
              }
              tmem_st_wait();
            }
            sum = 0.f;
#pragma unroll
            for (int c = 0; c < 4; ++c) {
              uint32_t pr[16];
#pragma unroll
              for (int j = 0; j < 16; ++j) {
                const float p0 = ex2(fmaf(sv[c * 32 + 2 * j], p.scale_log2, -m_used));
                const float p1 = ex2(fmaf(sv[c * 32 + 2 * j + 1], p.scale_log2, -m_used));
                sum += p0 + p1;
                pr[j] = pack_bf16x2(p0, p1);
              }
              store_p16(c, pr);
            }
          }
          l_run += sum;
        }
        // a tile that ends inside: rows of V behind the last real key become zeros.  One stream does it for both (the
        // issuer waits for stream 0's P before either product).
        if (real < kTile && (kAlt || s == 0)) {
          const int vpos = pos0 + min(n, i + LA + 1) + i, st = vpos % ST;      // loads before V_i: K_0 .. K_(i+LA), V_0 .. V_(i-1)
          ok = wait(bar_full(st), (vpos / ST) & 1);
          if (!ok) break;
          if (r >= real) {
            for (int c = 0; c < D / 8; ++c)
              st_shared_16(sR + (uint32_t)(st * C::kTileBytes + (c >> 3) * C::kSub + r * 128 + ((c & 7) << 4)), 0u, 0u, 0u, 0u);
          }
        }
        tc_fence_before();
        fence_proxy_async();                      // P and zeroed V rows: generic stores that the tensor core will read
        mbar_arrive(bar_p_full(s));
      }
      if (!ok) break;
      if (n > 0) {
        ok = wait(bar_o_final, iter & 1);
        if (!ok) break;
        tc_fence_after();
      }
      if (!any_key) {
        m_used = -INFINITY;
        l_run = 0.f;
      }
      // epilogue.  kAlt = true: stream 0 finishes the rows from both accumulators (same TMEM lanes, other columns)
      float f0 = any_key ? 1.f : 0.f, f1 = 0.f;   // weights of the accumulators; one of weight 0 may hold anything
      float m_all = m_used, l_all = l_run;
      if (kAlt && n > 0) {
        if (s == 1) {
          // stream 0 has read the previous item's values
          if (iter > 0) ok = wait(bar_o_free, (iter - 1) & 1);
          if (!ok) break;
          ml_x[r] = make_float2(m_used, l_run);
          mbar_arrive(bar_x);
        } else {
          ok = wait(bar_x, iter & 1);
          if (!ok) break;
          const float2 x1 = ml_x[r];
          m_all = fmaxf(m_used, x1.x);
          f0 = m_used == -INFINITY ? 0.f : ex2(m_used - m_all);
          f1 = x1.x == -INFINITY ? 0.f : ex2(x1.x - m_all);
          l_all = f0 * l_run + f1 * x1.y;
        }
      }
      const bool writes = !kAlt || s == 0;        // this stream's warps write the item's rows
      const int64_t gr = ((int64_t)row.b * a.n_q + row.t) * a.N_h + row.h;
      if (writes && p.direct) {
        // the finished rows are staged in the stream's P tile (its last product is complete) and leave as a box, or row by
        // row with 16-byte stores, a row or two per instruction
        if (staged > 0 && n == 0) {               // otherwise waited for before the item's first P
          ok = wait(bar_stage(s), (staged - 1) & 1);
          if (!ok) break;
        }
        const float inv = l_all > 0.f ? 1.f / l_all : 0.f;
        f0 *= inv;
        f1 *= inv;
        const uint32_t stage = sP + (uint32_t)(s * C::kPBytes + r * 128);
        if (warp_real) {
#pragma unroll
          for (int c = 0; c < D / 32; ++c) {
            float ov[32];
            tmem_ld32(tO + c * 32, ov);
            tmem_ld_wait();
#pragma unroll
            for (int j = 0; j < 32; ++j) ov[j] = f0 != 0.f ? ov[j] * f0 : 0.f;
            if constexpr (kAlt) {
              float o1[32];
              tmem_ld32(tm_O(1) + lane_off + c * 32, o1);
              tmem_ld_wait();
#pragma unroll
              for (int j = 0; j < 32; ++j) ov[j] += f1 != 0.f ? o1[j] * f1 : 0.f;
            }
#pragma unroll
            for (int q = 0; q < 4; ++q) {
              const int c16 = c * 4 + q;
              st_shared_16(stage + (uint32_t)((c16 >> 3) * C::kSub + (((c16 & 7) ^ (r & 7)) << 4)), pack_bf16x2(ov[q * 8 + 0], ov[q * 8 + 1]),
                           pack_bf16x2(ov[q * 8 + 2], ov[q * 8 + 3]), pack_bf16x2(ov[q * 8 + 4], ov[q * 8 + 5]),
                           pack_bf16x2(ov[q * 8 + 6], ov[q * 8 + 7]));
            }
          }
          if (row.real && a.lse)
            a.lse[((int64_t)row.b * a.N_h + row.h) * a.n_q + row.t] = l_all > 0.f ? (m_all + log2f(l_all)) * 0.6931471805599453f : -INFINITY;
        }
        if (n > 0) {
          tc_fence_before();
          mbar_arrive(bar_o_free);                // the accumulators have been read
        }
        if (x.box_out) {
          fence_proxy_async();
          mbar_arrive(bar_staged(s));
          if ((warp & 3) == 0) ok = wait(bar_staged(s), staged & 1);
          if (!ok) break;
          if ((warp & 3) == 0 && lane == 0) {
            if (row0 < a.n_q * p.g) {
              for (int db = 0; db < C::DB; ++db)
                tma_store_5d(&map_o, sP + s * C::kPBytes + db * C::kSub, db * 64, 0, row0 / p.g, d.h_kv, d.b0);
              tma_store_commit_wait();
            }
            mbar_arrive(bar_stage(s));
          }
        } else {
          __syncwarp();
          constexpr int CPR = D / 8, RPI = 32 / CPR;
          const int cc = lane % CPR, sub = lane / CPR;
          const int64_t off = row.real ? row.b * a.o_smp + row.t * a.o_tok + (int64_t)row.h * D : -1;
          const unsigned char* src = base_ptr + (sP - base) + s * C::kPBytes + (cc >> 3) * C::kSub + (warp & 3) * 32 * 128;
#pragma unroll 4
          for (int i = 0; i < 32 / RPI; ++i) {
            const int rl = i * RPI + sub;
            const int64_t o = __shfl_sync(0xffffffffu, off, rl);
            if (o >= 0)
              *reinterpret_cast<uint4*>((__nv_bfloat16*)a.out + o + cc * 8) =
                  *reinterpret_cast<const uint4*>(src + rl * 128 + (((cc & 7) ^ (rl & 7)) << 4));
          }
          __syncwarp();
          mbar_arrive(bar_stage(s));
        }
        ++staged;
      } else {
        if (writes && warp_real) {
          const int64_t pr = (int64_t)d.part * p.rows + gr;
#pragma unroll
          for (int c = 0; c < D / 32; ++c) {
            float ov[32];
            __syncwarp();
            tmem_ld32(tO + c * 32, ov);
            tmem_ld_wait();
#pragma unroll
            for (int j = 0; j < 32; ++j) ov[j] = f0 != 0.f ? ov[j] * f0 : 0.f;
            if constexpr (kAlt) {
              float o1[32];
              tmem_ld32(tm_O(1) + lane_off + c * 32, o1);
              tmem_ld_wait();
#pragma unroll
              for (int j = 0; j < 32; ++j) ov[j] += f1 != 0.f ? o1[j] * f1 : 0.f;
            }
            if (row.real) {
              float* dst = p.part_o + pr * D + c * 32;
#pragma unroll
              for (int q = 0; q < 8; ++q)
                *reinterpret_cast<float4*>(dst + q * 4) = make_float4(ov[q * 4], ov[q * 4 + 1], ov[q * 4 + 2], ov[q * 4 + 3]);
            }
          }
          if (row.real) p.part_ml[pr] = make_float2(m_all, l_all);
        }
        if (n > 0) {
          tc_fence_before();
          mbar_arrive(bar_o_free);
        }
      }
      if (n > 0) {
        ++iter;
        pos0 += 2 * n;
      }
    }
  }
  tc_fence_before();
  __syncthreads();
  if (threadIdx.x == 0 && *abort_flag) atomicOr(p.status, ST_TIMEOUT);
  if (warp == 8) {
    tc_fence_after();
    asm volatile("tcgen05.dealloc.cta_group::1.sync.aligned.b32 %0, 512;" ::"r"(tmem) : "memory");
  }
}

bool encode(CUtensorMap* map, const void* ptr, int rank, const cuuint64_t* dims, const cuuint64_t* strides, const cuuint32_t* box) {
  EncodeTiledFn fn = encode_fn();
  if (!fn) return false;
  const cuuint32_t estr[5] = {1, 1, 1, 1, 1};
  return fn(map, CU_TENSOR_MAP_DATA_TYPE_BFLOAT16, rank, const_cast<void*>(ptr), dims, strides, box, estr,
            CU_TENSOR_MAP_INTERLEAVE_NONE, CU_TENSOR_MAP_SWIZZLE_128B, CU_TENSOR_MAP_L2_PROMOTION_L2_256B,
            CU_TENSOR_MAP_FLOAT_OOB_FILL_NONE) == CUDA_SUCCESS;
}
// [blocks, n, N_kv, D] with strides, viewed as (d, row, head, block); box = 64 columns x 128 rows
bool make_kv_map(CUtensorMap* map, const void* ptr, int blocks, int n, int N_kv, int D, int64_t tok, int64_t smp) {
  const cuuint64_t dims[4] = {(cuuint64_t)D, (cuuint64_t)n, (cuuint64_t)N_kv, (cuuint64_t)blocks};
  const cuuint64_t strides[3] = {(cuuint64_t)tok * 2, (cuuint64_t)D * 2, (cuuint64_t)smp * 2};
  const cuuint32_t box[4] = {64, kTile, 1, 1};
  return encode(map, ptr, 4, dims, strides, box);
}
// [B, n_q, N_kv * g, D] viewed as (d, head of the group, token, group, sample); box = 64 columns x g heads x tokens x samples
bool make_q_map(CUtensorMap* map, const void* ptr, const SegArgs& a, int g, int64_t tok, int64_t smp, int box_tokens, int box_samples) {
  const cuuint64_t dims[5] = {(cuuint64_t)a.D, (cuuint64_t)g, (cuuint64_t)a.n_q, (cuuint64_t)a.N_kv, (cuuint64_t)a.B};
  const cuuint64_t strides[4] = {(cuuint64_t)a.D * 2, (cuuint64_t)tok * 2, (cuuint64_t)g * a.D * 2, (cuuint64_t)smp * 2};
  const cuuint32_t box[5] = {64, (cuuint32_t)g, (cuuint32_t)box_tokens, 1, (cuuint32_t)box_samples};
  return encode(map, ptr, 5, dims, strides, box);
}

template <int D, bool kAlt>
cudaError_t launch_tc(const SegParams& p, int pass, bool both, cudaStream_t st, int* launches) {
  const SegArgs& a = p.a;
  CUtensorMap mk[2], mv[2], mq, mo;
  memset(mk, 0, sizeof(mk));       // a segment without keys: its maps are never used
  memset(mv, 0, sizeof(mv));
  memset(&mq, 0, sizeof(mq));
  memset(&mo, 0, sizeof(mo));
  for (int s = 0; s < 2; ++s) {
    if (a.n[s] == 0) continue;
    const int blocks = s == 0 ? a.B / a.per_group : a.B;
    if (!make_kv_map(&mk[s], a.k[s], blocks, a.n[s], a.N_kv, D, a.k_tok[s], a.k_smp[s]) ||
        !make_kv_map(&mv[s], a.v[s], blocks, a.n[s], a.N_kv, D, a.v_tok[s], a.v_smp[s]))
      return cudaErrorInvalidValue;
  }
  // Row tiles that are boxes of the query tensor: whole tokens of one sample (the heads of a group divide the tile), or
  // whole samples (their rows divide it).
  SegTcArgs x;
  const bool mixed = p.pass[pass].block_samples > 1;
  const int per_sample = a.n_q * p.g;
  x.box_q = mixed ? per_sample <= kTile && kTile % per_sample == 0 : p.g <= kTile && kTile % p.g == 0;
  x.box_out = p.direct && !mixed && x.box_q;
  const int bt = mixed ? a.n_q : kTile / p.g, bs = mixed ? kTile / per_sample : 1;
  if (x.box_q && !make_q_map(&mq, a.q, a, p.g, a.q_tok, a.q_smp, bt, bs)) return cudaErrorInvalidValue;
  if (x.box_out && !make_q_map(&mo, a.out, a, p.g, a.o_tok, a.o_smp, bt, bs)) return cudaErrorInvalidValue;
  x.items = p.pass[pass].items + (both ? p.pass[1].items : 0);
  constexpr int smem = SegCfg<D, kAlt>::kBytes;
  cudaError_t e = cudaFuncSetAttribute(seg_tc_kernel<D, kAlt>, cudaFuncAttributeMaxDynamicSharedMemorySize, smem);
  if (e != cudaSuccess) return e;
  const int sms = sm_count(), grid = x.items < sms ? x.items : sms;
  ++*launches;
  seg_tc_kernel<D, kAlt><<<grid, kThreadsS, smem, st>>>(mq, mo, mk[0], mv[0], mk[1], mv[1], p, pass, x);
  return cudaGetLastError();
}

}  // namespace

cudaError_t launch_seg_tc(const SegParams& p, int pass, bool both, bool alt, cudaStream_t st, int* launches) {
  switch (p.a.D) {
    case 64: return alt ? launch_tc<64, true>(p, pass, both, st, launches) : launch_tc<64, false>(p, pass, both, st, launches);
    case 128: return alt ? launch_tc<128, true>(p, pass, both, st, launches) : launch_tc<128, false>(p, pass, both, st, launches);
    default: return cudaErrorInvalidConfiguration;
  }
}

}  // namespace swam
