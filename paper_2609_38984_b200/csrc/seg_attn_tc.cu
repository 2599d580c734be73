// Segment attention for bf16 tensors on the 5th-generation tensor cores (tcgen05 + TMEM), keys and values fed by TMA:
// the kernel for many query rows per key/value head (head dim 64 and 128).
//
// A persistent CTA per SM walks through work items (seg_attn.cuh): a row tile and a range of 128-key tiles.
//   warp 11      scheduler: decodes the items ahead of everybody else (divisions, lengths from memory) into a small ring of
//                descriptors that all other warps read
//   warp 9       TMA producer: K and V tiles into one ring of shared-memory slots, in the order the tensor pipe uses them,
//                and the queries where a row tile is a box of the query tensor
//   warp 10      fetches the query rows one by one where it is not (a number of heads per key/value head that does not
//                divide the tile, samples that do not tile it), with 16-byte asynchronous copies into the same layout;
//                where final results leave as boxes of the output tensor, it sends these instead
//   warp 8       one elected thread issues every tcgen05.mma: S = Q K^T into TMEM, then O += P V with P in TMEM and V in
//                shared memory; O stays in TMEM for the whole range of keys
//   warps 0-3    softmax of stream 0, one thread per row: S row from TMEM, exponentials against a running reference
//   warps 4-7    maximum (exp2 domain, raised only when the weights of 32 or 128 keys sum to more than 2^8 each on average: exact
//                either way), P as bf16; same for stream 1.  The streams' exponentials overlap each other's products.
// P goes back over its scores in TMEM (rounded to bf16, the operand type: half a step, 2^-8, of each weight).  TMEM holds three
// score buffers beside the outputs at head dim 64 and two at 128; P V of a unit (one key tile of one stream) frees the buffer
// that the Q K^T three (two) units on takes.  (At head dim 128 the chain softmax, P V, Q K^T then sets the period: 3110 clk a
// key tile for 2048 clk of tensor work.  P through shared memory breaks that chain, but its 64 KB are the second query
// buffer: a build of it, with some register spills, took 13.3 us instead of 11.1 for an item of 256 rows and 512 keys, and 65.1
// instead of 60.8 at 4096 keys.  P in halves, so that its first product starts earlier, was 3 % slower.)
// Q K^T runs ahead of P V across the borders of items.  An item's output is written after the first exponentials of the
// next one: the wait for its last product and the read of the accumulator then lie under work that is there anyway.  It
// leaves through the item's own query tiles, which are free by then; the next item's queries are in a second buffer.
// kAlt = false: a row tile has 256 rows; the streams are its two halves and share every key tile.
// kAlt = true: a row tile has at most 128 rows; both streams hold the same rows and take the key tiles in turn (over the
//   borders of items), each with its own maximum, sum and output accumulator, and are merged in the epilogue.  The memory of the second query tile
//   goes to the ring.
// A tile that ends early costs what its real keys cost: Q K^T and P V stop at the 16-key step of the last one, the exponentials
// at its 32.  Rows of V between it and the end of the step are overwritten with zeros in shared memory (0 * NaN would poison
// the row); scores behind a row's limit become -inf.
// Every wait on an mbarrier is bounded; when one runs out the kernel raises the timeout bit of the status word and every
// role falls through to the exit, where the copies and products in flight are waited for (again with a limit).
// What bounds it (cycles at the 1.65 to 1.85 GHz of this load): head dim 128, 3110 clk a key tile of an item (1.33 PFLOP/s at
// 4096 keys, 0.8 of the measured burst rate) and 4300 clk an item; head dim 64, 2300 clk a key tile, of which the exp2 unit
// (16 a clk) needs 1920, and 4400 clk an item: its first scores' maximum, the read of the accumulators, the bookkeeping between
// two items, and the instruction fetches of all that (83 % hits where items have some three key tiles; 96 % at head dim 128
// and 28).  So short items are bound by their change and not by the exp2 unit, which is 45 % active there.
#include <float.h>
#include <string.h>

#include <type_traits>

#include "tc_ptx.cuh"
#include "seg_attn.cuh"
#include "seg_maps.cuh"

namespace swam {
namespace {

constexpr int kThreadsS = 384;
constexpr int kDesc = 8;            // descriptors in flight

// One work item as every warp sees it: tiles [0, na) are 128-key tiles of segment 0 (the first one starts at key base0), the
// rest of segment 1 (tile i starts at key base1 + 128 i; base1 may be negative).  n = 0: no more items.
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
  static constexpr int NB = D == 64 ? 3 : 2;         // score buffers in TMEM
  static constexpr int kW = 32;
  static constexpr int NQ = kAlt ? 1 : 2;            // query tiles of an item
  static constexpr int kRows = NQ * kTile;
  // Query buffers.  A buffer is free again when its item's output has left through it, so Q K^T must not run into an item
  // whose buffer belongs to one with products that are still to be issued: with items of one tile it is LK items ahead.
  static constexpr int QB = D == 64 ? 3 : 2;
  static constexpr int ST = (14 - QB * NQ * DB) / DB;     // ring slots, 224 KB in all: 3 (kAlt 5) at D = 128, 8 (11) at 64
  // Key tiles that Q K^T has taken when P V takes its first one.  The ring holds K_0 .. K_(LK-1), then V_T, K_(T+LK) for
  // every T: the order on the tensor pipe.
  static constexpr int LK = kAlt ? NB : NB - 1;
  static constexpr int kData = QB * NQ * kTileBytes + ST * kTileBytes;
  static constexpr int kBars = 8 * (4 * QB + 2 * ST + 2 * kDesc + 2 * NB + 6);
  static constexpr int kDescOff = (kBars + 15) / 16 * 16;
  static constexpr int kTail = kDescOff + kDesc * (int)sizeof(SegDesc) + 16;
  static constexpr int kBytes = kData + 1024 /*alignment*/ + kTail + (kAlt ? kTile * 8 : 0) /*maxima and sums of stream 1*/;
  static_assert(ST >= 3 && kData <= 224 * 1024 && kBytes <= 227 * 1024, "shared memory");
  static constexpr uint32_t kIdescQK = (1u << 4) | (1u << 7) | (1u << 10) | ((uint32_t)(kTile >> 4) << 24);   // + N / 8 at bit 17
  static constexpr uint32_t kIdescPV = (1u << 4) | (1u << 7) | (1u << 10) | (1u << 16) | ((uint32_t)(D >> 3) << 17) | ((uint32_t)(kTile >> 4) << 24);
};

struct SegTcArgs {
  int box_q;        // queries come as boxes of map_q
  int box_out;      // finished tiles leave as boxes of map_o
  int items;        // of the passes of this launch
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
__device__ __forceinline__ void tmem_ld16(uint32_t taddr, uint32_t (&r)[16]) {
  asm volatile(
      "tcgen05.ld.sync.aligned.32x32b.x16.b32 "
      "{%0, %1, %2, %3, %4, %5, %6, %7, %8, %9, %10, %11, %12, %13, %14, %15}, [%16];"
      : "=r"(r[0]), "=r"(r[1]), "=r"(r[2]), "=r"(r[3]), "=r"(r[4]), "=r"(r[5]), "=r"(r[6]), "=r"(r[7]), "=r"(r[8]), "=r"(r[9]), "=r"(r[10]),
        "=r"(r[11]), "=r"(r[12]), "=r"(r[13]), "=r"(r[14]), "=r"(r[15])
      : "r"(taddr) : "memory");
}
// 32 bytes in one store (a whole sector)
__device__ __forceinline__ void st_global_32(void* dst, const uint32_t* v) {
  asm volatile("st.global.v8.b32 [%0], {%1, %2, %3, %4, %5, %6, %7, %8};"
               ::"l"(dst), "r"(v[0]), "r"(v[1]), "r"(v[2]), "r"(v[3]), "r"(v[4]), "r"(v[5]), "r"(v[6]), "r"(v[7]) : "memory");
}

template <int D, bool kAlt>
__global__ void __launch_bounds__(kThreadsS, 1)
seg_tc_kernel(const __grid_constant__ CUtensorMap map_q, const __grid_constant__ CUtensorMap map_o,
              const __grid_constant__ CUtensorMap map_k0, const __grid_constant__ CUtensorMap map_v0,
              const __grid_constant__ CUtensorMap map_k1, const __grid_constant__ CUtensorMap map_v1,
              const __grid_constant__ SegParams p, const int pass0, const SegTcArgs x) {
  using C = SegCfg<D, kAlt>;
  constexpr int ST = C::ST, LK = C::LK, QB = C::QB, NB = C::NB, kW = C::kW;
  extern __shared__ unsigned char smem_raw[];
  const uint32_t base = (smem_addr(smem_raw) + 1023u) & ~1023u;
  unsigned char* base_ptr = smem_raw + (base - smem_addr(smem_raw));
  const uint32_t sQ = base, sR = sQ + QB * C::NQ * C::kTileBytes;
  const uint32_t bars = base + C::kData;
  auto bar_q = [&](int b) { return bars + 8 * b; };                          // queries have arrived
  auto bar_q_free = [&](int b) { return bars + 8 * (QB + b); };              // last Q K^T has run, staged output has been read
  auto bar_full = [&](int s) { return bars + 8 * (2 * QB + s); };
  auto bar_empty = [&](int s) { return bars + 8 * (2 * QB + ST + s); };
  auto bar_d_full = [&](int s) { return bars + 8 * (2 * QB + 2 * ST + s); };
  auto bar_d_empty = [&](int s) { return bars + 8 * (2 * QB + 2 * ST + kDesc + s); };
  constexpr int kB = 2 * QB + 2 * ST + 2 * kDesc;
  auto bar_s_full = [&](int b) { return bars + 8 * (kB + b); };              // per score buffer
  auto bar_p_full = [&](int b) { return bars + 8 * (kB + NB + b); };
  auto bar_pv = [&](int s) { return bars + 8 * (kB + 2 * NB + s); };         // per stream
  const uint32_t bar_o_final = bars + 8 * (kB + 2 * NB + 2), bar_o_free = bars + 8 * (kB + 2 * NB + 3);
  const uint32_t bar_x = bars + 8 * (kB + 2 * NB + 4);                       // kAlt: stream 1 has left its maxima and sums
  // Every row of the output has been staged, per query buffer and stream.  (One barrier for all buffers could complete twice
  // before the warp that stores the tiles looks at it.)
  auto bar_staged = [&](int b, int s) { return bars + 8 * (kB + 2 * NB + 5 + 2 * b + s); };
  const uint32_t bar_drain = bars + 8 * (kB + 2 * NB + 5 + 2 * QB);          // the products in flight when a wait has run out
  SegDesc* desc = reinterpret_cast<SegDesc*>(base_ptr + C::kData + C::kDescOff);
  uint32_t* tmem_slot = reinterpret_cast<uint32_t*>(base_ptr + C::kData + C::kTail - 16);
  volatile int* abort_flag = reinterpret_cast<volatile int*>(base_ptr + C::kData + C::kTail - 8);
  float2* ml_x = reinterpret_cast<float2*>(base_ptr + C::kData + C::kTail);

  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
  const SegArgs& a = p.a;

  if (p.early && pass0 == 0) allow_next();

  if (threadIdx.x == 0) {
    for (int b = 0; b < QB; ++b) {
      mbar_init(bar_q(b), x.box_q ? 1 : 32);
      mbar_init(bar_q_free(b), 1 + (!p.direct ? 0 : C::NQ * (x.box_out ? 1 : 4)));
    }
    for (int s = 0; s < ST; ++s) {
      mbar_init(bar_full(s), 1);
      mbar_init(bar_empty(s), 1);
    }
    for (int s = 0; s < kDesc; ++s) {
      mbar_init(bar_d_full(s), 1);
      mbar_init(bar_d_empty(s), 11);        // producer, query warp, issuer, eight softmax warps
    }
    for (int b = 0; b < NB; ++b) {
      mbar_init(bar_s_full(b), 1);
      mbar_init(bar_p_full(b), 4);           // warps (an arrival of every thread would queue up at the barrier)
    }
    for (int s = 0; s < 2; ++s) {
      mbar_init(bar_pv(s), 1);
      for (int b = 0; b < QB; ++b) mbar_init(bar_staged(b, s), 4);
    }
    mbar_init(bar_o_final, 1);
    mbar_init(bar_o_free, 8);
    mbar_init(bar_x, 4);
    mbar_init(bar_drain, 1);
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
  auto tm_S = [&](int b) { return tmem + (uint32_t)(b * kTile); };
  auto tm_O = [&](int s) { return tmem + (uint32_t)(NB * kTile + s * D); };
  // (a warp leaves its loops together: the TMEM instructions and shuffles need it converged)
  auto wait = [&](uint32_t bar, uint32_t parity) {
    return __all_sync(0xffffffffu, mbar_wait(bar, parity, abort_flag) ? 1 : 0) != 0;
  };
  // one arrival for what all lanes of the warp have done
  auto arrive = [&](uint32_t bar) {
    __syncwarp();
    if (lane == 0) mbar_arrive(bar);
  };
  // 16-key steps of a tile with that many real keys
  auto steps16 = [&](int real) { return min(kTile / 16, (max(real, 1) + 15) / 16); };
  // next descriptor: false at the end (or when a wait ran out).  di counts the descriptors read so far.
  auto next_desc = [&](int& di, SegDesc& d) {
    const int slot = di % kDesc;
    if (!wait(bar_d_full(slot), (di / kDesc) & 1)) return false;
    d = desc[slot];
    __syncwarp();
    if (lane == 0) mbar_arrive(bar_d_empty(slot));
    ++di;
    return d.n > 0;
  };
  SegDesc d;
  int di = 0;

  // Every role walks through the same items, those with keys: all barrier phases count them and their tiles.  An item whose rows
  // see no key is only known to the scheduler, which writes its zeros.
  // (setmaxnreg: 384 threads start with 168 registers each; 72 for the third warpgroup frees exactly what 216 for the
  // other two takes)
  if (warp >= 8) {
    asm volatile("setmaxnreg.dec.sync.aligned.u32 72;");
    if (warp == 11) {
      // ------------------------------------------------------------------ scheduler
      // Items with keys first, for the other warps; then the rows of those without, which are written here: in the order of
      // the samples, a guided batch whose first half has no text would start 30 us late.
      int i = 0;
      bool ok = true, empty = false;               // has an item without keys been passed over
      auto walk = [&](bool keys) {
        for (int w = blockIdx.x; ok && w < x.items; w += gridDim.x) {
          const int q = pass0 == 0 && w >= p.pass[0].items ? 1 : pass0;
          const SegPass& ps = p.pass[q];
          const SegItem it = seg_item(ps, a.N_kv, C::kRows, q != pass0 ? w - p.pass[0].items : w);
          const SegKeys kk = seg_keys(p, ps, it, C::kRows, kTile);
          SegDesc o;
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
          if (o.n == 0) empty = true;
          if ((o.n > 0) != keys) continue;
          if (o.n == 0) {
            // rows of zeros (or a piece of weight 0)
            for (int r0 = 0; r0 < C::kRows; r0 += 32) {
              const SegRow r = seg_row(p, ps.block_samples, o.b0, o.h_kv, it.row0 + r0 + lane);
              if (!p.direct) {
                if (r.real) p.part_ml[(int64_t)o.part * p.rows + ((int64_t)r.b * a.n_q + r.t) * a.N_h + r.h] = make_float2(-INFINITY, 0.f);
                continue;
              }
              const int64_t off = r.real ? r.b * a.o_smp + r.t * a.o_tok + (int64_t)r.h * D : -1;
              if (r.real && a.lse) a.lse[((int64_t)r.b * a.N_h + r.h) * a.n_q + r.t] = -INFINITY;
              constexpr int CPR = D / 8, RPI = 32 / CPR;
              for (int j = 0; j < 32 / RPI; ++j) {
                const int64_t to = __shfl_sync(0xffffffffu, off, j * RPI + lane / CPR);
                if (to >= 0) *reinterpret_cast<uint4*>((__nv_bfloat16*)a.out + to + (lane % CPR) * 8) = make_uint4(0u, 0u, 0u, 0u);
              }
            }
            continue;
          }
          const int slot = i % kDesc;
          if (i >= kDesc) ok = wait(bar_d_empty(slot), ((i / kDesc) & 1) ^ 1);
          if (ok && lane == 0) {
            desc[slot] = o;
            mbar_arrive(bar_d_full(slot));
          }
          ++i;
        }
      };
      walk(true);
      const int slot = i % kDesc;
      if (ok && i >= kDesc) ok = wait(bar_d_empty(slot), ((i / kDesc) & 1) ^ 1);
      if (ok && lane == 0) {
        desc[slot].n = 0;                            // the end
        mbar_arrive(bar_d_full(slot));
      }
      if (empty) walk(false);
    } else if (warp == 10) {
      // ------------------------------------------------------------------ finished tiles, as boxes
      if (x.box_out) {
        int iter = 0;
        bool ok = true;
        while (ok && next_desc(di, d)) {
          for (int s = 0; s < C::NQ && ok; ++s) {
            ok = wait(bar_staged(iter % QB, s), (iter / QB) & 1);
            if (!ok) break;
            const int row0 = d.row0 + s * kTile;     // (one pass of single samples: no flag in row0)
            if (lane == 0) {
              if (row0 < a.n_q * p.g) {
                for (int db = 0; db < C::DB; ++db)
                  tma_store_5d(&map_o, sQ + ((iter % QB) * C::NQ + s) * C::kTileBytes + db * C::kSub, db * 64, 0, row0 / p.g, d.h_kv, d.b0);
                tma_store_commit_wait();
              }
              mbar_arrive(bar_q_free(iter % QB));
            }
            __syncwarp();
          }
          ++iter;
        }
      }
      // ------------------------------------------------------------------ or query rows one by one
      constexpr int CPR = D / 8, RPI = 32 / CPR;     // 16-byte chunks per row, rows per warp instruction
      const int cc = lane % CPR, sub = lane / CPR;
      const __nv_bfloat16* q = (const __nv_bfloat16*)a.q + cc * 8;
      int iter = 0;
      while (!x.box_out && next_desc(di, d)) {
        if (x.box_q) continue;
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
      // The key tiles of all items form one sequence T = 0, 1, ...  Behind the last K an empty slot takes the place of each
      // missing one, so that V_T is always load LK + 2 T.  A descriptor is released when the cursor of V leaves it.
      int pos = 0, iter = 0;                       // ring loads and items (of K) so far
      int ik = 0, nk = 0, iv = 0, nv = 0, dvi = 0; // next tile and tiles of the items of K (descriptor di - 1) and V (dvi - 1)
      bool ok = true, k_end = false;
      auto load = [&](const SegDesc& o, bool is_v, int i) {
        const int st = pos % ST;
        if (!wait(bar_empty(st), ((pos / ST) & 1) ^ 1)) return false;
        if (lane == 0) {
          const bool s1 = i >= o.na;
          const CUtensorMap* m = s1 ? (is_v ? &map_v1 : &map_k1) : (is_v ? &map_v0 : &map_k0);
          mbar_expect_tx(bar_full(st), C::kTileBytes);
          for (int db = 0; db < C::DB; ++db)
            tma_load_4d(sR + st * C::kTileBytes + db * C::kSub, m, bar_full(st), db * 64, (s1 ? o.base1 : o.base0) + i * kTile, o.h_kv,
                        s1 ? o.b0 : o.kv0);
        }
        ++pos;
        return true;
      };
      auto load_k = [&]() {
        if (ik == nk && !k_end) {
          const int slot = di % kDesc;
          if (!wait(bar_d_full(slot), (di / kDesc) & 1)) return false;
          ++di;
          ik = 0;
          nk = desc[slot].n;
          k_end = nk == 0;
          if (!k_end && x.box_q) {
            // the item's queries
            const int qb = iter % QB;
            if (iter >= QB && !wait(bar_q_free(qb), ((iter / QB) & 1) ^ 1)) return false;
            if (lane == 0) {
              const SegDesc& o = desc[slot];
              mbar_expect_tx(bar_q(qb), C::NQ * C::kTileBytes);
              const bool mixed = p.pass[o.row0 >> 30].block_samples > 1;
              for (int q = 0; q < C::NQ; ++q) {
                const int r = (o.row0 & 0x3fffffff) + q * kTile;
                const int smp = mixed ? r / (a.n_q * p.g) : 0, tok = mixed ? 0 : r / p.g;
                for (int db = 0; db < C::DB; ++db)
                  tma_load_5d(sQ + (qb * C::NQ + q) * C::kTileBytes + db * C::kSub, &map_q, bar_q(qb), db * 64, 0, tok, o.h_kv, o.b0 + smp);
              }
            }
          }
          ++iter;
        }
        if (!k_end) return load(desc[(di - 1) % kDesc], false, ik++);
        const int st = pos % ST;
        if (!wait(bar_empty(st), ((pos / ST) & 1) ^ 1)) return false;
        if (lane == 0) mbar_arrive(bar_full(st));
        ++pos;
        return true;
      };
      for (int j = 0; j < LK && ok; ++j) ok = load_k();
      while (ok) {
        if (iv == nv) {
          if (dvi > 0) {
            __syncwarp();
            if (lane == 0) mbar_arrive(bar_d_empty((dvi - 1) % kDesc));
          }
          // (K is a tile ahead at least, so an item that V could enter has been entered by K)
          if (dvi == di - (k_end ? 1 : 0)) break;
          nv = desc[dvi % kDesc].n;
          ++dvi;
          iv = 0;
        }
        ok = load(desc[(dvi - 1) % kDesc], true, iv++);
        if (ok) ok = load_k();
      }
      if (!ok) {
        drain_loads(bar_full(0), ST, pos);
        if (x.box_q) drain_loads(bar_q(0), QB, k_end ? iter - 1 : iter);
      }
    } else {
      // ------------------------------------------------------------------ MMA issuer (warp converged, one lane issues)
      const uint32_t el = elect_one();
      const uint32_t q_lo = desc_lo(sQ, 16), k_lo = desc_lo(sR, 16), v_lo = desc_lo(sR, C::kSub);
      // k16: 16-key steps with real keys.  A tile that ends early takes no more columns of Q K^T and steps of P V than these.
      auto issue_qk = [&](int qt, int buf, int st, int k16) {
        const uint32_t a_lo = q_lo + ((uint32_t)(qt * C::kTileBytes) >> 4), b_lo = k_lo + ((uint32_t)(st * C::kTileBytes) >> 4);
        const uint32_t idesc = C::kIdescQK + ((uint32_t)k16 << 18);
        mma_ss<false>(tm_S(buf), a_lo, b_lo, kDescHi, idesc, el);
#pragma unroll
        for (int ks = 1; ks < D / 16; ++ks) {
          constexpr int kSub16 = C::kSub >> 4;
          const uint32_t off = (uint32_t)((ks >> 2) * kSub16 + (ks & 3) * 2);
          mma_ss<true>(tm_S(buf), a_lo + off, b_lo + off, kDescHi, idesc, el);
        }
        tc_commit(bar_s_full(buf), el);
      };
      auto issue_pv = [&](int s, int buf, int st, bool accum, int k16) {
        const uint32_t b_lo = v_lo + ((uint32_t)(st * C::kTileBytes) >> 4);
        mma_ts(tm_O(s), tm_S(buf), b_lo, kDescHi, C::kIdescPV, accum ? 1u : 0u, el);
        if (k16 == kTile / 16) {
#pragma unroll
          for (int k = 1; k < kTile / 16; ++k) mma_ts(tm_O(s), tm_S(buf) + k * 8, b_lo + k * (2048 >> 4), kDescHi, C::kIdescPV, 1u, el);
        } else {
#pragma unroll 1
          for (int k = 1; k < k16; ++k) mma_ts(tm_O(s), tm_S(buf) + k * 8, b_lo + k * (2048 >> 4), kDescHi, C::kIdescPV, 1u, el);
        }
        tc_commit(bar_pv(s), el);
      };
      // The tiles of all items form one sequence for Q K^T, which runs ahead over the borders of items, and for P V behind it.
      // Every wait below ends without anything that this warp would have to issue first: the next item's queries are in the
      // other buffer, and the tensor pipe runs one thread's instructions in order, so that a score buffer is free for the
      // Q K^T issued behind the P V that reads it.
      bool ok = true, k_end = false;
      int pos = 0;                                  // ring slots taken so far
      int kn = 0, ki = 0, kiter = -1;               // item of Q K^T (descriptor di - 1): tiles, next tile, number
      int vn = 0, vi = 0, viter = -1;               // item of P V (descriptor viter)
      int kna = 0, kr0 = 0, kr1 = 0;                // their tiles of segment 0, and real keys ahead of each segment's first tile
      int vna = 0, vr0 = 0, vr1 = 0;
      int qk_u = 0, pv_u = 0;                       // units issued so far: unit u uses score buffer u % NB
      int k_st = 0, k_k16 = 0;                      // slot and steps of the current K tile
      // makes (kn, ki) the next tile of Q K^T and takes its ring slot; false at the end
      auto next_k = [&]() {
        if (ki == kn && !k_end) {
          const int slot = di % kDesc;
          ok = wait(bar_d_full(slot), (di / kDesc) & 1);
          if (!ok) return false;
          kn = desc[slot].n;
          kna = desc[slot].na;
          kr0 = desc[slot].len0 - desc[slot].base0;
          kr1 = desc[slot].len1 - desc[slot].base1;
          ++di;
          ki = 0;
          k_end = kn == 0;
        }
        if (k_end) {
          // the empty slot in the place of a missing K
          const int st = pos % ST;
          ok = wait(bar_full(st), (pos / ST) & 1);
          if (lane == 0) mbar_arrive(bar_empty(st));
          ++pos;
          return false;
        }
        if (ki == 0) {
          ++kiter;
          ok = wait(bar_q(kiter % QB), (kiter / QB) & 1);
          if (!ok) return false;
          if (!x.box_q) fence_proxy_async();
        }
        k_st = pos % ST;
        k_k16 = steps16((ki >= kna ? kr1 : kr0) - ki * kTile);
        ok = wait(bar_full(k_st), (pos / ST) & 1);
        ++pos;
        return ok;
      };
      // Q K^T of the current K tile and stream s; `last` releases the tile (and with the item's last tile the queries)
      auto qk = [&](int s, bool last) {
        tc_fence_after();
        issue_qk((kiter % QB) * C::NQ + (kAlt ? 0 : s), qk_u % NB, k_st, k_k16);
        ++qk_u;
        if (last) {
          tc_commit(bar_empty(k_st), el);
          if (++ki == kn) tc_commit(bar_q_free(kiter % QB), el);
        }
      };
      int v_st = 0, v_k16 = 0;
      // (between two steps Q K^T is a tile ahead at least: an item that P V could enter has been entered by it)
      auto v_left = [&]() { return ok && (vi < vn || viter < kiter); };
      // makes (vn, vi) the next tile of P V and takes its ring slot
      auto next_v = [&]() {
        if (vi == vn) {
          // a descriptor is released when P V leaves it
          __syncwarp();
          if (viter >= 0 && lane == 0) mbar_arrive(bar_d_empty(viter % kDesc));
          ++viter;
          vi = 0;
          const SegDesc& o = desc[viter % kDesc];
          vn = o.n;
          vna = o.na;
          vr0 = o.len0 - o.base0;
          vr1 = o.len1 - o.base1;
        }
        v_st = pos % ST;
        ok = wait(bar_full(v_st), (pos / ST) & 1);
        ++pos;
        const int real = (vi >= vna ? vr1 : vr0) - vi * kTile;
        v_k16 = steps16(real);
        if (ok && real < v_k16 * 16) {
          // rows of V behind the last real key become zeros up to the end of the product's last step
          for (int c = lane; c < (v_k16 * 16 - real) * (D / 8); c += 32) {
            const int rr = real + c / (D / 8), cc = c % (D / 8);
            st_shared_16(sR + (uint32_t)(v_st * C::kTileBytes + (cc >> 3) * C::kSub + rr * 128 + (((cc & 7) ^ (rr & 7)) << 4)), 0u, 0u, 0u, 0u);
          }
          fence_proxy_async();
          __syncwarp();
        }
        // the first product of an item overwrites the accumulators: the previous item's must have been read
        if (ok && vi == 0 && viter > 0) ok = wait(bar_o_free, (viter - 1) & 1);
        return ok;
      };
      auto pv = [&](int s, bool last) {
        ok = wait(bar_p_full(pv_u % NB), (pv_u / NB) & 1);
        if (!ok) return;
        tc_fence_after();
        issue_pv(s, pv_u % NB, v_st, kAlt ? vi > 1 : vi > 0, v_k16);
        ++pv_u;
        if (last) {
          tc_commit(bar_empty(v_st), el);
          if (++vi == vn) tc_commit(bar_o_final, el);
        }
      };
      if constexpr (!kAlt && NB == 2) {
        if (next_k()) qk(0, false), qk(1, true);
        while (v_left() && next_v()) {
          pv(0, false);
          const bool k = ok && next_k();            // (behind the last V too: only the descriptors tell that it was the last)
          if (k) qk(0, false);
          if (ok) pv(1, true);
          if (ok && k) qk(1, true);
        }
      } else if constexpr (!kAlt) {
        if (next_k()) qk(0, false), qk(1, true);
        bool half = ok && next_k();                 // stream 0 of a tile is out, stream 1 is not
        if (half) qk(0, false);
        while (v_left() && next_v()) {
          pv(0, false);
          if (ok && half) qk(1, true);
          if (ok) pv(1, true);
          half = v_left() && next_k();
          if (half) qk(0, false);
        }
      } else {
        auto qk_alt = [&]() {
          if (!next_k()) return;
          if (qk_u & 1) qk(1, true);
          else qk(0, true);
        };
        for (int j = 0; j < LK && ok; ++j) qk_alt();
        while (v_left() && next_v()) {
          if (pv_u & 1) pv(1, true);
          else pv(0, true);
          if (v_left()) qk_alt();
        }
      }
      if (!ok) {
        // a wait has run out: the products in flight must have ended before the tensor memory is given back
        tc_commit(bar_drain, el);
        drain_loads(bar_drain, 1, 1);
      }
    }
  } else {
    asm volatile("setmaxnreg.inc.sync.aligned.u32 216;");
    // ------------------------------------------------------------------ softmax: one thread per row and stream
    const int s = warp >> 2;                     // stream
    const int r = (warp & 3) * 32 + lane;        // row inside the tile == TMEM lane
    const uint32_t lane_off = (uint32_t)((warp & 3) * 32) << 16;
    const uint32_t tO = tm_O(s) + lane_off;
    bool ok = true;
    int iter = 0, cnt = 0, pos0 = 0, u0 = 0;     // items; tiles of this stream; tiles and units of finished items
    // the finished item whose output is still in the accumulators
    bool pend = false, pend_real = false, pend_warp = false;
    int pend_row = 0, pend_part = 0;             // row in the order (sample, query, head)
    int pend_lse = 0;                            // and in the order (sample, head, query)
    float pend_m = 0.f, pend_l = 0.f;
    // Writes one row: accumulators times their weights; an accumulator of weight 0 may hold anything.
    auto flush = [&]() {
      pend = false;
      if (kAlt && s == 1) return true;           // stream 0 writes for both
      if (!wait(bar_o_final, (iter - 1) & 1)) return false;
      const int qb = (iter - 1) % QB;
      // (the addresses are computed here, once per item: hoisted out of the loop over the items they would live, or be
      // spilled, across the softmax pass)
      int rr = r;
      asm volatile("" : "+r"(rr));
      const uint32_t stage = sQ + (uint32_t)((qb * C::NQ + s) * C::kTileBytes + rr * 128);
      float m = pend_m, l = pend_l, f0 = m == -INFINITY ? 0.f : 1.f, f1 = 0.f;
      if constexpr (kAlt) {
        if (!wait(bar_x, (iter - 1) & 1)) return false;
        const float2 x1 = ml_x[r];
        const float mm = fmaxf(m, x1.x);
        f0 = m == -INFINITY ? 0.f : ex2(m - mm);
        f1 = x1.x == -INFINITY ? 0.f : ex2(x1.x - mm);
        l = f0 * l + f1 * x1.y;
        m = mm;
      }
      tc_fence_after();
      if (pend_warp) {
        if (p.direct) {
          const float inv = seg_inverse(l);
          f0 *= inv;
          f1 *= inv;
          if (pend_real && a.lse) a.lse[pend_lse] = seg_lse(m, l);
        }
        const int64_t pr = (int64_t)pend_part * p.rows + pend_row;
        if (!p.direct && pend_real) p.part_ml[pr] = make_float2(m, l);
        const bool any_empty = __any_sync(0xffffffffu, f0 == 0.f);
#pragma unroll 1          // (unrolled: 257 instead of 251 us for the ragged multi-view batch, in instruction fetches)
        for (int c = 0; c < D / 32; ++c) {
          float ov[32];
          __syncwarp();
          tmem_ld32(tO + c * 32, ov);
          tmem_ld_wait();
          if (any_empty) {
#pragma unroll
            for (int j = 0; j < 32; ++j) ov[j] = f0 != 0.f ? ov[j] : 0.f;
          }
#pragma unroll
          for (int j = 0; j < 32; ++j) ov[j] *= f0;
          if constexpr (kAlt) {
            float o1[32];
            tmem_ld32(tm_O(1) + lane_off + c * 32, o1);
            tmem_ld_wait();
#pragma unroll
            for (int j = 0; j < 32; ++j) ov[j] = f1 != 0.f ? fmaf(o1[j], f1, ov[j]) : ov[j];
          }
          if (p.direct) {
#pragma unroll
            for (int q = 0; q < 4; ++q) {
              const int c16 = c * 4 + q;
              st_shared_16(stage + (uint32_t)((c16 >> 3) * C::kSub + (((c16 & 7) ^ (rr & 7)) << 4)), pack_bf16x2(ov[q * 8 + 0], ov[q * 8 + 1]),
                           pack_bf16x2(ov[q * 8 + 2], ov[q * 8 + 3]), pack_bf16x2(ov[q * 8 + 4], ov[q * 8 + 5]),
                           pack_bf16x2(ov[q * 8 + 6], ov[q * 8 + 7]));
            }
          } else if (pend_real) {
            uint32_t w[32];
#pragma unroll
            for (int j = 0; j < 32; ++j) w[j] = __float_as_uint(ov[j]);
#pragma unroll
            for (int q = 0; q < 4; ++q) st_global_32((unsigned char*)(p.part_o + pr * D) + c * 128 + q * 32, w + q * 8);
          }
        }
      }
      tc_fence_before();
      arrive(bar_o_free);                   // the accumulators have been read
      if (p.direct) {
        // the staged tile leaves as a box, or row by row with 16-byte stores, a row or two per instruction
        if (x.box_out) {
          fence_proxy_async();
          arrive(bar_staged(qb, s));        // warp 10 sends it
        } else {
          __syncwarp();
          constexpr int CPR = D / 8, RPI = 32 / CPR;
          int ln = lane;
          asm volatile("" : "+r"(ln));
          const int cc = ln % CPR, sub = ln / CPR;
          const int row = pend_real ? pend_row : -1;
          const unsigned char* src = base_ptr + (qb * C::NQ + s) * C::kTileBytes + (cc >> 3) * C::kSub + (warp & 3) * 32 * 128;
#pragma unroll 4
          for (int i = 0; i < 32 / RPI; ++i) {
            const int rl = i * RPI + sub;
            const int o = __shfl_sync(0xffffffffu, row, rl);
            const int bt = o / a.N_h, h = o - bt * a.N_h, b = bt / a.n_q, t = bt - b * a.n_q;
            if (o >= 0)
              *reinterpret_cast<uint4*>((__nv_bfloat16*)a.out + b * a.o_smp + t * a.o_tok + (int64_t)h * D + cc * 8) =
                  *reinterpret_cast<const uint4*>(src + rl * 128 + (((cc & 7) ^ (rl & 7)) << 4));
          }
          __syncwarp();
          fence_proxy_async();                   // the next loads of this buffer come through the other proxy
          arrive(bar_q_free(qb));
        }
      }
      return true;
    };
    while (ok && next_desc(di, d)) {
      const int n = d.n, na = d.na, part = d.part;
      const int row0 = (d.row0 & 0x3fffffff) + (kAlt ? 0 : s * kTile);       // of the stream's tile
      const SegRow row = seg_row(p, p.pass[d.row0 >> 30].block_samples, d.b0, d.h_kv, row0 + r);
      const int grow = (row.b * a.n_q + row.t) * a.N_h + row.h;
      const bool row_real = row.real, warp_real = __any_sync(0xffffffffu, row_real);
      // real keys ahead of each segment's first tile in this item, and those of segment 1 that this row sees
      const int real0 = d.len0 - d.base0, real1 = d.len1 - d.base1, sees1 = seg_limit1(a, d.own, row.t) - d.base1;
      float m_used = -INFINITY, l_run = 0.f;
      bool any_key = false;
      const int i0 = kAlt ? (s ^ pos0) & 1 : 0;                  // the stream's first tile of the item
      for (int i = i0; i < n; i += kAlt ? 2 : 1, ++cnt) {
        const int g = u0 + (kAlt ? i : 2 * i + s), buf = g % NB;      // unit
        const uint32_t tS = tm_S(buf) + lane_off;
        const bool s1 = i >= na;
        const int real = (s1 ? real1 : real0) - i * kTile;      // real keys of this tile
        const int valid = s1 ? sees1 - i * kTile : real;        // those that the row sees
        // kW scores at a time: chunks that every row of the warp sees, those that one of them sees something of, and those
        // that the product reads
        const int chunks_all = __reduce_min_sync(0xffffffffu, max(valid, 0) / kW);
        const int chunks = __reduce_max_sync(0xffffffffu, min(kTile / kW, (max(valid, 0) + kW - 1) / kW));
        const int chunks_pv = (steps16(real) * 16 + kW - 1) / kW;
        ok = wait(bar_s_full(buf), (g / NB) & 1);
        if (!ok) break;
        tc_fence_after();
        // rows behind the last one: nothing is computed, the barriers are kept in step (what their P rows hold only reaches
        // their own accumulator rows, which nobody reads)
        if (warp_real) {
          const bool first = i == i0;
          // weights of scores v[0 .. 2 n) as bf16 pairs, and their sum.  (A whole tile with a NaN is done again, in chunks.)
          auto weights = [&](auto n, const float* v, uint32_t* pk) {
            const uint64_t scale2 = pack2(p.scale_log2, p.scale_log2), negm2 = pack2(-m_used, -m_used);
            constexpr bool kWhole = decltype(n)::value == kTile / 2;
            uint64_t acc2[4] = {0ull, 0ull, 0ull, 0ull};
#pragma unroll
            for (int j = 0; j < decltype(n)::value; ++j) {
              const uint64_t v2 = pack2(v[2 * j], v[2 * j + 1]);
              // (a product as such and the sum would be made one fused operation again)
              const uint64_t x2 = kWhole ? fma2(v2, scale2, negm2) : add2(fma2(v2, scale2, 0ull), negm2);
              float p0, p1;
              if ((j & (D == 64 ? 15 : 7)) == 0) {
                // one pair in eight on the FMA pipes, which the exp2 unit leaves idle (in sixteen at head dim 64, where the
                // instructions cost more: ragged multi-view batch 245 us, 252 with eight, 240 with none; 608-row samples 72, 72, 74)
                exp2_poly2<true, !kWhole>(x2, p0, p1);
              } else {
                float t0, t1;
                unpack2(x2, t0, t1);
                p0 = ex2(t0);
                p1 = ex2(t1);
              }
              acc2[j & 3] = add2(acc2[j & 3], pack2(p0, p1));
              pk[j] = pack_bf16x2(p0, p1);
            }
            float a0, a1;
            unpack2(add2(add2(acc2[0], acc2[1]), add2(acc2[2], acc2[3])), a0, a1);
            return a0 + a1;
          };
          // The first scores fix the row's reference: any of them will do, since a row that outgrows it raises it.  A row that
          // sees none of its keys sees no later key either (limits are a prefix of segment 1, and segment 0 has no limits below
          // its length).
          auto reference = [&](const float* v) {
            any_key = valid > 0;
            float m4[4];
#pragma unroll
            for (int j = 0; j < 4; ++j) m4[j] = v[j];
#pragma unroll
            for (int b = 4; b < 32; b += 4) {
#pragma unroll
              for (int j = 0; j < 4; ++j) m4[j] = fmaxf(m4[j], v[b + j]);
            }
            // (a finite one: scores of -inf then weigh 0, and the first finite score raises it)
            m_used = any_key ? fmaxf(fmaxf(fmaxf(m4[0], m4[1]), fmaxf(m4[2], m4[3])) * p.scale_log2, -FLT_MAX) : 0.f;
          };
          bool whole = chunks_all >= kTile / kW;
          if (whole) {
            float sv[kTile];
            uint32_t pk[kTile / 2];
#pragma unroll
            for (int c = 0; c < 4; ++c) tmem_ld32(tS + c * 32, *reinterpret_cast<float(*)[32]>(&sv[c * 32]));
            tmem_ld_wait();
            if (first) reference(sv);
            const float sum = weights(std::integral_constant<int, kTile / 2>(), sv, pk);
            // no weight far above 1 and no large reference (kSegBig); else, inf and NaN too, below
            whole = !__any_sync(0xffffffffu, !(sum <= 256.f * kTile && fabsf(m_used) < kSegBig));
            if (whole) {
              // P overwrites the scores only now that the pass is known to stand
#pragma unroll
              for (int c = 0; c < 4; ++c) tmem_st16(tS + c * 16, &pk[c * 16]);
              l_run += sum;
            }
          }
          // Tiles of which some row of the warp does not see every key, and (rare) scores that outgrow the reference: kW scores
          // at a time, in a loop.  Unrolled too, this path costs more in instruction fetches than it saves (13 us of 265 where
          // half of the samples end inside a tile).
#pragma unroll 1
          for (int c = 0; !whole && c < chunks_pv; ++c) {
            uint32_t pk[kW / 2];
            if (c < chunks) {
              const int left = valid - c * kW;
              float sum;
#pragma unroll 1
              for (bool raised = false;; raised = true) {
                float v[kW];
#pragma unroll
                for (int j = 0; j < kW / 32; ++j) tmem_ld32(tS + c * kW + j * 32, *reinterpret_cast<float(*)[32]>(&v[j * 32]));
                tmem_ld_wait();
                if (c >= chunks_all) {
#pragma unroll
                  for (int j = 0; j < kW; ++j)
                    if (j >= left) v[j] = -INFINITY;
                }
                if (first && c == 0 && !raised && chunks_all < kTile / kW) reference(v);
                sum = weights(std::integral_constant<int, kW / 2>(), v, pk);
                const bool grew = !(sum <= 256.f * kW);          // weights far above 1; also inf and NaN
                if (raised || !__any_sync(0xffffffffu, grew)) break;
                // Rare: raise the reference to the row's maximum, in whole powers of two, so that the weights of this tile that
                // are written already rescale without another rounding; then repeat the chunk.  (A step of 2^8 or more leaves
                // nothing of them, and large numbers are whole: then the reference becomes the maximum itself, since a
                // sum of the two would be off by half a step of the larger one.)
                float mraw = -INFINITY;
#pragma unroll 1
                for (int b = 0; b < kW / 32; ++b) {
                  float w[32];
                  tmem_ld32(tS + c * kW + b * 32, w);
                  tmem_ld_wait();
#pragma unroll
                  for (int j = 0; j < 32; ++j)
                    if (b * 32 + j < left) mraw = fmaxf(mraw, w[j]);
                }
                const float delta = ceilf(fmaxf(fmaf(mraw, p.scale_log2, -m_used), 0.f));
                const bool near = delta < 256.f && fabsf(m_used) < kSegBig;
                const float next = !grew ? m_used : (near ? m_used + delta : fmaxf(m_used, mraw * p.scale_log2));
                const float f = !grew ? 1.f : ex2(near ? -delta : m_used - next);
                m_used = next;
                l_run *= f;
                tmem_st_wait();
#pragma unroll 1
                for (int b = 0; b < c * (kW / 32); ++b) {
                  uint32_t w[16];
                  tmem_ld16(tS + b * 16, w);
                  tmem_ld_wait();
#pragma unroll
                  for (int j = 0; j < 16; ++j) w[j] = pack_bf16x2(__uint_as_float(w[j] << 16) * f, __uint_as_float(w[j] & 0xffff0000u) * f);
                  tmem_st16(tS + b * 16, w);
                }
                if (!first) {
                  // the accumulator must hold every product issued against the old reference
                  ok = wait(bar_pv(s), (cnt - 1) & 1);
                  if (!ok) break;
                  tc_fence_after();
#pragma unroll 1
                  for (int b = 0; b < D / 32; ++b) {
                    float ov[32];
                    tmem_ld32(tO + b * 32, ov);
                    tmem_ld_wait();
                    uint32_t ou[32];
#pragma unroll
                    for (int j = 0; j < 32; ++j) ou[j] = __float_as_uint(ov[j] * f);
                    tmem_st32(tO + b * 32, ou);
                  }
                }
              }
              if (!ok) break;
              l_run += sum;
            } else {
#pragma unroll
              for (int j = 0; j < kW / 2; ++j) pk[j] = 0u;
            }
            // over scores that have been read
#pragma unroll
            for (int j = 0; j < kW / 32; ++j) tmem_st16(tS + c * (kW / 2) + j * 16, &pk[j * 16]);
          }
          if (!ok) break;
          if (first && chunks == 0) m_used = 0.f;            // a warp of rows that see no key
          tmem_st_wait();
        }
        tc_fence_before();
        arrive(bar_p_full(buf));
        if (pend) {
          ok = flush();
          if (!ok) break;
        }
      }
      if (!ok) break;
      if (pend) ok = flush();       // kAlt, stream 1: an item of one tile
      if (!ok) break;
      pend = true;
      pend_real = row_real;
      pend_warp = warp_real;
      pend_m = any_key ? m_used : -INFINITY;
      pend_l = any_key ? l_run : 0.f;
      pend_row = grow;
      pend_part = part;
      pend_lse = (row.b * a.N_h + row.h) * a.n_q + row.t;
      if (kAlt && s == 1) {
        // stream 0 has read the previous item's values
        if (iter > 0) ok = wait(bar_o_free, (iter - 1) & 1);
        if (!ok) break;
        ml_x[r] = make_float2(pend_m, pend_l);
        arrive(bar_x);
        arrive(bar_o_free);
      }
      ++iter;
      pos0 += n;
      u0 += kAlt ? n : 2 * n;
    }
    if (ok && pend) flush();
  }
  allow_next();
  tc_fence_before();
  __syncthreads();
  if (pass0 == 1) wait_previous();
  if (threadIdx.x == 0 && *abort_flag) atomicOr(p.status, ST_TIMEOUT);
  if (warp == 8) {
    tc_fence_after();
    asm volatile("tcgen05.dealloc.cta_group::1.sync.aligned.b32 %0, 512;" ::"r"(tmem) : "memory");
  }
}

// [B, n_q, N_kv * g, D] viewed as (d, head of the group, token, group, sample); box = 64 columns x g heads x tokens x samples
bool make_q_map(CUtensorMap* map, const void* ptr, const SegArgs& a, int g, int64_t tok, int64_t smp, int box_tokens, int box_samples) {
  const cuuint64_t dims[5] = {(cuuint64_t)a.D, (cuuint64_t)g, (cuuint64_t)a.n_q, (cuuint64_t)a.N_kv, (cuuint64_t)a.B};
  const cuuint64_t strides[4] = {(cuuint64_t)a.D * 2, (cuuint64_t)tok * 2, (cuuint64_t)g * a.D * 2, (cuuint64_t)smp * 2};
  const cuuint32_t box[5] = {64, (cuuint32_t)g, (cuuint32_t)box_tokens, 1, (cuuint32_t)box_samples};
  return encode_bf16(map, ptr, 5, dims, strides, box);
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
    if (!make_kv_map(&mk[s], a.k[s], blocks, a.n[s], a.N_kv, D, a.k_tok[s], a.k_smp[s], kTile) ||
        !make_kv_map(&mv[s], a.v[s], blocks, a.n[s], a.N_kv, D, a.v_tok[s], a.v_smp[s], kTile))
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
  static SmemOptIn opt_in;
  cudaError_t e = opt_in((const void*)seg_tc_kernel<D, kAlt>, smem, a.device);
  if (e != cudaSuccess) return e;
  const int grid = x.items < a.sms ? x.items : a.sms;
  ++*launches;
  if (pass == 1) return launch_after(seg_tc_kernel<D, kAlt>, dim3(grid), dim3(kThreadsS), smem, st, mq, mo, mk[0], mv[0], mk[1], mv[1], p, pass, x);
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
