// Head norms and rotary positions of q and k in one pass, and the same on the way into a paged cache (with v as it is).
//
// A row is one head of one token: y = x / sqrt(mean(x^2) + eps) * w in fp32, then the pairs (a, b) of its first rot elements become
// magnitude * (a cos - b sin, b cos + a sin), rounded once to the storage type.
// Angles.  A position times a frequency in fp32 would be off by half a step of the product, 0.004 radians at position 131072.  The
// frequencies arrive as turns per position in units of 2^-64 turns (the last three bits name the component of the position), so that
// position * turn modulo 2^64 IS the reduced angle: one 64-bit product, off by 2^-30 turns at most (five units of the turns
// times 2^31, and the product's last 32 bits), whatever the position and the frequency.  The nearest quarter turn is
// taken off as an integer; sine and cosine of the rest (at most an eighth of a turn) are their Taylor series up to x^9 and x^10,
// whose next terms are below 2e-9 (of sin) and 2e-10.
// Work: a CTA of eight warps owns a few tokens.  It finds out where they are and works out their cosines and sines once, in shared
// memory.  The rows of a token (of q, then k, then v) are cut into items, as many rows as a warp holds at two times 16 bytes a lane; a warp
// owns a token's items, or a share of them where tokens are few.  Items arrive by asynchronous copies, kRing ahead, the first of them
// requested before the tokens are looked up; a lane copies what it will read itself, so that no barrier is needed.  A lane holds both
// elements of each of its pairs, and keeps their cosines and sines, times the weights, for all items of a kind, so that an element costs a
// product, a fused one and the product with the reciprocal root.  Where rot/2 ends inside 16 bytes the other half of a pair is read again,
// element by element (L1), which takes 2.4 to 3.1 times as long (9280 tokens of 32 + 32 heads of 128: 160 us with 120 elements rotated, 51 with 128
// or with 120 in neighbouring pairs; 14631 tokens of 3 x 24 heads of 64 into a cache: 123 us with 56, 52 with 64).
// What bounds it: memory, and the issue of some 160 instructions an item (1 KB).  q and k of 9280 tokens, 32 heads of 128 each, 304 MB in
// 56 us (5.4 TB/s); 69376 tokens of 24 and 8 heads of 64, 569 MB in 107 us (5.3 TB/s, 73 % of the issue slots); 14631 tokens of 3 x 24 heads
// of 64 into a cache, 270 MB in 56 us (4.8 TB/s: the places in the cache are looked up first).  A ring of three or six, items in
// registers instead, one token a warp, cosines and sines unfolded: 0 to 30 % slower.  Few tokens: 4 to 5 us, a launch and one item.  Narrow heads
// and few of them spread what a token costs by itself over fewer items: 16449 tokens of 3 x 32 heads of 32 into a cache, 202 MB in 52 us (3.9
// TB/s); 6000 tokens of 32 + 2 x 8 heads of 128, 32 elements rotated, 147 MB in 37.5 us (3.9 TB/s).
// Three CTAs an SM leave 80 registers: bf16 instances spill 12 bytes a thread and load 16 (32 to 36 each where rot/2 ends inside 16
// bytes; none with neighbouring pairs outside the cache), fp32 ones nothing.
#include <string.h>

#include "seg_attn.cuh"

namespace swam {
namespace {

constexpr int kWarps = 8;
constexpr int kTokens = 32;        // of a CTA, at most
constexpr int kRing = 4;           // items in flight, of a warp

__device__ __forceinline__ uint64_t pair(float lo, float hi) {
  uint64_t r;
  asm("mov.b64 %0, {%1, %2};" : "=l"(r) : "f"(lo), "f"(hi));
  return r;
}
__device__ __forceinline__ float2 parts(uint64_t v) {
  float2 r;
  asm("mov.b64 {%0, %1}, %2;" : "=f"(r.x), "=f"(r.y) : "l"(v));
  return r;
}
__device__ __forceinline__ uint64_t fma2(uint64_t a, uint64_t b, uint64_t c) {
  uint64_t r;
  asm("fma.rn.f32x2 %0, %1, %2, %3;" : "=l"(r) : "l"(a), "l"(b), "l"(c));
  return r;
}
__device__ __forceinline__ uint64_t mul2(uint64_t a, uint64_t b) {
  uint64_t r;
  asm("mul.rn.f32x2 %0, %1, %2;" : "=l"(r) : "l"(a), "l"(b));
  return r;
}

template <typename T>
struct Chunk;                      // 16 bytes as pairs of neighbours
template <>
struct Chunk<float> {
  static constexpr int N = 4;
  static __device__ __forceinline__ void unpack(const uint4& u, uint64_t (&x)[2]) {
    x[0] = pair(__uint_as_float(u.x), __uint_as_float(u.y));
    x[1] = pair(__uint_as_float(u.z), __uint_as_float(u.w));
  }
  static __device__ __forceinline__ uint4 pack(const uint64_t (&x)[2]) {
    const float2 a = parts(x[0]), b = parts(x[1]);
    return make_uint4(__float_as_uint(a.x), __float_as_uint(a.y), __float_as_uint(b.x), __float_as_uint(b.y));
  }
};
template <>
struct Chunk<__nv_bfloat16> {
  static constexpr int N = 8;
  static __device__ __forceinline__ void unpack(const uint4& u, uint64_t (&x)[4]) {
    const uint32_t w[4] = {u.x, u.y, u.z, u.w};
#pragma unroll
    for (int i = 0; i < 4; ++i) x[i] = pair(__uint_as_float(w[i] << 16), __uint_as_float(w[i] & 0xffff0000u));
  }
  static __device__ __forceinline__ uint4 pack(const uint64_t (&x)[4]) {
    uint32_t w[4];
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      const float2 v = parts(x[i]);
      asm("cvt.rn.bf16x2.f32 %0, %1, %2;" : "=r"(w[i]) : "f"(v.y), "f"(v.x));
    }
    return make_uint4(w[0], w[1], w[2], w[3]);
  }
};

// cosine and sine of `phase` / 2^64 turns
__device__ __forceinline__ float2 cos_sin(uint64_t phase) {
  const uint32_t h = (uint32_t)(phase >> 32);
  const uint32_t quarter = (h + 0x20000000u) >> 30;
  const float x = (float)(int32_t)(h - (quarter << 30)) * 1.46291807926715968e-9f;       // 2 pi / 2^32
  const float z = x * x;
  float s = fmaf(z, 2.75573192e-6f, -1.98412698e-4f);
  s = fmaf(z, s, 8.33333333e-3f);
  s = fmaf(z, s, -1.66666667e-1f);
  s = fmaf(x * z, s, x);
  float c = fmaf(z, -2.75573192e-7f, 2.48015873e-5f);
  c = fmaf(z, c, -1.38888889e-3f);
  c = fmaf(z, c, 4.16666667e-2f);
  c = fmaf(z, c, -0.5f);
  c = fmaf(z, c, 1.f);
  const float a = quarter & 1 ? s : c, b = quarter & 1 ? c : s;
  return make_float2((quarter == 1) | (quarter == 2) ? -a : a, quarter >= 2 ? -b : b);
}

// A token: where its rows are (in elements; dst < 0: they are not written) and its position.
struct Token {
  int64_t src[3], dst[3], positions;
  int number;                      // default position
};

__device__ __forceinline__ void copy_16(uint32_t dst, const void* src) {
  asm volatile("cp.async.cg.shared.global [%0], [%1], 16;" ::"r"(dst), "l"(src) : "memory");
}
__device__ __forceinline__ uint4 shared_16(uint32_t src) {
  uint4 v;
  asm volatile("ld.shared.v4.b32 {%0, %1, %2, %3}, [%4];" : "=r"(v.x), "=r"(v.y), "=r"(v.z), "=r"(v.w) : "r"(src) : "memory");
  return v;
}

// kPair: 0 = (i, i + rot/2), 1 = (2i, 2i + 1), 2 = (i, i + rot/2) with a half that ends inside 16 bytes
template <typename T, int D, int kPair, bool kCache>
__global__ void __launch_bounds__(32 * kWarps, 3) norm_rope_kernel(const __grid_constant__ RopeParams p) {
  constexpr int N = Chunk<T>::N, N2 = N / 2;     // elements of 16 bytes, and pairs of neighbours
  constexpr int LPR = D / (2 * N);               // lanes of a row
  constexpr int RPW = 32 / LPR;                  // rows of an item
  extern __shared__ __align__(16) uint4 ring[];                  // [warp][kRing][2][lane], then the angles
  float* cosv = reinterpret_cast<float*>(ring + kWarps * kRing * 64);        // [token][half]
  float* sinv = cosv + p.per * (D / 2);
  __shared__ Token token[kTokens];
  __shared__ uint64_t turns[D / 2];
  __shared__ int owner[kTokens];                 // kCache: sample, -1: nobody's
  const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
  const int t0 = (int)blockIdx.x * p.per, count = min(p.per, (int)p.tokens - t0);
  const int l = lane % LPR, sub = lane / LPR, half = p.rot >> 1;
  // First elements of the lane's two times 16 bytes: kPair = 0: the halves of its pairs; otherwise, and where nothing turns, any two, so
  // that the lanes of a row follow one another (neighbouring chunks in one lane fetch and write every 32-byte sector twice: 145
  // instead of 107 us for the multi-view batch).
  const int turning = kPair == 0 ? half / N : 0;
  const int e0 = (kPair == 0 && l >= turning ? turning + l : l) * N;
  const int e1 = e0 + (kPair == 0 ? (l < turning ? half : (LPR - turning) * N) : D / 2);
  if (threadIdx.x < half) turns[threadIdx.x] = p.turn[threadIdx.x];
  // ---- where the tokens come from, one thread each (packed tokens are one sequence)
  const int t = t0 + (int)threadIdx.x;
  int b = 0, i = t;
  if (threadIdx.x < count) {
    if (!kCache) {
      b = t / p.n;
      i = t - b * p.n;
    }
    for (int j = 0; j < 3; ++j) token[threadIdx.x].src[j] = b * p.s_smp[j] + (int64_t)i * p.s_tok[j];
    if (kCache) owner[threadIdx.x] = p.cache.q_start ? -1 : t / p.cache.max_q;
  }
  __syncthreads();

  // ---- loads: the warp's items, one unit (a token, or share `u % split` of it) after the other
  const uint32_t slots = (uint32_t)__cvta_generic_to_shared(ring) + (uint32_t)(warp * kRing * 64 + lane) * 16;
  const int units = count * p.split;
  auto begin_of = [&](int u) { return p.split == 1 ? 0 : (u % p.split) * p.share; };
  auto end_of = [&](int u) { return p.split == 1 ? p.items : min((u % p.split + 1) * p.share, p.items); };
  int lu = warp, ln = begin_of(warp), lend = ln, lrows = 0, issued = 0;       // lend: items up to the end of the kind; lrows: rows left of it
  const T* lrow = nullptr;
  auto request = [&]() {
    if (ln == lend) {                    // another kind, or another unit
      while (lu < units && ln >= end_of(lu)) {
        lu += kWarps;
        ln = begin_of(lu);
      }
      lend = ln;
      lrows = 0;
      if (lu < units) {
        const int kind = ln < p.items_k ? 0 : (ln < p.items_v ? 1 : 2);
        lend = min(end_of(lu), kind == 0 ? p.items_k : (kind == 1 ? p.items_v : p.items));
        const int h = (ln - (kind == 0 ? 0 : (kind == 1 ? p.items_k : p.items_v))) * RPW + sub;
        lrows = (kind == 0 ? p.N_h : p.N_kv) - h;
        lrow = (const T*)p.src[kind] + token[p.split == 1 ? lu : lu / p.split].src[kind] + h * D;
      }
    }
    if (lrows > 0) {
      const uint32_t slot = slots + (issued % kRing) * 1024;
      copy_16(slot, lrow + e0);
      copy_16(slot + 512, lrow + e1);
    }
    lrow += RPW * D;
    lrows -= RPW;
    if (ln < lend) ++ln;
    ++issued;
    asm volatile("cp.async.commit_group;" ::: "memory");
  };
#pragma unroll 1
  for (int i = 0; i < kRing; ++i) request();

  // ---- where they go, and their positions
  if (kCache && p.cache.q_start) {
    // every sample claims its tokens
    for (int smp = threadIdx.x; smp < p.cache.samples; smp += 32 * kWarps) {
      const int q0 = __ldg(p.cache.q_start + smp), q1 = __ldg(p.cache.q_start + smp + 1);
      if (q0 < 0 || q0 > q1 || q1 > p.tokens) atomicOr(p.status, ST_BAD_LEN);
      else
        for (int x = max(q0, t0); x < min(q1, t0 + count); ++x) owner[x - t0] = smp;
    }
    __syncthreads();
  }
  if (threadIdx.x < count) {
    Token& k = token[threadIdx.x];
    int number = i;
    int64_t k_at = -1, v_at = -1;
    bool mine = true;                      // somebody's token
    if constexpr (kCache) {
      const PagedCache& c = p.cache;
      int bad = 0;
      const int smp = owner[threadIdx.x];
      mine = smp >= 0;
      const int q1 = !mine ? 0 : (c.q_start ? __ldg(c.q_start + smp + 1) : (smp + 1) * c.max_q);
      number = mine ? __ldg(c.kv_len + smp) - (q1 - t) : 0;
      if (mine && number >= 0 && number < c.max_kv) {
        const int page = __ldg(c.table + smp * c.table_stride + (number >> c.page_shift));
        const int row = number & ((1 << c.page_shift) - 1);
        if (page >= 0 && page < c.n_pages) {
          k_at = page * c.k_page + row * c.k_tok;
          v_at = page * c.v_page + row * c.v_tok;
        } else {
          bad = ST_BAD_MAP;
        }
      } else if (mine) {
        bad = ST_BAD_LEN;
      }
      if (bad) atomicOr(p.status, bad);
    }
    k.dst[0] = mine ? b * p.d_smp[0] + (int64_t)i * p.d_tok[0] : -1;
    k.dst[1] = kCache ? k_at : b * p.d_smp[1] + (int64_t)i * p.d_tok[1];
    k.dst[2] = v_at;
    k.positions = b * p.pos_smp + (int64_t)i * p.axes;
    k.number = number;
  }
  __syncthreads();
  // ---- their angles
  for (int x = threadIdx.x; x < count * half; x += 32 * kWarps) {
    const int k = x / half, j = x - k * half;
    const uint64_t turn = turns[j];
    const int pos = p.positions ? __ldg(p.positions + token[k].positions + (int)(turn & 7)) : token[k].number;
    const float2 v = cos_sin((turn & ~7ull) * (uint64_t)(int64_t)pos);
    cosv[k * (D / 2) + j] = v.x * p.magnitude;
    sinv[k * (D / 2) + j] = v.y * p.magnitude;
  }
  __syncthreads();

  int taken = 0;
  for (int u = warp; u < units; u += kWarps) {
    const int k = p.split == 1 ? u : u / p.split, end = end_of(u);
    for (int n = begin_of(u); n < end;) {
      const int kind = n < p.items_k ? 0 : (n < p.items_v ? 1 : 2);
      const int first = kind == 0 ? 0 : (kind == 1 ? p.items_k : p.items_v), last = min(end, kind == 0 ? p.items_k : (kind == 1 ? p.items_v : p.items));
      const int heads = kind == 0 ? p.N_h : p.N_kv;
      const float* weight = kind < 2 ? p.weight[kind] : nullptr;
      const int64_t to = token[k].dst[kind];
      int rows = heads - (n - first) * RPW - sub;          // of the lane's place, left
      T* dst = (T*)p.dst[kind] + to + (heads - rows) * D;
      if (to < 0) rows = 0;
      // what the lane's elements (x, y: its first and second 16 bytes) are multiplied with:
      //   kPair 0: x' = x xx + y xy, y' = y yy + x yx;   kPair 1: x' = x xx + swapped(x) xy, y' = y yy + swapped(y) yx
      uint64_t xx[N2], xy[N2], yx[N2], yy[N2];
      if (kind < 2) {
        const float* cv = cosv + k * (D / 2);
        const float* sv = sinv + k * (D / 2);
#pragma unroll
        for (int j = 0; j < N2; j += 2) {
          float4 wa = make_float4(1.f, 1.f, 1.f, 1.f), wb = wa;
          if (weight) {
            wa = __ldg(reinterpret_cast<const float4*>(weight + e0 + 2 * j));
            wb = __ldg(reinterpret_cast<const float4*>(weight + e1 + 2 * j));
          }
          xx[j] = pair(wa.x, wa.y);
          xx[j + 1] = pair(wa.z, wa.w);
          yy[j] = pair(wb.x, wb.y);
          yy[j + 1] = pair(wb.z, wb.w);
          xy[j] = xy[j + 1] = yx[j] = yx[j + 1] = 0ull;
          if constexpr (kPair == 0) {
            if (l < turning) {
              const float4 c = *reinterpret_cast<const float4*>(cv + e0 + 2 * j), sn = *reinterpret_cast<const float4*>(sv + e0 + 2 * j);
              xx[j] = pair(c.x * wa.x, c.y * wa.y);
              xx[j + 1] = pair(c.z * wa.z, c.w * wa.w);
              xy[j] = pair(-sn.x * wb.x, -sn.y * wb.y);
              xy[j + 1] = pair(-sn.z * wb.z, -sn.w * wb.w);
              yx[j] = pair(sn.x * wa.x, sn.y * wa.y);
              yx[j + 1] = pair(sn.z * wa.z, sn.w * wa.w);
              yy[j] = pair(c.x * wb.x, c.y * wb.y);
              yy[j + 1] = pair(c.z * wb.z, c.w * wb.w);
            }
          } else if constexpr (kPair == 1) {
            // two pairs of each 16 bytes; those behind rot / 2 do not turn
#pragma unroll
            for (int d = 0; d < 2; ++d) {
              const int pa = e0 / 2 + j + d, pb = e1 / 2 + j + d;
              const float2 va = d == 0 ? make_float2(wa.x, wa.y) : make_float2(wa.z, wa.w), vb = d == 0 ? make_float2(wb.x, wb.y) : make_float2(wb.z, wb.w);
              if (pa < half) {
                xx[j + d] = pair(cv[pa] * va.x, cv[pa] * va.y);
                xy[j + d] = pair(-sv[pa] * va.y, sv[pa] * va.x);
              }
              if (pb < half) {
                yy[j + d] = pair(cv[pb] * vb.x, cv[pb] * vb.y);
                yx[j + d] = pair(-sv[pb] * vb.y, sv[pb] * vb.x);
              }
            }
          }
        }
      }
      for (; n < last; ++n) {
        const uint32_t slot = slots + (taken % kRing) * 1024;
        asm volatile("cp.async.wait_group %0;" ::"n"(kRing - 1) : "memory");
        uint4 v0 = shared_16(slot), v1 = shared_16(slot + 512);
        if (kind < 2) {
          uint64_t x[N2], y[N2];
          Chunk<T>::unpack(v0, x);
          Chunk<T>::unpack(v1, y);
          float inv = 1.f;
          if (weight) {
            uint64_t sum2 = 0ull;
#pragma unroll
            for (int j = 0; j < N2; ++j) sum2 = fma2(x[j], x[j], fma2(y[j], y[j], sum2));
            float sum = parts(sum2).x + parts(sum2).y;
#pragma unroll
            for (int o = 1; o < LPR; o <<= 1) sum += __shfl_xor_sync(0xffffffffu, sum, o);
            inv = rsqrtf(fmaf(sum, 1.f / D, p.eps));
          }
          if constexpr (kPair == 0) {
            if (l < turning) {
#pragma unroll
              for (int j = 0; j < N2; ++j) {
                const uint64_t a = x[j];
                x[j] = fma2(a, xx[j], mul2(y[j], xy[j]));
                y[j] = fma2(y[j], yy[j], mul2(a, yx[j]));
              }
            } else {
#pragma unroll
              for (int j = 0; j < N2; ++j) {
                x[j] = mul2(x[j], xx[j]);
                y[j] = mul2(y[j], yy[j]);
              }
            }
          } else if constexpr (kPair == 1) {
            // (an element that does not turn keeps nothing of its neighbour, an infinite one included)
#pragma unroll
            for (int j = 0; j < N2; ++j) {
              const float2 a = parts(x[j]), c = parts(y[j]);
              const uint64_t xt = mul2(pair(a.y, a.x), xy[j]), yt = mul2(pair(c.y, c.x), yx[j]);
              x[j] = fma2(x[j], xx[j], p.rot == D || e0 + 2 * j < p.rot ? xt : 0ull);
              y[j] = fma2(y[j], yy[j], p.rot == D || e1 + 2 * j < p.rot ? yt : 0ull);
            }
          } else {
            const T* row = (const T*)p.src[kind] + token[k].src[kind] + ((n - first) * RPW + sub) * D;
            const bool there = (n - first) * RPW + sub < heads;
#pragma unroll
            for (int j = 0; j < N; ++j) {
              uint64_t& v = j < N2 ? x[j % N2] : y[j % N2];
              v = mul2(v, j < N2 ? xx[j % N2] : yy[j % N2]);
              float own[2] = {parts(v).x, parts(v).y};
#pragma unroll
              for (int d = 0; d < 2; ++d) {
                const int e = (j < N2 ? e0 : e1) + 2 * (j % N2) + d, o = e < half ? e + half : e - half, at = k * (D / 2) + (e < half ? e : o);
                if (e < p.rot && there) {
                  float other = (float)row[o];
                  if (weight) other *= __ldg(weight + o);
                  own[d] = fmaf(own[d], cosv[at], e < half ? -other * sinv[at] : other * sinv[at]);
                }
              }
              v = pair(own[0], own[1]);
            }
            __syncwarp();                          // (in place: every element of the rows has been read)
          }
          if (weight) {
            const uint64_t inv2 = pair(inv, inv);
#pragma unroll
            for (int j = 0; j < N2; ++j) {
              x[j] = mul2(x[j], inv2);
              y[j] = mul2(y[j], inv2);
            }
          }
          v0 = Chunk<T>::pack(x);
          v1 = Chunk<T>::pack(y);
        }
        if (rows > 0) {
          *reinterpret_cast<uint4*>(dst + e0) = v0;
          *reinterpret_cast<uint4*>(dst + e1) = v1;
        }
        dst += RPW * D;
        rows -= RPW;
        ++taken;
        request();                                 // (into the slot whose values have just been used)
      }
    }
  }
  asm volatile("cp.async.wait_all;" ::: "memory");
}

template <typename T, int D, int kPair>
cudaError_t launch_kind(RopeParams& p, cudaStream_t st, int* launches) {
  constexpr int rows = 32 / (D / (2 * Chunk<T>::N));           // of an item
  auto items = [&](int heads, int kind) { return p.src[kind] ? (heads + rows - 1) / rows : 0; };
  p.items_k = items(p.N_h, 0);
  p.items_v = p.items_k + items(p.N_kv, 1);
  p.items = p.items_v + items(p.N_kv, 2);
  // some sixteen items a warp (eight where the places in the cache have to be looked up first: 55 instead of 57 us for 16 chunks of
  // observations), but at least two CTAs for every SM; of few tokens, several warps share one
  const int64_t most = p.tokens / (2 * p.sms);
  int64_t per = ((p.paged ? 8 : 16) * kWarps + p.items - 1) / p.items;
  if (per > most) per = most;
  p.per = per < 1 ? 1 : (per > kTokens ? kTokens : (int)per);
  p.split = p.per >= kWarps ? 1 : kWarps / p.per;
  if (p.split > p.items) p.split = p.items;
  p.share = (p.items + p.split - 1) / p.split;
  if (p.split > 1) p.split = (p.items + p.share - 1) / p.share;
  const unsigned blocks = (unsigned)((p.tokens + p.per - 1) / p.per);
  const int smem = kWarps * kRing * 1024 + p.per * D * (int)sizeof(float);
  static SmemOptIn opt_in[2];
  const void* kernel = p.paged ? (const void*)norm_rope_kernel<T, D, kPair, true> : (const void*)norm_rope_kernel<T, D, kPair, false>;
  const cudaError_t e = opt_in[p.paged](kernel, kWarps * kRing * 1024 + kTokens * D * (int)sizeof(float), p.device);
  if (e != cudaSuccess) return e;
  ++*launches;
  if (p.paged) norm_rope_kernel<T, D, kPair, true><<<blocks, 32 * kWarps, smem, st>>>(p);
  else norm_rope_kernel<T, D, kPair, false><<<blocks, 32 * kWarps, smem, st>>>(p);
  return cudaGetLastError();
}
template <typename T, int D>
cudaError_t launch_pair(RopeParams& p, cudaStream_t st, int* launches) {
  if (p.interleaved) return launch_kind<T, D, 1>(p, st, launches);
  if ((p.rot / 2) % Chunk<T>::N == 0) return launch_kind<T, D, 0>(p, st, launches);
  return launch_kind<T, D, 2>(p, st, launches);
}
template <typename T>
cudaError_t launch_dim(RopeParams& p, cudaStream_t st, int* launches) {
  switch (p.D) {
    case 32: return launch_pair<T, 32>(p, st, launches);
    case 64: return launch_pair<T, 64>(p, st, launches);
    case 128: return launch_pair<T, 128>(p, st, launches);
    default: return cudaErrorInvalidConfiguration;
  }
}

}  // namespace

uint64_t turns_of(double freq) {
  // |freq| / (2 pi) turns in units of 2^-64, modulo a turn.  2 / pi = 0xa2f9836e4e441529fc2757d1f534ddc1 / 2^128, to half a unit: for the
  // largest frequency, 2^20, that is 2^-111 turns.  (With 2 / pi to 64 bits it would be 2^-52, and 2^-21 at the ends of int32.)
  uint64_t bits;
  memcpy(&bits, &freq, 8);
  const int e = (int)(bits >> 52 & 0x7ff);                               // |freq| = mantissa * 2^(e - 1075)
  if (e == 0) return 0;                                                  // (zero, and what is far below 2^-64 of a turn in 2^31 positions)
  const uint64_t mantissa = (bits & 0xfffffffffffffull) | 1ull << 52;
  // mantissa * (2 / pi * 2^128) = |freq| / (2 pi) * 2^(130 + 1075 - e), without its last 64 bits
  const unsigned __int128 low = (unsigned __int128)mantissa * 0xfc2757d1f534ddc1ull;
  const unsigned __int128 prod = (unsigned __int128)mantissa * 0xa2f9836e4e441529ull + (uint64_t)(low >> 64);
  const int shift = 1077 - e;                                            // to units of 2^-64; at least 34, as frequencies end at 2^20
  const uint64_t u = shift >= 128 ? 0 : (uint64_t)(prod >> shift);
  return bits >> 63 ? 0 - u : u;
}

cudaError_t launch_norm_rope(RopeParams& p, cudaStream_t st, int* launches) {
  return p.dtype == 0 ? launch_dim<float>(p, st, launches) : launch_dim<__nv_bfloat16>(p, st, launches);
}

}  // namespace swam
