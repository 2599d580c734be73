// Head norms and rotary positions of q and k in one pass, and the same on the way into a paged cache (with v as it is).
//
// A row is one head of one token: y = x / sqrt(mean(x^2) + eps) * w in fp32, then the pairs (a, b) of its first rot elements become
// magnitude * (a cos - b sin, b cos + a sin), rounded once to the storage type.
// Angles.  A position times a frequency in fp32 would be off by half a step of the product, 0.004 radians at position 131072.  The
// frequencies arrive as turns per position in units of 2^-64 turns, so that position * turn modulo 2^64 IS the reduced
// angle: one 64-bit product, exact but for the frequency's own rounding, whatever the position.  The nearest quarter turn is
// taken off as an integer; sine and cosine of the rest (at most an eighth of a turn) are their Taylor series up to x^9 and x^10,
// whose next terms are below 2e-9 (of sin) and 2e-10.
// Work: a warp owns a token and up to `per` slabs of its rows.  A slab is one kind of row (q, k or v), kBatch times as many as the warp
// holds at 16 bytes a lane, all loaded before the first is used.  The warp works out the token's cosines and sines once, in
// shared memory; a lane keeps those of its 16 bytes in registers for all rows.  The other half of a pair comes by shuffle (pairs i,
// i + rot/2) or is in the same 16 bytes (2i, 2i + 1); a rot/2 that ends inside 16 bytes reads it from memory again (L1).
#include <math.h>

#include "swam_internal.cuh"

namespace swam {
namespace {

constexpr int kWarps = 8;
constexpr int kBatch = 4;

template <typename T>
struct Chunk;                      // 16 bytes
template <>
struct Chunk<float> {
  static constexpr int N = 4;
  static __device__ __forceinline__ void unpack(const uint4& u, float (&x)[4]) {
    x[0] = __uint_as_float(u.x); x[1] = __uint_as_float(u.y); x[2] = __uint_as_float(u.z); x[3] = __uint_as_float(u.w);
  }
  static __device__ __forceinline__ uint4 pack(const float (&x)[4]) {
    return make_uint4(__float_as_uint(x[0]), __float_as_uint(x[1]), __float_as_uint(x[2]), __float_as_uint(x[3]));
  }
};
template <>
struct Chunk<__nv_bfloat16> {
  static constexpr int N = 8;
  static __device__ __forceinline__ void unpack(const uint4& u, float (&x)[8]) {
    const uint32_t w[4] = {u.x, u.y, u.z, u.w};
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      x[2 * i] = __uint_as_float(w[i] << 16);
      x[2 * i + 1] = __uint_as_float(w[i] & 0xffff0000u);
    }
  }
  static __device__ __forceinline__ uint4 pack(const float (&x)[8]) {
    uint32_t w[4];
#pragma unroll
    for (int i = 0; i < 4; ++i) asm("cvt.rn.bf16x2.f32 %0, %1, %2;" : "=r"(w[i]) : "f"(x[2 * i + 1]), "f"(x[2 * i]));
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

// The sample of packed token t, and t's place behind the sample's first one.  Two levels of 32 at a time.
__device__ __forceinline__ int find_sample(const int32_t* start, int n, int t, int lane) {
  int lo = 0, hi = n;              // start[lo] <= t, and start[hi] > t where hi < n
  while (hi - lo > 1) {
    const int step = (hi - lo + 31) / 32;
    const int i = lo + lane * step;
    const bool below = i < hi && (lane == 0 || __ldg(start + i) <= t);
    const uint32_t m = __ballot_sync(0xffffffffu, below);
    const int last = 31 - __clz(m);
    const int next = lo + last * step;
    hi = min(hi, next + step);
    lo = next;
  }
  return lo;
}

// kPair: 0 = (i, i + rot/2) by shuffle, 1 = (2i, 2i + 1), 2 = (i, i + rot/2) from memory
template <typename T, int D, int kPair, bool kCache>
__global__ void __launch_bounds__(32 * kWarps) norm_rope_kernel(const __grid_constant__ RopeParams p) {
  constexpr int N = Chunk<T>::N;           // elements of a lane
  constexpr int LPR = D / N;               // lanes of a row
  constexpr int RPW = 32 / LPR;            // rows of a warp
  __shared__ float2 turn[kWarps][64];
  const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
  const int64_t unit = (int64_t)blockIdx.x * kWarps + warp;
  const int64_t t64 = unit / p.parts;
  if (t64 >= p.tokens) return;
  const int t = (int)t64;
  const int slab0 = (int)(unit - t64 * p.parts) * p.per, slab1 = min(slab0 + p.per, p.slabs);
  const int col = (lane % LPR) * N, sub = lane / LPR;

  // where the token is, and its position
  int b = 0, i = t;
  bool real = true;                        // kCache: has the token a place in the cache
  int64_t k_at = 0, v_at = 0;
  int number = t;
  if constexpr (kCache) {
    const PagedCache& c = p.cache;
    int q0, q1;
    if (c.q_start) {
      b = find_sample(c.q_start, c.samples, t, lane);
      q0 = __ldg(c.q_start + b);
      q1 = __ldg(c.q_start + b + 1);
      if (t < q0 || t >= q1) return;       // in front of the first sample or behind the last one
      if (q0 < 0 || q1 > p.tokens) {
        if (lane == 0) atomicOr(p.status, ST_BAD_LEN);
        return;
      }
    } else {
      b = t / c.max_q;
      q0 = b * c.max_q;
      q1 = q0 + c.max_q;
    }
    number = __ldg(c.kv_len + b) - (q1 - t);
    const int slot = number;
    real = slot >= 0 && slot < c.max_kv;
    int bad = real ? 0 : ST_BAD_LEN;
    if (real) {
      const int page = __ldg(c.table + b * c.table_stride + (slot >> c.page_shift));
      const int row = slot & ((1 << c.page_shift) - 1);
      if (page < 0 || page >= c.n_pages) {
        real = false;
        bad = ST_BAD_MAP;
      }
      k_at = page * c.k_page + row * c.k_tok;
      v_at = page * c.v_page + row * c.v_tok;
    }
    if (bad && lane == 0) atomicOr(p.status, bad);
  } else {
    b = t / p.n;
    i = t - b * p.n;
    number = i;
  }
  float cs[N], sn[N];                      // of this lane's elements
  const int half = p.rot >> 1;
  const bool turned = col < p.rot;         // (some of) the lane's elements are
  if (p.rot > 0) {
    for (int j = lane; j < half; j += 32) {
      const int pos = p.positions ? __ldg(p.positions + (kCache ? 0 : b * p.pos_smp) + (int64_t)i * p.axes + p.axis[j]) : number;
      float2 x = cos_sin(p.turn[j] * (uint64_t)(int64_t)pos);
      turn[warp][j] = make_float2(x.x * p.magnitude, x.y * p.magnitude);
    }
    __syncwarp();
  }
#pragma unroll
  for (int j = 0; j < N; ++j) {
    const int e = col + j;
    const float2 x = e < p.rot ? turn[warp][kPair == 1 ? e >> 1 : (e < half ? e : e - half)] : make_float2(1.f, 0.f);
    cs[j] = x.x;
    // the sign of the other element's share
    sn[j] = (kPair == 1 ? (e & 1) == 0 : e < half) ? -x.y : x.y;
  }
  const int step = kPair == 0 ? half / N : 0;      // lanes to the other half of a pair
  const int other = kPair == 0 && turned ? (lane - lane % LPR) + (col < half ? lane % LPR + step : lane % LPR - step) : lane;

  for (int s = slab0; s < slab1; ++s) {
    const int kind = s < p.slab_k ? 0 : (s < p.slab_v ? 1 : 2);
    const int first = (s - (kind == 0 ? 0 : (kind == 1 ? p.slab_k : p.slab_v))) * (RPW * kBatch) + sub;
    const int heads = kind == 0 ? p.N_h : p.N_kv;
    // (packed tokens are one sequence: their sample does not matter to where they are)
    const T* src = (const T*)p.src[kind] + (kCache ? 0 : b * p.s_smp[kind]) + (int64_t)i * p.s_tok[kind] + col;
    T* dst;
    if (kCache && kind > 0) dst = (T*)p.dst[kind] + (kind == 1 ? k_at : v_at) + col;
    else dst = (T*)p.dst[kind] + (kCache ? 0 : b * p.d_smp[kind]) + (int64_t)i * p.d_tok[kind] + col;
    uint4 u[kBatch];
#pragma unroll
    for (int r = 0; r < kBatch; ++r) {
      const int h = first + r * RPW;
      u[r] = h < heads ? *reinterpret_cast<const uint4*>(src + (int64_t)h * D) : make_uint4(0u, 0u, 0u, 0u);
    }
    if (kind == 2) {
#pragma unroll
      for (int r = 0; r < kBatch; ++r) {
        const int h = first + r * RPW;
        if (real && h < heads) *reinterpret_cast<uint4*>(dst + (int64_t)h * D) = u[r];
      }
      continue;
    }
    float w[N];
    const float* weight = p.weight[kind];
    if (weight) {
#pragma unroll
      for (int j = 0; j < N; j += 4) *reinterpret_cast<float4*>(w + j) = __ldg(reinterpret_cast<const float4*>(weight + col + j));
    }
#pragma unroll
    for (int r = 0; r < kBatch; ++r) {
      const int h = first + r * RPW;
      float x[N], y[N];
      Chunk<T>::unpack(u[r], x);
      float inv = 1.f;
      if (weight) {
        float sum = 0.f;
#pragma unroll
        for (int j = 0; j < N; ++j) sum = fmaf(x[j], x[j], sum);
#pragma unroll
        for (int o = 1; o < LPR; o <<= 1) sum += __shfl_xor_sync(0xffffffffu, sum, o);
        inv = rsqrtf(fmaf(sum, 1.f / D, p.eps));
#pragma unroll
        for (int j = 0; j < N; ++j) x[j] *= inv * w[j];
      }
      if constexpr (kPair == 1) {
#pragma unroll
        for (int j = 0; j < N; ++j) y[j] = x[j ^ 1];
      } else if constexpr (kPair == 0) {
#pragma unroll
        for (int j = 0; j < N; ++j) y[j] = __shfl_sync(0xffffffffu, x[j], other);
      } else {
#pragma unroll
        for (int j = 0; j < N; ++j) {
          const int e = col + j, o = e < half ? e + half : e - half;
          y[j] = 0.f;
          if (e < p.rot && h < heads) {
            y[j] = (float)src[(int64_t)h * D + o - col];
            if (weight) y[j] *= inv * __ldg(weight + o);
          }
        }
        __syncwarp();                      // (in place: every element of the row has been read)
      }
#pragma unroll
      for (int j = 0; j < N; ++j)
        if (col + j < p.rot) x[j] = fmaf(x[j], cs[j], y[j] * sn[j]);
      if (real | (kind == 0) && h < heads) *reinterpret_cast<uint4*>(dst + (int64_t)h * D) = Chunk<T>::pack(x);
    }
  }
}

template <typename T, int D, int kPair>
cudaError_t launch_kind(RopeParams& p, cudaStream_t st, int* launches) {
  constexpr int rows = 32 / (D / Chunk<T>::N) * kBatch;        // of a slab
  auto slabs = [&](int heads, int kind) { return p.src[kind] ? (heads + rows - 1) / rows : 0; };
  p.slab_k = slabs(p.N_h, 0);
  p.slab_v = p.slab_k + slabs(p.N_kv, 1);
  p.slabs = p.slab_v + slabs(p.N_kv, 2);
  // a warp for each slab where that does not fill the SMs, else for each token
  p.per = (int64_t)p.tokens * p.slabs <= (int64_t)p.sms * 64 ? 1 : p.slabs;
  p.parts = (p.slabs + p.per - 1) / p.per;
  const int64_t blocks = ((int64_t)p.tokens * p.parts + kWarps - 1) / kWarps;
  if (blocks > 0x7fffffff) return cudaErrorInvalidConfiguration;
  ++*launches;
  if (p.paged) norm_rope_kernel<T, D, kPair, true><<<(unsigned)blocks, 32 * kWarps, 0, st>>>(p);
  else norm_rope_kernel<T, D, kPair, false><<<(unsigned)blocks, 32 * kWarps, 0, st>>>(p);
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
  // freq / (2 pi) turns in units of 2^-64, modulo a turn.  2 / pi = 0xa2f9836e4e44152a / 2^64, to half a unit.
  if (freq == 0.0) return 0;
  int e;
  const double m = frexp(freq < 0 ? -freq : freq, &e);                   // m in [0.5, 1)
  const unsigned __int128 prod = (unsigned __int128)(uint64_t)ldexp(m, 53) * 0xa2f9836e4e44152aull;      // |freq| / (2 pi) * 2^(66 + 53 - e)
  const int shift = 55 - e;                                              // to units of 2^-64
  const uint64_t u = shift >= 128 ? 0 : (shift >= 0 ? (uint64_t)(prod >> shift) : (shift > -64 ? (uint64_t)prod << -shift : 0));
  return freq < 0 ? 0 - u : u;
}

cudaError_t launch_norm_rope(RopeParams& p, cudaStream_t st, int* launches) {
  return p.dtype == 0 ? launch_dim<float>(p, st, launches) : launch_dim<__nv_bfloat16>(p, st, launches);
}

}  // namespace swam
