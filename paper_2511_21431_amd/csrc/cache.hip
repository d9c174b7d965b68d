// Rotation by position, and new tokens' way into a cache of pages, on gfx950.
//
//   y_a = x_a cos - x_b sin;  y_b = x_b cos + x_a sin
// for the pairs (a, b) = (i, i + D / 2), or (2 i, 2 i + 1) where interleaved, with
// the cosines and sines of the token's position (the inverse: -sin).
//
// Bound by memory: every element is loaded and stored once, in 16-byte pieces
// (MX8: 8 or 16 bytes stored).  D / 16 neighbouring threads own a head of a row, 8
// pairs each; 32 values of an MX8 block lie in 4 or 2 neighbouring lanes.
#include <algorithm>

#include "common.h"
#include "kernels.h"
#include "mx.h"

namespace memfine {
namespace {

// 16 elements of a head: 8 from `a` on, and 8 from `b` on.
template <typename T> struct Pairs {
  static constexpr int kV = 8 / Elem<T>::kVec;
  u32x4_t a[kV], b[kV];
  __device__ __forceinline__ void load(const T* pa, const T* pb) {
#pragma unroll
    for (int i = 0; i < kV; ++i) {
      a[i] = ((const u32x4_t*)pa)[i];
      b[i] = ((const u32x4_t*)pb)[i];
    }
  }
  __device__ __forceinline__ void values(float (&x)[8], float (&y)[8]) const {
    constexpr int E = Elem<T>::kVec;
#pragma unroll
    for (int i = 0; i < kV; ++i) {
      float f[E];
      unpack16(a[i], f, (T*)nullptr);
#pragma unroll
      for (int e = 0; e < E; ++e) x[i * E + e] = f[e];
      unpack16(b[i], f, (T*)nullptr);
#pragma unroll
      for (int e = 0; e < E; ++e) y[i * E + e] = f[e];
    }
  }
  __device__ __forceinline__ static void store(T* p, const float (&x)[8]) {
    constexpr int E = Elem<T>::kVec;
#pragma unroll
    for (int i = 0; i < kV; ++i) {
      float f[E];
#pragma unroll
      for (int e = 0; e < E; ++e) f[e] = x[i * E + e];
      ((u32x4_t*)p)[i] = pack16(f, (T*)nullptr);
    }
  }
};

// Turns 16 elements, x and y as Pairs holds them.
__device__ __forceinline__ void turn(float (&x)[8], float (&y)[8], const float (&cs)[8], const float (&sn)[8],
                                     bool interleaved) {
  if (interleaved) {
#pragma unroll
    for (int i = 0; i < 8; i += 2) {
      const float a = x[i], b = x[i + 1], p = y[i], q = y[i + 1];
      x[i] = a * cs[i / 2] - b * sn[i / 2];
      x[i + 1] = b * cs[i / 2] + a * sn[i / 2];
      y[i] = p * cs[4 + i / 2] - q * sn[4 + i / 2];
      y[i + 1] = q * cs[4 + i / 2] + p * sn[4 + i / 2];
    }
  } else {
#pragma unroll
    for (int i = 0; i < 8; ++i) {
      const float a = x[i], b = y[i];
      x[i] = a * cs[i] - b * sn[i];
      y[i] = b * cs[i] + a * sn[i];
    }
  }
}

// The 8 pairs' cosines and sines at a position; NaN past the tables (whose first row is
// read then: a branch around the loads keeps two of the values in memory).
__device__ __forceinline__ void angles(const RopeTable& r, int64_t pos, int at, int dim, float (&cs)[8],
                                       float (&sn)[8]) {
  const bool in = pos < r.positions;
  const int64_t row = (in ? pos : 0) * (dim / 2) + at;
  const float none = __uint_as_float(0x7fc00000u);
#pragma unroll
  for (int i = 0; i < 8; i += 4) {
    const f32x4_t c = *(const f32x4_t*)(r.cos + row + i), s = *(const f32x4_t*)(r.sin + row + i);
#pragma unroll
    for (int e = 0; e < 4; ++e) {
      cs[i + e] = in ? c[e] : none;
      sn[i + e] = in ? (r.inverse ? -s[e] : s[e]) : none;
    }
  }
}

// The sequence of row t, with its first row and length; false for a row of none.
// (The last sequence that begins at or before t; offsets are cut to [0, T].)
__device__ __forceinline__ bool sequence_of(const int32_t* __restrict__ offsets, int seqs, int64_t T, int64_t t,
                                            int& b, int64_t& begin, int64_t& end) {
  int lo = 0, hi = seqs;  // offsets[lo] <= t, offsets[hi] > t, as far as they ascend
  if (offsets[0] > t || offsets[seqs] <= t) return false;
  while (hi - lo > 1) {
    const int mid = (lo + hi) >> 1;
    if (offsets[mid] <= t) lo = mid;
    else hi = mid;
  }
  b = lo;
  begin = max(offsets[lo], 0);
  end = min((int64_t)offsets[lo + 1], T);
  return begin <= t && t < end;
}

// Rows of heads of D elements, turned.  A workgroup takes rows blockIdx.x,
// blockIdx.x + gridDim.x, ...; its threads the pieces of a row's heads (so that the row's
// angles are loaded once).  8192 rows of 256 heads of 128: 211 us, 5.1 TB/s.
template <typename T, int D>
__global__ __launch_bounds__(256) void rope_kernel(const RopeArgs g) {
  constexpr int kPer = D / 16;
  const int piece = threadIdx.x % kPer, step = 256 / kPer * gridDim.y;
  const int a = g.r.interleaved ? piece * 16 : piece * 8, b = g.r.interleaved ? a + 8 : a + D / 2;
  for (int64_t t = blockIdx.x; t < g.T; t += gridDim.x) {
    int seq;
    int64_t begin, end;
    if (!sequence_of(g.offsets, g.seqs, g.T, t, seq, begin, end)) continue;
    float cs[8], sn[8];
    angles(g.r, t - begin, piece * 8, D, cs, sn);
    for (int h = blockIdx.y * (256 / kPer) + threadIdx.x / kPer; h < g.heads; h += step) {
      const T* x = (const T*)g.X + t * g.ldx + h * D;
      Pairs<T> p;
      p.load(x + a, x + b);
      float u[8], v[8];
      p.values(u, v);
      turn(u, v, cs, sn, g.r.interleaved);
      T* y = (T*)g.Y + t * g.ldy + h * D;
      Pairs<T>::store(y + a, u);
      Pairs<T>::store(y + b, v);
    }
  }
}

// 32 values, of which this lane holds 8 and `N` lanes the block, as MX8.
template <int N> __device__ __forceinline__ u32x2_t mx8_of(const float (&x)[8], uint32_t& scale) {
  uint32_t m = 0;
#pragma unroll
  for (int i = 0; i < 8; ++i) m = umax(m, abs_bits(x[i]));
  m = lanes_umax<N>(m);
  scale = mx8_scale(m);
  const float inv = mx_inverse_scale(scale);
  return (u32x2_t){pack_e4m3x4(x[0] * inv, x[1] * inv, x[2] * inv, x[3] * inv),
                   pack_e4m3x4(x[4] * inv, x[5] * inv, x[6] * inv, x[7] * inv)};
}

// New rows: keys, turned, and values into the cache's pages, queries turned into rows of
// their own.  Heads in order: queries, keys, values.  8191 rows of 64 query and 8 key-value
// heads of 128 into MX8 pages 70 us, 4.6 TB/s; 64 rows 4 us, a launch's latency.
template <int D, bool MX8>
__global__ __launch_bounds__(256) void kv_write_kernel(const WriteArgs g) {
  constexpr int kPer = D / 16;
  const int piece = threadIdx.x % kPer, step = 256 / kPer * gridDim.y;
  const bool turned = g.r.cos != nullptr;
  const int all = g.heads + 2 * g.kv_heads;
  for (int64_t t = blockIdx.x; t < g.T; t += gridDim.x) {
    int seq = (int)t;
    int64_t begin = t, end = t + 1;
    if (g.offsets && !sequence_of(g.offsets, g.seqs, g.T, t, seq, begin, end)) continue;
    const int64_t pos = (int64_t)g.lengths[seq] - (end - t);
    if (pos < 0 || pos >= g.most) continue;
    const int32_t id = g.table[(int64_t)seq * g.width + (pos >> g.page_shift)];
    const bool held = (uint32_t)id < (uint32_t)g.pages;
    float cs[8], sn[8];
    if (turned) angles(g.r, pos, piece * 8, D, cs, sn);
    for (int h = blockIdx.y * (256 / kPer) + threadIdx.x / kPer; h < all; h += step) {
      // (all lanes of a head take the same branches)
      const bool is_q = h < g.heads, is_v = h >= g.heads + g.kv_heads;
      if (!is_q && !held) continue;
      const int kv = is_v ? h - g.heads - g.kv_heads : h - g.heads;
      const bf16_t* x = is_q ? (const bf16_t*)g.Q + t * g.ldq + h * D
                             : is_v ? (const bf16_t*)g.V + t * g.ldv + kv * D
                                    : (const bf16_t*)g.K + t * g.ldk + kv * D;
      const bool pairs = turned && !is_v && !g.r.interleaved;
      const int a = pairs ? piece * 8 : piece * 16, b = pairs ? a + D / 2 : a + 8;
      Pairs<bf16_t> p;
      p.load(x + a, x + b);
      float u[8], v[8];
      p.values(u, v);
      if (turned && !is_v) turn(u, v, cs, sn, g.r.interleaved);
      if (is_q) {
        bf16_t* y = (bf16_t*)g.R + (t * g.heads + h) * D;
        Pairs<bf16_t>::store(y + a, u);
        Pairs<bf16_t>::store(y + b, v);
        continue;
      }
      const int64_t row = ((int64_t)id * g.kv_heads + kv) * g.page + (pos & (g.page - 1));
      if constexpr (MX8) {
        uint8_t* y = (uint8_t*)(is_v ? g.v : g.k) + row * D;
        uint8_t* sc = (is_v ? g.vs : g.ks) + row * (D / 32);
        uint32_t s0, s1;
        u32x2_t lo, hi;
        if (pairs) {
          lo = mx8_of<4>(u, s0);
          hi = mx8_of<4>(v, s1);
          if ((piece & 3) == 0) {
            sc[a / 32] = (uint8_t)s0;
            sc[b / 32] = (uint8_t)s1;
          }
        } else {
          // a block is 16 values of this lane and 16 of its neighbour's
          uint32_t m = 0;
#pragma unroll
          for (int i = 0; i < 8; ++i) m = umax(m, umax(abs_bits(u[i]), abs_bits(v[i])));
          m = umax_dpp<0xb1>(m);
          s0 = mx8_scale(m);
          const float inv = mx_inverse_scale(s0);
          lo = (u32x2_t){pack_e4m3x4(u[0] * inv, u[1] * inv, u[2] * inv, u[3] * inv),
                         pack_e4m3x4(u[4] * inv, u[5] * inv, u[6] * inv, u[7] * inv)};
          hi = (u32x2_t){pack_e4m3x4(v[0] * inv, v[1] * inv, v[2] * inv, v[3] * inv),
                         pack_e4m3x4(v[4] * inv, v[5] * inv, v[6] * inv, v[7] * inv)};
          if ((piece & 1) == 0) sc[a / 32] = (uint8_t)s0;
        }
        *(u32x2_t*)(y + a) = lo;
        *(u32x2_t*)(y + b) = hi;
      } else {
        bf16_t* y = (bf16_t*)(is_v ? g.v : g.k) + row * D;
        Pairs<bf16_t>::store(y + a, u);
        Pairs<bf16_t>::store(y + b, v);
      }
    }
  }
}

// Workgroups: a row each, and a second dimension over its heads where rows are few.
dim3 row_grid(int64_t T, int heads, int dim, int cus) {
  const int per = 256 / (dim / 16);
  const int64_t x = std::min<int64_t>(T, 1 << 22);
  const int64_t most = (heads + per - 1) / per;
  const int64_t y = std::min<int64_t>(most, std::max<int64_t>(1, 8 * cus / x));
  return dim3((unsigned)x, (unsigned)y);
}

}  // namespace

hipError_t launch_rope(const RopeArgs& g, int cus, hipStream_t s) {
  const dim3 grid = row_grid(g.T, g.heads, g.dim, cus);
  if (g.f32) {
    if (g.dim == 64) rope_kernel<float, 64><<<grid, 256, 0, s>>>(g);
    else rope_kernel<float, 128><<<grid, 256, 0, s>>>(g);
  } else {
    if (g.dim == 64) rope_kernel<bf16_t, 64><<<grid, 256, 0, s>>>(g);
    else rope_kernel<bf16_t, 128><<<grid, 256, 0, s>>>(g);
  }
  return hipGetLastError();
}

hipError_t launch_kv_write(const WriteArgs& g, int cus, hipStream_t s) {
  const dim3 grid = row_grid(g.T, g.heads + 2 * g.kv_heads, g.dim, cus);
  if (g.dim == 64) {
    if (g.ks) kv_write_kernel<64, true><<<grid, 256, 0, s>>>(g);
    else kv_write_kernel<64, false><<<grid, 256, 0, s>>>(g);
  } else {
    if (g.ks) kv_write_kernel<128, true><<<grid, 256, 0, s>>>(g);
    else kv_write_kernel<128, false><<<grid, 256, 0, s>>>(g);
  }
  return hipGetLastError();
}

}  // namespace memfine
