// Residual addition and root-mean-square norm on gfx950, forward and backward,
// and the values of an MX8 tensor.
//
//   S = X + R (stored in the tensors' type; x = S below, or X without R)
//   r = 1 / sqrt(mean(x^2) + eps);   Y = x r w;   MX8 of the fp32 Y
//   dX = r (dY w - x r^2 mean(dY w x)) + dS;   dw = sum over rows of dY x r
//
// All are bound by memory: each element is loaded once, kept in registers
// across the row's reduction, and its results stored once (but the gradient of rows
// past 8192 elements, whose workgroups of up to 1024 threads have 128 registers a
// lane, keeps 44 bytes a lane in scratch memory in bf16 and 208 in fp32).  A workgroup
// of W waves owns a row at a time; lane-consecutive 16-byte vectors; sums in fp32.
// bf16: 32768 rows of 7168 with R, S, Y and MX8 365 us (2.12 GB, 5.8 TB/s), its
// values read back 143 us; 16385 rows of 4096 backward 102 us (537 MB, 5.2 TB/s).
#include <algorithm>

#include "common.h"
#include "kernels.h"
#include "mx.h"

namespace memfine {
namespace {

// Sum over a wave, in every lane.
__device__ __forceinline__ float wave_sum(float v) {
#pragma unroll
  for (int o = 32; o > 0; o >>= 1) v += __shfl_xor(v, o, 64);
  return v;
}

// One row per workgroup; V vectors per lane, vector i of lane l of wave w at
// column ((i W + w) 64 + l) VEC, W = blockDim.x / 64.  S may be X or R.
template <typename T, int V>
__global__ __launch_bounds__(1024) void norm_fwd_kernel(
    const T* X, const T* R, const T* __restrict__ w, float eps, int h, T* S, T* __restrict__ Y,
    uint8_t* __restrict__ Q, uint8_t* __restrict__ QS) {
  constexpr int E = Elem<T>::kVec;
  __shared__ float part[16];
  const int nv = h / E, W = blockDim.x >> 6, lane = threadIdx.x & 63, wv = threadIdx.x >> 6;
  const int64_t row = (int64_t)blockIdx.x * h;
  u32x4_t raw[V], res[V], wt[V];
#pragma unroll
  for (int i = 0; i < V; ++i) {
    const int c = i * blockDim.x + threadIdx.x;
    const int at = c < nv ? c : 0;
    raw[i] = ((const u32x4_t*)(X + row))[at];
    if (R) res[i] = ((const u32x4_t*)(R + row))[at];
    wt[i] = ((const u32x4_t*)w)[at];
  }
  float x[V][E], sq = 0.f;
#pragma unroll
  for (int i = 0; i < V; ++i) {
    const int c = i * blockDim.x + threadIdx.x;
    unpack16(raw[i], x[i], (T*)nullptr);
    if (R) {
      float a[E];
      unpack16(res[i], a, (T*)nullptr);
#pragma unroll
      for (int q = 0; q < E; ++q) a[q] += x[i][q];
      // the sum is rounded to the stream's type, and the norm is of what is stored
      const u32x4_t s = pack16(a, (T*)nullptr);
      unpack16(s, x[i], (T*)nullptr);
      if (S && c < nv) ((u32x4_t*)(S + row))[c] = s;
    }
    if (c < nv) {
#pragma unroll
      for (int q = 0; q < E; ++q) sq = fmaf(x[i][q], x[i][q], sq);
    }
  }
  sq = wave_sum(sq);
  if (W > 1) {
    if (lane == 0) part[wv] = sq;
    __syncthreads();
    sq = 0.f;
    for (int i = 0; i < W; ++i) sq += part[i];
  }
  const float r = 1.f / sqrtf(sq / (float)h + eps);
#pragma unroll
  for (int i = 0; i < V; ++i) {
    const int c = i * blockDim.x + threadIdx.x;
    float g[E];
    unpack16(wt[i], g, (T*)nullptr);
#pragma unroll
    for (int q = 0; q < E; ++q) g[q] = g[q] * x[i][q] * r;  // (bf16: w x is exact)
    if (Y && c < nv) ((u32x4_t*)(Y + row))[c] = pack16(g, (T*)nullptr);
    if (Q) {
      // 32 / E consecutive lanes hold a block (h is a multiple of 64, so a
      // block lies wholly inside or outside the row)
      uint32_t m = 0;
#pragma unroll
      for (int q = 0; q < E; ++q) m = umax(m, abs_bits(g[q]));
      const uint32_t s = mx8_scale(lanes_umax<kMxBlock / E>(m));
      const float inv = mx_inverse_scale(s);
      if (c < nv) {
#pragma unroll
        for (int q = 0; q < E; q += 4)
          ((uint32_t*)(Q + row))[(c * E + q) / 4] =
              pack_e4m3x4(g[q] * inv, g[q + 1] * inv, g[q + 2] * inv, g[q + 3] * inv);
        if ((lane & (kMxBlock / E - 1)) == 0) QS[(row + c * E) / kMxBlock] = (uint8_t)s;
      }
    }
  }
}

// Backward: workgroup b takes rows b, b + grid, ...; each lane keeps the sums
// of dw of its own columns in registers over its rows and writes them as row b
// of `part` [grid, h].  dX may be dY or dS: a row is loaded before it is stored, and
// the row loaded ahead belongs to this workgroup alone.
template <typename T, int V, int kThreads>
__global__ __launch_bounds__(kThreads) void norm_bwd_kernel(
    const T* __restrict__ X, const T* __restrict__ w, const T* dY, const T* dS, float eps,
    int64_t T_, int h, T* dX, float* __restrict__ partial) {
  constexpr int E = Elem<T>::kVec;
  __shared__ float part[2][2][16];
  const int nv = h / E, W = blockDim.x >> 6, lane = threadIdx.x & 63, wv = threadIdx.x >> 6;
  u32x4_t rw[V];
  float acc[V][E];
#pragma unroll
  for (int i = 0; i < V; ++i) {
    const int c = i * blockDim.x + threadIdx.x;
    rw[i] = ((const u32x4_t*)w)[c < nv ? c : 0];
#pragma unroll
    for (int q = 0; q < E; ++q) acc[i][q] = 0.f;
  }
  int parity = 0;
  u32x4_t rx[V], rd[V], rs[V];
  auto load = [&](int64_t t) {
    const int64_t row = t * h;
#pragma unroll
    for (int i = 0; i < V; ++i) {
      const int c = i * blockDim.x + threadIdx.x;
      const int at = c < nv ? c : 0;
      rx[i] = ((const u32x4_t*)(X + row))[at];
      rd[i] = ((const u32x4_t*)(dY + row))[at];
      if (dS) rs[i] = ((const u32x4_t*)(dS + row))[at];
    }
  };
  load(blockIdx.x);  // (no more workgroups than rows)
  for (int64_t t = blockIdx.x; t < T_; t += gridDim.x, parity ^= 1) {
    const int64_t row = t * h;
    float x[V][E], d[V][E], sq = 0.f, pr = 0.f;
#pragma unroll
    for (int i = 0; i < V; ++i) {
      const int c = i * blockDim.x + threadIdx.x;
      unpack16(rx[i], x[i], (T*)nullptr);
      unpack16(rd[i], d[i], (T*)nullptr);
      if (c < nv) {
        float wt[E];
        unpack16(rw[i], wt, (T*)nullptr);
#pragma unroll
        for (int q = 0; q < E; ++q) {
          sq = fmaf(x[i][q], x[i][q], sq);
          pr = fmaf(d[i][q] * wt[q], x[i][q], pr);
        }
      }
    }
    u32x4_t now[V];
#pragma unroll
    for (int i = 0; i < V; ++i) now[i] = rs[i];
    if (t + gridDim.x < T_) load(t + gridDim.x);  // the next row, in flight over this one's sums
    sq = wave_sum(sq);
    pr = wave_sum(pr);
    if (W > 1) {
      // two buffers by turns: a wave that writes a row's sums has passed the
      // barrier of the row before, so all have read those of two rows before
      if (lane == 0) {
        part[parity][0][wv] = sq;
        part[parity][1][wv] = pr;
      }
      __syncthreads();
      sq = pr = 0.f;
      for (int i = 0; i < W; ++i) {
        sq += part[parity][0][i];
        pr += part[parity][1][i];
      }
    }
    const float r = 1.f / sqrtf(sq / (float)h + eps);
    const float k = r * r * (pr / (float)h);
#pragma unroll
    for (int i = 0; i < V; ++i) {
      const int c = i * blockDim.x + threadIdx.x;
      float o[E], wt[E];
      if (dS) unpack16(now[i], o, (T*)nullptr);
      unpack16(rw[i], wt, (T*)nullptr);
#pragma unroll
      for (int q = 0; q < E; ++q) {
        acc[i][q] = fmaf(d[i][q], x[i][q] * r, acc[i][q]);
        const float g = r * (d[i][q] * wt[q] - x[i][q] * k);
        o[q] = dS ? o[q] + g : g;
      }
      if (c < nv) ((u32x4_t*)(dX + row))[c] = pack16(o, (T*)nullptr);
    }
  }
  float* out = partial + (int64_t)blockIdx.x * h;
#pragma unroll
  for (int i = 0; i < V; ++i) {
    const int c = i * blockDim.x + threadIdx.x;
    if (c >= nv) continue;
#pragma unroll
    for (int q = 0; q < E; q += 4)
      *(f32x4_t*)(out + c * E + q) =
          (f32x4_t){acc[i][q], acc[i][q + 1], acc[i][q + 2], acc[i][q + 3]};
  }
}

// dw (+)= the sum of the partial rows: a workgroup owns 64 columns, its sixteen
// waves every sixteenth row each, summed in a fixed order (four waves: a chain
// of loads four times as long, 12 us of the 117 of 16385 rows of 4096, now 5).
constexpr int kDwWaves = 16;
__global__ __launch_bounds__(64 * kDwWaves) void norm_dw_kernel(const float* __restrict__ partial,
                                                                int rows, int h, int accumulate,
                                                                float* __restrict__ dw) {
  __shared__ float part[kDwWaves][64];
  const int lane = threadIdx.x & 63, wv = threadIdx.x >> 6;
  const int c = blockIdx.x * 64 + lane;  // h is a multiple of 64
  float s = 0.f;
#pragma unroll 8
  for (int i = wv; i < rows; i += kDwWaves) s += partial[(int64_t)i * h + c];
  part[wv][lane] = s;
  __syncthreads();
  if (wv == 0) {
    s = 0.f;
#pragma unroll
    for (int i = 0; i < kDwWaves; ++i) s += part[i][lane];
    dw[c] = accumulate ? dw[c] + s : s;
  }
}

// The values of an MX8 tensor: a thread takes 8 (bf16) or 4 (fp32) of them.
template <typename T>
__global__ __launch_bounds__(256) void mx8_unpack_kernel(const uint8_t* __restrict__ Q,
                                                         const uint8_t* __restrict__ QS, int64_t n,
                                                         T* __restrict__ out) {
  constexpr int E = Elem<T>::kVec;
  const int64_t v = thread_id();
  if (v >= n / E) return;
  const float s = mx_scale_value(QS[v * E / kMxBlock]);
  float f[E];
#pragma unroll
  for (int q = 0; q < E; q += 4) {
    const int b = ((const int*)Q)[(v * E + q) / 4];
    const f32x2_t lo = __builtin_amdgcn_cvt_pk_f32_fp8(b, false);
    const f32x2_t hi = __builtin_amdgcn_cvt_pk_f32_fp8(b, true);
    f[q] = lo[0] * s;
    f[q + 1] = lo[1] * s;
    f[q + 2] = hi[0] * s;
    f[q + 3] = hi[1] * s;
  }
  ((u32x4_t*)out)[v] = pack16(f, (T*)nullptr);
}

// Workgroup of a row of nv vectors: two vectors per lane where at most 16
// waves can hold the row so, else four.
struct RowShape {
  int V, waves;
};
RowShape row_shape(int nv) {
  const int V = nv <= 64 ? 1 : nv <= 2048 ? 2 : 4;
  return {V, (nv + 64 * V - 1) / (64 * V)};
}

template <typename T, int V>
void run_norm_fwd(const void* X, const void* R, const void* w, float eps, int64_t rows, int h,
                  int waves, void* S, void* Y, uint8_t* Q, uint8_t* QS, hipStream_t s) {
  const int64_t most = kMostItems / (64 * waves);
  auto at = [](auto* p, int64_t i) { return p ? p + i : nullptr; };
  for (int64_t t = 0; t < rows; t += most) {
    const int64_t i = t * h;
    norm_fwd_kernel<T, V><<<(unsigned)std::min(most, rows - t), 64 * waves, 0, s>>>(
        (const T*)X + i, at((const T*)R, i), (const T*)w, eps, h, at((T*)S, i), at((T*)Y, i),
        at(Q, i), at(QS, i / kMxBlock));
  }
}

}  // namespace

hipError_t launch_norm_fwd(int dtype, const void* X, const void* R, const void* w, float eps,
                           int64_t T, int h, void* S, void* Y, uint8_t* Q, uint8_t* QS,
                           hipStream_t s) {
  if (T == 0) return hipSuccess;
  const RowShape rs = row_shape(h / (dtype == 0 ? 8 : 4));
  if (rs.waves > 16) return hipErrorInvalidValue;
#define MEMFINE_NORM(T_, V_) run_norm_fwd<T_, V_>(X, R, w, eps, T, h, rs.waves, S, Y, Q, QS, s)
  if (dtype == 0) {
    if (rs.V == 1) MEMFINE_NORM(bf16_t, 1);
    else MEMFINE_NORM(bf16_t, 2);  // (16384 elements are 16 waves of two vectors)
  } else {
    if (rs.V == 1) MEMFINE_NORM(float, 1);
    else if (rs.V == 2) MEMFINE_NORM(float, 2);
    else MEMFINE_NORM(float, 4);
  }
#undef MEMFINE_NORM
  return hipGetLastError();
}

// Rows of dw partials: one round of workgroups, of as many waves a CU as its
// registers hold (bf16, two vectors a lane: 12, else 16; 16 of them, in two
// rounds, 115 us at 16385 rows of 4096, 12 106).
int norm_bwd_blocks(int dtype, int64_t T, int h, int cus) {
  const RowShape rs = row_shape(h / (dtype == 0 ? 8 : 4));
  const int waves = dtype == 0 && rs.V > 1 ? 12 : 16;
  const int64_t want = (int64_t)cus * (waves / rs.waves > 0 ? waves / rs.waves : 1);
  return (int)(T < want ? T : want);
}

hipError_t launch_norm_bwd(int dtype, const void* X, const void* w, const void* dY, const void* dS,
                           float eps, int64_t T, int h, void* dX, float* partial, int blocks,
                           int accumulate, float* dw, hipStream_t s) {
  if (T == 0) return hipSuccess;
  const RowShape rs = row_shape(h / (dtype == 0 ? 8 : 4));
  const dim3 grid(blocks), block(64 * rs.waves);
  if (rs.waves > 16) return hipErrorInvalidValue;
#define MEMFINE_NORM(T_, V_, N_)                                                                  \
  norm_bwd_kernel<T_, V_, N_><<<grid, block, 0, s>>>((const T_*)X, (const T_*)w, (const T_*)dY,   \
                                                     (const T_*)dS, eps, T, h, (T_*)dX, partial)
  if (dtype == 0) {
    if (rs.V == 1) MEMFINE_NORM(bf16_t, 1, 512);
    else if (rs.waves <= 8) MEMFINE_NORM(bf16_t, 2, 512);
    else MEMFINE_NORM(bf16_t, 2, 1024);  // (16384 elements are 16 waves of two vectors)
  } else {
    if (rs.V == 1) MEMFINE_NORM(float, 1, 512);
    else if (rs.V == 2 && rs.waves <= 8) MEMFINE_NORM(float, 2, 512);
    else if (rs.V == 2) MEMFINE_NORM(float, 2, 1024);
    else MEMFINE_NORM(float, 4, 1024);
  }
#undef MEMFINE_NORM
  norm_dw_kernel<<<h / 64, 64 * kDwWaves, 0, s>>>(partial, blocks, h, accumulate, dw);
  return hipGetLastError();
}

hipError_t launch_mx8_unpack(int dtype, const uint8_t* Q, const uint8_t* QS, int64_t n, void* out,
                             hipStream_t s) {
  if (n == 0) return hipSuccess;
  const dim3 grid = grid_of(n / (dtype == 0 ? 8 : 4));
  if (dtype == 0) mx8_unpack_kernel<bf16_t><<<grid, 256, 0, s>>>(Q, QS, n, (bf16_t*)out);
  else mx8_unpack_kernel<float><<<grid, 256, 0, s>>>(Q, QS, n, (float*)out);
  return hipGetLastError();
}

}  // namespace memfine
