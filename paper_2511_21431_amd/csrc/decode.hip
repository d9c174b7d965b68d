// Attention of one new token a sequence over a cache of pages, on gfx950.
//
//   s_j = scale q . k_j over the sequence's tokens j (the last `window` of them,
//   where there is one);  o = sum_j exp(s_j - lse) v_j,  lse = log sum_j exp(s_j)
//
// Bound by memory: every key and value is read once for each 16 heads that share it (64 of them:
// four times, in runs that may lie far apart).  The tokens of all sequences
// and key-value heads are laid end to end in steps of 128, of which each
// workgroup takes an equal run, whatever the lengths are; runs end inside
// sequences, whose parts (sums relative to a maximum of their own) a second
// kernel joins in order.  A step's four waves take 32 tokens each.
//
// Up to 16 heads that share a key-value head are the columns of 16 x 16 products
// on the matrix cores (v_mfma_f32_16x16x32_bf16).  Keys go from memory into
// registers as the operand; values through LDS, from where a transposing load
// makes them one.  The scores' accumulators, as two bf16 values each, are the second
// product's other operand as they stand: value rows are read in the order that they have.
#include <algorithm>
#include <type_traits>

#include "common.h"
#include "kernels.h"
#include "mx.h"

namespace memfine {
namespace {

constexpr float kLog2e = 1.4426950408889634f, kLn2 = 0.6931471805599453f;
constexpr int kTokens = 32;              // of a wave's step
constexpr int kStep = 4 * kTokens;       // of a workgroup's

typedef short s16x4_t __attribute__((ext_vector_type(4)));
typedef __attribute__((address_space(3))) s16x4_t lds_s16x4;

__device__ __forceinline__ float exp2_(float x) { return __builtin_amdgcn_exp2f(x); }

// The largest and the sum over the lanes l, l ^ 16, l ^ 32, l ^ 48.
template <class F> __device__ __forceinline__ float over_quarters(float v, F f) {
  u32x2_t r = __builtin_bit_cast(
      u32x2_t, __builtin_amdgcn_permlane32_swap(__float_as_uint(v), __float_as_uint(v), false, false));
  v = f(__uint_as_float(r[0]), __uint_as_float(r[1]));
  r = __builtin_bit_cast(
      u32x2_t, __builtin_amdgcn_permlane16_swap(__float_as_uint(v), __float_as_uint(v), false, false));
  return f(__uint_as_float(r[0]), __uint_as_float(r[1]));
}
__device__ __forceinline__ float quarters_max(float v) {
  return over_quarters(v, [](float a, float b) { return fmaxf(a, b); });
}
__device__ __forceinline__ float quarters_sum(float v) {
  return over_quarters(v, [](float a, float b) { return a + b; });
}

// ------------------------------------------------------------- work to do
// A sequence's tokens that count: [lo, n), lo0 = lo cut down to a block of 16.
struct Span {
  int lo, lo0, n;
};
__device__ __forceinline__ Span span_of(const DecodeArgs& g, int b) {
  Span s;
  s.n = min(max(g.lengths[b], 0), g.most);
  s.lo = g.window > 0 ? max(0, s.n - g.window) : 0;
  s.lo0 = s.lo & ~15;
  return s;
}
__device__ __forceinline__ int steps_of(const Span& s) { return (s.n - s.lo0 + kStep - 1) / kStep; }

// Sum over the lanes up to this one, by DPP: row shifts, then each row's last lane to the next.
template <int kCtrl, int kRows> __device__ __forceinline__ int add_dpp(int v) {
  return v + __builtin_amdgcn_update_dpp(0, v, kCtrl, kRows, 0xf, false);
}
__device__ __forceinline__ int wave_scan(int v) {
  v = add_dpp<0x111, 0xf>(v);
  v = add_dpp<0x112, 0xf>(v);
  v = add_dpp<0x114, 0xf>(v);
  v = add_dpp<0x118, 0xf>(v);
  v = add_dpp<0x142, 0xa>(v);
  return add_dpp<0x143, 0xc>(v);
}
// a / b, in 32 bits where these hold a (all but caches of billions of tokens).
__device__ __forceinline__ int64_t quotient(int64_t a, int64_t b) {
  return (uint64_t)a >> 32 ? a / b : (int64_t)((uint32_t)a / (uint32_t)b);
}

// The steps of all sequences (of one pair each), for every thread of a workgroup, and
// the steps before some sequences.  Up to 64 sequences a wave sums them by itself;
// more are summed by the workgroup's 256 threads, `per` to each.
struct Plan {
  int64_t total;
  int64_t before;  // steps before this lane's sequence (few), or before this thread's
  int n, per;      // few: the lane's sequence's steps
};
__device__ __forceinline__ bool few(const DecodeArgs& g) { return g.seqs <= 64; }
__device__ __forceinline__ Plan plan_of(const DecodeArgs& g, int64_t* part) {
  Plan p;
  const int lane = threadIdx.x & 63, w = threadIdx.x >> 6;
  if (few(g)) {
    p.per = 1;
    p.n = steps_of(span_of(g, min(lane, g.seqs - 1)));
    if (lane >= g.seqs) p.n = 0;
    const int inc = wave_scan(p.n);  // (64 sequences of at most 2^23 steps)
    p.total = __builtin_amdgcn_readlane(inc, 63);
    p.before = inc - p.n;
    return p;
  }
  p.per = (g.seqs + 255) / 256;
  int64_t v = 0;
  const int first = threadIdx.x * p.per, last = min(first + p.per, g.seqs);
  for (int b = first; b < last; ++b) v += steps_of(span_of(g, b));
  int64_t inc = v;
#pragma unroll
  for (int o = 1; o < 64; o <<= 1) {
    const int64_t y = __shfl_up(inc, o, 64);
    if (lane >= o) inc += y;
  }
  if (lane == 63) part[w] = inc;
  __syncthreads();
  p.total = 0;
  p.before = inc - v;
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    if (i < w) p.before += part[i];
    p.total += part[i];
  }
  return p;
}
// The sequence whose pairs' steps hold step `at` < total pairs, and the steps of those
// before it; the same in every thread.
__device__ __forceinline__ int sequence_at(const DecodeArgs& g, const Plan& p, int64_t at, int64_t* found,
                                           int64_t& base) {
  if (few(g)) {
    const uint64_t past = __ballot((p.before + p.n) * g.pairs > at);
    const int b = __builtin_ctzll(past);
    base = (int64_t)__builtin_amdgcn_readlane((int)p.before, b) * g.pairs;
    return b;
  }
  int64_t before = p.before;
  const int first = threadIdx.x * p.per, last = min(first + p.per, g.seqs);
  for (int b = first; b < last; ++b) {
    const int64_t n = steps_of(span_of(g, b));
    if (at >= before * g.pairs && at < (before + n) * g.pairs) {
      found[0] = b;
      found[1] = before * g.pairs;
    }
    before += n;
  }
  __syncthreads();
  base = found[1];
  return __builtin_amdgcn_readfirstlane((int)found[0]);
}
// The steps before sequence b.
__device__ __forceinline__ int64_t steps_before(const DecodeArgs& g, const Plan& p, int b, int64_t* found) {
  if (few(g)) return __builtin_amdgcn_readlane((int)p.before, b);
  const int first = threadIdx.x * p.per;
  if (b >= first && b < first + p.per) {
    int64_t before = p.before;
    for (int i = first; i < b; ++i) before += steps_of(span_of(g, i));
    found[0] = before;
  }
  __syncthreads();
  return found[0];
}
// Steps a workgroup takes.
__device__ __forceinline__ int64_t share_of(const DecodeArgs& g, int64_t total) {
  const int64_t all = total * g.pairs;
  return std::max<int64_t>(quotient(all + g.groups - 1, g.groups), 1);
}

// --------------------------------------------------------------- operands
// D elements of 32 tokens, in two blocks of 16 that each lie in one page.  A
// lane of quarter g reads token t % 16 of a block for keys.  The reduction over a
// row goes in steps of 32 elements, of which a lane holds 8; in MX8 a 16-byte
// load holds two steps' 8.
template <int D, bool MX8> struct Held;
template <int D> struct Held<D, false> {
  static constexpr int kLoads = D / 32;  // 16-byte loads a lane and block
  // first element of a lane's part of load i
  __device__ __forceinline__ static int at(int i, int g) { return i * 32 + g * 8; }
};
template <int D> struct Held<D, true> {
  static constexpr int kLoads = D / 64;
  __device__ __forceinline__ static int at(int i, int g) { return i * 64 + g * 16; }
};

// Eight e4m3 values with their scale, exactly.
__device__ __forceinline__ bf16x8_t bf16_of(uint32_t a, uint32_t b, float scale) {
  const bf16x2_t p0 = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(a, scale, false);
  const bf16x2_t p1 = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(a, scale, true);
  const bf16x2_t p2 = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(b, scale, false);
  const bf16x2_t p3 = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(b, scale, true);
  return (bf16x8_t){p0[0], p0[1], p1[0], p1[1], p2[0], p2[1], p3[0], p3[1]};
}
// The conversion reads the scale's exponent field alone: byte 0 is 2^-127, 255 NaN.
__device__ __forceinline__ float cvt_scale(uint32_t s) { return __uint_as_float(s << 23); }

// Values of a wave's step in LDS: 32 rows of D bf16; 16-byte unit u of a row at u ^
// swizzle(row), so that a transposing load's 16 rows x 16 columns spread over the banks.
template <int D> struct Values {
  static constexpr int kPitch = 2 * D, kBytes = kTokens * kPitch;
  __device__ __forceinline__ static int swizzle(int row) {
    if constexpr (D == 128) return (row & 7) << 1;
    else return (row & 6);
  }
  __device__ __forceinline__ static int at(int row, int unit) {
    return row * kPitch + ((unit ^ swizzle(row)) << 4);
  }
  // columns col0 .. col0 + 15 as an operand's rows: lane quarter g has tokens 4 g ..
  // 4 g + 3 and 16 + 4 g .. 16 + 4 g + 3, as the scores' accumulators
  __device__ __forceinline__ static bf16x8_t col(const char* lds, int col0, int lane) {
    const int j = lane & 15, r = (lane >> 4) * 4 + (j >> 2);
    const int u = (col0 + 4 * (j & 3)) >> 3, in = (j & 1) << 3;
    const s16x4_t lo = __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds_s16x4*)(lds + at(r, u) + in));
    const s16x4_t hi = __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds_s16x4*)(lds + at(r + 16, u) + in));
    return __builtin_bit_cast(bf16x8_t, __builtin_shufflevector(lo, hi, 0, 1, 2, 3, 4, 5, 6, 7));
  }
};

// What a wave has in flight: keys and values of one step.
template <int D, bool MX8> struct Loaded {
  static constexpr int kK = 2 * Held<D, MX8>::kLoads;
  u32x4_t k[kK], v[kK];
  uint32_t ks[MX8 ? 2 : 1], vs[MX8 ? kK : 1];
};

// Sums of a (pair of a sequence and) key-value head's part: o relative to 2^m.
template <int D> struct Sums {
  f32x4_t o[D / 16];  // o^T: columns 16 i + 4 g + e of the query lane % 16
  float m, l;         // (l: of this lane quarter's tokens)
};

// Two workgroups a CU, all resident, with the next step's loads in flight while one is
// multiplied: 2 x 4 waves x 16 KiB a CU (bf16, D = 128), several times what the memory's
// latency needs.  One sequence of 131072 tokens, 8 key-value heads of 128: 93.5 us, 5.7 TB/s
// (a plain kernel that only reads: 7.1); 16 of 2048, 128 heads 377 us, 5.7 TB/s; in MX8 64 of
// 4096 on average, pages of 16, 64 heads in 8 groups 109 us, 5.1 TB/s (the values' way through
// LDS as bf16: two writes a load with conflicts on 39 % of the cycles that LDS is busy, and
// vector instructions for 34 %).
template <int D, bool MX8>
__global__ __launch_bounds__(256, 2) void decode_kernel(const DecodeArgs g) {
  typedef Held<D, MX8> H;
  typedef Values<D> LV;
  constexpr int kRowBytes = MX8 ? D : 2 * D, kLoads = H::kLoads;
  __shared__ __align__(1024) char smem[4 * LV::kBytes > 4 * 16 * (D + 4) * 4 ? 4 * LV::kBytes
                                                                             : 4 * 16 * (D + 4) * 4];
  __shared__ int64_t part[4];
  __shared__ int64_t found[2];
  const int lane = threadIdx.x & 63, w = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int lg = lane >> 4, col = lane & 15;
  const Plan plan = plan_of(g, part);
  const int64_t share = share_of(g, plan.total), end = std::min(plan.total * g.pairs, (blockIdx.x + 1) * share);
  int64_t at = blockIdx.x * share;
  if (at >= end) return;
  // (all pairs of a sequence follow each other)
  int64_t base;
  int b = sequence_at(g, plan, at, found, base);
  const float c = g.scale * kLog2e;
  char* mine = smem + w * LV::kBytes;
  bool first_run = true;
  for (; at < end; ++b) {
    if (b >= g.seqs) return;  // (not reached)
    const Span sp = span_of(g, b);
    const int n = steps_of(sp);
    if (n == 0) continue;
    const int32_t* table = g.table + (int64_t)b * g.width;
    const int64_t stop = std::min(end, base + (int64_t)n * g.pairs);
    while (at < stop) {
      const int pair = (int)quotient(at - base, n), x0 = (int)(at - base - (int64_t)pair * n);
      const int x1 = (int)std::min<int64_t>(n, x0 + (stop - at));
      const int kv = pair / g.tiles, h0 = kv * g.group + pair % g.tiles * 16;
      const int heads = min(16, g.group - pair % g.tiles * 16);
      // queries: columns; the reduction's order is that of the keys' loads
      bf16x8_t q[D / 32];
#pragma unroll
      for (int i = 0; i < kLoads; ++i) {
        const bf16_t* p = (const bf16_t*)g.Q + b * g.ldq + (h0 + (col < heads ? col : 0)) * D + H::at(i, lg);
        if constexpr (MX8) {
          q[2 * i] = *(const bf16x8_t*)p;
          q[2 * i + 1] = *(const bf16x8_t*)(p + 8);
        } else {
          q[i] = *(const bf16x8_t*)p;
        }
      }
      Sums<D> a;
#pragma unroll
      for (int i = 0; i < D / 16; ++i) a.o[i] = (f32x4_t){0.f, 0.f, 0.f, 0.f};
      a.m = -INFINITY;
      a.l = 0.f;

      // page of block j (16 tokens, from sp.lo0 on) of this wave's run, by lanes: two blocks a step
      const int t_first = sp.lo0 + x0 * kStep + w * kTokens;
      auto pages = [&](int step) {  // lane l: block l % 2 of step + l / 2
        const int t = t_first + (step + (lane >> 1)) * kStep + (lane & 1) * 16;
        int id = -1;
        if (t < sp.n && step + (lane >> 1) < x1 - x0) id = table[t >> g.page_shift];
        return (uint32_t)id < (uint32_t)g.pages ? id : -1;
      };
      int ids = pages(0);
      Loaded<D, MX8> next;
      auto load = [&](int x) {
        const int id0 = __builtin_amdgcn_readlane(ids, (x & 31) * 2);
        const int id1 = __builtin_amdgcn_readlane(ids, (x & 31) * 2 + 1);
        const int t = t_first + x * kStep;
#pragma unroll
        for (int h = 0; h < 2; ++h) {
          const int id = h ? id1 : id0;
          const int in = (t + 16 * h) & (g.page - 1);
          const int64_t row = ((int64_t)max(id, 0) * g.kv_heads + kv) * g.page + in;
          const char* kp = (const char*)g.k + row * kRowBytes + (int64_t)col * kRowBytes;
          const char* vp = (const char*)g.v + row * kRowBytes;
#pragma unroll
          for (int i = 0; i < kLoads; ++i) {
            next.k[h * kLoads + i] = *(const u32x4_t*)(kp + H::at(i, lg) * (MX8 ? 1 : 2));
            next.v[h * kLoads + i] = *(const u32x4_t*)(vp + i * 1024 + lane * 16);
          }
          if constexpr (MX8) {
            if constexpr (D == 128) next.ks[h] = *(const uint32_t*)(g.ks + (row + col) * 4);
            else next.ks[h] = *(const uint16_t*)(g.ks + (row + col) * 2);
#pragma unroll
            for (int i = 0; i < kLoads; ++i)
              next.vs[h * kLoads + i] = g.vs[row * (D / 32) + (i * 1024 + lane * 16) / 32];
          }
        }
      };
      load(0);
      for (int x = 0; x < x1 - x0; ++x) {
        const Loaded<D, MX8> now = next;
        const int t0 = t_first + x * kStep;
        const int id0 = __builtin_amdgcn_readlane(ids, (x & 31) * 2);
        const int id1 = __builtin_amdgcn_readlane(ids, (x & 31) * 2 + 1);
        if (x + 1 < x1 - x0) {
          if (((x + 1) & 31) == 0) ids = pages(x + 1);
          load(x + 1);
        }
        if (id0 < 0 && id1 < 0) continue;  // (nothing of this wave's in the step)
        // tokens of each block that count
        const int lo0 = id0 < 0 ? 16 : sp.lo - t0, hi0 = id0 < 0 ? 0 : sp.n - t0;
        const int lo1 = id1 < 0 ? 16 : sp.lo - t0 - 16, hi1 = id1 < 0 ? 0 : sp.n - t0 - 16;
        const bool all = lo0 <= 0 && lo1 <= 0 && hi0 >= 16 && hi1 >= 16;
        // values to LDS; rows that do not count are zeros (a weight of zero times what
        // the page happens to hold there could be a NaN)
#pragma unroll
        for (int h = 0; h < 2; ++h)
#pragma unroll
          for (int i = 0; i < kLoads; ++i) {
            constexpr int kPerRow = kRowBytes / 16;
            const int r = (i * 64 + lane) / kPerRow, u = (i * 64 + lane) % kPerRow;
            const bool counts = all || (r >= (h ? lo1 : lo0) && r < (h ? hi1 : hi0));
            u32x4_t v = now.v[h * kLoads + i];
            if constexpr (MX8) {
              const float s = cvt_scale(now.vs[h * kLoads + i]);
              u32x4_t x0v = __builtin_bit_cast(u32x4_t, bf16_of(v[0], v[1], s));
              u32x4_t x1v = __builtin_bit_cast(u32x4_t, bf16_of(v[2], v[3], s));
              if (!counts) x0v = x1v = (u32x4_t){0, 0, 0, 0};
              *(u32x4_t*)(mine + LV::at(16 * h + r, 2 * u)) = x0v;
              *(u32x4_t*)(mine + LV::at(16 * h + r, 2 * u + 1)) = x1v;
            } else {
              if (!counts) v = (u32x4_t){0, 0, 0, 0};
              *(u32x4_t*)(mine + LV::at(16 * h + r, u)) = v;
            }
          }
        f32x4_t s[2];
#pragma unroll
        for (int h = 0; h < 2; ++h) {
          s[h] = (f32x4_t){0.f, 0.f, 0.f, 0.f};
#pragma unroll
          for (int i = 0; i < kLoads; ++i) {
            const u32x4_t k = now.k[h * kLoads + i];
            if constexpr (MX8) {
              // elements 64 i + 16 g .. + 15: block 2 i + g / 2
              const float sc = cvt_scale(now.ks[h] >> (8 * (2 * i + (lg >> 1))) & 255u);
              s[h] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(bf16_of(k[0], k[1], sc), q[2 * i], s[h],
                                                             0, 0, 0);
              s[h] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(bf16_of(k[2], k[3], sc), q[2 * i + 1], s[h],
                                                             0, 0, 0);
            } else {
              s[h] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(__builtin_bit_cast(bf16x8_t, k), q[i], s[h], 0, 0, 0);
            }
          }
          if (!all) {
#pragma unroll
            for (int e = 0; e < 4; ++e) {
              const int r = 4 * lg + e;
              if (r < (h ? lo1 : lo0) || r >= (h ? hi1 : hi0)) s[h][e] = -INFINITY;
            }
          }
        }
        float top = s[0][0];
#pragma unroll
        for (int h = 0; h < 2; ++h)
#pragma unroll
          for (int e = 0; e < 4; ++e) top = fmaxf(top, s[h][e]);
        top = quarters_max(top) * c;
        // sums relative to a maximum that moves only past 2^8 (as in the prompt's kernel)
        if (__any(top > a.m + 8.f)) {
          const float m = fmaxf(a.m, top), f = m == -INFINITY ? 1.f : exp2_(a.m - m);
          a.m = m;
          a.l *= f;
#pragma unroll
          for (int i = 0; i < D / 16; ++i)
#pragma unroll
            for (int e = 0; e < 4; ++e) a.o[i][e] *= f;
        }
        const float ref = a.m == -INFINITY ? 0.f : a.m;
        float p[8];
#pragma unroll
        for (int e = 0; e < 8; ++e) {
          p[e] = exp2_(fmaf(s[e >> 2][e & 3], c, -ref));
          a.l += p[e];
        }
        // The matrix core's operands are bf16: a weight is the sum of two, its rounding and
        // what that leaves out, rounded, 2^-16 of it off.  (The first alone: outputs 2.4e-3 of
        // the 2-norm off where their own rounding is 1.65e-3.  The second costs 64 sequences of 4096
        // tokens in MX8 114.8 us instead of 113.7, and one of 131072 in bf16 nothing.)
        const u32x4_t hi = pack16(p, (bf16_t*)nullptr);
        float f[8];
        unpack16(hi, f, (bf16_t*)nullptr);
#pragma unroll
        for (int e = 0; e < 8; ++e) p[e] -= f[e];
        const bf16x8_t pw = __builtin_bit_cast(bf16x8_t, hi);
        const bf16x8_t pr = __builtin_bit_cast(bf16x8_t, pack16(p, (bf16_t*)nullptr));
#pragma unroll
        for (int i = 0; i < D / 16; ++i) {
          const bf16x8_t v = LV::col(mine, 16 * i, lane);
          a.o[i] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(v, pw, a.o[i], 0, 0, 0);
          a.o[i] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(v, pr, a.o[i], 0, 0, 0);
        }
      }
      // the four waves' sums, joined through LDS: [wave][query][D + m, l]
      a.l = quarters_sum(a.l);
      __syncthreads();  // (the values' LDS is free)
      float* mem = (float*)smem;
      constexpr int kRow = D + 4;
      {
        float* r = mem + (w * 16 + col) * kRow;
#pragma unroll
        for (int i = 0; i < D / 16; ++i) *(f32x4_t*)(r + 16 * i + 4 * lg) = a.o[i];
        if (lg == 0) {
          r[D] = a.m;
          r[D + 1] = a.l;
        }
      }
      __syncthreads();
      const bool whole = x0 == 0 && x1 == n;
      float* out = g.parts + ((int64_t)blockIdx.x * 2 + (first_run ? 0 : 1)) * 16 * kRow;
      for (int e = threadIdx.x; e < heads * (D / 4); e += 256) {
        const int qi = e / (D / 4), d = e % (D / 4) * 4;
        float m = -INFINITY;
#pragma unroll
        for (int i = 0; i < 4; ++i) m = fmaxf(m, mem[(i * 16 + qi) * kRow + D]);
        const float ref = m == -INFINITY ? 0.f : m;
        f32x4_t o = {0.f, 0.f, 0.f, 0.f};
        float l = 0.f;
#pragma unroll
        for (int i = 0; i < 4; ++i) {
          const float* r = mem + (i * 16 + qi) * kRow;
          const float f = exp2_(r[D] - ref);
          const f32x4_t v = *(const f32x4_t*)(r + d);
#pragma unroll
          for (int y = 0; y < 4; ++y) o[y] += v[y] * f;
          l += r[D + 1] * f;
        }
        if (whole) {
          const float inv = l > 0.f ? 1.f / l : l == 0.f ? 0.f : l;
          const float f[4] = {o[0] * inv, o[1] * inv, o[2] * inv, o[3] * inv};
          const int64_t head = (int64_t)b * g.heads + h0 + qi;
          Vec4<bf16_t>::store((bf16_t*)g.O + head * D + d, f);
          if (g.lse && d == 0) g.lse[head] = l == 0.f ? -INFINITY : m * kLn2 + logf(l);
        } else {
          *(f32x4_t*)(out + qi * kRow + d) = o;
          if (d == 0) {
            out[qi * kRow + D] = m;
            out[qi * kRow + D + 1] = l;
          }
        }
      }
      __syncthreads();  // (the next part's values may overwrite the sums)
      first_run = false;
      at += x1 - x0;
    }
    base += (int64_t)n * g.pairs;
  }
}

// One head's result from sums relative to 2^m: four columns.
__device__ __forceinline__ void store_head(const DecodeArgs& g, int64_t at, int dim, int d, const f32x4_t& o,
                                           float m, float l) {
  const float inv = l > 0.f ? 1.f / l : l == 0.f ? 0.f : l;
  const float f[4] = {o[0] * inv, o[1] * inv, o[2] * inv, o[3] * inv};
  Vec4<bf16_t>::store((bf16_t*)g.O + at * dim + d, f);
  if (g.lse && d == 0) g.lse[at] = l == 0.f ? -INFINITY : m * kLn2 + logf(l);
}
// Adds another part's sums.
__device__ __forceinline__ void join(f32x4_t& o, float& m, float& l, const f32x4_t& v, float pm, float pl) {
  const float now = fmaxf(m, pm), ref = now == -INFINITY ? 0.f : now;
  const float f = exp2_(m - ref), h = exp2_(pm - ref);
  m = now;
  l = l * f + pl * h;
#pragma unroll
  for (int e = 0; e < 4; ++e) o[e] = o[e] * f + v[e] * h;
}

// Joins the parts of one pair of a sequence whose steps lie in more than one
// workgroup's run, in order; writes zeros where there is no token.  Workgroup (x, y): pair
// x, its heads y, y + gridDim.y, ...  Bound by latency, 4 to 5 us, which a second
// launch needs anyway: the lengths' sums, then the parts, which lie in caches.
template <int D>
__global__ __launch_bounds__(256) void join_kernel(const DecodeArgs g) {
  constexpr int kRow = D + 4, kCols = D / 4, kAcross = 256 / kCols;
  __shared__ int64_t part[4];
  __shared__ int64_t found[2];
  __shared__ __align__(16) float mem[kAcross][kRow];
  const Plan plan = plan_of(g, part);
  const int b = blockIdx.x / g.pairs, pair = blockIdx.x % g.pairs;
  const int64_t before = steps_before(g, plan, b, found);
  const int kv = pair / g.tiles, first = pair % g.tiles * 16, heads = min(16, g.group - first);
  const int64_t h0 = (int64_t)b * g.heads + kv * g.group + first;
  const int n = steps_of(span_of(g, b));
  const int d = threadIdx.x % kCols * 4, y = threadIdx.x / kCols;
  if (n == 0) {
    for (int h = y * gridDim.y + blockIdx.y; h < heads; h += kAcross * gridDim.y)
      store_head(g, h0 + h, D, d, (f32x4_t){0.f, 0.f, 0.f, 0.f}, 0.f, 0.f);
    return;
  }
  const int64_t share = share_of(g, plan.total);
  const int64_t s0 = before * g.pairs + (int64_t)pair * n, s1 = s0 + n;
  const int64_t w0 = quotient(s0, share), w1 = quotient(s1 - 1, share);
  if (w0 == w1) return;  // one workgroup had it all
  auto row = [&](int64_t w, int h) {  // a run's first part is part 0
    const int which = w == w0 && w0 * share < s0 ? 1 : 0;
    return g.parts + ((w * 2 + which) * 16 + h) * kRow;
  };
  if (w1 - w0 < 8) {  // few parts: a thread joins four columns of a head
    for (int h = y * gridDim.y + blockIdx.y; h < heads; h += kAcross * gridDim.y) {
      float m = -INFINITY, l = 0.f;
      f32x4_t o = {0.f, 0.f, 0.f, 0.f};
#pragma unroll 2
      for (int64_t w = w0; w <= w1; ++w) {
        const float* r = row(w, h);
        join(o, m, l, *(const f32x4_t*)(r + d), r[D], r[D + 1]);
      }
      store_head(g, h0 + h, D, d, o, m, l);
    }
    return;
  }
  for (int h = blockIdx.y; h < heads; h += gridDim.y) {
    float m = -INFINITY, l = 0.f;
    f32x4_t o = {0.f, 0.f, 0.f, 0.f};
#pragma unroll 4
    for (int64_t w = w0 + y; w <= w1; w += kAcross) {
      const float* r = row(w, h);
      join(o, m, l, *(const f32x4_t*)(r + d), r[D], r[D + 1]);
    }
    *(f32x4_t*)(&mem[y][d]) = o;
    if (d == 0) {
      mem[y][D] = m;
      mem[y][D + 1] = l;
    }
    __syncthreads();
    if (y == 0) {
      for (int i = 1; i < kAcross; ++i) join(o, m, l, *(const f32x4_t*)(&mem[i][d]), mem[i][D], mem[i][D + 1]);
      store_head(g, h0 + h, D, d, o, m, l);
    }
    __syncthreads();
  }
}

}  // namespace

int decode_groups(const DecodeArgs& g) {
  // all resident at once: two workgroups a CU
  const int64_t most = (int64_t)g.seqs * g.pairs * ((g.most + kStep - 1) / kStep);
  return (int)std::max<int64_t>(1, std::min<int64_t>(2 * g.cus, most));
}
int64_t decode_part_floats(const DecodeArgs& g) { return (int64_t)decode_groups(g) * 2 * 16 * (g.dim + 4); }

hipError_t launch_decode(const DecodeArgs& g, hipStream_t s) {
  const int64_t pairs = (int64_t)g.seqs * g.pairs;
  if (pairs > kMostItems / 256) return hipErrorInvalidValue;
  // where pairs are few, a workgroup for each head
  const int64_t y = std::max<int64_t>(1, std::min<int64_t>(std::min(16, g.group), 2 * g.cus / pairs));
  const dim3 grid((unsigned)pairs, (unsigned)y);
  if (g.dim == 64) {
    if (g.ks) decode_kernel<64, true><<<g.groups, 256, 0, s>>>(g);
    else decode_kernel<64, false><<<g.groups, 256, 0, s>>>(g);
    join_kernel<64><<<grid, 256, 0, s>>>(g);
  } else {
    if (g.ks) decode_kernel<128, true><<<g.groups, 256, 0, s>>>(g);
    else decode_kernel<128, false><<<g.groups, 256, 0, s>>>(g);
    join_kernel<128><<<grid, 256, 0, s>>>(g);
  }
  return hipGetLastError();
}

}  // namespace memfine
