// Routing from logits on gfx950: scores, balance bias, expert groups, top-k
// and gates, and the gradient of the gates with respect to the logits.
//
//   p_e  = sigmoid(z_e), or softmax over the token's experts
//   v_e  = p_e + bias_e: the selection's value alone
//   group score = the sum of the group's two largest v; only the experts of
//          the top_groups best groups stay
//   the k largest v, equal ones by the lower id;  gate_j = scale p_j, or
//          scale p_j / sum of the selected p
//
// An expert whose logit is -inf, the lowest finite float or NaN is masked: p = 0,
// v = -inf, chosen only when fewer than k others are left, with gate 0.  +inf
// counts as the largest finite logit.
//
// Sixteen lanes hold a token (lane l: experts l v .. l v + v - 1, v = E / 16
// rounded up), so every reduction over the experts is four DPP steps inside a
// row of 16 lanes and a wave works on four tokens at once.
//
// The forward is bound by vector instructions, which take 95 % of the SIMDs'
// cycles (131072 tokens of 256 logits: 134 MB, 28 us at the copy rate).  Each lane sorts its values once (a network of
// minima and maxima, no ids); a round of the selection then takes the largest
// head of the 16 lists and pops it; the ids come last, all k at once: lane j
// looks its value up among the owning lane's values.  Searching the id and
// clearing it in every round took 71 us instead of 51.  The backward is bound by
// memory (100003 tokens of 160: 128 MB in 33 us).
#include <algorithm>
#include <cfloat>

#include "common.h"
#include "kernels.h"

namespace memfine {
namespace {

constexpr int kTokens = 16;  // tokens per workgroup of 256 threads

// e^x for x <= 0, to choose experts by and for the softmax's sum.  The rounding
// of x log2(e) is a relative error of |x| 2^-24: nothing beside the sum's own
// where e^x counts in it.
__device__ __forceinline__ float exp_neg(float x) {
  return __builtin_amdgcn_exp2f(fmaxf(x, -150.f) * 1.44269502f);
}
// The same for what is handed out, gates and gradients, where an expert far below
// the best counts by itself: what the rounded product x log2(e) lacks, in the
// product and in the constant, multiplies the result as 1 + it (to 2^-22 in all,
// where the product alone is off by 4e-6 at e^-80).
__device__ __forceinline__ float exp_neg_exact(float x) {
  constexpr float kLog2e = 1.44269502f;
  constexpr float kRest = (float)(1.4426950408889634074 - (double)kLog2e);
  x = fmaxf(x, -150.f);
  const float h = x * kLog2e;
  const float rest = fmaf(x, kRest, fmaf(x, kLog2e, -h));
  const float e = __builtin_amdgcn_exp2f(h);
  return fmaf(e, rest * 0.693147181f, e);
}
// sigmoid(z) and 1 - sigmoid(z), both without cancellation; e = e^-|z|, |z| finite.
__device__ __forceinline__ float sigmoid_pair(float z, float e, float* complement) {
  const float r = __builtin_amdgcn_rcpf(1.f + e);
  *complement = z >= 0.f ? e * r : r;
  return z >= 0.f ? r : e * r;
}

// Value of another lane of the row of 16 (kCtrl: a DPP row control).
template <int kCtrl> __device__ __forceinline__ float dpp_f(float v) {
  return __builtin_bit_cast(float, __builtin_amdgcn_update_dpp(0, __builtin_bit_cast(int, v), kCtrl,
                                                               0xf, 0xf, false));
}
template <int kCtrl> __device__ __forceinline__ int dpp_i(int v) {
  return __builtin_amdgcn_update_dpp(0, v, kCtrl, 0xf, 0xf, false);
}
constexpr int kXor1 = 0xb1, kXor2 = 0x4e, kHalfMirror = 0x141, kMirror = 0x140, kRor = 0x120;
// Sum, maximum over the row's 16 lanes, in every lane: after each step the
// lanes that are mirrored onto each other lie in groups with equal values.
__device__ __forceinline__ float row_sum(float v) {
  v += dpp_f<kXor1>(v);
  v += dpp_f<kXor2>(v);
  v += dpp_f<kHalfMirror>(v);
  return v + dpp_f<kMirror>(v);
}
__device__ __forceinline__ float row_max(float v) {
  v = fmaxf(v, dpp_f<kXor1>(v));
  v = fmaxf(v, dpp_f<kXor2>(v));
  v = fmaxf(v, dpp_f<kHalfMirror>(v));
  return fmaxf(v, dpp_f<kMirror>(v));
}
__device__ __forceinline__ uint32_t row_umax(uint32_t v) {
  v = max(v, (uint32_t)dpp_i<kXor1>((int)v));
  v = max(v, (uint32_t)dpp_i<kXor2>((int)v));
  v = max(v, (uint32_t)dpp_i<kHalfMirror>((int)v));
  return max(v, (uint32_t)dpp_i<kMirror>((int)v));
}
// (a, b) with a >= b: the two largest of (a, b) and another lane's pair.
template <int kCtrl> __device__ __forceinline__ void merge_two(float& a, float& b) {
  const float oa = dpp_f<kCtrl>(a), ob = dpp_f<kCtrl>(b);
  b = fmaxf(fminf(a, oa), fmaxf(b, ob));
  a = fmaxf(a, oa);
}
// The lowest lane of this lane's row of 16 where `yes` holds (it holds in one).
__device__ __forceinline__ int first_lane(bool yes, int lane) {
  return __builtin_ctz((uint32_t)(__ballot(yes) >> (lane & 48)) & 0xffffu);
}
// v sorted from the largest on (a merge-exchange network).
template <int V> __device__ __forceinline__ void sort_down(uint32_t (&v)[V]) {
#pragma unroll
  for (int p = 1; p < V; p *= 2)
#pragma unroll
    for (int k = p; k >= 1; k /= 2)
#pragma unroll
      for (int j = k % p; j <= V - 1 - k; j += 2 * k)
#pragma unroll
        for (int i = 0; i < k; ++i)
          if (i + j + k < V && (i + j) / (2 * p) == (i + j + k) / (2 * p)) {
            const uint32_t a = v[i + j], b = v[i + j + k];
            v[i + j] = max(a, b);
            v[i + j + k] = min(a, b);
          }
}
// How many of the lanes l - 1, ..., l - 15 of the row have this lane's (x, n),
// n >= 0; lanes that do not exist have n = -1.
template <int N> __device__ __forceinline__ void count_same(uint32_t x, int n, int& c) {
  const uint32_t ox = (uint32_t)__builtin_amdgcn_update_dpp(0, (int)x, 0x110 + N, 0xf, 0xf, false);
  const int on = __builtin_amdgcn_update_dpp(-1, n, 0x110 + N, 0xf, 0xf, false);
  c += (ox == x && on == n) ? 1 : 0;
  if constexpr (N < 15) count_same<N + 1>(x, n, c);
}

// Values of the selection: what is masked ranks below every number, what is no
// candidate (past E, outside the chosen groups) below that; and their keys,
// integers of the same order (0: no candidate).
constexpr float kMasked = -FLT_MAX, kNone = -INFINITY;
__device__ __forceinline__ uint32_t value_key(float v) {
  const uint32_t u = __float_as_uint(v + 0.f);  // (-0 as +0)
  return v == kNone ? 0u : u ^ ((uint32_t)((int32_t)u >> 31) | 0x80000000u);
}

__device__ __forceinline__ bool unmasked(float z) { return z > -FLT_MAX; }  // false for a NaN

// A lane's v experts (from e0 = l v on) of a row of E floats that starts `row`
// floats into a buffer: 16-, 8- or 4-byte loads, `fill` past the row.
template <int V>
__device__ __forceinline__ void load_share(__amdgpu_buffer_rsrc_t buf, int row, int E, int v, int l,
                                           float fill, float (&z)[V]) {
  constexpr uint32_t kPast = 0x80000000u;  // past the buffer: reads zero
  const int e0 = l * v;
  const uint32_t off = (uint32_t)(row + e0) * 4;
  auto in = [&](int q) { return q < v && e0 + q < E; };
  if (v % 4 == 0 && E % 4 == 0) {
#pragma unroll
    for (int q = 0; q < V; q += 4) {
      const f32x4_t x = __builtin_bit_cast(
          f32x4_t, __builtin_amdgcn_raw_buffer_load_b128(buf, in(q) ? off + 4 * q : kPast, 0, 0));
#pragma unroll
      for (int i = 0; i < 4; ++i) z[q + i] = x[i];
    }
  } else if (v % 2 == 0 && E % 2 == 0) {
#pragma unroll
    for (int q = 0; q < V; q += 2) {
      const f32x2_t x = __builtin_bit_cast(
          f32x2_t, __builtin_amdgcn_raw_buffer_load_b64(buf, in(q) ? off + 4 * q : kPast, 0, 0));
      z[q] = x[0];
      z[q + 1] = x[1];
    }
  } else {
#pragma unroll
    for (int q = 0; q < V; ++q)
      z[q] = __uint_as_float(__builtin_amdgcn_raw_buffer_load_b32(buf, in(q) ? off + 4 * q : kPast, 0, 0));
  }
  if (16 * V != E) {
#pragma unroll
    for (int q = 0; q < V; ++q) z[q] = in(q) ? z[q] : fill;
  }
}
__device__ __forceinline__ __amdgpu_buffer_rsrc_t floats(const float* p, int64_t n) {
  return __builtin_amdgcn_make_buffer_rsrc(const_cast<float*>(p), (short)0, (int32_t)(n * 4),
                                           0x00020000);
}

// The row's softmax statistics: maximum (a finite number) and 1 / sum of e^(z - max); 0 for a
// row without an unmasked expert.
template <int V>
__device__ __forceinline__ void softmax_stats(const float (&z)[V], float& m, float& inv) {
  m = -INFINITY;
#pragma unroll
  for (int q = 0; q < V; ++q) m = fmaxf(m, unmasked(z[q]) ? z[q] : -INFINITY);
  m = row_max(m);
  float s = 0.f;
#pragma unroll
  for (int q = 0; q < V; ++q) s += unmasked(z[q]) ? exp_neg(z[q] - m) : 0.f;
  s = row_sum(s);
  inv = s > 0.f ? 1.f / s : 0.f;
  if (!(m > -INFINITY)) m = 0.f;
}

// A slot's score over a factor that the row's slots share, so that the largest
// is 1/2 or more and scores far below the smallest float keep their ratios:
// softmax e^(z - max), sigmoid e^(min(z, 0) - min(max, 0)) / (1 + e^-|z|); the
// maximum is over the selected logits.  ok: the slot counts; 0 otherwise.
__device__ __forceinline__ float relative_score(int score, float zr, bool ok) {
  const float z = fminf(zr, FLT_MAX);
  const float top = row_max(ok ? z : -INFINITY);
  if (!ok) return 0.f;
  if (score == 0) return exp_neg_exact(z - top);
  return exp_neg_exact(fminf(z, 0.f) - fminf(top, 0.f)) *
         __builtin_amdgcn_rcpf(1.f + exp_neg(-fabsf(z)));
}

// H: the heads of a lane's list that the k rounds can reach (k <= 8: at most 8).
template <int V, int H>
__global__ __launch_bounds__(256) void route_fwd_kernel(const float* __restrict__ logits,
                                                        const float* __restrict__ bias, int64_t T,
                                                        RouteArgs a, int32_t* __restrict__ idx,
                                                        float* __restrict__ gates) {
  // every lane's values; 16-byte aligned rows, spread over the banks
  constexpr int kRow = V + 4;
  __shared__ __attribute__((aligned(16))) uint32_t held[kTokens][16][kRow];
  const int l = threadIdx.x & 15, tok = threadIdx.x >> 4, lane = threadIdx.x & 63;
  const int64_t t = (int64_t)blockIdx.x * kTokens + tok;
  const float* row = logits + min(t, T - 1) * a.E;  // tokens past T repeat the last, unstored
  const int v = a.v, E = a.E;
  float z[V], b[V];
  const int64_t t0 = (int64_t)blockIdx.x * kTokens;
  const int rows = (int)min((int64_t)kTokens, T - t0);
  load_share<V>(floats(logits + t0 * E, rows * E), min(tok, rows - 1) * E, E, v, l, -INFINITY, z);
  if (bias) load_share<V>(floats(bias, E), 0, E, v, l, 0.f, b);
#pragma unroll
  for (int q = 0; q < V; ++q) z[q] = z[q] > FLT_MAX ? FLT_MAX : z[q];
  float m = 0.f, inv = 0.f;
  if (a.score == 0) softmax_stats<V>(z, m, inv);
  float p[V];
  if (a.score == 0) {
#pragma unroll
    for (int q = 0; q < V; ++q) p[q] = exp_neg(z[q] - m) * inv;
  } else {
#pragma unroll
    for (int q = 0; q < V; ++q) {
      float c;
      p[q] = sigmoid_pair(z[q], exp_neg(-fabsf(z[q])), &c);
    }
  }
  if (bias) {
#pragma unroll
    for (int q = 0; q < V; ++q) p[q] += b[q];
  }
#pragma unroll
  for (int q = 0; q < V; ++q) {
    const bool ok = unmasked(z[q]) & (p[q] > kMasked);  // (a NaN of the bias masks too)
    const bool in = (l * v + q < E) & (q < v);
    const float val = ok ? p[q] : kMasked;
    z[q] = in ? val : kNone;
  }
  if (a.groups > 1) {
    const int gs = E / a.groups;  // experts per group
    uint32_t chosen = 0;          // by group
    float s = kNone;              // lane g, or every lane of group g: the group's score
    int id = l;                   // its group
    if (a.lane_groups) {          // a group is the experts of 16 / groups neighbouring lanes
      const int L = 1 << a.group_shift;
      float ga = -INFINITY, gb = -INFINITY;
#pragma unroll
      for (int q = 0; q < V; ++q) {
        gb = fmaxf(gb, fminf(ga, z[q]));
        ga = fmaxf(ga, z[q]);
      }
      if (L > 1) merge_two<kXor1>(ga, gb);
      if (L > 2) merge_two<kXor2>(ga, gb);
      if (L > 4) merge_two<kHalfMirror>(ga, gb);
      s = gs > 1 ? ga + gb : ga;
      id = l >> a.group_shift;
    } else {  // any division: one group after the other
      for (int g = 0; g < a.groups; ++g) {
        float ga = -INFINITY, gb = -INFINITY;
#pragma unroll
        for (int q = 0; q < V; ++q) {
          const int e = l * v + q;
          if (q < v && e >= g * gs && e < (g + 1) * gs) {
            gb = fmaxf(gb, fminf(ga, z[q]));
            ga = fmaxf(ga, z[q]);
          }
        }
        merge_two<kXor1>(ga, gb);
        merge_two<kXor2>(ga, gb);
        merge_two<kHalfMirror>(ga, gb);
        merge_two<kMirror>(ga, gb);
        if (l == g) s = gs > 1 ? ga + gb : ga;
      }
    }
    // a score with a masked expert in it is the lowest (equal ones: the lower group)
    if (id < a.groups) s = s > kMasked * 0.5f ? s : kMasked;
    for (int j = 0; j < a.top_groups; ++j) {
      const float best = row_max(s);
      const int g = first_lane(s == best, lane) >> a.group_shift;  // that lane's group
      chosen |= 1u << g;
      if (id == g) s = kNone;
    }
    if (a.lane_groups) {
      const bool in = (chosen >> id) & 1u;
#pragma unroll
      for (int q = 0; q < V; ++q) {
        const float was = z[q];
        z[q] = in ? was : kNone;
      }
    } else {
#pragma unroll
      for (int q = 0; q < V; ++q) {
        const float was = z[q];
        z[q] = (chosen >> ((l * v + q) / gs & 15)) & 1u ? was : kNone;
      }
    }
  }
  uint32_t key[V];
#pragma unroll
  for (int q = 0; q < V; ++q) key[q] = value_key(z[q]);
#pragma unroll
  for (int q = 0; q < V; q += 4)
    *(u32x4_t*)&held[tok][l][q] = (u32x4_t){key[q], key[q + 1], key[q + 2], key[q + 3]};
  sort_down<V>(key);
  // k rounds: the largest head of the row, of the lowest lane that has it (ids
  // rise with the lane, so equal values come in the order of their ids)
  uint32_t mine = 0;
  int owner = 0;
  for (int j = 0; j < a.k; ++j) {
    const uint32_t best = row_umax(key[0]);
    const int o = first_lane(key[0] == best, lane);
    const bool pop = l == o;
#pragma unroll
    for (int i = 0; i + 1 < H; ++i) {
      const uint32_t next = key[i + 1], now = key[i];
      key[i] = pop ? next : now;
    }
    key[H - 1] = pop ? 0u : key[H - 1];
    if (l == j) {
      mine = best;
      owner = o;
    }
  }
  __syncthreads();
  // slot l's expert: the owner's c-th with that value, c earlier slots having taken it
  const bool slot = l < a.k;
  // (values fall with the lane, so equal ones are neighbours)
  int c = 0;
  const uint32_t before = (uint32_t)__builtin_amdgcn_update_dpp(0, (int)mine, 0x111, 0xf, 0xf, false);
  if (__any(slot && before == mine)) count_same<1>(mine, owner, c);
  uint32_t has = 0;
#pragma unroll
  for (int q = 0; q < V; q += 4) {
    const u32x4_t x = *(const u32x4_t*)&held[tok][owner][q];
#pragma unroll
    for (int i = 0; i < 4; ++i) has |= x[i] == mine ? 1u << (q + i) : 0u;
  }
  for (; __any(slot && c > 0); --c)
    if (c > 0) has &= has - 1;
  const int e = slot ? owner * v + __builtin_ctz(has | 0x80000000u) : 0;
  const float zr = slot ? row[e] : -INFINITY;
  const bool ok = unmasked(zr);
  float g = 0.f, f = a.scale;
  if (a.renorm) {
    g = relative_score(a.score, zr, ok);
    const float sum = row_sum(g);  // 1/2 and more, or no slot counts
    f = sum > 0.f ? a.scale / sum : 0.f;
  } else if (ok) {
    const float zs = fminf(zr, FLT_MAX), e = exp_neg_exact(a.score == 0 ? zs - m : -fabsf(zs));
    float comp;
    g = a.score == 0 ? e * inv : sigmoid_pair(zs, e, &comp);
  }
  if (slot && t < T) {
    idx[t * a.k + l] = e;
    gates[t * a.k + l] = g * f;
  }
}

// Backward: lane j of a token's sixteen computes the gradient of slot j's
// logit; the rows are put together in LDS and written whole, 16 bytes a lane.
// Only the softmax gates without renormalisation reach every logit
// (dz_e = p_e (dp_e - sum p dp)) and read all of them.
template <int V>
__global__ __launch_bounds__(256) void route_bwd_kernel(const float* __restrict__ logits,
                                                        const int32_t* __restrict__ idx,
                                                        const float* __restrict__ dgates,
                                                        int64_t T, RouteArgs a,
                                                        float* __restrict__ dlogits) {
  extern __shared__ f32x4_t rows4[];  // kTokens rows of E
  float* rows = (float*)rows4;
  const int l = threadIdx.x & 15, tok = threadIdx.x >> 4;
  const int64_t t0 = (int64_t)blockIdx.x * kTokens, t = t0 + tok;
  const int64_t tr = min(t, T - 1);
  const int E = a.E;
  const bool dense = a.score == 0 && !a.renorm;
  const float* row = logits + tr * E;
  // slot l; an id outside [0, E) passes no gradient
  int id = l < a.k ? idx[tr * a.k + l] : -1;
  id = id >= 0 && id < E ? id : -1;
  const float zr = id >= 0 ? row[id] : -INFINITY;
  const bool ok = unmasked(zr);  // a masked expert's gate is 0 whatever the logits: no gradient
  const float dg = ok ? dgates[tr * a.k + l] * a.scale : 0.f;
  const float z = ok ? fminf(zr, FLT_MAX) : 0.f;
  float p = 0.f, dz = 0.f;
  if (dense) {
    float s[V], m, inv;
    const int held = (int)min((int64_t)kTokens, T - t0);
    load_share<V>(floats(logits + t0 * E, held * E), min(tok, held - 1) * E, E, a.v, l, -INFINITY, s);
#pragma unroll
    for (int q = 0; q < V; ++q) s[q] = s[q] > FLT_MAX ? FLT_MAX : s[q];
    softmax_stats<V>(s, m, inv);
    p = ok ? exp_neg_exact(z - m) * inv : 0.f;
    dz = p * dg;
    const float c = row_sum(dz);
#pragma unroll
    for (int q = 0; q < V; ++q)
      if (q < a.v && l * a.v + q < E)
        rows[tok * E + l * a.v + q] = unmasked(s[q]) ? -c * (exp_neg_exact(s[q] - m) * inv) : 0.f;
  } else {
    float comp = 1.f;  // sigmoid: 1 - p
    if (a.score != 0) {
      p = sigmoid_pair(z, exp_neg_exact(-fabsf(z)), &comp);
      if (!ok) p = 0.f;
    }
    if (a.renorm) {
      const float r = relative_score(a.score, zr, ok);
      const float sum = row_sum(r);
      const float g = sum > 0.f ? r / sum : 0.f;
      dz = g * comp * (dg - row_sum(g * dg));
    } else {
      dz = dg * p * comp;
    }
    for (int i = threadIdx.x; i < kTokens * E / 4; i += 256) rows4[i] = (f32x4_t){0.f, 0.f, 0.f, 0.f};
  }
  // slots of one token with the same id: the first adds the others' gradients
  bool lead = id >= 0;
  float sum = dz;
  for (int i = 0; i < a.k; ++i) {
    const int oid = __shfl(id, i, 16);
    const float od = __shfl(dz, i, 16);
    if (i != l && oid == id) {
      lead = lead && i > l;
      sum += od;
    }
  }
  __syncthreads();
  if (lead) rows[tok * E + id] += sum;
  __syncthreads();
  const int64_t n = min((int64_t)kTokens, T - t0) * E;
  float* out = dlogits + t0 * E;  // 16-byte aligned: kTokens rows of floats a workgroup
  for (int64_t i = threadIdx.x; i < n / 4; i += 256) ((f32x4_t*)out)[i] = rows4[i];
  if (threadIdx.x < (n & 3)) out[(n & ~3) + threadIdx.x] = rows[(n & ~3) + threadIdx.x];
}

// dlogits [T, E] as the operand rows of the router's gradient products: [T,
// EP] in the storage type, zero past E, and the split-K tables beside them.
template <typename T>
__global__ __launch_bounds__(256) void logit_rows_kernel(const float* __restrict__ dlogits,
                                                         int64_t n, int E, int EP,
                                                         T* __restrict__ D, RouterSplit sp,
                                                         int64_t T_) {
  const int64_t i = blockIdx.x * 256ll + threadIdx.x;
  if (blockIdx.x == 0)
    for (int s = threadIdx.x; s <= sp.S; s += 256) {
      sp.offsets[s] = (int32_t)(s * T_ / sp.S);
      if (s < sp.S) sp.order[s] = s;
    }
  if (i < T_) sp.tok[i] = (int32_t)i;
  if (i >= n) return;
  const int64_t el = i * 4;
  const int64_t t = el / EP;
  const int e = (int)(el - t * EP);  // EP is a multiple of 32
  float f[4];
#pragma unroll
  for (int q = 0; q < 4; ++q) f[q] = e + q < E ? dlogits[t * E + e + q] : 0.f;
  Vec4<T>::store(D + el, f);
}

// Tokens of a launch, 16 lanes each.
constexpr int64_t kMostTokens = kMostItems / 16;

}  // namespace

hipError_t launch_route_fwd(const float* logits, const float* bias, int64_t T, RouteArgs a,
                            int32_t* idx, float* gates, hipStream_t s) {
  if (T == 0) return hipSuccess;
  if (a.E > 256 || a.k > 16 || a.groups > 16) return hipErrorInvalidValue;
  a.v = (a.E + 15) / 16;
  a.lane_groups = a.E % 16 == 0 && 16 % a.groups == 0;
  a.group_shift = a.lane_groups ? __builtin_ctz(16 / a.groups) : 0;
  for (int64_t t0 = 0; t0 < T; t0 += kMostTokens) {
    const int64_t n = std::min(kMostTokens, T - t0);
    const unsigned g = (unsigned)((n + kTokens - 1) / kTokens);
    const float* z = logits + t0 * a.E;
    int32_t* id = idx + t0 * a.k;
    float* out = gates + t0 * a.k;
#define MEMFINE_ROUTE(V_, H_) route_fwd_kernel<V_, H_><<<g, 256, 0, s>>>(z, bias, n, a, id, out)
    if (a.v <= 4) MEMFINE_ROUTE(4, 4);
    else if (a.v <= 8) MEMFINE_ROUTE(8, 8);
    else if (a.k <= 8) MEMFINE_ROUTE(16, 8);
    else MEMFINE_ROUTE(16, 16);
#undef MEMFINE_ROUTE
  }
  return hipGetLastError();
}

hipError_t launch_route_bwd(const float* logits, const int32_t* idx, const float* dgates, int64_t T,
                            RouteArgs a, float* dlogits, hipStream_t s) {
  if (T == 0) return hipSuccess;
  if (a.E > 256 || a.k > 16) return hipErrorInvalidValue;
  a.v = (a.E + 15) / 16;
  const size_t lds = (size_t)kTokens * a.E * 4;
  for (int64_t t0 = 0; t0 < T; t0 += kMostTokens) {
    const int64_t n = std::min(kMostTokens, T - t0);
    const unsigned g = (unsigned)((n + kTokens - 1) / kTokens);
    const float *z = logits + t0 * a.E, *d = dgates + t0 * a.k;
    const int32_t* id = idx + t0 * a.k;
    float* out = dlogits + t0 * a.E;
    if (a.v <= 4) route_bwd_kernel<4><<<g, 256, lds, s>>>(z, id, d, n, a, out);
    else if (a.v <= 8) route_bwd_kernel<8><<<g, 256, lds, s>>>(z, id, d, n, a, out);
    else route_bwd_kernel<16><<<g, 256, lds, s>>>(z, id, d, n, a, out);
  }
  return hipGetLastError();
}

hipError_t launch_logit_rows(int dtype, const float* dlogits, int64_t T, int E, int EP, void* D,
                             const RouterSplit& sp, hipStream_t s) {
  const int64_t n = T * EP / 4;  // EP >= 32: at least T threads
  if (n == 0) return hipSuccess;
  const unsigned blocks = (unsigned)((n + 255) / 256);
  if (dtype == 0)
    logit_rows_kernel<bf16_t><<<blocks, 256, 0, s>>>(dlogits, n, E, EP, (bf16_t*)D, sp, T);
  else
    logit_rows_kernel<float><<<blocks, 256, 0, s>>>(dlogits, n, E, EP, (float*)D, sp, T);
  return hipGetLastError();
}

}  // namespace memfine
