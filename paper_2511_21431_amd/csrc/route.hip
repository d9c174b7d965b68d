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
#include <cfloat>

#include "common.h"
#include "kernels.h"

namespace memfine {
namespace {

constexpr int kTokens = 16;  // tokens per workgroup of 256 threads

// e^x for x <= 0, to about one unit in the last place: the product's rounding
// error is carried into the result (v_exp_f32 of the rounded product alone is
// off by |x| units).
__device__ __forceinline__ float exp_neg(float x) {
  constexpr float kLog2e = 1.44269502f, kLog2eLow = 1.92596303e-8f, kLn2 = 0.693147182f;
  x = fmaxf(x, -150.f);  // e^-150 is 0, and the product below stays finite
  const float t = x * kLog2e;
  const float lo = fmaf(x, kLog2eLow, fmaf(x, kLog2e, -t));
  const float e = __builtin_amdgcn_exp2f(t);
  return fmaf(e, lo * kLn2, e);
}
// sigmoid(z) and 1 - sigmoid(z), both without cancellation; |z| finite.
__device__ __forceinline__ float sigmoid_pair(float z, float* complement) {
  const float e = exp_neg(-fabsf(z));
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
// Rank of this lane's (score, id) among the row's 16 lanes: how many other
// lanes have a larger score, or the same with a lower id.
template <int N> __device__ __forceinline__ void count_better(float s, int id, int& n) {
  const float os = dpp_f<kRor + N>(s);
  const int oid = dpp_i<kRor + N>(id);
  n += (os > s || (os == s && oid < id)) ? 1 : 0;
  if constexpr (N < 15) count_better<N + 1>(s, id, n);
}

// Order-preserving key of a value (0: not a candidate, 1: masked or NaN).
__device__ __forceinline__ uint32_t value_key(float v) {
  const uint32_t u = __float_as_uint(v + 0.f);
  return v != v ? 1u : (u >> 31) ? ~u : u | 0x80000000u;
}

__device__ __forceinline__ bool unmasked(float z) { return z > -FLT_MAX; }  // false for a NaN

// A lane's v experts of a row of E floats: 16-, 8- or 4-byte loads, `fill`
// past the row.
template <int V>
__device__ __forceinline__ void load_share(const float* __restrict__ row, int E, int v, int l,
                                           float fill, float (&z)[V]) {
  const int e0 = l * v;
  if (v % 4 == 0 && E % 4 == 0) {
#pragma unroll
    for (int q = 0; q < V; q += 4) {
      f32x4_t x = {fill, fill, fill, fill};
      if (q < v && e0 + q < E) x = *(const f32x4_t*)(row + e0 + q);
#pragma unroll
      for (int i = 0; i < 4; ++i)
        if (q + i < V) z[q + i] = x[i];
    }
  } else if (v % 2 == 0 && E % 2 == 0) {
#pragma unroll
    for (int q = 0; q < V; q += 2) {
      f32x2_t x = {fill, fill};
      if (q < v && e0 + q < E) x = *(const f32x2_t*)(row + e0 + q);
      z[q] = x[0];
      if (q + 1 < V) z[q + 1] = x[1];
    }
  } else {
#pragma unroll
    for (int q = 0; q < V; ++q) z[q] = q < v && e0 + q < E ? row[e0 + q] : fill;
  }
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

template <int V>
__global__ __launch_bounds__(256) void route_fwd_kernel(const float* __restrict__ logits,
                                                        const float* __restrict__ bias, int64_t T,
                                                        RouteArgs a, int32_t* __restrict__ idx,
                                                        float* __restrict__ gates) {
  __shared__ int32_t won[kTokens][16];
  const int l = threadIdx.x & 15, tok = threadIdx.x >> 4, lane = threadIdx.x & 63;
  const int64_t t = (int64_t)blockIdx.x * kTokens + tok;
  const float* row = logits + min(t, T - 1) * a.E;  // tokens past T repeat the last, unstored
  const int v = a.v, E = a.E;
  float z[V], b[V];
  load_share<V>(row, E, v, l, -INFINITY, z);
  if (bias) load_share<V>(bias, E, v, l, 0.f, b);
#pragma unroll
  for (int q = 0; q < V; ++q) z[q] = z[q] > FLT_MAX ? FLT_MAX : z[q];
  float m = 0.f, inv = 0.f;
  if (a.score == 0) softmax_stats<V>(z, m, inv);
  // values of the selection, -inf where masked, and their keys
  uint32_t key[V];
#pragma unroll
  for (int q = 0; q < V; ++q) {
    float p, c;
    if (a.score == 0) p = exp_neg(z[q] - m) * inv;
    else p = sigmoid_pair(z[q], &c);
    const bool ok = unmasked(z[q]);
    const float val = bias ? p + b[q] : p;
    z[q] = ok && val == val ? val : -INFINITY;
    key[q] = q < v && l * v + q < E ? (ok ? value_key(val) : 1u) : 0u;
  }
  if (a.groups > 1) {
    float ga = -INFINITY, gb = -INFINITY;
    const int gs = E / a.groups;  // experts per group
    bool mine[V];
    if (a.lane_groups) {  // a group is the experts of 16 / groups neighbouring lanes
      const int L = 16 / a.groups;
#pragma unroll
      for (int q = 0; q < V; ++q) {
        gb = fmaxf(gb, fminf(ga, z[q]));
        ga = fmaxf(ga, z[q]);
      }
      if (L > 1) merge_two<kXor1>(ga, gb);
      if (L > 2) merge_two<kXor2>(ga, gb);
      if (L > 4) merge_two<kHalfMirror>(ga, gb);
      float s = gs > 1 ? ga + gb : ga;
      s = s == s ? s : -INFINITY;
      int better = 0;
      count_better<1>(s, l / L, better);
      const bool chosen = better < a.top_groups * L;
#pragma unroll
      for (int q = 0; q < V; ++q) mine[q] = chosen;
    } else {  // any division: one group after the other, lane g keeps group g's score
      float s = -INFINITY;
      for (int g = 0; g < a.groups; ++g) {
        ga = gb = -INFINITY;
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
        float sg = gs > 1 ? ga + gb : ga;
        sg = sg == sg ? sg : -INFINITY;
        if (l == g) s = sg;
      }
      int better = 0;
      count_better<1>(s, l, better);
      const uint64_t all = __ballot(better < a.top_groups && l < a.groups);
      const uint32_t chosen = (uint32_t)(all >> (lane & 48)) & 0xffffu;
#pragma unroll
      for (int q = 0; q < V; ++q) mine[q] = (chosen >> ((l * v + q) / gs & 15)) & 1u;
    }
#pragma unroll
    for (int q = 0; q < V; ++q) key[q] = mine[q] ? key[q] : 0u;
  }
  // k rounds: the row's largest key, the lowest lane that holds it, its first
  // expert with it (ids rise with the lane, then with q)
  for (int j = 0; j < a.k; ++j) {
    uint32_t top = key[0];
#pragma unroll
    for (int q = 1; q < V; ++q) top = max(top, key[q]);
    const uint32_t best = row_umax(top);
    const uint32_t holders = (uint32_t)(__ballot(top == best) >> (lane & 48)) & 0xffffu;
    int first = V;
#pragma unroll
    for (int q = V - 1; q >= 0; --q) first = key[q] == best ? q : first;
    if (l != __builtin_ctz(holders)) first = V;
#pragma unroll
    for (int q = 0; q < V; ++q) key[q] = first == q ? 0u : key[q];
    if (first < V) won[tok][j] = l * v + first;
  }
  __syncthreads();
  const bool slot = l < a.k;
  const int e = slot ? won[tok][l] : 0;
  float p = 0.f;
  if (slot) {
    const float zz = fminf(row[e], FLT_MAX);
    float c;
    if (unmasked(row[e])) p = a.score == 0 ? exp_neg(zz - m) * inv : sigmoid_pair(zz, &c);
  }
  float f = a.scale;
  if (a.renorm) {
    const float sum = row_sum(p);
    f = sum > 0.f ? a.scale / sum : 0.f;
  }
  if (slot && t < T) {
    idx[t * a.k + l] = e;
    gates[t * a.k + l] = p * f;
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
  const float dg = id >= 0 ? dgates[tr * a.k + l] * a.scale : 0.f;
  const float zr = id >= 0 ? row[id] : -INFINITY;
  const bool ok = unmasked(zr);
  const float z = ok ? fminf(zr, FLT_MAX) : 0.f;
  float p = 0.f, dz = 0.f;
  if (dense) {
    float s[V], m, inv;
    load_share<V>(row, E, a.v, l, -INFINITY, s);
#pragma unroll
    for (int q = 0; q < V; ++q) s[q] = s[q] > FLT_MAX ? FLT_MAX : s[q];
    softmax_stats<V>(s, m, inv);
    p = ok ? exp_neg(z - m) * inv : 0.f;
    dz = p * dg;
    const float c = row_sum(dz);
#pragma unroll
    for (int q = 0; q < V; ++q)
      if (q < a.v && l * a.v + q < E)
        rows[tok * E + l * a.v + q] = unmasked(s[q]) ? -c * (exp_neg(s[q] - m) * inv) : 0.f;
  } else {
    float comp = 1.f;
    if (a.score == 0) {
      const float m = row_max(ok ? z : -INFINITY);
      p = ok ? exp_neg(z - m) : 0.f;
    } else {
      p = sigmoid_pair(z, &comp);
      if (!ok) p = 0.f;
    }
    if (a.renorm) {
      const float sum = row_sum(p);
      const float g = sum > 0.f ? p / sum : 0.f;
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

}  // namespace

hipError_t launch_route_fwd(const float* logits, const float* bias, int64_t T, RouteArgs a,
                            int32_t* idx, float* gates, hipStream_t s) {
  if (T == 0) return hipSuccess;
  const int64_t blocks = (T + kTokens - 1) / kTokens;
  if (a.E > 256 || a.k > 16 || a.groups > 16 || blocks > INT32_MAX) return hipErrorInvalidValue;
  a.v = (a.E + 15) / 16;
  a.lane_groups = a.E % 16 == 0 && 16 % a.groups == 0;
  const unsigned g = (unsigned)blocks;
  if (a.v <= 4) route_fwd_kernel<4><<<g, 256, 0, s>>>(logits, bias, T, a, idx, gates);
  else if (a.v <= 8) route_fwd_kernel<8><<<g, 256, 0, s>>>(logits, bias, T, a, idx, gates);
  else route_fwd_kernel<16><<<g, 256, 0, s>>>(logits, bias, T, a, idx, gates);
  return hipGetLastError();
}

hipError_t launch_route_bwd(const float* logits, const int32_t* idx, const float* dgates, int64_t T,
                            RouteArgs a, float* dlogits, hipStream_t s) {
  if (T == 0) return hipSuccess;
  const int64_t blocks = (T + kTokens - 1) / kTokens;
  if (a.E > 256 || a.k > 16 || blocks > INT32_MAX) return hipErrorInvalidValue;
  a.v = (a.E + 15) / 16;
  const unsigned g = (unsigned)blocks;
  const size_t lds = (size_t)kTokens * a.E * 4;
  if (a.v <= 4) route_bwd_kernel<4><<<g, 256, lds, s>>>(logits, idx, dgates, T, a, dlogits);
  else if (a.v <= 8) route_bwd_kernel<8><<<g, 256, lds, s>>>(logits, idx, dgates, T, a, dlogits);
  else route_bwd_kernel<16><<<g, 256, lds, s>>>(logits, idx, dgates, T, a, dlogits);
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
