// Attention over packed sequences on gfx950, forward and backward.
//
//   s_ij = scale q_i . k_j over the tokens j that i sees (j <= i when causal; j >
//   i - window where there is one);  lse_i = log sum_j exp(s_ij)
//   p_ij = exp(s_ij - lse_i);   o_i = sum_j p_ij v_j
//   delta_i = do_i . o_i;   ds_ij = scale p_ij (do_i . v_j - delta_i)
//   dv_j = sum_i p_ij do_i;   dq_i = sum_j ds_ij k_j;   dk_j = sum_i ds_ij q_i
//   (dk and dv over the queries of every head that shares the key-value head)
//
// All products run on the matrix cores in blocks of 32 x 32 (v_mfma_f32_32x32x16
// _bf16, or _32x32x2_f32).  A wave owns 32 columns of the transposed scores and
// forms them from rows of the other operand in LDS, as rows: the accumulator
// then holds, in each lane, scores of one column alone, so that a row's maximum
// and sum need one exchange between the wave's halves, and its registers are,
// rounded, the operand of the second product as they stand: which of the 16
// values of a reduction step a register holds is the accumulator's choice, and
// the other operand, read from LDS with a transposing load, follows it.
//
// Bound by the matrix cores where sequences are long, and by the clock (1.7 to 1.9 GHz
// while the long calls of heads of 128 run, 2.4 in kernels that only move data); next to
// them every score costs vector instructions (exponent, sum, rounding), 35 to 60 % of the
// SIMDs' cycles, which only another wave's products hide: two or more waves a SIMD (fp32 with
// heads of 128 has one, for its registers).  Short sequences
// are bound by a workgroup's start (offsets, queries, first tile: about 4 us) and end.
#include <algorithm>
#include <cmath>
#include <type_traits>

#include "common.h"
#include "kernels.h"

namespace memfine {
namespace {

constexpr float kLog2e = 1.4426950408889634f, kLn2 = 0.6931471805599453f;

typedef short s16x4_t __attribute__((ext_vector_type(4)));
typedef __attribute__((address_space(3))) void lds_void;
typedef __attribute__((address_space(3))) s16x4_t lds_s16x4;

__device__ __forceinline__ float exp2_(float x) { return __builtin_amdgcn_exp2f(x); }

// The waits before a tile's barrier: this wave's copies have landed and its reads
// of the other stage have returned.  (A bare s_barrier: __syncthreads() adds a fence.)
__device__ __forceinline__ void stage_barrier() {
  __builtin_amdgcn_s_waitcnt(0 | (7 << 4) | (0 << 8) | (0 << 14));
  asm volatile("" ::: "memory");
  __builtin_amdgcn_s_barrier();
  asm volatile("" ::: "memory");
}

// The larger and the sum of a lane's value and that of the lane 32 apart.
__device__ __forceinline__ float halves_max(float v) {
  const u32x2_t r = __builtin_bit_cast(
      u32x2_t, __builtin_amdgcn_permlane32_swap(__float_as_uint(v), __float_as_uint(v), false, false));
  return fmaxf(__uint_as_float(r[0]), __uint_as_float(r[1]));
}
__device__ __forceinline__ float halves_sum(float v) {
  const u32x2_t r = __builtin_bit_cast(
      u32x2_t, __builtin_amdgcn_permlane32_swap(__float_as_uint(v), __float_as_uint(v), false, false));
  return __uint_as_float(r[0]) + __uint_as_float(r[1]);
}

// One reduction step of the 32 x 32 products: kStep values, of which each half of
// the wave holds half, 16 bytes a lane.
template <typename T> struct Mma;
template <> struct Mma<bf16_t> {
  static constexpr int kStep = 16;
  typedef bf16x8_t Frag;
  __device__ __forceinline__ static void mma(const Frag& a, const Frag& b, f32x16_t& c) {
    c = __builtin_amdgcn_mfma_f32_32x32x16_bf16(a, b, c, 0, 0, 0);
  }
  // accumulators 8 j .. 8 j + 7, rounded: rows 16 j + 8 (i / 4) + 4 hh + i % 4 of the block
  __device__ __forceinline__ static Frag of(const f32x16_t& c, int j) {
    u32x4_t v;
#pragma unroll
    for (int i = 0; i < 4; ++i) v[i] = pack_bf16x2(c[8 * j + 2 * i], c[8 * j + 2 * i + 1]);
    return __builtin_bit_cast(Frag, v);
  }
};
template <> struct Mma<float> {
  static constexpr int kStep = 8;
  typedef f32x4_t Frag;
  __device__ __forceinline__ static void mma(const Frag& a, const Frag& b, f32x16_t& c) {
#pragma unroll
    for (int s = 0; s < 4; ++s) c = __builtin_amdgcn_mfma_f32_32x32x2f32(a[s], b[s], c, 0, 0, 0);
  }
  // accumulators 4 j .. 4 j + 3: rows 8 j + 4 hh + i of the block
  __device__ __forceinline__ static Frag of(const f32x16_t& c, int j) {
    return (Frag){c[4 * j], c[4 * j + 1], c[4 * j + 2], c[4 * j + 3]};
  }
};
template <typename T> using Frag = typename Mma<T>::Frag;
// Row of accumulator i of a block.
__device__ __forceinline__ int acc_row(int i, int hh) { return 8 * (i >> 2) + 4 * hh + (i & 3); }

__device__ __forceinline__ void zero(f32x16_t& c) {
#pragma unroll
  for (int i = 0; i < 16; ++i) c[i] = 0.f;
}

// ------------------------------------------------------------------- tiles
// kRows rows of D elements in LDS.  16-byte unit u of a row sits at unit u ^
// swizzle(row): 16 consecutive rows' reads of one unit, and the reads of four
// (bf16) consecutive rows x 32 columns by a transposing load, or of 32 columns of rows 4
// apart (fp32), then fall on distinct banks.
template <typename T, int D, int R = sizeof(T) == 2 ? 64 : 32> struct Tile {
  static constexpr int ES = sizeof(T), kPitch = D * ES, kUnits = kPitch / 16;
  static constexpr int kRows = R, kBytes = kRows * kPitch;
  static constexpr int kBlocks = kRows / 32;           // blocks of 32 rows
  static constexpr int kSteps = D / Mma<T>::kStep;     // reduction steps along a row
  static constexpr int kDown = 32 / Mma<T>::kStep;     // reduction steps down a block of rows
  typedef typename Mma<T>::Frag F;

  __device__ __forceinline__ static int swizzle(int row) {
    if constexpr (ES == 4) return (row & 3) | (row & 4) << 1 | (row & 8) >> 1;
    else if constexpr (kUnits == 16) return (row & 3) << 2 | ((row >> 2) & 3);
    else return (row & 2) << 1 | ((row >> 2) & 3);
  }
  // What a lane's addresses begin with: further steps along a row and further columns are
  // other units, an exclusive or; 16 rows on, the swizzle is the same.
  struct At {
    int row, col;
  };
  __device__ __forceinline__ static At at(int lane) {
    const int r = lane & 31;
    At x;
    x.row = r * kPitch + (((lane >> 5) ^ swizzle(r)) << 4);
    if constexpr (ES == 2) {
      // lane j of each 16 supplies 4 columns of row j / 4 and gets 4 rows of column j
      const int j = lane & 15, G = lane >> 4, q = (G >> 1) * 4 + (j >> 2);
      x.col = q * kPitch + ((((G & 1) * 2 + ((j >> 1) & 1)) ^ swizzle(q)) << 4) + ((j & 1) << 3);
    } else {
      x.col = lane;
    }
    return x;
  }
  // operand rows row0 .. row0 + 31, step ks of D
  __device__ __forceinline__ static F row(const char* __restrict__ lds, int row0, int ks, const At& x) {
    return *(const F*)(lds + row0 * kPitch + (x.row ^ (ks << 5)));
  }
  // the transposed operand: its 32 rows are columns col0 .. col0 + 31, reduced over
  // step kk of the tile's rows, in the order in which Mma::of holds them
  __device__ __forceinline__ static F col(const char* __restrict__ lds, int col0, int kk, const At& x) {
    if constexpr (ES == 2) {
      const int c = x.col ^ (col0 << 1);
      const s16x4_t lo = __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds_s16x4*)(lds + kk * 16 * kPitch + c));
      const s16x4_t hi =  // (8 rows on)
          __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds_s16x4*)(lds + (kk * 16 + 8) * kPitch + (c ^ 32)));
      return __builtin_bit_cast(F, __builtin_shufflevector(lo, hi, 0, 1, 2, 3, 4, 5, 6, 7));
    } else {
      F f;
      const int lane = x.col, b = (col0 + (lane & 31)) * 4;
#pragma unroll
      for (int s = 0; s < 4; ++s) {
        const int r = kk * 8 + (lane >> 5) * 4 + s;
        f[s] = *(const float*)(lds + r * kPitch + (((b >> 4) ^ swizzle(r)) << 4) + (b & 15));
      }
      return f;
    }
  }
};

__device__ __forceinline__ __amdgpu_buffer_rsrc_t rsrc_of(const void* base, uint32_t bytes) {
  return __builtin_amdgcn_make_buffer_rsrc(const_cast<void*>(base), (short)0, (int32_t)bytes,
                                           0x00020000);
}
// `rows` rows of D elements, ld elements apart, from base on; what lies past
// them reads zero.  (The rows of one tile: below 2^31 bytes.)
template <typename T, int D>
__device__ __forceinline__ __amdgpu_buffer_rsrc_t rows_rsrc(const T* base, int64_t ld, int rows) {
  return rsrc_of(base, rows > 0 ? (uint32_t)((rows - 1) * ld + D) * (uint32_t)sizeof(T) : 0u);
}

// The copy of a tile into LDS by NW waves, straight from memory.
template <typename T, int D, int NW, class L = Tile<T, D>> struct Copy {
  static constexpr int kPer = 1024 / L::kPitch;               // rows an instruction
  static constexpr int kCount = L::kBytes / 1024 / NW;        // instructions a wave
  static_assert(kCount * NW * 1024 == L::kBytes, "a tile is split evenly over the waves");
  static constexpr int kApart = kPer * NW;                    // rows between a wave's instructions
  static constexpr int kKinds = kApart % 16 ? 2 : 1;          // (the swizzle repeats every 16 rows)
  static_assert(kApart * kKinds % 16 == 0 || kCount <= kKinds, "rows of an instruction");
  uint32_t voff[kKinds];  // from the instruction's first row on
  __device__ __forceinline__ void init(int64_t ld, int wave, int lane) {
#pragma unroll
    for (int i = 0; i < kKinds; ++i) {
      const int r = wave * kPer + lane / L::kUnits;
      voff[i] = (uint32_t)(r * ld) * L::ES + (((lane % L::kUnits) ^ L::swizzle(r + i * kApart)) << 4);
    }
  }
  // rows from base on, `rows` of them there
  __device__ __forceinline__ void issue(const T* base, int64_t ld, int rows, char* lds,
                                        int wave) const {
#pragma unroll
    for (int i = 0; i < kCount; ++i)
      __builtin_amdgcn_raw_ptr_buffer_load_lds(
          rows_rsrc<T, D>(base + i * kApart * ld, ld, min(rows - i * kApart, kApart)),
          (lds_void*)(lds + (i * NW + wave) * 1024), 16, voff[i % kKinds], 0, 0, 0);
  }
};

// A wave's 32 rows as an operand that stays in registers.
template <typename T, int D, int N>
__device__ __forceinline__ void load_rows(Frag<T> (&f)[N], const T* base, int64_t ld,
                                          int rows, int lane) {
  const __amdgpu_buffer_rsrc_t rs = rows_rsrc<T, D>(base, ld, rows);
  const uint32_t at = (uint32_t)((lane & 31) * ld) * (uint32_t)sizeof(T) + (lane >> 5) * 16;
#pragma unroll
  for (int k = 0; k < N; ++k)
    f[k] = __builtin_bit_cast(Frag<T>, __builtin_amdgcn_raw_buffer_load_b128(rs, at + k * 32, 0, 0));
}

// Transposed accumulators of 32 rows (a lane: row lane % 32), as rows of out.  They go
// through the wave's own 32 rows of LDS, so that whole rows are stored (straight from the
// accumulators a store writes 8 bytes of each of 64 lines: 8192 rows of 32 heads 27 us).
template <typename T, int D>
__device__ __forceinline__ void store_rows(const f32x16_t (&c)[D / 32], float scale, T* out, int64_t ld,
                                           int rows, char* lds, int lane) {
  constexpr int kPitch = D * (int)sizeof(T), kUnits = kPitch / 16, kVec = Elem<T>::kVec;
  const int r = lane & 31, hh = lane >> 5;
#pragma unroll
  for (int b = 0; b < D / 32; ++b)
#pragma unroll
    for (int g = 0; g < 4; ++g) {
      const float f[4] = {c[b][4 * g] * scale, c[b][4 * g + 1] * scale, c[b][4 * g + 2] * scale,
                          c[b][4 * g + 3] * scale};
      const int at = (b * 32 + g * 8 + hh * 4) * (int)sizeof(T);
      Vec4<T>::store((T*)(lds + r * kPitch + (((at >> 4) ^ (r & 15) % kUnits) << 4) + (at & 15)), f);
    }
#pragma unroll
  for (int i = 0; i < kUnits / 2; ++i) {
    const int row = i * (64 / kUnits) + lane / kUnits, u = lane % kUnits;
    const u32x4_t v = *(const u32x4_t*)(lds + row * kPitch + ((u ^ (row & 15) % kUnits) << 4));
    if (row < rows) *(u32x4_t*)(out + row * ld + u * kVec) = v;
  }
}

// Accumulators in LDS as a wave's lanes hold them, and added up: o mf + theirs of.
template <int D>
__device__ __forceinline__ void put_lanes(float* to, const f32x16_t (&o)[D / 32], int lane) {
#pragma unroll
  for (int b = 0; b < D / 32; ++b)
#pragma unroll
    for (int e = 0; e < 16; ++e) to[(b * 16 + e) * 64 + lane] = o[b][e];
}
template <int D>
__device__ __forceinline__ void add_lanes(const float* from, f32x16_t (&o)[D / 32], float mf, float of,
                                          int lane) {
#pragma unroll
  for (int b = 0; b < D / 32; ++b)
#pragma unroll
    for (int e = 0; e < 16; ++e) o[b][e] = o[b][e] * mf + from[(b * 16 + e) * 64 + lane] * of;
}

// ------------------------------------------------------------- work to do
// Block b of rows of the packed sequences, each cut into blocks of R.
struct Part {
  int begin, n;  // the sequence's first row and its length
  int block;     // of the sequence
};
// Sum over the lanes up to this one, by DPP: row shifts, then each row's last lane to the next.
template <int kCtrl, int kRows> __device__ __forceinline__ int add_dpp(int v) {
  return v + __builtin_amdgcn_update_dpp(0, v, kCtrl, kRows, 0xf, false);
}
__device__ __forceinline__ int wave_scan(int v) {
  v = add_dpp<0x111, 0xf>(v);  // row_shr 1, 2, 4, 8
  v = add_dpp<0x112, 0xf>(v);
  v = add_dpp<0x114, 0xf>(v);
  v = add_dpp<0x118, 0xf>(v);
  v = add_dpp<0x142, 0xa>(v);  // row_bcast 15 into rows 1 and 3
  return add_dpp<0x143, 0xc>(v);  // row_bcast 31 into rows 2 and 3
}
// Every wave looks for itself: its lanes add up the blocks of a 64th of the
// sequences each, and the search goes on in the one that holds block b.  (Offsets
// are cut to [0, T], so that nothing outside is touched whatever they are.)
__device__ __forceinline__ bool locate(const int32_t* __restrict__ offsets, int seqs, int T, int R, int b,
                                       Part& p) {
  const int lane = threadIdx.x & 63;
  int s0 = 0, count = seqs;
  while (count > 64) {
    const int per = (count + 63) / 64;
    const int first = s0 + lane * per, last = min(first + per, s0 + count);
    int n = 0;
    if (first < last) {
      int hi = min(max(offsets[first], 0), T);
      for (int s = first; s < last; ++s) {
        const int lo = hi;
        hi = min(max(offsets[s + 1], 0), T);
        n += hi > lo ? (hi - lo + R - 1) / R : 0;
      }
    }
    const int inc = wave_scan(n);
    const uint64_t past = __ballot(inc > b);
    if (past == 0) return false;
    const int w = __builtin_ctzll(past);
    b -= __builtin_amdgcn_readlane(inc - n, w);
    count = min(per, s0 + count - (s0 + w * per));
    s0 += w * per;
  }
  const int at = s0 + min(lane, count - 1);
  int lo = offsets[at], hi = offsets[at + 1];
  lo = min(max(lo, 0), T);
  hi = min(max(hi, 0), T);
  const int n = lane < count && hi > lo ? (hi - lo + R - 1) / R : 0;
  const int inc = wave_scan(n);
  const uint64_t past = __ballot(inc > b);
  if (past == 0) return false;
  const int w = __builtin_ctzll(past);
  p.begin = __builtin_amdgcn_readlane(lo, w);
  p.n = __builtin_amdgcn_readlane(hi, w) - p.begin;
  p.block = b - __builtin_amdgcn_readlane(inc - n, w);
  return true;
}
// Head and block of a workgroup.  All heads advance together through the blocks of the whole
// batch, in falling order with `down`: under a causal mask each sequence's longest come
// first, and the shortest of the first sequence even out the end (the longest of a first
// sequence that is longer than the others come late).  Workgroups go to the 8 XCDs in turn; with a multiple of 8 heads each
// XCD has an eighth of them, neighbours, which share keys and values in its L2.
__device__ __forceinline__ void work_item(int blocks, int heads, bool down, int& head, int& b) {
  const int id = blockIdx.x;
  if (heads % 8 == 0) {
    const int i = id >> 3, per = heads >> 3;
    head = (id & 7) * per + i % per;
    b = i / per;
  } else {
    head = id % heads;
    b = id / heads;
  }
  if (down) b = blocks - 1 - b;
}

// Which scores of a lane's own token count.
struct Seen {
  int lo, hi;  // tokens lo .. hi of the sequence
};
__device__ __forceinline__ Seen keys_of(const AttnArgs& g, int i, int n) {
  return {g.window > 0 ? i - g.window + 1 : 0, g.causal ? min(i, n - 1) : n - 1};
}
__device__ __forceinline__ Seen queries_of(const AttnArgs& g, int j, int n) {
  return {g.causal ? j : 0, g.window > 0 ? min(n - 1, j + min(g.window, n) - 1) : n - 1};
}
// Whether a wave's 32 own tokens from i0 on see all `rows` other tokens from r0 on.
__device__ __forceinline__ bool see_all(const Seen& first, const Seen& last, int r0, int rows) {
  return r0 >= max(first.lo, last.lo) && r0 + rows - 1 <= min(first.hi, last.hi);
}
// Scores of a block of rows from r0 on that do not count become v: one bit a row, two
// instructions a score.
__device__ __forceinline__ void hide(f32x16_t& c, const Seen& s, int r0, int hh, float v) {
  const int lo = s.lo - r0 - 4 * hh, hi = s.hi - r0 - 4 * hh;
  const uint32_t to = hi < 0 ? 0u : hi >= 31 ? ~0u : (2u << hi) - 1u;
  const uint32_t from = lo <= 0 ? ~0u : lo >= 32 ? 0u : ~0u << lo;
  const uint32_t bits = from & to;
#pragma unroll
  for (int i = 0; i < 16; ++i) {
    const uint32_t m = (uint32_t)((int32_t)(bits << (31 - acc_row(i, 0))) >> 31);
    c[i] = __uint_as_float((__float_as_uint(c[i]) & m) | (__float_as_uint(v) & ~m));
  }
}

// ----------------------------------------------------------------- forward
// NW waves of 32 queries each, which share the tiles of keys and values in LDS: heads of a
// group, where there are groups, for the same queries (under a causal mask they
// then need the same tiles), the rest further queries.  KS = 4, for so few queries that most
// CUs would have none: four waves take the same queries and a quarter of each tile's keys,
// of which there are twice as many; what they have is joined at the end, in order.
// D = 128: tiles of 32 keys in two stages, so that three workgroups of four waves share a CU:
// one starts or ends while others multiply.  Against tiles of 64, of which two fit, in
// workgroups of four waves or, for long sequences, of eight: 8192 tokens of 32 heads in 8
// groups, in sequences of 256 43 us against 47, of 668 66 and 71, one 515 and 514; with a window
// of 512 82 and 98; 4096 tokens of 128 heads 549 and 575 (in other runs, at other clocks, 560 to
// 620: 0.9 to 1.0 PFLOP/s).  D = 64: tiles of 64
// keys, of which four fit: 8 sequences of 1024 tokens, 32 heads 56 us against 57.5 with tiles
// of 32, two of 2048, 64 heads, not causal 146 and 160, but one of 8192, 16 heads 177 and 171.
// (Two halves of a workgroup that multiply and exponentiate in turns, a barrier
// between, were 2 % slower, 11 for heads of 64.)
template <typename T, int D, int NW, int KS>
__global__ __launch_bounds__(64 * NW, sizeof(T) == 4 || KS > 1 ? 1 : D == 128 ? 3 : 4)
void attn_fwd_kernel(const AttnArgs g, int blocks) {
  typedef Tile<T, D, KS != 1 ? 32 * KS : D == 64 ? Tile<T, D>::kRows : 32> L;
  constexpr int kOwn = L::kBlocks / KS;  // blocks of a tile that a wave takes
  typedef Mma<T> M;
  // (joined waves store through LDS that no other wave's sums are in)
  constexpr int kOutPitch = KS == 1 ? L::kPitch : (D / 2 + 2) * 8;
  constexpr int kNeed = 4 * L::kBytes, kSums = KS == 1 ? 0 : NW * (D / 2 + 2) * 256;
  __shared__ __align__(1024) char smem[kNeed > kSums ? kNeed : kSums];
  const int lane = threadIdx.x & 63, w = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int hh = lane >> 5;
  const typename L::At lds_at = L::at(lane);
  int head, b;
  Part p;
  // 2^share waves take the same queries for as many heads
  const int block = 32 * NW / KS >> g.share;
  work_item(blocks, g.heads >> g.share, g.causal, head, b);
  if (!locate(g.offsets, g.seqs, (int)g.T, block, b, p)) return;
  const int wq = w / KS, k0 = w % KS * kOwn;  // whose queries, first block of the tiles
  head = (head << g.share) + (wq & ((1 << g.share) - 1));
  const int kv = head / (g.heads / g.kv_heads);
  const int q0 = p.block * block, rows = min(block, p.n - q0);
  const int i0 = q0 + 32 * (wq >> g.share), mine = min(32, p.n - i0);
  const T* K = (const T*)g.K + p.begin * g.ldk + kv * D;
  const T* V = (const T*)g.V + p.begin * g.ldv + kv * D;

  // the tiles that the workgroup needs, and those that this wave does
  const Seen wg_first = keys_of(g, q0, p.n), wg_last = keys_of(g, q0 + rows - 1, p.n);
  const int t0 = max(wg_first.lo, 0) / L::kRows, t1 = wg_last.hi / L::kRows + 1;
  const Seen first = keys_of(g, i0, p.n), last = keys_of(g, i0 + 31, p.n);
  const Seen own = keys_of(g, i0 + (lane & 31), p.n);

  Copy<T, D, NW, L> ck, cv;
  ck.init(g.ldk, w, lane);
  cv.init(g.ldv, w, lane);
  auto issue = [&](int t, char* st) {
    const int64_t r = (int64_t)t * L::kRows;
    ck.issue(K + r * g.ldk, g.ldk, p.n - (int)r, st, w);
    cv.issue(V + r * g.ldv, g.ldv, p.n - (int)r, st + L::kBytes, w);
  };
  issue(t0, smem);
  Frag<T> q[L::kSteps];
  load_rows<T, D>(q, (const T*)g.Q + (p.begin + i0) * g.ldq + head * D, g.ldq, mine, lane);

  // (in base 2: a score's factor and, in the gradient, lse are rounded once more than for a
  // natural exponent, 2^-24 of each, beside the D roundings of the score's own sum)
  const float c = g.scale * kLog2e;
  f32x16_t o[D / 32];
#pragma unroll
  for (int i = 0; i < D / 32; ++i) zero(o[i]);
  float m = -INFINITY, l = 0.f;  // (l: of this half's tokens)
  // (the stage a constant: its addresses are then offsets in the reads)
  auto tile = [&](int t, auto stage) {
    constexpr int kAt = decltype(stage)::value * 2 * L::kBytes;
    stage_barrier();
    if (t + 1 < t1) issue(t + 1, smem + (2 * L::kBytes - kAt));
    const int r0 = t * L::kRows + 32 * k0;  // of the wave's own blocks
    if (mine <= 0 || r0 > last.hi || r0 + 32 * kOwn <= first.lo) return;
    const char* ks = smem + kAt;
    const char* vs = ks + L::kBytes;
    f32x16_t s[kOwn];
#pragma unroll
    for (int i = 0; i < kOwn; ++i) zero(s[i]);
#pragma unroll
    for (int k = 0; k < L::kSteps; ++k)
#pragma unroll
      for (int i = 0; i < kOwn; ++i) M::mma(L::row(ks, 32 * (k0 + i), k, lds_at), q[k], s[i]);
    if (!see_all(first, last, r0, 32 * kOwn)) {
#pragma unroll
      for (int i = 0; i < kOwn; ++i) hide(s[i], own, r0 + 32 * i, hh, -INFINITY);
    }
    float top = s[0][0];
#pragma unroll
    for (int i = 0; i < kOwn; ++i)
#pragma unroll
      for (int e = 0; e < 16; ++e) top = fmaxf(top, s[i][e]);
    top = halves_max(top) * c;
    // The sums are kept relative to 2^m, m a maximum seen so far: it moves, and they are
    // multiplied, only where a row's maximum has passed it by more than 8 (weights of up to
    // 2^8 are as exact).
    if (__any(top > m + 8.f)) {
      const float now = fmaxf(m, top);
      const float f = now == -INFINITY ? 1.f : exp2_(m - now);
      m = now;
      l *= f;
#pragma unroll
      for (int i = 0; i < D / 32; ++i)
#pragma unroll
        for (int e = 0; e < 16; ++e) o[i][e] *= f;
    }
    const float ref = m == -INFINITY ? 0.f : m;  // (a row that sees nothing yet)
#pragma unroll
    for (int i = 0; i < kOwn; ++i)
#pragma unroll
      for (int e = 0; e < 16; ++e) {
        s[i][e] = exp2_(fmaf(s[i][e], c, -ref));
        l += s[i][e];
      }
#pragma unroll
    for (int i = 0; i < kOwn; ++i)
#pragma unroll
      for (int j = 0; j < L::kDown; ++j) {
        // the weights are rounded to the values' type, the matrix core's operand (their
        // sum is not): half a step of bf16 each, with which outputs are 2.1e-3 of the
        // 2-norm off where their own rounding is 1.6e-3.  A second product with what the rounding
        // leaves out would be half as many again, and the matrix cores are the bound.
        const Frag<T> f = M::of(s[i], j);
#pragma unroll
        for (int d = 0; d < D / 32; ++d) M::mma(L::col(vs, 32 * d, (k0 + i) * L::kDown + j, lds_at), f, o[d]);
      }
  };
  for (int t = t0; t < t1; t += 2) {
    tile(t, std::integral_constant<int, 0>());
    if (t + 1 < t1) tile(t + 1, std::integral_constant<int, 1>());
  }
  stage_barrier();  // (all tiles are used: their LDS takes the results)
  if constexpr (KS > 1) {
    // the lanes of the four waves hold the same queries and columns
    float* mem = (float*)smem;
    constexpr int kEach = (D / 2 + 2) * 64;
    if (w % KS) {
      put_lanes<D>(mem + w * kEach, o, lane);
      mem[w * kEach + D / 2 * 64 + lane] = m;
      mem[w * kEach + (D / 2 + 1) * 64 + lane] = l;
    }
    stage_barrier();
    if (w % KS) return;
#pragma unroll 1
    for (int y = 1; y < KS; ++y) {
      const float* from = mem + (w + y) * kEach;
      const float om = from[D / 2 * 64 + lane], ol = from[(D / 2 + 1) * 64 + lane];
      const float now = fmaxf(m, om), at = now == -INFINITY ? 0.f : now;
      const float mf = exp2_(m - at), of = exp2_(om - at);
      m = now;
      l = l * mf + ol * of;
      add_lanes<D>(from, o, mf, of, lane);
    }
  }
  if (mine <= 0) return;
  l = halves_sum(l);
  store_rows<T, D>(o, l > 0.f ? 1.f / l : l == 0.f ? 0.f : l,
                   (T*)g.out + ((p.begin + i0) * (int64_t)g.heads + head) * D, (int64_t)g.heads * D, mine,
                   smem + w * 32 * kOutPitch, lane);
  if (g.lse && lane < mine)
    g.lse[head * g.T + p.begin + i0 + lane] = l == 0.f ? -INFINITY : m * kLn2 + logf(l);
}

// ---------------------------------------------------------------- backward
// Two kernels, each of which forms the scores: 7 products where 5 would do with dq added up
// in memory by atomics, whose order, and with it the result, would change from call to call.
//
// dq (shared out as in the forward), and their log2 of the weights' sum and delta for the
// kernel below.  A block's ds is all that is held between its products, so that queries,
// dO and dq stay in registers; four waves a workgroup, also for long sequences: 4096 tokens
// of 64 heads in 8 groups, causal, 372 us, with eight waves 389 (the shortest of a run; its
// median is 390 to 400); 6011 tokens of 16 heads of 64 in 9 sequences 34 us.  The first runs at
// 1.0 PFLOP/s, its matrix cores busy for 61 %.
template <typename T, int D, int NW, int KS>
__global__ __launch_bounds__(64 * NW, sizeof(T) == 2 && NW == 4 ? 2 : 1)
void attn_dq_kernel(const AttnArgs g, int blocks) {
  typedef Tile<T, D, KS == 1 ? Tile<T, D>::kRows : 32 * KS> L;
  constexpr int kOwn = L::kBlocks / KS;  // blocks of a tile that a wave takes
  typedef Mma<T> M;
  // (joined waves store through LDS that no other wave's sums are in)
  constexpr int kOutPitch = KS == 1 ? L::kPitch : (D / 2 + 2) * 8;
  constexpr int kNeed = 4 * L::kBytes, kSums = KS == 1 ? 0 : NW * (D / 2 + 2) * 256;
  __shared__ __align__(1024) char smem[kNeed > kSums ? kNeed : kSums];
  const int lane = threadIdx.x & 63, w = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int hh = lane >> 5;
  const typename L::At lds_at = L::at(lane);
  int head, b;
  Part p;
  // 2^share waves take the same queries for as many heads
  const int block = 32 * NW / KS >> g.share;
  work_item(blocks, g.heads >> g.share, g.causal, head, b);
  if (!locate(g.offsets, g.seqs, (int)g.T, block, b, p)) return;
  const int wq = w / KS, k0 = w % KS * kOwn;  // whose queries, first block of the tiles
  head = (head << g.share) + (wq & ((1 << g.share) - 1));
  const int kv = head / (g.heads / g.kv_heads);
  const int q0 = p.block * block, rows = min(block, p.n - q0);
  const int i0 = q0 + 32 * (wq >> g.share), mine = min(32, p.n - i0);
  const T* K = (const T*)g.K + p.begin * g.ldk + kv * D;
  const T* V = (const T*)g.V + p.begin * g.ldv + kv * D;
  const Seen wg_first = keys_of(g, q0, p.n), wg_last = keys_of(g, q0 + rows - 1, p.n);
  const int t0 = max(wg_first.lo, 0) / L::kRows, t1 = wg_last.hi / L::kRows + 1;
  const Seen first = keys_of(g, i0, p.n), last = keys_of(g, i0 + 31, p.n);
  const Seen own = keys_of(g, i0 + (lane & 31), p.n);
  Copy<T, D, NW, L> ck, cv;
  ck.init(g.ldk, w, lane);
  cv.init(g.ldv, w, lane);
  auto issue = [&](int t, char* st) {
    const int64_t r = (int64_t)t * L::kRows;
    ck.issue(K + r * g.ldk, g.ldk, p.n - (int)r, st, w);
    cv.issue(V + r * g.ldv, g.ldv, p.n - (int)r, st + L::kBytes, w);
  };
  issue(t0, smem);
  Frag<T> q[L::kSteps], d_o[L::kSteps];
  const int64_t ldo = (int64_t)g.heads * D, at = ((p.begin + i0) * (int64_t)g.heads + head) * D;
  load_rows<T, D>(q, (const T*)g.Q + (p.begin + i0) * g.ldq + head * D, g.ldq, mine, lane);
  load_rows<T, D>(d_o, (const T*)g.dO + at, ldo, mine, lane);
  // delta_i from O_i . dO_i of all the wave's rows, of which the diagonal counts: formed as dp is,
  // step by step, so that their difference is exactly zero for a token whose output is the
  // one value that it sees (vector instructions would add up in another order).
  float delta = 0.f;
  {
    Frag<T> f[L::kSteps];
    load_rows<T, D>(f, (const T*)g.O + at, ldo, mine, lane);
    f32x16_t x;
    zero(x);
#pragma unroll
    for (int k = 0; k < L::kSteps; ++k) M::mma(f[k], d_o[k], x);
#pragma unroll
    for (int e = 0; e < 16; ++e) delta = acc_row(e, hh) == (lane & 31) ? x[e] : delta;
  }
  delta = halves_sum(delta);
  const int64_t row = head * g.T + p.begin + i0;
  float lse = INFINITY;  // (rows past the sequence, and rows that see nothing: no weights)
  if ((lane & 31) < mine) {
    lse = g.lse[row + (lane & 31)];
    if (lse == -INFINITY) lse = INFINITY;
  }
  const float c = g.scale * kLog2e, ref = lse * kLog2e;
  if (lane < mine && w % KS == 0) {
    g.top[row + lane] = ref;
    g.delta[row + lane] = delta;
  }
  f32x16_t a[D / 32];
#pragma unroll
  for (int i = 0; i < D / 32; ++i) zero(a[i]);
  auto tile = [&](int t, auto stage) {  // (a constant stage, as in the forward)
    constexpr int kAt = decltype(stage)::value * 2 * L::kBytes;
    stage_barrier();
    if (t + 1 < t1) issue(t + 1, smem + (2 * L::kBytes - kAt));
    const int r0 = t * L::kRows + 32 * k0;  // of the wave's own blocks
    if (mine <= 0 || r0 > last.hi || r0 + 32 * kOwn <= first.lo) return;
    const char* ks = smem + kAt;
    const char* vs = ks + L::kBytes;
    const bool all = see_all(first, last, r0, 32 * kOwn);
#pragma unroll
    for (int i = 0; i < kOwn; ++i) {
      f32x16_t s, dp;
      zero(s);
      zero(dp);
#pragma unroll
      for (int k = 0; k < L::kSteps; ++k) {
        M::mma(L::row(ks, 32 * (k0 + i), k, lds_at), q[k], s);
        M::mma(L::row(vs, 32 * (k0 + i), k, lds_at), d_o[k], dp);
      }
#pragma unroll
      for (int e = 0; e < 16; ++e) s[e] = exp2_(fmaf(s[e], c, -ref)) * (dp[e] - delta);
      if (!all) hide(s, own, r0 + 32 * i, hh, 0.f);
#pragma unroll
      for (int j = 0; j < L::kDown; ++j) {
        // (rounded as the forward's weights, and for its reason: 2.5e-3 for 1.8e-3)
        const Frag<T> f = M::of(s, j);
#pragma unroll
        for (int d = 0; d < D / 32; ++d) M::mma(L::col(ks, 32 * d, (k0 + i) * L::kDown + j, lds_at), f, a[d]);
      }
    }
  };
  for (int t = t0; t < t1; t += 2) {
    tile(t, std::integral_constant<int, 0>());
    if (t + 1 < t1) tile(t + 1, std::integral_constant<int, 1>());
  }
  stage_barrier();
  if constexpr (KS > 1) {
    float* mem = (float*)smem;
    if (w % KS) put_lanes<D>(mem + w * D / 2 * 64, a, lane);
    stage_barrier();
    if (w % KS) return;
#pragma unroll 1
    for (int y = 1; y < KS; ++y) add_lanes<D>(mem + (w + y) * D / 2 * 64, a, 1.f, 1.f, lane);
  }
  if (mine > 0)
    store_rows<T, D>(a, g.scale, (T*)g.dQ + (p.begin + i0) * g.lddq + head * D, g.lddq, mine,
                     smem + w * 32 * kOutPitch, lane);
}

// dk and dv of 32 NW rows a workgroup: it goes through the queries of the heads that share
// them, head after head, so that every sum has one order.  With several parts each takes
// a run of these tiles and leaves its sums in fp32 for attn_sum_kernel.
// kHeld: the values stay in LDS, not in registers, of which two waves a SIMD have 256 each:
// keys, dk and dv take 160 of them (with the values too, or 64 keys a wave, they spill).
// 4096 tokens of 64 heads in 8 groups of 128, causal: 543 us in four parts and 23 for their
// sum, 1.0 PFLOP/s, matrix cores busy for 55 %, vector instructions 34; 6011 tokens of 16
// heads of 64 in 9 sequences 37 us (three waves a SIMD; two 41).
template <typename T, int D, int NW, bool kHeld>
__global__ __launch_bounds__(64 * NW, sizeof(T) == 2 && D == 64 && NW == 4 ? 3 : 1)
void attn_dkv_kernel(const AttnArgs g, int blocks) {
  typedef Tile<T, D> L;
  typedef Mma<T> M;
  constexpr int kBlock = 32 * NW;
  // two stages of queries, dO, and their rows' log2 of the sum and delta
  constexpr int kStage = 2 * L::kBytes;
  constexpr int kNeed = 2 * kStage + (kHeld ? kBlock * L::kPitch : 0), kOut = kBlock * D * 4;
  __shared__ __align__(1024) char smem[kNeed > kOut ? kNeed : kOut];
  __shared__ __align__(16) float stats[2][2][64];
  const int lane = threadIdx.x & 63, w = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int hh = lane >> 5;
  const typename L::At lds_at = L::at(lane);
  int kv, b;
  Part p;
  work_item(blocks * g.parts, g.kv_heads, false, kv, b);
  const int part = b % g.parts;
  if (!locate(g.offsets, g.seqs, (int)g.T, kBlock, b / g.parts, p)) return;
  const int group = g.heads / g.kv_heads;
  const int k0 = p.block * kBlock, rows = min(kBlock, p.n - k0);
  const int j0 = k0 + 32 * w, mine = min(32, p.n - j0);
  const Seen wg_first = queries_of(g, k0, p.n), wg_last = queries_of(g, k0 + rows - 1, p.n);
  const int t0 = wg_first.lo / L::kRows, tiles = wg_last.hi / L::kRows + 1 - t0;
  const Seen first = queries_of(g, j0, p.n), last = queries_of(g, j0 + 31, p.n);
  const Seen own = queries_of(g, j0 + (lane & 31), p.n);
  const int64_t ldo = (int64_t)g.heads * D;
  Copy<T, D, NW> cq, co;
  cq.init(g.ldq, w, lane);
  co.init(ldo, w, lane);
  // the part's first tile, and how many (group tiles parts < 2^31; all in scalar registers)
  const uint32_t run = (uint32_t)(group * tiles);
  const int x0 = __builtin_amdgcn_readfirstlane(run * part / g.parts);
  const int total = __builtin_amdgcn_readfirstlane(run * (part + 1) / g.parts) - x0;
  const int skip = __builtin_amdgcn_readfirstlane(x0 / tiles);
  int head = kv * group + skip, next = t0 + x0 - skip * tiles;  // of the tile to copy next
  auto issue = [&](int stage) {
    const int r0 = next * L::kRows;
    char* st = smem + stage * kStage;
    cq.issue((const T*)g.Q + (p.begin + r0) * g.ldq + head * D, g.ldq, p.n - r0, st, w);
    co.issue((const T*)g.dO + ((p.begin + r0) * (int64_t)g.heads + head) * D, ldo, p.n - r0,
             st + L::kBytes, w);
    // (rows past the sequence read zero, like their dO: they add nothing)
    if (w < 2) {
      const float* from = (w ? g.delta : g.top) + head * g.T + p.begin + r0;
      __builtin_amdgcn_raw_ptr_buffer_load_lds(rsrc_of(from, (uint32_t)min(p.n - r0, L::kRows) * 4),
                                               (lds_void*)stats[stage][w], 4, lane * 4, 0, 0, 0);
    }
    if (++next == t0 + tiles) {
      next = t0;
      ++head;
    }
  };
  const T* V = (const T*)g.V + (p.begin + k0) * g.ldv + kv * D;
  const char* held = smem + 2 * kStage;
  Frag<T> k[L::kSteps], v[kHeld ? 1 : L::kSteps];
  if constexpr (kHeld) {
    Copy<T, D, NW> cv;
    cv.init(g.ldv, w, lane);
#pragma unroll
    for (int i = 0; i < kBlock / L::kRows; ++i)
      cv.issue(V + i * L::kRows * g.ldv, g.ldv, rows - i * L::kRows, smem + 2 * kStage + i * L::kBytes, w);
  } else {
    load_rows<T, D>(v, V + 32 * w * g.ldv, g.ldv, mine, lane);
  }
  load_rows<T, D>(k, (const T*)g.K + (p.begin + j0) * g.ldk + kv * D, g.ldk, mine, lane);
  int now = next;  // the tile to use
  if (total > 0) issue(0);
  f32x16_t dk[D / 32], dv[D / 32];
#pragma unroll
  for (int i = 0; i < D / 32; ++i) {
    zero(dk[i]);
    zero(dv[i]);
  }
  const float scale = g.scale * kLog2e;
  auto tile = [&](int x, auto stage) {  // (a constant stage, as in the forward)
    constexpr int kAt = decltype(stage)::value;
    stage_barrier();
    const int r0 = now * L::kRows;
    now = next;
    if (x + 1 < total) issue(1 - kAt);
    if (mine <= 0 || r0 + L::kRows <= first.lo || r0 > last.hi) return;
    const char* qs = smem + kAt * kStage;
    const char* os = qs + L::kBytes;
    const bool all = see_all(first, last, r0, L::kRows);
#pragma unroll
    for (int i = 0; i < L::kBlocks; ++i) {
      // (what is read from LDS is read where it is used: registers are full)
      if constexpr (kHeld) asm volatile("" ::: "memory");
      f32x16_t s, dp;
      zero(s);
      zero(dp);
      // (the addresses are formed where they are used, not held in registers, which are full)
      typename L::At here = lds_at;
      if constexpr (kHeld) asm volatile("" : "+v"(here.row), "+v"(here.col));
      // (a step's operands are read while the one before it multiplies, and no earlier)
      Frag<T> a[2], o[2], u[2];
      auto rows_of = [&](int e) {
        a[e & 1] = L::row(qs, 32 * i, e, here);
        o[e & 1] = L::row(os, 32 * i, e, here);
        if constexpr (kHeld) u[e & 1] = L::row(held, 32 * w, e, here);
      };
      rows_of(0);
#pragma unroll
      for (int e = 0; e < L::kSteps; ++e) {
        if (e + 1 < L::kSteps) rows_of(e + 1);
        M::mma(a[e & 1], k[e], s);
        if constexpr (kHeld) M::mma(o[e & 1], u[e & 1], dp);
        else M::mma(o[e & 1], v[e], dp);
        __builtin_amdgcn_sched_barrier(0);
      }
      const float* top = &stats[kAt][0][32 * i + 4 * hh];
      const float* del = &stats[kAt][1][32 * i + 4 * hh];
#pragma unroll
      for (int e = 0; e < 16; e += 4) {
        const f32x4_t a = *(const f32x4_t*)(top + 2 * e);
#pragma unroll
        for (int y = 0; y < 4; ++y) s[e + y] = exp2_(fmaf(s[e + y], scale, -a[y]));
      }
      if (!all) hide(s, own, r0 + 32 * i, hh, 0.f);
#pragma unroll
      for (int e = 0; e < 16; e += 4) {
        const f32x4_t a = *(const f32x4_t*)(del + 2 * e);
#pragma unroll
        for (int y = 0; y < 4; ++y) dp[e + y] = s[e + y] * (dp[e + y] - a[y]);
      }
      constexpr int kCols = D / 32;
      auto cols_of = [&](int x) {
        o[x & 1] = L::col(os, 32 * (x % kCols), i * L::kDown + x / kCols, here);
        a[x & 1] = L::col(qs, 32 * (x % kCols), i * L::kDown + x / kCols, here);
      };
      cols_of(0);
#pragma unroll
      for (int j = 0; j < L::kDown; ++j) {
        const Frag<T> f = M::of(s, j), h = M::of(dp, j);
#pragma unroll
        for (int d = 0; d < kCols; ++d) {
          const int x = j * kCols + d;
          if (x + 1 < L::kDown * kCols) cols_of(x + 1);
          M::mma(o[x & 1], f, dv[d]);
          M::mma(a[x & 1], h, dk[d]);
          __builtin_amdgcn_sched_barrier(0);
        }
      }
    }
  };
  for (int x = 0; x < total; x += 2) {
    tile(x, std::integral_constant<int, 0>());
    if (x + 1 < total) tile(x + 1, std::integral_constant<int, 1>());
  }
  stage_barrier();
  if (mine <= 0) return;
  const int64_t j = p.begin + j0;
  if (g.parts > 1) {
    const int64_t kvd = (int64_t)g.kv_heads * D;
    float* out = g.sums + (part * 2 * g.T + j) * kvd + kv * D;
    char* lds = smem + w * 32 * D * 4;
    store_rows<float, D>(dk, g.scale, out, kvd, mine, lds, lane);
    store_rows<float, D>(dv, 1.f, out + g.T * kvd, kvd, mine, lds, lane);
  } else {
    char* lds = smem + w * 32 * L::kPitch;
    store_rows<T, D>(dk, g.scale, (T*)g.dK + j * g.lddk + kv * D, g.lddk, mine, lds, lane);
    store_rows<T, D>(dv, 1.f, (T*)g.dV + j * g.lddv + kv * D, g.lddv, mine, lds, lane);
  }
}

// dK and dV from the parts' sums [parts][dK, dV][T][kv_heads dim], added in order: four
// elements a thread, of rows that lie in a sequence.  Bound by memory: four parts of 4096
// rows of 8 heads of 128, 151 MB, 23 us (6.5 TB/s, some of it out of caches).
template <typename T>
__global__ __launch_bounds__(256) void attn_sum_kernel(const AttnArgs g) {
  const int64_t kvd = (int64_t)g.kv_heads * g.dim, n = g.T * kvd / 4;
  for (int64_t i = blockIdx.x * 256ll + threadIdx.x; i < 2 * n; i += gridDim.x * 256ll) {
    const bool v = i >= n;
    const int64_t at = (v ? i - n : i) * 4, row = at / kvd, col = at % kvd;
    bool in = false;  // of a sequence (the last that begins at or before it)
    {
      int lo = 0, hi = g.seqs;
      while (hi - lo > 1) {
        const int mid = (lo + hi) >> 1;
        if (g.offsets[mid] <= row) lo = mid;
        else hi = mid;
      }
      in = g.offsets[lo] <= row && row < g.offsets[lo + 1];
    }
    if (!in) continue;
    float f[4] = {0.f, 0.f, 0.f, 0.f};
    for (int p = 0; p < g.parts; ++p) {
      const f32x4_t x = *(const f32x4_t*)(g.sums + (p * 2 + v) * g.T * kvd + at);
#pragma unroll
      for (int e = 0; e < 4; ++e) f[e] += x[e];
    }
    Vec4<T>::store(v ? (T*)g.dV + row * g.lddv + col : (T*)g.dK + row * g.lddk + col, f);
  }
}

// Blocks of R rows of seqs sequences that share T rows, at most.
int64_t blocks_of(int64_t T, int64_t seqs, int R) {
  const int64_t full = std::min(seqs, T);
  return (T + full * (R - 1)) / R;
}

// (The compiler leaves out host stubs of kernels that only templates launch.)
#define MEMFINE_FWD(T, D, NW, KS) \
  template __global__ void attn_fwd_kernel<T, D, NW, KS>(const AttnArgs, int);
#define MEMFINE_DQ(T, D, NW, KS) \
  template __global__ void attn_dq_kernel<T, D, NW, KS>(const AttnArgs, int);
#define MEMFINE_DKV(T, D, NW, HELD) \
  template __global__ void attn_dkv_kernel<T, D, NW, HELD>(const AttnArgs, int);
MEMFINE_FWD(bf16_t, 64, 4, 1)
MEMFINE_FWD(bf16_t, 64, 8, 1)
MEMFINE_FWD(bf16_t, 64, 8, 4)
MEMFINE_FWD(bf16_t, 128, 4, 1)
MEMFINE_FWD(bf16_t, 128, 8, 4)
MEMFINE_FWD(float, 64, 4, 1)
MEMFINE_FWD(float, 128, 4, 1)
MEMFINE_DQ(bf16_t, 64, 4, 1)
MEMFINE_DQ(bf16_t, 64, 8, 4)
MEMFINE_DQ(bf16_t, 128, 4, 1)
MEMFINE_DQ(bf16_t, 128, 8, 4)
MEMFINE_DQ(float, 64, 4, 1)
MEMFINE_DQ(float, 128, 4, 1)
MEMFINE_DKV(bf16_t, 64, 4, false)
MEMFINE_DKV(bf16_t, 64, 8, false)
MEMFINE_DKV(bf16_t, 128, 8, true)
MEMFINE_DKV(float, 64, 4, false)
MEMFINE_DKV(float, 128, 4, false)
#undef MEMFINE_FWD
#undef MEMFINE_DQ
#undef MEMFINE_DKV
template __global__ void attn_sum_kernel<bf16_t>(const AttnArgs);
template __global__ void attn_sum_kernel<float>(const AttnArgs);

// Heads of a group that a workgroup for `sets` sets of 32 queries takes together: the largest
// power of two that divides the group.
int share_of(const AttnArgs& g, int sets) {
  int share = 0;
  while ((g.heads / g.kv_heads) % (2 << share) == 0 && (2 << share) <= sets) ++share;
  return share;
}
template <typename T, int D, int NW, int KS> void run_fwd(AttnArgs g, hipStream_t s) {
  g.share = share_of(g, NW / KS);
  const int blocks = (int)blocks_of(g.T, g.seqs, 32 * NW / KS >> g.share);
  attn_fwd_kernel<T, D, NW, KS><<<(unsigned)blocks * (g.heads >> g.share), 64 * NW, 0, s>>>(g, blocks);
}
template <typename T, int D, int NW, int KS> void run_dq(AttnArgs g, hipStream_t s) {
  g.share = share_of(g, NW / KS);
  const int blocks = (int)blocks_of(g.T, g.seqs, 32 * NW / KS >> g.share);
  attn_dq_kernel<T, D, NW, KS><<<(unsigned)blocks * (g.heads >> g.share), 64 * NW, 0, s>>>(g, blocks);
}
template <typename T, int D, int NW, bool kHeld> void run_dkv(const AttnArgs& g, hipStream_t s) {
  const int blocks = (int)blocks_of(g.T, g.seqs, 32 * NW);
  attn_dkv_kernel<T, D, NW, kHeld>
      <<<(unsigned)blocks * g.kv_heads * g.parts, 64 * NW, 0, s>>>(g, blocks);
  if (g.parts > 1) {
    const int64_t n = (g.T * g.kv_heads * D / 2 + 255) / 256;
    attn_sum_kernel<T><<<(unsigned)std::min<int64_t>(n, 8192), 256, 0, s>>>(g);
  }
}

// So few sets of 32 queries (at most 4 a CU) of so long sequences that the longest ones' tiles,
// one after the other, are the time: four waves a set, each with a quarter of the keys.  The
// forward of two heads of 6783 tokens 141 us with one wave, 69 with four; 16 heads in 2 groups,
// 2048 tokens 48 and 37; 32 heads in 8 groups, 512 tokens 15.6 and 13.3, 1024 tokens 26.9 both,
// 2048 tokens 54 and 71; 8 sequences of 256 tokens, 8 heads 10.6 and 11.2.
// Where no mask, or a window of at most half the sequence, makes all chains alike, none is left
// to run alone at the end, and heads of 128 are better off from two sets a CU on: 16 heads in 4
// groups, 2048 tokens, a window of 512 18 us with one wave and 28 with four, without a mask 48 and
// 54; 8 heads in 2 groups, a window of 512 17 and 15 (16 heads of 64: 15.5 and 14.5).
bool few_queries(const AttnArgs& g) {
  const int64_t sets = blocks_of(g.T, g.seqs, 32) * g.heads, mean = g.T / std::max(g.seqs, 1);
  const bool alike = !g.causal || (g.window > 0 && g.window <= mean / 2);
  return sets <= (alike && g.dim == 128 ? 2 : 4) * g.cus && mean >= 384 && mean * g.cus > 200 * sets;
}
// Sequences so short, on average, that the starts and ends of workgroups weigh more than
// what twice the rows save of copies: four waves, several workgroups a CU, else eight (heads of
// 64).  Forward, 32 heads, sequences of 256 tokens 29 us against 30, of 1024 56 and 60, of 2048
// 92 and 94, of 4096 178 and 165; dk and dv of 16 heads, sequences of 668 tokens 38 us against
// 50, of 4096 68 and 60.
bool short_rows(const AttnArgs& g) { return g.T < 2048 * (int64_t)g.seqs; }

}  // namespace

// Parts that the tiles of a group's queries are shared out in for dk and dv: one workgroup's
// chain, all queries of the group that see any of 256 keys (fp32: 128), is the shortest time
// it can take, and few keys leave CUs idle; but parts are written and read again.  In
// microseconds:
//   tile x max(chain / parts + 4, (load chain / parts + 4) workgroups per CU) + sums
// (a start and an end weigh four tiles; load: the mean chain over the longest, .6 under a
// causal mask, 1 where a short window or no mask makes all alike; tile: 3.5, fp32 8; sums: 6
// and 16 bytes an element of dk at 3 TB/s.)  Dim 128, the whole gradient with one, two and four
// parts: 32 heads in 8 groups, 8192 tokens 2.33, 1.79 and 1.81 ms (two are taken), a window of
// 128 160, 208 and 271 us (one), 4 sequences of 1024 without a mask, 4 groups 481, 311 and 248 us
// (four); 64 heads in 8 groups, 4096 tokens 1.85, 1.18 and 0.94 ms (four), a window of 512 399,
// 309 and 335 us (two).
int attn_parts(const AttnArgs& g) {
  const int group = g.heads / g.kv_heads, keys = g.f32 ? 128 : 256, rows = g.f32 ? 32 : 64;
  const double items = (double)blocks_of(g.T, g.seqs, keys) * g.kv_heads;
  const double mean = (double)g.T / std::max<int64_t>(std::min<int64_t>(g.seqs, g.T), 1);
  const double seen = g.window > 0 ? std::min<double>(mean, g.window) : mean;
  const double chain = group * std::ceil(std::min(mean, seen + keys) / rows);
  const double load = g.causal ? 1. - .4 * seen / std::max(mean, 1.) : 1.;
  int best = 1;
  double least = 0.;
  for (int p = 1; p <= 32 && p <= chain; p *= 2) {
    const double t = std::max(chain / p + 4., (load * chain / p + 4.) * items * p / g.cus) * (g.f32 ? 8. : 3.5) +
                     (p > 1 ? 6. + p * (double)g.T * g.kv_heads * g.dim * 16. / 3e6 : 0.);
    if (p == 1 || t < least) {
      best = p;
      least = t;
    }
  }
  return best;
}
int64_t attn_bwd_floats(const AttnArgs& g) {
  return (2 * g.heads + (g.parts > 1 ? 2 * (int64_t)g.parts * g.kv_heads * g.dim : 0)) * g.T;
}

// (blocks of 32 rows: workgroups of 512 threads for more rows, or of several heads, are fewer)
bool attn_fits(const AttnArgs& g) {
  return blocks_of(g.T, g.seqs, 32) * g.heads <= kMostItems / 512;
}

hipError_t launch_attn_fwd(const AttnArgs& g, hipStream_t s) {
  if (!attn_fits(g)) return hipErrorInvalidValue;
  if (g.f32) {
    if (g.dim == 64) run_fwd<float, 64, 4, 1>(g, s);
    else run_fwd<float, 128, 4, 1>(g, s);
  } else if (few_queries(g)) {
    if (g.dim == 64) run_fwd<bf16_t, 64, 8, 4>(g, s);
    else run_fwd<bf16_t, 128, 8, 4>(g, s);
  } else {
    if (g.dim == 128) run_fwd<bf16_t, 128, 4, 1>(g, s);
    else if (short_rows(g)) run_fwd<bf16_t, 64, 4, 1>(g, s);
    else run_fwd<bf16_t, 64, 8, 1>(g, s);
  }
  return hipGetLastError();
}

hipError_t launch_attn_bwd(const AttnArgs& g, hipStream_t s) {
  if (!attn_fits(g)) return hipErrorInvalidValue;
  // (dq's kernel writes top and delta, which dkv's reads)
  if (g.f32) {
    if (g.dim == 64) {
      run_dq<float, 64, 4, 1>(g, s);
      run_dkv<float, 64, 4, false>(g, s);
    } else {
      run_dq<float, 128, 4, 1>(g, s);
      run_dkv<float, 128, 4, false>(g, s);
    }
  } else if (g.dim == 64) {
    if (few_queries(g)) run_dq<bf16_t, 64, 8, 4>(g, s);
    else run_dq<bf16_t, 64, 4, 1>(g, s);
    if (short_rows(g)) run_dkv<bf16_t, 64, 4, false>(g, s);
    else run_dkv<bf16_t, 64, 8, false>(g, s);
  } else {
    if (few_queries(g)) run_dq<bf16_t, 128, 8, 4>(g, s);
    else run_dq<bf16_t, 128, 4, 1>(g, s);
    run_dkv<bf16_t, 128, 8, true>(g, s);
  }
  return hipGetLastError();
}

}  // namespace memfine
