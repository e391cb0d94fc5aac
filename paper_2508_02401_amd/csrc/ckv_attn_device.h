// Device helpers of the attention and decode kernels: waits, operand rounding, values
// that are not finite, and how a paged batch is cut into workgroups.
#pragma once

#include "ckv_device.h"

namespace ckv {
namespace dev {

typedef short s16x4 __attribute__((ext_vector_type(4)));

// Wait until at most N vector-memory operations of this wave are outstanding
// and its LDS operations are done; nothing is moved across.
template <int N>
__device__ __forceinline__ void wait_vm() {
  asm volatile("" ::: "memory");
  __builtin_amdgcn_s_waitcnt(0x070 | (N & 15) | ((N >> 4) << 14));
  asm volatile("" ::: "memory");
}
__device__ __forceinline__ void barrier() {
  asm volatile("" ::: "memory");
  __builtin_amdgcn_s_barrier();
  asm volatile("" ::: "memory");
}

// f16 weights are kept 2^8 larger than exp2(s - max), out of the subnormals
// for all but weights below 2^-22; the running maximum is moved when a row
// passes it by more than kSlack (in exp2 units), so weights stay below 2^14.
constexpr float kF16Bias = 8.f;
constexpr float kSlack = 6.f;

// exp2 of a logit's distance to the maximum. fp32 caches keep weights below
// 2^-126, which the bare instruction flushes to zero; V may be that large. The
// 16-bit types' weights are rounded to operands that end sooner.
template <int DT>
__device__ __forceinline__ float weight_exp2(float x) {
  return DT == 2 ? exp2f(x) : fast_exp2(x);
}

// Eight fp32 values rounded to the 16-bit operand chunk of an MFMA.
template <int DT>
__device__ __forceinline__ uint4 round_chunk(const float* x) {
  if constexpr (DT == 0) {
    bf16x8 v;
#pragma unroll
    for (int i = 0; i < 8; ++i) v[i] = (__bf16)x[i];
    return __builtin_bit_cast(uint4, v);
  } else {
    f16x8 v;
#pragma unroll
    for (int i = 0; i < 8; ++i) v[i] = (_Float16)x[i];
    return __builtin_bit_cast(uint4, v);
  }
}

// 8 (16-bit) or 4 (fp32) fp32 values -> one operand chunk, and for 16-bit types
// the chunk of the rounded remainders.
template <int DT>
__device__ __forceinline__ void split_chunk(const float* x, uint4& hi, uint4& lo) {
  if constexpr (DT == 2) {
    hi = make_uint4(__float_as_uint(x[0]), __float_as_uint(x[1]), __float_as_uint(x[2]),
                    __float_as_uint(x[3]));
  } else if constexpr (DT == 0) {
    bf16x8 h, l;
#pragma unroll
    for (int i = 0; i < 8; ++i) {
      h[i] = (__bf16)x[i];
      l[i] = (__bf16)(x[i] - (float)h[i]);
    }
    hi = __builtin_bit_cast(uint4, h);
    lo = __builtin_bit_cast(uint4, l);
  } else {
    f16x8 h, l;
#pragma unroll
    for (int i = 0; i < 8; ++i) {
      h[i] = (_Float16)x[i];
      l[i] = (_Float16)(x[i] - (float)h[i]);
    }
    hi = __builtin_bit_cast(uint4, h);
    lo = __builtin_bit_cast(uint4, l);
  }
}

// A chunk of V without its values that are not finite, and these in x as numbers
// that add up without getting mixed over the (at most 64) keys of a tile.
constexpr float kPlusInf = 1.f, kMinusInf = 128.f, kNan = 16384.f;
template <int DT>
__device__ __forceinline__ uint4 strip_chunk(uint4 v, uint4& x) {
  constexpr uint16_t kExp = DT == 0 ? 0x7F80 : 0x7C00;
  typedef uint16_t u16x8 __attribute__((ext_vector_type(8)));
  u16x8 a = __builtin_bit_cast(u16x8, v);
  float f[8];
#pragma unroll
  for (int i = 0; i < 8; ++i) {
    const uint16_t mag = a[i] & 0x7FFF;
    f[i] = mag < kExp ? 0.f : mag > kExp ? kNan : a[i] >> 15 ? kMinusInf : kPlusInf;
    a[i] = mag < kExp ? a[i] : 0;
  }
  x = round_chunk<DT>(f);
  return __builtin_bit_cast(uint4, a);
}
// acc and 0 times the chunk's values: NaN where one of them is not finite.
template <int DT>
__device__ __forceinline__ float zero_times(uint4 v, float acc) {
  const uint32_t w[4] = {v.x, v.y, v.z, v.w};
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    if constexpr (DT == 0) {
      typedef __bf16 bf16x2 __attribute__((ext_vector_type(2)));
      acc = __builtin_amdgcn_fdot2_f32_bf16(__builtin_bit_cast(bf16x2, w[i]), bf16x2{0, 0}, acc, false);
    } else {
      typedef _Float16 f16x2 __attribute__((ext_vector_type(2)));
      acc = __builtin_amdgcn_fdot2(__builtin_bit_cast(f16x2, w[i]), f16x2{0, 0}, acc, false);
    }
  }
  return acc;
}
__device__ __forceinline__ float strip_f32(float v, float& x) {
  x = fabsf(v) < INFINITY ? 0.f : v == INFINITY ? kPlusInf : v == -INFINITY ? kMinusInf : kNan;
  return fabsf(v) < INFINITY ? v : 0.f;
}
// What a sum of such numbers adds to a row's output.
__device__ __forceinline__ float stripped_sum(float c) {
  const float minus = floorf(c * (1.f / kMinusInf)) * kMinusInf;
  const float x = minus == 0.f ? INFINITY : minus == c && c < kNan ? -INFINITY : NAN;
  return c == 0.f ? 0.f : x;
}
// Operand of 8 keys (bits 0..3 and 8..11): 1 for those that the row sees.
template <int DT>
__device__ __forceinline__ uint4 seen_chunk(uint32_t bits) {
  float one[8];
#pragma unroll
  for (int i = 0; i < 8; ++i) one[i] = bits & (1u << (8 * (i >> 2) + (i & 3))) ? 1.f : 0.f;
  return round_chunk<DT>(one);
}
__device__ __forceinline__ f32x16 mfma_f32(float a, float b, f32x16 c) {
  return __builtin_amdgcn_mfma_f32_32x32x2f32(a, b, c, 0, 0, 0);
}

// Four fp32 values to an output row.
template <int DT>
__device__ __forceinline__ void store4(char* p, float a, float b, float c, float d) {
  if constexpr (DT == 2) {
    *reinterpret_cast<f32x4*>(p) = f32x4{a, b, c, d};
  } else if constexpr (DT == 0) {
    typedef __bf16 bf16x4 __attribute__((ext_vector_type(4)));
    *reinterpret_cast<bf16x4*>(p) = bf16x4{(__bf16)a, (__bf16)b, (__bf16)c, (__bf16)d};
  } else {
    typedef _Float16 f16x4 __attribute__((ext_vector_type(4)));
    *reinterpret_cast<f16x4*>(p) = f16x4{(_Float16)a, (_Float16)b, (_Float16)c, (_Float16)d};
  }
}


__device__ __forceinline__ int clamp_int(int x, int lo, int hi) {
  return x < lo ? lo : (x > hi ? hi : x);
}

// ---- packed prompts ----
// Block b of the grid: KV head b % n_kv (neighbouring blocks go to different
// XCDs, so with 8 KV heads each XCD's L2 holds one head's K and V), row tiles in
// the launch's order, a range of a prompt's tiles from its last on.
struct PromptTile {
  int tok0, T, g, rt;
};
__device__ __forceinline__ PromptTile prompt_tile(const PrefillArgs& A) {
  PromptTile p;
  const int b = (int)blockIdx.x / A.a.n_kv;
  p.g = (int)blockIdx.x - b * A.a.n_kv;
  int lo = 0, hi = A.n;  // the last range whose first tile is at most b
  while (hi - lo > 1) {
    const int mid = (lo + hi) / 2;
    if (A.tile[mid] <= b) lo = mid; else hi = mid;
  }
  p.tok0 = A.tok[lo];
  p.T = A.len[lo];
  p.rt = A.top[lo] - (b - A.tile[lo]);
  return p;
}

// ---- paged batches -----------------------------------------------------------
__device__ __forceinline__ int page_at(const PageDiv& d, int x) {
  return (int)(((uint64_t)(uint32_t)x * d.mul) >> d.shift);
}

// A request of a paged batch, whatever the device arrays hold.
struct PagedSeq {
  int tok0, T, n;  // first row, rows, tokens
};
__device__ __forceinline__ PagedSeq paged_seq(const PagedArgs& A, int s) {
  PagedSeq q;
  q.tok0 = clamp_int(to_global(A.cu_q)[s], 0, A.total_q);
  const int end = clamp_int(to_global(A.cu_q)[s + 1], 0, A.total_q);
  q.T = end > q.tok0 ? end - q.tok0 : 0;
  q.n = clamp_int(to_global(A.kv_len)[s], 0, A.max_kv);
  return q;
}
__device__ __forceinline__ bool paged_few(const PagedArgs& A, const PagedSeq& q) {
  return q.T * A.a.G <= A.few_rows;
}

// What follows is worked out by every wave for itself, 64 requests at a time, one
// per lane, with no barrier: for 64 requests and fewer they are read once and stay
// in registers. Sums and searches over the whole workgroup took 1.7 us more a kernel.
__device__ __forceinline__ PagedSeq lane_seq(const PagedArgs& A, int s) {
  PagedSeq q = {};
  if (s < A.num_seqs) q = paged_seq(A, s);
  return q;
}
// f(request) for this lane's requests.
template <class F>
__device__ __forceinline__ void each_seq(const PagedArgs& A, const PagedSeq& first, F f) {
  f(first);
  for (int s = 64 + (threadIdx.x & 63); s < A.num_seqs; s += 64) f(paged_seq(A, s));
}
template <int K>
__device__ __forceinline__ void wave_sums(int64_t (&x)[K]) {
#pragma unroll
  for (int i = 32; i > 0; i >>= 1)
#pragma unroll
    for (int k = 0; k < K; ++k) x[k] += __shfl_xor(x[k], i);
}

// Keys per workgroup of a kernel, its share. Every workgroup works it out for itself
// from the requests' lengths (the host knows bounds only). `work` is the sum of the
// keys over the `base` items (row tiles times KV heads) of the launch, `target` its
// workgroups in one round. Up to half a round of items, all workgroups are to fit
// into one round: an even share of work / target keys does where the lengths divide
// well; otherwise it leaves up to one short workgroup per item over, and with
// work / (target - base) they always fit.
// Shares are whole UNITs and at least LEAST.
constexpr int kUnsplit = 0x7FFFFF80;
template <int LEAST, int UNIT>
__device__ __forceinline__ int paged_share(int64_t work, int64_t parts) {
  const double c = ceil((double)work / (double)parts * (1.0 / UNIT)) * UNIT;  // exact below 2^53
  return c < LEAST ? LEAST : c > kUnsplit ? kUnsplit : (int)c;
}

// The kernel for few rows: a 32-key tile for each of the four waves. Past half a round
// of items it takes small shares, of which the short requests' and the long ones'
// add up evenly.
__device__ __forceinline__ int few_share(const PagedArgs& A, const PagedSeq& first) {
  int64_t x[2] = {};  // keys and items
  each_seq(A, first, [&](const PagedSeq& q) {
    const bool mine = q.T > 0 && paged_few(A, q);
    x[0] += mine ? q.n : 0;
    x[1] += mine ? 1 : 0;
  });
  wave_sums(x);
  x[0] *= A.a.n_kv;
  x[1] *= A.a.n_kv;
  auto share = [&](int64_t parts) { return paged_share<kFewLeast, 32 * kWaves>(x[0], parts); };
  const bool fits = 2 * x[1] <= A.few_target;
  int c = share(fits ? A.few_target : (int64_t)A.few_target * kFewRounds);
  if (fits) {
    int64_t y[1] = {};  // workgroups with even shares
    each_seq(A, first, [&](const PagedSeq& q) { y[0] += q.T > 0 && paged_few(A, q) ? paged_chunks(q.n, c) : 0; });
    wave_sums(y);
    if (y[0] * A.a.n_kv > A.few_target) c = share(A.few_target - x[1]);
  }
  return __builtin_amdgcn_readfirstlane(c);  // the same in every lane: in scalar registers from here on
}

// The tile kernel: it does not split past half a round of items. Where even shares do not
// fit, the smallest of 64 shares up to work / (target - base) that does, one per lane (500,
// 300 and 100 tokens over 8000 each: 302 us with that last share, 213 so; for few rows the
// search costs more than it saves, 31 to 37 us for 16 single tokens).
__device__ __forceinline__ int many_share(const PagedArgs& A, const PagedSeq& first) {
  auto tiles = [&](int T) { return (T * A.a.G + kAttnRows - 1) / kAttnRows; };
  int64_t x[2] = {};  // keys and items
  each_seq(A, first, [&](const PagedSeq& q) {
    const int n = q.T > 0 && !paged_few(A, q) ? tiles(q.T) : 0;
    x[0] += (int64_t)n * q.n;
    x[1] += n;
  });
  wave_sums(x);
  x[0] *= A.a.n_kv;
  x[1] *= A.a.n_kv;
  if (2 * x[1] > A.many_target) return kUnsplit;
  auto share = [&](int64_t parts) { return paged_share<kManyLeast, 64>(x[0], parts); };
  int lo = share(A.many_target);
  const int hi = share(A.many_target - x[1]);
  const int lane = threadIdx.x & 63;
  // lane 0 tries lo, lane 63 hi, with which all fit
  const int64_t step = ((int64_t)(hi - lo) * lane / 63 + 63) / 64 * 64;
  const int c = lo + step > hi ? hi : (int)(lo + step);
  const float r = 1.f / (float)c;
  int64_t count = 0;
  for (int s0 = 0; s0 < A.num_seqs; s0 += 64) {
    const PagedSeq q = s0 == 0 ? first : lane_seq(A, s0 + lane);
    for (uint64_t m = __ballot(q.T > 0 && !paged_few(A, q)); m; m &= m - 1) {
      const int l = __ffsll((unsigned long long)m) - 1;
      const int n = __builtin_amdgcn_readlane(q.n, l), T = __builtin_amdgcn_readlane(q.T, l);
      int e = (int)((float)n * r);  // n / c rounded up: at most a few hundred, so at most one off
      e += (int64_t)e * c < n ? 1 : 0;
      e += (int64_t)e * c < n ? 1 : 0;
      e -= (int64_t)(e - 1) * c >= n ? 1 : 0;
      count += (int64_t)tiles(T) * (n <= c ? 1 : e);
    }
  }
  const uint64_t fits = __ballot(count * A.a.n_kv <= A.many_target) | 1ull << 63;
  return __builtin_amdgcn_readlane(c, __ffsll((unsigned long long)fits) - 1);
}

// The request that entry b of a list of requests' entries belongs to, with
// count(q) entries (x) each; and a second number (y) summed over the requests
// before it.
struct Found {
  PagedSeq q;         // the request
  int s, within;      // its number, entry within it
  uint32_t before;    // sum of y
};
template <class Count>
__device__ __forceinline__ bool find_entry(const PagedArgs& A, const PagedSeq& first, int b, Count count, Found& f) {
  const int lane = threadIdx.x & 63;
  uint32_t x0 = 0, y0 = 0;
  for (int s0 = 0; s0 < A.num_seqs; s0 += 64) {
    const PagedSeq q = s0 == 0 ? first : lane_seq(A, s0 + lane);
    uint2 c = make_uint2(0u, 0u);
    if (q.T > 0) c = count(q);
    const uint32_t x = x0 + wave_incl_scan(c.x), y = y0 + wave_incl_scan(c.y);
    const uint64_t hit = __ballot((uint32_t)b < x && (uint32_t)b >= x - c.x);
    if (hit) {
      const int l = __ffsll((unsigned long long)hit) - 1;
      auto of = [&](int v) { return __builtin_amdgcn_readlane(v, l); };
      f.q.tok0 = of(q.tok0);
      f.q.T = of(q.T);
      f.q.n = of(q.n);
      f.s = s0 + l;
      f.within = of((int)((uint32_t)b - (x - c.x)));
      f.before = (uint32_t)of((int)(y - c.y));
      return true;
    }
    x0 = (uint32_t)__builtin_amdgcn_readlane((int)x, 63);
    y0 = (uint32_t)__builtin_amdgcn_readlane((int)y, 63);
  }
  return false;
}

// The factor of a partial result (maximum, sum) towards the maximum m: 0 for
// one without keys, 1 for one whose logits were all NaN.
__device__ __forceinline__ float part_weight(float2 x, float m) {
  return x.x == -INFINITY ? (x.y == 0.f ? 0.f : 1.f) : exp2f(x.x - m);
}

// Partial results of a split item, in its slot: `rows` rows of D floats, then
// their (maximum, sum) pairs.
__device__ __forceinline__ float* partial_o(float* part, int64_t slot, int rows, int D) {
  return part + slot * partial_words(rows, D);
}
__device__ __forceinline__ float2* partial_ml(float* part, int64_t slot, int rows, int D) {
  return reinterpret_cast<float2*>(partial_o(part, slot, rows, D) + rows * D);
}

__device__ __forceinline__ RowNote row_note(int64_t slot, int n_chunks, int row, bool many) {
  RowNote x = {};
  if (slot >= 0) {
    x.where = (uint32_t)slot | (many ? 0x80000000u : 0u);
    x.what = (uint32_t)n_chunks | (uint32_t)row << 16;
  }
  return x;
}

// A row's log-sum-exp from its running maximum (in exp2 units) and sum.
__device__ __forceinline__ float row_lse(float m, float l) {
  return l > 0.f ? (float)((m + log2f(l)) * 0.6931471805599453) : l == 0.f ? -INFINITY : NAN;
}
__device__ __forceinline__ float row_scale(float l) { return l > 0.f ? 1.f / l : l == 0.f ? 0.f : NAN; }

}  // namespace dev
}  // namespace ckv
