// Device helpers of the attention kernels: waits, operand rounding, values that
// are not finite, and how a paged batch is cut into workgroups.
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

// exp2 of a logit's distance to the maximum. fp32 keeps weights below 2^-126,
// which the bare instruction flushes to zero.
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
// Chunks that a request's keys are cut into (one where it has none: its rows
// are written all the same).
__device__ __forceinline__ int paged_chunks(int n, int chunk) {
  return n <= chunk ? 1 : (n + chunk - 1) / chunk;
}

// Sum over the workgroup, for every thread of it.
template <int NT>
__device__ __forceinline__ int64_t block_sum(int64_t x, int64_t* part) {
#pragma unroll
  for (int i = 32; i > 0; i >>= 1) x += __shfl_xor(x, i);
  if ((threadIdx.x & 63) == 0) part[threadIdx.x >> 6] = x;
  __syncthreads();
  int64_t sum = 0;
#pragma unroll
  for (int i = 0; i < NT / 64; ++i) sum += part[i];
  __syncthreads();
  return sum;
}

// Keys per workgroup. Every workgroup of the batch's launches works this out for
// itself from the requests' lengths (the host knows bounds only). `work` is the
// sum of the keys over the `base` items (row tiles times KV heads) of a launch,
// `target` its workgroups in one round. An even share of work / target keys would
// leave up to one short workgroup per item over, in a second round; with
// work / (target - base) all fit into one. Past half a round of items the share
// would grow to more than twice the even one, and the even one stays. Shares are
// whole tiles of 64 keys and at least `least`.
constexpr int kUnsplit = 0x7FFFFFC0;
__device__ __forceinline__ int paged_share(int64_t work, int64_t base, int target, int least, bool split) {
  if (!split && 2 * base > target) return kUnsplit;
  const int64_t parts = 2 * base <= target ? target - base : target;
  const int64_t c = ((work + parts - 1) / parts + 63) / 64 * 64;
  return (int)(c < least ? least : c > kUnsplit ? kUnsplit : c);
}

struct PagedCut {
  int few, many;  // keys per workgroup of the two kernels
};
template <int NT>
__device__ __forceinline__ PagedCut paged_cut(const PagedArgs& A, int64_t* part) {
  int64_t few = 0, few_n = 0, many = 0, many_n = 0;
  for (int s = threadIdx.x; s < A.num_seqs; s += NT) {
    const PagedSeq q = paged_seq(A, s);
    if (q.T == 0) continue;
    if (paged_few(A, q)) {
      few += q.n;
      few_n += 1;
    } else {
      const int tiles = (q.T * A.a.G + kAttnRows - 1) / kAttnRows;
      many += (int64_t)tiles * q.n;
      many_n += tiles;
    }
  }
  PagedCut c = {};
  if (A.few_rows > 0) {
    // at most 4096 requests and 2^43 keys: both fit one number
    const int64_t f = block_sum<NT>(few * 8192 + few_n, part);
    c.few = paged_share((f >> 13) * A.a.n_kv, (f & 8191) * A.a.n_kv, A.few_target, kFewLeast, true);
  }
  if (A.has_many) {
    const int64_t m = block_sum<NT>(many, part), n = block_sum<NT>(many_n, part);
    c.many = paged_share(m * A.a.n_kv, n * A.a.n_kv, A.many_target, kManyLeast, false);
  }
  return c;
}

// The request that entry b of a list of requests' entries belongs to, with
// count(s, q) entries (x) each; and a second number (y) summed over the
// requests before it.
struct Found {
  int s, within;      // request, entry within it
  uint32_t before;    // sum of y
};
template <int NT, class Count>
__device__ __forceinline__ bool find_entry(const PagedArgs& A, int b, Count count, Found& f) {
  __shared__ uint32_t wsum[NT / 64];
  __shared__ int res[3];
  if (threadIdx.x == 0) res[0] = -1;
  uint32_t x0 = 0, y0 = 0;
  for (int s0 = 0; s0 < A.num_seqs; s0 += NT) {
    const int s = s0 + (int)threadIdx.x;
    uint2 c = make_uint2(0u, 0u);
    if (s < A.num_seqs) c = count(paged_seq(A, s));
    uint32_t x_all, y_all;
    const uint32_t x = x0 + block_excl_scan<NT>(c.x, wsum, x_all);
    const uint32_t y = y0 + block_excl_scan<NT>(c.y, wsum, y_all);
    if ((uint32_t)b >= x && (uint32_t)b - x < c.x) {
      res[0] = s;
      res[1] = (int)((uint32_t)b - x);
      res[2] = (int)y;
    }
    __syncthreads();
    if (res[0] >= 0) break;
    x0 += x_all;
    y0 += y_all;
  }
  f.s = __builtin_amdgcn_readfirstlane(res[0]);
  f.within = __builtin_amdgcn_readfirstlane(res[1]);
  f.before = (uint32_t)__builtin_amdgcn_readfirstlane(res[2]);
  return f.s >= 0;
}

// The factor of a partial result (maximum, sum) towards the maximum m: 0 for
// one without keys, 1 for one whose logits were all NaN.
__device__ __forceinline__ float part_weight(float2 x, float m) {
  return x.x == -INFINITY ? (x.y == 0.f ? 0.f : 1.f) : exp2f(x.x - m);
}

// Partial results of a split item, in its slot: `rows` rows of D floats, then
// their (maximum, sum) pairs.
__device__ __forceinline__ float* partial_o(float* part, int64_t slot, int rows, int D) {
  return part + slot * rows * (D + 2);
}
__device__ __forceinline__ float2* partial_ml(float* part, int64_t slot, int rows, int D) {
  return reinterpret_cast<float2*>(part + slot * rows * (D + 2) + rows * D);
}

// A row's log-sum-exp from its running maximum (in exp2 units) and sum.
__device__ __forceinline__ float row_lse(float m, float l) {
  return l > 0.f ? (float)((m + log2f(l)) * 0.6931471805599453) : l == 0.f ? -INFINITY : NAN;
}
__device__ __forceinline__ float row_scale(float l) { return l > 0.f ? 1.f / l : l == 0.f ? 0.f : NAN; }

}  // namespace dev
}  // namespace ckv
