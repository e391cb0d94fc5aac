// gfx950 (MI355X) attention of whole prompts and of new tokens over a paged
// cache: out = softmax(scale * Q K^T, causal) V with the rows' log-sum-exp.
//
// A workgroup takes a tile of query rows of one KV head g: row r of a request
// is token r / G, head g * G + r % G, so the G heads that share K and V are
// neighbouring rows and K and V are read once for all of them. Every wave owns
// 32 rows and walks the keys tile by tile, all waves together: K and V tiles go
// from memory straight into LDS (the next tile's while this one is reduced).
// Per tile: S^T = K Q^T with MFMA, which leaves each query row's logits in two
// lanes; the running maximum and sum of the softmax; O^T += V^T P^T with MFMA,
// whose P operand is the lane's own logits in place. V is transposed on the
// way out of LDS (ds_read_b64_tr_b16).
//
// What bounds it: a wave and tile of 64 keys (bf16, d 128) take 1024 cycles of the
// matrix units and about 950 of the vector units (528 of them the 32 exponentials),
// and the two waves of a SIMD hardly overlap the one with the other: 4200
// cycles per tile of 256 rows. 32768 tokens of 32 heads over 8 take 8.2 to 8.6 ms
// by the card, 1.02 to 1.07 PFLOP/s, where a library product of 8192^3 reaches 1.22. Running the second
// four waves half a step behind the first, so that one half multiplies while
// the other works out its weights, took 9.0 ms; alternating the two chains of
// QK^T made no difference.
#include <math.h>

#include <type_traits>

#include "ckv_attn_device.h"

namespace ckv {
namespace {

using namespace dev;

// A workgroup's part of the call: T query tokens from row tok0 on that are the
// last of n keys, KV head g, row tile rt.
struct Item {
  int tok0, T, n, g, rt;
  int j0, j1;            // its keys of the n: all, or a chunk
  int slot;              // where its partial result goes, -1 where the keys are not split
  int n_chunks;
  const int32_t* table;  // paged: the request's block table
};

template <int ROWS>
__device__ __forceinline__ bool find_item(const PrefillArgs& A, Item& it) {
  const PromptTile p = prompt_tile(A);
  it.tok0 = p.tok0;
  it.T = it.n = p.T;
  it.g = p.g;
  it.rt = p.rt;
  it.j0 = 0;
  it.j1 = it.n;
  it.slot = -1;
  it.n_chunks = 1;
  it.table = nullptr;
  return true;
}

template <int ROWS>
__device__ __forceinline__ bool find_item(const PagedArgs& A, Item& it) {
  static_assert(ROWS == kAttnRows, "tiles as many_share counts them");
  const int b = (int)blockIdx.x / A.a.n_kv;
  it.g = (int)blockIdx.x - b * A.a.n_kv;
  const PagedSeq first = lane_seq(A, threadIdx.x & 63);
  const int chunk = many_share(A, first);
  auto tiles = [&](const PagedSeq& q) { return (q.T * A.a.G + ROWS - 1) / ROWS; };
  Found f;
  if (!find_entry(A, first, b, [&](const PagedSeq& q) {
        return make_uint2(paged_few(A, q) ? 0u : (uint32_t)(tiles(q) * paged_chunks(q.n, chunk)), 0u);
      }, f))
    return false;
  const PagedSeq q = f.q;
  const int n_chunks = paged_chunks(q.n, chunk), back = f.within / n_chunks, c = f.within - back * n_chunks;
  it.tok0 = q.tok0;
  it.T = q.T;
  it.n = q.n;
  it.rt = tiles(q) - 1 - back;
  it.j0 = c * chunk;
  it.j1 = paged_chunk_end(q.n, chunk, c);
  it.slot = n_chunks > 1 ? (int)blockIdx.x : -1;
  it.n_chunks = n_chunks;
  it.table = A.table + (int64_t)f.s * A.table_stride;
  return true;
}

// How a pass over the tiles treats values that are not finite.
enum Pass { kPlain, kStripped, kLeftOut };

template <int DT, int D, int NW, bool PAGED, class Args>
__global__ __launch_bounds__(NW * 64) __attribute__((amdgpu_waves_per_eu(2)))
void attn_kernel(const Args A) {
  constexpr int EB = Elt<DT>::bytes;
  constexpr int ROWB = D * EB;            // bytes per K or V row
  constexpr int NV = ROWB / 16;           // 16-byte chunks per row: 8, 16 or 32
  constexpr int NC = NV / 2;              // operand chunks per lane
  constexpr int KT = DT == 2 ? 32 : 64;   // keys per tile
  constexpr int KB = KT / 32;             // 32-key blocks of it
  constexpr int VEC = KT * NV;            // 16-byte chunks per tile
  constexpr int PT = VEC / 64 / NW;       // load instructions per wave and tile, for K and V each
  constexpr int RPL = 64 / NV;            // tile rows per load instruction
  constexpr int NB = D / 32;
  constexpr int ROWS = NW * 32;
  static_assert(PT >= 1 && VEC % (64 * NW) == 0, "tile loads");
  constexpr uint64_t kAll = KT == 64 ? ~0ull : 0xFFFFFFFFull;
  constexpr float kBias = DT == 1 ? kF16Bias : 0.f;
  __shared__ uint4 k0[VEC], k1[VEC];  // chunk c of row t at position c ^ swz(t), V's at c ^ vswz(t)
  __shared__ uint4 v0[VEC], v1[VEC];
  const int tid = threadIdx.x, lane = tid & 63, h = lane >> 5, l32 = lane & 31;
  const int wave = __builtin_amdgcn_readfirstlane(tid >> 6);
  Item it;
  if (!find_item<ROWS>(A, it)) return;
  const AttnArgs& a = A.a;
  const int G = a.G, R = it.T * G;
  // this lane's query row (column of S^T and O^T); row r sees keys 0..limit
  const int first = it.rt * ROWS + wave * 32;        // of the wave
  const int shift = it.n - it.T;
  const bool active = first < R;
  const int r = first + l32;
  const bool row_ok = r < R;
  const int rc = row_ok ? r : R - 1;
  const int t = rc / G, head = it.g * G + rc - t * G;
  const int limit = shift + t;
  const int lim_lo = shift + (active ? first / G : 0);               // the wave's first row's
  const int lim_hi = active ? shift + (first + 31 < R ? first + 31 : R - 1) / G : -1;
  const int last_row = it.rt * ROWS + ROWS - 1 < R ? it.rt * ROWS + ROWS - 1 : R - 1;
  const int keys = min(shift + last_row / G + 1, it.j1);  // seen by the tile's last row
  const int tl0 = it.j0 / KT;                        // chunks are whole tiles
  const int nt = keys > it.j0 ? (keys + KT - 1) / KT : tl0;

  auto swz = [](int row) { return ROWB >= 256 ? (row & 15) : ((row >> 1) & 7); };
  // V of 16-bit types is read 4 keys of 64 bytes at a time, which meet every bank once if
  // they lie in different quarters of the 256 bytes (with K's swizzle, 59% of the LDS
  // cycles were bank conflicts and a prompt of 8192 tokens took 574 us, not 542);
  // rows of fp32 are read along their columns, which does as it is
  auto vswz = [&](int row) { return DT == 2 ? 0 : ROWB >= 256 ? (row & 3) * 4 : (row & 2) * 2; };
  const int lrow = lane / NV, lpos = lane % NV;
  const char* kbase = a.k + (int64_t)it.g * a.kv_sh;
  const char* vbase = a.v + (int64_t)it.g * a.kv_sh;
  if constexpr (!PAGED) {
    kbase += (int64_t)it.tok0 * a.kv_st;
    vbase += (int64_t)it.tok0 * a.kv_st;
  }
  // paged: the page of this lane's key of tile tl, -1 for keys that are not there
  auto page_of = [&](int tl) {
    int id = -1;
    if constexpr (PAGED) {
      const int key = tl * KT + (lane & (KT - 1));
      if (key < it.j1) {
        const int p = page_at(A.div, key);
        if ((uint32_t)p < (uint32_t)A.table_width) id = to_global(it.table)[p];
        if ((uint32_t)id >= (uint32_t)A.n_pages) id = -1;
      }
    }
    return id;
  };
  // the keys of tile tl that are there
  auto there = [&](int tl, int page) -> uint64_t {
    if constexpr (PAGED) return __ballot(page >= 0) & kAll;
    const int left = it.n - tl * KT;
    return left >= KT ? kAll : (1ull << left) - 1;
  };
  // Requests a tile's rows of K or V. Keys that are not there read some valid row.
  auto fetch_one = [&](const char* base, int tl, int page, uint4* dst, auto swizzle) {
#pragma unroll
    for (int i = 0; i < PT; ++i) {
      const int row = (i * NW + wave) * RPL + lrow;  // of the tile
      int64_t off;
      if constexpr (PAGED) {
        const int key = tl * KT + row;
        const int id = __shfl(page, row);
        const int p = page_at(A.div, key);
        const int slot = key - p * A.page_size;
        off = (int64_t)(id < 0 ? 0 : id) * A.kv_sp + (int64_t)slot * a.kv_st;
      } else {
        const int key = tl * KT + row < it.n ? tl * KT + row : it.n - 1;
        off = (int64_t)key * a.kv_st;
      }
      __builtin_amdgcn_global_load_lds(reinterpret_cast<const uint4*>(base + off + (lpos ^ swizzle(row)) * 16),
                                       dst + (i * NW + wave) * 64, 16, 0, 0);
    }
  };
  auto fetch = [&](int tl, int page, uint4* ks, uint4* vs) {
    fetch_one(kbase, tl, page, ks, swz);
    fetch_one(vbase, tl, page, vs, vswz);
  };
  // Keys that are not there count as zeros in V: for the rows that this wave requested.
  auto clear_v = [&](uint64_t seen, uint4* vs) {
    if (seen == kAll) return;
#pragma unroll
    for (int i = 0; i < PT; ++i) {
      const int row = (i * NW + wave) * RPL + lrow;
      if (!((seen >> row) & 1)) vs[(i * NW + wave) * 64 + lane] = make_uint4(0u, 0u, 0u, 0u);
    }
    wait_vm<0>();
  };

  // lane half h holds chunks 2c + h of its query row
  uint4 q[NC];
  {
    const CKV_GLOBAL u32x4* src =
        (const CKV_GLOBAL u32x4*)(to_global(a.q) + (int64_t)(it.tok0 + t) * a.q_st +
                                  (int64_t)head * a.q_sh) + h;
#pragma unroll
    for (int c = 0; c < NC; ++c) {
      const u32x4 x = src[2 * c];
      q[c] = make_uint4(x.x, x.y, x.z, x.w);
    }
  }
  const float alpha = a.alpha;
  const int i16 = lane & 15;
  // V^T operand of columns nb * 32 .. + 31 and the 16 keys of MFMA step km: lane i
  // of a 16-lane group reads columns 4 * (i % 4) .. + 3 of key 8 * jj + 4 * h + i / 4,
  // and receives column i of the 4 keys
  auto v_chunk = [&](const char* vt, int nb, int km) {
    uint2 part[2];
#pragma unroll
    for (int jj = 0; jj < 2; ++jj) {
      typedef __attribute__((address_space(3))) s16x4* LdsPtr;
      const int key = 8 * jj + 4 * h + (i16 >> 2);
      const int col = nb * 32 + (lane & 16) + 4 * (i16 & 3);
      const int at = key * ROWB + ((col >> 3) ^ vswz(key)) * 16 + (col & 7) * 2;
      part[jj] = __builtin_bit_cast(uint2, __builtin_amdgcn_ds_read_tr16_b64_v4i16((LdsPtr)(vt + at + km * 16 * ROWB)));
    }
    return make_uint4(part[0].x, part[0].y, part[1].x, part[1].y);
  };
  auto v_elem = [&](const char* vt, int nb, int v) {
    return *reinterpret_cast<const float*>(vt + acc_row(v, h) * ROWB + (nb * 32 + l32) * 4);
  };

  f32x16 o[NB];
  float m_run, l_run;
  // S^T = K Q^T of a tile
  auto logits = [&](const uint4* ks, f32x16 (&s)[KB]) {
#pragma unroll
    for (int kb = 0; kb < KB; ++kb) {
      __builtin_amdgcn_sched_barrier(0);
      s[kb] = f32x16{};
#pragma unroll
      for (int c = 0; c < NC; ++c)
        s[kb] = mfma_chunk<DT>(ks[(kb * 32 + l32) * NV + ((2 * c + h) ^ swz(l32))], q[c], s[kb]);
    }
    __builtin_amdgcn_sched_barrier(0);
  };
  // logits to weights, with the keys `sees` (if `hides`), and the running maximum and sum
  auto weights = [&](f32x16 (&s)[KB], bool hides, uint64_t sees) {
    if (hides) {
#pragma unroll
      for (int kb = 0; kb < KB; ++kb) {
        const uint32_t bits = (uint32_t)(sees >> (32 * kb)) >> (4 * h);
#pragma unroll
        for (int v = 0; v < 16; ++v)
          if (!(bits & (1u << acc_row(v, 0)))) s[kb][v] = -INFINITY;
      }
    }
    float mx = s[0][0];
#pragma unroll
    for (int kb = 0; kb < KB; ++kb)
#pragma unroll
      for (int v = 0; v < 16; ++v) mx = fmaxf(mx, s[kb][v]);
    mx = fmaxf(mx, __shfl_xor(mx, 32)) * alpha;
    if (__any(mx > m_run + kSlack)) {
      const float m_new = fmaxf(m_run, mx);
      const float resc = m_run == -INFINITY ? 0.f : weight_exp2<DT>(m_run - m_new);
      l_run *= resc;
#pragma unroll
      for (int nb = 0; nb < NB; ++nb) o[nb] *= resc;
      m_run = m_new;
    }
    const float ms = m_run == -INFINITY ? 0.f : m_run - kBias;
    float psum = 0.f;
#pragma unroll
    for (int kb = 0; kb < KB; ++kb)
#pragma unroll
      for (int v = 0; v < 16; ++v) {
        s[kb][v] = weight_exp2<DT>(fmaf(s[kb][v], alpha, -ms));
        psum += s[kb][v];
      }
    l_run += psum;
  };
  // the keys of tile tl, of which `vis` are there, that this lane's row sees, one bit each
  auto seen_keys = [&](int tl, uint64_t vis, bool& hides) {
    const int rel = limit - tl * KT;
    hides = vis != kAll || tl * KT + KT - 1 > lim_lo;
    uint64_t sees = vis;
    if (hides && rel < KT - 1) sees &= rel < 0 ? 0 : (2ull << rel) - 1;
    return sees;
  };
  // P^T operands: MFMA step km takes this lane's keys acc_row(8km .. 8km+7, h)
  // = 16km + 4h + (0..3) and 16km + 8 + 4h + (0..3), in that order
  // Rounded once to the type: a second product for the rounding's remainders took 12.0 ms
  // in place of 8.6 for 32768 tokens and 775 us in place of 562 for 8192, and brought the
  // relative error of bf16 outputs from 2.1e-3 to the 1.6e-3 of their own rounding
  auto p_chunk = [&](const f32x16 (&s)[KB], int km) {
    float p[8];
#pragma unroll
    for (int i = 0; i < 8; ++i) p[i] = s[km >> 1][8 * (km & 1) + i];
    return round_chunk<DT>(p);
  };
  auto not_finite = [&]() {
    float bad = 0.f;
#pragma unroll
    for (int nb = 0; nb < NB; ++nb)
#pragma unroll
      for (int v = 0; v < 16; ++v) bad = fmaf(o[nb][v], 0.f, bad);
    return active && bad != 0.f;
  };
  // A row's hidden keys have weight 0, but 0 times a value that is not finite
  // is not 0. If an output came out not finite, the tiles are taken again, first
  // without such values, then for what every row sees of them.
  auto pass = [&](auto mode) {
    constexpr Pass MODE = decltype(mode)::value;
    if constexpr (MODE != kLeftOut) {
#pragma unroll
      for (int nb = 0; nb < NB; ++nb) o[nb] = f32x16{};
      m_run = -INFINITY;
      l_run = 0.f;
    }
    int page = page_of(tl0);
    uint64_t seen = nt > tl0 ? there(tl0, page) : 0;
    if (nt > tl0) fetch(tl0, page, k0, v0);
    page = page_of(tl0 + 1);
    auto step = [&](int tl, uint4* ks, uint4* vs, uint4* ks_next, uint4* vs_next) {
      wait_vm<0>();  // this wave's part of the tile
      clear_v(seen, vs);
      barrier();
      const uint64_t vis = seen;
      if (tl + 1 < nt) {
        seen = there(tl + 1, page);
        fetch(tl + 1, page, ks_next, vs_next);
        page = page_of(tl + 2);
      }
      const int j0 = tl * KT;
      if (!active || j0 > lim_hi) return;
      bool hides;
      const uint64_t sees = seen_keys(tl, vis, hides);
      const char* vt = reinterpret_cast<const char*>(vs);
      if constexpr (MODE == kLeftOut) {
#pragma unroll
        for (int nb = 0; nb < NB; ++nb) {
          f32x16 c = f32x16{};
          if constexpr (DT != 2) {
#pragma unroll
            for (int km = 0; km < KB * 2; ++km) {
              uint4 x;
              strip_chunk<DT>(v_chunk(vt, nb, km), x);
              c = mfma_chunk<DT>(x, seen_chunk<DT>((uint32_t)(sees >> (16 * km)) >> (4 * h)), c);
            }
          } else {
#pragma unroll
            for (int v = 0; v < 16; ++v) {
              float x;
              strip_f32(v_elem(vt, nb, v), x);
              c = mfma_f32(x, (sees >> acc_row(v, h)) & 1 ? 1.f : 0.f, c);
            }
          }
#pragma unroll
          for (int v = 0; v < 16; ++v) o[nb][v] += stripped_sum(c[v]);
          __builtin_amdgcn_sched_barrier(0);
        }
        return;
      }
      f32x16 s[KB];
      logits(ks, s);
      weights(s, hides, sees);
      if constexpr (DT != 2) {
#pragma unroll
        for (int km = 0; km < KB * 2; ++km) {
          __builtin_amdgcn_sched_barrier(0);
          const uint4 ph = p_chunk(s, km);
#pragma unroll
          for (int nb = 0; nb < NB; ++nb) {
            uint4 x, va = v_chunk(vt, nb, km);
            if constexpr (MODE == kStripped) va = strip_chunk<DT>(va, x);
            o[nb] = mfma_chunk<DT>(va, ph, o[nb]);
          }
        }
      } else {
#pragma unroll
        for (int v = 0; v < 16; ++v) {
          if (v % 4 == 0) __builtin_amdgcn_sched_barrier(0);
#pragma unroll
          for (int nb = 0; nb < NB; ++nb) {
            float x, va = v_elem(vt, nb, v);
            if constexpr (MODE == kStripped) va = strip_f32(va, x);
            o[nb] = mfma_f32(va, s[0][v], o[nb]);
          }
        }
      }
    };
    for (int tl = tl0; tl < nt; tl += 2) {
      step(tl, k0, v0, k1, v1);
      if (tl + 1 < nt) step(tl + 1, k1, v1, k0, v0);
    }
    return not_finite();
  };
  if (__syncthreads_or(pass(std::integral_constant<Pass, kPlain>()))) {
    pass(std::integral_constant<Pass, kStripped>());
    __syncthreads();
    pass(std::integral_constant<Pass, kLeftOut>());
  }
  if (!row_ok) return;
  const float l = l_run + __shfl_xor(l_run, 32);
  if constexpr (PAGED) {
    const int row = wave * 32 + l32;
    if (A.notes && h == 0 && it.j0 == 0)
      A.notes[(int64_t)(it.tok0 + t) * a.H + head] = row_note(it.slot, it.n_chunks, row, true);
    if (it.slot >= 0) {
      float* orow = partial_o(A.part_many, it.slot, ROWS, D) + row * D;
#pragma unroll
      for (int nb = 0; nb < NB; ++nb)
#pragma unroll
        for (int v = 0; v < 16; v += 4)
          *reinterpret_cast<f32x4*>(orow + nb * 32 + acc_row(v, h)) =
              f32x4{o[nb][v], o[nb][v + 1], o[nb][v + 2], o[nb][v + 3]};
      if (h == 0) partial_ml(A.part_many, it.slot, ROWS, D)[row] = make_float2(m_run - kBias, l);
      return;
    }
  }
  const float inv = row_scale(l);
  char* dst = a.out + (int64_t)(it.tok0 + t) * a.o_st + (int64_t)head * a.o_sh;
#pragma unroll
  for (int nb = 0; nb < NB; ++nb)
#pragma unroll
    for (int v = 0; v < 16; v += 4)
      store4<DT>(dst + (nb * 32 + acc_row(v, h)) * EB, o[nb][v] * inv, o[nb][v + 1] * inv,
                 o[nb][v + 2] * inv, o[nb][v + 3] * inv);
  if (a.lse && h == 0) a.lse[(int64_t)head * a.lse_sh + it.tok0 + t] = row_lse(m_run - kBias, l);
}

template <bool PAGED, class Args>
hipError_t launch_attn(int dtype, int d, const Args& A, int grid, hipStream_t st) {
  if (grid == 0) return hipSuccess;
  const Timing none;
  if (d == 128) {
    if (dtype == CKV_BF16) return launch(attn_kernel<0, 128, 8, PAGED, Args>, grid, 512, st, none, A);
    if (dtype == CKV_F16) return launch(attn_kernel<1, 128, 8, PAGED, Args>, grid, 512, st, none, A);
    return launch(attn_kernel<2, 128, 8, PAGED, Args>, grid, 512, st, none, A);
  }
  if (dtype == CKV_BF16) return launch(attn_kernel<0, 64, 8, PAGED, Args>, grid, 512, st, none, A);
  if (dtype == CKV_F16) return launch(attn_kernel<1, 64, 8, PAGED, Args>, grid, 512, st, none, A);
  return launch(attn_kernel<2, 64, 8, PAGED, Args>, grid, 512, st, none, A);
}

}  // namespace

hipError_t launch_prefill(int dtype, int d, const PrefillArgs& p, int grid, hipStream_t st) {
  return launch_attn<false>(dtype, d, p, grid, st);
}
hipError_t launch_paged_many(int dtype, int d, const PagedArgs& p, int grid, hipStream_t st) {
  return launch_attn<true>(dtype, d, p, grid, st);
}

}  // namespace ckv
