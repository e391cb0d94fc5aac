// gfx950 (MI355X) attention of few new tokens per request over a paged cache
// (decoding steps), and the join of what is split along the keys.
//
// paged_few_kernel: up to 32 query rows (a KV head's G heads x T tokens), a
//   workgroup per (request, KV head, chunk of its keys). A cache row is read
//   once, so the bound is the stream, and what counts is how much of it is in
//   flight: every wave owns 32-key tiles, whose K and V go from memory straight
//   into the wave's part of LDS, the next tile's K requested as soon as this
//   one's is in registers (the same for V), with no barrier between waves. The
//   waves' results meet in LDS.
// paged_merge_kernel: the chunks' partial results (of this kernel and of the tile
//   kernel) rescaled to the common maximum and added in order.
#include <math.h>

#include "ckv_attn_device.h"

namespace ckv {
namespace {

using namespace dev;

template <int DT, int D>
__global__ __launch_bounds__(kThreads) __attribute__((amdgpu_waves_per_eu(DT == 2 ? 1 : 2)))
void paged_few_kernel(const PagedArgs A) {
  constexpr int EB = Elt<DT>::bytes;
  constexpr int ROWB = D * EB;       // bytes per cache row
  constexpr int NV = ROWB / 16;      // 16-byte chunks per row: 8, 16 or 32
  constexpr int NC = NV / 2;         // operand chunks per lane
  constexpr int KT = 32;             // keys per tile
  constexpr int VEC = KT * NV;       // 16-byte chunks per tile
  constexpr int PT = VEC / 64;       // load instructions per tile
  constexpr int RPL = 64 / NV;       // tile rows per load instruction
  constexpr int NB = D / 32;
  constexpr float kBias = DT == 1 ? kF16Bias : 0.f;
  __shared__ uint4 kl[kWaves][VEC];  // chunk c of row t at position c ^ swz(t), V's at c ^ vswz(t)
  __shared__ uint4 vl[kWaves][VEC];
  __shared__ float2 ml[kWaves][32];
  __shared__ int64_t sums[kWaves];
  const AttnArgs& a = A.a;
  const int tid = threadIdx.x, lane = tid & 63, h = lane >> 5, l32 = lane & 31;
  const int wave = __builtin_amdgcn_readfirstlane(tid >> 6);
  const int b = (int)blockIdx.x / a.n_kv, g = (int)blockIdx.x - b * a.n_kv;
  const int chunk = paged_cut<kThreads>(A, sums).few;
  Found f;
  if (!find_entry<kThreads>(A, b, [&](const PagedSeq& q) {
        const uint32_t n = q.T > 0 && paged_few(A, q) ? paged_chunks(q.n, chunk) : 0;
        return make_uint2(n, n > 1 ? n : 0);
      }, f))
    return;
  const PagedSeq sq = paged_seq(A, f.s);
  const int n_chunks = paged_chunks(sq.n, chunk);
  const int32_t* table = A.table + (int64_t)f.s * A.table_stride;
  const int G = a.G, R = sq.T * G;
  const int j0 = f.within * chunk;
  const int j1 = n_chunks == 1 || sq.n - j0 < chunk ? sq.n : j0 + chunk;
  const int nt = (j1 - j0 + KT - 1) / KT;
  const char* kbase = a.k + (int64_t)g * a.kv_sh;
  const char* vbase = a.v + (int64_t)g * a.kv_sh;
  const float alpha = a.alpha;

  auto swz = [](int t) { return ROWB >= 256 ? (t & 15) : ((t >> 1) & 7); };
  // V rows of fp32 are read along their columns, which meets every bank as it is
  auto vswz = [&](int t) { return DT == 2 ? 0 : swz(t); };
  const int lrow = lane / NV, lpos = lane % NV;
  // the page of key l32 of tile tl, -1 for keys that are not there
  auto page_of = [&](int tl) {
    const int key = j0 + tl * KT + l32;
    int id = -1;
    if (key < j1) {
      const int p = page_at(A.div, key);
      if (p < A.table_width) id = to_global(table)[p];
      if ((uint32_t)id >= (uint32_t)A.n_pages) id = -1;
    }
    return id;
  };
  // tile tl of base: non-temporal, each cache row is read once. Keys that are not
  // there read a row of page 0.
  auto fetch = [&](const char* base, int tl, int page, uint4* slot, auto swizzle) {
#pragma unroll
    for (int i = 0; i < PT; ++i) {
      const int t = i * RPL + lrow, key = j0 + tl * KT + t;
      const int id = __shfl(page, t);
      const int64_t off = (int64_t)(id < 0 ? 0 : id) * A.kv_sp +
                          (int64_t)(key - page_at(A.div, key) * A.page_size) * a.kv_st;
      __builtin_amdgcn_global_load_lds(
          reinterpret_cast<const uint4*>(base + off + (lpos ^ swizzle(t)) * 16), slot + i * 64, 16, 0, 2);
    }
  };
  // query row r = token * G + head; lane half h holds chunks 2c + h of it
  const int r = l32 < R ? l32 : R - 1;
  const int t = r / G, limit = sq.n - sq.T + t;
  uint4 q[NC];
  {
    const CKV_GLOBAL u32x4* src =
        (const CKV_GLOBAL u32x4*)(to_global(a.q) + (int64_t)(sq.tok0 + t) * a.q_st +
                                  (int64_t)(g * G + r - t * G) * a.q_sh) + h;
#pragma unroll
    for (int c = 0; c < NC; ++c) {
      const u32x4 x = src[2 * c];
      q[c] = make_uint4(x.x, x.y, x.z, x.w);
    }
  }
  int tile = wave;
  int page = page_of(tile), page_next = page_of(tile + kWaves);
  if (tile < nt) {
    fetch(kbase, tile, page, kl[wave], swz);
    fetch(vbase, tile, page, vl[wave], vswz);
  }

  f32x16 o[NB];
#pragma unroll
  for (int nb = 0; nb < NB; ++nb) o[nb] = f32x16{};
  float m_run = -INFINITY, l_run = 0.f;  // the maximum in exp2 units
  // lane i of a 16-lane group reads columns 4 * (i % 4) .. + 3 of key
  // 8 * jj + 4 * h + i / 4, and receives column i of the 4 keys
  const int i16 = lane & 15;
  auto v_chunk = [&](const char* vt, int nb, int m) {
    uint2 part[2];
#pragma unroll
    for (int jj = 0; jj < 2; ++jj) {
      typedef __attribute__((address_space(3))) s16x4* LdsPtr;
      const int key = 8 * jj + 4 * h + (i16 >> 2);
      const int col = nb * 32 + (lane & 16) + 4 * (i16 & 3);
      const int at = key * ROWB + ((col >> 3) ^ vswz(key)) * 16 + (col & 7) * 2;
      part[jj] = __builtin_bit_cast(uint2, __builtin_amdgcn_ds_read_tr16_b64_v4i16((LdsPtr)(vt + at + m * 16 * ROWB)));
    }
    return make_uint4(part[0].x, part[0].y, part[1].x, part[1].y);
  };
  auto v_elem = [&](const char* vt, int nb, int v) {
    return *reinterpret_cast<const float*>(vt + acc_row(v, h) * ROWB + (nb * 32 + l32) * 4);
  };

  for (; tile < nt; tile += kWaves) {
    const bool more = tile + kWaves < nt;
    wait_vm<PT>();  // this tile's K; its V may still be on the way
    uint4 kr[NC];
#pragma unroll
    for (int c = 0; c < NC; ++c) kr[c] = kl[wave][l32 * NV + ((2 * c + h) ^ swz(l32))];
    wait_vm<63>();  // K is in registers: its part of LDS is free
    const uint32_t vis = (uint32_t)__ballot(page >= 0);  // the keys that are there
    page = page_next;
    page_next = page_of(tile + 2 * kWaves);
    if (more) fetch(kbase, tile + kWaves, page, kl[wave], swz);
    // the keys that this lane's row sees, one bit each
    const int first = j0 + tile * KT, rel = limit - first;
    const uint32_t sees = rel >= KT - 1 ? vis : rel < 0 ? 0u : vis & ((2u << rel) - 1u);
    const bool hides = __any(sees != ~0u);
    f32x16 s = f32x16{};
#pragma unroll
    for (int c = 0; c < NC; ++c) s = mfma_chunk<DT>(kr[c], q[c], s);
    if (hides) {
      const uint32_t bits = sees >> (4 * h);
#pragma unroll
      for (int v = 0; v < 16; ++v)
        if (!(bits & (1u << acc_row(v, 0)))) s[v] = -INFINITY;
    }
    float mx = s[0];
#pragma unroll
    for (int v = 1; v < 16; ++v) mx = fmaxf(mx, s[v]);
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
    for (int v = 0; v < 16; ++v) {
      s[v] = weight_exp2<DT>(fmaf(s[v], alpha, -ms));
      psum += s[v];
    }
    l_run += psum;
    if (more) wait_vm<PT>();  // this tile's V; the next K may still be on the way
    else wait_vm<0>();
    if (vis != ~0u) {  // keys that are not there count as zeros
#pragma unroll
      for (int i = 0; i < PT; ++i)
        if (!((vis >> (i * RPL + lrow)) & 1)) vl[wave][i * 64 + lane] = make_uint4(0u, 0u, 0u, 0u);
      wait_vm<63>();
    }
    const char* vt = reinterpret_cast<const char*>(vl[wave]);
    // A hidden key's weight is 0, but 0 times a value that is not finite is not:
    // where keys are hidden such values are left out of the product, and what a
    // row sees of them is added.
    if constexpr (DT != 2) {
      // P^T operands: MFMA step m takes this lane's keys acc_row(8m .. 8m+7, h)
      // = 16m + 4h + (0..3) and 16m + 8 + 4h + (0..3), in that order
      uint4 vr[2][NB];
#pragma unroll
      for (int m = 0; m < 2; ++m)
#pragma unroll
        for (int nb = 0; nb < NB; ++nb) vr[m][nb] = v_chunk(vt, nb, m);
      wait_vm<63>();  // V is in registers
      if (more) fetch(vbase, tile + kWaves, page, vl[wave], vswz);
      uint4 ph[2];
#pragma unroll
      for (int m = 0; m < 2; ++m) {
        float p[8];
#pragma unroll
        for (int i = 0; i < 8; ++i) p[i] = s[8 * m + i];
        ph[m] = round_chunk<DT>(p);
      }
      if (hides) {
#pragma unroll
        for (int nb = 0; nb < NB; ++nb) {
          f32x16 c = f32x16{};
#pragma unroll
          for (int m = 0; m < 2; ++m) {
            uint4 x;
            vr[m][nb] = strip_chunk<DT>(vr[m][nb], x);
            c = mfma_chunk<DT>(x, seen_chunk<DT>((sees >> (16 * m)) >> (4 * h)), c);
          }
#pragma unroll
          for (int v = 0; v < 16; ++v) o[nb][v] += stripped_sum(c[v]);
        }
      }
#pragma unroll
      for (int m = 0; m < 2; ++m)
#pragma unroll
        for (int nb = 0; nb < NB; ++nb) o[nb] = mfma_chunk<DT>(vr[m][nb], ph[m], o[nb]);
    } else {
      float vr[16][NB];
#pragma unroll
      for (int v = 0; v < 16; ++v)
#pragma unroll
        for (int nb = 0; nb < NB; ++nb) vr[v][nb] = v_elem(vt, nb, v);
      wait_vm<63>();
      if (more) fetch(vbase, tile + kWaves, page, vl[wave], vswz);
      if (hides) {
#pragma unroll
        for (int nb = 0; nb < NB; ++nb) {
          f32x16 c = f32x16{};
#pragma unroll
          for (int v = 0; v < 16; ++v) {
            float x;
            vr[v][nb] = strip_f32(vr[v][nb], x);
            c = mfma_f32(x, (sees >> acc_row(v, h)) & 1 ? 1.f : 0.f, c);
          }
#pragma unroll
          for (int v = 0; v < 16; ++v) o[nb][v] += stripped_sum(c[v]);
        }
      }
#pragma unroll
      for (int v = 0; v < 16; ++v)
#pragma unroll
        for (int nb = 0; nb < NB; ++nb) o[nb] = mfma_f32(vr[v][nb], s[v], o[nb]);
    }
  }

  // the waves' results, rescaled to the common maximum and added in wave order
  // through the tiles' LDS. A wave's O^T (32 rows of D floats) fills its K and V
  // parts when elements are 2 bytes (columns below and from D / 2), its K part
  // when they are 4. 16-byte chunks of row r are XOR-ed with r % 8.
  constexpr int OC = EB == 2 ? D / 8 : D / 4;  // 16-byte chunks of a row in one part
  __syncthreads();
  const float l = l_run + __shfl_xor(l_run, 32);
  if (h == 0) ml[wave][l32] = make_float2(m_run, l);
#pragma unroll
  for (int nb = 0; nb < NB; ++nb)
#pragma unroll
    for (int v4 = 0; v4 < 4; ++v4) {
      const int c = nb * 8 + v4 * 2 + h;  // chunk of the row: columns 4c .. 4c + 3
      float4* part = reinterpret_cast<float4*>(c < OC ? kl[wave] : vl[wave]);
      part[l32 * OC + ((c % OC) ^ (l32 & 7))] =
          make_float4(o[nb][4 * v4], o[nb][4 * v4 + 1], o[nb][4 * v4 + 2], o[nb][4 * v4 + 3]);
    }
  __syncthreads();
  const int64_t slot = (int64_t)f.before * a.n_kv + (int64_t)g * n_chunks + f.within;
  for (int e = tid; e < R * (D / 4); e += kThreads) {
    const int rr = e / (D / 4), c = e - rr * (D / 4);
    float m = ml[0][rr].x;
#pragma unroll
    for (int w = 1; w < kWaves; ++w) m = fmaxf(m, ml[w][rr].x);
    float ls = 0.f;
    float4 acc = make_float4(0.f, 0.f, 0.f, 0.f);
#pragma unroll
    for (int w = 0; w < kWaves; ++w) {
      const float2 x = ml[w][rr];
      const float fct = part_weight(x, m);
      const float4* part = reinterpret_cast<const float4*>(c < OC ? kl[w] : vl[w]);
      const float4 y = part[rr * OC + ((c % OC) ^ (rr & 7))];
      ls += x.y * fct;
      acc.x += y.x * fct;
      acc.y += y.y * fct;
      acc.z += y.z * fct;
      acc.w += y.w * fct;
    }
    if (n_chunks > 1) {
      *reinterpret_cast<float4*>(partial_o(A.part, slot, A.few_rows, D) + rr * D + 4 * c) = acc;
      if (c == 0) partial_ml(A.part, slot, A.few_rows, D)[rr] = make_float2(m - kBias, ls);
    } else {
      const int tt = rr / G, head = g * G + rr - tt * G;
      const float inv = row_scale(ls);
      store4<DT>(a.out + (int64_t)(sq.tok0 + tt) * a.o_st + (int64_t)head * a.o_sh + 4 * c * EB,
                 acc.x * inv, acc.y * inv, acc.z * inv, acc.w * inv);
      if (c == 0 && a.lse) a.lse[(int64_t)head * a.lse_sh + sq.tok0 + tt] = row_lse(m - kBias, ls);
    }
  }
}

// One row of a request of few rows (all thread groups of D / 4 lanes share its
// chunks), or a thread group per row of the others.
template <int DT, int D>
__global__ __launch_bounds__(kThreads) void paged_merge_kernel(const PagedArgs A) {
  constexpr int C4 = D / 4, NG = kThreads / C4, U = 8;
  constexpr int EB = Elt<DT>::bytes;
  __shared__ float4 acc_l[NG][C4];
  __shared__ float2 ml_l[NG];
  __shared__ int64_t sums[kWaves];
  const AttnArgs& a = A.a;
  const int grp = threadIdx.x / C4, c = threadIdx.x % C4;
  const PagedCut cut = paged_cut<kThreads>(A, sums);
  // entries are this launch's workgroups; y counts the slots per KV head of the two
  // kernels, few in the low half (at most 2 * few_target), many in the high half
  // (at most many_target, where any are split)
  Found f;
  if (!find_entry<kThreads>(A, (int)blockIdx.x, [&](const PagedSeq& q) {
        if (q.T == 0) return make_uint2(0u, 0u);
        const bool few = paged_few(A, q);
        const uint32_t n = (uint32_t)paged_chunks(q.n, few ? cut.few : cut.many), R = q.T * a.G;
        if (few) return n < 2 ? make_uint2(0u, 0u) : make_uint2(R * a.n_kv, n);
        if (cut.many == kUnsplit) return make_uint2(0u, 0u);
        return make_uint2(n < 2 ? 0u : (R + NG - 1) / NG * a.n_kv, ((R + kAttnRows - 1) / kAttnRows * n) << 16);
      }, f))
    return;
  const PagedSeq q = paged_seq(A, f.s);
  const bool few = paged_few(A, q);
  const int R = q.T * a.G, n = paged_chunks(q.n, few ? cut.few : cut.many);
  int r, g;
  int64_t slot0;     // of the row's first chunk
  int step;          // slots between chunks
  const float* part;
  int rows;
  if (few) {
    g = f.within / R;
    r = f.within - g * R;
    slot0 = (int64_t)(f.before & 0xFFFF) * a.n_kv + (int64_t)g * n;
    step = 1;
    part = A.part;
    rows = A.few_rows;
  } else {
    // split requests' items are the blocks of the tile kernel's launch, in the
    // order in which find_item numbers them
    const int per = (R + NG - 1) / NG;
    g = f.within / per;
    r = (f.within - g * per) * NG + grp;
    if (r >= R) r = R - 1;
    const int tiles = (R + kAttnRows - 1) / kAttnRows, back = tiles - 1 - r / kAttnRows;
    slot0 = (int64_t)((f.before >> 16) + back * n) * a.n_kv + g;
    step = a.n_kv;
    part = A.part_many;
    rows = kAttnRows;
  }
  const int row = few ? r : r % kAttnRows;
  const int64_t words = (int64_t)rows * (D + 2);
  const int first = few ? grp : 0, stride = few ? NG : 1;
  float m = -INFINITY, l = 0.f;
  float4 acc = make_float4(0.f, 0.f, 0.f, 0.f);
  for (int i0 = first; i0 < n; i0 += U * stride) {
    float2 x[U];
    float4 y[U];
#pragma unroll
    for (int u = 0; u < U; ++u) {
      const int i = i0 + u * stride;
      const float* p = part + (slot0 + (int64_t)(i < n ? i : first) * step) * words;
      x[u] = reinterpret_cast<const float2*>(p + rows * D)[row];
      y[u] = reinterpret_cast<const float4*>(p + row * D)[c];
      if (i >= n) x[u] = make_float2(-INFINITY, 0.f);
    }
#pragma unroll
    for (int u = 0; u < U; ++u) {
      const float m_new = fmaxf(m, x[u].x);
      const float old = part_weight(make_float2(m, l), m_new), f_new = part_weight(x[u], m_new);
      m = m_new;
      l = l * old + x[u].y * f_new;
      acc.x = acc.x * old + (f_new == 0.f ? 0.f : y[u].x * f_new);
      acc.y = acc.y * old + (f_new == 0.f ? 0.f : y[u].y * f_new);
      acc.z = acc.z * old + (f_new == 0.f ? 0.f : y[u].z * f_new);
      acc.w = acc.w * old + (f_new == 0.f ? 0.f : y[u].w * f_new);
    }
  }
  if (few) {
    acc_l[grp][c] = acc;
    if (c == 0) ml_l[grp] = make_float2(m, l);
    __syncthreads();
    if (grp > 0) return;
    for (int i = 1; i < NG; ++i) {
      const float2 x = ml_l[i];
      const float4 y = acc_l[i][c];
      const float m_new = fmaxf(m, x.x);
      const float old = part_weight(make_float2(m, l), m_new), f_new = part_weight(x, m_new);
      m = m_new;
      l = l * old + x.y * f_new;
      acc.x = acc.x * old + y.x * f_new;
      acc.y = acc.y * old + y.y * f_new;
      acc.z = acc.z * old + y.z * f_new;
      acc.w = acc.w * old + y.w * f_new;
    }
  }
  const int t = r / a.G, head = g * a.G + r - t * a.G;
  const float inv = row_scale(l);
  store4<DT>(a.out + (int64_t)(q.tok0 + t) * a.o_st + (int64_t)head * a.o_sh + 4 * c * EB, acc.x * inv,
             acc.y * inv, acc.z * inv, acc.w * inv);
  if (c == 0 && a.lse) a.lse[(int64_t)head * a.lse_sh + q.tok0 + t] = row_lse(m, l);
}

}  // namespace

hipError_t launch_paged_few(int dtype, int d, const PagedArgs& p, int grid, hipStream_t st) {
  if (grid == 0) return hipSuccess;
  const Timing none;
  if (d == 128) {
    if (dtype == CKV_BF16) return launch(paged_few_kernel<0, 128>, grid, kThreads, st, none, p);
    if (dtype == CKV_F16) return launch(paged_few_kernel<1, 128>, grid, kThreads, st, none, p);
    return launch(paged_few_kernel<2, 128>, grid, kThreads, st, none, p);
  }
  if (dtype == CKV_BF16) return launch(paged_few_kernel<0, 64>, grid, kThreads, st, none, p);
  if (dtype == CKV_F16) return launch(paged_few_kernel<1, 64>, grid, kThreads, st, none, p);
  return launch(paged_few_kernel<2, 64>, grid, kThreads, st, none, p);
}

hipError_t launch_paged_merge(int dtype, int d, const PagedArgs& p, int grid, hipStream_t st) {
  if (grid == 0) return hipSuccess;
  const Timing none;
  if (d == 128) {
    if (dtype == CKV_BF16) return launch(paged_merge_kernel<0, 128>, grid, kThreads, st, none, p);
    if (dtype == CKV_F16) return launch(paged_merge_kernel<1, 128>, grid, kThreads, st, none, p);
    return launch(paged_merge_kernel<2, 128>, grid, kThreads, st, none, p);
  }
  if (dtype == CKV_BF16) return launch(paged_merge_kernel<0, 64>, grid, kThreads, st, none, p);
  if (dtype == CKV_F16) return launch(paged_merge_kernel<1, 64>, grid, kThreads, st, none, p);
  return launch(paged_merge_kernel<2, 64>, grid, kThreads, st, none, p);
}

}  // namespace ckv
