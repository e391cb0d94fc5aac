// gfx950 (MI355X) attention of 32 query rows per workgroup: few new tokens per
// request over a paged cache (decoding steps), and prompts too small to fill the
// chip with larger tiles; and the join of what is split along the keys.
//
// few_kernel: up to 32 query rows (of a KV head's G heads x T tokens), a
//   workgroup per (request, KV head, chunk of its keys) or per (prompt, KV head,
//   row tile). The keys go round the waves, which need no barrier between them:
//   every wave owns 32-key tiles, whose K and V go from memory straight into the
//   wave's part of LDS. The waves' results meet in LDS. Over a cache each row is
//   read once, so the bound is the stream, and a prompt's rows come from L2.
//   The next tile's K (V) is requested once this one's is in registers, and a tile starts
//   when both are there. In 16-bit types the next K does not stay open over the reads of
//   V: the compiler, which cannot tell the parts of LDS apart, waits for it there, as it
//   waits for the page numbers read ahead over a cache. Counted waits, which let a tile
//   start on K while V is on the way, took the same time: what keeps the stream up are
//   the CU's other waves.
// paged_merge_kernel: the chunks' partial results (of this kernel and of the tile
//   kernel) rescaled to the common maximum and added in order.
#include <math.h>

#include "ckv_attn_device.h"

namespace ckv {
namespace {

using namespace dev;

// A workgroup's part: rows row0 .. of the T * G of a request whose last T of n keys
// are its query tokens from row tok0 on; keys j0 .. j1.
struct FewItem {
  int tok0, T, n, g, row0, j0, j1;
  int64_t slot;           // where its partial result goes, -1 where the keys are not split
  int n_chunks;
  const int32_t* table;   // paged: the request's block table
};

__device__ __forceinline__ bool find_few(const PagedArgs& A, FewItem& it) {
  const int b = (int)blockIdx.x / A.a.n_kv;
  it.g = (int)blockIdx.x - b * A.a.n_kv;
  const PagedSeq first = lane_seq(A, threadIdx.x & 63);
  const int chunk = few_share(A, first);
  Found f;
  if (!find_entry(A, first, b, [&](const PagedSeq& q) {
        const uint32_t n = paged_few(A, q) ? paged_chunks(q.n, chunk) : 0;
        return make_uint2(n, n > 1 ? n : 0);
      }, f))
    return false;
  const PagedSeq q = f.q;
  const int n_chunks = paged_chunks(q.n, chunk);
  it.tok0 = q.tok0;
  it.T = q.T;
  it.n = q.n;
  it.row0 = 0;
  it.j0 = f.within * chunk;
  it.j1 = paged_chunk_end(q.n, chunk, f.within);
  it.slot = n_chunks > 1 ? (int64_t)f.before * A.a.n_kv + (int64_t)it.g * n_chunks + f.within : -1;
  it.n_chunks = n_chunks;
  it.table = A.table + (int64_t)f.s * A.table_stride;
  return true;
}

__device__ __forceinline__ bool find_few(const PrefillArgs& A, FewItem& it) {
  const PromptTile p = prompt_tile(A);
  it.tok0 = p.tok0;
  it.T = it.n = p.T;
  it.g = p.g;
  it.row0 = p.rt * kFewRows;
  const int last = it.row0 + kFewRows < p.T * A.a.G ? it.row0 + kFewRows - 1 : p.T * A.a.G - 1;
  it.j0 = 0;
  it.j1 = last / A.a.G + 1;
  it.slot = -1;
  it.n_chunks = 1;
  it.table = nullptr;
  return true;
}

template <int DT, int D, bool PAGED, class Args>
__global__ __launch_bounds__(kThreads) __attribute__((amdgpu_waves_per_eu(DT == 2 ? 1 : 2)))
void few_kernel(const Args A) {
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
  const AttnArgs& a = A.a;
  const int tid = threadIdx.x, lane = tid & 63, h = lane >> 5, l32 = lane & 31;
  const int wave = __builtin_amdgcn_readfirstlane(tid >> 6);
  FewItem it;
  if (!find_few(A, it)) return;
  const int G = a.G, g = it.g, j0 = it.j0, j1 = it.j1;
  const int R = it.T * G - it.row0 < kFewRows ? it.T * G - it.row0 : kFewRows;  // rows of this workgroup
  const int nt = (j1 - j0 + KT - 1) / KT;
  const char* kbase = a.k + (int64_t)g * a.kv_sh;
  const char* vbase = a.v + (int64_t)g * a.kv_sh;
  if constexpr (!PAGED) {
    kbase += (int64_t)it.tok0 * a.kv_st;
    vbase += (int64_t)it.tok0 * a.kv_st;
  }
  const float alpha = a.alpha;

  auto swz = [](int t) { return ROWB >= 256 ? (t & 15) : ((t >> 1) & 7); };
  // V of 16-bit types is read 4 keys of 64 bytes at a time, which meet every bank once if
  // they lie in different quarters of the 256 bytes; rows of fp32 are read along
  // their columns, which does as it is
  auto vswz = [&](int t) { return DT == 2 ? 0 : ROWB >= 256 ? (t & 3) * 4 : (t & 2) * 2; };
  const int lrow = lane / NV, lpos = lane % NV;
  // the page of key l32 of tile tl (0 where there are no pages), -1 for keys that are not there
  auto page_of = [&](int tl) {
    const int key = j0 + tl * KT + l32;
    int id = -1;
    if (key < j1) {
      if constexpr (PAGED) {
        const int p = page_at(A.div, key);
        if ((uint32_t)p < (uint32_t)A.table_width) id = to_global(it.table)[p];
        if ((uint32_t)id >= (uint32_t)A.n_pages) id = -1;
      } else {
        id = 0;
      }
    }
    return id;
  };
  // tile tl of base; a cache's rows, read once, are non-temporal. Keys that are not
  // there read some valid row.
  auto fetch = [&](const char* base, int tl, int page, uint4* slot, auto swizzle) {
#pragma unroll
    for (int i = 0; i < PT; ++i) {
      const int t = i * RPL + lrow, key = j0 + tl * KT + t;
      int64_t off;
      if constexpr (PAGED) {
        const int id = __shfl(page, t);
        off = (int64_t)(id < 0 ? 0 : id) * A.kv_sp + (int64_t)(key - page_at(A.div, key) * A.page_size) * a.kv_st;
      } else {
        off = (int64_t)(key < j1 ? key : j1 - 1) * a.kv_st;
      }
      __builtin_amdgcn_global_load_lds(reinterpret_cast<const uint4*>(base + off + (lpos ^ swizzle(t)) * 16),
                                       slot + i * 64, 16, 0, PAGED ? 2 : 0);
    }
  };
  // query row r = token * G + head; lane half h holds chunks 2c + h of it
  const int r = it.row0 + (l32 < R ? l32 : R - 1);
  const int t = r / G, limit = it.n - it.T + t;
  uint4 q[NC];
  {
    const CKV_GLOBAL u32x4* src =
        (const CKV_GLOBAL u32x4*)(to_global(a.q) + (int64_t)(it.tok0 + t) * a.q_st +
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
    wait_vm<0>();  // this tile's K and V
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
    if (vis != ~0u) {  // keys that are not there count as zeros
#pragma unroll
      for (int i = 0; i < PT; ++i)
        if (!((vis >> (i * RPL + lrow)) & 1)) vl[wave][i * 64 + lane] = make_uint4(0u, 0u, 0u, 0u);
      wait_vm<63>();
    }
    const char* vt = reinterpret_cast<const char*>(vl[wave]);
    // A hidden key's weight is 0, but 0 times a value that is not finite is not:
    // where keys are hidden such values are left out of the product, and what a
    // row sees of them is added; likewise where a weight's low part, of either sign
    // or 0, would make a NaN of an infinity.
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
      // A cache's weights keep a high and a low part, as ckv_decode_attention's do: its rows
      // are few and the stream bounds it (64 single tokens 82.9 us with both, 81.9 rounded
      // once), and the outputs are as exact as their type (rounded once they were 1.3 to 1.4
      // times as far off). A prompt's are rounded once, in either kernel: both parts took
      // 5% longer here and 35% in the large tiles.
      uint4 ph[2], pl[2];
#pragma unroll
      for (int m = 0; m < 2; ++m) {
        float p[8];
#pragma unroll
        for (int i = 0; i < 8; ++i) p[i] = s[8 * m + i];
        if constexpr (PAGED) split_chunk<DT>(p, ph[m], pl[m]);
        else ph[m] = round_chunk<DT>(p);
      }
      bool strip = hides;
      if constexpr (PAGED) {
        float zero = 0.f;
#pragma unroll
        for (int m = 0; m < 2; ++m)
#pragma unroll
          for (int nb = 0; nb < NB; ++nb) zero = zero_times<DT>(vr[m][nb], zero);
        strip = strip || __any(zero != 0.f);
      }
      if (strip) {
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
        for (int nb = 0; nb < NB; ++nb) {
          o[nb] = mfma_chunk<DT>(vr[m][nb], ph[m], o[nb]);
          if constexpr (PAGED) o[nb] = mfma_chunk<DT>(vr[m][nb], pl[m], o[nb]);
        }
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
    const int tt = (it.row0 + rr) / G, head = g * G + it.row0 + rr - tt * G;
    if constexpr (PAGED) {
      if (A.notes && c == 0 && j0 == 0)
        A.notes[(int64_t)(it.tok0 + tt) * a.H + head] = row_note(it.slot, it.n_chunks, rr, false);
      if (it.slot >= 0) {
        *reinterpret_cast<float4*>(partial_o(A.part, it.slot, A.few_rows, D) + rr * D + 4 * c) = acc;
        if (c == 0) partial_ml(A.part, it.slot, A.few_rows, D)[rr] = make_float2(m - kBias, ls);
        continue;
      }
    }
    const float inv = row_scale(ls);
    store4<DT>(a.out + (int64_t)(it.tok0 + tt) * a.o_st + (int64_t)head * a.o_sh + 4 * c * EB,
               acc.x * inv, acc.y * inv, acc.z * inv, acc.w * inv);
    if (c == 0 && a.lse) a.lse[(int64_t)head * a.lse_sh + it.tok0 + tt] = row_lse(m - kBias, ls);
  }
}

// Joins the partial results of the rows whose keys were split, which the two kernels
// noted per row. A workgroup takes a row with all its thread groups of D / 4 lanes,
// or, where there are many rows, a row per thread group unless they have many chunks.
// Bound by the latency of its three dependent reads: 5.5 us for the 32 rows of one long
// request, 8 us for 2048 rows of 64; with every workgroup working the cuts out again in
// place of reading the notes it took 8 and 12 us.
__host__ __device__ inline int merge_rows_per(const PagedArgs& A, int groups) {
  return (int64_t)A.total_q * A.a.H <= 16 * kCUs ? 1 : groups;
}
template <int DT, int D>
__global__ __launch_bounds__(kThreads) void paged_merge_kernel(const PagedArgs A) {
  constexpr int C4 = D / 4, NG = kThreads / C4, U = 8;
  constexpr int EB = Elt<DT>::bytes;
  __shared__ float4 acc_l[NG][C4];
  __shared__ float2 ml_l[NG];
  const AttnArgs& a = A.a;
  const int grp = threadIdx.x / C4, c = threadIdx.x % C4;
  const int rows_per = merge_rows_per(A, NG);
  const int64_t lo = (int64_t)clamp_int(to_global(A.cu_q)[0], 0, A.total_q) * a.H;
  const int64_t hi = (int64_t)clamp_int(to_global(A.cu_q)[A.num_seqs], 0, A.total_q) * a.H;
  // Row's note, one without chunks where it has none. The notes of rows that no
  // request covers may hold anything: what they name stays inside the workspace.
  auto note_of = [&](int64_t row) {
    RowNote x = {};
    if (row >= lo && row < hi) x = A.notes[row];
    const int cap = x.many() ? A.many_slots : A.few_slots, step = x.many() ? a.n_kv : 1;
    const bool ok = x.n() >= 2 && (int64_t)x.slot() + (int64_t)(x.n() - 1) * step < cap &&
                    x.row() < (x.many() ? kAttnRows : A.few_rows);
    return ok ? x : RowNote{};
  };
  // chunks first, first + stride, .. of a row. One of factor 0 is multiplied all the same:
  // what it holds that is not finite reaches the row.
  auto gather = [&](const RowNote x, int first, int stride, float& m, float& l, float4& acc) {
    const int rows = x.many() ? kAttnRows : A.few_rows, step = x.many() ? a.n_kv : 1, n = x.n(), row = x.row();
    const int64_t words = partial_words(rows, D);
    const float* part = (x.many() ? A.part_many : A.part) + x.slot() * words;
    m = -INFINITY;
    l = 0.f;
    acc = make_float4(0.f, 0.f, 0.f, 0.f);
    for (int i0 = first; i0 < n; i0 += U * stride) {
      float2 x[U];
      float4 y[U];
#pragma unroll
      for (int u = 0; u < U; ++u) {
        const int i = i0 + u * stride;
        const float* p = part + (int64_t)(i < n ? i : first) * step * words;
        x[u] = reinterpret_cast<const float2*>(p + rows * D)[row];
        y[u] = reinterpret_cast<const float4*>(p + row * D)[c];
      }
#pragma unroll
      for (int u = 0; u < U; ++u) {
        if (i0 + u * stride >= n) break;  // what was read past the last one does not count
        const float m_new = fmaxf(m, x[u].x);
        const float old = part_weight(make_float2(m, l), m_new), f_new = part_weight(x[u], m_new);
        m = m_new;
        l = l * old + x[u].y * f_new;
        acc.x = acc.x * old + y[u].x * f_new;
        acc.y = acc.y * old + y[u].y * f_new;
        acc.z = acc.z * old + y[u].z * f_new;
        acc.w = acc.w * old + y[u].w * f_new;
      }
    }
  };
  auto put = [&](int64_t row, float m, float l, float4 acc) {
    const int tok = (int)(row / a.H), head = (int)(row - (int64_t)tok * a.H);
    const float inv = row_scale(l);
    store4<DT>(a.out + (int64_t)tok * a.o_st + (int64_t)head * a.o_sh + 4 * c * EB, acc.x * inv, acc.y * inv,
               acc.z * inv, acc.w * inv);
    if (c == 0 && a.lse) a.lse[(int64_t)head * a.lse_sh + tok] = row_lse(m, l);
  };
  auto together = [&](int64_t row, const RowNote x) {  // for the whole workgroup
    if (x.n() < 2) return;
    float m, l;
    float4 acc;
    gather(x, grp, NG, m, l, acc);
    acc_l[grp][c] = acc;
    if (c == 0) ml_l[grp] = make_float2(m, l);
    __syncthreads();
    if (grp == 0) {
      for (int i = 1; i < NG; ++i) {
        const float2 z = ml_l[i];
        const float4 y = acc_l[i][c];
        const float m_new = fmaxf(m, z.x);
        const float old = part_weight(make_float2(m, l), m_new), f_new = part_weight(z, m_new);
        m = m_new;
        l = l * old + z.y * f_new;
        acc.x = acc.x * old + y.x * f_new;
        acc.y = acc.y * old + y.y * f_new;
        acc.z = acc.z * old + y.z * f_new;
        acc.w = acc.w * old + y.w * f_new;
      }
      put(row, m, l, acc);
    }
    __syncthreads();
  };
  for (int64_t row0 = (int64_t)blockIdx.x * rows_per; row0 < hi; row0 += (int64_t)gridDim.x * rows_per) {
    if (rows_per == 1) {
      together(row0, note_of(row0));
      continue;
    }
    const RowNote mine = note_of(row0 + grp);
    if (__syncthreads_or(mine.n() > 8 * U)) {
      for (int i = 0; i < NG; ++i) together(row0 + i, note_of(row0 + i));
    } else if (mine.n() >= 2) {
      float m, l;
      float4 acc;
      gather(mine, 0, 1, m, l, acc);
      put(row0 + grp, m, l, acc);
    }
  }
}

template <int D>
hipError_t launch_merge(int dtype, const PagedArgs& p, hipStream_t st) {
  constexpr int NG = kThreads / (D / 4);
  const int64_t rows = (int64_t)p.total_q * p.a.H, per = merge_rows_per(p, NG), most = 64 * kCUs;
  const int grid = (int)((rows + per - 1) / per < most ? (rows + per - 1) / per : most);
  auto kernel = dtype == CKV_BF16 ? paged_merge_kernel<0, D> : dtype == CKV_F16 ? paged_merge_kernel<1, D> : paged_merge_kernel<2, D>;
  return launch(kernel, grid, kThreads, st, Timing(), p);
}

template <bool PAGED, class Args>
hipError_t launch_few(int dtype, int d, const Args& p, int grid, hipStream_t st) {
  if (grid == 0) return hipSuccess;
  const Timing none;
  if (d == 128) {
    if (dtype == CKV_BF16) return launch(few_kernel<0, 128, PAGED, Args>, grid, kThreads, st, none, p);
    if (dtype == CKV_F16) return launch(few_kernel<1, 128, PAGED, Args>, grid, kThreads, st, none, p);
    return launch(few_kernel<2, 128, PAGED, Args>, grid, kThreads, st, none, p);
  }
  if (dtype == CKV_BF16) return launch(few_kernel<0, 64, PAGED, Args>, grid, kThreads, st, none, p);
  if (dtype == CKV_F16) return launch(few_kernel<1, 64, PAGED, Args>, grid, kThreads, st, none, p);
  return launch(few_kernel<2, 64, PAGED, Args>, grid, kThreads, st, none, p);
}

}  // namespace

hipError_t launch_paged_few(int dtype, int d, const PagedArgs& p, int grid, hipStream_t st) {
  return launch_few<true>(dtype, d, p, grid, st);
}
hipError_t launch_prefill_few(int dtype, int d, const PrefillArgs& p, int grid, hipStream_t st) {
  return launch_few<false>(dtype, d, p, grid, st);
}

hipError_t launch_paged_merge(int dtype, int d, const PagedArgs& p, hipStream_t st) {
  return d == 128 ? launch_merge<128>(dtype, p, st) : launch_merge<64>(dtype, p, st);
}

}  // namespace ckv
