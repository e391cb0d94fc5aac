// gfx950 (MI355X) kernels that keep a paged KV cache: block tables and slot
// maps of a step from its requests' lengths, and K/V rows into their slots.
#include "ckv_attn_device.h"

namespace ckv {
namespace {

using namespace dev;

// Pages that hold x tokens, at most `width`.
__device__ __forceinline__ int pages_of(const PageDiv& d, int size, int x, int width) {
  const int q = page_at(d, x);
  const int n = q + ((int64_t)q * size < x ? 1 : 0);
  return n < width ? n : width;
}

// A request's lengths, whatever the device arrays hold.
struct Request {
  int cached, add, have, need;  // tokens; pages that it has, and that it lacks
};
__device__ __forceinline__ Request request(const PagePlanArgs& a, int s) {
  Request r;
  const int c = to_global(a.p.cached)[s], n = to_global(a.p.add)[s];
  r.cached = c > 0 ? c : 0;
  r.add = n > 0 ? n : 0;
  const int64_t full = (int64_t)r.cached + r.add;
  r.have = pages_of(a.div, a.p.page_size, r.cached, a.p.table_width);
  r.need = pages_of(a.div, a.p.page_size, full < 0x7FFFFFFF ? (int)full : 0x7FFFFFFF, a.p.table_width) - r.have;
  return r;
}

// One launch: every workgroup scans all requests' tokens and pages for itself
// (a request is two numbers), then workgroups share out the new table entries
// and the slots. A token's page is read from the table only if it was there
// before, and taken from the free list otherwise, so that no workgroup reads
// what another one writes.
__global__ __launch_bounds__(kThreads) void page_plan_kernel(const PagePlanArgs A) {
  __shared__ int tok[CKV_MAX_PAGED_SEQS + 1];    // first row of every request
  __shared__ int taken[CKV_MAX_PAGED_SEQS + 1];  // pages taken by the requests before
  __shared__ uint32_t wsum[kWaves];
  const ckv_page_plan& p = A.p;
  const int tid = threadIdx.x, N = p.num_seqs;
  const int per = (N + kThreads - 1) / kThreads;  // consecutive requests per thread
  const int s0 = tid * per, s1 = s0 + per < N ? s0 + per : N;
  uint32_t rows = 0, pages = 0;
  for (int s = s0; s < s1; ++s) {
    const Request r = request(A, s);
    tok[s] = (int)rows;
    taken[s] = (int)pages;
    rows += (uint32_t)r.add;
    pages += (uint32_t)r.need;
  }
  uint32_t all_rows, all_pages;
  const uint32_t row0 = block_excl_scan<kThreads>(rows, wsum, all_rows);
  const uint32_t page0 = block_excl_scan<kThreads>(pages, wsum, all_pages);
  for (int s = s0; s < s1; ++s) {
    tok[s] += (int)row0;
    taken[s] += (int)page0;
  }
  if (tid == 0) {
    tok[N] = (int)all_rows;
    taken[N] = (int)all_pages;
  }
  __syncthreads();
  const int head = p.free_head ? to_global(p.free_head)[0] : 0;
  if (blockIdx.x == 0) {
    for (int s = tid; s <= N; s += kThreads) to_global(p.cu_q)[s] = tok[s];
    for (int s = tid; s < N; s += kThreads) {
      const Request r = request(A, s);
      to_global(p.kv_len)[s] = (int)((uint32_t)r.cached + (uint32_t)r.add);
    }
    if (tid == 0) to_global(p.free_head_out)[0] = (int)((uint32_t)head + all_pages);
  }
  // page k of those that the step needs, or -1 past the free list
  auto free_page = [&](int64_t k) {
    const int64_t at = (int64_t)head + k;
    return k >= 0 && at >= 0 && at < p.n_free ? to_global(p.free_pages)[at] : -1;
  };
  // the request with entry i of an array of first entries
  auto owner = [&](const int* first, int i) {
    int lo = 0, hi = N;
    while (hi - lo > 1) {
      const int mid = (lo + hi) / 2;
      if (first[mid] <= i) lo = mid; else hi = mid;
    }
    return lo;
  };
  const int at = (int)blockIdx.x * kThreads + tid, step = (int)gridDim.x * kThreads;
  for (int64_t k = at; k < (int64_t)(int)all_pages; k += step) {
    const int s = owner(taken, (int)k);
    const int e = request(A, s).have + (int)k - taken[s];
    if (e >= 0 && e < p.table_width)
      to_global(p.table)[(int64_t)s * p.table_stride + e] = free_page(k);
  }
  for (int64_t i = at; i < p.n_slots; i += step) {
    int64_t slot = -1;
    if (i < (int64_t)(int)all_rows) {
      const int s = owner(tok, (int)i);
      const Request r = request(A, s);
      const uint32_t pos = (uint32_t)r.cached + (uint32_t)((int)i - tok[s]);
      const int e = pos < 0x80000000u ? page_at(A.div, (int)pos) : p.table_width;
      if (e < p.table_width) {
        const int id = e < r.have ? to_global(p.table)[(int64_t)s * p.table_stride + e]
                                  : free_page((int64_t)taken[s] + e - r.have);
        slot = (int64_t)id * p.page_size + ((int)pos - e * p.page_size);
        if (id < 0 || slot > 0x7FFFFFFF) slot = -1;
      }
    }
    to_global(p.slots)[i] = (int)slot;
  }
}

// Rows per workgroup of one KV head: each of its 16-lane groups (8 or 32 lanes
// for other row lengths) copies kWriteRows rows' K and V, all loads issued
// before the first store.
constexpr int kWriteRows = 4;

template <int NV>
__global__ __launch_bounds__(kThreads) void page_write_kernel(const PageWriteArgs A) {
  constexpr int PER = kThreads / NV;  // rows per pass
  const int g = (int)blockIdx.x % A.n_kv;
  const int64_t r0 = (int64_t)((int)blockIdx.x / A.n_kv) * (PER * kWriteRows) + threadIdx.x / NV;
  const int c = threadIdx.x % NV;
  u32x4 kr[kWriteRows], vr[kWriteRows];
  int slot[kWriteRows];
#pragma unroll
  for (int u = 0; u < kWriteRows; ++u) {
    const int64_t r = r0 + u * PER;
    slot[u] = r < A.n ? to_global(A.slots)[r] : -1;
  }
#pragma unroll
  for (int u = 0; u < kWriteRows; ++u) {
    const int64_t r = r0 + u * PER;
    const int64_t off = (int64_t)g * A.sh + (r < A.n ? r : A.n - 1) * A.st;
    kr[u] = __builtin_nontemporal_load((const CKV_GLOBAL u32x4*)(to_global(A.k) + off) + c);
    vr[u] = __builtin_nontemporal_load((const CKV_GLOBAL u32x4*)(to_global(A.v) + off) + c);
  }
#pragma unroll
  for (int u = 0; u < kWriteRows; ++u) {
    if (slot[u] < 0) continue;
    const int id = page_at(A.div, slot[u]);
    if (id >= A.n_pages) continue;
    const int64_t off = (int64_t)id * A.sp + (int64_t)g * A.csh + (int64_t)(slot[u] - id * A.page_size) * A.cst;
    ((CKV_GLOBAL u32x4*)(to_global(A.ck) + off))[c] = kr[u];
    ((CKV_GLOBAL u32x4*)(to_global(A.cv) + off))[c] = vr[u];
  }
}

template <int NV>
hipError_t launch_write(const PageWriteArgs& w, hipStream_t st) {
  constexpr int rows = kThreads / NV * kWriteRows;
  const int64_t grid = (w.n + rows - 1) / rows * w.n_kv;
  if (grid > 0x7FFFFFFF) return hipErrorInvalidConfiguration;
  return launch(page_write_kernel<NV>, (int)grid, kThreads, st, Timing(), w);
}

}  // namespace

hipError_t launch_page_write(const PageWriteArgs& w, hipStream_t st) {
  if (w.n == 0) return hipSuccess;
  if (w.row_bytes == 128) return launch_write<8>(w, st);
  if (w.row_bytes == 256) return launch_write<16>(w, st);
  return launch_write<32>(w, st);
}

// A workgroup per 1024 slots; the new table entries are at most about as many.
hipError_t launch_page_plan(const PagePlanArgs& a, hipStream_t st) {
  const int64_t grid = ((int64_t)a.p.n_slots + 1023) / 1024;
  return launch(page_plan_kernel, (int)(grid < 1 ? 1 : grid > 1024 ? 1024 : grid), kThreads, st,
                Timing(), a);
}

}  // namespace ckv
