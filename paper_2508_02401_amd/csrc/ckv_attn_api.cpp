// C ABI of prompt attention and of the paged cache: argument validation and
// launches. Declarations and the contract of every entry point are in
// include/ckv.h.
#include "ckv.h"

#include <hip/hip_runtime.h>
#include <math.h>
#include <string.h>

#include <algorithm>

#include "ckv_internal.h"
#include "ckv_plan.h"

namespace {

int elt_bytes(int dtype) { return dtype == CKV_F32 ? 4 : 2; }
bool aligned(const void* p, uintptr_t n) { return ((uintptr_t)p & (n - 1)) == 0; }
int64_t ceil_div(int64_t a, int64_t b) { return (a + b - 1) / b; }

int status(hipError_t e) { return e == hipSuccess ? CKV_OK : ckv::record_hip_error((int)e); }

int check_desc(const ckv_attn_desc* d) {
  if (!d || d->num_q_heads < 1 || d->num_kv_heads < 1 || d->num_q_heads % d->num_kv_heads)
    return CKV_ERR_INVALID_ARG;
  if (d->num_q_heads > CKV_MAX_Q_HEADS || d->num_kv_heads > CKV_MAX_KV_HEADS) return CKV_ERR_UNSUPPORTED;
  if (d->head_dim != 64 && d->head_dim != 128) return CKV_ERR_UNSUPPORTED;
  if (d->dtype != CKV_BF16 && d->dtype != CKV_F16 && d->dtype != CKV_F32) return CKV_ERR_UNSUPPORTED;
  if (!(d->scale > 0.f) && !(d->scale <= 0.f)) return CKV_ERR_INVALID_ARG;  // NaN
  if (isinf(d->scale)) return CKV_ERR_INVALID_ARG;
  return CKV_OK;
}

// A stride in elements: not negative, a multiple of 16 bytes and, where there is
// a second index along it, at least `least`.
bool stride_ok(int64_t s, int64_t eb, int64_t least, bool used) {
  return s >= 0 && (s * eb) % 16 == 0 && (!used || s >= least);
}

// Queries, outputs and log-sum-exp of `rows` rows.
int check_rows(const ckv_attn_desc* d, const ckv_packed_attn* a, int64_t rows) {
  const int64_t eb = elt_bytes(d->dtype), dim = d->head_dim;
  if (!a->q || !a->out || !aligned(a->q, 16) || !aligned(a->out, 16)) return CKV_ERR_INVALID_ARG;
  const bool heads = d->num_q_heads > 1;
  if (!stride_ok(a->q_stride_tok, eb, dim, rows > 1) || !stride_ok(a->q_stride_head, eb, dim, heads) ||
      !stride_ok(a->out_stride_tok, eb, dim, rows > 1) || !stride_ok(a->out_stride_head, eb, dim, heads))
    return CKV_ERR_INVALID_ARG;
  if (a->lse && (!aligned(a->lse, 4) || a->lse_stride_head < 0 || (heads && a->lse_stride_head < rows)))
    return CKV_ERR_INVALID_ARG;
  return CKV_OK;
}

void fill(const ckv_attn_desc* d, const ckv_packed_attn* a, ckv::AttnArgs& r) {
  const int64_t eb = elt_bytes(d->dtype);
  memset(&r, 0, sizeof(r));
  r.q = static_cast<const char*>(a->q);
  r.out = static_cast<char*>(a->out);
  r.lse = a->lse;
  r.q_st = a->q_stride_tok * eb;
  r.q_sh = a->q_stride_head * eb;
  r.o_st = a->out_stride_tok * eb;
  r.o_sh = a->out_stride_head * eb;
  r.lse_sh = a->lse_stride_head;
  r.H = d->num_q_heads;
  r.n_kv = d->num_kv_heads;
  r.G = d->num_q_heads / d->num_kv_heads;
  const float scale = d->scale > 0.f ? d->scale : 1.0f / sqrtf((float)d->head_dim);
  r.alpha = (float)((double)scale * 1.4426950408889634);  // log2(e)
}

int check_cache(const ckv_attn_desc* d, const ckv_paged_cache* c) {
  const int64_t eb = elt_bytes(d->dtype), dim = d->head_dim;
  if (!c || !c->k || !c->v || !aligned(c->k, 16) || !aligned(c->v, 16)) return CKV_ERR_INVALID_ARG;
  if (c->n_pages < 1 || c->page_size < 1 || (int64_t)c->n_pages * c->page_size >= ((int64_t)1 << 31))
    return CKV_ERR_INVALID_ARG;
  if (!stride_ok(c->stride_page, eb, dim, c->n_pages > 1) ||
      !stride_ok(c->stride_head, eb, dim, d->num_kv_heads > 1) ||
      !stride_ok(c->stride_tok, eb, dim, c->page_size > 1))
    return CKV_ERR_INVALID_ARG;
  return CKV_OK;
}

int check_batch(const ckv_attn_desc* d, const ckv_paged_batch* b) {
  if (!b || b->num_seqs < 1 || b->total_q < 0 || b->max_q < 0 || b->max_kv < 0) return CKV_ERR_INVALID_ARG;
  if (b->num_seqs > CKV_MAX_PAGED_SEQS) return CKV_ERR_UNSUPPORTED;
  // positions of the tiles that are requested ahead, in 32 bits
  if (b->max_kv > CKV_MAX_PAGED_KV) return CKV_ERR_UNSUPPORTED;
  // rows of a KV head, counted in 32 bits
  if ((int64_t)b->total_q * (d->num_q_heads / d->num_kv_heads) >= ((int64_t)1 << 30)) return CKV_ERR_UNSUPPORTED;
  return CKV_OK;
}

// Workgroups of one round of the kernel for few rows: two on a CU, one in fp32.
int32_t few_target(const ckv_attn_desc* d) {
  return ckv::kCUs * ckv::decode_wgs_per_cu(d->dtype == CKV_F32, d->head_dim, ckv::kFewRows);
}
constexpr int32_t kManyTarget = ckv::kCUs;  // and of the tile kernel

// What a batch of these bounds needs of the workspace: partial results of requests
// of few rows (slots for twice kFewRounds rounds, as a split request has two chunks
// at least) and of the tile kernel (one round), and a note per row.
struct PagedSpace {
  int32_t few_slots;
  size_t few, many, notes;  // bytes
};
PagedSpace paged_space(const ckv_attn_desc* d, const ckv_paged_batch* b) {
  const int64_t rows = (int64_t)b->max_q * (d->num_q_heads / d->num_kv_heads);
  auto slot = [&](int64_t n) { return (size_t)ckv::partial_words((int32_t)n, d->head_dim) * sizeof(float); };
  PagedSpace s = {};
  if (b->max_kv > ckv::kFewLeast) {
    s.few_slots = 2 * ckv::kFewRounds * few_target(d);
    s.few = s.few_slots * slot(std::min<int64_t>(rows, ckv::kFewRows));
    s.notes = (size_t)b->total_q * d->num_q_heads * sizeof(ckv::RowNote);
  }
  if (rows > ckv::kFewRows && b->max_kv > ckv::kManyLeast) s.many = (size_t)kManyTarget * slot(ckv::kAttnRows);
  return s;
}

// Whether [a, a + n) and [b, b + m) (numbers of int32) share an element.
bool overlap(const int32_t* a, int64_t n, const int32_t* b, int64_t m) {
  return a && b && (uintptr_t)a < (uintptr_t)(b + m) && (uintptr_t)b < (uintptr_t)(a + n);
}

}  // namespace

extern "C" {

int ckv_prefill_attention(const ckv_attn_desc* desc, const ckv_packed_attn* a,
                          const int32_t* cu_seqlens, int32_t num_seqs, void* stream) {
  int rc = check_desc(desc);
  if (rc != CKV_OK) return rc;
  if (!a || !cu_seqlens || num_seqs < 1 || cu_seqlens[0] < 0) return CKV_ERR_INVALID_ARG;
  for (int32_t i = 0; i < num_seqs; ++i)
    if (cu_seqlens[i + 1] < cu_seqlens[i]) return CKV_ERR_INVALID_ARG;
  const int64_t rows = cu_seqlens[num_seqs], eb = elt_bytes(desc->dtype);
  if (rows == cu_seqlens[0]) return CKV_OK;  // no token
  const int64_t G = desc->num_q_heads / desc->num_kv_heads;
  if (rows * G >= ((int64_t)1 << 30)) return CKV_ERR_UNSUPPORTED;  // rows of a KV head, counted in 32 bits
  if ((rc = check_rows(desc, a, rows)) != CKV_OK) return rc;
  if (!a->k || !a->v || !aligned(a->k, 16) || !aligned(a->v, 16) ||
      !stride_ok(a->kv_stride_tok, eb, desc->head_dim, rows > 1) ||
      !stride_ok(a->kv_stride_head, eb, desc->head_dim, desc->num_kv_heads > 1))
    return CKV_ERR_INVALID_ARG;
  ckv::PrefillArgs p;
  fill(desc, a, p.a);
  p.a.k = static_cast<const char*>(a->k);
  p.a.v = static_cast<const char*>(a->v);
  p.a.kv_st = a->kv_stride_tok * eb;
  p.a.kv_sh = a->kv_stride_head * eb;
  for (int32_t i0 = 0; i0 < num_seqs; i0 += ckv::kPrefillSeqs) {
    p.n = num_seqs - i0 < ckv::kPrefillSeqs ? num_seqs - i0 : ckv::kPrefillSeqs;
    const int32_t* cu = cu_seqlens + i0;
    const int32_t n = p.n;
    auto len = [&](int32_t i) { return cu[i + 1] - cu[i]; };
    int32_t longest = 0;
    for (int32_t i = 0; i < n; ++i) longest = std::max(longest, len(i));
    const bool few = ckv::prefill_small_tiles(desc->dtype == CKV_F32, desc->head_dim, ckv::kCUs, ckv::kFewRows, G,
                                              desc->num_kv_heads, cu, n);
    const int64_t rows_per = few ? ckv::kFewRows : ckv::kAttnRows;
    // A tile's work is its last row's position. Tiles run from long to short, in
    // bands of position over all prompts, so that no long one starts when the others
    // end: seven prompts of 1 to 4013 tokens
    // took 192 us one after the other and take 189 so.
    const int32_t bands = n == 1 ? 1 : std::min(ckv::kPrefillSeqs / n, 16);
    p.n = 0;
    p.tile[0] = 0;
    for (int32_t b = bands - 1; b >= 0; --b) {
      auto below = [&](int32_t i, int32_t band) {  // prompt i's tiles in the bands under this one
        const int64_t rows = std::min((int64_t)longest * band / bands, (int64_t)len(i)) * G;
        return (int32_t)(rows == len(i) * G ? ceil_div(rows, rows_per) : rows / rows_per);
      };
      for (int32_t i = 0; i < n; ++i) {
        const int32_t lo = below(i, b), hi = below(i, b + 1);
        if (hi == lo) continue;
        p.tok[p.n] = cu[i];
        p.len[p.n] = len(i);
        p.top[p.n] = hi - 1;
        p.tile[p.n + 1] = p.tile[p.n] + hi - lo;
        ++p.n;
      }
    }
    if (p.n == 0) continue;  // no token
    const int grid = p.tile[p.n] * desc->num_kv_heads;
    const hipError_t e = few ? ckv::launch_prefill_few(desc->dtype, desc->head_dim, p, grid, (hipStream_t)stream)
                             : ckv::launch_prefill(desc->dtype, desc->head_dim, p, grid, (hipStream_t)stream);
    if (e != hipSuccess) return status(e);
  }
  return CKV_OK;
}

int ckv_paged_plan(const ckv_page_plan* p, void* stream) {
  if (!p || p->num_seqs < 1 || p->page_size < 1 || p->table_width < 1 || p->n_free < 0 || p->n_slots < 0)
    return CKV_ERR_INVALID_ARG;
  if (p->num_seqs > CKV_MAX_PAGED_SEQS) return CKV_ERR_UNSUPPORTED;
  if (!p->cached || !p->add || !p->table || (!p->free_pages && p->n_free > 0) || !p->cu_q || !p->kv_len ||
      (!p->slots && p->n_slots > 0) || !p->free_head_out)
    return CKV_ERR_INVALID_ARG;
  if (p->num_seqs > 1 && p->table_stride < p->table_width) return CKV_ERR_INVALID_ARG;
  struct Range {
    const int32_t* at;
    int64_t n;
  };
  const int64_t N = p->num_seqs;
  const int64_t table_n = (N > 1 ? (N - 1) * p->table_stride : 0) + p->table_width;
  const Range in[] = {{p->cached, N}, {p->add, N}, {p->free_pages, p->n_free}, {p->free_head, 1}};
  const Range out[] = {{p->table, table_n}, {p->cu_q, N + 1}, {p->kv_len, N}, {p->slots, p->n_slots}, {p->free_head_out, 1}};
  for (const Range& r : in)
    if (!aligned(r.at, 4)) return CKV_ERR_INVALID_ARG;
  for (const Range& o : out) {
    if (!aligned(o.at, 4)) return CKV_ERR_INVALID_ARG;
    for (const Range& r : in)
      if (overlap(o.at, o.n, r.at, r.n)) return CKV_ERR_INVALID_ARG;
    for (const Range& r : out)
      if (&r != &o && overlap(o.at, o.n, r.at, r.n)) return CKV_ERR_INVALID_ARG;
  }
  ckv::PagePlanArgs a;
  a.p = *p;
  a.div = ckv::page_div(p->page_size);
  return status(ckv::launch_page_plan(a, (hipStream_t)stream));
}

int ckv_paged_write(const ckv_attn_desc* desc, const ckv_paged_cache* cache, const void* k,
                    const void* v, int64_t stride_tok, int64_t stride_head, const int32_t* slots,
                    int64_t n, void* stream) {
  int rc = check_desc(desc);
  if (rc != CKV_OK) return rc;
  if ((rc = check_cache(desc, cache)) != CKV_OK) return rc;
  const int64_t eb = elt_bytes(desc->dtype);
  if (n < 0 || n >= ((int64_t)1 << 31)) return CKV_ERR_INVALID_ARG;
  if (n == 0) return CKV_OK;
  if (!k || !v || !slots || !aligned(k, 16) || !aligned(v, 16) || !aligned(slots, 4)) return CKV_ERR_INVALID_ARG;
  if (!stride_ok(stride_tok, eb, desc->head_dim, n > 1) ||
      !stride_ok(stride_head, eb, desc->head_dim, desc->num_kv_heads > 1))
    return CKV_ERR_INVALID_ARG;
  ckv::PageWriteArgs w;
  w.k = static_cast<const char*>(k);
  w.v = static_cast<const char*>(v);
  w.st = stride_tok * eb;
  w.sh = stride_head * eb;
  w.ck = static_cast<char*>(cache->k);
  w.cv = static_cast<char*>(cache->v);
  w.sp = cache->stride_page * eb;
  w.csh = cache->stride_head * eb;
  w.cst = cache->stride_tok * eb;
  w.slots = slots;
  w.n = n;
  w.n_kv = desc->num_kv_heads;
  w.row_bytes = (int32_t)(desc->head_dim * eb);
  w.n_pages = cache->n_pages;
  w.page_size = cache->page_size;
  w.div = ckv::page_div(cache->page_size);
  return status(ckv::launch_page_write(w, (hipStream_t)stream));
}

size_t ckv_paged_workspace_bytes(const ckv_attn_desc* desc, const ckv_paged_batch* batch) {
  if (check_desc(desc) != CKV_OK || check_batch(desc, batch) != CKV_OK) return 0;
  const PagedSpace s = paged_space(desc, batch);
  return s.few + s.many + s.notes + 256;
}

int ckv_paged_attention(const ckv_attn_desc* desc, const ckv_paged_cache* cache,
                        const ckv_paged_batch* batch, const ckv_packed_attn* a, void* workspace,
                        size_t workspace_bytes, void* stream) {
  int rc = check_desc(desc);
  if (rc != CKV_OK) return rc;
  if ((rc = check_cache(desc, cache)) != CKV_OK) return rc;
  if ((rc = check_batch(desc, batch)) != CKV_OK) return rc;
  if (!a || !batch->cu_q || !batch->kv_len || !batch->table || !aligned(batch->cu_q, 4) ||
      !aligned(batch->kv_len, 4) || !aligned(batch->table, 4) || batch->table_width < 1 ||
      (batch->num_seqs > 1 && batch->table_stride < batch->table_width))
    return CKV_ERR_INVALID_ARG;
  if (batch->total_q == 0 || batch->max_q == 0) return CKV_OK;  // no row
  if ((rc = check_rows(desc, a, batch->total_q)) != CKV_OK) return rc;
  if (!workspace || !aligned(workspace, 16) ||
      workspace_bytes < ckv_paged_workspace_bytes(desc, batch))
    return CKV_ERR_WORKSPACE;
  const int64_t eb = elt_bytes(desc->dtype);
  ckv::PagedArgs p;
  fill(desc, a, p.a);
  p.a.k = static_cast<const char*>(cache->k);
  p.a.v = static_cast<const char*>(cache->v);
  p.a.kv_st = cache->stride_tok * eb;
  p.a.kv_sh = cache->stride_head * eb;
  p.kv_sp = cache->stride_page * eb;
  p.cu_q = batch->cu_q;
  p.kv_len = batch->kv_len;
  p.table = batch->table;
  p.table_stride = batch->table_stride;
  p.table_width = batch->table_width;
  p.num_seqs = batch->num_seqs;
  p.total_q = batch->total_q;
  p.max_kv = batch->max_kv;
  p.n_pages = cache->n_pages;
  p.page_size = cache->page_size;
  p.div = ckv::page_div(cache->page_size);
  p.part = static_cast<float*>(workspace);
  const PagedSpace space = paged_space(desc, batch);
  p.part_many = reinterpret_cast<float*>(static_cast<char*>(workspace) + space.few);
  p.notes = space.notes ? reinterpret_cast<ckv::RowNote*>(static_cast<char*>(workspace) + space.few + space.many) : nullptr;
  p.few_slots = space.few_slots;
  p.many_slots = space.many ? kManyTarget : 0;
  // Requests of few and of many rows have a kernel each; one request with many
  // takes the latter whatever its rows turn out to be
  const int64_t N = batch->num_seqs, n_kv = desc->num_kv_heads, G = desc->num_q_heads / n_kv;
  const int64_t most = batch->max_q * G;  // rows of a request and KV head
  p.has_many = most > ckv::kFewRows;
  p.few_rows = !p.has_many ? (int32_t)most : N > 1 ? ckv::kFewRows : 0;
  p.few_target = few_target(desc);
  p.many_target = kManyTarget;
  const hipStream_t st = (hipStream_t)stream;
  hipError_t e = hipSuccess;
  if (p.has_many) {
    // row tiles: whole ones of all rows, and one more each for what is left
    int64_t tiles = batch->total_q * G / ckv::kAttnRows + N;
    if (N * ceil_div(most, ckv::kAttnRows) < tiles) tiles = N * ceil_div(most, ckv::kAttnRows);
    int64_t split = tiles * n_kv * ceil_div(batch->max_kv, ckv::kManyLeast);
    if (split > p.many_target) split = p.many_target;
    const int64_t grid = split > tiles * n_kv ? split : tiles * n_kv;
    if ((e = ckv::launch_paged_many(desc->dtype, desc->head_dim, p, (int)grid, st)) != hipSuccess) return status(e);
  }
  if (p.few_rows > 0) {
    int64_t grid = N * n_kv + ckv::kFewRounds * p.few_target;
    if (N * n_kv * ceil_div(batch->max_kv, ckv::kFewLeast) < grid)
      grid = N * n_kv * ceil_div(batch->max_kv, ckv::kFewLeast);
    if (grid < N * n_kv) grid = N * n_kv;
    if ((e = ckv::launch_paged_few(desc->dtype, desc->head_dim, p, (int)grid, st)) != hipSuccess) return status(e);
  }
  return p.notes ? status(ckv::launch_paged_merge(desc->dtype, desc->head_dim, p, st)) : CKV_OK;
}

}  // extern "C"
