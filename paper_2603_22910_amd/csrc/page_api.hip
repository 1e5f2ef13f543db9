// libechokv: C-ABI entry points of the paged 8-bit cache.  Host side only validates and launches; lengths, tables and the sharing out
// of work live on the device (page_kernels.h), so that a captured step follows its sequences as they grow.
#include "../../include/echokv.h"

#include <hip/hip_runtime.h>

#include <algorithm>
#include <cmath>
#include <initializer_list>
#include <type_traits>

#include "page_attn.h"

using namespace echokv;

namespace {

#define LAUNCH_CHECK() do { if (hipGetLastError() != hipSuccess) return ECHOKV_ERR_HIP; } while (0)

struct Sizes { int H_q, H_kv, G, d, D; bool out_bf16; float scale; };

int check_shape(const echokv_shape* s, Sizes* o) {
  if (!s) return ECHOKV_ERR_NULL;
  if (s->dtype != ECHOKV_BF16 && s->dtype != ECHOKV_F32) return ECHOKV_ERR_DTYPE;
  if (s->out_dtype != ECHOKV_BF16 && s->out_dtype != ECHOKV_F32) return ECHOKV_ERR_DTYPE;
  if (s->n_q_heads <= 0 || s->n_kv_heads <= 0 || s->head_dim <= 0 || s->n_q_heads % s->n_kv_heads) return ECHOKV_ERR_SHAPE;
  if (s->n_kv_heads > 4096 || s->n_q_heads > 65536 || !std::isfinite(s->softmax_scale)) return ECHOKV_ERR_SHAPE;
  if (s->head_dim != 64 && s->head_dim != 128) return ECHOKV_ERR_UNSUPPORTED;
  if (s->dtype != ECHOKV_BF16 || s->flags) return ECHOKV_ERR_UNSUPPORTED;
  *o = {s->n_q_heads, s->n_kv_heads, s->n_q_heads / s->n_kv_heads, s->head_dim, s->n_kv_heads * s->head_dim, s->out_dtype == ECHOKV_BF16,
        s->softmax_scale > 0.f ? s->softmax_scale : 1.0f / std::sqrt((float)s->head_dim)};
  // scale * log2(e), scale / cap and slope / scale stay normal numbers
  return o->scale < 1e-10f || o->scale > 1e10f ? ECHOKV_ERR_SHAPE : ECHOKV_OK;
}

int check_table(const echokv_page_table* t) {
  if (!t) return ECHOKV_ERR_NULL;
  if (t->batch <= 0 || t->max_pages <= 0 || t->n_pages <= 0) return ECHOKV_ERR_SHAPE;
  if (t->batch > page::kMaxBatch || t->max_pages >= 1 << 23 || t->n_pages >= 1 << 24) return ECHOKV_ERR_UNSUPPORTED;      // lengths below 2^30, slots below 2^31
  if (!t->table || !t->seq_len || !t->free_list || !t->n_free) return ECHOKV_ERR_NULL;
  return ECHOKV_OK;
}

bool aligned16(std::initializer_list<const void*> ps) {
  return std::all_of(ps.begin(), ps.end(), [](const void* p) { return ((uintptr_t)p & 15) == 0; });
}

int check_cache(const echokv_page_cache* c) {
  if (!c || !c->k || !c->v || !c->k_exp || !c->v_exp || !c->k_tail || !c->v_tail) return ECHOKV_ERR_NULL;
  return aligned16({c->k, c->v, c->k_tail, c->v_tail}) ? ECHOKV_OK : ECHOKV_ERR_SHAPE;
}

size_t plan_bytes(int batch) { return ((page::kHeadWords + (size_t)page::Plan::kArrays * (batch + 1)) * 4 + 255) / 256 * 256; }

int check_plan(const echokv_page_plan* p, const Sizes& z, int batch) {
  if (!p || !p->buf) return ECHOKV_ERR_NULL;
  if (p->max_rows < 0 || p->max_rows > 1 << 30) return ECHOKV_ERR_SHAPE;
  if ((int64_t)p->max_rows * z.G >= (int64_t)1 << 30) return ECHOKV_ERR_UNSUPPORTED;      // (query, query head) columns in 32 bits
  if (p->bytes < plan_bytes(batch) || !aligned16({p->buf})) return ECHOKV_ERR_WORKSPACE;
  return ECHOKV_OK;
}

// ---- launches: items at most, and what they are shared out to.  grow (on the device) and the attention entry points go by the same numbers.
struct Schedule {
  int col_tiles, dec_items, pf_items, nw_items;
  int64_t dec_grid, pf_grid;                // items of a launch, at most
  int64_t pf_rows;                          // columns in a split prefill launch that leave partial results, of a KV head
  int64_t nw_grid, nw_parts;                // items of few columns, and those of them that leave partial results, at most
};
Schedule schedule(const Sizes& z, int batch, int max_rows) {
  Schedule s;
  s.col_tiles = (z.G + 15) / 16;
  s.dec_items = std::max(1, page::kDecodeItems / (z.H_kv * s.col_tiles));
  s.dec_grid = s.dec_items + 2 * (int64_t)batch;
  const int64_t cols = (int64_t)max_rows * z.G, seqs = std::min(batch, max_rows);
  const int64_t wide_seqs = cols > page::kNarrow ? std::min<int64_t>(seqs, cols / page::kNarrow) : 0, full = page::kPfFill / z.H_kv + 1;
  // blocks of 128 columns only where those of 384 (of 256 with a cap) are fewer than kPfMany, hence at most three times as many
  const int64_t few = 3 * ((int64_t)page::kPfMany / z.H_kv + 1);
  // split: fewer blocks than fill the chip, and no more shares than that beside each block's last one
  s.pf_items = std::max(1, page::kPfFill / z.H_kv);
  s.pf_grid = s.pf_rows = 0;
  for (int of : {page::kLCols, page::kMCols, page::kSCols}) {
    if (!wide_seqs) break;
    const int64_t all = cols / of + wide_seqs, n = of == page::kSCols ? std::min(all, few) : all, parts = s.pf_items + std::min(n, full);
    s.pf_grid = std::max(s.pf_grid, std::max(n, parts));
    s.pf_rows = std::max(s.pf_rows, parts * of);
  }
  // A block whose keys are split has more halves than a share: there are at most as many such blocks as shares' worth of work
  s.nw_items = std::max(1, page::kNarrowItems / z.H_kv);
  s.nw_grid = s.nw_items + std::min(seqs * ((page::kNarrow + page::kNCols - 1) / page::kNCols), cols / page::kNCols + seqs);
  s.nw_parts = 2 * (int64_t)s.nw_items;
  return s;
}

int launch_dims(int64_t blocks, int threads, dim3* grid) {
  if (blocks * threads >= (int64_t)1 << 32) return ECHOKV_ERR_UNSUPPORTED;
  *grid = dim3((unsigned)blocks);
  return ECHOKV_OK;
}

int attn_args(const Sizes& z, const echokv_page_table* t, const echokv_page_cache* c, const echokv_page_plan* p, const void* q,
              const echokv_score_extras* x, void* out, float* lse, const Schedule& s, page::AttnArgs* a) {
  if (!q || !out) return ECHOKV_ERR_NULL;
  if (!aligned16({q, out}) || ((uintptr_t)lse & 3)) return ECHOKV_ERR_SHAPE;
  if (x && (!std::isfinite(x->softcap) || x->softcap < 0.f || x->softcap > 1e20f || (x->softcap > 0.f && x->softcap < 1e-20f))) return ECHOKV_ERR_SHAPE;
  *a = page::AttnArgs{};
  a->k = (const uint8_t*)c->k; a->v = (const uint8_t*)c->v; a->ke = c->k_exp; a->ve = c->v_exp;
  a->kt = (const bf16_t*)c->k_tail; a->vt = (const bf16_t*)c->v_tail; a->q = (const bf16_t*)q;
  a->table = t->table; a->out = out; a->lse = lse;
  a->plan = {(int32_t*)p->buf, t->batch};
  a->key = {t->batch, z.H_q, z.H_kv, p->max_rows};
  a->scale = z.scale; a->max_pages = t->max_pages; a->n_pages = t->n_pages; a->G = z.G; a->col_tiles = s.col_tiles;
  if (x && x->softcap > 0.f) {
    // cap2 tanh(to_arg x) as x times a polynomial in x^2, where its coefficients are numbers of fp32
    const double k[4] = {0.99999997, -0.33332517, 0.13298439, -0.04913415}, arg = (double)z.scale / x->softcap;
    a->to_arg = (float)arg;
    if (arg > 1e-5 && arg < 1e4)
      for (int i = 0; i < 4; ++i) a->tanh_k[i] = (float)(k[i] * std::pow(arg, 2 * i + 1) * x->softcap * page::kLog2e);
  }
  a->capped = x && x->softcap > 0.f;
  if (x) { a->cap = x->softcap; a->slopes = x->slopes; a->prefix = x->prefix_len; }
  return ECHOKV_OK;
}

// Partials in the workspace: outputs, then (maximum, sum) pairs.
size_t part_bytes(int64_t rows, int d) { return (size_t)rows * (d + 2) * 4; }

int64_t wide_rows(const Sizes& z, const Schedule& s) { return s.pf_rows * z.H_kv; }
int64_t prefill_rows(const Sizes& z, const Schedule& s) { return wide_rows(z, s) + s.nw_parts * page::kNCols * z.H_kv; }

template <class F> int by_type(const Sizes& z, const page::AttnArgs& a, F f) {
  auto typed = [&](auto hd, auto mode) { return z.out_bf16 ? f(hd, mode, bf16_t{}) : f(hd, mode, float{}); };
  auto modal = [&](auto hd) {
    if (a.cap > 0.f) return a.slopes ? typed(hd, std::integral_constant<int, page::kCapBias>{}) : typed(hd, std::integral_constant<int, page::kCap>{});
    return a.slopes ? typed(hd, std::integral_constant<int, page::kBias>{}) : typed(hd, std::integral_constant<int, page::kPlain>{});
  };
  return z.d == 64 ? modal(std::integral_constant<int, 64>{}) : modal(std::integral_constant<int, 128>{});
}

}  // namespace

extern "C" {

size_t echokv_page_plan_bytes(int32_t batch) { return batch > 0 && batch <= page::kMaxBatch ? plan_bytes(batch) : 0; }

size_t echokv_page_workspace_bytes(const echokv_shape* shape, int32_t batch, int32_t max_rows) {
  Sizes z;
  if (check_shape(shape, &z) || batch <= 0 || batch > page::kMaxBatch || max_rows < 0 || (int64_t)max_rows * z.G >= (int64_t)1 << 30) return 0;
  const Schedule s = schedule(z, batch, max_rows);
  const size_t dec = part_bytes(s.dec_grid * z.H_q, z.d), pf = max_rows ? part_bytes(prefill_rows(z, s), z.d) : 0;
  return (std::max(dec, pf) + 255) / 256 * 256;
}

int echokv_pages_grow(const echokv_shape* shape, const echokv_page_table* t, const int32_t* n_new, int32_t* seq_len_out, int32_t* n_free_out,
                      int32_t* row_slot, int32_t* row_pos, const echokv_page_plan* plan, void* hip_stream) {
  Sizes z;
  int rc = check_shape(shape, &z);
  if (rc) return rc;
  if ((rc = check_table(t)) || (rc = check_plan(plan, z, t->batch))) return rc;
  if (!n_new || !seq_len_out || !n_free_out) return ECHOKV_ERR_NULL;
  const Schedule s = schedule(z, t->batch, plan->max_rows);
  page::GrowArgs a;
  a.len0 = t->seq_len; a.n_new = n_new; a.free_list = t->free_list; a.n_free0 = t->n_free;
  a.len1 = seq_len_out; a.n_free1 = n_free_out; a.table = t->table; a.slot = row_slot; a.pos = row_pos;
  a.plan = {(int32_t*)plan->buf, t->batch};
  a.max_pages = t->max_pages; a.n_pages = t->n_pages; a.max_rows = plan->max_rows; a.H_q = z.H_q; a.H_kv = z.H_kv;
  a.dec_items = s.dec_items; a.pf_items = s.pf_items; a.nw_items = s.nw_items;
  a.rows_here = plan->max_rows <= 4096 && t->batch <= 1024;      // (batch: what the workgroup below has threads for)
  const hipStream_t st = (hipStream_t)hip_stream;
  if (t->batch <= 256 && plan->max_rows <= 1024) hipLaunchKernelGGL(page::grow_kernel<256>, dim3(1), dim3(256), 0, st, a);
  else if (t->batch <= 512) hipLaunchKernelGGL(page::grow_kernel<512>, dim3(1), dim3(512), 0, st, a);
  else hipLaunchKernelGGL(page::grow_kernel<1024>, dim3(1), dim3(1024), 0, st, a);
  LAUNCH_CHECK();
  if (!a.rows_here && plan->max_rows > 0) {
    hipLaunchKernelGGL(page::grow_rows_kernel, dim3((plan->max_rows + page::kRowsPerBlock - 1) / page::kRowsPerBlock), dim3(page::kRowsPerBlock), 0, st, a);
    LAUNCH_CHECK();
  }
  return ECHOKV_OK;
}

int echokv_pages_slots(const echokv_page_table* t, const int32_t* row_start, const int32_t* first_pos, int32_t n_rows, int32_t* row_slot,
                       void* hip_stream) {
  const int rc = check_table(t);
  if (rc) return rc;
  if (n_rows < 0) return ECHOKV_ERR_SHAPE;
  if (n_rows == 0) return ECHOKV_OK;
  if (!row_start || !first_pos || !row_slot) return ECHOKV_ERR_NULL;
  const page::SlotArgs a = {t->table, t->seq_len, row_start, first_pos, row_slot, t->batch, t->max_pages, n_rows};
  hipLaunchKernelGGL(page::slots_kernel, dim3((unsigned)(((int64_t)n_rows + 255) / 256)), dim3(256), 0, (hipStream_t)hip_stream, a);
  LAUNCH_CHECK();
  return ECHOKV_OK;
}

int echokv_pages_release(const echokv_page_table* t, const int32_t* which, void* hip_stream) {
  const int rc = check_table(t);
  if (rc) return rc;
  if (!which) return ECHOKV_ERR_NULL;
  const page::ReleaseArgs a = {which, t->table, t->seq_len, t->free_list, t->n_free, t->batch, t->max_pages, t->n_pages};
  hipLaunchKernelGGL(page::release_kernel<1024>, dim3(1), dim3(1024), 0, (hipStream_t)hip_stream, a);
  LAUNCH_CHECK();
  return ECHOKV_OK;
}

int echokv_page_append(const echokv_shape* shape, const echokv_page_table* t, const echokv_page_cache* c, const echokv_page_plan* plan,
                       const void* k_new, const void* v_new, void* hip_stream) {
  Sizes z;
  int rc = check_shape(shape, &z);
  if (rc) return rc;
  if ((rc = check_table(t)) || (rc = check_cache(c)) || (rc = check_plan(plan, z, t->batch))) return rc;
  if (plan->max_rows == 0) return ECHOKV_OK;
  if (!k_new || !v_new) return ECHOKV_ERR_NULL;
  if (!aligned16({k_new, v_new})) return ECHOKV_ERR_SHAPE;
  page::StoreArgs a;
  a.k = (uint8_t*)c->k; a.v = (uint8_t*)c->v; a.ke = c->k_exp; a.ve = c->v_exp; a.kt = (bf16_t*)c->k_tail; a.vt = (bf16_t*)c->v_tail;
  a.kn = (const bf16_t*)k_new; a.vn = (const bf16_t*)v_new; a.table = t->table;
  a.plan = {(int32_t*)plan->buf, t->batch};
  a.key = {t->batch, z.H_q, z.H_kv, plan->max_rows};
  a.max_pages = t->max_pages; a.n_pages = t->n_pages;
  dim3 grid;
  // a sequence has an item for every block that is completed, at least one if it has new rows at all
  const int64_t items = plan->max_rows / page::kTokens + std::min(t->batch, plan->max_rows);
  if ((rc = launch_dims(items * z.H_kv * 2, 256, &grid))) return rc;
  if (z.d == 64) hipLaunchKernelGGL(page::append_kernel<64>, grid, dim3(256), 0, (hipStream_t)hip_stream, a);
  else hipLaunchKernelGGL(page::append_kernel<128>, grid, dim3(256), 0, (hipStream_t)hip_stream, a);
  LAUNCH_CHECK();
  return ECHOKV_OK;
}

int echokv_page_read(const echokv_shape* shape, const echokv_page_table* t, const echokv_page_cache* c, const int32_t* row_slot, int32_t n_rows,
                     void* k_out, void* v_out, void* hip_stream) {
  Sizes z;
  int rc = check_shape(shape, &z);
  if (rc) return rc;
  if ((rc = check_table(t)) || (rc = check_cache(c))) return rc;
  if (n_rows < 0) return ECHOKV_ERR_SHAPE;
  if (n_rows > 1 << 30) return ECHOKV_ERR_UNSUPPORTED;
  if (n_rows == 0) return ECHOKV_OK;
  if (!row_slot || !k_out || !v_out) return ECHOKV_ERR_NULL;
  if (!aligned16({k_out, v_out})) return ECHOKV_ERR_SHAPE;
  dim3 grid;
  if ((rc = launch_dims(((int64_t)n_rows + page::kTokens - 1) / page::kTokens * z.H_kv, 256, &grid))) return rc;
  auto run = [&](auto hd, auto to) {
    using TO = decltype(to);
    page::ReadArgs<TO> a = {(const uint8_t*)c->k, (const uint8_t*)c->v, c->k_exp, c->v_exp, (const bf16_t*)c->k_tail, (const bf16_t*)c->v_tail,
                            row_slot, (TO*)k_out, (TO*)v_out, n_rows, t->n_pages, t->batch, z.H_kv};
    hipLaunchKernelGGL((page::read_kernel<decltype(hd)::value, TO>), grid, dim3(256), 0, (hipStream_t)hip_stream, a);
  };
  auto typed = [&](auto hd) { if (z.out_bf16) run(hd, bf16_t{}); else run(hd, float{}); };
  if (z.d == 64) typed(std::integral_constant<int, 64>{}); else typed(std::integral_constant<int, 128>{});
  LAUNCH_CHECK();
  return ECHOKV_OK;
}

int echokv_page_decode_attn(const echokv_shape* shape, const echokv_page_table* t, const echokv_page_cache* c, const echokv_page_plan* plan,
                            const void* q, const echokv_score_extras* extras, void* out, float* lse_out, void* workspace,
                            size_t workspace_bytes, void* hip_stream) {
  Sizes z;
  int rc = check_shape(shape, &z);
  if (rc) return rc;
  if ((rc = check_table(t)) || (rc = check_cache(c)) || (rc = check_plan(plan, z, t->batch))) return rc;
  const Schedule s = schedule(z, t->batch, plan->max_rows);
  page::AttnArgs a;
  if ((rc = attn_args(z, t, c, plan, q, extras, out, lse_out, s, &a))) return rc;
  const int64_t rows = s.dec_grid * z.H_q;
  if (!workspace || !aligned16({workspace}) || workspace_bytes < part_bytes(rows, z.d)) return ECHOKV_ERR_WORKSPACE;
  a.part_o = (float*)workspace;
  a.part_ml = a.part_o + rows * z.d;
  dim3 grid, merge;
  if ((rc = launch_dims(s.dec_grid * z.H_kv * s.col_tiles, 256, &grid)) || (rc = launch_dims((int64_t)t->batch * z.H_q, 256, &merge))) return rc;
  return by_type(z, a, [&](auto hd, auto mode, auto to) -> int {
    constexpr int HD = decltype(hd)::value;
    using TO = decltype(to);
    hipLaunchKernelGGL((page::decode_kernel<HD, decltype(mode)::value, TO>), grid, dim3(256), 0, (hipStream_t)hip_stream, a);
    LAUNCH_CHECK();
    hipLaunchKernelGGL((page::decode_merge_kernel<HD, TO>), merge, dim3(256), 0, (hipStream_t)hip_stream, a);
    LAUNCH_CHECK();
    return ECHOKV_OK;
  });
}

int echokv_page_prefill_attn(const echokv_shape* shape, const echokv_page_table* t, const echokv_page_cache* c, const echokv_page_plan* plan,
                             const void* q, const echokv_score_extras* extras, void* out, float* lse_out, void* workspace,
                             size_t workspace_bytes, void* hip_stream) {
  Sizes z;
  int rc = check_shape(shape, &z);
  if (rc) return rc;
  if ((rc = check_table(t)) || (rc = check_cache(c)) || (rc = check_plan(plan, z, t->batch))) return rc;
  if (plan->max_rows == 0) return ECHOKV_OK;
  const Schedule s = schedule(z, t->batch, plan->max_rows);
  page::AttnArgs a;
  if ((rc = attn_args(z, t, c, plan, q, extras, out, lse_out, s, &a))) return rc;
  const int64_t rows = wide_rows(z, s), all = prefill_rows(z, s);
  if (!workspace || !aligned16({workspace}) || workspace_bytes < part_bytes(all, z.d)) return ECHOKV_ERR_WORKSPACE;
  a.part_o = (float*)workspace;
  a.nw_o = a.part_o + rows * z.d;
  a.part_ml = a.part_o + all * z.d;
  a.nw_ml = a.part_ml + rows * 2;
  dim3 grid;
  const dim3 merge((unsigned)std::min<int64_t>((int64_t)plan->max_rows * z.H_q, page::kMergeBlocks));
  if ((rc = launch_dims((s.pf_grid + s.nw_grid) * z.H_kv, page::kPfThreads, &grid))) return rc;
  return by_type(z, a, [&](auto hd, auto mode, auto to) -> int {
    constexpr int HD = decltype(hd)::value;
    using TO = decltype(to);
    hipLaunchKernelGGL((page::prefill_kernel<HD, decltype(mode)::value, TO>), grid, dim3(page::kPfThreads), 0, (hipStream_t)hip_stream, a, (int)s.pf_grid);
    LAUNCH_CHECK();
    hipLaunchKernelGGL((page::prefill_merge_kernel<HD, TO>), merge, dim3(256), 0, (hipStream_t)hip_stream, a);
    LAUNCH_CHECK();
    return ECHOKV_OK;
  });
}

}  // extern "C"
