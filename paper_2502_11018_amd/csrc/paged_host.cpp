// Host side of the 8-bit paged cache's entry points (griffin_paged_*): checks
// of the arguments and the launches.  No device memory is allocated and
// nothing is copied or waited for, so the calls can be captured.

#include <hip/hip_runtime.h>

#include <cmath>

#include "griffin_verify.h"
#include "paged.h"
#include "paged_host.h"

using namespace griffin;

namespace griffin {

namespace {

int type_bytes(int dtype) { return dtype == PT_F32 ? 4 : 2; }
bool aligned(const void* p, size_t n) { return (reinterpret_cast<uintptr_t>(p) & (n - 1)) == 0; }

// rows of `heads` heads: 1 if 8 consecutive values are always aligned to their size
int vector_rows(const void* p, long long sb, long long sr, long long sh, int dtype) {
  const int n = 16 / type_bytes(dtype);  // values of a 16-byte access
  return aligned(p, 16) && sb % n == 0 && sr % n == 0 && sh % n == 0;
}

PagedRows rows_of(const griffin_rows& r, int dtype) {
  return PagedRows{r.data, r.stride_seq, r.stride_row, r.stride_head,
                   vector_rows(r.data, r.stride_seq, r.stride_row, r.stride_head, dtype)};
}

int check_rows(const griffin_rows& r, int dtype) {
  return r.data && aligned(r.data, type_bytes(dtype)) && r.stride_seq >= 0 && r.stride_row >= 0 && r.stride_head >= 0;
}

}  // namespace

int paged_pool_of(const griffin_pool& p, PagedPool* out) {
  if (!p.k || !p.v || !p.k_exp || !p.v_exp || !aligned(p.k, 16) || !aligned(p.v, 16)) return GRIFFIN_EINVAL;
  if ((p.head_dim != 64 && p.head_dim != 128) || p.n_kv_heads < 1 || p.page_slots < 32 || p.page_slots % 32 != 0 ||
      p.n_pages < 1)
    return GRIFFIN_ESHAPE;
  if ((long long)p.n_pages * p.n_kv_heads * (p.page_slots / 32) > 0x7fffffffLL) return GRIFFIN_ESHAPE;
  *out = PagedPool{static_cast<uint8_t*>(p.k), static_cast<uint8_t*>(p.v), static_cast<int8_t*>(p.k_exp),
                   static_cast<int8_t*>(p.v_exp), p.n_pages, p.page_slots / 32, p.n_kv_heads, p.head_dim};
  return GRIFFIN_OK;
}

bool paged_sizes(const PagedPool& pool, int batch, int nodes, int n_q_heads) {
  return (long long)batch * nodes <= PAGED_MAX_GROUPS && (long long)batch * pool.Hkv <= PAGED_MAX_GROUPS &&
         (long long)n_q_heads * nodes <= (1 << 18);
}

// max_length < 0: the table's capacity
int paged_table_of(const griffin_pool& pool, const int32_t* table, int stride, int cols, const int32_t* lengths,
                   int max_length, PagedTable* out) {
  if (!table || !lengths || cols < 1 || stride < cols) return GRIFFIN_EINVAL;
  const long long cap = (long long)cols * pool.page_slots;
  if (cap > 0x7fffffffLL - 4096) return GRIFFIN_ESHAPE;  // positions of nodes stay 32-bit
  if (max_length > cap) return GRIFFIN_ECAPACITY;
  *out = PagedTable{table, stride, cols, lengths, max_length < 0 ? (int)cap : max_length};
  return GRIFFIN_OK;
}

void paged_frequencies(double base, int dh, double* inv_rev) {
  for (int i = 0; i < dh / 2; ++i) inv_rev[i] = std::pow(base, -2.0 * i / dh) / 6.283185307179586476925;
}

}  // namespace griffin

namespace {

int attention_args(const griffin_attention* g, PagedAttn* out) {
  PagedAttn& a = *out;
  a = PagedAttn{};
  int rc = paged_pool_of(g->pool, &a.pool);
  if (rc != GRIFFIN_OK) return rc;
  if (g->dtype < PT_BF16 || g->dtype > PT_F32) return GRIFFIN_EINVAL;
  if (g->batch < 1 || g->window < 0 || g->sinks < 0 || !(g->scale > 0.f) || !std::isfinite(g->scale)) return GRIFFIN_EINVAL;
  if (g->nodes < 1 || g->nodes > 64) return GRIFFIN_ETREE;
  if (g->n_q_heads < 1 || g->n_q_heads % a.pool.Hkv != 0) return GRIFFIN_ESHAPE;
  if (!paged_sizes(a.pool, g->batch, g->nodes, g->n_q_heads)) return GRIFFIN_ESHAPE;
  a.dtype = g->dtype;
  a.batch = g->batch;
  a.nodes = a.stride = g->nodes;
  a.Hq = g->n_q_heads;
  a.scale_log2 = (float)((double)g->scale * 1.4426950408889634);
  a.cut.window = g->window;
  a.cut.sinks = g->window ? g->sinks : 0;
  rc = paged_table_of(g->pool, g->table, g->table_stride, g->table_cols, g->lengths, g->max_length, &a.tab);
  if (rc != GRIFFIN_OK) return rc;
  return paged_plan(a, a.tab.most) == 0 ? GRIFFIN_OK : GRIFFIN_ESHAPE;
}

}  // namespace

extern "C" {

int griffin_paged_append(const griffin_append* g, void* hip_stream) {
  if (!g) return GRIFFIN_EINVAL;
  PagedAppend a{};
  int rc = paged_pool_of(g->pool, &a.pool);
  if (rc != GRIFFIN_OK) return rc;
  if (g->dtype < PT_BF16 || g->dtype > PT_F32 || g->batch < 1 || g->rows < 1 || g->max_new < 0) return GRIFFIN_EINVAL;
  if (!check_rows(g->k, g->dtype) || !check_rows(g->v, g->dtype)) return GRIFFIN_EINVAL;
  if (g->path ? g->path_stride < g->max_new : g->max_new > g->rows) return GRIFFIN_EINVAL;
  if (!(g->rope_base >= 0.0) || !std::isfinite(g->rope_base)) return GRIFFIN_EINVAL;
  rc = paged_table_of(g->pool, g->table, g->table_stride, g->table_cols, g->lengths, -1, &a.tab);
  if (rc != GRIFFIN_OK) return rc;
  if (g->max_new == 0) return GRIFFIN_OK;
  if ((long long)g->batch * (g->max_new / 32 + 2) > PAGED_MAX_GROUPS) return GRIFFIN_ESHAPE;
  a.counts = g->counts;
  a.counts_stride = 1;
  a.path = g->path;
  a.path_stride = g->path_stride;
  a.k = rows_of(g->k, g->dtype);
  a.v = rows_of(g->v, g->dtype);
  a.dtype = g->dtype;
  a.batch = g->batch;
  a.rows = g->rows;
  a.max_new = g->max_new;
  a.rotate = g->rope_base > 0.0;
  if (a.rotate) paged_frequencies(g->rope_base, a.pool.dh, a.inv_rev);
  a.layers = 1;
  a.status = g->status;
  return launch_paged_append(a, static_cast<hipStream_t>(hip_stream)) == hipSuccess ? GRIFFIN_OK : GRIFFIN_EHIP;
}

size_t griffin_paged_attention_workspace(const griffin_attention* g) {
  PagedAttn a;
  if (!g || attention_args(g, &a) != GRIFFIN_OK) return 0;
  return paged_workspace(a, nullptr);
}

int griffin_paged_attention(const griffin_attention* g, void* workspace, size_t workspace_bytes, void* hip_stream) {
  if (!g) return GRIFFIN_EINVAL;
  PagedAttn a;
  int rc = attention_args(g, &a);
  if (rc != GRIFFIN_OK) return rc;
  for (const griffin_rows* r : {&g->q, &g->k, &g->v, &g->out})
    if (!check_rows(*r, g->dtype)) return GRIFFIN_EINVAL;
  const size_t need = paged_workspace(a, workspace);
  if (need && (!workspace || !aligned(workspace, 16))) return GRIFFIN_EINVAL;
  if (need > workspace_bytes) return GRIFFIN_ENOMEM;
  a.counts = g->counts;
  a.anc = g->anc;
  a.q = rows_of(g->q, g->dtype);
  a.k = rows_of(g->k, g->dtype);
  a.v = rows_of(g->v, g->dtype);
  const PagedRows o = rows_of(g->out, g->dtype);
  a.out = const_cast<void*>(g->out.data);
  a.ob = o.sb;
  a.orow = o.sr;
  a.oh = o.sh;
  a.out_vec = o.vec;
  a.status = g->status;
  return launch_paged_attention(a, static_cast<hipStream_t>(hip_stream)) == hipSuccess ? GRIFFIN_OK : GRIFFIN_EHIP;
}

}  // extern "C"
