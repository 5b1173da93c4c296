// Host side of the 4-bit cache's entry points: validation and launches.  No allocation of device memory, no synchronisation.
#include <string.h>

#include <new>

#include "host_objects.hpp"

using namespace ts;

namespace {

int check_sizes(const trispec_mx_cache *c, size_t *slots_all) {
  if (!c) return TRISPEC_ENULL;
  if (c->batch < 1 || c->batch > kMaxBatch) return TRISPEC_ENODES;
  if (c->n_kv_heads < 1 || c->n_kv_heads > 65535 || (c->head_dim != 64 && c->head_dim != 128)) return TRISPEC_ESHAPE;
  if (c->page_table) {
    if (c->n_pages < 1 || c->n_pages > (1 << 22) || c->max_pages < 1 || c->max_pages > (1 << 22) / kKvPage) return TRISPEC_ECAPACITY;
  } else if (c->capacity < 64 || c->capacity % 64 || c->capacity > (1 << 26)) {
    return TRISPEC_ECAPACITY;
  }
  *slots_all = (c->page_table ? (size_t)c->n_pages * kKvPage : (size_t)c->batch * c->capacity) * c->n_kv_heads;
  return TRISPEC_OK;
}

int capacity_of(const trispec_mx_cache *c) { return c->page_table ? c->max_pages * kKvPage : c->capacity; }

int check_cache(const trispec_mx_cache *c, size_t *slots_all) {
  const int rc = check_sizes(c, slots_all);
  if (rc) return rc;
  if (!c->k_codes || !c->k_scales || !c->v_codes || !c->v_scales) return TRISPEC_ENULL;
  if (((uintptr_t)c->k_codes | (uintptr_t)c->k_scales | (uintptr_t)c->v_codes | (uintptr_t)c->v_scales) & 15) return TRISPEC_EARG;
  if ((uintptr_t)c->page_table & 3) return TRISPEC_EARG;
  return TRISPEC_OK;
}

MxMap map_of(const trispec_mx_cache *c) {
  MxMap m;
  m.k_codes = (uint8_t *)c->k_codes; m.k_scales = (uint8_t *)c->k_scales;
  m.v_codes = (uint8_t *)c->v_codes; m.v_scales = (uint8_t *)c->v_scales;
  m.page_table = c->page_table;
  m.max_pages = c->max_pages; m.n_pages = c->n_pages;
  m.slots = c->page_table ? kKvPage : c->capacity;
  m.n_kv = c->n_kv_heads;
  return m;
}

bool dtype_ok(int32_t dtype) { return dtype == TRISPEC_F32 || dtype == TRISPEC_BF16; }

bool rows_ok(const trispec_mx_rows &r, int32_t dtype) {
  const int64_t unit = dtype == TRISPEC_F32 ? 4 : 8;   // elements of 16 bytes
  return !((uintptr_t)r.data & 15) && r.row_stride >= 0 && r.seq_stride >= 0 && r.row_stride % unit == 0 && r.seq_stride % unit == 0;
}

MxRows rows_of(const trispec_mx_rows &r) { return MxRows{r.data, r.row_stride, r.seq_stride}; }

// Whether no two of the batch * n rows of `width` elements share one: sequences behind one another, or rows of all sequences side by side
bool rows_apart(const trispec_mx_rows &r, int batch, int64_t n, int64_t width) {
  if (n > 1 && r.row_stride < width) return false;
  if (batch > 1 && r.seq_stride < width) return false;
  return batch == 1 || n <= 1 || r.seq_stride >= (n - 1) * r.row_stride + width || r.row_stride >= (batch - 1) * r.seq_stride + width;
}

// start and count of every sequence, checked; the largest count
int take_range(const trispec_mx_cache *c, const int32_t *start, const int32_t *count, int32_t *to_start, int32_t *to_count, int *most) {
  if (!start || !count) return TRISPEC_ENULL;
  const int cap = capacity_of(c);
  *most = 0;
  for (int b = 0; b < kMaxBatch; ++b) to_start[b] = to_count[b] = 0;
  for (int b = 0; b < c->batch; ++b) {
    if (start[b] < 0 || count[b] < 0 || start[b] > cap || count[b] > cap - start[b]) return TRISPEC_ECAPACITY;
    to_start[b] = start[b];
    to_count[b] = count[b];
    if (count[b] > *most) *most = count[b];
  }
  return TRISPEC_OK;
}

struct AttendLayout {
  size_t o, m, l, total;
};
AttendLayout attend_layout(int batch, int n_nodes, int group, int n_kv, int head_dim) {
  const size_t rows = mx_max_parts(batch, n_kv, group, n_nodes) * n_kv * group * n_nodes;
  auto up = [](size_t v) { return (v + 255) / 256 * 256; };
  AttendLayout L;
  L.o = 0;
  L.m = up(rows * head_dim * sizeof(float));
  L.l = L.m + up(rows * sizeof(float));
  L.total = L.l + up(rows * sizeof(float));
  return L;
}

int check_heads(int batch, int n_nodes, int n_q_heads, int n_kv_heads, int head_dim) {
  if (batch < 1 || batch > kMaxBatch || n_nodes < 1 || n_nodes > kMaxNodes || batch * n_nodes > kMaxRows) return TRISPEC_ENODES;
  if (n_kv_heads < 1 || n_kv_heads > 65535 || n_q_heads < 1 || n_q_heads % n_kv_heads || n_q_heads / n_kv_heads > kMaxGroup ||
      (head_dim != 64 && head_dim != 128))
    return TRISPEC_ESHAPE;
  if (n_q_heads / n_kv_heads * n_nodes > 512) return TRISPEC_ENODES;
  return TRISPEC_OK;
}

}  // namespace

extern "C" {

int trispec_mx_cache_bytes(const trispec_mx_cache *c, size_t *code_bytes, size_t *scale_bytes) {
  if (!code_bytes || !scale_bytes) return TRISPEC_ENULL;
  size_t slots;
  const int rc = check_sizes(c, &slots);
  if (rc) return rc;
  *code_bytes = slots * (c->head_dim / 2);
  *scale_bytes = slots * (c->head_dim / kMxBlock);
  return TRISPEC_OK;
}

int trispec_mx_append(const trispec_mx_cache *c, const trispec_mx_rows *k, const trispec_mx_rows *v, int32_t dtype,
                      const int32_t *start_host, const int32_t *count_host, void *stream) {
  if (!c || !k || !v || !k->data || !v->data) return TRISPEC_ENULL;
  size_t slots;
  int rc = check_cache(c, &slots);
  if (rc) return rc;
  if (!dtype_ok(dtype) || !rows_ok(*k, dtype) || !rows_ok(*v, dtype)) return TRISPEC_EARG;
  MxAppendArgs a;
  memset(&a, 0, sizeof(a));
  int most;
  rc = take_range(c, start_host, count_host, a.start, a.count, &most);
  if (rc) return rc;
  if (most == 0) return TRISPEC_OK;
  a.c = map_of(c);
  a.k = rows_of(*k);
  a.v = rows_of(*v);
  a.head_dim = c->head_dim;
  a.dtype = dtype;
  (void)hipGetLastError();
  launch_mx_append((hipStream_t)stream, a, c->batch);
  return hipGetLastError() == hipSuccess ? TRISPEC_OK : TRISPEC_ELAUNCH;
}

int trispec_mx_read(const trispec_mx_cache *c, const trispec_mx_rows *k, const trispec_mx_rows *v, int32_t dtype,
                    const int32_t *start_host, const int32_t *count_host, void *stream) {
  if (!c || (!k && !v) || (k && !k->data) || (v && !v->data)) return TRISPEC_ENULL;
  size_t slots;
  int rc = check_cache(c, &slots);
  if (rc) return rc;
  if (!dtype_ok(dtype) || (k && !rows_ok(*k, dtype)) || (v && !rows_ok(*v, dtype))) return TRISPEC_EARG;
  MxReadArgs a;
  memset(&a, 0, sizeof(a));
  int most;
  rc = take_range(c, start_host, count_host, a.start, a.count, &most);
  if (rc) return rc;
  const int64_t width = (int64_t)c->n_kv_heads * c->head_dim;
  if ((k && !rows_apart(*k, c->batch, most, width)) || (v && !rows_apart(*v, c->batch, most, width))) return TRISPEC_EARG;
  if (most == 0) return TRISPEC_OK;
  a.c = map_of(c);
  if (k) { a.k = k->data; a.k_row = k->row_stride; a.k_seq = k->seq_stride; }
  if (v) { a.v = v->data; a.v_row = v->row_stride; a.v_seq = v->seq_stride; }
  a.head_dim = c->head_dim;
  a.dtype = dtype;
  (void)hipGetLastError();
  launch_mx_read((hipStream_t)stream, a, c->batch);
  return hipGetLastError() == hipSuccess ? TRISPEC_OK : TRISPEC_ELAUNCH;
}

int trispec_mx_attend_workspace_bytes(int32_t batch, int32_t n_nodes, int32_t n_q_heads, int32_t n_kv_heads, int32_t head_dim,
                                      size_t *bytes) {
  if (!bytes) return TRISPEC_ENULL;
  const int rc = check_heads(batch, n_nodes, n_q_heads, n_kv_heads, head_dim);
  if (rc) return rc;
  *bytes = attend_layout(batch, n_nodes, n_q_heads / n_kv_heads, n_kv_heads, head_dim).total;
  return TRISPEC_OK;
}

int trispec_mx_attend(const trispec_mx_cache *c, const int32_t *ctx_len_host, const int32_t *tree_parents, const trispec_mx_attend_args *x) {
  if (!c || !ctx_len_host || !x || !x->q.data || !x->out || !x->k.data != !x->v.data) return TRISPEC_ENULL;
  const bool own = x->k.data != nullptr;
  if (x->append && !own) return TRISPEC_ENULL;
  size_t slots;
  int rc = check_cache(c, &slots);
  if (rc) return rc;
  const int B = c->batch, M = x->n_nodes, D = c->head_dim;
  rc = check_heads(B, M, x->n_q_heads, c->n_kv_heads, D);
  if (rc) return rc;
  if (!dtype_ok(x->dtype) || !rows_ok(x->q, x->dtype) || (own && (!rows_ok(x->k, x->dtype) || !rows_ok(x->v, x->dtype)))) return TRISPEC_EARG;
  if (x->append != 0 && x->append != 1) return TRISPEC_EARG;
  if (((uintptr_t)x->out & 15) || x->out_row_stride < (int64_t)x->n_q_heads * D || x->out_row_stride % (x->dtype == TRISPEC_F32 ? 4 : 8)) return TRISPEC_EARG;
  const int cap = capacity_of(c), group = x->n_q_heads / c->n_kv_heads;
  MxAttnArgs a;
  memset(&a, 0, sizeof(a));
  for (int b = 0; b < B; ++b) {
    const int n = ctx_len_host[b];
    if (n < 0 || n > cap || (x->append && M > cap - n)) return TRISPEC_ECAPACITY;
    a.ctx.v[b] = n;
  }
  a.chain = tree_parents == nullptr;
  if (tree_parents)
    for (int i = 0; i < B * M; ++i) {
      const int node = i % M, p = tree_parents[i];
      if (node == 0 ? p != -1 : (p < 0 || p >= node)) return TRISPEC_ETREE;
      a.parent[i] = (uint8_t)(node == 0 ? 0 : p);
    }
  const AttendLayout L = attend_layout(B, M, group, c->n_kv_heads, D);
  if (!x->workspace || ((uintptr_t)x->workspace & 255) || x->workspace_bytes < L.total) return TRISPEC_EWORKSPACE;
  const MxPlan p = plan_mx(B, c->n_kv_heads, group, M, own, x->dtype == TRISPEC_F32, a.ctx.v);
  a.c = map_of(c);
  a.q = rows_of(x->q);
  a.k = rows_of(x->k);
  a.v = rows_of(x->v);
  a.batch = B; a.n_nodes = M; a.n_q_heads = x->n_q_heads; a.group = group; a.head_dim = D; a.dtype = x->dtype;
  a.append = x->append;
  a.whole = p.whole; a.form = p.form; a.n_row_groups = p.n_row_groups;
  a.n_own = p.n_own; a.keys = p.keys;
  mx_split_table(p, B, a.ctx.v, a.split0);
  char *ws = (char *)x->workspace;
  a.part_o = (float *)(ws + L.o);
  a.part_m = (float *)(ws + L.m);
  a.part_l = (float *)(ws + L.l);
  a.out = x->out;
  a.out_row = x->out_row_stride;
  (void)hipGetLastError();
  launch_mx_attn((hipStream_t)x->stream, a);
  return hipGetLastError() == hipSuccess ? TRISPEC_OK : TRISPEC_ELAUNCH;
}

int trispec_kv_create_mx(const trispec_model *m, const trispec_mx_cache *c, trispec_kv **out) {
  if (!m || !c || !out) return TRISPEC_ENULL;
  size_t slots;
  const int rc = check_cache(c, &slots);
  if (rc) return rc;
  if (m->cfg.dtype != TRISPEC_BF16) return TRISPEC_ESHAPE;
  if (c->n_kv_heads != m->cfg.n_kv_heads || c->head_dim != m->cfg.head_dim) return TRISPEC_EMISMATCH;
  trispec_kv *kv = new (std::nothrow) trispec_kv;
  if (!kv) return TRISPEC_EARG;
  kv->model = m;
  kv->k = kv->v = nullptr;
  kv->batch = c->batch;
  kv->capacity = capacity_of(c);
  kv->page_table = c->page_table;
  kv->max_pages = c->page_table ? c->max_pages : 0;
  kv->n_pages = c->page_table ? c->n_pages : 0;
  kv->held_in_mx = true;
  kv->mx = map_of(c);
  kv->mx_slots = slots;
  for (int b = 0; b < kMaxBatch; ++b) kv->ctx_len[b] = 0;
  *out = kv;
  return TRISPEC_OK;
}

}  // extern "C"
