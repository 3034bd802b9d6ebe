// C entry points of the operators outside of a state: argument checks and launches.
#include <math.h>

#include <limits>

#include "../../include/skd.h"
#include "kv_ops.h"
#include "sample_rows.h"

using namespace skd;

namespace {

bool aligned(const void *p) { return ((uintptr_t)p & 15) == 0; }
// 4-byte elements
bool aligned4(std::initializer_list<const void *> ps) {
  for (const void *p : ps)
    if ((uintptr_t)p & 3) return false;
  return true;
}

int check_kv(const skd_kv *kv) {
  if (!kv) return SKD_ERR_NULL;
  if (kv->elem != SKD_KV_BF16 && kv->elem != SKD_KV_FP8) return SKD_ERR_SHAPE;
  if (kv->head_dim != 64 && kv->head_dim != 128) return SKD_ERR_SHAPE;
  if (kv->kv_heads < 1 || kv->kv_heads > 65536 || kv->page_tokens < 32 || kv->page_tokens % 32 || kv->pages < 1 || kv->rows < 0 || kv->max_pages < 1) return SKD_ERR_SHAPE;
  if ((int64_t)kv->max_pages * kv->page_tokens >= 1 << 30) return SKD_ERR_RANGE;  // positions are counted in 32 bits
  return SKD_OK;
}
int check_call(const skd_kv *kv, const skd_kv_chunk *ch) {
  const int rc = check_kv(kv);
  if (rc != SKD_OK) return rc;
  if (!ch) return SKD_ERR_NULL;
  if (ch->tokens < 0 || ch->max_new < 0 || ch->max_past < 0) return SKD_ERR_RANGE;
  return SKD_OK;
}
// The device memory of a call, which is the current device's: a pointer of another one, or of memory that no device knows, is
// refused before it reaches a kernel.
int check_memory(std::initializer_list<const void *> ps) {
  int device = 0;
  if (const hipError_t e = hipGetDevice(&device); e != hipSuccess) return hip_failed(e);
  for (const void *p : ps) {
    hipPointerAttribute_t at{};
    if (hipPointerGetAttributes(&at, p) != hipSuccess) {
      (void)hipGetLastError();
      return SKD_ERR_RANGE;
    }
    if (at.type == hipMemoryTypeUnregistered || (at.type == hipMemoryTypeDevice && at.device != device)) return SKD_ERR_RANGE;
  }
  return SKD_OK;
}
int check_rows(const void *p, int64_t stride, int64_t width) {
  if (!p) return SKD_ERR_NULL;
  if (stride < width || stride % 8 || !aligned(p)) return SKD_ERR_SHAPE;
  return SKD_OK;
}

KvView view(const skd_kv *kv) {
  KvView v{};
  v.g.page_tokens = kv->page_tokens;
  v.g.max_pages = kv->max_pages;
  v.g.H = kv->kv_heads;
  v.g.dh = kv->head_dim;
  v.fp8 = kv->elem == SKD_KV_FP8;
  v.pages = kv->pages;
  v.rows = kv->rows;
  v.page_bytes = (long)skd_kv_page_bytes(kv);
  v.pool = (unsigned char *)kv->pool;
  v.table = kv->block_table;
  return v;
}
KvTokens tokens(const skd_kv *kv, const skd_kv_chunk *ch) {
  KvTokens t{};
  t.kind = KvTokens::RAGGED;
  t.first = ch->first;
  t.past = ch->past;
  t.tokens = ch->tokens;
  t.step = 1;
  // no row has more positions than its pages hold, nor more new tokens than there are
  const int64_t room = (int64_t)kv->max_pages * kv->page_tokens;
  t.max_new = (int)std::min<int64_t>(std::min(ch->max_new, ch->tokens), room);
  t.max_past = (int)std::min<int64_t>(ch->max_past, room);
  t.room = (int)room;
  return t;
}
KvRows rows_of(const void *p, int64_t stride) { return KvRows{const_cast<void *>(p), (long)stride, 0, false}; }

int launched() {
  const hipError_t e = hipGetLastError();
  return e == hipSuccess ? SKD_OK : hip_failed(e);
}
bool fits_int(__int128 n) { return n <= std::numeric_limits<int32_t>::max(); }

#define CHECK(expr)          \
  do {                       \
    const int r_ = (expr);   \
    if (r_ < 0) return r_;   \
  } while (0)

}  // namespace

extern "C" int64_t skd_kv_page_bytes(const skd_kv *kv) {
  CHECK(check_kv(kv));
  return kv->elem == SKD_KV_FP8 ? (int64_t)kv8_page_bytes(kv->kv_heads, kv->head_dim, kv->page_tokens)
                                : (int64_t)kv->kv_heads * kv->page_tokens * 4 * kv->head_dim;
}

extern "C" int skd_kv_append(const skd_kv *kv, const skd_kv_chunk *ch, const void *k, int64_t k_stride, const void *v, int64_t v_stride,
                             void *hip_stream) {
  CHECK(check_call(kv, ch));
  const KvTokens tk = tokens(kv, ch);
  if (!tk.max_new || !kv->rows) return SKD_OK;
  if (!kv->pool || !kv->block_table || !ch->first || !ch->past) return SKD_ERR_NULL;
  const int64_t width = (int64_t)kv->kv_heads * kv->head_dim;
  CHECK(check_rows(k, k_stride, width));
  CHECK(check_rows(v, v_stride, width));
  if (!aligned(kv->pool) || !aligned4({kv->block_table, ch->first, ch->past})) return SKD_ERR_SHAPE;
  if (!fits_int((__int128)kv->kv_heads * kv->rows * ((tk.max_new + 62LL) / 32))) return SKD_ERR_RANGE;
  CHECK(check_memory({kv->pool, kv->block_table, ch->first, ch->past, k, v}));
  kv_append((hipStream_t)hip_stream, view(kv), tk, rows_of(k, k_stride), rows_of(v, v_stride));
  return launched();
}

extern "C" int skd_kv_read(const skd_kv *kv, const skd_kv_chunk *ch, int32_t elem, void *k_out, int64_t k_stride, void *v_out,
                           int64_t v_stride, void *hip_stream) {
  CHECK(check_call(kv, ch));
  if (elem != SKD_W_FP32 && elem != SKD_W_BF16) return SKD_ERR_SHAPE;
  const KvTokens tk = tokens(kv, ch);
  if (!tk.max_new || !kv->rows) return SKD_OK;
  if (!kv->pool || !kv->block_table || !ch->first || !ch->past) return SKD_ERR_NULL;
  const int64_t width = (int64_t)kv->kv_heads * kv->head_dim;
  CHECK(check_rows(k_out, k_stride, width));
  CHECK(check_rows(v_out, v_stride, width));
  if (!aligned(kv->pool) || !aligned4({kv->block_table, ch->first, ch->past})) return SKD_ERR_SHAPE;
  if (!fits_int((__int128)kv->kv_heads * kv->rows * ((tk.max_new + 62LL) / 32))) return SKD_ERR_RANGE;
  CHECK(check_memory({kv->pool, kv->block_table, ch->first, ch->past, k_out, v_out}));
  kv_read((hipStream_t)hip_stream, view(kv), tk, elem == SKD_W_BF16, rows_of(k_out, k_stride), rows_of(v_out, v_stride));
  return launched();
}

static int check_attend(const skd_kv *kv, const skd_kv_chunk *ch, int32_t heads) {
  CHECK(check_call(kv, ch));
  if (heads < 1 || heads % kv->kv_heads) return SKD_ERR_SHAPE;
  const KvTokens tk = tokens(kv, ch);
  if (!fits_int((int64_t)heads * kv->head_dim)) return SKD_ERR_RANGE;  // columns of a token
  const int64_t group = heads / kv->kv_heads;
  const int64_t queries = tk.max_new * group;
  if (!fits_int(queries + 128) || !fits_int((int64_t)kv->kv_heads * kv->rows + 8)) return SKD_ERR_RANGE;
  return kv_attend_fits(view(kv), tk, heads) ? SKD_OK : SKD_ERR_RANGE;
}

extern "C" int64_t skd_kv_attend_workspace(const skd_kv *kv, const skd_kv_chunk *ch, int32_t heads) {
  CHECK(check_attend(kv, ch, heads));
  const KvView v = view(kv);
  const KvTokens tk = tokens(kv, ch);
  if (!tk.max_new || !kv->rows) return 0;
  return (int64_t)(kv_attend_part(v, tk, heads, kv_attend_splits(v, tk, heads)) * sizeof(float));
}

extern "C" int skd_kv_attend(const skd_kv *kv, const skd_kv_chunk *ch, int32_t heads, float scale, const void *q, int64_t q_stride,
                             const void *k, int64_t k_stride, const void *v, int64_t v_stride, void *out, int64_t out_stride,
                             void *workspace, int64_t workspace_bytes, void *hip_stream) {
  CHECK(check_attend(kv, ch, heads));
  const float c = scale * 1.4426950408889634f;
  if (!(scale > 0.f) || !std::isfinite(c)) return SKD_ERR_RANGE;
  KvAttend a{};
  a.kv = view(kv);
  a.tk = tokens(kv, ch);
  if (!a.tk.max_new || !kv->rows) return SKD_OK;
  if (!kv->pool || !kv->block_table || !ch->first || !ch->past || !k != !v) return SKD_ERR_NULL;
  const int64_t width = (int64_t)kv->kv_heads * kv->head_dim;
  CHECK(check_rows(q, q_stride, (int64_t)heads * kv->head_dim));
  CHECK(check_rows(out, out_stride, (int64_t)heads * kv->head_dim));
  if (k) {
    CHECK(check_rows(k, k_stride, width));
    CHECK(check_rows(v, v_stride, width));
  }
  if (!aligned(kv->pool) || !aligned4({kv->block_table, ch->first, ch->past})) return SKD_ERR_SHAPE;
  a.heads = heads;
  a.group = heads / kv->kv_heads;
  a.c = c;
  a.q = rows_of(q, q_stride);
  a.o = rows_of(out, out_stride);
  a.splits = kv_attend_splits(a.kv, a.tk, heads);
  if (a.splits > 1) {
    if (!workspace) return SKD_ERR_NULL;
    if (!aligned(workspace)) return SKD_ERR_SHAPE;
    if (workspace_bytes < (int64_t)(kv_attend_part(a.kv, a.tk, heads, a.splits) * sizeof(float))) return SKD_ERR_NOMEM;
    a.part = (float *)workspace;
  }
  CHECK(check_memory({kv->pool, kv->block_table, ch->first, ch->past, q, out}));
  if (k) CHECK(check_memory({k, v}));
  if (a.splits > 1) CHECK(check_memory({workspace}));
  if (k) {
    a.k = rows_of(k, k_stride);
    a.v = rows_of(v, v_stride);
  }
  kv_attend((hipStream_t)hip_stream, a);
  return launched();
}

extern "C" int64_t skd_sample_workspace(int32_t rows, int32_t vocab) {
  if (rows < 0) return SKD_ERR_RANGE;
  if (vocab < 1 || vocab > SAMPLE_ROWS_VOCAB) return SKD_ERR_SHAPE;
  if (!sample_rows_fit(rows, vocab)) return SKD_ERR_RANGE;
  return (int64_t)(sample_rows_bins(rows, vocab) * sizeof(SampleBins));
}

extern "C" int skd_sample(const float *logits, int64_t stride, int32_t rows, int32_t vocab, const skd_sampling *params, const float *u,
                          int32_t *tokens_out, void *workspace, int64_t workspace_bytes, void *hip_stream) {
  const int64_t need = skd_sample_workspace(rows, vocab);
  if (need < 0) return (int)need;
  if (stride < vocab) return SKD_ERR_SHAPE;
  if (!rows) return SKD_OK;
  if (!logits || !u || !tokens_out || !workspace) return SKD_ERR_NULL;
  if (!aligned(workspace) || !aligned4({logits, u, tokens_out})) return SKD_ERR_SHAPE;
  if (params && !aligned4({params->temperature, params->top_k, params->top_p, params->min_p})) return SKD_ERR_SHAPE;
  if (workspace_bytes < need) return SKD_ERR_NOMEM;
  SampleRows a{};
  a.bins = (SampleBins *)workspace;
  a.logits = logits;
  a.stride = (long)stride;
  a.rows = rows;
  a.vocab = vocab;
  if (params) {
    a.temperature = params->temperature;
    a.top_k = params->top_k;
    a.top_p = params->top_p;
    a.min_p = params->min_p;
  }
  a.u = u;
  a.tokens = tokens_out;
  CHECK(check_memory({logits, u, tokens_out, workspace}));
  for (const void *p : {(const void *)a.temperature, (const void *)a.top_k, (const void *)a.top_p, (const void *)a.min_p})
    if (p) CHECK(check_memory({p}));
  sample_rows((hipStream_t)hip_stream, a);
  return launched();
}
