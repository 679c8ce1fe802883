// C entry points of the decoding-stage operators: argument checks and launches.
#include <algorithm>
#include <atomic>
#include <cstdarg>
#include <cstdio>
#include <new>

#include "wf_decoder.h"
#include "wf_ptx.cuh"

using namespace wf;

struct wf_decoder {
  wf_decoder_config cfg;
  bool no_waits;  // wf_selftest_attention_timeout
  char err[512];
};

namespace {

wf_status fail(wf_decoder* d, wf_status st, const char* fmt, ...) {
  va_list ap;
  va_start(ap, fmt);
  vsnprintf(d->err, sizeof(d->err), fmt, ap);
  va_end(ap);
  return st;
}

bool aligned16(const void* p) { return ((uintptr_t)p & 15) == 0; }

int path_bytes(const wf_decoder_config& c) { return c.dtype == WF_BF16 ? 2 : 4; }
int code_bytes(const wf_decoder_config& c) { return c.cache_format == WF_CACHE_PATH ? path_bytes(c) : 1; }
int log2_of(int v) {
  int s = 0;
  while ((1 << s) < v) ++s;
  return s;
}

wf_status cuda_result(wf_decoder* d, const char* what, cudaError_t e) {
  if (e == cudaSuccess) return WF_OK;
  return fail(d, WF_ERR_CUDA, "%s: %s", what, cudaGetErrorString(e));
}

// The checks that every cache operator makes.
wf_status check_cache(wf_decoder* d, const char* what, const wf_cache* c) {
  if (!c || !c->k || !c->v || c->n_pages < 1) return fail(d, WF_ERR_INVALID_ARG, "%s: NULL cache or no pages", what);
  if ((long)c->n_pages * d->cfg.n_kv_head * d->cfg.page_size >= (1L << 32) - 1)
    return fail(d, WF_ERR_CAPACITY, "%s: more than 2^32 vectors in a cache", what);
  if (!aligned16(c->k) || !aligned16(c->v)) return fail(d, WF_ERR_INVALID_ARG, "%s: cache pages must be 16-byte aligned", what);
  if (d->cfg.cache_format != WF_CACHE_PATH) {
    if (!c->k_scale || !c->v_scale) return fail(d, WF_ERR_INVALID_ARG, "%s: a quantised cache needs scales", what);
    if (!aligned16(c->k_scale) || !aligned16(c->v_scale))
      return fail(d, WF_ERR_INVALID_ARG, "%s: scales must be 16-byte aligned", what);
  }
  return WF_OK;
}

wf_status check_rows(wf_decoder* d, const char* what, const wf_rows* r) {
  if (!r || r->n_seq < 0 || r->n_rows < 0) return fail(d, WF_ERR_INVALID_ARG, "%s: NULL rows or a negative size", what);
  if (r->n_seq == 0 || r->n_rows == 0) return WF_OK;
  if (!r->cu_rows || !r->start || !r->page_table || r->table_stride < 1)
    return fail(d, WF_ERR_INVALID_ARG, "%s: NULL prefix sums, starts or page table", what);
  if (r->n_rows > (1 << 27)) return fail(d, WF_ERR_CAPACITY, "%s: more than 2^27 rows", what);
  return WF_OK;
}

CacheView view_of(const wf_decoder* d, const wf_cache* c) {
  const bool q = d->cfg.cache_format != WF_CACHE_PATH;
  return CacheView{c->k, c->v, q ? (__nv_bfloat16*)c->k_scale : nullptr, q ? (__nv_bfloat16*)c->v_scale : nullptr, c->n_pages,
                   d->cfg.n_kv_head, log2_of(d->cfg.page_size)};
}
RowsView view_of(const wf_rows* r) { return RowsView{r->n_seq, r->n_rows, r->cu_rows, r->start, r->page_table, r->table_stride}; }

wf_status check_vectors(wf_decoder* d, const char* what, const wf_rows* r, const void* k, long k_stride, const void* v, long v_stride) {
  const int esz = path_bytes(d->cfg);
  const long row = (long)d->cfg.n_kv_head * d->cfg.d_head;
  if ((long)r->n_rows * d->cfg.n_kv_head >= (1L << 32) - 1)  // as in check_cache; a launch's blocks fit its grid then
    return fail(d, WF_ERR_CAPACITY, "%s: more than 2^32 vectors in a call", what);
  if (!k || !v) return fail(d, WF_ERR_INVALID_ARG, "%s: NULL keys or values", what);
  if (!aligned16(k) || !aligned16(v) || k_stride * esz % 16 || v_stride * esz % 16)
    return fail(d, WF_ERR_INVALID_ARG, "%s: keys and values need 16-byte aligned pointers and row strides", what);
  if (k_stride < row || v_stride < row)
    return fail(d, WF_ERR_INVALID_ARG, "%s: a row stride is shorter than a row of %ld elements", what, row);
  return WF_OK;
}

// Whether two states of n rows certainly share bytes: the first row of one begins inside a row of the other, or (strides alike) a
// row's end reaches into one.
bool share_bytes(const wf_beam_state& a, const wf_beam_state& b, long n) {
  if (a.row_bytes == 0 || b.row_bytes == 0) return false;
  const uintptr_t a0 = (uintptr_t)a.ptr, b0 = (uintptr_t)b.ptr;
  if (a0 >= b0 + (n - 1) * b.stride_bytes + b.row_bytes || b0 >= a0 + (n - 1) * a.stride_bytes + a.row_bytes) return false;
  if (a0 >= b0 && (long)((a0 - b0) % b.stride_bytes) < b.row_bytes) return true;
  if (b0 >= a0 && (long)((b0 - a0) % a.stride_bytes) < a.row_bytes) return true;
  // the extents meet and neither begins inside a row: with one stride, one begins in a gap of the other that it overruns or fits
  if (a.stride_bytes != b.stride_bytes) return false;
  return a0 > b0 ? b.stride_bytes - (long)((a0 - b0) % b.stride_bytes) < a.row_bytes : a.stride_bytes - (long)((b0 - a0) % a.stride_bytes) < b.row_bytes;
}

}  // namespace

extern "C" {

wf_status wf_decoder_create(const wf_decoder_config* cfg, wf_decoder** out) {
  if (!cfg || !out) return WF_ERR_INVALID_ARG;
  *out = nullptr;
  wf_decoder* d = new (std::nothrow) wf_decoder();
  if (!d) return WF_ERR_INVALID_ARG;
  d->cfg = *cfg;
  d->no_waits = false;
  d->err[0] = 0;
  *out = d;  // returned even on failure so that the caller can read the message, then destroy
  const wf_decoder_config& c = d->cfg;
  if (c.n_head < 1 || c.n_head > 1024 || c.n_kv_head < 1 || c.n_head % c.n_kv_head)
    return fail(d, WF_ERR_INVALID_ARG, "n_kv_head must divide n_head (1 .. 1024)");
  if (c.d_head != 64 && c.d_head != 128) return fail(d, WF_ERR_INVALID_ARG, "d_head must be 64 or 128");
  if (c.dtype != WF_F32 && c.dtype != WF_BF16) return fail(d, WF_ERR_INVALID_ARG, "unknown dtype");
  if (c.cache_format < WF_CACHE_PATH || c.cache_format > WF_CACHE_INT8)
    return fail(d, WF_ERR_INVALID_ARG, "unknown cache format");
  if (c.page_size < 16 || c.page_size > 256 || (c.page_size & (c.page_size - 1)))
    return fail(d, WF_ERR_INVALID_ARG, "page_size must be a power of two from 16 to 256");
  return WF_OK;
}

wf_status wf_decoder_destroy(wf_decoder* d) {
  delete d;
  return WF_OK;
}

const char* wf_decoder_last_error(const wf_decoder* d) { return d ? d->err : "null decoder"; }

wf_status wf_cache_write(wf_decoder* d, const wf_cache* cache, const wf_rows* rows, const void* k, long k_stride, const void* v,
                         long v_stride, int* status, void* stream) {
  if (!d) return WF_ERR_INVALID_ARG;
  wf_status st = check_rows(d, "wf_cache_write", rows);
  if (st != WF_OK) return st;
  st = check_cache(d, "wf_cache_write", cache);
  if (st != WF_OK) return st;
  if (rows->n_seq == 0 || rows->n_rows == 0) return WF_OK;
  st = check_vectors(d, "wf_cache_write", rows, k, k_stride, v, v_stride);
  if (st != WF_OK) return st;
  return cuda_result(d, "wf_cache_write",
                     launch_cache_write(view_of(d, cache), view_of(rows), d->cfg.d_head, d->cfg.dtype, d->cfg.cache_format, k, k_stride,
                                        v, v_stride, status, (cudaStream_t)stream));
}

wf_status wf_cache_read(wf_decoder* d, const wf_cache* cache, const wf_rows* rows, void* k, long k_stride, void* v, long v_stride,
                        int* status, void* stream) {
  if (!d) return WF_ERR_INVALID_ARG;
  wf_status st = check_rows(d, "wf_cache_read", rows);
  if (st != WF_OK) return st;
  st = check_cache(d, "wf_cache_read", cache);
  if (st != WF_OK) return st;
  if (rows->n_seq == 0 || rows->n_rows == 0) return WF_OK;
  st = check_vectors(d, "wf_cache_read", rows, k, k_stride, v, v_stride);
  if (st != WF_OK) return st;
  return cuda_result(d, "wf_cache_read",
                     launch_cache_read(view_of(d, cache), view_of(rows), d->cfg.d_head, d->cfg.dtype, d->cfg.cache_format, k, k_stride, v,
                                       v_stride, status, (cudaStream_t)stream));
}

namespace {
// Number of SMs of the current device (asked once per device; the same for every thread that asks).
wf_status sm_count(wf_decoder* d, int* n) {
  static std::atomic<int> known[64];
  int dev = 0;
  cudaError_t e = cudaGetDevice(&dev);
  if (e == cudaSuccess && dev < 64 && (*n = known[dev].load(std::memory_order_relaxed)) > 0) return WF_OK;
  if (e == cudaSuccess) e = cudaDeviceGetAttribute(n, cudaDevAttrMultiProcessorCount, dev);
  if (e != cudaSuccess) return cuda_result(d, "device query", e);
  if (dev < 64) known[dev].store(*n, std::memory_order_relaxed);
  return WF_OK;
}
wf_status check_attention_sizes(wf_decoder* d, int n_seq, int n_rows, int max_rows, int max_len) {
  if (n_seq < 0 || n_rows < 0 || max_rows < 0 || max_len < 0)
    return fail(d, WF_ERR_INVALID_ARG, "wf_tree_attention: a negative size");
  if (n_seq > 65535) return fail(d, WF_ERR_CAPACITY, "wf_tree_attention: more than 65535 sequences");
  if (max_len > (1 << 30)) return fail(d, WF_ERR_CAPACITY, "wf_tree_attention: max_len above 2^30");
  if (n_rows > (1 << 27) || max_rows > (1 << 16)) return fail(d, WF_ERR_CAPACITY, "wf_tree_attention: more than 2^27 rows, or 2^16 in a sequence");
  return WF_OK;
}
}  // namespace

wf_status wf_tree_attention_workspace(wf_decoder* d, int n_seq, int n_rows, int max_rows, int max_len, size_t* bytes) {
  if (!d) return WF_ERR_INVALID_ARG;
  if (!bytes) return fail(d, WF_ERR_INVALID_ARG, "wf_tree_attention_workspace: NULL argument");
  *bytes = 0;
  wf_status st = check_attention_sizes(d, n_seq, n_rows, max_rows, max_len);
  if (st != WF_OK || n_seq == 0 || n_rows == 0 || max_rows == 0) return st;
  int sms = 0;
  st = sm_count(d, &sms);
  if (st != WF_OK) return st;
  const wf_decoder_config& c = d->cfg;
  *bytes = plan_tree_attention(c.dtype, c.d_head, c.n_head, c.n_kv_head, n_seq, n_rows, max_rows, max_len, sms).bytes;
  return WF_OK;
}

wf_status wf_tree_attention(wf_decoder* d, const wf_cache* cache, const wf_rows* rows, const void* q, long q_stride, float scale,
                            int tail, const unsigned* mask, int mask_words, int max_rows, int max_len, void* out, long out_stride,
                            float* lse, void* workspace, size_t workspace_bytes, int* status, void* stream) {
  if (!d) return WF_ERR_INVALID_ARG;
  wf_status st = check_rows(d, "wf_tree_attention", rows);
  if (st != WF_OK) return st;
  st = check_cache(d, "wf_tree_attention", cache);
  if (st != WF_OK) return st;
  st = check_attention_sizes(d, rows->n_seq, rows->n_rows, max_rows, max_len);
  if (st != WF_OK) return st;
  if (tail < WF_TAIL_NONE || tail > WF_TAIL_MASK) return fail(d, WF_ERR_INVALID_ARG, "wf_tree_attention: unknown tail %d", tail);
  if (tail == WF_TAIL_MASK && (mask_words < 0 || (long)mask_words * 32 < max_rows || (max_rows > 0 && !mask)))
    return fail(d, WF_ERR_INVALID_ARG, "wf_tree_attention: WF_TAIL_MASK needs a mask of at least max_rows bits per row");
  if (!(scale == scale) || scale - scale != 0.f) return fail(d, WF_ERR_INVALID_ARG, "wf_tree_attention: scale must be finite");
  if (rows->n_seq == 0 || rows->n_rows == 0 || max_rows == 0) return WF_OK;
  const wf_decoder_config& c = d->cfg;
  if ((long)max_len > (long)rows->table_stride * c.page_size)
    return fail(d, WF_ERR_INVALID_ARG, "wf_tree_attention: max_len %d exceeds the page table (%d pages of %d)", max_len,
                rows->table_stride, c.page_size);
  const int esz = path_bytes(c);
  const long row = (long)c.n_head * c.d_head;
  if (!q || !out) return fail(d, WF_ERR_INVALID_ARG, "wf_tree_attention: NULL queries or output");
  if (!aligned16(q) || !aligned16(out) || q_stride * esz % 16 || out_stride * esz % 16 || q_stride < row || out_stride < row)
    return fail(d, WF_ERR_INVALID_ARG, "wf_tree_attention: queries and outputs need 16-byte aligned pointers and row strides of at least %ld elements", row);
  int sms = 0;
  st = sm_count(d, &sms);
  if (st != WF_OK) return st;
  const TreeAttnPlan plan = plan_tree_attention(c.dtype, c.d_head, c.n_head, c.n_kv_head, rows->n_seq, rows->n_rows, max_rows, max_len, sms);
  if (plan.bytes > 0 && (!workspace || workspace_bytes < plan.bytes || !aligned16(workspace)))
    return fail(d, WF_ERR_INVALID_ARG, "wf_tree_attention: needs %zu bytes of 16-byte aligned workspace, got %zu", plan.bytes, workspace_bytes);
  TreeAttnParams p{};
  p.cache = view_of(d, cache);
  p.rows = view_of(rows);
  p.q = q;
  p.out = out;
  p.q_stride = q_stride;
  p.out_stride = out_stride;
  p.lse = lse;
  p.mask = mask;
  p.mask_words = mask_words;
  p.tail = tail;
  p.max_rows = max_rows;
  p.max_len = max_len;
  p.n_head = c.n_head;
  p.group = c.n_head / c.n_kv_head;
  p.scale = scale;
  p.n_splits = plan.n_splits;
  p.chunk = plan.chunk;
  p.unit_warps = plan.unit_warps;
  p.part_o = (float*)workspace;
  p.part_ml = plan.bytes ? (float2*)((float*)workspace + (size_t)rows->n_rows * c.n_head * plan.n_splits * c.d_head) : nullptr;
  p.status = status;
  p.wait_limit = d->no_waits ? 0 : ptx::kWaitLimit;
  return cuda_result(d, "wf_tree_attention", launch_tree_attention(p, c.d_head, c.dtype, c.cache_format, (cudaStream_t)stream));
}

wf_status wf_selftest_attention_timeout(wf_decoder* d, int on) {
  if (!d) return WF_ERR_INVALID_ARG;
  d->no_waits = on != 0;
  return WF_OK;
}

wf_status wf_beam_select(wf_decoder* d, const void* logits, int logits_dtype, long ld, int B, int n_beam, int vocab, const float* scores,
                         const int* beams, const unsigned char* finished, int end_token, const unsigned* suppress, int keep,
                         float* out_scores, int* out_parents, int* out_tokens, unsigned char* out_finished, int* status, void* stream) {
  if (!d) return WF_ERR_INVALID_ARG;
  if (B < 0 || n_beam < 1 || n_beam > kMaxBeams || keep < 1 || keep > kMaxKeep || vocab < 1 || (long)vocab * n_beam >= (1L << 31))
    return fail(d, WF_ERR_INVALID_ARG, "wf_beam_select: needs 1 .. %d beams, 1 .. %d to keep and a vocabulary below 2^31 / n_beam", kMaxBeams, kMaxKeep);
  if (B > (1 << 24) || vocab > (1 << 28)) return fail(d, WF_ERR_CAPACITY, "wf_beam_select: more than 2^24 sequences or 2^28 tokens");
  const int esz = logits_dtype == WF_BF16 ? 2 : 4;
  if ((logits_dtype != WF_F32 && logits_dtype != WF_BF16) || ld < vocab)
    return fail(d, WF_ERR_INVALID_ARG, "wf_beam_select: unknown logits type, or rows shorter than the vocabulary");
  if (end_token < -1 || end_token >= vocab || (finished && end_token < 0))
    return fail(d, WF_ERR_INVALID_ARG, "wf_beam_select: end_token %d outside the vocabulary (finished beams need one)", end_token);
  if (B == 0) return WF_OK;
  if (!logits || !scores || !out_scores || !out_parents || !out_tokens) return fail(d, WF_ERR_INVALID_ARG, "wf_beam_select: NULL argument");
  if ((uintptr_t)logits % esz) return fail(d, WF_ERR_INVALID_ARG, "wf_beam_select: logits are not aligned to their type");
  int sms = 0;
  const wf_status st = sm_count(d, &sms);
  if (st != WF_OK) return st;
  BeamSelectParams p{};
  p.logits = logits;
  p.ld = ld;
  p.n_beam = n_beam;
  p.vocab = vocab;
  p.keep = keep;
  p.scores = scores;
  p.beams = beams;
  p.finished = finished;
  p.end_token = end_token;
  p.suppress = suppress;
  p.out_scores = out_scores;
  p.out_parents = out_parents;
  p.out_tokens = out_tokens;
  p.out_finished = out_finished;
  p.status = status;
  return cuda_result(d, "wf_beam_select", launch_beam_select(p, B, logits_dtype, sms, (cudaStream_t)stream));
}

wf_status wf_beam_reorder(wf_decoder* d, const int* parents, int B, int n_beam, const wf_beam_state* states, int n_states,
                          const wf_cache* caches, int n_caches, int* page_table, int table_stride, const int* lengths, int* status,
                          void* stream) {
  if (!d) return WF_ERR_INVALID_ARG;
  if (B < 0 || n_beam < 1 || n_beam > kMaxBeams || n_states < 0 || n_caches < 0)
    return fail(d, WF_ERR_INVALID_ARG, "wf_beam_reorder: a negative size, or n_beam outside 1 .. %d", kMaxBeams);
  if (B > 65535) return fail(d, WF_ERR_CAPACITY, "wf_beam_reorder: more than 65535 sequences");
  if ((n_states > 0 && !states) || (n_caches > 0 && (!caches || !page_table || !lengths || table_stride < 1)) || (B > 0 && !parents))
    return fail(d, WF_ERR_INVALID_ARG, "wf_beam_reorder: NULL argument");
  for (int i = 0; i < n_states; ++i) {
    const wf_beam_state& x = states[i];
    if (x.row_bytes < 0 || x.stride_bytes < x.row_bytes || (x.row_bytes > 0 && !x.ptr))
      return fail(d, WF_ERR_INVALID_ARG, "wf_beam_reorder: state %d has %ld bytes every %ld", i, x.row_bytes, x.stride_bytes);
    if (x.row_bytes > (1L << 36)) return fail(d, WF_ERR_CAPACITY, "wf_beam_reorder: a row of more than 2^36 bytes");
  }
  for (int i = 0; i < n_caches; ++i) {
    const wf_status st = check_cache(d, "wf_beam_reorder", caches + i);
    if (st != WF_OK) return st;
    if (caches[i].n_pages != caches[0].n_pages)
      return fail(d, WF_ERR_INVALID_ARG, "wf_beam_reorder: caches that share a page table have the same number of pages");
  }
  if (B == 0 || n_beam == 1) return WF_OK;  // one beam can only have grown from itself
  // What a call is given twice would be moved twice, in any order.  (A table of pages is a state of its own here.)
  const wf_beam_state table_state{page_table, n_caches > 0 ? (long)table_stride * 4 : 0, (long)table_stride * 4};
  for (int i = 0; i < n_states; ++i) {
    for (int j = 0; j < i; ++j)
      if (share_bytes(states[i], states[j], (long)B * n_beam))
        return fail(d, WF_ERR_INVALID_ARG, "wf_beam_reorder: states %d and %d share memory", j, i);
    if (share_bytes(states[i], table_state, (long)B * n_beam))
      return fail(d, WF_ERR_INVALID_ARG, "wf_beam_reorder: state %d and the page table share memory", i);
  }
  const bool scaled = d->cfg.cache_format != WF_CACHE_PATH;
  for (int i = 0; i < n_caches; ++i)
    for (int j = 0; j <= i; ++j) {
      const wf_cache &x = caches[i], &y = caches[j];
      const bool pages = x.k == y.v || (i != j && (x.k == y.k || x.v == y.k || x.v == y.v));
      const bool scales = scaled && (x.k_scale == y.v_scale || (i != j && (x.k_scale == y.k_scale || x.v_scale == y.k_scale || x.v_scale == y.v_scale)));
      if (pages || scales) return fail(d, WF_ERR_INVALID_ARG, "wf_beam_reorder: caches %d and %d (or the sides of one) share memory", j, i);
    }
  const wf_decoder_config& c = d->cfg;
  ReorderPlan p{};
  p.parents = parents;
  p.n_beam = n_beam;
  p.page_table = page_table;
  p.table_stride = table_stride;
  p.lengths = lengths;
  p.page_shift = log2_of(c.page_size);
  p.head_units = c.page_size * c.d_head * code_bytes(c) / 16;
  p.n_kv_head = c.n_kv_head;
  p.n_pages = n_caches > 0 ? caches[0].n_pages : 0;
  p.status = status;
  long blocks = 0;
  cudaError_t e = cudaSuccess;
  auto flush = [&]() {
    if (p.n_items > 0 && e == cudaSuccess) e = launch_beam_reorder(p, B, (int)blocks, (cudaStream_t)stream);
    p.n_items = 0;
    blocks = 0;
  };
  auto add = [&](ReorderItem it, long threads) {
    const long need = (threads + kReorderThreads - 1) / kReorderThreads;
    if (need == 0) return;
    if (p.n_items == kReorderItems || blocks + need > (1L << 30)) flush();
    it.first_block = (int)blocks;
    p.item[p.n_items++] = it;
    blocks += need;
  };
  for (int i = 0; i < n_caches; ++i)
    for (int side = 0; side < 2; ++side) {
      ReorderItem it{};
      it.kind = 1;
      it.ptr = (char*)(side == 0 ? caches[i].k : caches[i].v);
      it.scale = c.cache_format == WF_CACHE_PATH ? nullptr : (__nv_bfloat16*)(side == 0 ? caches[i].k_scale : caches[i].v_scale);
      it.units = (long)p.head_units * c.n_kv_head;
      it.stride = it.units * 16;
      add(it, it.units + (it.scale ? (long)c.n_kv_head * c.page_size : 0));
    }
  if (n_caches > 0) {
    ReorderItem it{};
    it.kind = 2;
    it.units = table_stride;
    add(it, table_stride);
  }
  for (int i = 0; i < n_states; ++i) {
    ReorderItem it{};
    const uintptr_t bits = (uintptr_t)states[i].ptr | (uintptr_t)states[i].row_bytes | (uintptr_t)states[i].stride_bytes;
    it.kind = 0;
    it.ptr = (char*)states[i].ptr;
    it.stride = states[i].stride_bytes;
    it.unit = bits % 16 == 0 ? 16 : bits % 4 == 0 ? 4 : 1;
    it.units = states[i].row_bytes / it.unit;
    add(it, it.units);
  }
  flush();
  return cuda_result(d, "wf_beam_reorder", e);
}

}  // extern "C"
