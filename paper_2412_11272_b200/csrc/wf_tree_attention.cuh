// Device helpers shared by the attention kernels over the paged cache.
#pragma once

#include "wf_decoder.h"

namespace wf {

// What a block needs to know about its sequence.
struct Sequence {
  int first_row, n_rows;  // rows of the batch
  int start;              // committed positions
  int len;                // positions to look at, the rows' own included
};

// The same for every thread of the block.
__device__ __forceinline__ Sequence load_sequence(const TreeAttnParams& p, int seq, bool reporter) {
  Sequence s;
  s.first_row = __ldg(p.rows.cu_rows + seq);
  s.n_rows = __ldg(p.rows.cu_rows + seq + 1) - s.first_row;
  s.start = __ldg(p.rows.start + seq);
  bool bad = s.first_row < 0 || s.n_rows < 0 || (long)s.first_row + s.n_rows > p.rows.n_rows || s.start < 0;
  if (bad) s.n_rows = 0, s.start = 0;
  long len = (long)s.start + (p.tail == WF_TAIL_NONE ? 0 : s.n_rows);
  if (s.n_rows > 0 && len > p.max_len) {
    bad = true;
    len = p.max_len;
  }
  if (s.n_rows > p.max_rows) bad = true;
  s.len = (int)len;
  if (bad && reporter) report(p.status, kBadRows);
  return s;
}

// Whether batch row i of the sequence sees position start + t (t >= 0).
__device__ __forceinline__ bool sees_tail(const TreeAttnParams& p, const Sequence& s, int i, int t) {
  if (p.tail == WF_TAIL_CAUSAL) return t <= i;
  const int w = t >> 5;
  if (w >= p.mask_words) return false;
  return (__ldg(p.mask + (long)(s.first_row + i) * p.mask_words + w) >> (t & 31)) & 1;
}

__device__ __forceinline__ int page_of(const TreeAttnParams& p, int seq, int pos) {
  const int page = __ldg(p.rows.page_table + (long)seq * p.rows.table_stride + (pos >> p.cache.page_shift));
  if (page < 0 || page >= p.cache.n_pages) {
    report(p.status, kBadPage);
    return -1;
  }
  return page;
}

// bfloat16 path: tiles of few query rows (wf_tree_attention_tc.cu; rows_tile is 8, 16 or 32) and of 128 (wf_tree_attention_wide.cu).
cudaError_t launch_tree_attention_tc(const TreeAttnParams& p, int d_head, int format, int rows_tile, cudaStream_t s);
cudaError_t launch_tree_attention_wide(const TreeAttnParams& p, int d_head, int format, cudaStream_t s);

}  // namespace wf
