// Internal declarations of the decoding-stage operators (not part of the ABI).
#pragma once

#include <cuda_bf16.h>
#include <cuda_fp16.h>
#include <cuda_fp8.h>
#include <cuda_runtime.h>
#include <stdint.h>

#include "wf_internal.h"

namespace wf {

// Bits of the caller's status word.
enum DeviceStatus : int { kBadPage = 1, kBadRows = 2, kBadParent = 4, kGaveUp = 8, kPutOff = 16, kBadValue = 32 };

constexpr int kMaxBeams = 16;

// One layer's cache as the kernels see it.
struct CacheView {
  void *k, *v;
  __nv_bfloat16 *k_scale, *v_scale;
  int n_pages;
  int n_kv_head;
  int page_shift;  // log2 of the page size
};

struct RowsView {
  int n_seq, n_rows;
  const int *cu_rows, *start, *page_table;
  int table_stride;
};

__device__ __forceinline__ void report(int* status, int bit) {
  if (status) atomicOr(status, bit);
}

// Sequence that can have a row: the largest s with cu[s] <= row, searched by a whole warp 32 entries at a time (two
// dependent loads for up to 1024 sequences).  All lanes ask for one row.  Always one of 0 .. n_seq - 1: whether the row lies
// within it is the caller's to check (rows in front of the first sequence, rows behind the last one, sums that decrease).
__device__ __forceinline__ int warp_find_sequence(const int* __restrict__ cu, int n_seq, int row) {
  const int lane = threadIdx.x & 31;
  int lo = 0, n = n_seq;  // the answer lies in [lo, lo + n)
  while (n > 1) {
    const int step = (n + 31) / 32;
    const int at = lo + lane * step;
    const unsigned le = __ballot_sync(0xffffffffu, lane * step < n && __ldg(cu + at) <= row);
    const int last = le ? 31 - __clz(le) : 0;
    const int next = lo + last * step;
    n = min(step, lo + n - next);
    lo = next;
  }
  return lo;
}

// ---- launchers
cudaError_t launch_cache_write(const CacheView& c, const RowsView& r, int d_head, int dtype, int format, const void* k,
                               long k_stride, const void* v, long v_stride, int* status, cudaStream_t s);
cudaError_t launch_cache_read(const CacheView& c, const RowsView& r, int d_head, int dtype, int format, void* k,
                              long k_stride, void* v, long v_stride, int* status, cudaStream_t s);

// ---- attention over the paged cache (wf_tree_attention.cu)
struct TreeAttnParams {
  CacheView cache;
  RowsView rows;
  const void* q;
  void* out;
  long q_stride, out_stride;  // elements
  float* lse;
  const unsigned* mask;
  int mask_words, tail;
  int max_rows, max_len;
  int n_head, group;  // group = n_head / n_kv_head
  float scale;
  // split of the positions: split i of a sequence has [i chunk, (i + 1) chunk); with more than one split the
  // unnormalised sums go to part_o [n_rows][n_head][n_splits][d_head] and (maximum, sum) to part_ml
  int n_splits, chunk;
  int unit_warps;  // warps that share a tile of few rows (1, 2 or 4); 0: the kernel for many rows
  float* part_o;
  float2* part_ml;
  int* status;
  unsigned wait_limit;  // polls of a wait of the 128-row kernel; 0: every wait gives up at once
};
struct TreeAttnPlan {
  int n_splits, chunk, unit_warps;
  size_t bytes;
};
TreeAttnPlan plan_tree_attention(int dtype, int d_head, int n_head, int n_kv_head, int n_seq, int n_rows, int max_rows, int max_len,
                                 int num_sms);
cudaError_t launch_tree_attention(const TreeAttnParams& p, int d_head, int dtype, int format, cudaStream_t s);

// ---- beam selection (wf_beam_search.cu)
constexpr int kMaxKeep = 32;
struct BeamSelectParams {
  const void* logits;
  long ld;
  int n_beam, vocab, keep;
  const float* scores;
  const int* beams;
  const unsigned char* finished;
  int end_token;
  const unsigned* suppress;
  float* out_scores;
  int *out_parents, *out_tokens;
  unsigned char* out_finished;
  int* status;
  int slice;   // elements of a row per block of the cluster (a multiple of 8)
  int groups;  // items that a block makes of its slice of a row
  int tiles;   // tiles of an item
};
cudaError_t launch_beam_select(BeamSelectParams p, int B, int dtype, int num_sms, cudaStream_t s);

// An item of the reorder kernel: a contiguous state, one side (keys or values) of a paged cache, or the
// page table itself.
struct ReorderItem {
  char* ptr;
  __nv_bfloat16* scale;  // paged, quantised: the side's scales
  long stride;           // state: bytes between rows; paged: bytes of a page
  long units;            // state: units of `unit` bytes in a row; paged: 16-byte units of a page, all heads
  int kind;              // 0 state, 1 paged, 2 page table
  int unit;              // state: 16, 4 or 1 bytes
  int first_block;
};
constexpr int kReorderItems = 64;
struct ReorderPlan {
  ReorderItem item[kReorderItems];
  int n_items;
  const int* parents;
  int n_beam;
  int* page_table;
  int table_stride;
  const int* lengths;
  int page_shift;
  int head_units;  // paged: 16-byte units of one head of a page
  int n_kv_head;
  int n_pages;
  int* status;
};
constexpr int kReorderThreads = 256;
cudaError_t launch_beam_reorder(const ReorderPlan& p, int B, int n_blocks, cudaStream_t s);

// ---- rows and pages of a round (wf_page_plan.cu)
constexpr int kMaxPlanned = 8192;  // sequences: five integers each in shared memory
struct PagePlanParams {
  int *ring, *pool;
  int n_pages, page_shift;
  int n_seq, n_rows;
  const int* new_rows;
  const unsigned char* ended;
  int *lengths, *held, *table;
  int table_stride;
  int *cu_rows, *row_seq, *row_pos;
  long long* row_slot;
  int* status;
};
cudaError_t launch_page_plan(const PagePlanParams& p, cudaStream_t s);

// ---- verification and commit of drafted tokens (wf_draft.cu)
constexpr int kMaxDrafts = 1024;  // rows of a sequence
struct DraftVerifyParams {
  const void* logits;
  long ld;
  int vocab, n_seq, n_rows, max_rows;
  const int *cu_rows, *tokens, *parents;
  const float* draft;
  long draft_ld;
  const float *temperature, *accept_u, *sample_u;
  int *kept, *out_tokens, *path;
  int* status;
};
cudaError_t launch_draft_verify(const DraftVerifyParams& p, int dtype, int num_sms, cudaStream_t s);

// One side (keys or values) of a layer's cache.
struct CommitItem {
  char* ptr;
  __nv_bfloat16* scale;  // NULL: not quantised
};
constexpr int kCommitItems = 128;
struct CommitPlan {
  CommitItem item[kCommitItems];
  int n_items;
  int n_seq;
  const int *start, *kept, *path;
  int path_stride;
  int* lengths;  // NULL: not this launch
  const int* page_table;
  int table_stride, page_shift, n_pages, n_kv_head;
  int vec_units;  // 16-byte units of a vector
  int* status;
};
cudaError_t launch_draft_commit(const CommitPlan& p, cudaStream_t s);
cudaError_t launch_draft_lengths(const CommitPlan& p, cudaStream_t s);

// ---- products with 8-bit codes (wf_gemm_e4m3.cu)
constexpr int kScaleBlock = 128;  // channels of a row that share a scale
struct E4m3Operand {
  const void* codes;
  const uint32_t* scales;  // words of four blocks' bytes: [ceil(k / 512)][scale_ld], a word for each row
  long ld, scale_ld;       // bytes between rows of codes; words between groups of blocks
};
cudaError_t launch_quantise_e4m3(const void* x, int dtype, long ldx, long rows, int k, void* codes, long ld_codes, unsigned char* scales,
                                 long ld_scales, cudaStream_t s);
struct E4m3GemmParams {
  E4m3Operand a, w;  // [m, k], [n, k]
  int m, n, k;
  const float* bias;
  int gelu;
  void* out;
  int out_dtype;
  long ldc;
  int* status;
  unsigned wait_limit;
  int hasty_warp;  // a warp that gives up at its first wait (-1: none)
};
cudaError_t launch_gemm_e4m3(const E4m3GemmParams& p, int num_sms, cudaStream_t s);

}  // namespace wf
