// Device side of beam search: reordering of the beams' states.
//
// In place without a second buffer: a thread owns one unit (16 bytes where alignment allows) of a
// column, loads that unit of every parent that some other beam grew from, and stores only then.  Units of
// different threads do not meet, so no thread sees a half-moved state.  Bound by memory: a row that
// moves is written once and its parent read once (several children of one parent hit L1 / L2).
// Rows that stay (parent = itself) cost nothing.
#include "wf_decoder.h"

namespace wf {

namespace {

// Parents of one sequence's beams, in shared memory; out-of-range ones stay in place.
__device__ __forceinline__ void load_parents(const ReorderPlan& p, int b, int* parent, bool* any) {
  if (threadIdx.x < (unsigned)p.n_beam) {
    const int w = threadIdx.x;
    int q = __ldg(p.parents + (long)b * p.n_beam + w);
    if (q >= p.n_beam) {
      report(p.status, kBadParent);
      q = w;
    }
    if (q < 0) q = w;
    parent[w] = q;
    if (q != w) *any = true;
  }
}

// new[w] = old[parent[w]] for one unit of every beam; `at(w)` is its address in beam w's row (null: absent).
template <int kBeams, typename U, typename At>
__device__ __forceinline__ void move_unit(const int* parent, int n_beam, At at) {
  U u[kBeams];
  bool moves[kBeams];
#pragma unroll
  for (int w = 0; w < kBeams; ++w) {
    moves[w] = false;
    if (w < n_beam && parent[w] != w) {
      const U* src = reinterpret_cast<const U*>(at(parent[w]));
      moves[w] = src != nullptr && at(w) != nullptr;
      if (moves[w]) u[w] = *src;
    }
  }
#pragma unroll
  for (int w = 0; w < kBeams; ++w)
    if (moves[w]) *reinterpret_cast<U*>(at(w)) = u[w];
}

template <int kBeams>
__global__ void __launch_bounds__(kReorderThreads) beam_reorder_kernel(const __grid_constant__ ReorderPlan p) {
  __shared__ int parent[kMaxBeams];
  __shared__ int page_of[kMaxBeams];
  __shared__ bool any;
  const int b = blockIdx.y;
  if (threadIdx.x == 0) any = false;
  __syncthreads();
  load_parents(p, b, parent, &any);
  int i = 0;
  while (i + 1 < p.n_items && p.item[i + 1].first_block <= (int)blockIdx.x) ++i;
  const ReorderItem& it = p.item[i];
  const long unit = (long)((int)blockIdx.x - it.first_block) * kReorderThreads + threadIdx.x;
  const long row0 = (long)b * p.n_beam;

  int length = 0;
  if (it.kind != 0) {
    length = __ldg(p.lengths + b);
    if (length < 0 || (length >> p.page_shift) > p.table_stride ||
        ((length & ((1 << p.page_shift) - 1)) != 0 && (length >> p.page_shift) >= p.table_stride)) {
      if (threadIdx.x == 0) report(p.status, kBadRows);
      length = 0;
    }
  }
  const int full = length >> p.page_shift;  // pages that are full
  const int rest = length & ((1 << p.page_shift) - 1);
  if (it.kind == 1 && threadIdx.x < (unsigned)p.n_beam) {
    int page = -1;
    if (rest != 0) {
      page = __ldg(p.page_table + (row0 + threadIdx.x) * p.table_stride + full);
      if (page < 0 || page >= p.n_pages) {
        report(p.status, kBadPage);
        page = -1;
      }
    }
    page_of[threadIdx.x] = page;
  }
  __syncthreads();
  if (!any) return;

  if (it.kind == 0) {
    if (unit >= it.units) return;
    char* base = it.ptr + row0 * it.stride + unit * it.unit;
    auto at = [&](int w) { return base + w * it.stride; };
    if (it.unit == 16) move_unit<kBeams, uint4>(parent, p.n_beam, at);
    else if (it.unit == 4) move_unit<kBeams, uint32_t>(parent, p.n_beam, at);
    else move_unit<kBeams, unsigned char>(parent, p.n_beam, at);
  } else if (it.kind == 1) {
    // the rows [0, rest) of every head of the page being filled; a head's rows are contiguous
    if (rest == 0) return;
    if (unit < it.units) {
      const int within = (int)(unit % p.head_units);
      if (((long)within << p.page_shift) >= (long)rest * p.head_units) return;
      auto at = [&](int w) -> char* { return page_of[w] < 0 ? nullptr : it.ptr + page_of[w] * it.stride + unit * 16; };
      move_unit<kBeams, uint4>(parent, p.n_beam, at);
    } else if (it.scale != nullptr) {
      const long j = unit - it.units;  // (head, row)
      if (j >= ((long)p.n_kv_head << p.page_shift) || (int)(j & ((1 << p.page_shift) - 1)) >= rest) return;
      auto at = [&](int w) -> char* {
        return page_of[w] < 0 ? nullptr : (char*)(it.scale + (((long)page_of[w] * p.n_kv_head) << p.page_shift) + j);
      };
      move_unit<kBeams, unsigned short>(parent, p.n_beam, at);
    }
  } else {
    if (unit >= full) return;
    auto at = [&](int w) { return (char*)(p.page_table + (row0 + w) * p.table_stride + unit); };
    move_unit<kBeams, uint32_t>(parent, p.n_beam, at);
  }
}

}  // namespace

cudaError_t launch_beam_reorder(const ReorderPlan& p, int B, int n_blocks, cudaStream_t s) {
  const dim3 grid((unsigned)n_blocks, (unsigned)B);
  // registers hold one unit per beam: a narrower variant keeps more threads resident
  auto kernel = p.n_beam <= 4 ? beam_reorder_kernel<4> : p.n_beam <= 8 ? beam_reorder_kernel<8> : beam_reorder_kernel<16>;
  return launch_dependent(kernel, grid, dim3(kReorderThreads), 0, s, 1, false, p);
}

}  // namespace wf
