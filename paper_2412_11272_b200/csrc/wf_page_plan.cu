// Rows and pages of one round, planned on the device: which sequences get the rows they ask for, which free pages they
// take, what the ended ones give back, and for every row its sequence, position and place in the cache.
//
//   need_s = max(0, ceil((len_s + n_s) / P) - held_s)      granted_s = (sum_{t<=s} n_t <= rows) and (need_s = 0 or sum_{t<=s} need_t <= free)
//   cu = prefix sums of the granted n;   new page i of s = ring[head + sum_{t<s} need_t + i]
//
// Everything but the rows is a few prefix sums over the sequences; what bounds a call is latency (one chain of loads, two
// scans, the writes) and for prompts the 16 bytes written per row.  So one launch of one cluster: every block makes all
// prefix sums for itself in shared memory (no exchange), and the blocks share the pages and rows.  The state is updated in
// place, so a cluster barrier stands between its last read and its first write.
#include <limits.h>

#include "wf_decoder.h"
#include "wf_ptx.cuh"

namespace wf {
namespace {

constexpr int kPlanThreads = 512;
constexpr int kPlanWarps = kPlanThreads / 32;

// Exclusive prefix sum over the block's threads; `total` gets the sum.
__device__ __forceinline__ long long block_scan(long long x, long long* warp_sum, long long* total) {
  const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
  long long sum = x;
#pragma unroll
  for (int o = 1; o < 32; o *= 2) {
    const long long up = __shfl_up_sync(0xffffffffu, sum, o);
    if (lane >= o) sum += up;
  }
  __syncthreads();  // the sums of the scan before have been read
  if (lane == 31) warp_sum[warp] = sum;
  __syncthreads();
  long long before = 0, all = 0;
#pragma unroll
  for (int w = 0; w < kPlanWarps; ++w) {
    const long long y = warp_sum[w];
    if (w < warp) before += y;
    all += y;
  }
  *total = all;
  return before + sum - x;
}

// The largest s in [0, n) with sums[s] <= i, where sums[0] <= i (sums does not decrease).
__device__ __forceinline__ int find(const int* sums, int n, int i) {
  int lo = 0, hi = n;
  while (hi - lo > 1) {
    const int mid = (lo + hi) >> 1;
    if (sums[mid] <= i) lo = mid;
    else hi = mid;
  }
  return lo;
}

__global__ void __launch_bounds__(kPlanThreads) page_plan_kernel(const __grid_constant__ PagePlanParams p, int cluster) {
  extern __shared__ int sums[];
  __shared__ long long warp_sum[kPlanWarps];
  const int n = p.n_seq, tid = threadIdx.x, page = 1 << p.page_shift;
  int* cu = sums;             // [n + 1] granted rows, summed
  int* base = cu + n + 1;     // [n + 1] new pages, summed
  int* back = base + n + 1;   // [n + 1] pages given back, summed
  int* len = back + n + 1;    // [n] positions held
  int* held = len + n;        // [n] pages held before the new ones
  const int rank = cluster > 1 ? (int)ptx::cluster_ctarank() : 0;

  int head = __ldcg(p.pool), free = __ldcg(p.pool + 1);
  const bool bad_pool = head < 0 || head >= p.n_pages || free < 0 || free > p.n_pages;
  if (bad_pool) head = free = 0;
  int problems = bad_pool ? kBadRows : 0;

  // ---- what every sequence asks for
  for (int s = tid; s < n; s += kPlanThreads) {
    int l = __ldcg(p.lengths + s), h = __ldcg(p.held + s), want = __ldg(p.new_rows + s), gone = 0;
    const bool ended = p.ended != nullptr && p.ended[s] != 0;
    if (l < 0 || h < 0 || h > p.table_stride || (long long)l > (long long)h * page || want < 0) {
      problems |= kBadRows;  // left as it is, and without rows
      want = 0;
      h |= INT_MIN;          // (no length or pages to be written)
    } else if (ended && !bad_pool) {
      gone = h;
      l = h = 0;
    }
    int need = 0;
    if (want > 0) {
      const long long end = (long long)l + want;
      if (end > (long long)p.table_stride * page) {
        problems |= kBadRows;
        want = 0;
      } else {
        need = max(0, (int)((end + page - 1) >> p.page_shift) - h);
        want = min(want, p.n_rows + 1);
      }
    }
    cu[s] = want;
    base[s] = need;
    back[s] = gone;
    len[s] = l;
    held[s] = h;
  }
  __syncthreads();

  // ---- prefix sums: a thread takes consecutive sequences
  const int each = (n + kPlanThreads - 1) / kPlanThreads, first = min(n, tid * each), last = min(n, first + each);
  long long rows = 0, pages = 0, given = 0, total;
  for (int s = first; s < last; ++s) {
    rows += cu[s];
    pages += base[s];
    given += back[s];
  }
  rows = block_scan(rows, warp_sum, &total);
  pages = block_scan(pages, warp_sum, &total);
  given = block_scan(given, warp_sum, &total);
  const int room = p.n_pages - free;  // more cannot come back
  if (total > room) problems |= kBadRows;
  const int returned = (int)min(total, (long long)room);
  long long granted = 0;
  for (int s = first; s < last; ++s) {
    const int want = cu[s], need = base[s], gone = back[s];
    rows += want;
    pages += need;
    const bool ok = !bad_pool && rows <= p.n_rows && (need == 0 || pages <= free);
    if (want > 0 && !ok) problems |= kPutOff;
    cu[s] = ok ? want : 0;
    // Whoever gets pages comes behind sequences that all got theirs (one without would have left too few for it as
    // well), so its pages begin behind all that was asked for before.  The sums of the others are cut to what is free.
    base[s] = (int)min(pages - need, (long long)free);
    back[s] = (int)min(given, (long long)returned);
    given += gone;
    granted += cu[s];
    if (need > 0 && !ok) base[s] |= INT_MIN;  // marks: asked, and got none
  }
  granted = block_scan(granted, warp_sum, &total);
  __syncthreads();
  for (int s = first; s < last; ++s) {
    const int want = cu[s];
    cu[s] = (int)granted;
    granted += want;
  }
  __syncthreads();
  const int n_rows = (int)total;
  // New pages of a sequence end where the next one's begin.  Behind the first that got none nobody gets any: all sums from
  // there on stand for the number of pages handed out.
  __shared__ int handed;
  if (tid == 0) {
    handed = INT_MAX;
    cu[n] = n_rows;
    back[n] = returned;
  }
  __syncthreads();
  for (int s = tid; s < n; s += kPlanThreads)
    if (base[s] < 0) atomicMin(&handed, base[s] & INT_MAX);
  __syncthreads();
  if (handed == INT_MAX) {
    if (last == n && first < last) base[n] = (int)pages;  // all were granted: their sum
    if (n == 0 && tid == 0) base[n] = 0;
  } else {
    for (int s = tid; s <= n; s += kPlanThreads) base[s] = s < n ? min(base[s] & INT_MAX, handed) : handed;
  }
  __syncthreads();
  const int n_new = base[n];

  // ---- the last read of what is updated in place lies behind
  if (cluster > 1) ptx::cluster_sync_all();
  const int at = rank * kPlanThreads + tid, step = cluster * kPlanThreads;
  for (int i = at; i < returned; i += step) {
    const int s = find(back, n, i);
    const int x = __ldcg(p.table + (long)s * p.table_stride + (i - back[s]));
    if (x < 0 || x >= p.n_pages) problems |= kBadPage;
    const long to = (long)head + free + i;
    p.ring[to % p.n_pages] = x;
  }
  if (returned > 0 && n_new > 0) {  // an ended sequence's table is read before its successor's pages are written to it
    __syncwarp();
    if (cluster > 1) ptx::cluster_sync_all();
    else __syncthreads();
  }
  for (int i = at; i < n_new; i += step) {
    const int s = find(base, n, i);
    const int x = p.ring[((long)head + i) % p.n_pages];
    if (x < 0 || x >= p.n_pages) problems |= kBadPage;
    p.table[(long)s * p.table_stride + held[s] + (i - base[s])] = x;
  }
  for (int s = at; s < n; s += step) {
    p.cu_rows[s] = cu[s];
    if (held[s] >= 0) {
      p.held[s] = held[s] + base[s + 1] - base[s];
      p.lengths[s] = len[s];
    }
  }
  if (at == 0) {
    p.cu_rows[n] = n_rows;
    if (!bad_pool) {
      p.pool[0] = (int)(((long)head + n_new) % p.n_pages);
      p.pool[1] = free - n_new + returned;
    }
  }
  // ---- the rows; those behind the last sequence belong to none
  for (int r = at; r < p.n_rows; r += step) {
    int s = -1, pos = -1;
    long long slot = -1;
    if (r < n_rows) {
      s = find(cu, n, r);
      pos = len[s] + (r - cu[s]);
      const int index = pos >> p.page_shift, mine = index - held[s];
      // pages that were held before are in the table, new ones still at the front of the ring as well
      const int x = mine < 0 ? __ldcg(p.table + (long)s * p.table_stride + index) : __ldcg(p.ring + ((long)head + base[s] + mine) % p.n_pages);
      if (x < 0 || x >= p.n_pages) problems |= kBadPage;
      else slot = ((long long)x << p.page_shift) + (pos & (page - 1));
    }
    if (p.row_seq) p.row_seq[r] = s;
    if (p.row_pos) p.row_pos[r] = pos;
    if (p.row_slot) p.row_slot[r] = slot;
  }
  if (problems != 0) report(p.status, problems);
}

}  // namespace

cudaError_t launch_page_plan(const PagePlanParams& p, cudaStream_t s) {
  // one block where it writes a few rows per thread, else a cluster of eight
  const int cluster = p.n_rows <= 4 * kPlanThreads ? 1 : 8;
  const size_t smem = (size_t)(5 * (long)p.n_seq + 3) * sizeof(int);
  cudaError_t e = cudaFuncSetAttribute(page_plan_kernel, cudaFuncAttributeMaxDynamicSharedMemorySize, (int)smem);
  if (e != cudaSuccess) return e;
  return launch_dependent(page_plan_kernel, dim3((unsigned)cluster), dim3(kPlanThreads), smem, s, cluster, false, p, cluster);
}

}  // namespace wf
