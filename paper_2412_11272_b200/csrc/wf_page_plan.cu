// Rows and pages of one round, planned on the device: which sequences get the rows they ask for, which free pages they
// take, what the ended ones give back, and for every row its sequence, position and place in the cache.
//
//   need_s = max(0, ceil((len_s + n_s) / P) - held_s)      granted_s = (sum_{t<=s} n_t <= rows) and (need_s = 0 or sum_{t<=s} need_t <= free)
//   cu = prefix sums of the granted n;   new page i of s = ring[head + sum_{t<s} need_t + i]
//
// Everything but the rows is a few prefix sums over the sequences; what bounds a call is latency (one chain of loads, two
// scans, the writes) and for prompts the instructions of the rows.  So one launch for an ordinary round: a block makes all sums
// in shared memory and writes the pages and rows.  For prompts a cluster of blocks, each of which makes all prefix sums for
// itself (no exchange), shares the pages, and the rows, 16 bytes each, are written by a grid of their own behind it: 213 thousand
// rows of 256 prompts in 15 us, in the cluster itself 55.  The state is updated in place, so a barrier stands between its last
// read and its first write.
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

__device__ __forceinline__ int wrap(long i, int n) { return (int)(i >= n ? i - n : i); }  // i < 2 n

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
      if (end > (long long)p.table_stride * page || end > INT_MAX) {
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
    p.ring[wrap((long)head + free + i, p.n_pages)] = x;
  }
  if (returned > 0 && n_new > 0) {  // an ended sequence's table is read before its successor's pages are written to it
    __syncwarp();
    if (cluster > 1) ptx::cluster_sync_all();
    else __syncthreads();
  }
  for (int i = at; i < n_new; i += step) {
    const int s = find(base, n, i);
    const int x = p.ring[wrap((long)head + i, p.n_pages)];
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
      p.pool[0] = wrap((long)head + n_new, p.n_pages);
      p.pool[1] = free - n_new + returned;
    }
  }
  // ---- the rows, where they are not left to a launch of their own; those behind the last sequence belong to none
  if (cluster == 1)
    for (int r = tid; r < p.n_rows; r += kPlanThreads) {
      int s = -1, pos = -1;
      long long slot = -1;
      if (r < n_rows) {
        s = find(cu, n, r);
        pos = len[s] + (r - cu[s]);
        const int index = pos >> p.page_shift, mine = index - held[s];
        // pages that were held before are in the table, new ones still at the front of the ring as well
        const int x = mine < 0 ? __ldcg(p.table + (long)s * p.table_stride + index) : __ldcg(p.ring + wrap((long)head + base[s] + mine, p.n_pages));
        if (x < 0 || x >= p.n_pages) problems |= kBadPage;
        else slot = ((long long)x << p.page_shift) + (pos & (page - 1));
      }
      if (p.row_seq) p.row_seq[r] = s;
      if (p.row_pos) p.row_pos[r] = pos;
      if (p.row_slot) p.row_slot[r] = slot;
    }
  if (problems != 0) report(p.status, problems);
}

// The rows of a planned round: four consecutive ones per thread, so that most look for their sequence once.
constexpr int kRowThreads = 256;
__global__ void __launch_bounds__(kRowThreads) plan_rows_kernel(const __grid_constant__ PagePlanParams p) {
  extern __shared__ int cu[];
  for (int s = threadIdx.x; s <= p.n_seq; s += kRowThreads) cu[s] = __ldg(p.cu_rows + s);
  __syncthreads();
  const int n_rows = cu[p.n_seq], r0 = (int)(blockIdx.x * kRowThreads + threadIdx.x) * 4, page = 1 << p.page_shift;
  int seq[4], pos[4], s = 0, problems = 0;
  long long slot[4];
  for (int i = 0; i < 4; ++i) {
    const int r = r0 + i;
    seq[i] = pos[i] = -1;
    slot[i] = -1;
    if (r >= n_rows) continue;
    if (i == 0 || r >= cu[s + 1]) s = find(cu, p.n_seq, r);
    seq[i] = s;
    pos[i] = __ldg(p.lengths + s) + (r - cu[s]);
    const int x = __ldg(p.table + (long)s * p.table_stride + (pos[i] >> p.page_shift));
    if (x < 0 || x >= p.n_pages) problems |= kBadPage;
    else slot[i] = ((long long)x << p.page_shift) + (pos[i] & (page - 1));
  }
  if (problems != 0) report(p.status, problems);
  const bool whole = r0 + 4 <= p.n_rows;
  auto put4 = [&](int* to, const int (&v)[4]) {
    if (to == nullptr) return;
    if (whole && ((uintptr_t)to & 15) == 0) *reinterpret_cast<int4*>(to + r0) = make_int4(v[0], v[1], v[2], v[3]);
    else
      for (int i = 0; i < 4; ++i)
        if (r0 + i < p.n_rows) to[r0 + i] = v[i];
  };
  put4(p.row_seq, seq);
  put4(p.row_pos, pos);
  if (p.row_slot == nullptr) return;
  if (whole && ((uintptr_t)p.row_slot & 15) == 0) {
    longlong2* to = reinterpret_cast<longlong2*>(p.row_slot + r0);
    to[0] = make_longlong2(slot[0], slot[1]);
    to[1] = make_longlong2(slot[2], slot[3]);
  } else {
    for (int i = 0; i < 4; ++i)
      if (r0 + i < p.n_rows) p.row_slot[r0 + i] = slot[i];
  }
}

}  // namespace

cudaError_t launch_page_plan(const PagePlanParams& p, cudaStream_t s) {
  // One block up to four rows per thread, else a cluster of eight and a launch for the rows (64 sequences, 2048 rows: 7.0 us in one
  // block, 7.9 so; 4096: 9.4 and 7.8).
  const int cluster = p.n_rows <= 4 * kPlanThreads ? 1 : 8;
  const size_t smem = (size_t)(5 * (long)p.n_seq + 3) * sizeof(int);
  cudaError_t e = cudaFuncSetAttribute(page_plan_kernel, cudaFuncAttributeMaxDynamicSharedMemorySize, (5 * kMaxPlanned + 3) * (int)sizeof(int));
  if (e != cudaSuccess) return e;
  e = launch_dependent(page_plan_kernel, dim3((unsigned)cluster), dim3(kPlanThreads), smem, s, cluster, false, p, cluster);
  if (e != cudaSuccess || cluster == 1 || (p.row_seq == nullptr && p.row_pos == nullptr && p.row_slot == nullptr)) return e;
  return launch_dependent(plan_rows_kernel, dim3((unsigned)((p.n_rows + 4 * kRowThreads - 1) / (4 * kRowThreads))), dim3(kRowThreads),
                          (size_t)(p.n_seq + 1) * sizeof(int), s, 1, false, p);
}

}  // namespace wf
