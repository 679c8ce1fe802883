// Device side of beam search: selection over beams and vocabulary, and reordering of the beams' states.
//
// Reordering, in place without a second buffer: a thread owns one unit (16 bytes where alignment allows) of a
// column, loads that unit of every parent that some other beam grew from, and stores only then.  Units of
// different threads do not meet, so no thread sees a half-moved state.  Bound by memory: a row that
// moves is written once and its parent read once (several children of one parent hit L1 / L2).
// Rows that stay (parent = itself) cost nothing.
#include "wf_decoder.h"
#include "wf_ptx.cuh"

namespace wf {

namespace {

// ---------------------------------------------------------------------------------------------
// Selection.  One cluster of blocks per sequence; a block has one slice of the vocabulary of all its beams, cut
// into items (one beam, up to `tiles` tiles of 1024 elements) that its warps take in turn.  A warp holds a tile in
// registers (32 elements a lane) and makes, in one pass over the logits:
//   * the running maximum and sum of exponentials of its lanes;
//   * the item's best `keep` elements: the keep-th largest of the 32 lane maxima is a lower bound of the
//     keep-th largest element, few elements reach it (the bound's own lanes and little more), those are collected and
//     ranked by (value, index).
// After a cluster barrier every block knows every beam's log-sum (partial sums joined in a fixed order, in
// float64), turns its items' elements into float64 scores and keeps the best; the first block joins the blocks'
// lists.  No workspace, no atomics that decide an order, one launch.

constexpr int kSelThreads = 256, kSelWarps = kSelThreads / 32;
constexpr int kPerLane = 32, kTile = 32 * kPerLane;
constexpr int kRanked = 64;  // elements a warp collects and ranks at once; more (many ties) are picked one by one

struct Pick {  // an element with its place in the order: larger value first, then lower index
  float x;
  int v;
};

// Order-preserving map of a float to an unsigned integer above 0 (NaN excluded).
__device__ __forceinline__ uint32_t ordered(float x) {
  const uint32_t b = __float_as_uint(x + 0.f);  // -0 counts as 0
  return b & 0x80000000u ? ~b : b | 0x80000000u;
}
__device__ __forceinline__ float from_ordered(uint32_t k) { return __uint_as_float(k & 0x80000000u ? k & 0x7fffffffu : ~k); }
__device__ __forceinline__ uint64_t ordered(double x) {
  const uint64_t b = (uint64_t)__double_as_longlong(x + 0.0);
  return b >> 63 ? ~b : b | (1ull << 63);
}

// keep-th largest of the lanes' keys (0 counts as none; 0 if there are fewer).
__device__ __forceinline__ uint32_t kth_lane_key(uint32_t key, int keep) {
  uint32_t top = 0;
  for (int i = 0; i < keep; ++i) {
    top = __reduce_max_sync(0xffffffffu, key);
    const unsigned who = __ballot_sync(0xffffffffu, key == top);
    if ((threadIdx.x & 31) == __ffs(who) - 1) key = 0;
  }
  return top;
}

// The best `keep` of n entries by (key descending, tie ascending), found by one warp; entries with key 0 are absent.
// emit(rank, i) is called once for each of them, by one lane.  `found` is the warp's list of n indexes.
template <typename Key, typename Tie, typename Emit>
__device__ void warp_best(int n, int keep, Key key, Tie tie, unsigned short* found, Emit emit) {
  const int lane = threadIdx.x & 31;
  uint32_t high = 0;
  for (int i = lane; i < n; i += 32) high = max(high, (uint32_t)(key(i) >> 32));
  const uint32_t bound = max(kth_lane_key(high, keep), 1u);  // present keys have a high half above 0
  int c = 0;
  for (int i0 = 0; i0 < n; i0 += 32) {
    const int i = i0 + lane;
    const bool in = i < n && (uint32_t)(key(i) >> 32) >= bound;
    const unsigned who = __ballot_sync(0xffffffffu, in);
    if (in) found[c + __popc(who & ((1u << lane) - 1))] = (unsigned short)i;
    c += __popc(who);
  }
  __syncwarp();
  if (c <= kRanked) {
    for (int a = lane; a < c; a += 32) {
      const int i = found[a];
      const uint64_t ki = key(i);
      const uint32_t ti = tie(i);
      int rank = 0;
      for (int b = 0; b < c; ++b) {
        const int j = found[b];
        const uint64_t kj = key(j);
        rank += kj > ki || (kj == ki && tie(j) < ti);
      }
      if (rank < keep) emit(rank, i);
    }
  } else {  // many ties: one after the other, each the best of what comes after the one before
    uint64_t last_k = ~0ull;
    uint32_t last_t = 0;
    for (int r = 0; r < keep; ++r) {
      uint64_t bk = 0;
      uint32_t bt = 0xffffffffu;
      int bi = -1;
      for (int a = lane; a < c; a += 32) {
        const int i = found[a];
        const uint64_t k = key(i);
        const uint32_t t = tie(i);
        const bool after = r == 0 || k < last_k || (k == last_k && t > last_t);
        if (after && (k > bk || (k == bk && t < bt))) bk = k, bt = t, bi = i;
      }
      const uint32_t h = __reduce_max_sync(0xffffffffu, (uint32_t)(bk >> 32));
      const uint32_t l = __reduce_max_sync(0xffffffffu, (uint32_t)(bk >> 32) == h ? (uint32_t)bk : 0u);
      const uint64_t k = ((uint64_t)h << 32) | l;
      if (k == 0) break;
      const uint32_t t = __reduce_min_sync(0xffffffffu, bk == k ? bt : 0xffffffffu);
      if (bk == k && bt == t && bi >= 0) emit(r, bi);
      last_k = k;
      last_t = t;
    }
  }
  __syncwarp();
}

template <typename T>
struct Vec;
template <>
struct Vec<float> {
  static constexpr int n = 4;
  static __device__ __forceinline__ void load(const float* p, float* x) {
    const float4 r = __ldcs(reinterpret_cast<const float4*>(p));
    x[0] = r.x; x[1] = r.y; x[2] = r.z; x[3] = r.w;
  }
};
template <>
struct Vec<__nv_bfloat16> {
  static constexpr int n = 8;
  static __device__ __forceinline__ void load(const __nv_bfloat16* p, float* x) {
    const uint4 r = __ldcs(reinterpret_cast<const uint4*>(p));
    const uint32_t w[4] = {r.x, r.y, r.z, r.w};
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      x[2 * i] = __uint_as_float(w[i] << 16);
      x[2 * i + 1] = __uint_as_float(w[i] & 0xffff0000u);
    }
  }
};
__device__ __forceinline__ float one(const float* p) { return __ldg(p); }
__device__ __forceinline__ float one(const __nv_bfloat16* p) { return __bfloat162float(*p); }

// Best `keep` elements of a tile held in registers (element (j, e) of a lane has index first + (j * 32 + lane) * n + e),
// joined with the `have` elements that the item's earlier tiles left in out[]; returns how many there are now.
template <int kVec>
__device__ int best_of_tile(const float (&x)[kPerLane], float lane_max, int first, int keep, Pick* buf, Pick* out, int have) {
  const int lane = threadIdx.x & 31;
  uint32_t bound = kth_lane_key(lane_max > -INFINITY ? ordered(lane_max) : 0u, keep);
  if (have == keep) bound = max(bound, ordered(out[keep - 1].x));  // the list is full: its last element is a bound too
  const float least = bound ? from_ordered(bound) : -INFINITY;
  int mine = 0;
#pragma unroll
  for (int i = 0; i < kPerLane; ++i) mine += x[i] >= least && x[i] > -INFINITY;
  int before = mine;  // inclusive prefix sum over the lanes
#pragma unroll
  for (int o = 1; o < 32; o <<= 1) {
    const int y = __shfl_up_sync(0xffffffffu, before, o);
    if (lane >= o) before += y;
  }
  const int c = __shfl_sync(0xffffffffu, before, 31);
  if (c == 0) return have;
  if (c + have <= kRanked) {
    int at = before - mine;
    if (mine) {
#pragma unroll
      for (int i = 0; i < kPerLane; ++i)
        if (x[i] >= least && x[i] > -INFINITY) buf[at++] = Pick{x[i], first + ((i / kVec) * 32 + lane) * kVec + i % kVec};
    }
    for (int i = lane; i < have; i += 32) buf[c + i] = out[i];
    __syncwarp();
    const int total = c + have;
    Pick p[2];
    int rank[2];
#pragma unroll
    for (int h = 0; h < 2; ++h) {
      const int i = h * 32 + lane;
      rank[h] = keep;
      if (i < total) {
        p[h] = buf[i];
        rank[h] = 0;
        for (int j = 0; j < total; ++j) {
          const Pick q = buf[j];
          rank[h] += q.x > p[h].x || (q.x == p[h].x && q.v < p[h].v);
        }
      }
    }
    __syncwarp();
#pragma unroll
    for (int h = 0; h < 2; ++h)
      if (rank[h] < keep) out[rank[h]] = p[h];
    __syncwarp();
    return min(total, keep);
  }
  // many elements reach the bound: pick the best one by one, from the registers and the old list alike
  for (int i = lane; i < have; i += 32) buf[i] = out[i];
  __syncwarp();
  float last_x = INFINITY;
  int last_v = -1, r = 0;
  for (; r < keep; ++r) {
    float bx = -INFINITY;
    int bv = 0x7fffffff;
    auto consider = [&](float y, int v) {
      const bool after = r == 0 || y < last_x || (y == last_x && v > last_v);
      if (after && y > -INFINITY && (y > bx || (y == bx && v < bv))) bx = y, bv = v;
    };
#pragma unroll
    for (int i = 0; i < kPerLane; ++i) consider(x[i], first + ((i / kVec) * 32 + lane) * kVec + i % kVec);
    for (int i = lane; i < have; i += 32) consider(buf[i].x, buf[i].v);
    const uint32_t k = __reduce_max_sync(0xffffffffu, bx > -INFINITY ? ordered(bx) : 0u);
    if (k == 0) break;
    last_x = from_ordered(k);
    last_v = (int)__reduce_min_sync(0xffffffffu, bx > -INFINITY && ordered(bx) == k ? (unsigned)bv : 0xffffffffu);
    if (lane == 0) out[r] = Pick{last_x, last_v};
  }
  __syncwarp();
  return r;
}

static_assert(kSelWarps >= 8, "the join of a cluster's lists uses the warps' lists");
struct SelectShared {  // sizes of the dynamic shared memory's parts
  int items, entries;
  size_t pick, stat, rows, found, best, total;
};
__host__ __device__ inline SelectShared select_shared(int n_beam, int groups, int keep) {
  SelectShared s;
  s.items = n_beam * groups;
  s.entries = s.items * keep + n_beam;
  size_t at = 0;
  s.best = at; at += (size_t)kSelWarps * keep * 16;                 // per warp: (key, tie, -); the first `keep` also: the block's list
  s.pick = at; at += (size_t)s.entries * sizeof(Pick);
  s.stat = at; at += (size_t)s.items * 8;
  s.rows = at; at += (size_t)((s.entries + 15) / 16 * 16);          // beam of each entry
  s.found = at; at += (size_t)(s.entries + 8 * kMaxKeep) * 2 + 16;  // index lists of all warps, or of one
  s.total = (at + 15) / 16 * 16;
  return s;
}

struct Ranked {
  uint64_t key;
  uint32_t flat;
  uint32_t unused;
};

template <typename T>
__global__ void __launch_bounds__(kSelThreads) beam_select_kernel(const __grid_constant__ BeamSelectParams p, int cluster) {
  extern __shared__ __align__(16) unsigned char dyn[];
  __shared__ Pick buf[kSelWarps][kRanked];
  __shared__ int live_row[kMaxBeams];  // beams whose logits are read
  __shared__ int n_live, n_done;
  __shared__ double block_l[kMaxBeams], lse[kMaxBeams];
  __shared__ float block_m[kMaxBeams];
  __shared__ Ranked list[kMaxKeep];
  const SelectShared sh = select_shared(p.n_beam, p.groups, p.keep);
  Ranked* best = reinterpret_cast<Ranked*>(dyn + sh.best);
  Pick* pick = reinterpret_cast<Pick*>(dyn + sh.pick);
  float2* stat = reinterpret_cast<float2*>(dyn + sh.stat);
  unsigned char* beam_of = dyn + sh.rows;
  unsigned short* found = reinterpret_cast<unsigned short*>(dyn + sh.found);
  const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5;
  const int rank = (int)blockIdx.x % cluster, b = (int)blockIdx.x / cluster;
  constexpr int kVec = Vec<T>::n;

  if (tid == 0) {
    int live = p.n_beam;
    if (p.beams) {
      const int asked = __ldg(p.beams + b);
      live = min(max(asked, 0), p.n_beam);
      if (live != asked && rank == 0) report(p.status, kBadRows);
    }
    int n = 0, done = 0;
    for (int w = 0; w < live; ++w) {
      if (p.finished && p.finished[(long)b * p.n_beam + w]) {
        if (rank == 0) {  // the one continuation of a finished beam, behind the items' entries
          pick[sh.items * p.keep + done] = Pick{0.f, p.end_token};
          beam_of[sh.items * p.keep + done] = (unsigned char)w;
          ++done;
        }
        lse[w] = 0.0;
      } else {
        live_row[n++] = w;
      }
    }
    n_live = n;
    n_done = done;
  }
  __syncthreads();
  const int n_items = n_live * p.groups;

  // ---- items: statistics and best elements
  for (int item = warp; item < n_items; item += kSelWarps) {
    const int w = live_row[item / p.groups], g = item % p.groups;
    const T* row = reinterpret_cast<const T*>(p.logits) + ((long)b * p.n_beam + w) * p.ld;
    const int shift = (int)(((uintptr_t)row / sizeof(T)) % kVec);  // windows start at 16-byte borders
    const int slice_end = min(p.vocab, (rank + 1) * p.slice - shift);
    float m = -INFINITY, l = 0.f;
    int have = 0;
    Pick* out = pick + item * p.keep;
    for (int t = 0; t < p.tiles; ++t) {
      const int first = rank * p.slice - shift + (g * p.tiles + t) * kTile;
      if (first >= slice_end) break;
      float x[kPerLane];
#pragma unroll
      for (int j = 0; j < kPerLane / kVec; ++j) {
        const int v = first + (j * 32 + lane) * kVec;
        if (v >= 0 && v + kVec <= slice_end) {
          Vec<T>::load(row + v, x + j * kVec);
        } else {
#pragma unroll
          for (int e = 0; e < kVec; ++e) x[j * kVec + e] = v + e >= 0 && v + e < slice_end ? one(row + v + e) : -INFINITY;
        }
      }
      if (p.suppress) {
        const unsigned char* bits = reinterpret_cast<const unsigned char*>(p.suppress);
        const int n_bytes = (p.vocab + 31) / 32 * 4;
#pragma unroll
        for (int j = 0; j < kPerLane / kVec; ++j) {
          const int v = first + (j * 32 + lane) * kVec;
          if (v + kVec <= 0 || v >= slice_end) continue;
          const int at = max(v, 0) >> 3, off = max(v, 0) & 7;
          unsigned word = __ldg(bits + at);
          if (at + 1 < n_bytes) word |= (unsigned)__ldg(bits + at + 1) << 8;
          word = (word >> off) << (max(v, 0) - v);
          if (word & ((1u << kVec) - 1)) {
#pragma unroll
            for (int e = 0; e < kVec; ++e)
              if ((word >> e) & 1) x[j * kVec + e] = -INFINITY;
          }
        }
      }
      float top = -INFINITY;
#pragma unroll
      for (int i = 0; i < kPerLane; ++i) top = fmaxf(top, x[i]);
      const float m_new = fmaxf(m, top);
      const float base = m_new == -INFINITY ? 0.f : m_new;
      l *= exp2f((m - base) * 1.4426950408889634f);
#pragma unroll
      for (int i = 0; i < kPerLane; ++i) l += exp2f((x[i] - base) * 1.4426950408889634f);
      m = m_new;
      have = best_of_tile<kVec>(x, top, first, p.keep, buf[warp], out, have);
    }
    float wm = m;
#pragma unroll
    for (int o = 16; o > 0; o >>= 1) wm = fmaxf(wm, __shfl_xor_sync(0xffffffffu, wm, o));
    float wl = l * exp2f((m - (wm == -INFINITY ? 0.f : wm)) * 1.4426950408889634f);
#pragma unroll
    for (int o = 16; o > 0; o >>= 1) wl += __shfl_xor_sync(0xffffffffu, wl, o);
    if (lane == 0) stat[item] = make_float2(wm, wl);
    for (int i = lane; i < p.keep; i += 32) {
      if (i >= have) out[i].v = -1;
      beam_of[item * p.keep + i] = (unsigned char)w;
    }
  }
  __syncthreads();
  if (tid < n_live) {
    float m = -INFINITY;
    for (int g = 0; g < p.groups; ++g) m = fmaxf(m, stat[tid * p.groups + g].x);
    double l = 0.0;
    for (int g = 0; g < p.groups; ++g) {
      const float2 s = stat[tid * p.groups + g];
      if (s.y != 0.f) l += (double)s.y * exp((double)s.x - (double)m);
    }
    block_m[tid] = m;
    block_l[tid] = l;
  }
  __syncwarp();
  ptx::cluster_sync_all();
  if (tid < n_live) {  // log-sum of a beam from all blocks' parts, in rank order
    const uint32_t am = ptx::smem_u32(block_m + tid), al = ptx::smem_u32(block_l + tid);
    float m = -INFINITY;
    for (int r = 0; r < cluster; ++r) m = fmaxf(m, ptx::ld_cluster_f32(ptx::map_to_cta(am, r)));
    double l = 0.0;
    for (int r = 0; r < cluster; ++r) {
      const double lr = ptx::ld_cluster_f64(ptx::map_to_cta(al, r));
      const float mr = ptx::ld_cluster_f32(ptx::map_to_cta(am, r));
      if (lr != 0.0) l += lr * exp((double)mr - (double)m);
    }
    lse[live_row[tid]] = (double)m + log(l);  // NaN if the row holds one, or +infinity
  }
  __syncthreads();

  // ---- the block's best: every warp of a share of the entries, then the first warp of the warps' lists
  const float* scores = p.scores + (long)b * p.n_beam;
  auto key_of = [&](int e) -> uint64_t {
    const Pick q = pick[e];
    if (q.v < 0) return 0;
    const int w = beam_of[e];
    const double c = (double)__ldg(scores + w) + ((double)q.x - lse[w]);
    return c > -INFINITY ? ordered(c) : 0;  // false for NaN
  };
  auto flat_of = [&](int e) -> uint32_t { return (uint32_t)beam_of[e] * (uint32_t)p.vocab + (uint32_t)pick[e].v; };
  const int n_entries = n_items * p.keep;
  {
    const int share = (n_entries + kSelWarps - 1) / kSelWarps, e0 = min(warp * share, n_entries), n = min(share, n_entries - e0);
    for (int i = lane; i < p.keep; i += 32) best[warp * p.keep + i].key = 0;
    __syncwarp();
    warp_best(n, p.keep, [&](int i) { return key_of(e0 + i); }, [&](int i) { return flat_of(e0 + i); }, found + e0, [&](int r, int i) {
      best[warp * p.keep + r].key = key_of(e0 + i);
      best[warp * p.keep + r].flat = flat_of(e0 + i);
    });
  }
  __syncthreads();
  if (warp == 0) {
    const int done0 = sh.items * p.keep, n = kSelWarps * p.keep + n_done;
    auto key = [&](int i) { return i < kSelWarps * p.keep ? best[i].key : key_of(done0 + i - kSelWarps * p.keep); };
    auto flat = [&](int i) { return i < kSelWarps * p.keep ? best[i].flat : flat_of(done0 + i - kSelWarps * p.keep); };
    for (int i = lane; i < p.keep; i += 32) list[i].key = 0;
    __syncwarp();
    warp_best(n, p.keep, key, flat, found, [&](int r, int i) {
      list[r].key = key(i);
      list[r].flat = flat(i);
    });
  }
  __syncwarp();
  ptx::cluster_sync_all();

  // ---- the sequence's best
  if (rank == 0 && warp == 0) {
    for (int i = lane; i < cluster * p.keep; i += 32) {
      const uint32_t a = ptx::map_to_cta(ptx::smem_u32(list + i % p.keep), i / p.keep);
      best[i].key = ptx::ld_cluster_u64(a);
      best[i].flat = ptx::ld_cluster_u32(a + 8);
    }
    __syncwarp();
    const long o = (long)b * p.keep;
    for (int i = lane; i < p.keep; i += 32) {
      p.out_scores[o + i] = -INFINITY;
      p.out_parents[o + i] = p.out_tokens[o + i] = -1;
      if (p.out_finished) p.out_finished[o + i] = 0;
    }
    __syncwarp();
    warp_best(cluster * p.keep, p.keep, [&](int i) { return best[i].key; }, [&](int i) { return best[i].flat; }, found, [&](int r, int i) {
      const uint64_t k = best[i].key;
      const double c = __longlong_as_double((long long)(k >> 63 ? k & ~(1ull << 63) : ~k));
      const int w = (int)(best[i].flat / (uint32_t)p.vocab), v = (int)(best[i].flat % (uint32_t)p.vocab);
      p.out_scores[o + r] = (float)c;
      p.out_parents[o + r] = w;
      p.out_tokens[o + r] = v;
      if (p.out_finished) p.out_finished[o + r] = v == p.end_token || (p.finished && p.finished[(long)b * p.n_beam + w]);
    });
  }
  __syncwarp();
  ptx::cluster_sync_all();  // the lists stay until they have been read
}

// ---------------------------------------------------------------------------------------------
// Reordering.

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

cudaError_t launch_beam_select(BeamSelectParams p, int B, int dtype, int num_sms, cudaStream_t s) {
  // enough blocks for two on every SM, at least one tile of every row each, at most the 8 of a portable cluster
  int cluster = 1;
  while (cluster < 8 && (long)B * cluster < 2L * num_sms && p.vocab > cluster * kTile) cluster *= 2;
  p.slice = ((p.vocab + 8 + cluster - 1) / cluster + 7) / 8 * 8;
  const int n_tiles = (p.slice + kTile - 1) / kTile;
  p.tiles = (n_tiles + 15) / 16;  // at most 16 items of a row in a block
  p.groups = (n_tiles + p.tiles - 1) / p.tiles;
  const size_t smem = select_shared(p.n_beam, p.groups, p.keep).total;
  auto kernel = dtype == WF_BF16 ? beam_select_kernel<__nv_bfloat16> : beam_select_kernel<float>;
  cudaError_t e = cudaSuccess;
  if (smem > 40 * 1024) e = cudaFuncSetAttribute(kernel, cudaFuncAttributeMaxDynamicSharedMemorySize, (int)smem);
  if (e != cudaSuccess) return e;
  return launch_dependent(kernel, dim3((unsigned)(B * cluster)), dim3(kSelThreads), smem, s, cluster, false, p, cluster);
}

cudaError_t launch_beam_reorder(const ReorderPlan& p, int B, int n_blocks, cudaStream_t s) {
  const dim3 grid((unsigned)n_blocks, (unsigned)B);
  // registers hold one unit per beam: a narrower variant keeps more threads resident
  auto kernel = p.n_beam <= 4 ? beam_reorder_kernel<4> : p.n_beam <= 8 ? beam_reorder_kernel<8> : beam_reorder_kernel<16>;
  return launch_dependent(kernel, grid, dim3(kReorderThreads), 0, s, 1, false, p);
}

}  // namespace wf
