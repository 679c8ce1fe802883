// Drafted tokens verified against the target's distribution, and the accepted rows moved behind the committed ones.
//
// Verification.  A sequence's rows are its last committed token (row 0) and drafts, each the child of an earlier row.  At
// a row w the target's distribution is p = softmax(logits_w / T); children are tried in row order.  A child with token x
// is taken if u q(x) < p(x), q being the distribution it was drawn from (a drafted token that was not drawn: q(x) = 1);
// otherwise p becomes max(p - q, 0), normalised, and the next child is tried.  Where no child is taken the token that follows
// is drawn from p: the first v whose running sum, in the order of the vocabulary, exceeds u' times the whole.
//
// Bytes: the logits of the rows on the path, once, and one row of q; what bounds a call is the chain of row after row, each
// a pass over the vocabulary and an exchange.  So one cluster of blocks per sequence walks its path in one launch: a pass is
// shared by the blocks, partial results go to every block's shared memory, and all blocks then take the same decision from
// the same numbers.  Rows off the path are not read.  The sums that decide a drawn token are float64, exponentials
// included: a vocabulary's running sum has steps of 1e-6 or less, so in float32 the token would depend on the order of
// summation.  Acceptance needs the row's sum alone, where float32 exponentials (1e-7) are enough.
#include <math.h>

#include "wf_decoder.h"
#include "wf_ptx.cuh"

namespace wf {
namespace {

constexpr int kVerThreads = 512;
constexpr int kVerWarps = kVerThreads / 32;
constexpr int kVerTiles = 1024;  // runs of the vocabulary whose sums a block keeps
constexpr int kMaxCluster = 8;

template <typename T>
struct VecOf;
template <>
struct VecOf<float> {
  static constexpr int n = 4;
  static __device__ __forceinline__ void unpack(uint4 u, float (&y)[n]) {
    y[0] = __uint_as_float(u.x), y[1] = __uint_as_float(u.y), y[2] = __uint_as_float(u.z), y[3] = __uint_as_float(u.w);
  }
  static __device__ __forceinline__ float one(const float* x) { return __ldg(x); }
};
template <>
struct VecOf<__nv_bfloat16> {
  static constexpr int n = 8;
  static __device__ __forceinline__ void unpack(uint4 u, float (&y)[n]) {
    const uint32_t w[4] = {u.x, u.y, u.z, u.w};
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      y[2 * i] = __uint_as_float(w[i] << 16);
      y[2 * i + 1] = __uint_as_float(w[i] & 0xffff0000u);
    }
  }
  static __device__ __forceinline__ float one(const __nv_bfloat16* x) { return __bfloat162float(*x); }
};

// A row of logits cut into 16-byte pieces from the boundary at or below its first element: piece i holds the elements
// i n - shift .. ; what lies outside the row counts as -infinity.
template <typename T>
struct LogitRow {
  const T* x;
  int vocab, shift, pieces;
  __device__ __forceinline__ LogitRow(const T* row, int v) : x(row), vocab(v) {
    shift = (int)(((uintptr_t)row & 15) / sizeof(T));
    pieces = (int)(((long)v + shift + VecOf<T>::n - 1) / VecOf<T>::n);
  }
  __device__ __forceinline__ int first(int i) const { return i * VecOf<T>::n - shift; }
  __device__ __forceinline__ void load(int i, float (&y)[VecOf<T>::n]) const {
    const int v = first(i);
    if (i < pieces && v >= 0 && v <= vocab - VecOf<T>::n) {
      VecOf<T>::unpack(__ldg(reinterpret_cast<const uint4*>(x + v)), y);
    } else {
#pragma unroll
      for (int e = 0; e < VecOf<T>::n; ++e) y[e] = i < pieces && v + e >= 0 && v + e < vocab ? VecOf<T>::one(x + v + e) : -INFINITY;
    }
  }
};

// What blocks and warps tell each other about a pass: the largest logit, its first place, and a sum.
struct __align__(16) Part {
  float top;
  int at;
  double sum;
};

template <typename T>
__global__ void __launch_bounds__(kVerThreads) draft_verify_kernel(const __grid_constant__ DraftVerifyParams p, int cluster) {
  constexpr int kVec = VecOf<T>::n;
  __shared__ Part gather[2][kMaxCluster * kVerWarps];
  __shared__ double tile_sum[kVerTiles];
  __shared__ double inverse[kMaxDrafts];  // of the sums left after each refusal at the present row
  __shared__ int token[kMaxDrafts], parent[kMaxDrafts];
  __shared__ float chance[kMaxDrafts];
  __shared__ int refused[kMaxDrafts];     // tokens that were not drawn and not taken at the present row
  const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5;
  const int rank = cluster > 1 ? (int)ptx::cluster_ctarank() : 0;
  const int s = (int)blockIdx.x / cluster;
  int turn = 0;  // which of the two gather buffers the next exchange uses

  const int row0 = __ldg(p.cu_rows + s), end = __ldg(p.cu_rows + s + 1);
  int n = end - row0, problems = 0;
  if (row0 < 0 || end < row0 || end > p.n_rows) {
    problems |= kBadRows;
    n = 0;
  }
  if (n > p.max_rows) {
    problems |= kBadRows;
    n = p.max_rows;
  }
  for (int i = tid; i < n; i += kVerThreads) {
    const int x = __ldg(p.tokens + row0 + i);
    int up = p.parents ? __ldg(p.parents + row0 + i) : i - 1;
    if (i > 0 && (up < 0 || up >= i)) {
      problems |= kBadParent;
      up = -1;  // never tried
    }
    if (i > 0 && (x < 0 || x >= p.vocab)) {
      problems |= kBadValue;
      up = -1;
    }
    token[i] = x;
    parent[i] = i > 0 ? up : -1;
    chance[i] = __ldg(p.accept_u + row0 + i);
  }
  const float t = p.temperature ? __ldg(p.temperature + s) : 1.f;
  if (n > 0 && !(t >= 0.f && t < INFINITY)) {
    problems |= kBadValue;
    n = 0;
  }
  if (problems != 0) report(p.status, problems);
  const bool greedy = t == 0.f;
  const double per_t = greedy ? 0.0 : 1.0 / (double)t;
  // (a temperature near the smallest float must not make 0 x infinity of the largest logit)
  const float per_t_log2 = greedy ? 0.f : fminf((float)(1.4426950408889634 * per_t), 3.0e38f);
  if (cluster > 1) ptx::cluster_sync_all();  // every block of the cluster runs: its memory may be written
  else __syncthreads();

  // Hands every block what each warp of the cluster holds and returns the whole; the same numbers in the same order everywhere.
  auto exchange = [&](Part mine) -> Part {
    Part* to = &gather[turn][rank * kVerWarps + warp];
    if (lane < cluster) {
      if (cluster > 1) {
        const long long bits = __double_as_longlong(mine.sum);
        ptx::st_cluster_v4(ptx::map_to_cta(ptx::smem_u32(to), lane), __float_as_uint(mine.top), (uint32_t)mine.at, (uint32_t)bits, (uint32_t)(bits >> 32));
      } else {
        *to = mine;
      }
    }
    __syncwarp();
    if (cluster > 1) ptx::cluster_sync_all();
    else __syncthreads();
    Part all{-INFINITY, 0x7fffffff, 0.0};
    for (int i = lane; i < cluster * kVerWarps; i += 32) {
      const Part x = gather[turn][i];
      if (x.top > all.top || (x.top == all.top && x.at < all.at)) all.top = x.top, all.at = x.at;
    }
#pragma unroll
    for (int o = 16; o > 0; o /= 2) {
      const float top = __shfl_xor_sync(0xffffffffu, all.top, o);
      const int at = __shfl_xor_sync(0xffffffffu, all.at, o);
      if (top > all.top || (top == all.top && at < all.at)) all.top = top, all.at = at;
    }
    // sums of exponentials relative to each part's own largest logit
    double sum = 0.0;
    for (int i = lane; i < cluster * kVerWarps; i += 32) {
      const Part x = gather[turn][i];
      sum += greedy || x.top == all.top ? x.sum : x.sum * (double)exp2f((x.top - all.top) * per_t_log2);
    }
#pragma unroll
    for (int o = 16; o > 0; o /= 2) sum += __shfl_xor_sync(0xffffffffu, sum, o);
    all.sum = sum;
    turn ^= 1;
    return all;
  };

  const float* q_row = nullptr;
  int kept = n > 0 ? 1 : 0, cur = 0;
  int next = -1;          // the token that follows the path
  bool draws = false;     // it is drawn from what is left of p
  Part row{};             // largest logit and sum of the row `cur`
  double whole = 0.0;     // its sum in float64, once something needs it (0: not yet)
  int n_cut = 0;          // refusals that changed p: sums in `inverse` (drawn drafts) or tokens in `refused`
  double gone = 0.0;      // probability of the refused tokens (drafts that were not drawn)
  int have = -1;          // tile_sum holds the sums of p after this many refusals
  double have_total = 0.0;

  // p's weight at an element, after `cuts` refusals; unnormalised by the last of them
  auto weight = [&](float y, int v, float q, int cuts) -> double {
    double r = exp(((double)y - (double)row.top) * per_t);
    if (y == row.top) r = 1.0;
    if (q_row == nullptr) {
      for (int i = 0; i < cuts; ++i)
        if (refused[i] == v) r = 0.0;
    } else if (cuts > 0) {
      r *= 1.0 / whole;
      for (int i = 0; i < cuts; ++i) {
        const double d = r - (double)q;
        r = d > 0.0 ? d : 0.0;
        if (i + 1 < cuts) r *= inverse[i];
      }
    }
    return r;
  };

  // One float64 pass over the row: sums of runs of 32 `sub` pieces in tile_sum, the whole returned.
  auto slice = [&](const LogitRow<T>& x, int& sub, int& first, int& tiles) {
    const int share = (x.pieces + cluster - 1) / cluster;
    sub = (share + 32 * kVerTiles - 1) / (32 * kVerTiles);
    tiles = (share + 32 * sub - 1) / (32 * sub);
    first = rank * tiles * 32 * sub;
  };
  auto weights_of = [&](const LogitRow<T>& x, int i, int cuts, double (&w)[kVec]) {
    float y[kVec];
    x.load(i, y);
    const int v = x.first(i);
#pragma unroll
    for (int e = 0; e < kVec; ++e) {
      const bool in = i < x.pieces && v + e >= 0 && v + e < p.vocab;
      const float q = in && cuts > 0 && q_row != nullptr ? __ldg(q_row + v + e) : 0.f;
      w[e] = in ? weight(y[e], v + e, q, cuts) : 0.0;
    }
  };
  auto sum_pass = [&](const LogitRow<T>& x, int cuts) -> double {
    int sub, first, tiles;
    slice(x, sub, first, tiles);
    double mine = 0.0;
    for (int k = warp; k < tiles; k += kVerWarps) {
      double sum = 0.0;
      for (int u = 0; u < sub; ++u) {
        double w[kVec];
        weights_of(x, first + (k * sub + u) * 32 + lane, cuts, w);
#pragma unroll
        for (int e = 0; e < kVec; ++e) sum += w[e];
      }
#pragma unroll
      for (int o = 16; o > 0; o /= 2) sum += __shfl_xor_sync(0xffffffffu, sum, o);
      if (lane == 0) tile_sum[k] = sum;
      mine += sum;
    }
    have = cuts;
    have_total = exchange(Part{0.f, 0, mine}).sum;
    return have_total;
  };
  auto row_at = [&](int i) { return LogitRow<T>(reinterpret_cast<const T*>(p.logits) + (long)(row0 + i) * p.ld, p.vocab); };

  while (kept > 0) {
    // ---- the row's largest logit and sum of exponentials
    const LogitRow<T> x = row_at(cur);
    q_row = p.draft ? p.draft + (long)(row0 + cur) * p.draft_ld : nullptr;
    float top = -INFINITY, sum = 0.f;
    int at = 0x7fffffff;
    bool odd = false;  // a NaN
    const int share = (x.pieces + cluster - 1) / cluster, stop = min(x.pieces, (rank + 1) * share);
    constexpr int kAhead = 4;
    for (int i0 = rank * share + tid; i0 < stop; i0 += kAhead * kVerThreads) {
      float y[kAhead][kVec];
#pragma unroll
      for (int a = 0; a < kAhead; ++a) x.load(i0 + a * kVerThreads < stop ? i0 + a * kVerThreads : x.pieces, y[a]);
      float high = top;
#pragma unroll
      for (int a = 0; a < kAhead; ++a)
#pragma unroll
        for (int e = 0; e < kVec; ++e) {
          if (y[a][e] > high) {
            high = y[a][e];
            at = x.first(i0 + a * kVerThreads) + e;
          }
          odd |= y[a][e] != y[a][e];
        }
      if (!greedy && high > -INFINITY) {
        sum *= top == high ? 1.f : exp2f((top - high) * per_t_log2);
#pragma unroll
        for (int a = 0; a < kAhead; ++a)
#pragma unroll
          for (int e = 0; e < kVec; ++e) sum += ptx::ex2_approx((y[a][e] - high) * per_t_log2);
      }
      top = high;
    }
    float high = top;
    int place = at;
#pragma unroll
    for (int o = 16; o > 0; o /= 2) {
      const float h = __shfl_xor_sync(0xffffffffu, high, o);
      const int a = __shfl_xor_sync(0xffffffffu, place, o);
      if (h > high || (h == high && a < place)) high = h, place = a;
    }
    double wide = greedy || top == high ? (double)sum : (double)(sum * exp2f((top - high) * per_t_log2));
#pragma unroll
    for (int o = 16; o > 0; o /= 2) wide += __shfl_xor_sync(0xffffffffu, wide, o);
    if (__any_sync(0xffffffffu, odd)) wide = __longlong_as_double(0x7ff8000000000000ll);
    row = exchange(Part{high, place, wide});
    if (row.at >= p.vocab) row.at = 0;  // (nothing but -infinity)
    whole = gone = 0.0;
    n_cut = 0;
    have = -1;
    if (!(row.top > -INFINITY && row.top < INFINITY) || row.sum != row.sum) break;  // no distribution: nothing follows

    // ---- its children, in row order
    int taken = -1;
    for (int base = (cur + 1) & ~31; base < n && taken < 0; base += 32) {
      unsigned who = __ballot_sync(0xffffffffu, base + lane < n && base + lane > cur && parent[base + lane] == cur);
      while (who != 0 && taken < 0) {
        const int i = base + __ffs(who) - 1, v = token[i];
        who &= who - 1;
        if (greedy) {
          if (v == row.at) taken = i;
          continue;
        }
        const float y = VecOf<T>::one(x.x + v);
        double e = y == row.top ? 1.0 : exp(((double)y - (double)row.top) * per_t);
        if (q_row == nullptr) {
          for (int j = 0; j < n_cut; ++j)
            if (refused[j] == v) e = 0.0;
          const double share_v = e / row.sum;
          if ((double)chance[i] * (1.0 - gone) < share_v) {
            taken = i;
          } else if (share_v > 0.0 && 1.0 - gone - share_v > 0.0) {
            __syncthreads();  // all warps have read the list
            if (tid == 0) refused[n_cut] = v;
            __syncthreads();
            ++n_cut;
            gone += share_v;
          }
        } else {
          const float qv = __ldg(q_row + v);
          double r = n_cut == 0 ? e / row.sum : e * (1.0 / whole);
          for (int j = 0; j < n_cut; ++j) r = (r - (double)qv > 0.0 ? r - (double)qv : 0.0) * inverse[j];
          if ((double)chance[i] * (double)qv < r) {
            taken = i;
          } else {
            if (whole == 0.0) whole = sum_pass(x, 0);
            const double left = sum_pass(x, n_cut + 1);
            if (left > 0.0) {
              if (tid == 0) inverse[n_cut] = 1.0 / left;
              __syncthreads();
              ++n_cut;
            }
          }
        }
      }
    }
    if (taken < 0) {
      if (greedy) next = row.at;
      else draws = true;
      break;
    }
    if (rank == 0 && tid == 0) {
      p.path[(long)s * p.max_rows + kept] = taken;
      p.out_tokens[(long)s * p.max_rows + kept - 1] = token[taken];
    }
    cur = taken;
    ++kept;
  }

  // ---- the token behind the path
  if (draws) {
    const LogitRow<T> x = row_at(cur);
    if (have != n_cut) sum_pass(x, n_cut);
    if (!(have_total > 0.0) && n_cut > 0) sum_pass(x, n_cut = 0);
    const double target = (double)__ldg(p.sample_u + s) * have_total;
    // the block whose run of the vocabulary holds the target (behind all: the last with any weight)
    const Part* parts = gather[turn ^ 1];
    double before = 0.0, at_owner = 0.0;
    int owner = 0;
    bool found = false;
    for (int r = 0; r < cluster && !found; ++r) {
      double sum = 0.0;
      for (int w = 0; w < kVerWarps; ++w) sum += parts[r * kVerWarps + w].sum;
      if (sum > 0.0) owner = r, at_owner = before;
      before += sum;
      found = sum > 0.0 && before > target;
    }
    if (owner == rank && warp == 0) {
      int sub, first, tiles;
      slice(x, sub, first, tiles);
      const double want = target - at_owner;
      const int each = (tiles + 31) / 32, k0 = min(tiles, lane * each), k1 = min(tiles, k0 + each);
      double sum = 0.0;
      for (int k = k0; k < k1; ++k) sum += tile_sum[k];
      double run = sum;
#pragma unroll
      for (int o = 1; o < 32; o *= 2) {
        const double up = __shfl_up_sync(0xffffffffu, run, o);
        if (lane >= o) run += up;
      }
      run -= sum;
      // the first run of pieces whose end lies behind the target, else the last that has any weight
      int k_hit = -1, k_last = -1;
      double hit_before = 0.0, last_before = 0.0;
      for (int k = k0; k < k1; ++k) {
        const double y = tile_sum[k];
        if (y > 0.0) {
          k_last = k, last_before = run;
          if (k_hit < 0 && run + y > want) k_hit = k, hit_before = run;
        }
        run += y;
      }
      const unsigned hit = __ballot_sync(0xffffffffu, k_hit >= 0), any = __ballot_sync(0xffffffffu, k_last >= 0);
      const int from = hit ? __ffs(hit) - 1 : 31 - __clz(any | 1);
      const int k = __shfl_sync(0xffffffffu, hit ? k_hit : k_last, from);
      double done = __shfl_sync(0xffffffffu, hit ? hit_before : last_before, from);
      int best = -1, last = -1;
      for (int u = 0; k >= 0 && u < sub && best < 0; ++u) {
        const int i = first + (k * sub + u) * 32 + lane;
        double w[kVec], mine = 0.0;
        weights_of(x, i, n_cut, w);
#pragma unroll
        for (int e = 0; e < kVec; ++e) mine += w[e];
        double up_to = mine;
#pragma unroll
        for (int o = 1; o < 32; o *= 2) {
          const double up = __shfl_up_sync(0xffffffffu, up_to, o);
          if (lane >= o) up_to += up;
        }
        double here = done + (up_to - mine);
        int mine_hit = -1, mine_last = -1;
#pragma unroll
        for (int e = 0; e < kVec; ++e) {
          here += w[e];
          if (w[e] > 0.0) {
            mine_last = x.first(i) + e;
            if (mine_hit < 0 && here > want) mine_hit = x.first(i) + e;
          }
        }
        const unsigned h = __ballot_sync(0xffffffffu, mine_hit >= 0), l = __ballot_sync(0xffffffffu, mine_last >= 0);
        if (h) best = __shfl_sync(0xffffffffu, mine_hit, __ffs(h) - 1);
        if (l) last = __shfl_sync(0xffffffffu, mine_last, 31 - __clz(l));
        done += __shfl_sync(0xffffffffu, up_to, 31);
      }
      if (lane == 0) p.out_tokens[(long)s * p.max_rows + kept - 1] = best >= 0 ? best : last;
    }
  }
  if (rank == 0) {
    if (tid == 0) {
      p.kept[s] = kept;
      if (kept > 0) {
        p.path[(long)s * p.max_rows] = 0;
        if (!draws) p.out_tokens[(long)s * p.max_rows + kept - 1] = next;
      }
    }
    for (int i = kept + tid; i < p.max_rows; i += kVerThreads) {
      p.path[(long)s * p.max_rows + i] = -1;
      p.out_tokens[(long)s * p.max_rows + i] = -1;
    }
  }
}

// ---------------------------------------------------------------------------------------------
// Commit.  Row path[i] of a sequence's batch rows becomes row i, in every layer's keys and values: a move towards the
// front, so that one thread that takes 16 bytes of every row in turn (eight in flight) can do it in place.
constexpr int kCommitThreads = 256;

__device__ __forceinline__ int committed(const CommitPlan& p, int s, int start, int* problems) {
  const int kept = __ldg(p.kept + s);
  if (kept < 0 || (p.path != nullptr && kept > p.path_stride) || start < 0 || start > 0x7fffffff - max(kept, 0)) {
    *problems |= kBadRows;
    return 0;
  }
  return kept;
}

template <typename U>
__device__ __forceinline__ void move_rows(char* base, int each, const uint32_t* from, const uint32_t* to, int n) {
  for (int i0 = 0; i0 < n; i0 += 8) {
    U u[8];
#pragma unroll
    for (int i = 0; i < 8; ++i)
      if (i0 + i < n) u[i] = *reinterpret_cast<const U*>(base + (long)from[i0 + i] * each);
#pragma unroll
    for (int i = 0; i < 8; ++i)
      if (i0 + i < n) *reinterpret_cast<U*>(base + (long)to[i0 + i] * each) = u[i];
  }
}

__global__ void __launch_bounds__(kCommitThreads) draft_commit_kernel(const __grid_constant__ CommitPlan p) {
  __shared__ uint32_t from[kMaxDrafts], to[kMaxDrafts];  // vectors of head 0
  __shared__ int n_moves;
  const int s = (int)blockIdx.y, tid = threadIdx.x, lane = tid & 31;
  int problems = 0;
  const int start = __ldg(p.start + s), kept = committed(p, s, start, &problems);
  if (p.lengths != nullptr && blockIdx.x == 0 && tid == 0) p.lengths[s] = start + kept;
  if (tid < 32) {  // the moves, in order
    const int* path = p.path + (long)s * p.path_stride;
    int n = 0;
    for (int i0 = 0; i0 < kept; i0 += 32) {
      const int i = i0 + lane;
      bool moves = false;
      uint32_t src = 0, dst = 0;
      if (i < kept) {
        const int row = __ldg(path + i), last = i > 0 ? __ldg(path + i - 1) : -1;
        if (row < i || row <= last) {
          problems |= kBadParent;
        } else if (row != i) {
          const long a = (long)start + row, b = (long)start + i;
          const int mask = (1 << p.page_shift) - 1;
          if ((a >> p.page_shift) >= p.table_stride) {
            problems |= kBadRows;
          } else {
            const int* table = p.page_table + (long)s * p.table_stride;
            const int pa = __ldg(table + (a >> p.page_shift)), pb = __ldg(table + (b >> p.page_shift));
            if (pa < 0 || pa >= p.n_pages || pb < 0 || pb >= p.n_pages) {
              problems |= kBadPage;
            } else {
              moves = true;
              src = (((uint32_t)pa * (uint32_t)p.n_kv_head) << p.page_shift) + (uint32_t)(a & mask);
              dst = (((uint32_t)pb * (uint32_t)p.n_kv_head) << p.page_shift) + (uint32_t)(b & mask);
            }
          }
        }
      }
      const unsigned who = __ballot_sync(0xffffffffu, moves);
      if (moves) {
        const int k = n + __popc(who & ((1u << lane) - 1));
        from[k] = src;
        to[k] = dst;
      }
      n += __popc(who);
    }
    if (lane == 0) n_moves = n;
  }
  if (problems != 0 && blockIdx.x == 0) report(p.status, problems);
  __syncthreads();
  const int n = n_moves;
  if (n == 0) return;
  const int units = p.n_kv_head * p.vec_units, per_item = units + (p.item[0].scale ? p.n_kv_head : 0);
  const long flat = (long)blockIdx.x * kCommitThreads + tid;
  const int item = (int)(flat / per_item), unit = (int)(flat % per_item);
  if (item >= p.n_items) return;
  const CommitItem& it = p.item[item];
  if (unit < units) {
    const long head = unit / p.vec_units, within = unit % p.vec_units;
    move_rows<uint4>(it.ptr + ((head << p.page_shift) * p.vec_units + within) * 16, p.vec_units * 16, from, to, n);
  } else {
    move_rows<unsigned short>(reinterpret_cast<char*>(it.scale + ((long)(unit - units) << p.page_shift)), 2, from, to, n);
  }
}

__global__ void draft_lengths_kernel(const __grid_constant__ CommitPlan p) {
  const int s = (int)(blockIdx.x * blockDim.x + threadIdx.x);
  if (s >= p.n_seq) return;
  int problems = 0;
  const int start = p.start[s];
  p.lengths[s] = start + committed(p, s, start, &problems);
  if (problems != 0) report(p.status, problems);
}

}  // namespace

cudaError_t launch_draft_verify(const DraftVerifyParams& p, int dtype, int num_sms, cudaStream_t s) {
  // up to two blocks on every SM, at least a 16-byte piece of a row for every thread
  const int piece = dtype == WF_BF16 ? VecOf<__nv_bfloat16>::n : VecOf<float>::n;
  int cluster = 1;
  while (cluster < kMaxCluster && (long)p.n_seq * cluster <= num_sms && p.vocab > cluster * kVerThreads * piece) cluster *= 2;
  auto kernel = dtype == WF_BF16 ? draft_verify_kernel<__nv_bfloat16> : draft_verify_kernel<float>;
  return launch_dependent(kernel, dim3((unsigned)(p.n_seq * cluster)), dim3(kVerThreads), 0, s, cluster, false, p, cluster);
}

cudaError_t launch_draft_commit(const CommitPlan& p, cudaStream_t s) {
  const long threads = (long)p.n_items * (p.n_kv_head * p.vec_units + (p.n_items > 0 && p.item[0].scale ? p.n_kv_head : 0));
  const dim3 grid((unsigned)((threads + kCommitThreads - 1) / kCommitThreads), (unsigned)p.n_seq);
  return launch_dependent(draft_commit_kernel, grid, dim3(kCommitThreads), 0, s, 1, false, p);
}

cudaError_t launch_draft_lengths(const CommitPlan& p, cudaStream_t s) {
  return launch_dependent(draft_lengths_kernel, dim3((unsigned)((p.n_seq + 255) / 256)), dim3(256), 0, s, 1, false, p);
}

}  // namespace wf
