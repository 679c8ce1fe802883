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
// the same numbers.  Rows off the path are not read.  The sums that decide are float64, exponentials included: a
// vocabulary's running sum has steps of 1e-6 or less, so in float32 the token would depend on the order of summation, and after refusals
// what is left of p may be small beside what it is taken from.  A first child is weighed against the row's sum in float32,
// which the first pass makes beside the largest logit; where that sum's error could decide (1e-5 of all cases), against one in float64.
#include <math.h>

#include "wf_decoder.h"
#include "wf_ptx.cuh"

namespace wf {
namespace {

constexpr int kVerThreads = 512;
constexpr int kVerWarps = kVerThreads / 32;
constexpr int kAhead = 4;  // 16-byte pieces of a row that a thread has in flight
constexpr int kMaxCluster = 8;
constexpr int kRowBytes = 24;  // shared memory for a row of the sequence
constexpr int kHoldBytes = 216 * 1024;  // shared memory that a block may ask for

template <typename T>
struct VecOf;
template <>
struct VecOf<float> {
  static constexpr int n = 4;
  static __device__ __forceinline__ void unpack(uint4 u, float (&y)[n]) {
    y[0] = __uint_as_float(u.x), y[1] = __uint_as_float(u.y), y[2] = __uint_as_float(u.z), y[3] = __uint_as_float(u.w);
  }
  static __device__ __forceinline__ float one(const float* x) { return __ldg(x); }
  static constexpr uint32_t nothing = 0xff800000u;  // -infinity
  static __device__ __forceinline__ void put(uint32_t (&w)[4], int e, const float* x) { w[e] = __float_as_uint(*x); }
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
  static constexpr uint32_t nothing = 0xff80ff80u;
  static __device__ __forceinline__ void put(uint32_t (&w)[4], int e, const __nv_bfloat16* x) {
    const uint32_t h = __bfloat16_as_ushort(*x);
    w[e >> 1] = e & 1 ? (w[e >> 1] & 0xffffu) | h << 16 : (w[e >> 1] & 0xffff0000u) | h;
  }
};

// Elements v .. of a row, those outside it -infinity (its first and last piece: kept out of line, the kernel's code is fetched anew
// by every launch, and its size shows in the time of a small one).
template <typename T>
__device__ __noinline__ uint4 partial_piece(const T* x, int vocab, int v) {
  uint32_t w[4];
#pragma unroll
  for (int e = 0; e < 4; ++e) w[e] = VecOf<T>::nothing;
#pragma unroll
  for (int e = 0; e < VecOf<T>::n; ++e)
    if (v + e >= 0 && v + e < vocab) VecOf<T>::put(w, e, x + v + e);
  return make_uint4(w[0], w[1], w[2], w[3]);
}

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
  __device__ __forceinline__ uint4 load(int i) const {
    const int v = first(i);
    if (i < pieces && v >= 0 && v <= vocab - VecOf<T>::n) return __ldg(reinterpret_cast<const uint4*>(x + v));
    return i < pieces ? partial_piece(x, vocab, v) : make_uint4(VecOf<T>::nothing, VecOf<T>::nothing, VecOf<T>::nothing, VecOf<T>::nothing);
  }
};

// What blocks and warps tell each other about a pass: the largest logit, its first place, and a sum.
struct __align__(16) Part {
  float top;
  int at;
  double sum;
};

// 2^(z / 64) for z <= 0 to some 1e-15: 2^(j / 64) from a table (z's nearest whole number is 64 i + j), the rest, at most half a
// 64th, by the exponential series to the fifth power.  Eleven float64 operations where exp() takes about three times as many; the
// draws are bound by them.
// z below -64000 gives no number: the caller takes 0 there.
constexpr double kLn2By64 = 0.010830424696249145;
__constant__ double kSeries[6] = {kLn2By64,
                                  kLn2By64 * kLn2By64 / 2.0,
                                  kLn2By64 * kLn2By64 * kLn2By64 / 6.0,
                                  kLn2By64 * kLn2By64 * kLn2By64 * kLn2By64 / 24.0,
                                  kLn2By64 * kLn2By64 * kLn2By64 * kLn2By64 * kLn2By64 / 120.0,
                                  6755399441055744.0};  // 1.5 * 2^52: a sum with it is rounded to a whole number
__device__ __forceinline__ double exp2_64th(double z, const double* table) {
  const double sum = z + kSeries[5], f = z - (sum - kSeries[5]);
  const int k = __double2loint(sum);
  double q = fma(f, kSeries[4], kSeries[3]);
  q = fma(f, q, kSeries[2]);
  q = fma(f, q, kSeries[1]);
  q = fma(f, q, kSeries[0]) * f;
  const double t = table[k & 63], r = fma(t, q, t);
  return __hiloint2double(__double2hiint(r) + ((k >> 6) << 20), __double2loint(r));
}

// exp(x / T)'s parts of a power of two: 2^((y - top) per_t / 64), in float64.
__device__ __forceinline__ double power_of(float y, double top, double per_t, const double* table) {
  const double z = ((double)y - top) * per_t, r = exp2_64th(z, table);
  return z > -64000.0 ? r : 0.0;
}

// A row's sum in float64 without some tokens, handed to all blocks by way of `sums`: for the few cases in which the float32 sum's
// error could decide.  Out of line and plain: once in 1e5 rows, and the kernel's registers are short.
template <typename T>
__device__ __noinline__ double exact_sum(const T* row, int vocab, double top, double per_t, const double* table, const int* refused, int n_refused, double* sums,
                                         int cluster) {
  const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5, rank = cluster > 1 ? (int)ptx::cluster_ctarank() : 0;
  double sum = 0.0;
  for (int v = rank * kVerThreads + (int)threadIdx.x; v < vocab; v += cluster * kVerThreads) {
    double w = power_of(VecOf<T>::one(row + v), top, per_t, table);
    for (int j = 0; j < n_refused; ++j)
      if (refused[j] == v) w = 0.0;
    sum += w;
  }
  for (int o = 16; o > 0; o /= 2) sum += __shfl_xor_sync(0xffffffffu, sum, o);
  double* to = sums + rank * kVerWarps + warp;
  if (cluster == 1) {
    if (lane == 0) *to = sum;
    __syncthreads();
  } else {
    const long long bits = __double_as_longlong(sum);
    if (lane < cluster) ptx::st_cluster_v2(ptx::map_to_cta(ptx::smem_u32(to), lane), (uint32_t)bits, (uint32_t)(bits >> 32));
    __syncwarp();
    ptx::cluster_sync_all();
  }
  sum = 0.0;
  for (int i = lane; i < cluster * kVerWarps; i += 32) sum += sums[i];
  for (int o = 16; o > 0; o /= 2) sum += __shfl_xor_sync(0xffffffffu, sum, o);
  return sum;
}

// kHold: the block keeps its part of p in shared memory (`hold`), so that a refusal costs a subtraction for each element and
// not an exponential; vocabularies whose part does not fit are computed anew.
template <typename T, bool kHold>
__global__ void __launch_bounds__(kVerThreads, 2) draft_verify_kernel(const __grid_constant__ DraftVerifyParams p, int cluster, int hold_length) {
  constexpr int kVec = VecOf<T>::n;
  extern __shared__ __align__(16) double dynamic[];
  __shared__ Part gather[2][kMaxCluster * kVerWarps];
  __shared__ double table[64];
  __shared__ float bound[kVerWarps];  // of the error of a row's float32 sum, each warp's own copy (a register fewer)
  double* inverse = dynamic;                                   // of the sums left after each refusal at the present row
  int* token = reinterpret_cast<int*>(dynamic + p.max_rows);
  int* parent = token + p.max_rows;
  float* chance = reinterpret_cast<float*>(parent + p.max_rows);
  int* refused = reinterpret_cast<int*>(chance + p.max_rows);  // tokens that were not drawn and not taken at the present row
  double* hold = dynamic + kRowBytes / 8 * p.max_rows;
  const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5;
  const int rank = cluster > 1 ? (int)ptx::cluster_ctarank() : 0;
  const int s = (int)blockIdx.x / cluster;
  int turn = 0;  // which of the two gather buffers the next exchange uses

  const int row0 = __ldg(p.cu_rows + s), end = __ldg(p.cu_rows + s + 1);
  const float t = p.temperature ? __ldg(p.temperature + s) : 1.f, draw = __ldg(p.sample_u + s);
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
  if (tid < 64) table[tid] = exp2((double)tid / 64.0);
  if (n > 0 && !(t >= 0.f && t < INFINITY)) {
    problems |= kBadValue;
    n = 0;
  }
  if (problems != 0) report(p.status, problems);
  const bool greedy = t == 0.f;
  const double per_t = greedy ? 0.0 : 64.0 * 1.4426950408889634 / (double)t;  // exp(x / T) = 2^(x per_t / 64)
  // (a temperature near the smallest float must not make 0 x infinity of the largest logit)
  const float per_t_log2 = greedy ? 0.f : fminf((float)(per_t / 64.0), 3.0e38f);
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
    Part all{-INFINITY, 0x7fffffff, 0.0}, part[kMaxCluster * kVerWarps / 32];
#pragma unroll
    for (int i = 0; i < kMaxCluster * kVerWarps / 32; ++i) {
      part[i] = Part{-INFINITY, 0x7fffffff, 0.0};
      if (i * 32 + lane < cluster * kVerWarps) part[i] = gather[turn][i * 32 + lane];
      if (part[i].top > all.top || (part[i].top == all.top && part[i].at < all.at)) all.top = part[i].top, all.at = part[i].at;
    }
#pragma unroll
    for (int o = 16; o > 0; o /= 2) {
      const float top = __shfl_xor_sync(0xffffffffu, all.top, o);
      const int at = __shfl_xor_sync(0xffffffffu, all.at, o);
      if (top > all.top || (top == all.top && at < all.at)) all.top = top, all.at = at;
    }
    // sums of exponentials relative to each part's own largest logit
#pragma unroll
    for (int i = 0; i < kMaxCluster * kVerWarps / 32; ++i)
      all.sum += greedy || part[i].top == all.top ? part[i].sum : part[i].sum * (double)exp2f((part[i].top - all.top) * per_t_log2);
#pragma unroll
    for (int o = 16; o > 0; o /= 2) all.sum += __shfl_xor_sync(0xffffffffu, all.sum, o);
    turn ^= 1;
    return all;
  };

  // The same for a sum alone: each warp's goes to gather's memory as doubles, in the order of the warps.
  auto exchange_sum = [&](double mine) -> double {
    double* sums = reinterpret_cast<double*>(gather[turn]);
    if (lane < cluster) {
      if (cluster > 1) {
        const long long bits = __double_as_longlong(mine);
        ptx::st_cluster_v2(ptx::map_to_cta(ptx::smem_u32(sums + rank * kVerWarps + warp), lane), (uint32_t)bits, (uint32_t)(bits >> 32));
      } else {
        sums[warp] = mine;
      }
    }
    __syncwarp();
    if (cluster > 1) ptx::cluster_sync_all();
    else __syncthreads();
    double all = 0.0;
#pragma unroll
    for (int i = 0; i < kMaxCluster * kVerWarps / 32; ++i)
      if (i * 32 + lane < cluster * kVerWarps) all += sums[i * 32 + lane];
#pragma unroll
    for (int o = 16; o > 0; o /= 2) all += __shfl_xor_sync(0xffffffffu, all, o);
    turn ^= 1;
    return all;
  };

  const float* q_row = nullptr;
  int kept = n > 0 ? 1 : 0, cur = 0;
  int next = -1;          // the token that follows the path
  bool draws = false;     // it is drawn from what is left of p
  Part row{};             // largest logit and sum of the row `cur`
  double whole = 0.0;     // its sum (of drafts that were not drawn: without those refused), in float64 once something needs that
  int n_cut = 0;          // refusals that changed p: sums in `inverse` (drawn drafts) or tokens in `refused`
  int have = -1;          // the last pass (and hold) has p after this many refusals, not divided by the last one's sum; -1: no sum in float64 at this row
                          // so far, -2: none that can be gone on from
  double have_total = 0.0;

  auto row_at = [&](int i) { return LogitRow<T>(reinterpret_cast<const T*>(p.logits) + (long)(row0 + i) * p.ld, p.vocab); };
  double top64 = 0.0;     // row.top
  auto power = [&](float y) { return power_of(y, top64, per_t, table); };
  // A row is cut into runs of 32 `length` pieces, one for every warp of the cluster, in order.
  const int runs = cluster * kVerWarps;
  auto run_length = [&](const LogitRow<T>& x) { return (x.pieces + runs * 32 - 1) / (runs * 32); };
  // p's weights at the elements of piece i, after `cuts` refusals
  auto weights_of = [&](const LogitRow<T>& x, int i, uint4 raw, int cuts, double (&w)[kVec]) {
    float y[kVec];
    VecOf<T>::unpack(raw, y);
    const int v = x.first(i);
    float q[kVec];
#pragma unroll
    for (int e = 0; e < kVec; ++e) q[e] = cuts > 0 && q_row != nullptr && i < x.pieces && v + e >= 0 && v + e < p.vocab ? __ldg(q_row + v + e) : 0.f;
#pragma unroll
    for (int e = 0; e < kVec; ++e) w[e] = power(y[e]);  // (what lies outside the row is -infinity)
    if (cuts == 0) return;
    if (q_row == nullptr) {
#pragma unroll 1
      for (int c = 0; c < cuts; ++c)
#pragma unroll
        for (int e = 0; e < kVec; ++e)
          if (refused[c] == v + e) w[e] = 0.0;
      return;
    }
#pragma unroll
    for (int e = 0; e < kVec; ++e) w[e] *= 1.0 / whole;
#pragma unroll 1
    for (int c = 0; c < cuts; ++c)
#pragma unroll
      for (int e = 0; e < kVec; ++e) {
        w[e] = fmax(w[e] - (double)q[e], 0.0);
        if (c + 1 < cuts) w[e] *= inverse[c];
      }
  };
  auto held = [&](int u, int e) -> double& { return hold[((warp * hold_length + u) * 32 + lane) * kVec + (e ^ (lane & (kVec - 1)))]; };
  // One pass over the row; returns the whole.  `on`: from what is held, one refusal further.
  auto sum_pass = [&](const LogitRow<T>& x, int cuts, bool on) -> double {
    const int length = run_length(x), first = (rank * kVerWarps + warp) * length * 32 + lane;
    double sum = 0.0;
    if (kHold && on) {
      const double factor = cuts == 1 ? 1.0 / whole : inverse[cuts - 2];
#pragma unroll 1
      for (int u = 0; u < length; ++u) {
        const int i = first + u * 32, v = x.first(i);
        float q[kVec];
#pragma unroll
        for (int e = 0; e < kVec; ++e) q[e] = i < x.pieces && v + e >= 0 && v + e < p.vocab ? __ldg(q_row + v + e) : 0.f;
#pragma unroll
        for (int e = 0; e < kVec; ++e) {
          double& w = held(u, e);
          w = fmax(w * factor - (double)q[e], 0.0);
          sum += w;
        }
      }
    } else {
      uint4 raw = x.load(first);
#pragma unroll 1
      for (int u = 0; u < length; ++u) {
        const uint4 now = raw;
        if (u + 1 < length) raw = x.load(first + (u + 1) * 32);
        double w[kVec];
        weights_of(x, first + u * 32, now, cuts, w);
#pragma unroll
        for (int e = 0; e < kVec; ++e) {
          if (kHold) held(u, e) = w[e];
          sum += w[e];
        }
      }
    }
#pragma unroll
    for (int o = 16; o > 0; o /= 2) sum += __shfl_xor_sync(0xffffffffu, sum, o);
    have = cuts;
    have_total = exchange_sum(sum);
    return have_total;
  };
  // The first child of the present row behind row `after`, n if there is none.
  auto child_behind = [&](int after) {
    for (int base = (after + 1) & ~31; base < n; base += 32) {
      const unsigned who = __ballot_sync(0xffffffffu, base + lane < n && base + lane > after && parent[base + lane] == cur);
      if (who != 0) return base + __ffs(who) - 1;
    }
    return n;
  };

  while (kept > 0) {
    // ---- the row's largest logit and sum of exponentials; what its first child needs is on its way meanwhile
    const LogitRow<T> x = row_at(cur);
    q_row = p.draft ? p.draft + (long)(row0 + cur) * p.draft_ld : nullptr;
    int child = child_behind(cur);
    float child_y = 0.f, child_q = 0.f;
    auto look = [&]() {
      if (child >= n) return;
      child_y = VecOf<T>::one(x.x + token[child]);
      if (q_row != nullptr) child_q = __ldg(q_row + token[child]);
    };
    look();
    float top = -INFINITY, sum = 0.f;
    int at = 0x7fffffff;
    const int length = run_length(x), mine = (rank * kVerWarps + warp) * length * 32 + lane;
#pragma unroll 1
    for (int u0 = 0; u0 < length; u0 += kAhead) {
      uint4 raw[kAhead];
#pragma unroll
      for (int a = 0; a < kAhead; ++a) raw[a] = x.load(u0 + a < length ? mine + (u0 + a) * 32 : x.pieces);
      if (greedy) {
#pragma unroll
        for (int a = 0; a < kAhead; ++a) {
          if (u0 + a >= length) break;
          float y[kVec];
          VecOf<T>::unpack(raw[a], y);
#pragma unroll
          for (int e = 0; e < kVec; ++e) {
            if (y[e] > top) top = y[e], at = x.first(mine + (u0 + a) * 32) + e;
            sum += y[e] != y[e] ? y[e] : 0.f;  // a NaN shows
          }
        }
        continue;
      }
      float high = top;  // of all the pieces first: one rescaling, and no chain from piece to piece
#pragma unroll
      for (int a = 0; a < kAhead; ++a) {
        if (u0 + a >= length) break;
        float y[kVec];
        VecOf<T>::unpack(raw[a], y);
#pragma unroll
        for (int e = 0; e < kVec; ++e) high = fmaxf(high, y[e]);
      }
      if (high > top) sum *= exp2f((top - high) * per_t_log2);
      const float from = high > -INFINITY ? high : 0.f;  // (nothing but -infinity: no weight; a NaN shows)
      float part[kAhead];
#pragma unroll
      for (int a = 0; a < kAhead; ++a) {
        part[a] = 0.f;
        if (u0 + a >= length) continue;
        float y[kVec];
        VecOf<T>::unpack(raw[a], y);
#pragma unroll
        for (int e = 0; e < kVec; ++e) part[a] += ptx::ex2_approx((y[e] - from) * per_t_log2);
      }
#pragma unroll
      for (int a = 0; a < kAhead; ++a) sum += part[a];
      top = high;
    }
    // (as ordered integers: one instruction takes the largest of a warp; a sum with +0 makes -0 and +0 one number)
    const int bits = __float_as_int(top + 0.f), order = bits ^ ((bits >> 31) & 0x7fffffff), most = __reduce_max_sync(0xffffffffu, order);
    const float high = __int_as_float(most ^ ((most >> 31) & 0x7fffffff));
    const int place = greedy ? (int)__reduce_min_sync(0xffffffffu, (unsigned)(order == most ? at : 0x7fffffff)) : 0x7fffffff;
    float part = greedy || top == high ? sum : sum * exp2f((top - high) * per_t_log2);
#pragma unroll
    for (int o = 16; o > 0; o /= 2) part += __shfl_xor_sync(0xffffffffu, part, o);
    const double wide = (double)part;
    row = exchange(Part{high, place, wide});
    if (row.at >= p.vocab) row.at = 0;  // (nothing but -infinity)
    top64 = (double)row.top;
    whole = row.sum;
    n_cut = 0;
    have = -1;
    if (!(row.top > -INFINITY && row.top < INFINITY) || row.sum != row.sum) break;  // no distribution: nothing follows

    // ---- its children, in row order.  A draft is weighed against float32 sums where that is beyond doubt, and else against
    // sums in float64 (then a pass has been made).  The bound: an exponential's own error and its argument's (rounded thrice, and 28
    // binary digits are as much as a row's weights differ where they count), the additions of a lane and a warp.
    // (Temperatures above 2^100 give weight to logits that differ by more than float32 holds, and where 1 / T is more than float32
    // holds it has been cut: the sum says nothing then.)
    if (lane == 0) bound[warp] = per_t_log2 < 0x1p-100f || per_t_log2 >= 3.0e38f ? INFINITY : (float)whole * ((float)(96 + 4 * length) * (1.f / (1 << 23)));
    __syncwarp();
    int taken = -1;
    for (; child < n && taken < 0; child = child_behind(child), look()) {
      const int v = token[child];
      if (greedy) {
        if (v == row.at) taken = child;
        continue;
      }
      double e = power(child_y), against = (double)chance[child];
      if (q_row != nullptr) {
        against *= (double)child_q;
        if (n_cut > 0) {
          e *= 1.0 / whole;
          for (int j = 0; j < n_cut; ++j) e = fmax(e - (double)child_q, 0.0) * inverse[j];
        }
      } else {
        for (int j = 0; j < n_cut; ++j)
          if (refused[j] == v) e = 0.0;
      }
      if (q_row == nullptr || n_cut == 0) {
        if (have == -1 && fabs(against * whole - e) <= against * (double)bound[warp]) {
          whole = exact_sum<T>(x.x, p.vocab, top64, per_t, table, refused, q_row == nullptr ? n_cut : 0, reinterpret_cast<double*>(gather[turn]), cluster);
          turn ^= 1;
          have = -2;
        }
        against *= whole;
      }
      if (against < e) {
        taken = child;
        continue;
      }
      if (q_row == nullptr) {
        if (!(e > 0.0)) continue;  // (nothing is taken from p)
        __syncthreads();           // all warps have read the list
        if (tid == 0) refused[n_cut] = v;
        __syncthreads();
        // what is left by subtraction, while that says enough (in float64: halved sixteen times at most)
        if (have == -1 ? whole - e > 2.0 * (double)bound[warp] : e <= 0.5 * whole && n_cut - have < 16) {
          whole -= e;
          ++n_cut;
          continue;
        }
      }
      double left = 0.0;
#pragma unroll 1
      for (int step = q_row != nullptr && have < 0 ? 0 : 1; step < 2; ++step) {  // p itself first, where nothing has needed it so far
        left = sum_pass(x, step == 0 ? 0 : n_cut + 1, q_row != nullptr && step != 0 && have == n_cut);
        if (step == 0) whole = left;
      }
      if (left > 0.0) {
        if (q_row == nullptr) whole = left;
        if (tid == 0) inverse[n_cut] = 1.0 / left;
        __syncthreads();
        ++n_cut;
      } else if (q_row == nullptr) {  // the refusal does not count
        have = -2;
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
#pragma unroll 1
    while (have != n_cut || (n_cut > 0 && !(have_total > 0.0))) {  // (where the refusals leave nothing they do not count)
      if (have == n_cut) n_cut = 0;
      sum_pass(x, n_cut, false);
    }
    draws = have_total > 0.0;  // (always so: the largest logit's weight is 1)
    const double target = (double)draw * have_total;
    // the run that holds the target (behind all: the last with any weight); a lane looks at four of the at most 128
    static_assert(kMaxCluster * kVerWarps == 128, "four runs for each lane");
    const double* sums = reinterpret_cast<const double*>(gather[turn ^ 1]);
    double part[4], run = 0.0;
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      part[i] = 4 * lane + i < runs ? sums[4 * lane + i] : 0.0;
      run += part[i];
    }
    double before = run;
#pragma unroll
    for (int o = 1; o < 32; o *= 2) {
      const double up = __shfl_up_sync(0xffffffffu, before, o);
      if (lane >= o) before += up;
    }
    before -= run;
    int hit = -1, last = -1;
    double hit_before = 0.0, last_before = 0.0;
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      if (part[i] > 0.0) {
        last = 4 * lane + i, last_before = before;
        if (hit < 0 && before + part[i] > target) hit = 4 * lane + i, hit_before = before;
      }
      before += part[i];
    }
    const unsigned hits = __ballot_sync(0xffffffffu, hit >= 0), some = __ballot_sync(0xffffffffu, last >= 0);
    const int from = hits ? __ffs(hits) - 1 : 31 - __clz(some | 1);
    const int owner = __shfl_sync(0xffffffffu, hits ? hit : last, from);
    const double want = target - __shfl_sync(0xffffffffu, hits ? hit_before : last_before, from);
    if (draws && owner == rank * kVerWarps + warp) {
      // ---- its warp goes through it once more, up to the element
      const int length = run_length(x), first = owner * length * 32 + lane;
      double done = 0.0;
      int best = -1, best_last = -1;  // (where rounding has moved the target out of reach: the last element with any weight)
#pragma unroll 1
      for (int u = 0; u < length && best < 0; ++u) {
        const int i = first + u * 32;
        double w[kVec], mine = 0.0;
        if (kHold) {
#pragma unroll
          for (int e = 0; e < kVec; ++e) w[e] = held(u, e);
        } else {
          weights_of(x, i, x.load(i), n_cut, w);
        }
#pragma unroll
        for (int e = 0; e < kVec; ++e) mine += w[e];
        double up_to = mine;
#pragma unroll
        for (int o = 1; o < 32; o *= 2) {
          const double up = __shfl_up_sync(0xffffffffu, up_to, o);
          if (lane >= o) up_to += up;
        }
        double here = done + (up_to - mine);
        int e_hit = -1, e_last = -1;
#pragma unroll
        for (int e = 0; e < kVec; ++e) {
          here += w[e];
          if (w[e] > 0.0) {
            e_last = x.first(i) + e;
            if (e_hit < 0 && here > want) e_hit = e_last;
          }
        }
        const unsigned h = __ballot_sync(0xffffffffu, e_hit >= 0), l = __ballot_sync(0xffffffffu, e_last >= 0);
        if (h) best = __shfl_sync(0xffffffffu, e_hit, __ffs(h) - 1);
        if (l) best_last = __shfl_sync(0xffffffffu, e_last, 31 - __clz(l));
        done += __shfl_sync(0xffffffffu, up_to, 31);
      }
      if (lane == 0) p.out_tokens[(long)s * p.max_rows + kept - 1] = best >= 0 ? best : best_last;
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
// front, so that one thread that takes 16 bytes of every row in turn (eight in flight) can do it in place.  Bound by memory in
// pieces: a vector is 64 to 256 bytes of a head's run of positions, a scale two of its 32 (64 sequences, 38 MB: 18 us with
// vectors of 64 bytes and their scales, 11 us with 128 bytes and none; more or fewer moves per thread change nothing).
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
        } else {  // (a row that stays is looked up like one that moves, so that it is reported where it has no place)
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
              moves = row != i;
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
  const int start = p.start[s], kept = committed(p, s, start, &problems);
  if (kept > 0 && p.page_table != nullptr && (long)start + kept > (long)p.table_stride << p.page_shift) problems |= kBadRows;
  p.lengths[s] = start + kept;
  if (problems != 0) report(p.status, problems);
}

}  // namespace

cudaError_t launch_draft_verify(const DraftVerifyParams& p, int dtype, int num_sms, cudaStream_t s) {
  // up to two blocks on every SM, at least a 16-byte piece of a row for every thread
  const int piece = dtype == WF_BF16 ? VecOf<__nv_bfloat16>::n : VecOf<float>::n;
  int cluster = 1;
  while (cluster < kMaxCluster && (long)p.n_seq * cluster <= num_sms && p.vocab > cluster * kVerThreads * piece) cluster *= 2;
  // pieces of a run at any alignment of a row, and what a block holds of them
  const long pieces = ((long)p.vocab + 2 * piece - 2) / piece, per = (long)cluster * kVerWarps * 32, length = (pieces + per - 1) / per;
  const size_t rows = (size_t)p.max_rows * kRowBytes, part = (size_t)(length * kVerThreads * piece) * sizeof(double);
  // Held where it fits and pays: for drawn drafts, whose refusals go on from it, and where a block has its SM to itself, so that the
  // draw is read back and not computed again (one stream 20 -> 19 us; 64 streams of drafts that were not drawn 30 -> 36: not there).
  const bool hold = rows + part <= kHoldBytes && (p.draft != nullptr || (long)p.n_seq * cluster <= num_sms);
  auto kernel = dtype == WF_BF16 ? (hold ? draft_verify_kernel<__nv_bfloat16, true> : draft_verify_kernel<__nv_bfloat16, false>)
                                 : (hold ? draft_verify_kernel<float, true> : draft_verify_kernel<float, false>);
  const cudaError_t e = cudaFuncSetAttribute(kernel, cudaFuncAttributeMaxDynamicSharedMemorySize, kHoldBytes);
  if (e != cudaSuccess) return e;
  return launch_dependent(kernel, dim3((unsigned)(p.n_seq * cluster)), dim3(kVerThreads), rows + (hold ? part : 0), s, cluster, false, p, cluster, (int)length);
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
