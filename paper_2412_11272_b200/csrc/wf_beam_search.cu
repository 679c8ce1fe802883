// Device side of beam search: selection over beams and vocabulary, and reordering of the beams' states.
//
// Reordering, in place without a second buffer: a thread owns one unit (16 bytes where alignment allows) of a
// column, loads that unit of every parent that some other beam grew from, and stores only then.  Units of
// different threads do not meet, so no thread sees a half-moved state.  Bound by memory: a row that
// moves is written once and its parent read once (several children of one parent hit L1 / L2).
// Rows that stay (parent = itself) cost nothing.  345 MB of contiguous rows: 56 us, 6.2 TB/s read and written; the pages of 16 x 5
// beams in 12 layers (13.9 MB in runs of 512 to 960 bytes): 8.9 us.
#include "wf_decoder.h"
#include "wf_ptx.cuh"

namespace wf {

namespace {

// ---------------------------------------------------------------------------------------------
// Selection.  One cluster of blocks per sequence; a block has one slice of the vocabulary of all its beams, cut
// into items (one beam, up to `tiles` tiles) that its warps take in turn, loading the next tile while they work on
// one.  The pass over the logits only keeps, per lane, the maximum and the sum of exponentials: a lane's
// maximum stands for its 32 (float32: 16) elements of every tile.  Then
//   * the blocks exchange the beams' partial sums (through distributed shared memory) and know every log-sum;
//   * the keep-th largest of lane maxima, turned into scores, bounds the keep-th best score from below; only the few lanes
//     whose maximum reaches the bound can hold one of the best: their elements are read once more and ranked by
//     (score, index) in float64;
//   * the first block joins the blocks' lists.
// Where many elements tie at the bound, the lists overflow and the block picks its best one by one instead.  No workspace
// and one launch; sums are joined in a fixed order and a shared list's order decides nothing, so results are reproducible.
// Bound by the latency of its phases, one after another: 5 beams of 50,021 float32 logits 11.3 us (5 us of it the pass over the logits);
// 64 x 5 beams of bfloat16 logits 18.6 us (1.5 TB/s, half of the issue slots busy).

constexpr int kSelThreads = 512, kSelWarps = kSelThreads / 32;
constexpr int kMaxCluster = 8;
constexpr float kLog2e = 1.4426950408889634f;
constexpr int kVecs = 4;            // 16-byte vectors of a lane per tile
constexpr int kMaxGroups = 16;      // items of one beam in a block
constexpr int kLaneList = 1024;     // lanes that reach the first bound
constexpr int kCandidates = 512;    // elements that reach the second
constexpr int kFewLanes = 64;       // lanes that reach the second bound

// Order-preserving maps to unsigned integers above 0 (NaN excluded).
__device__ __forceinline__ uint32_t ordered(float x) {
  const uint32_t b = __float_as_uint(x + 0.f);  // -0 counts as 0
  return b & 0x80000000u ? ~b : b | 0x80000000u;
}
__device__ __forceinline__ float from_ordered(uint32_t k) { return __uint_as_float(k & 0x80000000u ? k & 0x7fffffffu : ~k); }
__device__ __forceinline__ uint64_t ordered(double x) {
  const uint64_t b = (uint64_t)__double_as_longlong(x + 0.0);
  return b >> 63 ? ~b : b | (1ull << 63);
}

struct __align__(16) Ranked {
  uint64_t key;   // ordered score; 0: none
  uint32_t flat;  // beam * vocab + token
  uint32_t pad;
  __device__ __forceinline__ bool before(const Ranked& o) const { return (key > o.key) | ((key == o.key) & (flat < o.flat)); }
};

// keep-th largest of the lanes' keys (0 if fewer lanes have one), by counting for every lane the keys before its own;
// `space`: 32 words of shared memory of the warp's own.
__device__ __forceinline__ uint32_t kth_lane_key(uint32_t key, int keep, uint32_t* space) {
  const int lane = threadIdx.x & 31;
  space[lane] = key;
  __syncwarp();
  int before = 0;
#pragma unroll
  for (int i = 0; i < 32; i += 4) {
    const uint4 k = *reinterpret_cast<const uint4*>(space + i);
    before += (k.x > key) | ((k.x == key) & (i < lane));
    before += (k.y > key) | ((k.y == key) & (i + 1 < lane));
    before += (k.z > key) | ((k.z == key) & (i + 2 < lane));
    before += (k.w > key) | ((k.w == key) & (i + 3 < lane));
  }
  __syncwarp();
  const unsigned who = __ballot_sync(0xffffffffu, before == keep - 1);  // one lane: the places are 0 .. 31
  return __shfl_sync(0xffffffffu, key, __ffs(who) - 1);
}

// The best of the lanes' entries, in every lane.
__device__ __forceinline__ Ranked warp_first(Ranked x) {
  const uint32_t h = __reduce_max_sync(0xffffffffu, (uint32_t)(x.key >> 32));
  const uint32_t l = __reduce_max_sync(0xffffffffu, (uint32_t)(x.key >> 32) == h ? (uint32_t)x.key : 0u);
  Ranked r;
  r.key = ((uint64_t)h << 32) | l;
  r.flat = __reduce_min_sync(0xffffffffu, x.key == r.key ? x.flat : 0xffffffffu);
  r.pad = 0;
  return r;
}

// Gives the best `keep` of n entries to out(rank, entry), by all threads of the block: every entry against all others.
template <typename Emit>
__device__ __forceinline__ void block_best(const Ranked* from, int n, int keep, Emit out) {
  for (int i = threadIdx.x; i < n; i += kSelThreads) {
    const Ranked x = from[i];
    if (x.key == 0) continue;
    int rank = 0;
#pragma unroll 8
    for (int j = 0; j < n; ++j) {
      const uint4 r = *reinterpret_cast<const uint4*>(from + j);  // one load, no branch
      rank += Ranked{((uint64_t)r.y << 32) | r.x, r.z, 0}.before(x);
    }
    if (rank < keep) out(rank, x);
  }
}

template <typename T>
struct Vec {  // 16 bytes of logits
  static constexpr int n = 16 / (int)sizeof(T);
  static constexpr int tile = kVecs * 32 * n;
  // largest element; NaN counts as nothing
  static __device__ __forceinline__ float max(const uint4& r) {
    if constexpr (sizeof(T) == 4) {
      return fmaxf(fmaxf(fmaxf(__uint_as_float(r.x), __uint_as_float(r.y)), fmaxf(__uint_as_float(r.z), __uint_as_float(r.w))), -INFINITY);
    } else {
      uint32_t a, b;
      asm("max.bf16x2 %0, %1, %2;" : "=r"(a) : "r"(r.x), "r"(r.y));
      asm("max.bf16x2 %0, %1, %2;" : "=r"(b) : "r"(r.z), "r"(r.w));
      asm("max.bf16x2 %0, %1, %2;" : "=r"(a) : "r"(a), "r"(b));
      return fmaxf(fmaxf(__uint_as_float(a << 16), __uint_as_float(a & 0xffff0000u)), -INFINITY);
    }
  }
  static __device__ __forceinline__ void unpack(const uint4& r, float* x) {
    const uint32_t w[4] = {r.x, r.y, r.z, r.w};
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      if constexpr (sizeof(T) == 4) {
        x[i] = __uint_as_float(w[i]);
      } else {
        x[2 * i] = __uint_as_float(w[i] << 16);
        x[2 * i + 1] = __uint_as_float(w[i] & 0xffff0000u);
      }
    }
  }
};
__device__ __forceinline__ uint32_t bits_of(float x) { return __float_as_uint(x); }
__device__ __forceinline__ uint32_t bits_of(__nv_bfloat16 x) { return (uint32_t)__bfloat16_as_ushort(x); }
template <typename T>
__device__ __forceinline__ T minus_infinity();
template <>
__device__ __forceinline__ float minus_infinity<float>() { return -INFINITY; }
template <>
__device__ __forceinline__ __nv_bfloat16 minus_infinity<__nv_bfloat16>() { return __ushort_as_bfloat16(0xff80); }
__device__ __forceinline__ float to_f32(float x) { return x; }
__device__ __forceinline__ float to_f32(__nv_bfloat16 x) { return __bfloat162float(x); }

__device__ __forceinline__ bool suppressed(const BeamSelectParams& p, int v) { return p.suppress && ((__ldg(p.suppress + (v >> 5)) >> (v & 31)) & 1); }

// Elements v .. v + n - 1 of a row; those outside [0, end) are -infinity.
template <typename T>
__device__ __forceinline__ uint4 load_vec(const T* row, int v, int end) {
  constexpr int n = Vec<T>::n;
  if (v >= 0 && v + n <= end) return __ldcs(reinterpret_cast<const uint4*>(row + v));
  uint32_t w[4];
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    w[i] = sizeof(T) == 4 ? 0xff800000u : 0xff80ff80u;
    if constexpr (sizeof(T) == 4) {
      if (v + i >= 0 && v + i < end) w[i] = bits_of(row[v + i]);
    } else {
      if (v + 2 * i >= 0 && v + 2 * i < end) w[i] = (w[i] & 0xffff0000u) | bits_of(row[v + 2 * i]);
      if (v + 2 * i + 1 >= 0 && v + 2 * i + 1 < end) w[i] = (w[i] & 0x0000ffffu) | (bits_of(row[v + 2 * i + 1]) << 16);
    }
  }
  return make_uint4(w[0], w[1], w[2], w[3]);
}
// Bits of elements v .. v + n - 1 (bit e: element v + e is suppressed); those outside [0, end) are anything.
__device__ __forceinline__ unsigned suppress_bits(const BeamSelectParams& p, int v, int end) {
  if (!p.suppress || v >= end || v <= -8) return 0;
  const unsigned char* bytes = reinterpret_cast<const unsigned char*>(p.suppress);
  const int from = max(v, 0), at = from >> 3;
  const unsigned lo = __ldg(bytes + at), hi = __ldg(bytes + min(at + 1, (p.vocab - 1) >> 3));
  return ((lo | (hi << 8)) >> (from & 7)) << (from - v);
}
template <typename T>
__device__ __forceinline__ void suppress_vec(unsigned bits, uint4& r) {
  if (bits & ((1u << Vec<T>::n) - 1)) {
    uint32_t* w = &r.x;
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      if constexpr (sizeof(T) == 4) {
        if ((bits >> i) & 1) w[i] = 0xff800000u;
      } else {
        if ((bits >> (2 * i)) & 1) w[i] = (w[i] & 0xffff0000u) | 0xff80u;
        if ((bits >> (2 * i)) & 2) w[i] = (w[i] & 0x0000ffffu) | 0xff800000u;
      }
    }
  }
}

__device__ __forceinline__ float exp_diff(float x, float base) { return ptx::ex2_approx((x - base) * kLog2e); }

// Starts the copy of elements v .. v + n - 1 of a row to 16 bytes of shared memory; those outside [0, end) are not read and
// anything there.
template <typename T>
__device__ __forceinline__ void copy_vec(const T* row, int v, int end, uint4* to) {
  constexpr int n = Vec<T>::n;
  if (v >= 0) {
    if (v < end) ptx::cp_async_16_partial(ptx::smem_u32(to), row + v, (uint32_t)min(n, end - v) * (uint32_t)sizeof(T));
  } else if (v > -n) {
    *to = load_vec(row, v, end);
  }
}

template <typename T, int kStages>
__global__ void __launch_bounds__(kSelThreads, 2) beam_select_kernel(const __grid_constant__ BeamSelectParams p, int cluster) {
  // [item][lane]: (maximum, sum) of the lane's elements; later .x is the high half of its ordered best score
  extern __shared__ __align__(16) float2 lane_stat[];
  uint4* ring = reinterpret_cast<uint4*>(lane_stat + p.n_beam * p.groups * 32) + (threadIdx.x >> 5) * (kStages * kVecs * 32);  // the warp's tiles in flight
  __shared__ float2 part[kMaxCluster][kMaxBeams];       // of a beam, from every block
  __shared__ Ranked gather[kMaxCluster * kMaxKeep];     // first block: the blocks' lists
  __shared__ Ranked cand[kCandidates + kMaxBeams];
  __shared__ unsigned short lanes[kLaneList], few[kFewLanes];
  __shared__ Ranked warp_top[kSelWarps];
  __shared__ __align__(16) uint32_t space[kSelWarps][32];
  __shared__ double lse[kMaxBeams];
  __shared__ float score[kMaxBeams];
  __shared__ int live_row[kMaxBeams];  // beams whose logits are read
  struct Place {
    const T* row;
    int first, end;  // first element of the item's first tile, end of the slice
  };
  __shared__ __align__(16) Place place[kMaxBeams * kMaxGroups];   // of an item
  __shared__ unsigned char beam_of[kMaxBeams * kMaxGroups];
  __shared__ int n_live, n_done, n_lanes, n_few, n_cand;
  __shared__ unsigned bound, bound2;
  const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5;
  const int rank = (int)blockIdx.x % cluster, b = (int)blockIdx.x / cluster;
  constexpr int kVec = Vec<T>::n, kTile = Vec<T>::tile, kPerTile = kVecs * kVec;
  ptx::cluster_arrive();

  if (warp == 0) {
    const int asked = p.beams ? __ldg(p.beams + b) : p.n_beam;
    const bool flag = p.finished && lane < p.n_beam && __ldg(p.finished + (long)b * p.n_beam + lane);
    const float mine = lane < p.n_beam ? __ldg(p.scores + (long)b * p.n_beam + lane) : 0.f;
    if (lane < p.n_beam) score[lane] = mine;
    const int live = min(max(asked, 0), p.n_beam);
    if (live != asked && rank == 0 && lane == 0) report(p.status, kBadRows);
    const bool done = lane < live && flag;
    const unsigned ended = __ballot_sync(0xffffffffu, done), open = __ballot_sync(0xffffffffu, lane < live && !done);
    if (lane < live && !done) live_row[__popc(open & ((1u << lane) - 1))] = lane;
    if (done && rank == 0) {  // the one continuation of a finished beam
      const double c = (double)mine;
      cand[__popc(ended & ((1u << lane) - 1))] = Ranked{c > -INFINITY ? ordered(c) : 0, (uint32_t)lane * (uint32_t)p.vocab + (uint32_t)p.end_token, 0};
    }
    if (lane == 0) {
      n_live = __popc(open);
      n_done = rank == 0 ? __popc(ended) : 0;
      n_cand = n_done;
      n_lanes = n_few = 0;
      bound = bound2 = 0;
    }
  }
  __syncthreads();
  const int n_items = n_live * p.groups;
  for (int i = tid; i < n_items; i += kSelThreads) {
    const int r = i / p.groups, w = live_row[r];
    const T* row = reinterpret_cast<const T*>(p.logits) + ((long)b * p.n_beam + w) * p.ld;
    const int shift = (int)(((uintptr_t)row / sizeof(T)) % kVec);  // vectors start at 16-byte borders
    place[i] = Place{row, rank * p.slice - shift + (i - r * p.groups) * p.tiles * kTile, min(p.vocab, (rank + 1) * p.slice - shift)};
    beam_of[i] = (unsigned char)w;
  }
  __syncthreads();

  // ---- one pass over the logits
  // A warp's tiles are copied to shared memory kStages ahead; every lane copies and reads its own pieces, so no barrier is
  // needed.  (Held in registers instead, one tile ahead, the compiler waited for each tile at the end of the one before.)
  int ahead_item = warp, ahead_tile = 0;
  auto start_next = [&](int stage) {
    if (ahead_item < n_items) {
      const Place x = place[ahead_item];
      const int v = x.first + ahead_tile * kTile + lane * kVec;
      uint4* to = ring + stage * (kVecs * 32) + lane;
      if (v - lane * kVec >= 0 && v - lane * kVec + kTile <= x.end) {
        const uint32_t at = ptx::smem_u32(to);
        const T* from = x.row + v;
#pragma unroll
        for (int j = 0; j < kVecs; ++j) ptx::cp_async_16(at + j * 512, from + j * 32 * kVec, true);
      } else {
#pragma unroll
        for (int j = 0; j < kVecs; ++j) copy_vec(x.row, v + j * 32 * kVec, x.end, to + j * 32);
      }
      if (++ahead_tile == p.tiles) {
        ahead_tile = 0;
        ahead_item += kSelWarps;
      }
    }
    ptx::cp_async_commit();
  };
#pragma unroll
  for (int i = 0; i < kStages; ++i) start_next(i);
  int stage = 0;
  float m = -INFINITY, l = 0.f;
  for (int item = warp, tile = 0; item < n_items;) {
    const Place at = place[item];
    const int first = at.first + tile * kTile, now_item = item;
    if (++tile == p.tiles) {
      tile = 0;
      item += kSelWarps;
    }
    // words of suppression bits of the tile: lane i has the i-th, lane 0 also the one behind the lanes'
    unsigned word = 0, word_end = 0;
    if (p.suppress) {
      const int w = (max(first, 0) >> 5) + lane, last = (p.vocab - 1) >> 5;
      if (w <= last && lane <= kTile / 32) word = __ldg(p.suppress + w);
      if (kTile == 1024 && lane == 0 && w + 32 <= last) word_end = __ldg(p.suppress + w + 32);
    }
    ptx::cp_async_wait<kStages - 1>();
    uint4* mine = ring + stage * (kVecs * 32);
    if (__any_sync(0xffffffffu, (word | word_end) != 0)) {  // suppressed elements become -infinity
      __syncwarp();
      const int base = (max(first, 0) >> 5) * 32;
      auto poke = [&](unsigned bits, int at) {
        while (bits) {
          const int v = base + at * 32 + __ffs(bits) - 1;
          bits &= bits - 1;
          if (v >= first && v < first + kTile) reinterpret_cast<T*>(mine)[v - first] = minus_infinity<T>();
        }
      };
      poke(word, lane);
      poke(word_end, 32);
      __syncwarp();
    }
    uint4 raw[kVecs];
#pragma unroll
    for (int j = 0; j < kVecs; ++j) raw[j] = mine[j * 32 + lane];
    __syncwarp();  // other lanes' pieces may have been written above: all are read before the next copies land
    start_next(stage);
    stage = stage + 1 == kStages ? 0 : stage + 1;
    if (first < 0 || first + kTile > at.end) {  // elements outside the slice are -infinity too
#pragma unroll
      for (int j = 0; j < kVecs; ++j) {
        const int v = first + (j * 32 + lane) * kVec;
        unsigned off = 0;
        if (v < 0) off |= (1u << min(-v, kVec)) - 1;
        if (v + kVec > at.end) off |= ~0u << min(max(at.end - v, 0), 31);
        suppress_vec<T>(off, raw[j]);
      }
    }
    float top = m;
#pragma unroll
    for (int j = 0; j < kVecs; ++j) top = fmaxf(top, Vec<T>::max(raw[j]));
    const float base = top > -INFINITY ? top : 0.f;  // an all-NaN lane has top = -infinity: base 0, the sum is NaN
    // sum of exp(x - base), two elements per arithmetic instruction
    const uint64_t minus = ptx::pack_f32x2(-base, -base), log2e = ptx::pack_f32x2(kLog2e, kLog2e);
    uint64_t sum[2] = {ptx::pack_f32x2(l * exp_diff(m, base), 0.f), 0ull};
#pragma unroll
    for (int j = 0; j < kVecs; ++j) {
      float x[kVec];
      Vec<T>::unpack(raw[j], x);
#pragma unroll
      for (int e = 0; e < kVec; e += 2) {
        float lo, hi;
        ptx::unpack_f32x2(ptx::mul_f32x2(ptx::add_f32x2(ptx::pack_f32x2(x[e], x[e + 1]), minus), log2e), lo, hi);
        sum[(e / 2) % 2] = ptx::add_f32x2(sum[(e / 2) % 2], ptx::pack_f32x2(ptx::ex2_approx(lo), ptx::ex2_approx(hi)));
      }
    }
    float s0, s1, s2, s3;
    ptx::unpack_f32x2(sum[0], s0, s1);
    ptx::unpack_f32x2(sum[1], s2, s3);
    l = (s0 + s1) + (s2 + s3);
    m = top;
    if (tile == 0) {  // the item is complete
      lane_stat[now_item * 32 + lane] = make_float2(m, l);
      m = -INFINITY;
      l = 0.f;
    }
  }
  __syncthreads();

  // ---- the beams' log-sums: lanes of a block, then blocks of the cluster, in a fixed order; one warp per beam
  ptx::cluster_wait();  // every block of the cluster runs
  for (int i = warp; i < n_live; i += kSelWarps) {
    const float2* from = lane_stat + i * p.groups * 32 + lane;
    float top = -INFINITY;
    for (int g = 0; g < p.groups; ++g) top = fmaxf(top, from[g * 32].x);
    const float wm = from_ordered(__reduce_max_sync(0xffffffffu, ordered(top)));
    float wl = 0.f;
    for (int g = 0; g < p.groups; ++g) {
      const float2 s = from[g * 32];
      if (s.y != 0.f) wl += s.y * exp_diff(s.x, wm > -INFINITY ? wm : 0.f);
    }
#pragma unroll
    for (int o = 16; o > 0; o >>= 1) wl += __shfl_xor_sync(0xffffffffu, wl, o);
    if (lane < cluster) ptx::st_cluster_v2(ptx::map_to_cta(ptx::smem_u32(&part[rank][i]), lane), __float_as_uint(wm), __float_as_uint(wl));
  }
  __syncwarp();
  ptx::cluster_arrive();
  ptx::cluster_wait();
  for (int i = warp; i < n_live; i += kSelWarps) {
    const float2 s = lane < cluster ? part[lane][i] : make_float2(-INFINITY, 0.f);
    const float wm = from_ordered(__reduce_max_sync(0xffffffffu, ordered(s.x)));
    float wl = s.y == 0.f ? 0.f : s.y * exp_diff(s.x, wm > -INFINITY ? wm : 0.f);
#pragma unroll
    for (int o = 4; o > 0; o >>= 1) wl += __shfl_xor_sync(0xffffffffu, wl, o);
    // log of 2^e f as e log 2 + log f: the float32 logarithm of 1 <= f < 2 is off by 2^-24 at most
    const uint32_t bits = __float_as_uint(wl);
    const double log_l = wl > 0.f && wl < INFINITY ? (double)((int)(bits >> 23) - 127) * 0.6931471805599453 + (double)logf(__uint_as_float((bits & 0x7fffffu) | 0x3f800000u))
                                                   : (double)logf(wl);
    if (lane == 0) lse[live_row[i]] = (double)wm + log_l;  // NaN if the row holds one, or +infinity; all -infinity: no score
  }
  __syncthreads();

  auto key_of = [&](int w, float x) -> uint64_t {
    const double c = (double)score[w] + ((double)x - lse[w]);
    return x > -INFINITY && c > -INFINITY ? ordered(c) : 0;  // false for NaN
  };
  // ---- the lanes that can hold one of the best
  uint32_t high = 0;
  for (int i = warp; i < n_items; i += kSelWarps) {
    const int e = i * 32 + lane;
    const uint32_t k = (uint32_t)(key_of(beam_of[i], lane_stat[e].x) >> 32);
    lane_stat[e].x = __uint_as_float(k);
    high = max(high, k);
  }
  const uint32_t mine = kth_lane_key(high, p.keep, space[warp]);
  if (lane == 0) atomicMax(&bound, mine);
  auto lane_key = [&](int e) { return __float_as_uint(lane_stat[e].x); };
  __syncthreads();
  {
    const uint32_t least = max(bound, 1u);
    for (int i = warp; i < n_items; i += kSelWarps) {
      const int e = i * 32 + lane;
      const bool in = lane_key(e) >= least;
      const unsigned who = __ballot_sync(0xffffffffu, in);
      if (who == 0) continue;
      int to = 0;
      if (lane == 0) to = atomicAdd(&n_lanes, __popc(who));
      to = __shfl_sync(0xffffffffu, to, 0) + __popc(who & ((1u << lane) - 1));
      if (in && to < kLaneList) lanes[to] = (unsigned short)e;
    }
  }
  __syncthreads();
  if (warp == 0 && n_lanes <= kLaneList) {
    uint32_t h = 0;
    for (int i = lane; i < n_lanes; i += 32) h = max(h, lane_key(lanes[i]));
    const uint32_t least = max(max(kth_lane_key(h, p.keep, space[0]), bound), 1u);
    int n = 0;
    for (int i0 = 0; i0 < n_lanes; i0 += 32) {
      const bool in = i0 + lane < n_lanes && lane_key(lanes[i0 + lane]) >= least;
      const unsigned who = __ballot_sync(0xffffffffu, in);
      const int to = n + __popc(who & ((1u << lane) - 1));
      if (in && to < kFewLanes) few[to] = lanes[i0 + lane];
      n += __popc(who);
    }
    if (lane == 0) n_few = n, bound2 = least;
  }
  __syncthreads();
  bool fits = n_lanes <= kLaneList && n_few <= kFewLanes;
  if (fits) {
    // ---- their elements once more
    for (int q = warp; q < n_few; q += kSelWarps) {
      const int e = few[q], w = beam_of[e >> 5], L = e & 31;
      const Place x = place[e >> 5];
      for (int k = lane; k < p.tiles * kPerTile; k += 32) {
        const int within = k % kPerTile, v = x.first + k / kPerTile * kTile + (within / kVec * 32 + L) * kVec + within % kVec;
        if (v < 0 || v >= x.end) continue;
        const float y = to_f32(x.row[v]);
        const uint64_t key = suppressed(p, v) ? 0 : key_of(w, y);
        if ((uint32_t)(key >> 32) >= bound2) {
          const int i = atomicAdd(&n_cand, 1);
          if (i < kCandidates) cand[i] = Ranked{key, (uint32_t)w * (uint32_t)p.vocab + (uint32_t)v, 0};
        }
      }
    }
    __syncthreads();
    fits = n_cand <= kCandidates;
  }
  const uint32_t to_first = ptx::map_to_cta(ptx::smem_u32(gather + rank * p.keep), 0);
  auto send = [&](int r, const Ranked& x) {
    ptx::st_cluster_v4(to_first + r * 16, (uint32_t)x.key, (uint32_t)(x.key >> 32), x.flat, 0);
  };
  if (fits) {
    block_best(cand, n_cand, p.keep, send);
    if (warp == 0) {  // a finished beam of score -infinity has no key
      const int keyless = __popc(__ballot_sync(0xffffffffu, lane < n_done && cand[lane].key == 0));
      for (int r = n_cand - keyless + lane; r < p.keep; r += 32) send(r, Ranked{0, 0, 0});
    }
  } else {
    // ---- many ties: one by one, each the best element of the slice behind the one before
    Ranked last{~0ull, 0, 0};
    const int done = n_done;
    for (int r = 0; r < p.keep; ++r) {
      Ranked best{0, 0xffffffffu, 0};
      for (int i = warp; i < n_items; i += kSelWarps) {
        const Place x = place[i];
        const int w = beam_of[i];
        for (int k = 0; k < p.tiles * kVecs; ++k) {
          const int v = x.first + k / kVecs * kTile + (k % kVecs * 32 + lane) * kVec;
          float y[kVec];
          uint4 bits = load_vec(x.row, v, x.end);
          suppress_vec<T>(suppress_bits(p, v, x.end), bits);
          Vec<T>::unpack(bits, y);
#pragma unroll
          for (int e = 0; e < kVec; ++e) {
            const Ranked z{key_of(w, y[e]), (uint32_t)w * (uint32_t)p.vocab + (uint32_t)(v + e), 0};
            if ((r == 0 || last.before(z)) && z.before(best)) best = z;
          }
        }
      }
      if (tid < done) {
        const Ranked z = cand[tid];
        if ((r == 0 || last.before(z)) && z.before(best)) best = z;
      }
      best = warp_first(best);
      if (lane == 0) warp_top[warp] = best;
      __syncthreads();
      last = warp_top[0];
#pragma unroll
      for (int i = 1; i < kSelWarps; ++i)
        if (warp_top[i].before(last)) last = warp_top[i];
      __syncthreads();
      if (tid == 0) send(r, last);
      if (last.key == 0) {
        for (int q = r + 1 + tid; q < p.keep; q += kSelThreads) send(q, Ranked{0, 0, 0});
        break;
      }
    }
  }
  __syncwarp();
  ptx::cluster_arrive();
  if (rank != 0) return;

  // ---- the sequence's best
  ptx::cluster_wait();
  const long o = (long)b * p.keep;
  const int n = cluster * p.keep;
  block_best(gather, n, p.keep, [&](int r, const Ranked& x) {
    const double c = __longlong_as_double((long long)(x.key >> 63 ? x.key & ~(1ull << 63) : ~x.key));
    const int w = (int)(x.flat / (uint32_t)p.vocab), v = (int)(x.flat - (uint32_t)w * (uint32_t)p.vocab);
    p.out_scores[o + r] = (float)c;
    p.out_parents[o + r] = w;
    p.out_tokens[o + r] = v;
    if (p.out_finished) p.out_finished[o + r] = v == p.end_token;  // what a finished beam offers is end_token
  });
  if (warp == kSelWarps - 1) {  // places without a continuation
    int found = 0;
    for (int i0 = 0; i0 < n; i0 += 32) found += __popc(__ballot_sync(0xffffffffu, i0 + lane < n && gather[i0 + lane].key != 0));
    for (int i = found + lane; i < p.keep; i += 32) {
      p.out_scores[o + i] = -INFINITY;
      p.out_parents[o + i] = p.out_tokens[o + i] = -1;
      if (p.out_finished) p.out_finished[o + i] = 0;
    }
  }
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
  const int tile = dtype == WF_BF16 ? Vec<__nv_bfloat16>::tile : Vec<float>::tile;
  // up to two blocks on every SM (what their registers allow), at least one tile of every row each, at most the 8 of a
  // portable cluster
  int cluster = 1;
  while (cluster < kMaxCluster && (long)B * cluster <= num_sms && p.vocab > cluster * tile) cluster *= 2;
  p.slice = ((p.vocab + 8 + cluster - 1) / cluster + 7) / 8 * 8;
  const int n_tiles = (p.slice + tile - 1) / tile;
  p.tiles = (n_tiles + kMaxGroups - 1) / kMaxGroups;
  p.groups = (n_tiles + p.tiles - 1) / p.tiles;
  // with a block or less per SM there is room for four tiles of every warp in flight, else for two
  const bool alone = (long)B * cluster <= num_sms;
  const size_t smem = (size_t)p.n_beam * p.groups * 32 * sizeof(float2) + (size_t)(alone ? 4 : 2) * kSelWarps * kVecs * 32 * sizeof(uint4);  // at most 192 KB
  auto kernel = dtype == WF_BF16 ? (alone ? beam_select_kernel<__nv_bfloat16, 4> : beam_select_kernel<__nv_bfloat16, 2>)
                                 : (alone ? beam_select_kernel<float, 4> : beam_select_kernel<float, 2>);
  cudaError_t e = cudaFuncSetAttribute(kernel, cudaFuncAttributeMaxDynamicSharedMemorySize, (int)smem);
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
