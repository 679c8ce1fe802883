// Attention over the paged cache on the 5th-generation tensor cores, for many query rows per key/value head (trees of
// drafted tokens, grouped heads, prompts).
//
// A block has one tile of 128 query rows of one key/value head over one split of the positions, and takes 64 keys a step:
//   warps 0-3   softmax, one thread per query row: scores from tensor memory, probabilities back to it as packed bfloat16
//               (two buffers), the running maximum raised (and the accumulator rescaled in place) only when it is exceeded
//               by more than 2^8 (so a row's largest probability is rounded like the others, where it would be 1 otherwise: error against
//               float64 0.0023, raised at every step 0.0019);
//   warps 5-7   load keys and values from their pages into registers one step ahead, turn codes into bfloat16 (exact, so a
//               scale multiplies the float32 score or the float32 probability, never a key or value) and write them to shared
//               memory in the swizzled layout the tensor core reads;
//   warp 4      issues S = Q K^T (128 x 64 x d) and O += P V (128 x d x 64), O staying in tensor memory.
// Against the kernel for few rows, which converts every code once per 8 .. 32 query rows and feeds the legacy matrix
// instructions, a code is converted once per 128 rows and the products cost no register traffic.
// Two blocks run per SM (256 tensor-memory columns each: S [0, 64), P [64, 96) and [96, 128), O [128, 128 + d)), so that one
// computes while the other waits.  Every wait is bounded; where one gives up, the block's rows become NaN and the caller's status word says so.
//
// Bound by the loading warps, at 1.2 us per 64-key step of an SM (128 channels, int8): a step's keys and values are waited for
// together, one step after their issue, and converted; the softmax waits for more than half of its time, the tensor cores and
// the memory are far from theirs.  8 heads of 128 channels, 16 sequences of up to 4144 positions with 8 .. 192 rows a head:
// 95 us, of which 78 MB from memory need 12; 37 sequences of 768 positions, 128 rows a head: 38 us, 390 TFLOP/s.
#include <type_traits>

#include "wf_ptx.cuh"
#include "wf_tree_attention.cuh"

namespace wf {

using namespace ptx;

namespace {

constexpr int kTileRows = 128, kStep = 64;
constexpr int kThreads = 256, kLoaders = 96;
constexpr float kLog2e = 1.4426950408889634f, kLn2 = 0.6931471805599453f;
constexpr int kHalfBytes = kStep * 128;  // 64 keys x 64 channels of bfloat16

template <int kDim>
struct Smem {  // offsets from a 1024-byte border
  static constexpr int kHalves = kDim / 64;
  static constexpr int kQ = 0;                                             // [half][128 rows][128 bytes]
  static constexpr int kK = kQ + kHalves * kTileRows * 128;                // [stage][half][64 keys][128 bytes]
  static constexpr int kV = kK + 2 * kHalves * kHalfBytes;
  static constexpr int kScale = kV + 2 * kHalves * kHalfBytes;             // [stage][keys: 64 factors, values: 64 scales] float32
  static constexpr int kValid = kScale + 2 * 2 * kStep * 4;                // [stage][2] words: the key exists
  static constexpr int kBars = kValid + 2 * 2 * 4;
  // k_full, k_free, v_full, v_free (two each), s_full, s_free, p_full (2), o_full (2), drain
  static constexpr int kNumBars = 15;
  static constexpr int kSlot = kBars + 8 * kNumBars;                       // tensor memory address, abort flag, odd values
  // at least a third of an SM's shared memory and more: two blocks share the SM's 512 tensor-memory columns
  static constexpr int kTotal = kSlot + 16 + 1024 > 80 * 1024 ? kSlot + 16 + 1024 : 80 * 1024;
};

// MN-major operand: rows are keys, the 64 contiguous elements of a row are channels.
__device__ __forceinline__ uint64_t desc_mn_sw128(uint32_t addr) {
  return (uint64_t)((addr >> 4) & 0x3FFF) | (uint64_t)1 << 16 | (uint64_t)(1024 >> 4) << 32 | (uint64_t)1 << 46 | (uint64_t)2 << 61;
}
// Byte offset of 16-byte chunk c (0 .. 7) of a row in the 128-byte swizzle.
__device__ __forceinline__ uint32_t swizzled(int row, int c) { return (uint32_t)(row * 128 + ((c ^ (row & 7)) << 4)); }

__device__ __forceinline__ uint32_t pack_bf16(float lo, float hi) {
  const __nv_bfloat162 h = __floats2bfloat162_rn(lo, hi);
  return *reinterpret_cast<const uint32_t*>(&h);
}

// Four codes as two bfloat16 pairs, exactly.
template <int kFormat>
__device__ __forceinline__ void codes_bf16(uint32_t w, uint32_t& lo, uint32_t& hi) {
  if (kFormat == WF_CACHE_E4M3) {
    // sign, then the seven other bits where bfloat16 has its low exponent bits: the value times 2^-120
    const uint32_t a = __byte_perm(w, 0, 0x1404), b = __byte_perm(w, 0, 0x3424);
    asm("mul.rn.bf16x2 %0, %1, %2;" : "=r"(lo) : "r"(((a >> 4) & 0x07f007f0u) | (a & 0x80008000u)), "r"(0x7b807b80u));
    asm("mul.rn.bf16x2 %0, %1, %2;" : "=r"(hi) : "r"(((b >> 4) & 0x07f007f0u) | (b & 0x80008000u)), "r"(0x7b807b80u));
  } else {
    // (128 + low seven bits) - (128, or 256 for a negative code)
    const uint32_t a = __byte_perm(w, 0x43434343u, 0x4140), b = __byte_perm(w, 0x43434343u, 0x4342);
    asm("sub.rn.bf16x2 %0, %1, %2;" : "=r"(lo) : "r"(a & 0xff7fff7fu), "r"(a & 0xff80ff80u));
    asm("sub.rn.bf16x2 %0, %1, %2;" : "=r"(hi) : "r"(b & 0xff7fff7fu), "r"(b & 0xff80ff80u));
  }
}

__device__ __forceinline__ bool odd_bf16x2(uint32_t w) { return (w & 0x7f80u) == 0x7f80u || (w & 0x7f800000u) == 0x7f800000u; }

template <int kFormat, int kDim>
__global__ void __launch_bounds__(kThreads, 2) tree_attention_wide_kernel(const __grid_constant__ TreeAttnParams p) {
  using S = Smem<kDim>;
  constexpr bool kQuant = kFormat != WF_CACHE_PATH;
  constexpr int kVecBytes = kDim * (kQuant ? 1 : 2);
  constexpr int kPieces = kVecBytes / 16;          // 16-byte pieces of a vector
  constexpr int kPasses = (kStep * kPieces + kLoaders - 1) / kLoaders;  // pieces per loading thread and step
  extern __shared__ unsigned char smem_raw[];

  const int seq = blockIdx.z, kvh = blockIdx.y;
  const int split = (int)blockIdx.x % p.n_splits, tile = (int)blockIdx.x / p.n_splits;
  const int tid = threadIdx.x, warp = tid >> 5, lane = tid & 31;
  const Sequence s = load_sequence(p, seq, tid == 0 && blockIdx.x == 0 && kvh == 0);
  const int rows = min(s.n_rows, p.max_rows) * p.group;
  const int r0 = tile * kTileRows;
  if (r0 >= rows) return;
  const int begin = split * p.chunk, end = min(s.len, begin + p.chunk);
  if (split > 0 && begin >= s.len) return;
  const int n_steps = end > begin ? (end - begin + kStep - 1) / kStep : 0;

  const uint32_t sbase = (smem_u32(smem_raw) + 1023u) & ~1023u;
  unsigned char* const sgen = smem_raw + (sbase - smem_u32(smem_raw));
  auto bar = [&](int i) { return sbase + S::kBars + 8u * i; };
  auto k_full = [&](int st) { return bar(st); };
  auto k_free = [&](int st) { return bar(2 + st); };
  auto v_full = [&](int st) { return bar(4 + st); };
  auto v_free = [&](int st) { return bar(6 + st); };
  const uint32_t s_full = bar(8), s_free = bar(9);
  auto p_full = [&](int b) { return bar(10 + b); };
  auto o_full = [&](int b) { return bar(12 + b); };
  const uint32_t drain = bar(14);
  volatile uint32_t* tmem_slot = reinterpret_cast<volatile uint32_t*>(sgen + S::kSlot);
  volatile int* abort_flag = reinterpret_cast<volatile int*>(sgen + S::kSlot + 4);
  volatile int* odd_values = reinterpret_cast<volatile int*>(sgen + S::kSlot + 8);
  float* const scales = reinterpret_cast<float*>(sgen + S::kScale);
  unsigned* const valid = reinterpret_cast<unsigned*>(sgen + S::kValid);

  if (tid == 0) {
    for (int i = 0; i < 2; ++i) {
      mbar_init(k_full(i), kLoaders);
      mbar_init(k_free(i), 1);
      mbar_init(v_full(i), kLoaders);
      mbar_init(v_free(i), 1);
      mbar_init(p_full(i), 128);
      mbar_init(o_full(i), 1);
    }
    mbar_init(s_full, 1);
    mbar_init(s_free, 128);
    mbar_init(drain, 1);
    *abort_flag = 0;
    *odd_values = 0;
    fence_mbar_init();
  }
  if (warp == 4) {
    tmem_alloc(smem_u32(const_cast<uint32_t*>(tmem_slot)), 256);
    tmem_relinquish();
  }
  // ---- the query tile, rows behind the last one as zeros
  {
    constexpr int kEach = kTileRows * (kDim / 8) / kThreads;  // 16-byte pieces per thread
    uint4 x[kEach];
#pragma unroll
    for (int k = 0; k < kEach; ++k) {
      const int i = k * kThreads + tid, rr = i / (kDim / 8), c = i % (kDim / 8), r = r0 + rr;
      x[k] = make_uint4(0, 0, 0, 0);
      if (r < rows) {
        const int row = r / p.group;
        x[k] = __ldg(reinterpret_cast<const uint4*>(reinterpret_cast<const __nv_bfloat16*>(p.q) + (long)(s.first_row + row) * p.q_stride +
                                                    (long)(kvh * p.group + r - row * p.group) * kDim) + c);
      }
    }
#pragma unroll
    for (int k = 0; k < kEach; ++k) {
      const int i = k * kThreads + tid, rr = i / (kDim / 8), c = i % (kDim / 8);
      st_shared_v4(sbase + S::kQ + (c / 8) * (kTileRows * 128) + swizzled(rr, c % 8), x[k].x, x[k].y, x[k].z, x[k].w);
    }
  }
  fence_proxy_async_smem();
  tc_fence_before();
  __syncthreads();
  tc_fence_after();
  const uint32_t tmem = *tmem_slot;
  bool ok = true, issuer = false;  // issuer: the thread that starts the products

  if (warp > 4) {
    // ------------------------------------------------------------------ loads and conversion
    const int lt = tid - (kThreads - kLoaders);
    // this thread's i-th piece of a step: piece `piece_of(i)` of key `key_of(i)`; the last pass may have none for it
    auto key_of = [&](int i) { return (i * kLoaders + lt) / kPieces; };
    auto piece_of = [&](int i) { return (i * kLoaders + lt) % kPieces; };
    auto has = [&](int i) { return (i + 1) * kLoaders <= kStep * kPieces || i * kLoaders + lt < kStep * kPieces; };
    const int shift = p.cache.page_shift;
    const int* table = p.rows.page_table + (long)seq * p.rows.table_stride;
    constexpr uint32_t kAbsent = 0xffffffffu;
    uint4 kraw[kPasses], vraw[kPasses];
    unsigned short kscale = 0, vscale = 0;  // bfloat16 bits, of key lt
    bool there = false;
    // Lanes 0 .. 3 of a warp look up the pages of the step's four 16-key tiles, a step before their vectors are loaded.
    uint32_t page = 0, tile = kAbsent, vtile = kAbsent;  // vtile: of the values in registers
    auto look_up = [&](int j) {
      const int pos = begin + j * kStep + 16 * (lane & 3);
      page = (uint32_t)__ldg(table + (min(pos, end - 1) >> shift));
    };
    auto find = [&](int j) {  // index of the lane's tile's first vector in the cache
      const int pos = begin + j * kStep + 16 * (lane & 3);
      tile = kAbsent;
      if (pos < end) {
        if (page < (uint32_t)p.cache.n_pages) tile = ((page * (uint32_t)p.cache.n_kv_head + (uint32_t)kvh) << shift) + (uint32_t)(pos & ((1 << shift) - 1));
        else report(p.status, kBadPage);
      }
    };
    // vector of a key of the step; an absent one's place is taken by the cache's first (it is masked)
    auto vector_of = [&](int key) -> uint32_t {
      const uint32_t first = __shfl_sync(0xffffffffu, tile, key >> 4);
      return first == kAbsent ? 0u : first + (uint32_t)(key & 15);
    };
    auto load_keys = [&]() {
#pragma unroll
      for (int i = 0; i < kPasses; ++i) {
        const uint32_t v = vector_of(min(key_of(i), kStep - 1));
        kraw[i] = __ldcs(reinterpret_cast<const uint4*>(p.cache.k) + (uint64_t)v * kPieces + piece_of(i));
      }
    };
    auto load_values = [&](int j) {
      vtile = tile;
#pragma unroll
      for (int i = 0; i < kPasses; ++i) {
        const uint32_t v = vector_of(min(key_of(i), kStep - 1));
        vraw[i] = __ldcs(reinterpret_cast<const uint4*>(p.cache.v) + (uint64_t)v * kPieces + piece_of(i));
      }
      const int key = min(lt, kStep - 1);
      const uint32_t v = vector_of(key);
      there = __shfl_sync(0xffffffffu, tile, key >> 4) != kAbsent && begin + j * kStep + key < end;
      if constexpr (kQuant) {
        kscale = __ldg(reinterpret_cast<const unsigned short*>(p.cache.k_scale) + v);
        vscale = __ldg(reinterpret_cast<const unsigned short*>(p.cache.v_scale) + v);
      }
    };
    auto put = [&](uint32_t base, const uint4 (&raw)[kPasses]) {
#pragma unroll
      for (int i = 0; i < kPasses; ++i) {
        if (!has(i)) continue;
        const int key = key_of(i), piece = piece_of(i);
        const uint4 x = raw[i];
        if constexpr (kQuant) {
          uint32_t a[4], b[4];
          codes_bf16<kFormat>(x.x, a[0], a[1]);
          codes_bf16<kFormat>(x.y, a[2], a[3]);
          codes_bf16<kFormat>(x.z, b[0], b[1]);
          codes_bf16<kFormat>(x.w, b[2], b[3]);
          const uint32_t half = base + (uint32_t)(piece / 4) * kHalfBytes;
          st_shared_v4(half + swizzled(key, 2 * piece % 8), a[0], a[1], a[2], a[3]);
          st_shared_v4(half + swizzled(key, 2 * piece % 8 + 1), b[0], b[1], b[2], b[3]);
        } else {
          st_shared_v4(base + (uint32_t)(piece / 8) * kHalfBytes + swizzled(key, piece % 8), x.x, x.y, x.z, x.w);
        }
      }
    };
    if (n_steps > 0) {
      look_up(0);
      find(0);
      load_keys();
      load_values(0);
      look_up(1);
    }
    // The next step's keys and values are loaded side by side at the end of a step, past the last one too (absent keys stand for
    // the cache's first): with a condition around them, or the keys' loads between the two conversions, loads were
    // waited for where they were issued (107 and 100 us instead of 97).
    for (int j = 0; j < n_steps; ++j) {
      const int st = j & 1;
      const uint32_t parity = ((j >> 1) & 1u) ^ 1u;
      if (!__all_sync(0xffffffffu, mbar_wait_limited(k_free(st), parity, abort_flag, p.wait_limit))) { ok = false; break; }
      put(sbase + S::kK + st * S::kHalves * kHalfBytes, kraw);
      fence_proxy_async_smem();
      mbar_arrive(k_full(st));
      if (!__all_sync(0xffffffffu, mbar_wait_limited(v_free(st), parity, abort_flag, p.wait_limit))) { ok = false; break; }
      if constexpr (!kQuant) {
        // A batch row's value that is not finite must not reach rows that do not see it through 0 * inf: it is left out here
        // and added, at the end, to the rows that see it.
        // (Positions behind the end and absent ones are zeros.)
        const unsigned pages = __ballot_sync(0xffffffffu, vtile != kAbsent) & 15u;
        if (begin + (j + 1) * kStep > min(s.start, end) || pages != 15u) {
#pragma unroll
          for (int i = 0; i < kPasses; ++i) {
            uint32_t* w = &vraw[i].x;
            const int pos = begin + j * kStep + key_of(i);
            const bool batch_row = pos >= s.start;
            if (pos >= end || !((pages >> (key_of(i) >> 4 & 3)) & 1)) vraw[i] = make_uint4(0, 0, 0, 0);
#pragma unroll
            for (int e = 0; e < 4; ++e)
              if (batch_row && odd_bf16x2(w[e])) {
                *odd_values = 1;
                if ((w[e] & 0x7f80u) == 0x7f80u) w[e] &= 0xffff0000u;
                if ((w[e] & 0x7f800000u) == 0x7f800000u) w[e] &= 0x0000ffffu;
              }
          }
        }
      }
      put(sbase + S::kV + st * S::kHalves * kHalfBytes, vraw);
      if (kQuant && lt < kStep) {
        scales[st * 2 * kStep + lt] = __uint_as_float((uint32_t)kscale << 16) * (p.scale * kLog2e);
        scales[st * 2 * kStep + kStep + lt] = __uint_as_float((uint32_t)vscale << 16);
      }
      const unsigned exists = __ballot_sync(0xffffffffu, there);
      if (lt < kStep && lane == 0) valid[st * 2 + lt / 32] = exists;
      fence_proxy_async_smem();
      mbar_arrive(v_full(st));
      find(j + 1);
      load_keys();
      load_values(j + 1);
      look_up(j + 2);
    }
  } else if (warp == 4) {
    // ------------------------------------------------------------------ matrix products
    const bool leader = issuer = elect_one();
    constexpr uint32_t idesc_s = umma_idesc_bf16(kTileRows, kStep, 0, 0);
    constexpr uint32_t idesc_o = umma_idesc_bf16(kTileRows, 64, 0, 1);
    auto wait_all = [&](uint32_t b, uint32_t parity) -> bool { return __all_sync(0xffffffffu, mbar_wait_limited(b, parity, abort_flag, p.wait_limit)); };
    auto issue_scores = [&](int j) -> bool {
      const int st = j & 1;
      if (j > 0 && !wait_all(s_free, (j - 1) & 1u)) return false;
      if (!wait_all(k_full(st), (j >> 1) & 1u)) return false;
      tc_fence_after();
      if (leader) {
#pragma unroll
        for (int h = 0; h < S::kHalves; ++h) {
          const uint64_t qd = umma_desc_k_sw128(sbase + S::kQ + h * kTileRows * 128);
          const uint64_t kd = umma_desc_k_sw128(sbase + S::kK + (st * S::kHalves + h) * kHalfBytes);
#pragma unroll
          for (int k = 0; k < 4; ++k) umma_bf16(tmem, qd + 2 * k, kd + 2 * k, idesc_s, h > 0 || k > 0);
        }
        umma_commit(s_full);
        umma_commit(k_free(st));
      }
      __syncwarp();
      return true;
    };
    auto issue_output = [&](int j) -> bool {
      const int st = j & 1;
      if (!wait_all(v_full(st), (j >> 1) & 1u) || !wait_all(p_full(st), (j >> 1) & 1u)) return false;
      tc_fence_after();
      if (leader) {
#pragma unroll
        for (int h = 0; h < S::kHalves; ++h) {
          const uint64_t vd = desc_mn_sw128(sbase + S::kV + (st * S::kHalves + h) * kHalfBytes);
#pragma unroll
          for (int k = 0; k < 4; ++k) umma_bf16_ts(tmem + 128 + 64 * h, tmem + 64 + 32 * st + 8 * k, vd + 128 * k, idesc_o, j > 0 || k > 0);
        }
        umma_commit(o_full(st));
        umma_commit(v_free(st));
      }
      __syncwarp();
      return true;
    };
    // the scores of a step run while the softmax works on those of the step before
    if (n_steps > 0) ok = issue_scores(0);
    for (int j = 0; ok && j < n_steps; ++j) ok = (j + 1 >= n_steps || issue_scores(j + 1)) && issue_output(j);
  } else {
    // ------------------------------------------------------------------ softmax, one query row per thread
    const int r = r0 + tid;
    const uint32_t ta = tmem + ((uint32_t)(warp * 32) << 16);
    const bool active = r0 + warp * 32 < rows;  // of the warp
    const bool mine = r < rows;
    const int i_row = mine ? r / p.group : 0;
    constexpr float kRaise = 8.f, kRaiseSum = 256.f;
    float m = -INFINITY, l = 0.f;
    auto wait_warp = [&](uint32_t b, uint32_t parity) -> bool { return __all_sync(0xffffffffu, mbar_wait_limited(b, parity, abort_flag, p.wait_limit)); };
    for (int j = 0; j < n_steps; ++j) {
      const int st = j & 1, pos0 = begin + j * kStep;
      if (!wait_warp(s_full, j & 1u)) { ok = false; break; }
      tc_fence_after();
      uint32_t x[kStep];
      if (active) {
        tmem_ld_32x32(ta, *reinterpret_cast<uint32_t(*)[32]>(&x[0]));
        tmem_ld_32x32(ta + 32, *reinterpret_cast<uint32_t(*)[32]>(&x[32]));
        tmem_ld_wait();
      }
      tc_fence_before();
      mbar_arrive(s_free);  // the scores are in registers: the next product may overwrite them
      if (!wait_warp(v_full(st), (j >> 1) & 1u)) { ok = false; break; }  // the step's scales are there
      if (active) {
        const float4* kf = reinterpret_cast<const float4*>(scales + st * 2 * kStep);
        const float4* vs = kf + kStep / 4;
        const uint64_t plain = pack_f32x2(p.scale * kLog2e, p.scale * kLog2e);
#pragma unroll
        for (int i = 0; i < kStep; i += 4) {
          uint64_t f0 = plain, f1 = plain;
          if constexpr (kQuant) {
            const float4 f = kf[i / 4];
            f0 = pack_f32x2(f.x, f.y);
            f1 = pack_f32x2(f.z, f.w);
          }
          float a, b;
          unpack_f32x2(mul_f32x2(pack_f32x2(__uint_as_float(x[i]), __uint_as_float(x[i + 1])), f0), a, b);
          x[i] = __float_as_uint(a);
          x[i + 1] = __float_as_uint(b);
          unpack_f32x2(mul_f32x2(pack_f32x2(__uint_as_float(x[i + 2]), __uint_as_float(x[i + 3])), f1), a, b);
          x[i + 2] = __float_as_uint(a);
          x[i + 3] = __float_as_uint(b);
        }
        // what the row does not see
        const unsigned v0 = valid[st * 2], v1 = valid[st * 2 + 1];
        const bool clean = pos0 + kStep <= s.start && (v0 & v1) == 0xffffffffu;
        unsigned see[2] = {v0, v1};
        if (!clean) {
#pragma unroll
          for (int h = 0; h < 2; ++h) {
            unsigned bits = see[h];
            const int t0 = pos0 + 32 * h - s.start;  // batch row of bit 0
            if (t0 + 32 > 0 && p.tail != WF_TAIL_NONE) {
              unsigned may;  // bit b: batch row t0 + b is seen, or the position is a committed one
              if (p.tail == WF_TAIL_CAUSAL) {
                const int n = i_row - t0 + 1;  // rows t0 .. i
                may = n >= 32 ? 0xffffffffu : n <= 0 ? 0u : (1u << n) - 1;
              } else {
                auto word = [&](int w) -> unsigned {
                  if (w < 0) return 0xffffffffu;
                  return w < p.mask_words ? __ldg(p.mask + (long)(s.first_row + i_row) * p.mask_words + w) : 0u;
                };
                const int w = t0 >> 5;  // (rounds down)
                may = __funnelshift_r(word(w), word(w + 1), (unsigned)t0 & 31u);
              }
              if (t0 < 0) may |= (1u << -t0) - 1;  // -t0 < 32 committed positions
              bits &= may;
            }
            see[h] = mine ? bits : 0u;
          }
#pragma unroll
          for (int i = 0; i < kStep; ++i)
            if (!((see[i / 32] >> (i % 32)) & 1)) x[i] = 0xff800000u;
        }
        auto row_max = [&]() {
          float a = -INFINITY, b = -INFINITY, c = -INFINITY, d = -INFINITY;
#pragma unroll
          for (int i = 0; i < kStep; i += 4) {
            a = fmaxf(a, __uint_as_float(x[i]));
            b = fmaxf(b, __uint_as_float(x[i + 1]));
            c = fmaxf(c, __uint_as_float(x[i + 2]));
            d = fmaxf(d, __uint_as_float(x[i + 3]));
          }
          return fmaxf(fmaxf(a, b), fmaxf(c, d));
        };
        if (__any_sync(0xffffffffu, m == -INFINITY)) {
          const float top = row_max();
          if (m == -INFINITY) m = top;  // nothing has been added up yet
        }
        float sum;
        auto exponentials_of = [&](auto clean_tag) {
          constexpr bool kClean = decltype(clean_tag)::value;
          const float base = m == -INFINITY ? 0.f : m;
          const uint64_t minus = pack_f32x2(-base, -base);
          uint64_t s0 = 0, s1 = 0;
#pragma unroll
          for (int c = 0; c < 2; ++c) {
            uint32_t pk[16];
#pragma unroll
            for (int i = 0; i < 16; i += 2) {
              const int e = 32 * c + 2 * i;
              float a0, a1, b0, b1;
              unpack_f32x2(add_f32x2(pack_f32x2(__uint_as_float(x[e]), __uint_as_float(x[e + 1])), minus), a0, a1);
              unpack_f32x2(add_f32x2(pack_f32x2(__uint_as_float(x[e + 2]), __uint_as_float(x[e + 3])), minus), b0, b1);
              uint64_t wa = pack_f32x2(ex2_approx(a0), ex2_approx(a1)), wb = pack_f32x2(ex2_approx(b0), ex2_approx(b1));
              s0 = add_f32x2(s0, wa);
              s1 = add_f32x2(s1, wb);
              if constexpr (kQuant) {
                const float4 f = vs[e / 4];
                wa = mul_f32x2(wa, pack_f32x2(f.x, f.y));
                wb = mul_f32x2(wb, pack_f32x2(f.z, f.w));
              }
              unpack_f32x2(wa, a0, a1);
              unpack_f32x2(wb, b0, b1);
              if constexpr (kQuant && !kClean) {  // a vector that the row does not see may have any scale, NaN too
                if (!((see[c] >> (2 * i)) & 1)) a0 = 0.f;
                if (!((see[c] >> (2 * i)) & 2)) a1 = 0.f;
                if (!((see[c] >> (2 * i)) & 4)) b0 = 0.f;
                if (!((see[c] >> (2 * i)) & 8)) b1 = 0.f;
              }
              pk[i] = pack_bf16(a0, a1);
              pk[i + 1] = pack_bf16(b0, b1);
            }
            __syncwarp();
            tmem_st_32x16(ta + 64 + 32 * st + 16 * c, pk);
          }
          float q0, q1, q2, q3;
          unpack_f32x2(s0, q0, q1);
          unpack_f32x2(s1, q2, q3);
          sum = (q0 + q1) + (q2 + q3);
        };
        auto exponentials = [&]() {
          if (!kQuant || clean) exponentials_of(std::true_type{});
          else exponentials_of(std::false_type{});
        };
        // The buffer of these probabilities was last read by the product of two steps ago, which had landed when this step's
        // scores came (its issue precedes theirs in the same thread, and their commit covers it).
        exponentials();
        if (j > 0 && __any_sync(0xffffffffu, !(sum <= kRaiseSum))) {
          const float top = row_max();
          const bool raise = top > m + kRaise;
          if (__any_sync(0xffffffffu, raise)) {
            if (!wait_warp(o_full(st ^ 1), ((j - 1) >> 1) & 1u)) { ok = false; break; }
            tc_fence_after();
            const float f = raise ? ex2_approx(m - top) : 1.f;
            if (raise) m = top, l *= f;
#pragma unroll
            for (int c = 0; c < kDim / 16; ++c) {
              uint32_t a[16];
              tmem_ld_32x16(ta + 128 + 16 * c, a);
              tmem_ld_wait();
#pragma unroll
              for (int i = 0; i < 16; ++i) a[i] = __float_as_uint(__uint_as_float(a[i]) * f);
              tmem_st_32x16(ta + 128 + 16 * c, a);
            }
            tmem_st_wait();
            exponentials();
          }
        }
        l += sum;
        tmem_st_wait();
      }
      tc_fence_before();
      mbar_arrive(p_full(st));
    }
    // the last two products
    if (ok && n_steps >= 2) ok = wait_warp(o_full(n_steps & 1), ((n_steps - 2) >> 1) & 1u);
    if (ok && n_steps >= 1) ok = wait_warp(o_full((n_steps - 1) & 1), ((n_steps - 1) >> 1) & 1u);
    tc_fence_after();
    if (ok && active) {
      const long row = s.first_row + i_row;
      const int head = kvh * p.group + r % p.group;
      const float inv = l == 0.f ? 0.f : 1.f / l;
      const bool odd = !kQuant && *odd_values != 0;
      const long at = (row * p.n_head + head) * p.n_splits + split;
      for (int c = 0; c < kDim / 16; ++c) {
        uint32_t a[16];
        if (n_steps > 0) {
          tmem_ld_32x16(ta + 128 + 16 * c, a);
          tmem_ld_wait();
        }
        if (mine) {
        float y[16];
#pragma unroll
        for (int i = 0; i < 16; ++i) y[i] = l == 0.f ? 0.f : __uint_as_float(a[i]);
        if (odd) {  // values that are not finite, of the batch rows that this one sees
          for (int pos = max(begin, s.start); pos < end; ++pos) {
            if (!sees_tail(p, s, i_row, pos - s.start)) continue;
            const int page = page_of(p, seq, pos);
            if (page < 0) continue;
            const __nv_bfloat16* v = reinterpret_cast<const __nv_bfloat16*>(p.cache.v) +
                                     ((((long)page * p.cache.n_kv_head + kvh) << p.cache.page_shift) + (pos & ((1 << p.cache.page_shift) - 1))) * kDim + 16 * c;
#pragma unroll
            for (int i = 0; i < 16; ++i) {
              const float z = __bfloat162float(v[i]);
              if ((__float_as_uint(z) & 0x7f800000u) == 0x7f800000u) y[i] += z;
            }
          }
        }
        if (p.n_splits > 1) {
          float4* to = reinterpret_cast<float4*>(p.part_o + at * kDim + 16 * c);
#pragma unroll
          for (int i = 0; i < 4; ++i) to[i] = make_float4(y[4 * i], y[4 * i + 1], y[4 * i + 2], y[4 * i + 3]);
        } else {
          uint4* to = reinterpret_cast<uint4*>(reinterpret_cast<__nv_bfloat16*>(p.out) + row * p.out_stride + (long)head * kDim + 16 * c);
#pragma unroll
          for (int i = 0; i < 2; ++i)
            to[i] = make_uint4(pack_bf16(y[8 * i] * inv, y[8 * i + 1] * inv), pack_bf16(y[8 * i + 2] * inv, y[8 * i + 3] * inv),
                               pack_bf16(y[8 * i + 4] * inv, y[8 * i + 5] * inv), pack_bf16(y[8 * i + 6] * inv, y[8 * i + 7] * inv));
        }
        }
        __syncwarp();
      }
      if (mine) {
        if (p.n_splits > 1) p.part_ml[at] = make_float2(m * kLn2, l);
        else if (p.lse) p.lse[row * p.n_head + head] = l == 0.f ? -INFINITY : (m + log2f(l)) * kLn2;
      }
    }
    if (!ok && mine) {  // a wait gave up: the row is NaN (with splits, the join makes NaN of a NaN sum)
      const long row = s.first_row + i_row;
      const int head = kvh * p.group + r % p.group;
      const float nan = __int_as_float(0x7fc00000);
      if (p.n_splits > 1) {
        p.part_ml[(row * p.n_head + head) * p.n_splits + split] = make_float2(nan, nan);
      } else {
        uint4* to = reinterpret_cast<uint4*>(reinterpret_cast<__nv_bfloat16*>(p.out) + row * p.out_stride + (long)head * kDim);
        for (int c = 0; c < kDim / 8; ++c) to[c] = make_uint4(0x7fc07fc0u, 0x7fc07fc0u, 0x7fc07fc0u, 0x7fc07fc0u);
        if (p.lse) p.lse[row * p.n_head + head] = nan;
      }
    }
  }
  if (!ok && lane == 0) report(p.status, kGaveUp);
  tc_fence_before();
  __syncthreads();
  if (warp == 4) {
    if (*abort_flag) {  // products may be in flight: they land before tensor memory and shared memory are given back
      if (issuer) umma_commit(drain);
      __syncwarp();
      int never = 0;
      mbar_wait_limited(drain, 0, &never, kWaitLimit);
      __syncwarp();
    }
    tc_fence_after();
    tmem_dealloc(tmem, 256);
  }
}

template <int kFormat, int kDim>
cudaError_t launch(const TreeAttnParams& p, cudaStream_t s) {
  const long rows = (long)p.max_rows * p.group;
  const int tiles = (int)((rows + kTileRows - 1) / kTileRows);
  const dim3 grid((unsigned)(tiles * p.n_splits), (unsigned)p.cache.n_kv_head, (unsigned)p.rows.n_seq);
  auto kernel = tree_attention_wide_kernel<kFormat, kDim>;
  cudaError_t e = cudaFuncSetAttribute(kernel, cudaFuncAttributeMaxDynamicSharedMemorySize, Smem<kDim>::kTotal);
  if (e != cudaSuccess) return e;
  return launch_dependent(kernel, grid, dim3(kThreads), Smem<kDim>::kTotal, s, 1, false, p);
}

template <int kFormat>
cudaError_t launch_dim(const TreeAttnParams& p, int d_head, cudaStream_t s) {
  return d_head == 64 ? launch<kFormat, 64>(p, s) : launch<kFormat, 128>(p, s);
}

}  // namespace

cudaError_t launch_tree_attention_wide(const TreeAttnParams& p, int d_head, int format, cudaStream_t s) {
  if (format == WF_CACHE_PATH) return launch_dim<WF_CACHE_PATH>(p, d_head, s);
  if (format == WF_CACHE_E4M3) return launch_dim<WF_CACHE_E4M3>(p, d_head, s);
  return launch_dim<WF_CACHE_INT8>(p, d_head, s);
}

}  // namespace wf
