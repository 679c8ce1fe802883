// Attention over the paged cache on the tensor cores, for few query rows per key/value head.
//
// The cache is read once and everything else is small, so the kernel is built around the loads.  The scores
// are computed transposed, S^T = K Q^T, with the keys as the 16-row operand and 8 query rows as the columns.  A
// lane then needs whole 16-byte pieces of a key (the sum over channels may run in any order, so a lane's piece
// serves several steps of the product).  Every lane copies its own pieces to shared memory, a few blocks of keys ahead
// (cp.async), and reads them back into operand registers: no barrier, no bank conflict, every byte moved once.  The output is
// transposed as well, O^T = V^T P^T; the value operand's pairs of neighbouring keys are made by byte permutation of
// two keys' pieces, and P^T comes from S^T by one 8 x 8 transposition in registers.
// The warps of a unit take blocks of keys in turn, each with its own running maximum and sums, and are joined at the end.
//
// Quantised caches: a code is exact in float16 and in bfloat16.  Scores: codes as float16 times the queries
// scaled by a power of two per row into float16 (exact up to 2^-24 of the row's largest element), the vector's scale
// multiplies the float32 score.  Values: codes as bfloat16, and the probability times the vector's scale rounded once
// to bfloat16, whose range holds any scale.  Unquantised: bfloat16 throughout, the probability rounded to it.
//
// Bound by memory where few heads share long histories: 2 sequences of 119 and 131 thousand positions, 8 heads of 128
// channels, bfloat16: 200 us, 5.1 TB/s.  Many short ones are bound by the starts and ends of their blocks and by issue: 64 sequences
// of 75 .. 775 positions, 20 heads of 64 channels, e4m3: 27 us, 2.8 TB/s, half of the issue slots busy.  One token,
// 20 heads, 151 positions: 4.6 us, the latency of three dependent loads (lengths, page, keys) and the join of the warps.
#include "wf_ptx.cuh"
#include "wf_tree_attention.cuh"

namespace wf {

namespace {

constexpr int kThreads = 128;  // four warps
constexpr float kLog2e = 1.4426950408889634f, kLn2 = 0.6931471805599453f;

__device__ __forceinline__ void mma_f16(float (&c)[4], const uint32_t (&a)[4], uint32_t b0, uint32_t b1) {
  asm volatile("mma.sync.aligned.m16n8k16.row.col.f32.f16.f16.f32 {%0, %1, %2, %3}, {%4, %5, %6, %7}, {%8, %9}, {%0, %1, %2, %3};"
               : "+f"(c[0]), "+f"(c[1]), "+f"(c[2]), "+f"(c[3])
               : "r"(a[0]), "r"(a[1]), "r"(a[2]), "r"(a[3]), "r"(b0), "r"(b1));
}
__device__ __forceinline__ void mma_bf16(float (&c)[4], const uint32_t (&a)[4], uint32_t b0, uint32_t b1) {
  asm volatile("mma.sync.aligned.m16n8k16.row.col.f32.bf16.bf16.f32 {%0, %1, %2, %3}, {%4, %5, %6, %7}, {%8, %9}, {%0, %1, %2, %3};"
               : "+f"(c[0]), "+f"(c[1]), "+f"(c[2]), "+f"(c[3])
               : "r"(a[0]), "r"(a[1]), "r"(a[2]), "r"(a[3]), "r"(b0), "r"(b1));
}
__device__ __forceinline__ uint32_t transpose8x8(uint32_t x) {
  uint32_t y;
  asm volatile("movmatrix.sync.aligned.m8n8.trans.b16 %0, %1;" : "=r"(y) : "r"(x));
  return y;
}
__device__ __forceinline__ uint32_t pack_bf16(float lo, float hi) {
  const __nv_bfloat162 h = __floats2bfloat162_rn(lo, hi);
  return *reinterpret_cast<const uint32_t*>(&h);
}
__device__ __forceinline__ uint32_t pack_f16(float lo, float hi) {
  const __half2 h = __floats2half2_rn(lo, hi);
  return *reinterpret_cast<const uint32_t*>(&h);
}

// Four codes (bytes 0..3 of w) as float16 pairs (0, 1) and (2, 3), exactly.
template <int kFormat>
__device__ __forceinline__ void codes_f16(uint32_t w, uint32_t& lo, uint32_t& hi) {
  if (kFormat == WF_CACHE_E4M3) {
    asm("cvt.rn.f16x2.e4m3x2 %0, %1;" : "=r"(lo) : "h"((unsigned short)(w & 0xffffu)));
    asm("cvt.rn.f16x2.e4m3x2 %0, %1;" : "=r"(hi) : "h"((unsigned short)(w >> 16)));
  } else {
    // 1024 + (code + 128) is a float16 whose low mantissa byte is the biased code
    const uint32_t u = w ^ 0x80808080u, bias = 0x64806480u;
    const uint32_t a = __byte_perm(u, 0x64646464u, 0x4140), b = __byte_perm(u, 0x64646464u, 0x4342);
    asm("sub.rn.f16x2 %0, %1, %2;" : "=r"(lo) : "r"(a), "r"(bias));
    asm("sub.rn.f16x2 %0, %1, %2;" : "=r"(hi) : "r"(b), "r"(bias));
  }
}
// Codes in two bytes of w (kSel 0: bytes 0 and 1, 1: bytes 2 and 3) as a bfloat16 pair, exactly.
template <int kFormat, int kSel>
__device__ __forceinline__ uint32_t codes_bf16(uint32_t w) {
  uint32_t r;
  if (kFormat == WF_CACHE_E4M3) {
    // sign, then the seven other bits where bfloat16 has its low exponent bits: the value times 2^-120
    const uint32_t x = __byte_perm(w, 0, kSel == 0 ? 0x1404 : 0x3424);
    const uint32_t y = ((x >> 4) & 0x07f007f0u) | (x & 0x80008000u);
    asm("mul.rn.bf16x2 %0, %1, %2;" : "=r"(r) : "r"(y), "r"(0x7b807b80u));
  } else {
    // (128 + low seven bits) - (128, or 256 for a negative code)
    const uint32_t x = __byte_perm(w, 0x43434343u, kSel == 0 ? 0x4140 : 0x4342);
    asm("sub.rn.bf16x2 %0, %1, %2;" : "=r"(r) : "r"(x & 0xff7fff7fu), "r"(x & 0xff80ff80u));
  }
  return r;
}

template <int kFormat, int kDim>
struct Layout {
  static constexpr int kEsz = kFormat == WF_CACHE_PATH ? 2 : 1;
  static constexpr int kVecBytes = kDim * kEsz;
  static constexpr int kTiles = kVecBytes == 64 ? 2 : 1;  // 16-key tiles of a block of keys
  static constexpr int kKeys = 16 * kTiles;           // 32 or 16
  static constexpr int kKChunks = kVecBytes / 64;     // 16-byte pieces of a key per lane
  static constexpr int kVWords = kVecBytes / 32;      // 32-bit words of a value per lane
  static constexpr int kSteps = kDim / 16;            // steps of S^T's product = 16-channel tiles of O^T
  // a warp's blocks of keys in flight, and the bytes of one: keys' pieces, values' pieces, scales
  static constexpr int kStages = 2;
  static constexpr int kKeyBytes = kKeys * kVecBytes;
  static constexpr int kStageBytes = 2 * kKeyBytes + (kFormat == WF_CACHE_PATH ? 0 : 64 * kTiles);
  static constexpr int kVPieces = kVecBytes == 256 ? 2 : 1;             // pieces of a value per lane
  static constexpr int kVPieceBytes = kVecBytes == 64 ? 8 : 16;
  // channel of element e (0 .. 3) of the lane's share of step s
  static __device__ __forceinline__ int key_channel(int s, int t) {
    return kEsz == 2 ? 32 * (s / 2) + 8 * t + 4 * (s % 2) : 64 * (s / 4) + 16 * t + 4 * (s % 4);
  }
  // channel of rows g and g + 8 (the next one) of 16-channel tile j
  static __device__ __forceinline__ int value_channel(int j, int g) {
    return kVecBytes == 256 ? 64 * (j / 4) + 8 * g + 2 * (j % 4) : kDim / 8 * g + 2 * j;
  }
};

// A unit of work is one tile of query rows of one key/value head over one split of the positions; kW warps share it.
// Shared memory of a warp: its copies in flight, and at the end its rows' sums.
template <int kFormat, int kDim, int kNT>
__host__ __device__ constexpr int warp_bytes() {
  constexpr int copies = Layout<kFormat, kDim>::kStages * Layout<kFormat, kDim>::kStageBytes, rows = 8 * kNT * (kDim + 6) * 4;
  return copies > rows ? copies : (rows + 15) / 16 * 16;
}

template <int kFormat, int kDim, int kNT, int kW>
__global__ void __launch_bounds__(kThreads, kNT == 1 ? 5 : kNT == 2 && kDim == 64 ? 3 : 2) tree_attention_tc_kernel(const __grid_constant__ TreeAttnParams p, int tiles) {
  using L = Layout<kFormat, kDim>;
  constexpr bool kQuant = kFormat != WF_CACHE_PATH;
  constexpr int kRows = 8 * kNT;
  extern __shared__ __align__(16) unsigned char smem[];
  constexpr int kWarpBytes = warp_bytes<kFormat, kDim, kNT>();
  const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5, g = lane >> 2, t = lane & 3;
  const int seq = blockIdx.y;
  const int unit = (int)blockIdx.x * (4 / kW) + warp / kW, rest = unit / p.n_splits;
  const int split = unit - rest * p.n_splits, kvh = rest / tiles, tile = rest - kvh * tiles;
  if (kvh >= p.cache.n_kv_head) return;
  const int begin = split * p.chunk, shift = p.cache.page_shift;
  const int* table = p.rows.page_table + (long)seq * p.rows.table_stride;
  // The warp's 16-key tiles, T = 0, 1, ...: lane i holds the page of tile 32 b + i for the current b and the next one.
  auto tile_pos = [&](int T) -> long { return (long)begin + (long)(warp % kW + T / L::kTiles * kW) * L::kKeys + 16 * (T % L::kTiles); };
  auto load_pages = [&](int b) {
    const long index = tile_pos(32 * b + lane) >> shift;
    return index < p.rows.table_stride ? __ldg(table + index) : -1;
  };
  int page_next = load_pages(0);
  const Sequence s = load_sequence(p, seq, tid == 0 && blockIdx.x == 0);
  const int rows = min(s.n_rows, p.max_rows) * p.group;
  const int r0 = tile * kRows;
  if (r0 >= rows) return;
  const int end = min(s.len, begin + p.chunk);
  if (split > 0 && begin >= s.len) return;
  // ---- copies
  constexpr uint32_t kAbsent = 0xffffffffu;  // (at most 2^32 vectors of 64 bytes or more fit a GPU)
  auto first_vector = [&](int page, int b) -> uint32_t {  // index of the lane's tile's first vector in the cache
    const long at = tile_pos(32 * b + lane);
    if (at >= end) return kAbsent;
    if ((unsigned)page >= (unsigned)p.cache.n_pages) {
      report(p.status, kBadPage);
      return kAbsent;
    }
    return (((uint32_t)page * (uint32_t)p.cache.n_kv_head + (uint32_t)kvh) << shift) + (uint32_t)((int)at & ((1 << shift) - 1));
  };
  const int w0 = begin + warp % kW * L::kKeys;
  const int n_blocks = w0 < end ? (end - w0 + kW * L::kKeys - 1) / (kW * L::kKeys) : 0;
  uint32_t vec = first_vector(page_next, 0);
  page_next = load_pages(1);
  unsigned char* const ring = smem + warp * kWarpBytes;
  const char* const key_base = reinterpret_cast<const char*>(p.cache.k) + g * L::kVecBytes + t * 16;
  const char* const value_base = reinterpret_cast<const char*>(p.cache.v) + 2 * t * L::kVecBytes + g * L::kVPieceBytes;
  // lanes 0, 1: the scales of a tile's 16 keys; 2, 3: of its values
  const char* const scale_base = reinterpret_cast<const char*>(lane < 2 ? p.cache.k_scale : p.cache.v_scale) + (lane & 1) * 16;
  uint32_t id[L::kTiles];   // of the block whose copies are being started
  unsigned absent = 0;      // bit (stage, tile): the tile has no page
  auto copy_keys = [&](int n, int stage) {
    if (n < n_blocks) {
      if (n > 0 && (n * L::kTiles) % 32 == 0) {
        vec = first_vector(page_next, n * L::kTiles / 32);
        page_next = load_pages(n * L::kTiles / 32 + 1);
      }
      const uint32_t at = ptx::smem_u32(ring + stage * L::kStageBytes) + lane * 16;
#pragma unroll
      for (int i = 0; i < L::kTiles; ++i) {
        id[i] = __shfl_sync(0xffffffffu, vec, (n * L::kTiles + i) % 32);
        const unsigned bit = 1u << (stage * L::kTiles + i);
        absent = id[i] == kAbsent ? absent | bit : absent & ~bit;
        if (id[i] == kAbsent) continue;
        const char* from = key_base + (uint64_t)id[i] * L::kVecBytes;
#pragma unroll
        for (int h = 0; h < 2; ++h)
#pragma unroll
          for (int c = 0; c < L::kKChunks; ++c)
            ptx::cp_async_16_stream(at + ((i * 2 + h) * L::kKChunks + c) * 512, from + 8 * h * L::kVecBytes + c * 64);
        if constexpr (kQuant) {
          if (lane < 4) ptx::cp_async_16(at + 2 * L::kKeyBytes + i * 64, scale_base + (uint64_t)id[i] * 2, true);
        }
      }
    }
    ptx::cp_async_commit();
  };
  auto copy_values = [&](int n, int stage) {
    if (n < n_blocks) {
      const uint32_t at = ptx::smem_u32(ring + stage * L::kStageBytes) + L::kKeyBytes + lane * L::kVPieceBytes;
#pragma unroll
      for (int i = 0; i < L::kTiles; ++i) {
        if (id[i] == kAbsent) continue;
        const char* from = value_base + (uint64_t)id[i] * L::kVecBytes;
#pragma unroll
        for (int k = 0; k < 4; ++k)
#pragma unroll
          for (int c = 0; c < L::kVPieces; ++c) {
            const uint32_t to = at + ((i * 4 + k) * L::kVPieces + c) * 32 * L::kVPieceBytes;
            const char* src = from + ((k & 1) + 8 * (k >> 1)) * L::kVecBytes + c * 128;
            if constexpr (L::kVPieceBytes == 16) ptx::cp_async_16_stream(to, src);
            else ptx::cp_async_8(to, src);
          }
      }
    }
    ptx::cp_async_commit();
  };
  // commit groups alternate, keys of block 0, values of block 0, keys of block 1, ...: 2 kStages of them are open
#pragma unroll
  for (int i = 0; i < L::kStages; ++i) {
    copy_keys(i, i);
    copy_values(i, i);
  }
  // ---- queries: the second operand of S^T, element pairs matching the lane's pieces of a key
  uint32_t qf[kNT][L::kSteps][2];
  float factor[kNT][2];  // of the scores of rows 2t and 2t + 1: scale * log2(e), and the row's power of two
#pragma unroll
  for (int nt = 0; nt < kNT; ++nt) {
    const int r = r0 + nt * 8 + g;
    uint2 raw[L::kSteps];
    const __nv_bfloat16* q = reinterpret_cast<const __nv_bfloat16*>(p.q) + (long)(s.first_row + r / p.group) * p.q_stride +
                             (long)(kvh * p.group + r % p.group) * kDim;
#pragma unroll
    for (int i = 0; i < L::kSteps; ++i)
      raw[i] = r < rows ? __ldg(reinterpret_cast<const uint2*>(q + L::key_channel(i, t))) : make_uint2(0, 0);
    if constexpr (kQuant) {
      uint32_t top = 0;
#pragma unroll
      for (int i = 0; i < L::kSteps; ++i)
        top = max(max(top, max(raw[i].x << 16 & 0x7fff0000u, raw[i].x & 0x7fff0000u)), max(raw[i].y << 16 & 0x7fff0000u, raw[i].y & 0x7fff0000u));
      top = max(top, __shfl_xor_sync(0xffffffffu, top, 1));
      top = max(top, __shfl_xor_sync(0xffffffffu, top, 2));
      // the row's largest element becomes 1 .. 2; exponents at either end of the range stay within normal floats
      const int e = min(max((int)(top >> 23), 2), 252);
      const float down = __uint_as_float((uint32_t)(254 - e) << 23), up = __uint_as_float((uint32_t)e << 23);  // 2^(127 - e), 2^(e - 127)
#pragma unroll
      for (int i = 0; i < L::kSteps; ++i) {
        qf[nt][i][0] = pack_f16(__uint_as_float(raw[i].x << 16) * down, __uint_as_float(raw[i].x & 0xffff0000u) * down);
        qf[nt][i][1] = pack_f16(__uint_as_float(raw[i].y << 16) * down, __uint_as_float(raw[i].y & 0xffff0000u) * down);
      }
      factor[nt][0] = __shfl_sync(0xffffffffu, up, 8 * t) * (p.scale * kLog2e);
      factor[nt][1] = __shfl_sync(0xffffffffu, up, 8 * t + 4) * (p.scale * kLog2e);
    } else {
#pragma unroll
      for (int i = 0; i < L::kSteps; ++i) qf[nt][i][0] = raw[i].x, qf[nt][i][1] = raw[i].y;
      factor[nt][0] = factor[nt][1] = p.scale * kLog2e;
    }
  }

  float o[kNT][L::kSteps][4];
  float m[kNT][2], l[kNT][2];
#pragma unroll
  for (int nt = 0; nt < kNT; ++nt) {
#pragma unroll
    for (int j = 0; j < L::kSteps; ++j)
#pragma unroll
      for (int i = 0; i < 4; ++i) o[nt][j][i] = 0.f;
    m[nt][0] = m[nt][1] = -INFINITY;
    l[nt][0] = l[nt][1] = 0.f;
  }

  int stage = 0;
  for (int n = 0; n < n_blocks; ++n) {
    const int pos = w0 + n * kW * L::kKeys;
    const unsigned char* slot = ring + stage * L::kStageBytes;
    const unsigned no_page = absent >> (stage * L::kTiles);  // bit i: tile i
    ptx::cp_async_wait<2 * L::kStages - 1>();
    if constexpr (kQuant) __syncwarp();  // the scales are copied by some lanes for all
    // ---- S^T
    float sc[L::kTiles][kNT][4];
#pragma unroll
    for (int i = 0; i < L::kTiles; ++i) {
#pragma unroll
      for (int nt = 0; nt < kNT; ++nt) sc[i][nt][0] = sc[i][nt][1] = sc[i][nt][2] = sc[i][nt][3] = 0.f;
      uint4 piece[2][L::kKChunks];
#pragma unroll
      for (int h = 0; h < 2; ++h)
#pragma unroll
        for (int c = 0; c < L::kKChunks; ++c) piece[h][c] = reinterpret_cast<const uint4*>(slot)[((i * 2 + h) * L::kKChunks + c) * 32 + lane];
      auto word = [&](int h, int c, int w) { return w == 0 ? piece[h][c].x : w == 1 ? piece[h][c].y : w == 2 ? piece[h][c].z : piece[h][c].w; };
#pragma unroll
      for (int st = 0; st < L::kSteps; ++st) {
        uint32_t a[4];
        if constexpr (kQuant) {
          codes_f16<kFormat>(word(0, st / 4, st % 4), a[0], a[2]);
          codes_f16<kFormat>(word(1, st / 4, st % 4), a[1], a[3]);
        } else {
          a[0] = word(0, st / 2, (st % 2) * 2);
          a[1] = word(1, st / 2, (st % 2) * 2);
          a[2] = word(0, st / 2, (st % 2) * 2 + 1);
          a[3] = word(1, st / 2, (st % 2) * 2 + 1);
        }
#pragma unroll
        for (int nt = 0; nt < kNT; ++nt) {
          if constexpr (kQuant) mma_f16(sc[i][nt], a, qf[nt][st][0], qf[nt][st][1]);
          else mma_bf16(sc[i][nt], a, qf[nt][st][0], qf[nt][st][1]);
        }
      }
    }
    float kscale[L::kTiles][2], vscale[L::kTiles][2];  // of keys g and g + 8 of each tile
    if constexpr (kQuant) {
#pragma unroll
      for (int i = 0; i < L::kTiles; ++i) {
        const unsigned short* x = reinterpret_cast<const unsigned short*>(slot + 2 * L::kKeyBytes + i * 64);
        kscale[i][0] = __uint_as_float((uint32_t)x[g] << 16);
        kscale[i][1] = __uint_as_float((uint32_t)x[g + 8] << 16);
        vscale[i][0] = __uint_as_float((uint32_t)x[g + 16] << 16);
        vscale[i][1] = __uint_as_float((uint32_t)x[g + 24] << 16);
      }
      __syncwarp();
    }
    const bool clean = pos + L::kKeys <= min(end, s.start) && (no_page & ((1u << L::kTiles) - 1)) == 0;
    copy_keys(n + L::kStages, stage);

    // ---- softmax over the keys (rows of S^T: lanes with the same t hold the same query rows)
#pragma unroll
    for (int i = 0; i < L::kTiles; ++i)
#pragma unroll
      for (int nt = 0; nt < kNT; ++nt)
#pragma unroll
        for (int h = 0; h < 2; ++h) {  // key g + 8 h, rows 2t and 2t + 1
          uint64_t f = ptx::pack_f32x2(factor[nt][0], factor[nt][1]);
          if constexpr (kQuant) f = ptx::mul_f32x2(f, ptx::pack_f32x2(kscale[i][h], kscale[i][h]));
          ptx::unpack_f32x2(ptx::mul_f32x2(ptx::pack_f32x2(sc[i][nt][2 * h], sc[i][nt][2 * h + 1]), f), sc[i][nt][2 * h], sc[i][nt][2 * h + 1]);
        }
    if (!clean) {
#pragma unroll
      for (int i = 0; i < L::kTiles; ++i)
#pragma unroll
        for (int nt = 0; nt < kNT; ++nt)
#pragma unroll
          for (int c = 0; c < 4; ++c) {
            const int at = pos + 16 * i + g + 8 * (c >> 1), r = r0 + nt * 8 + 2 * t + (c & 1);
            const bool see = !((no_page >> i) & 1) && at < end && r < rows && (at < s.start || sees_tail(p, s, r / p.group, at - s.start));
            if (!see) sc[i][nt][c] = -INFINITY;
          }
    }
    bool grew = false;
    float m_new[kNT][2];
#pragma unroll
    for (int nt = 0; nt < kNT; ++nt)
#pragma unroll
      for (int h = 0; h < 2; ++h) {
        float x = m[nt][h];
#pragma unroll
        for (int i = 0; i < L::kTiles; ++i) x = fmaxf(x, fmaxf(sc[i][nt][h], sc[i][nt][h + 2]));
        x = fmaxf(x, __shfl_xor_sync(0xffffffffu, x, 4));
        x = fmaxf(x, __shfl_xor_sync(0xffffffffu, x, 8));
        x = fmaxf(x, __shfl_xor_sync(0xffffffffu, x, 16));
        m_new[nt][h] = x;
        grew |= x != m[nt][h];
      }
    if (__any_sync(0xffffffffu, grew)) {
#pragma unroll
      for (int nt = 0; nt < kNT; ++nt)
#pragma unroll
        for (int h = 0; h < 2; ++h) {
          const float f = m_new[nt][h] == -INFINITY ? 1.f : exp2f(m[nt][h] - m_new[nt][h]);
          m[nt][h] = m_new[nt][h];
          l[nt][h] *= f;
#pragma unroll
          for (int j = 0; j < L::kSteps; ++j) o[nt][j][h] *= f, o[nt][j][h + 2] *= f;
        }
    }
    uint32_t pf[L::kTiles][kNT][2];
#pragma unroll
    for (int nt = 0; nt < kNT; ++nt) {
      const float base0 = m[nt][0] == -INFINITY ? 0.f : m[nt][0], base1 = m[nt][1] == -INFINITY ? 0.f : m[nt][1];
      const uint64_t minus = ptx::pack_f32x2(-base0, -base1);
      uint64_t sum = ptx::pack_f32x2(l[nt][0], l[nt][1]);
#pragma unroll
      for (int i = 0; i < L::kTiles; ++i)
#pragma unroll
        for (int h = 0; h < 2; ++h) {
          float w0, w1;
          ptx::unpack_f32x2(ptx::add_f32x2(ptx::pack_f32x2(sc[i][nt][2 * h], sc[i][nt][2 * h + 1]), minus), w0, w1);
          w0 = ptx::ex2_approx(w0);
          w1 = ptx::ex2_approx(w1);
          const uint64_t w = ptx::pack_f32x2(w0, w1);
          sum = ptx::add_f32x2(sum, w);
          if constexpr (kQuant) {
            ptx::unpack_f32x2(ptx::mul_f32x2(w, ptx::pack_f32x2(vscale[i][h], vscale[i][h])), w0, w1);
            if (!clean) {  // a masked vector's scale may be NaN
              if (sc[i][nt][2 * h] == -INFINITY) w0 = 0.f;
              if (sc[i][nt][2 * h + 1] == -INFINITY) w1 = 0.f;
            }
          }
          pf[i][nt][h] = transpose8x8(pack_bf16(w0, w1));
        }
      ptx::unpack_f32x2(sum, l[nt][0], l[nt][1]);
    }

    // ---- O^T
    ptx::cp_async_wait<2 * L::kStages - 1>();
    uint32_t vreg[L::kTiles][4][L::kVWords];
#pragma unroll
    for (int i = 0; i < L::kTiles; ++i)
#pragma unroll
      for (int k = 0; k < 4; ++k) {
        if constexpr (L::kVPieceBytes == 8) {
          const uint2 x = reinterpret_cast<const uint2*>(slot + L::kKeyBytes)[(i * 4 + k) * 32 + lane];
          vreg[i][k][0] = x.x;
          vreg[i][k][1] = x.y;
        } else {
#pragma unroll
          for (int c = 0; c < L::kVPieces; ++c) {
            const uint4 x = reinterpret_cast<const uint4*>(slot + L::kKeyBytes)[((i * 4 + k) * L::kVPieces + c) * 32 + lane];
            vreg[i][k][4 * c] = x.x;
            vreg[i][k][4 * c + 1] = x.y;
            vreg[i][k][4 * c + 2] = x.z;
            vreg[i][k][4 * c + 3] = x.w;
          }
        }
      }
    if constexpr (!kQuant) {
      if (!clean) {
        // Values behind the end are not the sequence's, and a batch row's value that is not finite must not reach rows that do not
        // see it through 0 * inf: such elements are taken out here and added to the rows that see them.
#pragma unroll
        for (int i = 0; i < L::kTiles; ++i) {
          bool odd = false;
#pragma unroll
          for (int k = 0; k < 4; ++k) {
            const bool in = !((no_page >> i) & 1) && pos + 16 * i + 2 * t + (k & 1) + 8 * (k >> 1) < end;
#pragma unroll
            for (int w = 0; w < L::kVWords; ++w) {
              if (!in) vreg[i][k][w] = 0;
              odd |= (vreg[i][k][w] & 0x7f80u) == 0x7f80u || (vreg[i][k][w] & 0x7f800000u) == 0x7f800000u;
            }
          }
          if (!__any_sync(0xffffffffu, odd)) continue;
#pragma unroll
          for (int k = 0; k < 4; ++k)
            for (int owner = 0; owner < 4; ++owner) {
              const int at = pos + 16 * i + 2 * owner + (k & 1) + 8 * (k >> 1);
#pragma unroll
              for (int j = 0; j < L::kVWords; ++j) {
                const uint32_t w = __shfl_sync(0xffffffffu, vreg[i][k][j], (lane & ~3) | owner);
#pragma unroll
                for (int half = 0; half < 2; ++half) {
                  const uint32_t bits = half == 0 ? w << 16 : w & 0xffff0000u;
                  if ((bits & 0x7f800000u) != 0x7f800000u) continue;
#pragma unroll
                  for (int nt = 0; nt < kNT; ++nt)
#pragma unroll
                    for (int h = 0; h < 2; ++h) {
                      const int r = r0 + nt * 8 + 2 * t + h;
                      if (at < end && r < rows && (at < s.start || sees_tail(p, s, r / p.group, at - s.start)))
                        o[nt][j][2 * half + h] += __uint_as_float(bits);
                    }
                }
              }
            }
#pragma unroll
          for (int k = 0; k < 4; ++k)
#pragma unroll
            for (int w = 0; w < L::kVWords; ++w) {
              if ((vreg[i][k][w] & 0x7f80u) == 0x7f80u) vreg[i][k][w] &= 0xffff0000u;
              if ((vreg[i][k][w] & 0x7f800000u) == 0x7f800000u) vreg[i][k][w] &= 0x0000ffffu;
            }
        }
      }
    }
#pragma unroll
    for (int i = 0; i < L::kTiles; ++i)
#pragma unroll
      for (int j = 0; j < L::kSteps; ++j) {
        uint32_t a[4];
        if constexpr (kQuant) {
          const uint32_t x = __byte_perm(vreg[i][0][j / 2], vreg[i][1][j / 2], j % 2 == 0 ? 0x5140 : 0x7362);
          const uint32_t y = __byte_perm(vreg[i][2][j / 2], vreg[i][3][j / 2], j % 2 == 0 ? 0x5140 : 0x7362);
          a[0] = codes_bf16<kFormat, 0>(x);
          a[1] = codes_bf16<kFormat, 1>(x);
          a[2] = codes_bf16<kFormat, 0>(y);
          a[3] = codes_bf16<kFormat, 1>(y);
        } else {
          a[0] = __byte_perm(vreg[i][0][j], vreg[i][1][j], 0x5410);
          a[1] = __byte_perm(vreg[i][0][j], vreg[i][1][j], 0x7632);
          a[2] = __byte_perm(vreg[i][2][j], vreg[i][3][j], 0x5410);
          a[3] = __byte_perm(vreg[i][2][j], vreg[i][3][j], 0x7632);
        }
#pragma unroll
        for (int nt = 0; nt < kNT; ++nt) mma_bf16(o[nt][j], a, pf[i][nt][0], pf[i][nt][1]);
      }
    copy_values(n + L::kStages, stage);
    stage = stage + 1 == L::kStages ? 0 : stage + 1;
  }
  ptx::cp_async_wait<0>();

  // ---- output
#pragma unroll
  for (int nt = 0; nt < kNT; ++nt)
#pragma unroll
    for (int h = 0; h < 2; ++h) {  // the lanes' shares of a row's sum
      float x = l[nt][h];
      x += __shfl_xor_sync(0xffffffffu, x, 4);
      x += __shfl_xor_sync(0xffffffffu, x, 8);
      x += __shfl_xor_sync(0xffffffffu, x, 16);
      l[nt][h] = x;
    }
  // eight neighbouring channels of a row
  auto finish = [&](int r, int ch, float top, float sum, const float (&x)[8], bool first) {
    const long row = s.first_row + r / p.group;
    const int head = kvh * p.group + r % p.group;
    if (p.n_splits > 1) {
      const long at = (row * p.n_head + head) * p.n_splits + split;
      float4* to = reinterpret_cast<float4*>(p.part_o + at * kDim + ch);
      to[0] = make_float4(x[0], x[1], x[2], x[3]);
      to[1] = make_float4(x[4], x[5], x[6], x[7]);
      if (first) p.part_ml[at] = make_float2(top * kLn2, sum);
    } else {
      const float inv = sum == 0.f ? 0.f : 1.f / sum;
      uint4 out;
      out.x = pack_bf16(x[0] * inv, x[1] * inv);
      out.y = pack_bf16(x[2] * inv, x[3] * inv);
      out.z = pack_bf16(x[4] * inv, x[5] * inv);
      out.w = pack_bf16(x[6] * inv, x[7] * inv);
      *reinterpret_cast<uint4*>(reinterpret_cast<__nv_bfloat16*>(p.out) + row * p.out_stride + (long)head * kDim + ch) = out;
      if (first && p.lse) p.lse[row * p.n_head + head] = sum == 0.f ? -INFINITY : (top + log2f(sum)) * kLn2;
    }
  };
  if constexpr (kW == 1) {
#pragma unroll
    for (int nt = 0; nt < kNT; ++nt)
#pragma unroll
      for (int h = 0; h < 2; ++h) {
        const int r = r0 + nt * 8 + 2 * t + h;
        if (r >= rows) continue;
#pragma unroll
        for (int j = 0; j < L::kSteps; j += 4) {
          float x[8];
#pragma unroll
          for (int e = 0; e < 4; ++e) x[2 * e] = o[nt][j + e][h], x[2 * e + 1] = o[nt][j + e][h + 2];
          finish(r, L::value_channel(j, g), m[nt][h], l[nt][h], x, j == 0 && g == 0);
        }
      }
  } else {
    // join the unit's warps
    auto rows_of = [&](int w) { return reinterpret_cast<float*>(smem + w * kWarpBytes); };  // [row][kDim + 4], then [row] m, [row] l
    constexpr int kStat = kRows * (kDim + 4);
    float* mine = rows_of(warp);
    __syncwarp();
#pragma unroll
    for (int nt = 0; nt < kNT; ++nt)
#pragma unroll
      for (int h = 0; h < 2; ++h) {
        const int r = nt * 8 + 2 * t + h;
        if (g == 0) mine[kStat + r] = m[nt][h], mine[kStat + kRows + r] = l[nt][h];
#pragma unroll
        for (int j = 0; j < L::kSteps; ++j)
          *reinterpret_cast<float2*>(mine + r * (kDim + 4) + L::value_channel(j, g)) = make_float2(o[nt][j][h], o[nt][j][h + 2]);
      }
    const int first_warp = warp / kW * kW;
    asm volatile("bar.sync %0, %1;" ::"r"(1 + first_warp / kW), "n"(kW * 32) : "memory");
    constexpr int kUnits = kRows * kDim / 8;
    for (int u = tid - first_warp * 32; u < kUnits; u += kW * 32) {
      const int rr = u / (kDim / 8), ch = u % (kDim / 8) * 8;
      if (r0 + rr >= rows) break;
      float top = -INFINITY;
#pragma unroll
      for (int w = 0; w < kW; ++w) top = fmaxf(top, rows_of(first_warp + w)[kStat + rr]);
      const float base = top == -INFINITY ? 0.f : top;
      float sum = 0.f, x[8];
#pragma unroll
      for (int e = 0; e < 8; ++e) x[e] = 0.f;
#pragma unroll
      for (int w = 0; w < kW; ++w) {
        const float* x_of = rows_of(first_warp + w);
        const float f = exp2f(x_of[kStat + rr] - base);
        sum += x_of[kStat + kRows + rr] * f;
        const float* from = x_of + rr * (kDim + 4) + ch;
#pragma unroll
        for (int e = 0; e < 8; ++e) x[e] += from[e] * f;
      }
      finish(r0 + rr, ch, top, sum, x, ch == 0);
    }
  }
}

template <int kFormat, int kDim, int kNT, int kW>
cudaError_t launch_tile(const TreeAttnParams& p, cudaStream_t s) {
  const long rows = (long)p.max_rows * p.group;
  const int tiles = (int)((rows + 8 * kNT - 1) / (8 * kNT));
  const long units = (long)tiles * p.n_splits * p.cache.n_kv_head;
  const dim3 grid((unsigned)((units + 4 / kW - 1) / (4 / kW)), (unsigned)p.rows.n_seq);
  auto kernel = tree_attention_tc_kernel<kFormat, kDim, kNT, kW>;
  constexpr size_t smem = (size_t)4 * warp_bytes<kFormat, kDim, kNT>();
  cudaError_t e = cudaSuccess;
  if (smem > 48 * 1024) e = cudaFuncSetAttribute(kernel, cudaFuncAttributeMaxDynamicSharedMemorySize, (int)smem);
  if (e != cudaSuccess) return e;
  return launch_dependent(kernel, grid, dim3(kThreads), smem, s, 1, false, p, tiles);
}

template <int kFormat, int kDim, int kNT>
cudaError_t launch_warps(const TreeAttnParams& p, cudaStream_t s) {
  if (p.unit_warps == 1) return launch_tile<kFormat, kDim, kNT, 1>(p, s);
  if (p.unit_warps == 2) return launch_tile<kFormat, kDim, kNT, 2>(p, s);
  return launch_tile<kFormat, kDim, kNT, 4>(p, s);
}

template <int kFormat>
cudaError_t launch_dim(const TreeAttnParams& p, int d_head, int rows_tile, cudaStream_t s) {
  if (d_head == 64) {
    if (rows_tile == 8) return launch_warps<kFormat, 64, 1>(p, s);
    if (rows_tile == 16) return launch_warps<kFormat, 64, 2>(p, s);
    return launch_warps<kFormat, 64, 4>(p, s);
  }
  return rows_tile == 8 ? launch_warps<kFormat, 128, 1>(p, s) : launch_warps<kFormat, 128, 2>(p, s);
}

}  // namespace

cudaError_t launch_tree_attention_tc(const TreeAttnParams& p, int d_head, int format, int rows_tile, cudaStream_t s) {
  if (format == WF_CACHE_PATH) return launch_dim<WF_CACHE_PATH>(p, d_head, rows_tile, s);
  if (format == WF_CACHE_E4M3) return launch_dim<WF_CACHE_E4M3>(p, d_head, rows_tile, s);
  return launch_dim<WF_CACHE_INT8>(p, d_head, rows_tile, s);
}

}  // namespace wf
