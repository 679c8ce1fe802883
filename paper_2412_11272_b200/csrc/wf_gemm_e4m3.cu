// Products with 8-bit codes: C = act(A W^T + bias), A [m, k] and W [n, k] as e4m3 codes with one power-of-two scale (a byte b,
// 2^(b - 127)) for each 128 channels of a row.
//
// The tensor cores take such scales themselves (kind::mxf8f6f4, block scaled: a byte per row and 32 channels, held in tensor
// memory), so a scale costs nothing in the main loop: the products of a block are multiplied by both scales, exactly, on their
// way into the float32 accumulator.  One byte serves the four 32-channel instructions of its block; the four bytes of a
// 32-bit column of tensor memory are four consecutive blocks, picked by the instruction's scale number.
#include <atomic>

#include "wf_decoder.h"
#include "wf_epilogue.cuh"
#include "wf_ptx.cuh"

namespace wf {
namespace {

using namespace ptx;

// ---------------------------------------------------------------------------------------------
// Codes of the rows of x: eight lanes take the 128 channels of a block, sixteen each.
//   s = the least power of two with max |x| / s <= 448, code = x / s (exact) rounded to the nearest e4m3 value, ties to even.
// Bound by memory for large matrices, once the instructions a value are few: sixteen values a lane share the look-up of
// their place and the exchange of the maximum, and the maximum of bfloat16 values is taken two at a time.
constexpr int kQuantThreads = 256;
constexpr int kQuantItems = 2;  // blocks that a group of lanes has in flight
constexpr int kQuantEach = 16, kQuantLanes = kScaleBlock / kQuantEach;

// What sixteen elements are before they are needed as numbers: bits, two bfloat16 or one float32 a word.
template <typename T>
struct Sixteen {
  static constexpr int words = kQuantEach * (int)sizeof(T) / 4;
  uint32_t w[words];
};
template <typename T>
__device__ __forceinline__ void load_whole(const T* x, Sixteen<T>& r) {
#pragma unroll
  for (int i = 0; i < Sixteen<T>::words / 4; ++i) {
    const uint4 u = __ldg(reinterpret_cast<const uint4*>(x) + i);
    r.w[4 * i] = u.x, r.w[4 * i + 1] = u.y, r.w[4 * i + 2] = u.z, r.w[4 * i + 3] = u.w;
  }
}
// The first n of them (n <= 0: none), the rest zero.
__device__ __forceinline__ void load_some(const float* x, int n, Sixteen<float>& r) {
#pragma unroll
  for (int i = 0; i < 16; ++i) r.w[i] = i < n ? __float_as_uint(__ldg(x + i)) : 0u;
}
__device__ __forceinline__ void load_some(const __nv_bfloat16* x, int n, Sixteen<__nv_bfloat16>& r) {
  const unsigned short* h = reinterpret_cast<const unsigned short*>(x);
#pragma unroll
  for (int i = 0; i < 8; ++i) r.w[i] = (2 * i < n ? (uint32_t)__ldg(h + 2 * i) : 0u) | (2 * i + 1 < n ? (uint32_t)__ldg(h + 2 * i + 1) << 16 : 0u);
}
// The bits of the largest magnitude as float32 (a NaN or an infinity is the largest).
__device__ __forceinline__ uint32_t top_of(const Sixteen<float>& r) {
  uint32_t top = 0;
#pragma unroll
  for (int i = 0; i < 16; ++i) top = max(top, r.w[i] & 0x7fffffffu);
  return top;
}
__device__ __forceinline__ uint32_t top_of(const Sixteen<__nv_bfloat16>& r) {
  uint32_t two = 0;
#pragma unroll
  for (int i = 0; i < 8; ++i) two = __vmaxu2(two, r.w[i] & 0x7fff7fffu);
  return max(two << 16, two & 0xffff0000u);
}
__device__ __forceinline__ float2 pair_of(const Sixteen<float>& r, int i) { return make_float2(__uint_as_float(r.w[2 * i]), __uint_as_float(r.w[2 * i + 1])); }
__device__ __forceinline__ float2 pair_of(const Sixteen<__nv_bfloat16>& r, int i) {
  return make_float2(__uint_as_float(r.w[i] << 16), __uint_as_float(r.w[i] & 0xffff0000u));
}

// The blocks of `rows_each` rows are counted through: block i of them is block i % blocks of row i / blocks (`magic`: 2^32 / blocks
// rounded up; exact as i * blocks < 2^32).
template <typename T, bool kAligned>
__global__ void __launch_bounds__(kQuantThreads) quantise_e4m3_kernel(const T* __restrict__ x, long ldx, long rows, int k, int blocks,
                                                                     uint32_t magic, int rows_each, unsigned char* __restrict__ codes,
                                                                     long ld_codes, unsigned char* __restrict__ scales, long ld_scales) {
  griddep_launch_dependents();
  constexpr int kGroups = kQuantThreads / kQuantLanes;
  const int lane = threadIdx.x % kQuantLanes;
  const long row0 = (long)blockIdx.y * rows_each;
  const uint32_t items = (uint32_t)min((long)rows_each, rows - row0) * (uint32_t)blocks;
  const uint32_t first = (uint32_t)blockIdx.x * (kGroups * kQuantItems) + threadIdx.x / kQuantLanes;
  x += row0 * ldx;
  codes += row0 * ld_codes;
  scales += row0 * 4;
  Sixteen<T> raw[kQuantItems];
  uint32_t row[kQuantItems];
  int b[kQuantItems], n[kQuantItems];  // block of the row; this lane's elements of it
#pragma unroll
  for (int u = 0; u < kQuantItems; ++u) {
    const uint32_t item = first + u * kGroups;
    row[u] = __umulhi(item, magic) + (blocks == 1 ? item : 0u);
    b[u] = (int)(item - row[u] * blocks);
    const int c = b[u] * kScaleBlock + lane * kQuantEach;
    n[u] = item < items ? min(kQuantEach, k - c) : 0;
    const T* from = x + (long)row[u] * ldx + c;
    if (kAligned && n[u] == kQuantEach) load_whole(from, raw[u]);
    else load_some(from, n[u], raw[u]);
  }
#pragma unroll
  for (int u = 0; u < kQuantItems; ++u) {
    uint32_t top = top_of(raw[u]);
#pragma unroll
    for (int o = kQuantLanes / 2; o > 0; o /= 2) top = max(top, __shfl_xor_sync(0xffffffffu, top, o));
    if (first + u * kGroups >= items) continue;
    const int e = (int)(top >> 23);
    const int scale = top == 0 ? 127 : e == 255 ? 255 : max(e - 8 + ((top & 0x7fffffu) > 0x600000u ? 1 : 0), 1);
    // 1 / s is a power of two as well: the products are exact, or so small that their code is zero either way
    const float inv = scale == 255 ? 0.f : __uint_as_float((uint32_t)(254 - scale) << 23);
    uint32_t word[4];
#pragma unroll
    for (int h = 0; h < 4; ++h) {
      const float2 p = pair_of(raw[u], 2 * h), q = pair_of(raw[u], 2 * h + 1);
      const uint32_t lo = __nv_cvt_float2_to_fp8x2(make_float2(p.x * inv, p.y * inv), __NV_SATFINITE, __NV_E4M3);
      const uint32_t hi = __nv_cvt_float2_to_fp8x2(make_float2(q.x * inv, q.y * inv), __NV_SATFINITE, __NV_E4M3);
      word[h] = scale == 255 ? 0u : lo | (hi << 16);
    }
    unsigned char* to = codes + (long)row[u] * ld_codes + b[u] * kScaleBlock + lane * kQuantEach;
    if (n[u] == kQuantEach) {
      *reinterpret_cast<uint4*>(to) = make_uint4(word[0], word[1], word[2], word[3]);
    } else {
#pragma unroll
      for (int i = 0; i < kQuantEach; ++i)
        if (i < n[u]) to[i] = (unsigned char)(word[i >> 2] >> (8 * (i & 3)));
    }
    unsigned char* mark = scales + ((b[u] >> 2) * ld_scales + (long)row[u]) * 4 + (b[u] & 3);
    if (lane == 0) *mark = (unsigned char)scale;
    // a row's last word has all its bytes
    if (b[u] == blocks - 1 && lane > 0 && lane <= 3 - (b[u] & 3)) mark[lane] = 127;
  }
}

// ---------------------------------------------------------------------------------------------
constexpr int kTileN = 128;  // rows of W that a block has in a tile: the accumulator's lanes
constexpr int kBlockBytes = 128;
constexpr int kEpiWarps = 16, kScaleWarp = kEpiWarps, kCopyWarp = kScaleWarp + 4, kMathWarp = kCopyWarp + 1;
constexpr int kEpiTurns = kEpiWarps / 4;
constexpr int kGemmThreads = (kMathWarp + 1) * 32;
constexpr int kStoreRows = 16;                         // rows of C, all 128 columns, that four warps turn round in shared memory at a time
constexpr int kStoreBytes = kStoreRows * kTileN * 2;   // two such pieces for each four warps
constexpr int kScaleCols = 512 - 24;  // tensor memory: two buffers of 4 columns of W's scales and 8 of A's

// Whether a barrier's phase is over, without waiting for it.
__device__ __forceinline__ bool mbar_test(uint32_t bar, uint32_t parity) {
  uint32_t ok;
  asm volatile(
      "{\n\t.reg .pred p;\n\t"
      "mbarrier.test_wait.parity.shared::cta.b64 p, [%1], %2;\n\t"
      "selp.u32 %0, 1, 0, p;\n\t}"
      : "=r"(ok)
      : "r"(bar), "r"(parity)
      : "memory");
  return ok != 0;
}
template <int CG>
__device__ __forceinline__ void umma_e4m3(uint32_t d_tmem, uint64_t adesc, uint64_t bdesc, uint32_t idesc, uint32_t sa, uint32_t sb,
                                          uint32_t accumulate) {
  if constexpr (CG == 1)
    asm volatile(
        "{\n\t.reg .pred p;\n\t"
        "setp.ne.b32 p, %6, 0;\n\t"
        "tcgen05.mma.cta_group::1.kind::mxf8f6f4.block_scale.scale_vec::1X [%0], %1, %2, %3, [%4], [%5], p;\n\t}"
        ::"r"(d_tmem), "l"(adesc), "l"(bdesc), "r"(idesc), "r"(sa), "r"(sb), "r"(accumulate)
        : "memory");
  else
    asm volatile(
        "{\n\t.reg .pred p;\n\t"
        "setp.ne.b32 p, %6, 0;\n\t"
        "tcgen05.mma.cta_group::2.kind::mxf8f6f4.block_scale.scale_vec::1X [%0], %1, %2, %3, [%4], [%5], p;\n\t}"
        ::"r"(d_tmem), "l"(adesc), "l"(bdesc), "r"(idesc), "r"(sa), "r"(sb), "r"(accumulate)
        : "memory");
}
// Instruction descriptor: e4m3 operands, both K-major, scales 2^(b - 127); `number` picks the byte of a scale column.
__device__ __forceinline__ constexpr uint32_t e4m3_idesc(int M, int N, int number) {
  return ((uint32_t)number << 4) | ((uint32_t)(N >> 3) << 17) | (1u << 23) | ((uint32_t)(M >> 7) << 27) | ((uint32_t)number << 29);
}
__device__ __forceinline__ void tmem_st_x4(uint32_t taddr, const uint32_t* r) {
  asm volatile("tcgen05.st.sync.aligned.32x32b.x4.b32 [%0], {%1, %2, %3, %4};" ::"r"(taddr), "r"(r[0]), "r"(r[1]), "r"(r[2]), "r"(r[3]) : "memory");
}
__device__ __forceinline__ void tmem_ld_x8(uint32_t taddr, uint32_t (&r)[8]) {
  asm volatile("tcgen05.ld.sync.aligned.32x32b.x8.b32 {%0, %1, %2, %3, %4, %5, %6, %7}, [%8];"
               : "=r"(r[0]), "=r"(r[1]), "=r"(r[2]), "=r"(r[3]), "=r"(r[4]), "=r"(r[5]), "=r"(r[6]), "=r"(r[7])
               : "r"(taddr)
               : "memory");
}
// 16 lanes x 16 columns as matrix fragments: thread t has columns 2 (t % 4), + 1 of lane t / 4 (r[0], r[1]) and of lane
// t / 4 + 8 (r[2], r[3]), and the same eight columns further on (r[4] .. r[7]).
__device__ __forceinline__ void tmem_ld_fragments(uint32_t taddr, uint32_t* r) {
  asm volatile("tcgen05.ld.sync.aligned.16x256b.x2.b32 {%0, %1, %2, %3, %4, %5, %6, %7}, [%8];"
               : "=r"(r[0]), "=r"(r[1]), "=r"(r[2]), "=r"(r[3]), "=r"(r[4]), "=r"(r[5]), "=r"(r[6]), "=r"(r[7])
               : "r"(taddr)
               : "memory");
}
// Four 8 x 8 matrices of 16-bit elements, transposed on their way: thread t names the 16 bytes of row t % 8 of matrix t / 8.
__device__ __forceinline__ void stmatrix_trans(uint32_t addr, uint32_t a, uint32_t b, uint32_t c, uint32_t d) {
  asm volatile("stmatrix.sync.aligned.m8n8.x4.trans.shared.b16 [%0], {%1, %2, %3, %4};" ::"r"(addr), "r"(a), "r"(b), "r"(c), "r"(d) : "memory");
}
__device__ __forceinline__ void tmem_st_x8(uint32_t taddr, const uint32_t* r) {
  asm volatile("tcgen05.st.sync.aligned.32x32b.x8.b32 [%0], {%1, %2, %3, %4, %5, %6, %7, %8};" ::"r"(taddr), "r"(r[0]), "r"(r[1]), "r"(r[2]),
               "r"(r[3]), "r"(r[4]), "r"(r[5]), "r"(r[6]), "r"(r[7])
               : "memory");
}

// Shared memory of a block.  BN: rows of A in a tile; CG: blocks that share the tile (each has 128 rows of W and BN / CG of A);
// kSplit: room for the partial sums of a split, 128 x BN float32, in place of the pieces of C that are turned round.
template <int BN, int CG, bool kSplit>
struct E4m3Plan {
  static constexpr int kWBytes = kTileN * kBlockBytes, kABytes = BN / CG * kBlockBytes;
  static constexpr int kStageBytes = kWBytes + kABytes;
  static constexpr int kSideBytes = kSplit ? kTileN * BN * 4 : kEpiTurns * 2 * kStoreBytes;
  static constexpr int kFit = (225 * 1024 - kSideBytes) / kStageBytes;
  static constexpr int kStages = kFit > 12 ? 12 : kFit;
  static constexpr int kBars = 2 * kStages + 9;  // full, empty, scales full / empty, accumulator full / empty, drain
  static constexpr int kSideOffset = kStages * kStageBytes;
  static constexpr int kBarOffset = kSideOffset + kSideBytes;
  static constexpr int kBytes = kBarOffset + 8 * kBars + 16 + 1024;
  static_assert(2 * BN <= kScaleCols && kABytes % 1024 == 0 && kStages >= 4 && kBytes <= 227 * 1024, "tile plan");
};

// The four bytes of scales of `row` that belong to blocks 4 g .. 4 g + 3; rows that do not exist count as 1.
__device__ __forceinline__ uint32_t scale_word(const E4m3Operand& x, long row, long rows, int g) {
  return row < rows ? __ldg(x.scales + g * x.scale_ld + row) : 0x7f7f7f7fu;
}

// GELU for bfloat16 outputs, two values: x Phi(x) = max(x, 0) - |x| h, h = erfc(|x| / sqrt 2) / 2 = 2^q with q(|x|) a polynomial
// of degree 7 fitted to log2 h over [0, 7], evaluated in float32: relative error 4e-6 up to |x| = 3, 8e-6 to 5, 6e-5 to 7, 4e-3 at
// 8; from there it falls faster than h does, to 0 at 16.  Half a step of bfloat16 is 4e-3.  (Degree 5 over [0, 5.5] was one
// instruction a value shorter, but 1.6e-4 off, and a constant below -5.5.)  Some eight instructions a value; erff takes some 30, which would
// bound the kernel (at 1280 channels a tile's products take 20 issue slots per value of C).  NaN for NaN and -infinity, as gelu_erf.
__device__ __forceinline__ void gelu_pair(float& x0, float& x1) {
  auto both = [](float c) { return pack_f32x2(c, c); };
  const uint64_t n = pack_f32x2(fmaxf(-fabsf(x0), -16.f), fmaxf(-fabsf(x1), -16.f));
  uint64_t q = fma_f32x2(n, both(1.76883373e-06f), both(6.03389999e-05f));
  q = fma_f32x2(n, q, both(9.21197818e-04f));
  q = fma_f32x2(n, q, both(8.47389456e-03f));
  q = fma_f32x2(n, q, both(5.38961962e-02f));
  q = fma_f32x2(n, q, both(-4.58523482e-01f));
  q = fma_f32x2(n, q, both(1.15122795f));
  q = fma_f32x2(n, q, both(-0.999997795f));
  float q0, q1;
  unpack_f32x2(q, q0, q1);
  const uint64_t p = fma_f32x2(pack_f32x2(x0, x1), both(0.5f), pack_f32x2(0.5f * fabsf(x0), 0.5f * fabsf(x1)));  // max(x, 0), exactly
  unpack_f32x2(fma_f32x2(n, pack_f32x2(ex2_approx(q0), ex2_approx(q1)), p), x0, x1);
}

// Whether all 128 threads that share barrier `id` say so.
__device__ __forceinline__ bool all_of_128(int id, bool mine) {
  uint32_t all;
  asm volatile(
      "{\n\t.reg .pred p, q;\n\t"
      "setp.ne.u32 p, %2, 0;\n\t"
      "bar.red.and.pred q, %1, 128, p;\n\t"
      "selp.u32 %0, 1, 0, q;\n\t}"
      : "=r"(all)
      : "r"(id), "r"((uint32_t)mine)
      : "memory");
  return all != 0;
}

// Bias and activation of NC accumulator columns, and their store: v[i] belongs to row r0 + i of C and to this lane's column.
template <int NC>
__device__ __forceinline__ void finish(const E4m3GemmParams& p, int r0, int col, float bias, float (&v)[NC]) {
  const bool wide = p.out_dtype == WF_F32;
  const uint64_t b2 = pack_f32x2(bias, bias);
#pragma unroll
  for (int i = 0; i < NC; i += 2) unpack_f32x2(add_f32x2(pack_f32x2(v[i], v[i + 1]), b2), v[i], v[i + 1]);
  if (p.gelu) {
#pragma unroll
    for (int i = 0; i < NC; i += 2) {
      if (wide) v[i] = gelu_erf(v[i]), v[i + 1] = gelu_erf(v[i + 1]);
      else gelu_pair(v[i], v[i + 1]);
    }
  }
  const bool whole = r0 + NC <= p.m;
  if (wide) {
    float* out = reinterpret_cast<float*>(p.out) + (long)r0 * p.ldc + col;
    if (col < p.n) {
#pragma unroll
      for (int i = 0; i < NC; ++i)
        if (whole || r0 + i < p.m) out[(long)i * p.ldc] = v[i];
    }
    return;
  }
  __nv_bfloat16* out = reinterpret_cast<__nv_bfloat16*>(p.out);
  if (((p.ldc & 1) == 0) && ((uintptr_t)p.out & 3) == 0) {
    // two lanes swap halves of two rows, so that each writes four bytes of one of them
    const int odd = threadIdx.x & 1, even_col = col - odd;
    const uint32_t pick = odd ? 0x3276u : 0x5410u;
    __nv_bfloat16* to = out + (long)(r0 + odd) * p.ldc + even_col;
    const bool both = even_col + 1 < p.n, one = even_col < p.n;
#pragma unroll
    for (int i = 0; i < NC; i += 2) {
      const __nv_bfloat162 mine = __floats2bfloat162_rn(v[i], v[i + 1]);
      const uint32_t word = *reinterpret_cast<const uint32_t*>(&mine);
      const uint32_t two = __byte_perm(word, __shfl_xor_sync(0xffffffffu, word, 1), pick);
      if (whole || r0 + i + odd < p.m) {
        if (both) *reinterpret_cast<uint32_t*>(to) = two;
        else if (one) *to = __ushort_as_bfloat16((unsigned short)two);
      }
      to += 2 * p.ldc;
    }
  } else if (col < p.n) {
#pragma unroll
    for (int i = 0; i < NC; ++i)
      if (whole || r0 + i < p.m) out[(long)(r0 + i) * p.ldc + col] = __float2bfloat16_rn(v[i]);
  }
}

template <int NC>
__device__ __forceinline__ void finish_nan(const E4m3GemmParams& p, int r0, int col) {
  float v[NC];
#pragma unroll
  for (int i = 0; i < NC; ++i) v[i] = __uint_as_float(0x7fc00000u);
  finish(p, r0, col, 0.f, v);
}

// A tile is 128 rows of W for each block by BN rows of A: W's rows are the lanes of the accumulator, so that a handful of rows
// of A costs a handful of columns, and C's rows are written in runs of 128 columns (by way of shared memory, bfloat16 rows of whole
// 16-byte chunks) or of 32 per warp (float32, other rows, the last columns, splits).
//   warps 0..15   read the accumulator (warp w the quarter w % 4 of its lanes; four turns, w / 4, take pieces of its columns alternately), apply
//                 bias and activation, store
//   warps 16..19  bring the scales of 512 channels to tensor memory (each its quarter of the lanes, which hold copies)
//   warp 20       one lane issues the TMA copies of the codes
//   warp 21       issues the products: all of it walks along, one lane issues
// CG = 2: a pair of blocks shares a tile of 256 rows of W by BN of A, each block stages its own 128 rows of W and half of A's.
// The copies of both signal the first block's barriers, which alone issues the products; its commits reach both.
// The queue of products is short: what the issuing warp does between two stages shows (it walks whole, so that descriptors stay in
// uniform registers: without GELU 344 us with a single lane, 287 so, 49,600 x 5120 x 1280), and the epilogue shares its schedulers.
// That product takes 259 us in a short burst (2.51 PFLOP/s; by the box 254 to 277) and 298 for seconds on end (SMs at 1.3 GHz under the power
// cap), with GELU 285 (to 308) and 327; n and k exchanged 221 to 239 and 265.  Float32 outputs: 318 us, 464 with GELU (erff).  64 rows by
// 50,021 x 1280, float32 out: 15.3 us, with the output 77 % of the copy rate; bfloat16 rows of odd length, stored by two bytes a lane, 15.0
// (50,048: 14.2), 4000 of them 291 us (231).
// kSplit: a cluster of blocks shares a tile, each has a part of the channels; every block sums a part of the columns, in the
// order of the blocks, from what the others leave in its shared memory.
template <int BN, int CG, bool kSplit>
__global__ void __launch_bounds__(kGemmThreads, 1) gemm_e4m3_kernel(const __grid_constant__ CUtensorMap tmap_w,
                                                                   const __grid_constant__ CUtensorMap tmap_a,
                                                                   const __grid_constant__ E4m3GemmParams p, int split, int wide_rows) {
  static_assert(CG == 1 || !kSplit, "pairs do not split");
  using Plan = E4m3Plan<BN, CG, kSplit>;
  constexpr int kStages = Plan::kStages;
  extern __shared__ uint8_t smem_raw[];
  const uint32_t smem_base = (smem_u32(smem_raw) + 1023u) & ~1023u;
  uint8_t* smem_gen = smem_raw + (smem_base - smem_u32(smem_raw));
  const uint32_t bars = smem_base + Plan::kBarOffset;
  auto full_bar = [&](int s) { return bars + 8u * s; };
  auto empty_bar = [&](int s) { return bars + 8u * (kStages + s); };
  auto sfull_bar = [&](int b) { return bars + 8u * (2 * kStages + b); };
  auto sempty_bar = [&](int b) { return bars + 8u * (2 * kStages + 2 + b); };
  auto tfull_bar = [&](int a) { return bars + 8u * (2 * kStages + 4 + a); };
  auto tempty_bar = [&](int a) { return bars + 8u * (2 * kStages + 6 + a); };
  const uint32_t drain_bar = bars + 8u * (2 * kStages + 8);
  volatile uint32_t* tmem_slot = reinterpret_cast<volatile uint32_t*>(smem_gen + Plan::kBarOffset + 8 * Plan::kBars);
  volatile int* abort_flag = reinterpret_cast<volatile int*>(smem_gen + Plan::kBarOffset + 8 * Plan::kBars + 8);
  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
  const int rank = CG == 2 || kSplit ? (int)cluster_ctarank() : 0;

  if (threadIdx.x == 0) {
    for (int s = 0; s < kStages; ++s) {
      mbar_init(full_bar(s), 1);
      mbar_init(empty_bar(s), 1);
    }
    for (int b = 0; b < 2; ++b) {
      mbar_init(sfull_bar(b), 4 * CG);
      mbar_init(sempty_bar(b), 1);
      mbar_init(tfull_bar(b), 1);
      mbar_init(tempty_bar(b), kEpiWarps * CG);
    }
    mbar_init(drain_bar, 1);
    *abort_flag = 0;
    fence_mbar_init();
  }
  if (warp == kMathWarp) {
    if constexpr (CG == 2) {
      tmem_alloc_pair(smem_u32(const_cast<uint32_t*>(tmem_slot)), 512);
      tmem_relinquish_pair();
    } else {
      tmem_alloc(smem_u32(const_cast<uint32_t*>(tmem_slot)), 512);
      tmem_relinquish();
    }
  }
  tc_fence_before();
  if constexpr (CG == 2 || kSplit) cluster_sync_all();  // every block's barriers and memory are there before another one uses them
  else __syncthreads();
  tc_fence_after();
  const uint32_t tmem = *tmem_slot;
  griddep_wait();
  griddep_launch_dependents();

  const int num_w = (p.n + CG * kTileN - 1) / (CG * kTileN), num_a = (p.m + BN - 1) / BN;
  const int num_k = (p.k + kScaleBlock - 1) / kScaleBlock;
  const int num_tiles = num_w * num_a;
  const int share = CG == 2 ? 2 : kSplit ? split : 1;  // blocks of a tile
  const int tile0 = (int)blockIdx.x / share, tile_step = (int)gridDim.x / share;
  const int kb0 = kSplit ? (int)((long)rank * num_k / split) : 0, kb1 = kSplit ? (int)((long)(rank + 1) * num_k / split) : num_k;
  auto wait = [&](uint32_t bar, uint32_t parity) { return mbar_wait_limited(bar, parity, abort_flag, p.wait_limit); };
  // Whether a warp begins at all.  (A limit of its own for each warp would say the same, and cost 0.4 us a call.)
  auto begins = [&]() {
    if (warp != p.hasty_warp) return true;
    *abort_flag = 1;
    return false;
  };
  bool done = true;  // epilogue warps of a split: the accumulator is complete
  uint32_t armed = 0, armed_parity = 0;  // copying lane: stages that copies went to, and the parity of the last ones
  bool one = false;                      // the lane that issues the products

  if (warp == kCopyWarp) {
    if (lane == 0) {
      prefetch_tmap(&tmap_w);
      prefetch_tmap(&tmap_a);
      int stage = 0;
      uint32_t phase = 0;
      bool ok = begins();
      for (int tile = tile0; ok && tile < num_tiles; tile += tile_step) {
        const int n0 = (tile % num_w * CG + (CG == 2 ? rank : 0)) * kTileN;
        const int m0 = tile / num_w * BN + (CG == 2 ? rank * (BN / 2) : 0);
        for (int kb = kb0; kb < kb1; ++kb) {
          if (!wait(empty_bar(stage), phase ^ 1u)) { ok = false; break; }
          const uint32_t at = smem_base + stage * Plan::kStageBytes;
          if constexpr (CG == 2) {
            const uint32_t bar = map_to_cta(full_bar(stage), 0);
            if (rank == 0) mbar_arrive_expect_tx(full_bar(stage), 2 * Plan::kStageBytes);
            tma_load_2d_pair(at, &tmap_w, kb * kBlockBytes, n0, bar);
            tma_load_2d_pair(at + Plan::kWBytes, &tmap_a, kb * kBlockBytes, m0, bar);
          } else {
            mbar_arrive_expect_tx(full_bar(stage), Plan::kStageBytes);
            tma_load_2d(at, &tmap_w, kb * kBlockBytes, n0, full_bar(stage));
            tma_load_2d(at + Plan::kWBytes, &tmap_a, kb * kBlockBytes, m0, full_bar(stage));
          }
          armed |= 1u << stage;
          armed_parity = (armed_parity & ~(1u << stage)) | (phase << stage);
          if (++stage == kStages) { stage = 0; phase ^= 1u; }
        }
      }
    }
  } else if (warp == kMathWarp) {
    // The whole warp walks along (so that descriptors stay in uniform registers), one lane issues.
    if (CG == 1 || rank == 0) {
      one = elect_one();
      auto commit = [&](uint32_t bar) {  // (by the electing lane)
        if constexpr (CG == 2) umma_commit_pair(bar, 3);
        else umma_commit(bar);
      };
      auto ready = [&](uint32_t bar, uint32_t parity) { return __all_sync(0xffffffffu, wait(bar, parity)); };
      auto seen = [&](uint32_t bar, uint32_t parity) { return __all_sync(0xffffffffu, mbar_test(bar, parity)); };
      const uint64_t desc = umma_desc_k_sw128(0) + ((smem_base & 0x3ffff) >> 4);
      int stage = 0, acc = 0, buf = 0;
      uint32_t phase = 0, acc_phase = 0, buf_phase = 0;
      bool ok = begins(), full_seen = false, scales_seen = false;
      for (int tile = tile0; ok && tile < num_tiles; tile += tile_step) {
        if (!ready(tempty_bar(acc), acc_phase ^ 1u)) { ok = false; break; }
        const uint32_t to = tmem + acc * BN;
        uint32_t more = 0;  // the tile's first product overwrites the accumulator
        for (int g = kb0 >> 2; ok && 4 * g < kb1; ++g) {
          if (!scales_seen && !ready(sfull_bar(buf), buf_phase)) { ok = false; break; }
          const uint32_t scales = tmem + kScaleCols + 12 * buf, free_scales = sempty_bar(buf);
          if (++buf == 2) { buf = 0; buf_phase ^= 1u; }
#pragma unroll
          for (int number = 0; number < 4; ++number) {
            const int kb = 4 * g + number;
            if ((kSplit && kb < kb0) || kb >= kb1) continue;
            if (!full_seen && !ready(full_bar(stage), phase)) { ok = false; break; }
            tc_fence_after();
            const uint64_t wdesc = desc + (uint32_t)stage * (uint32_t)(Plan::kStageBytes >> 4), adesc = wdesc + (Plan::kWBytes >> 4);
            const uint32_t empty = empty_bar(stage);
            const bool last = number == 3 || kb == kb1 - 1;
            if (++stage == kStages) { stage = 0; phase ^= 1u; }
            if (one) {
#pragma unroll
              for (int j = 0; j < 4; ++j)  // 32 channels: 32 bytes further inside the swizzled row
                umma_e4m3<CG>(to, wdesc + 2 * j, adesc + 2 * j, e4m3_idesc(CG * kTileN, BN, number), scales, scales + 4, j != 0 ? 1u : more);
              commit(empty);
              if (last) commit(free_scales);
              if (kb == kb1 - 1) commit(tfull_bar(acc));
            }
            __syncwarp();
            more = 1;
            // The next stage (and scales) are looked for while these products run: the queue of products is short, and
            // waiting behind them would leave the tensor cores idle for the time of a look.
            full_seen = seen(full_bar(stage), phase);
            if (last) scales_seen = seen(sfull_bar(buf), buf_phase);
          }
        }
        if (!ok) break;
        if (++acc == 2) { acc = 0; acc_phase ^= 1u; }
      }
    }
  } else if (warp >= kScaleWarp) {
    const uint32_t lanes = (uint32_t)((warp & 3) * 32) << 16;
    int buf = 0;
    uint32_t buf_phase = 0;
    bool ok = begins();
    // words are loaded two groups ahead: a load takes longer than the products of a group
    struct Words {
      uint32_t w[4], a[8];
    };
    int tile_next = tile0;
    int g_next = kb0 >> 2;
    auto load = [&](Words& x) {
      if (tile_next >= num_tiles) return;
      const int n0 = (tile_next % num_w * CG + (CG == 2 ? rank : 0)) * kTileN, m0 = tile_next / num_w * BN;
#pragma unroll
      for (int i = 0; i < 4; ++i) x.w[i] = scale_word(p.w, n0 + 32 * i + lane, p.n, g_next);
#pragma unroll
      for (int i = 0; i < 8; ++i) x.a[i] = 32 * i < BN ? scale_word(p.a, m0 + 32 * i + lane, p.m, g_next) : 0x7f7f7f7fu;
      if (4 * ++g_next >= kb1) {
        g_next = kb0 >> 2;
        tile_next += tile_step;
      }
    };
    auto pass = [&](const Words& x) {  // to tensor memory, behind the last product that used the buffer
      ok = __all_sync(0xffffffffu, wait(sempty_bar(buf), buf_phase ^ 1u));
      if (!ok) return;
      tc_fence_after();
      const uint32_t to = tmem + lanes + kScaleCols + 12 * buf;
      tmem_st_x4(to, x.w);
      if (BN <= 128) tmem_st_x4(to + 4, x.a);
      else tmem_st_x8(to + 4, x.a);
      tmem_st_wait();
      tc_fence_before();
      __syncwarp();
      if (lane == 0) {
        if constexpr (CG == 2) mbar_arrive_cluster(map_to_cta(sfull_bar(buf), 0));
        else mbar_arrive(sfull_bar(buf));
      }
      if (++buf == 2) { buf = 0; buf_phase ^= 1u; }
    };
    const int groups = tile0 < num_tiles ? ((num_tiles - tile0 + tile_step - 1) / tile_step) * (((kb1 + 3) >> 2) - (kb0 >> 2)) : 0;
    Words even, odd;
    load(even);
    load(odd);
    for (int i = 0; ok && i < groups; i += 2) {
      pass(even);
      load(even);
      if (!ok || i + 1 >= groups) break;
      pass(odd);
      load(odd);
    }
  } else if constexpr (!kSplit) {
    const int quarter = warp & 3, turn = warp >> 2;
    int acc = 0, pieces = 0;
    uint32_t acc_phase = 0;
    bool ok = begins();
    // What does not depend on the tile.  Pieces of 16 rows by 128 columns: in shared memory a row is two halves of 128 bytes,
    // 16-byte chunks exclusive-or'd with the row against bank conflicts.  A thread names a row of a matrix to be stored, and
    // copies a chunk of two rows out.
    const int chunk_in = (quarter & 1) * 4 + (lane >> 3), row_out = quarter * 4 + (lane >> 4), chunk_out = lane & 15;
    const uint32_t area = smem_base + Plan::kSideOffset + (uint32_t)(turn * 2 * kStoreBytes);
    const uint32_t in = area + (quarter >> 1) * (kStoreBytes / 2) + (lane & 7) * 128 + ((chunk_in ^ (lane & 7)) << 4);
    const uint32_t out_a = area + (chunk_out >> 3) * (kStoreBytes / 2) + row_out * 128 + (((chunk_out & 7) ^ (row_out & 7)) << 4);
    const uint32_t out_b = out_a ^ ((2u << 4) | (2u * 128u));  // two rows on (row_out is even in its second bit: 0, 1, 4, 5, ..)
    const long two_rows = 2 * p.ldc, next_piece = 16L * kEpiTurns * p.ldc - two_rows;
    const uint32_t lanes_at = (uint32_t)(quarter * 32) << 16;
    int wn = tile0 % num_w, wm = tile0 / num_w;
    const int step_n = tile_step % num_w, step_m = tile_step / num_w;
    for (int tile = tile0; tile < num_tiles; tile += tile_step) {
      const int n0 = (wn * CG + (CG == 2 ? rank : 0)) * kTileN, m0 = wm * BN;
      wn += step_n;
      wm += step_m;
      if (wn >= num_w) wn -= num_w, ++wm;
      const int col = n0 + quarter * 32 + lane, stop = min(BN, p.m - m0);
      // (the four warps of a turn share barriers further down: they go on together or not at all)
      ok = all_of_128(1 + turn, ok && __all_sync(0xffffffffu, wait(tfull_bar(acc), acc_phase)));
      const bool pieces_of_16 = wide_rows && n0 + kTileN <= p.n;
      const int begin = turn ^ (acc << 1);  // (14 pieces for four turns: those that take one more change with the tile)
      if (!ok) {  // what was not computed is NaN: the rows that these warps would have stored, the other turns may have theirs
        if (lane == 0) report(p.status, kGaveUp);
        const int each = pieces_of_16 ? 16 : 8;
        for (int c = (pieces_of_16 ? begin : turn) * each; c < stop; c += each * kEpiTurns)
          for (int i = 0; i < each; i += 8) finish_nan<8>(p, m0 + c + i, col);
        acc ^= 1;
        continue;
      }
      tc_fence_after();
      const uint32_t from = tmem + lanes_at + acc * BN;
      if (pieces_of_16) {
        float b4[4] = {0.f, 0.f, 0.f, 0.f};  // of this thread's lanes of the fragments
        if (p.bias) {
          const int first = n0 + quarter * 32 + (lane >> 2);
#pragma unroll
          for (int i = 0; i < 4; ++i)
            b4[i] = __ldg(p.bias + first + 8 * i);
        }
        __nv_bfloat16* to = reinterpret_cast<__nv_bfloat16*>(p.out) + (long)(m0 + begin * 16 + row_out) * p.ldc + n0 + chunk_out * 8;
        auto copy_out = [&](uint32_t from_smem, bool exists) {
          uint4 u;
          ld_shared_v4(from_smem, u.x, u.y, u.z, u.w);
          if (exists) *reinterpret_cast<uint4*>(to) = u;
        };
#pragma unroll 1
        for (int c = begin * 16; c < stop; c += 16 * kEpiTurns) {
          uint32_t r[16];
          tmem_ld_fragments(from + c, r);
          tmem_ld_fragments(from + (16u << 16) + c, r + 8);
          tmem_ld_wait();
          float v[16];
          uint32_t word[8];  // [lanes 0 .. 7, 8 .. 15, 16 .. 23, 24 .. 31] of eight columns, then of the next eight
#pragma unroll
          for (int i = 0; i < 8; ++i) {
            const float b = b4[(i & 1) | (i >> 2) << 1];
            unpack_f32x2(add_f32x2(pack_f32x2(__uint_as_float(r[2 * i]), __uint_as_float(r[2 * i + 1])), pack_f32x2(b, b)), v[2 * i], v[2 * i + 1]);
          }
          if (p.gelu) {
#pragma unroll
            for (int i = 0; i < 8; ++i) gelu_pair(v[2 * i], v[2 * i + 1]);
          }
#pragma unroll
          for (int i = 0; i < 8; ++i) {
            const __nv_bfloat162 two = __floats2bfloat162_rn(v[2 * i], v[2 * i + 1]);
            word[((i >> 1) & 1) * 4 + ((i & 1) | (i >> 2) << 1)] = *reinterpret_cast<const uint32_t*>(&two);
          }
          const uint32_t side = (uint32_t)(pieces++ & 1) * kStoreBytes;
          stmatrix_trans(in + side, word[0], word[1], word[2], word[3]);
          stmatrix_trans(in + side + 8 * 128, word[4], word[5], word[6], word[7]);
          asm volatile("bar.sync %0, 128;" ::"r"(1 + turn) : "memory");  // (the other piece has been read by then)
          copy_out(out_a + side, c + row_out < stop);
          to += two_rows;
          copy_out(out_b + side, c + row_out + 2 < stop);
          to += next_piece;
        }
      } else {
        const float bias = p.bias && col < p.n ? __ldg(p.bias + col) : 0.f;
        uint32_t next[8];
        if (turn * 8 < stop) tmem_ld_x8(from + turn * 8, next);
#pragma unroll 1
        for (int c = turn * 8; c < stop; c += 8 * kEpiTurns) {
          float v[8];
          tmem_ld_wait();
#pragma unroll
          for (int i = 0; i < 8; ++i) v[i] = __uint_as_float(next[i]);
          if (c + 8 * kEpiTurns < stop) tmem_ld_x8(from + c + 8 * kEpiTurns, next);
          finish(p, m0 + c, col, bias, v);
        }
      }
      tc_fence_before();
      __syncwarp();
      if (lane == 0) {
        if constexpr (CG == 2) mbar_arrive_cluster(map_to_cta(tempty_bar(acc), 0));
        else mbar_arrive(tempty_bar(acc));
      }
      if (++acc == 2) { acc = 0; acc_phase ^= 1u; }
    }
  } else {
    // ---- a split: this block's sums of every other block's columns go there (one tile per cluster).  Partial sums of block r
    // lie at [r][column / 4][row][4] of the receiving block.
    const int quarter = warp & 3, turn = warp >> 2, row = quarter * 32 + lane, mine = BN / split;
    done = begins() && __all_sync(0xffffffffu, wait(tfull_bar(0), 0));
    tc_fence_after();
    const uint32_t from = tmem + ((uint32_t)(quarter * 32) << 16);
#pragma unroll 1
    for (int c = turn * 8; c < BN; c += 8 * kEpiTurns) {
      uint32_t r[8];
      if (done) {
        tmem_ld_x8(from + c, r);
        tmem_ld_wait();
      } else {
#pragma unroll
        for (int i = 0; i < 8; ++i) r[i] = 0x7fc00000u;
      }
#pragma unroll
      for (int q = 0; q < 2; ++q) {
        const int column = c + 4 * q, owner = column / mine, within = (rank * mine + column - owner * mine) / 4;
        st_cluster_v4(map_to_cta(smem_base + Plan::kSideOffset + (uint32_t)(within * kTileN + row) * 16u, owner), r[4 * q], r[4 * q + 1],
                      r[4 * q + 2], r[4 * q + 3]);
      }
    }
    if (!done && lane == 0) report(p.status, kGaveUp);
  }

  tc_fence_before();
  __syncwarp();
  if constexpr (CG == 2) {  // what one block of a pair has given up, the other one hears of
    __syncthreads();
    if (threadIdx.x == 0 && *abort_flag) st_cluster_v2(map_to_cta(bars + 8u * Plan::kBars + 8u, rank ^ 1), 1u, 0u);
    __syncwarp();
  }
  if constexpr (CG == 2 || kSplit) cluster_sync_all();  // partial sums are there; nobody leaves while another one may still use its memory
  else __syncthreads();
  if (*abort_flag) {
    // Somebody has given up.  Copies and products in flight, which those who issued them need not have waited for, end before the
    // block's memory and tensor memory are given back (where nobody has, the accumulators were complete, and so all copies).
    // The second block of a pair sees its copies only by their stages being released, and the first one waits for both blocks'
    // bytes: where these do not come, what is still in flight has the time of the looks, hundreds of microseconds or more.
    if (warp == kCopyWarp && lane == 0) {
      uint32_t looks = CG == 2 ? 1u << 14 : kWaitLimit;
#pragma unroll 1
      for (int s = 0; s < kStages; ++s)
        if (armed >> s & 1u) {
          const uint32_t bar = CG == 2 && rank == 1 ? empty_bar(s) : full_bar(s);
          while (looks > 0 && !mbar_try_wait(bar, armed_parity >> s & 1u)) --looks;
        }
    } else if (warp == kMathWarp && (CG == 1 || rank == 0)) {
      if (one) {
        if constexpr (CG == 2) umma_commit_pair(drain_bar, 1);
        else umma_commit(drain_bar);
      }
      __syncwarp();
      for (uint32_t it = 0; it < kWaitLimit && !mbar_try_wait(drain_bar, 0); ++it) {}
    }
    if constexpr (CG == 2) {
      __syncwarp();
      cluster_sync_all();
    }
  }
  if (warp == kMathWarp) {
    tc_fence_after();
    if constexpr (CG == 2) tmem_dealloc_pair(tmem, 512);
    else tmem_dealloc(tmem, 512);
  }
  if constexpr (kSplit) {
    if (warp < kEpiWarps) {
      const int quarter = warp & 3, turn = warp >> 2, row = quarter * 32 + lane, mine = BN / split;
      const int n0 = tile0 % num_w * kTileN, m0 = tile0 / num_w * BN + rank * mine;
      const int col = n0 + row;
      const float bias = p.bias && col < p.n ? __ldg(p.bias + col) : 0.f;
      for (int c = turn * 4; c < mine && m0 + c < p.m; c += 4 * kEpiTurns) {
        float v[4] = {0.f, 0.f, 0.f, 0.f};
        for (int r = 0; r < split; ++r) {
          uint32_t q[4];
          ld_shared_v4(smem_base + Plan::kSideOffset + (uint32_t)((r * mine + c) / 4 * kTileN + row) * 16u, q[0], q[1], q[2], q[3]);
#pragma unroll
          for (int i = 0; i < 4; ++i) v[i] += __uint_as_float(q[i]);
        }
        finish(p, m0 + c, col, bias, v);
      }
    }
  }
}

typedef CUresult (*EncodeTiled)(CUtensorMap*, CUtensorMapDataType, cuuint32_t, void*, const cuuint64_t*, const cuuint64_t*, const cuuint32_t*,
                                const cuuint32_t*, CUtensorMapInterleave, CUtensorMapSwizzle, CUtensorMapL2promotion, CUtensorMapFloatOOBfill);

// A matrix [rows, cols] in device memory, rows `ld` bytes apart, as boxes; what lies outside reads as zeros and is not written.
bool matrix_map(CUtensorMap* m, CUtensorMapDataType type, const void* base, long cols, long rows, long ld, int box_cols, int box_rows,
                CUtensorMapSwizzle swizzle) {
  static std::atomic<void*> encode{nullptr};  // the driver's entry point, the same for every caller
  void* fn = encode.load(std::memory_order_relaxed);
  if (fn == nullptr) {
    TmaApi api{};
    if (!tma_api_init(&api)) return false;
    encode.store(fn = api.encode_tiled, std::memory_order_relaxed);
  }
  const cuuint64_t dims[2] = {(cuuint64_t)cols, (cuuint64_t)rows}, strides[1] = {(cuuint64_t)ld};
  const cuuint32_t box[2] = {(cuuint32_t)box_cols, (cuuint32_t)box_rows}, steps[2] = {1, 1};
  return reinterpret_cast<EncodeTiled>(fn)(m, type, 2, const_cast<void*>(base), dims, strides, box, steps, CU_TENSOR_MAP_INTERLEAVE_NONE, swizzle,
                                           CU_TENSOR_MAP_L2_PROMOTION_L2_256B, CU_TENSOR_MAP_FLOAT_OOB_FILL_NONE) == CUDA_SUCCESS;
}
bool codes_map(CUtensorMap* m, const E4m3Operand& x, long rows, int k, int box_rows) {
  return matrix_map(m, CU_TENSOR_MAP_DATA_TYPE_UINT8, x.codes, k, rows, x.ld, kBlockBytes, box_rows, CU_TENSOR_MAP_SWIZZLE_128B);
}

template <int BN, int CG, bool kSplit>
cudaError_t launch_tiles(const E4m3GemmParams& p, int split, int num_sms, cudaStream_t s) {
  using Plan = E4m3Plan<BN, CG, kSplit>;
  CUtensorMap tw, ta;
  if (!codes_map(&tw, p.w, p.n, p.k, kTileN) || !codes_map(&ta, p.a, p.m, p.k, BN / CG)) return cudaErrorInvalidValue;
  // bfloat16 rows of whole 16-byte chunks go through shared memory, others (and the last columns) straight from registers
  const bool wide = p.out_dtype == WF_BF16 && ((uintptr_t)p.out & 15) == 0 && p.ldc % 8 == 0;
  const long tiles = (long)((p.n + CG * kTileN - 1) / (CG * kTileN)) * ((p.m + BN - 1) / BN);
  if (tiles * 8 > 0x7fffffffL) return cudaErrorInvalidValue;  // (C would have 2^39 elements)
  const int share = CG == 2 ? 2 : kSplit ? split : 1;
  const long groups = kSplit ? tiles : tiles < num_sms / share ? tiles : num_sms / share;
  auto kernel = gemm_e4m3_kernel<BN, CG, kSplit>;
  const cudaError_t e = cudaFuncSetAttribute(kernel, cudaFuncAttributeMaxDynamicSharedMemorySize, Plan::kBytes);
  if (e != cudaSuccess) return e;
  return launch_dependent(kernel, dim3((unsigned)(groups * share)), dim3(kGemmThreads), Plan::kBytes, s, share, true, tw, ta, p, split, (int)wide);
}

template <int BN>
cudaError_t launch_single(const E4m3GemmParams& p, int split, int num_sms, cudaStream_t s) {
  return split > 1 ? launch_tiles<BN, 1, true>(p, split, num_sms, s) : launch_tiles<BN, 1, false>(p, 1, num_sms, s);
}

}  // namespace

cudaError_t launch_quantise_e4m3(const void* x, int dtype, long ldx, long rows, int k, void* codes, long ld_codes, unsigned char* scales,
                                 long ld_scales, cudaStream_t s) {
  const int blocks = (k + kScaleBlock - 1) / kScaleBlock, per_block = kQuantThreads / kQuantLanes * kQuantItems;
  // rows that are counted through together: as many as fill 16 thread blocks, so that it counts in 32 bits (a grid has 65535 of them in y)
  long rows_each = 16 * per_block / blocks > 0 ? 16 * per_block / blocks : 1;
  if ((rows + rows_each - 1) / rows_each > 65535) rows_each = (rows + 65534) / 65535;
  if (rows_each > rows) rows_each = rows;
  const bool aligned = ((uintptr_t)x & 15) == 0 && ldx * (dtype == WF_BF16 ? 2 : 4) % 16 == 0;
  const dim3 grid((unsigned)((rows_each * blocks + per_block - 1) / per_block), (unsigned)((rows + rows_each - 1) / rows_each));
  const uint32_t magic = (uint32_t)(((1ull << 32) + blocks - 1) / blocks);
  unsigned char* c = (unsigned char*)codes;
  auto go = [&](auto kernel, auto* from) {
    return launch_dependent(kernel, grid, dim3(kQuantThreads), 0, s, 1, false, from, ldx, rows, k, blocks, magic, (int)rows_each, c, ld_codes, scales,
                            ld_scales);
  };
  if (dtype == WF_BF16) {
    auto* from = (const __nv_bfloat16*)x;
    return aligned ? go(quantise_e4m3_kernel<__nv_bfloat16, true>, from) : go(quantise_e4m3_kernel<__nv_bfloat16, false>, from);
  }
  auto* from = (const float*)x;
  return aligned ? go(quantise_e4m3_kernel<float, true>, from) : go(quantise_e4m3_kernel<float, false>, from);
}

// Which tile: rows of A (224 of them: on pairs of blocks), and over how many blocks its channels are split.  Estimated time of
// a call in us, fitted to the choice between the times measured for 55 shapes of m = 1 .. 4000, n = 640 .. 50021, k = 512 .. 5120 (it is
// within 8 % of the best tile for all but one, which loses 23 %): a launch 3.6 (1.8 more on pairs), then as many rounds of tiles as
// the SMs need, a block of 128 channels taking the time of its bytes.  One SM draws 85 GB/s, all of them together 9.4 TB/s.  A split
// costs an exchange.  Examples, one tile of the kind against another: m = 1, n = k = 1280: 16 rows split 4: 4.5, whole 4.9;
// m = 320, n = 1280, k = 5120: 128 rows split 4: 9.7, whole 12.9, pairs 14.7; m = 775, n = 5120, k = 1280: 128 rows 9.9, 64: 14.2,
// pairs 10.7; m = 4000: pairs 23, 128 rows 30.
double estimate_us(long m, long n, long k, int bn, int split, int num_sms) {
  const int cg = bn == 224 ? 2 : 1, share = cg * split;
  const long tiles = (n + kTileN * cg - 1) / (kTileN * cg) * ((m + bn - 1) / bn), blocks_k = (k + kScaleBlock - 1) / kScaleBlock;
  if (split > 1 && (tiles * split * 20 > num_sms * 19 || split > blocks_k)) return 1e30;  // (a cluster needs its blocks at one time)
  const long at_once = num_sms > share ? num_sms / share : 1, rounds = (tiles + at_once - 1) / at_once;
  const double active = (double)(tiles < at_once ? tiles : at_once) * share;
  const double rate = active * 85e3 < 9.4e6 ? 85e3 : 9.4e6 / active;  // bytes per us and SM
  const double block = (kTileN + bn / cg) * (double)kBlockBytes / rate;
  return 3.6 + (cg == 2 ? 1.8 : 0.0) + (split > 1 ? 0.8 + 0.012 * bn : 0.0) +
         (double)rounds * ((double)((blocks_k + split - 1) / split) * block + 0.006 * bn);
}

cudaError_t launch_gemm_e4m3(const E4m3GemmParams& p, int num_sms, cudaStream_t s) {
  static const int tiles[][2] = {{16, 1}, {16, 2}, {16, 4}, {32, 1}, {32, 2}, {32, 4}, {32, 8}, {64, 1}, {64, 2}, {64, 4},
                                 {64, 8}, {128, 1}, {128, 2}, {128, 4}, {128, 8}, {224, 1}};
  int bn = 0, split = 1;
  double least = 1e30;
  for (const auto& t : tiles) {
    const double us = estimate_us(p.m, p.n, p.k, t[0], t[1], num_sms);
    if (us < least) least = us, bn = t[0], split = t[1];
  }
  switch (bn) {
    case 16: return launch_single<16>(p, split, num_sms, s);
    case 32: return launch_single<32>(p, split, num_sms, s);
    case 64: return launch_single<64>(p, split, num_sms, s);
    case 128: return launch_single<128>(p, split, num_sms, s);
    default: return launch_tiles<224, 2, false>(p, 1, num_sms, s);
  }
}

}  // namespace wf
