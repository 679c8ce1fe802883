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
// Codes of the rows of x: sixteen lanes take the 128 channels of a block, eight each.
//   s = the least power of two with max |x| / s <= 448, code = x / s (exact) rounded to the nearest e4m3 value, ties to even.
constexpr int kQuantThreads = 256;
constexpr int kQuantItems = 4;  // blocks that a group of lanes has in flight

__device__ __forceinline__ void load8(const float* x, float (&v)[8]) {
  const float4 a = __ldg(reinterpret_cast<const float4*>(x)), b = __ldg(reinterpret_cast<const float4*>(x) + 1);
  v[0] = a.x, v[1] = a.y, v[2] = a.z, v[3] = a.w, v[4] = b.x, v[5] = b.y, v[6] = b.z, v[7] = b.w;
}
__device__ __forceinline__ void load8(const __nv_bfloat16* x, float (&v)[8]) {
  const uint4 u = __ldg(reinterpret_cast<const uint4*>(x));
  const uint32_t w[4] = {u.x, u.y, u.z, u.w};
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    v[2 * i] = __uint_as_float(w[i] << 16);
    v[2 * i + 1] = __uint_as_float(w[i] & 0xffff0000u);
  }
}
__device__ __forceinline__ float load1(const float* x) { return __ldg(x); }
__device__ __forceinline__ float load1(const __nv_bfloat16* x) { return __bfloat162float(*x); }

template <typename T, bool kAligned>
__global__ void __launch_bounds__(kQuantThreads) quantise_e4m3_kernel(const T* __restrict__ x, long ldx, long items, int k, int blocks,
                                                                     unsigned char* __restrict__ codes, long ld_codes,
                                                                     unsigned char* __restrict__ scales, long ld_scales) {
  griddep_launch_dependents();
  const int lane16 = threadIdx.x & 15;
  const long group = ((long)blockIdx.x * kQuantThreads + threadIdx.x) >> 4, groups = ((long)gridDim.x * kQuantThreads) >> 4;
  float v[kQuantItems][8];
#pragma unroll
  for (int u = 0; u < kQuantItems; ++u) {
    const long item = group + u * groups, row = item / blocks;
    const int c = (int)(item - row * blocks) * kScaleBlock + lane16 * 8;
    if (item < items && kAligned && c + 8 <= k) {
      load8(x + row * ldx + c, v[u]);
    } else {
#pragma unroll
      for (int e = 0; e < 8; ++e) v[u][e] = item < items && c + e < k ? load1(x + row * ldx + c + e) : 0.f;
    }
  }
#pragma unroll
  for (int u = 0; u < kQuantItems; ++u) {
    const long item = group + u * groups, row = item / blocks;
    const int b = (int)(item - row * blocks), c = b * kScaleBlock + lane16 * 8;
    uint32_t top = 0;  // as bits: a NaN or an infinity is the largest
#pragma unroll
    for (int e = 0; e < 8; ++e) top = max(top, __float_as_uint(v[u][e]) & 0x7fffffffu);
#pragma unroll
    for (int o = 8; o > 0; o /= 2) top = max(top, __shfl_xor_sync(0xffffffffu, top, o));
    if (item >= items) continue;
    const int e = (int)(top >> 23);
    const int scale = top == 0 ? 127 : e == 255 ? 255 : max(e - 8 + ((top & 0x7fffffu) > 0x600000u ? 1 : 0), 1);
    // 1 / s is a power of two as well: the products are exact, or so small that their code is zero either way
    const float inv = scale == 255 ? 0.f : __uint_as_float((uint32_t)(254 - scale) << 23);
    uint32_t word[2];
#pragma unroll
    for (int h = 0; h < 2; ++h) {
      uint32_t two[2];
#pragma unroll
      for (int j = 0; j < 2; ++j)
        two[j] = __nv_cvt_float2_to_fp8x2(make_float2(v[u][4 * h + 2 * j] * inv, v[u][4 * h + 2 * j + 1] * inv), __NV_SATFINITE, __NV_E4M3);
      word[h] = scale == 255 ? 0u : two[0] | (two[1] << 16);
    }
    unsigned char* to = codes + row * ld_codes + c;
    if (c + 8 <= k) {
      *reinterpret_cast<uint2*>(to) = make_uint2(word[0], word[1]);
    } else {
      for (int i = 0; c + i < k && i < 8; ++i) to[i] = (unsigned char)(word[i >> 2] >> (8 * (i & 3)));
    }
    if (lane16 == 0) scales[row * ld_scales + b] = (unsigned char)scale;
    // the row's scales end with the four of a word
    if (b == blocks - 1 && lane16 > 0 && lane16 <= 3 - ((blocks - 1) & 3)) scales[row * ld_scales + b + lane16] = 127;
  }
}

// ---------------------------------------------------------------------------------------------
constexpr int kTileN = 128;  // rows of W in a tile: the accumulator's lanes
constexpr int kBlockBytes = 128;
constexpr int kGemmThreads = 320;
constexpr int kScaleCols = 512 - 24;  // tensor memory: two buffers of 4 columns of W's scales and 8 of A's

__device__ __forceinline__ void umma_e4m3(uint32_t d_tmem, uint64_t adesc, uint64_t bdesc, uint32_t idesc, uint32_t sa, uint32_t sb,
                                          uint32_t accumulate) {
  asm volatile(
      "{\n\t.reg .pred p;\n\t"
      "setp.ne.b32 p, %6, 0;\n\t"
      "tcgen05.mma.cta_group::1.kind::mxf8f6f4.block_scale.scale_vec::1X [%0], %1, %2, %3, [%4], [%5], p;\n\t}"
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
__device__ __forceinline__ void tmem_st_x8(uint32_t taddr, const uint32_t* r) {
  asm volatile("tcgen05.st.sync.aligned.32x32b.x8.b32 [%0], {%1, %2, %3, %4, %5, %6, %7, %8};" ::"r"(taddr), "r"(r[0]), "r"(r[1]), "r"(r[2]),
               "r"(r[3]), "r"(r[4]), "r"(r[5]), "r"(r[6]), "r"(r[7])
               : "memory");
}

template <int BN>
struct E4m3Plan {
  static constexpr int kWBytes = kTileN * kBlockBytes, kABytes = BN * kBlockBytes;
  static constexpr int kStageBytes = kWBytes + kABytes;
  static constexpr int kFit = 216 * 1024 / kStageBytes;
  static constexpr int kStages = kFit > 12 ? 12 : kFit;
  static constexpr int kBars = 2 * kStages + 9;  // full, empty, scales full / empty, accumulator full / empty, drain
  static constexpr int kBarOffset = kStages * kStageBytes;
  static constexpr int kBytes = kBarOffset + 8 * kBars + 16 + 1024;
  static_assert(2 * BN <= kScaleCols && kStageBytes % 1024 == 0 && kBytes <= 227 * 1024, "tile plan");
};

// The four bytes of scales of `row` that belong to blocks 4 g .. 4 g + 3; rows that do not exist count as 1.
__device__ __forceinline__ uint32_t scale_word(const E4m3Operand& x, long row, long rows, int g) {
  return row < rows ? __ldg(reinterpret_cast<const uint32_t*>(x.scales + row * x.scale_ld) + g) : 0x7f7f7f7fu;
}

// One accumulator column block: `v` are 16 rows of C (from row `r0`) at column `col` (one per lane).
__device__ __forceinline__ void store16(const E4m3GemmParams& p, int r0, int col, const float (&v)[16]) {
  const int lane = threadIdx.x & 31;
  if (p.out_dtype == WF_F32) {
    float* out = reinterpret_cast<float*>(p.out) + (long)r0 * p.ldc + col;
#pragma unroll
    for (int i = 0; i < 16; ++i)
      if (r0 + i < p.m && col < p.n) out[(long)i * p.ldc] = v[i];
    return;
  }
  __nv_bfloat16* out = reinterpret_cast<__nv_bfloat16*>(p.out);
  if (((p.ldc & 1) == 0) && ((uintptr_t)p.out & 3) == 0) {
    // two lanes swap halves of two rows, so that each writes four bytes of one of them
    const int odd = lane & 1, even_col = col - odd;
#pragma unroll
    for (int i = 0; i < 16; i += 2) {
      const float other = __shfl_xor_sync(0xffffffffu, odd ? v[i] : v[i + 1], 1);
      const __nv_bfloat162 two = __floats2bfloat162_rn(odd ? other : v[i], odd ? v[i + 1] : other);
      const int r = r0 + i + odd;
      if (r < p.m) {
        __nv_bfloat16* to = out + (long)r * p.ldc + even_col;
        if (even_col + 1 < p.n) *reinterpret_cast<__nv_bfloat162*>(to) = two;
        else if (even_col < p.n) *to = two.x;
      }
    }
  } else {
#pragma unroll
    for (int i = 0; i < 16; ++i)
      if (r0 + i < p.m && col < p.n) out[(long)(r0 + i) * p.ldc + col] = __float2bfloat16_rn(v[i]);
  }
}

// A tile is 128 rows of W by BN rows of A: W's rows are the lanes of the accumulator, so that a handful of rows of A costs a
// handful of columns, and C's rows are written in runs of 32 columns per warp.
//   warps 0..3  read the accumulator, apply bias and activation, store
//   warps 4..7  bring the scales of 512 channels to tensor memory (each its quarter of the lanes, which hold copies)
//   warp 8      one lane issues the TMA copies of the codes;   warp 9  one lane issues the products
template <int BN>
__global__ void __launch_bounds__(kGemmThreads, 1) gemm_e4m3_kernel(const __grid_constant__ CUtensorMap tmap_w,
                                                                   const __grid_constant__ CUtensorMap tmap_a,
                                                                   const __grid_constant__ E4m3GemmParams p) {
  using Plan = E4m3Plan<BN>;
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

  if (threadIdx.x == 0) {
    for (int s = 0; s < kStages; ++s) {
      mbar_init(full_bar(s), 1);
      mbar_init(empty_bar(s), 1);
    }
    for (int b = 0; b < 2; ++b) {
      mbar_init(sfull_bar(b), 4);
      mbar_init(sempty_bar(b), 1);
      mbar_init(tfull_bar(b), 1);
      mbar_init(tempty_bar(b), 4);
    }
    mbar_init(drain_bar, 1);
    *abort_flag = 0;
    fence_mbar_init();
  }
  if (warp == 9) {
    tmem_alloc(smem_u32(const_cast<uint32_t*>(tmem_slot)), 512);
    tmem_relinquish();
  }
  tc_fence_before();
  __syncthreads();
  tc_fence_after();
  const uint32_t tmem = *tmem_slot;
  griddep_wait();
  griddep_launch_dependents();

  const int num_w = (p.n + kTileN - 1) / kTileN, num_a = (p.m + BN - 1) / BN, num_k = (p.k + kScaleBlock - 1) / kScaleBlock;
  const long num_tiles = (long)num_w * num_a;
  auto wait = [&](uint32_t bar, uint32_t parity) { return mbar_wait_limited(bar, parity, abort_flag, p.wait_limit); };

  if (warp == 8) {
    if (lane == 0) {
      prefetch_tmap(&tmap_w);
      prefetch_tmap(&tmap_a);
      int stage = 0;
      uint32_t phase = 0, armed = 0, armed_parity = 0;
      bool ok = true;
      for (long tile = blockIdx.x; ok && tile < num_tiles; tile += gridDim.x) {
        const int n0 = (int)(tile % num_w) * kTileN, m0 = (int)(tile / num_w) * BN;
        for (int kb = 0; kb < num_k; ++kb) {
          if (!wait(empty_bar(stage), phase ^ 1u)) { ok = false; break; }
          const uint32_t at = smem_base + stage * Plan::kStageBytes;
          mbar_arrive_expect_tx(full_bar(stage), Plan::kStageBytes);
          tma_load_2d(at, &tmap_w, kb * kBlockBytes, n0, full_bar(stage));
          tma_load_2d(at + Plan::kWBytes, &tmap_a, kb * kBlockBytes, m0, full_bar(stage));
          armed |= 1u << stage;
          armed_parity = (armed_parity & ~(1u << stage)) | (phase << stage);
          if (++stage == kStages) { stage = 0; phase ^= 1u; }
        }
      }
      if (!ok)  // no copy may land after the block has gone
        for (int s = 0; s < kStages; ++s)
          if (armed >> s & 1u)
            for (uint32_t it = 0; it < kWaitLimit && !mbar_try_wait(full_bar(s), armed_parity >> s & 1u); ++it) {}
    }
  } else if (warp == 9) {
    if (lane == 0) {
      int stage = 0, acc = 0, buf = 0;
      uint32_t phase = 0, acc_phase = 0, buf_phase = 0;
      bool ok = true;
      for (long tile = blockIdx.x; ok && tile < num_tiles; tile += gridDim.x) {
        if (!wait(tempty_bar(acc), acc_phase ^ 1u)) { ok = false; break; }
        tc_fence_after();
        for (int kb = 0; kb < num_k; ++kb) {
          if ((kb & 3) == 0 && !wait(sfull_bar(buf), buf_phase)) { ok = false; break; }
          if (!wait(full_bar(stage), phase)) { ok = false; break; }
          tc_fence_after();
          const uint32_t at = smem_base + stage * Plan::kStageBytes;
          const uint64_t wdesc = umma_desc_k_sw128(at), adesc = umma_desc_k_sw128(at + Plan::kWBytes);
          const uint32_t idesc = e4m3_idesc(kTileN, BN, kb & 3), scales = tmem + kScaleCols + 12 * buf;
#pragma unroll
          for (int j = 0; j < 4; ++j)  // 32 channels: 32 bytes further inside the swizzled row
            umma_e4m3(tmem + acc * BN, wdesc + 2 * j, adesc + 2 * j, idesc, scales, scales + 4, (kb | j) != 0 ? 1u : 0u);
          umma_commit(empty_bar(stage));
          if (++stage == kStages) { stage = 0; phase ^= 1u; }
          if ((kb & 3) == 3 || kb == num_k - 1) {
            umma_commit(sempty_bar(buf));
            if (++buf == 2) { buf = 0; buf_phase ^= 1u; }
          }
        }
        if (!ok) break;
        umma_commit(tfull_bar(acc));
        if (++acc == 2) { acc = 0; acc_phase ^= 1u; }
      }
      if (!ok) {  // products in flight end before tensor memory is given back
        umma_commit(drain_bar);
        for (uint32_t it = 0; it < kWaitLimit && !mbar_try_wait(drain_bar, 0); ++it) {}
      }
    }
  } else if (warp >= 4) {
    const uint32_t lanes = (uint32_t)((warp & 3) * 32) << 16;
    int buf = 0;
    uint32_t buf_phase = 0;
    bool ok = true;
    for (long tile = blockIdx.x; ok && tile < num_tiles; tile += gridDim.x) {
      const long n0 = (tile % num_w) * kTileN, m0 = (tile / num_w) * BN;
      for (int g = 0; 4 * g < num_k; ++g) {
        uint32_t sw[4], sa[8];
#pragma unroll
        for (int i = 0; i < 4; ++i) sw[i] = scale_word(p.w, n0 + 32 * i + lane, p.n, g);
#pragma unroll
        for (int i = 0; i < 8; ++i) sa[i] = 32 * i < BN ? scale_word(p.a, m0 + 32 * i + lane, p.m, g) : 0x7f7f7f7fu;
        ok = __all_sync(0xffffffffu, wait(sempty_bar(buf), buf_phase ^ 1u));
        if (!ok) break;
        tc_fence_after();
        const uint32_t to = tmem + lanes + kScaleCols + 12 * buf;
        tmem_st_x4(to, sw);
        if (BN <= 128) tmem_st_x4(to + 4, sa);
        else tmem_st_x8(to + 4, sa);
        tmem_st_wait();
        tc_fence_before();
        __syncwarp();
        if (lane == 0) mbar_arrive(sfull_bar(buf));
        if (++buf == 2) { buf = 0; buf_phase ^= 1u; }
      }
    }
  } else {
    int acc = 0;
    uint32_t acc_phase = 0;
    bool ok = true;
    for (long tile = blockIdx.x; tile < num_tiles; tile += gridDim.x) {
      const int n0 = (int)(tile % num_w) * kTileN, m0 = (int)(tile / num_w) * BN;
      const int col = n0 + warp * 32 + lane;
      const float bias = p.bias && col < p.n ? __ldg(p.bias + col) : 0.f;
      ok = ok && __all_sync(0xffffffffu, wait(tfull_bar(acc), acc_phase));
      if (ok) tc_fence_after();
      else if (lane == 0) report(p.status, kGaveUp);  // what was not computed is NaN
      const uint32_t from = tmem + ((uint32_t)(warp * 32) << 16) + acc * BN;
#pragma unroll 1
      for (int c = 0; c < BN && m0 + c < p.m; c += 16) {
        float v[16];
        if (ok) {
          uint32_t r[16];
          tmem_ld_32x16(from + c, r);
          tmem_ld_wait();
#pragma unroll
          for (int i = 0; i < 16; ++i) {
            v[i] = __uint_as_float(r[i]) + bias;
            if (p.gelu) v[i] = gelu_erf(v[i]);
          }
        } else {
#pragma unroll
          for (int i = 0; i < 16; ++i) v[i] = __uint_as_float(0x7fc00000u);
        }
        store16(p, m0 + c, col, v);
      }
      if (ok) {
        tc_fence_before();
        __syncwarp();
        if (lane == 0) mbar_arrive(tempty_bar(acc));
        if (++acc == 2) { acc = 0; acc_phase ^= 1u; }
      }
    }
  }

  tc_fence_before();
  __syncthreads();
  if (warp == 9) {
    tc_fence_after();
    tmem_dealloc(tmem, 512);
  }
}

typedef CUresult (*EncodeTiled)(CUtensorMap*, CUtensorMapDataType, cuuint32_t, void*, const cuuint64_t*, const cuuint64_t*, const cuuint32_t*,
                                const cuuint32_t*, CUtensorMapInterleave, CUtensorMapSwizzle, CUtensorMapL2promotion, CUtensorMapFloatOOBfill);

// Codes [rows, k] as tiles of 128 channels by `box_rows` rows; channels and rows that do not exist read as zeros.
bool codes_map(CUtensorMap* m, const E4m3Operand& x, long rows, int k, int box_rows) {
  static std::atomic<void*> encode{nullptr};  // the driver's entry point, the same for every caller
  void* fn = encode.load(std::memory_order_relaxed);
  if (fn == nullptr) {
    TmaApi api{};
    if (!tma_api_init(&api)) return false;
    encode.store(fn = api.encode_tiled, std::memory_order_relaxed);
  }
  const cuuint64_t dims[2] = {(cuuint64_t)k, (cuuint64_t)rows}, strides[1] = {(cuuint64_t)x.ld};
  const cuuint32_t box[2] = {(cuuint32_t)kBlockBytes, (cuuint32_t)box_rows}, steps[2] = {1, 1};
  return reinterpret_cast<EncodeTiled>(fn)(m, CU_TENSOR_MAP_DATA_TYPE_UINT8, 2, const_cast<void*>(x.codes), dims, strides, box, steps,
                                           CU_TENSOR_MAP_INTERLEAVE_NONE, CU_TENSOR_MAP_SWIZZLE_128B, CU_TENSOR_MAP_L2_PROMOTION_L2_256B,
                                           CU_TENSOR_MAP_FLOAT_OOB_FILL_NONE) == CUDA_SUCCESS;
}

template <int BN>
cudaError_t launch_tiles(const E4m3GemmParams& p, int num_sms, cudaStream_t s) {
  CUtensorMap tw, ta;
  if (!codes_map(&tw, p.w, p.n, p.k, kTileN) || !codes_map(&ta, p.a, p.m, p.k, BN)) return cudaErrorInvalidValue;
  const long tiles = (long)((p.n + kTileN - 1) / kTileN) * ((p.m + BN - 1) / BN);
  const cudaError_t e = cudaFuncSetAttribute(gemm_e4m3_kernel<BN>, cudaFuncAttributeMaxDynamicSharedMemorySize, E4m3Plan<BN>::kBytes);
  if (e != cudaSuccess) return e;
  return launch_dependent(gemm_e4m3_kernel<BN>, dim3((unsigned)(tiles < num_sms ? tiles : num_sms)), dim3(kGemmThreads), E4m3Plan<BN>::kBytes, s, 1,
                          true, tw, ta, p);
}

}  // namespace

cudaError_t launch_quantise_e4m3(const void* x, int dtype, long ldx, long rows, int k, void* codes, long ld_codes, unsigned char* scales,
                                 long ld_scales, cudaStream_t s) {
  const int blocks = (k + kScaleBlock - 1) / kScaleBlock;
  const long items = rows * blocks, per_block = (long)kQuantThreads / 16 * kQuantItems;
  const bool aligned = ((uintptr_t)x & 15) == 0 && ldx * (dtype == WF_BF16 ? 2 : 4) % 16 == 0;
  const dim3 grid((unsigned)((items + per_block - 1) / per_block));
  unsigned char* c = (unsigned char*)codes;
  auto go = [&](auto kernel, auto* from) {
    return launch_dependent(kernel, grid, dim3(kQuantThreads), 0, s, 1, false, from, ldx, items, k, blocks, c, ld_codes, scales, ld_scales);
  };
  if (dtype == WF_BF16) {
    auto* from = (const __nv_bfloat16*)x;
    return aligned ? go(quantise_e4m3_kernel<__nv_bfloat16, true>, from) : go(quantise_e4m3_kernel<__nv_bfloat16, false>, from);
  }
  auto* from = (const float*)x;
  return aligned ? go(quantise_e4m3_kernel<float, true>, from) : go(quantise_e4m3_kernel<float, false>, from);
}

cudaError_t launch_gemm_e4m3(const E4m3GemmParams& p, int num_sms, cudaStream_t s) {
  if (p.m <= 16) return launch_tiles<16>(p, num_sms, s);
  if (p.m <= 32) return launch_tiles<32>(p, num_sms, s);
  if (p.m <= 64) return launch_tiles<64>(p, num_sms, s);
  if (p.m <= 128) return launch_tiles<128>(p, num_sms, s);
  return launch_tiles<224>(p, num_sms, s);
}

}  // namespace wf
