// Paged key/value cache of the decoder: quantised as it is written, and read back.
//
// A vector (one position, one head, keys or values; d_head = 64 or 128 elements) is handled by
// d_head / 8 neighbouring lanes with 8 elements each, so its absolute maximum is a shuffle reduction
// and its codes leave as one 8-byte store per lane (coalesced: a position's heads are read side by side,
// each written as d_head consecutive bytes of its page).  A thread takes the key and the value vector
// of its (row, head), so two (float32: four) 16-byte loads are in flight per thread.
// Bound by memory: d_head (esz + 1) + 2 bytes per vector, once.
#include "wf_decoder.h"

namespace wf {

namespace {

constexpr int kThreads = 256;

template <typename T>
struct Raw8;  // 8 elements as loaded
template <>
struct Raw8<__nv_bfloat16> {
  uint4 a;
};
template <>
struct Raw8<float> {
  float4 a, b;
};

__device__ __forceinline__ void load8(const __nv_bfloat16* p, Raw8<__nv_bfloat16>& r) {
  r.a = __ldcs(reinterpret_cast<const uint4*>(p));
}
__device__ __forceinline__ void load8(const float* p, Raw8<float>& r) {
  r.a = __ldcs(reinterpret_cast<const float4*>(p));
  r.b = __ldcs(reinterpret_cast<const float4*>(p) + 1);
}
__device__ __forceinline__ void unpack(const Raw8<__nv_bfloat16>& r, float (&x)[8]) {
  const uint32_t w[4] = {r.a.x, r.a.y, r.a.z, r.a.w};
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    x[2 * i] = __uint_as_float(w[i] << 16);
    x[2 * i + 1] = __uint_as_float(w[i] & 0xffff0000u);
  }
}
__device__ __forceinline__ void unpack(const Raw8<float>& r, float (&x)[8]) {
  x[0] = r.a.x; x[1] = r.a.y; x[2] = r.a.z; x[3] = r.a.w;
  x[4] = r.b.x; x[5] = r.b.y; x[6] = r.b.z; x[7] = r.b.w;
}
__device__ __forceinline__ void store8(__nv_bfloat16* p, const float (&x)[8]) {
  uint4 r;
  uint32_t* w = &r.x;
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    const __nv_bfloat162 h = __floats2bfloat162_rn(x[2 * i], x[2 * i + 1]);
    w[i] = *reinterpret_cast<const uint32_t*>(&h);
  }
  *reinterpret_cast<uint4*>(p) = r;
}
__device__ __forceinline__ void store8(float* p, const float (&x)[8]) {
  reinterpret_cast<float4*>(p)[0] = make_float4(x[0], x[1], x[2], x[3]);
  reinterpret_cast<float4*>(p)[1] = make_float4(x[4], x[5], x[6], x[7]);
}

// Scale of a vector from the largest magnitude bits `top` (as an integer: finite magnitudes order like
// their bits, infinities and NaN lie above them).
template <int kFormat>
__device__ __forceinline__ float scale_of(uint32_t top) {
  if (top >= 0x7f800000u) return __uint_as_float(0x7fc00000u);
  if (top == 0) return 1.f;
  if (kFormat == WF_CACHE_E4M3) {
    // a = m 2^e with 1 <= m < 2, and 448 = 1.75 2^8: s = 2^(e - 8) for m <= 1.75, else 2^(e - 7).
    // Subnormal a (exponent field 0) ends at the floor.
    const int e = (int)(top >> 23) - 8 + ((top & 0x7fffffu) > 0x600000u ? 1 : 0);
    return __uint_as_float((uint32_t)max(e, 1) << 23);
  }
  const float q = __fdiv_rn(__uint_as_float(top), 127.f);
  return __uint_as_float(max((__float_as_uint(q) + 0xffffu) & 0xffff0000u, 0x00800000u));
}

// 8 codes of a vector with scale s.
__device__ __forceinline__ uint2 quantise_e4m3(const float (&x)[8], float s) {
  const float inv = 1.f / s;  // a power of two: x * inv is exact
  uint32_t w[4];
#pragma unroll
  for (int i = 0; i < 4; ++i)
    w[i] = __nv_cvt_float2_to_fp8x2(make_float2(x[2 * i] * inv, x[2 * i + 1] * inv), __NV_SATFINITE, __NV_E4M3);
  return make_uint2(w[0] | (w[1] << 16), w[2] | (w[3] << 16));
}
// x / s rounded to the nearest whole number.  The product with the reciprocal is within 2^-15 of the
// quotient (|x / s| <= 127.5, two roundings of 2^-24 relative), so only a product that close to a
// border needs the quotient itself; and that one, rounded to float32, is the border exactly or lies on
// the right side of it, in the first case the remainder tells (it is exact in float32).
__device__ __forceinline__ int whole_quotient(float x, float s, float inv) {
  const float p = x * inv;
  float r = rintf(p);
  if (fabsf(fabsf(p - r) - 0.5f) < 0x1p-14f) {
    const float q = __fdiv_rn(x, s);
    r = rintf(q);
    if (fabsf(q - truncf(q)) == 0.5f) {
      const float rest = fmaf(-q, s, x);
      if (rest > 0.f) r = ceilf(q);
      if (rest < 0.f) r = floorf(q);
    }
  }
  return (int)r;
}
__device__ __forceinline__ uint2 quantise_int8(const float (&x)[8], float s) {
  const float inv = __fdiv_rn(1.f, s);
  uint32_t w[2] = {0, 0};
#pragma unroll
  for (int i = 0; i < 8; ++i) w[i / 4] |= (uint32_t)(whole_quotient(x[i], s, inv) & 0xff) << (8 * (i % 4));
  return make_uint2(w[0], w[1]);
}
template <int kFormat>
__device__ __forceinline__ void dequantise(uint2 c, float s, float (&x)[8]) {
  const uint32_t w[2] = {c.x, c.y};
  if (kFormat == WF_CACHE_E4M3) {
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      const __half2_raw h = __nv_cvt_fp8x2_to_halfraw2((__nv_fp8x2_storage_t)(w[i / 2] >> (16 * (i % 2))), __NV_E4M3);
      const float2 f = __half22float2(*reinterpret_cast<const __half2*>(&h));
      x[2 * i] = f.x * s;
      x[2 * i + 1] = f.y * s;
    }
  } else {
#pragma unroll
    for (int i = 0; i < 8; ++i) x[i] = (float)(int)(int8_t)(w[i / 4] >> (8 * (i % 4))) * s;
  }
}

// Where the thread's (row, head) lives in the cache: index of its vector among all vectors of a side,
// or -1 (padding rows, bad tables).
__device__ __forceinline__ long locate(const CacheView& c, const RowsView& r, long row, int head, int seq_hint, int* status) {
  if (row >= r.n_rows) return -1;
  int seq = seq_hint;
  while (seq + 1 < r.n_seq && __ldg(r.cu_rows + seq + 1) <= row) ++seq;
  const int first = __ldg(r.cu_rows + seq), next = __ldg(r.cu_rows + seq + 1);
  if (row < first || row >= next) {
    if (row < first || next < first) report(status, kBadRows);
    return -1;
  }
  const long pos = (long)__ldg(r.start + seq) + (row - first);
  const long index = pos >> c.page_shift;
  if (pos < 0 || index >= r.table_stride) {
    report(status, kBadRows);
    return -1;
  }
  const int page = __ldg(r.page_table + (long)seq * r.table_stride + index);
  if (page < 0 || page >= c.n_pages) {
    report(status, kBadPage);
    return -1;
  }
  return (((long)page * c.n_kv_head + head) << c.page_shift) + (pos & ((1L << c.page_shift) - 1));
}

template <typename T, int kFormat, int kDim>
__global__ void __launch_bounds__(kThreads) cache_write_kernel(CacheView c, RowsView r, const T* __restrict__ k, long k_stride,
                                                               const T* __restrict__ v, long v_stride, int* status) {
  constexpr int kLanes = kDim / 8;
  const long first = (long)blockIdx.x * kThreads + (threadIdx.x & ~31);
  const int hint = warp_find_sequence(r.cu_rows, r.n_seq, (int)min(first / kLanes / c.n_kv_head, (long)r.n_rows));
  const long t = (long)blockIdx.x * kThreads + threadIdx.x;
  if (t == 0 && __ldg(r.cu_rows + r.n_seq) > r.n_rows) report(status, kBadRows);
  const int sub = (int)(t % kLanes);
  const long item = t / kLanes;
  const long row = item / c.n_kv_head;
  const int head = (int)(item - row * c.n_kv_head);
  const long at = locate(c, r, row, head, hint, sub == 0 ? status : nullptr);
  if (at < 0) return;  // the lanes of one vector agree
  const unsigned group = ((kLanes == 16 ? 0xffffu : 0xffu)) << (threadIdx.x & 31 & ~(kLanes - 1));
  Raw8<T> raw[2];
  load8(k + row * k_stride + (long)head * kDim + sub * 8, raw[0]);
  load8(v + row * v_stride + (long)head * kDim + sub * 8, raw[1]);
#pragma unroll
  for (int side = 0; side < 2; ++side) {
    void* out = side == 0 ? c.k : c.v;
    if (kFormat == WF_CACHE_PATH) {
      reinterpret_cast<Raw8<T>*>(out)[at * kLanes + sub] = raw[side];
    } else {
      float x[8];
      unpack(raw[side], x);
      uint32_t top = 0;
#pragma unroll
      for (int i = 0; i < 8; ++i) top = max(top, __float_as_uint(x[i]) & 0x7fffffffu);
#pragma unroll
      for (int o = kLanes / 2; o > 0; o >>= 1) top = max(top, __shfl_xor_sync(group, top, o));
      const float s = scale_of<kFormat>(top);
      uint2 codes = make_uint2(0, 0);
      if (top < 0x7f800000u) codes = kFormat == WF_CACHE_E4M3 ? quantise_e4m3(x, s) : quantise_int8(x, s);
      reinterpret_cast<uint2*>(out)[at * kLanes + sub] = codes;
      if (sub == 0) (side == 0 ? c.k_scale : c.v_scale)[at] = __float2bfloat16_rn(s);  // exact: s is a bfloat16
    }
  }
}

template <typename T, int kFormat, int kDim>
__global__ void __launch_bounds__(kThreads) cache_read_kernel(CacheView c, RowsView r, T* __restrict__ k, long k_stride,
                                                              T* __restrict__ v, long v_stride, int* status) {
  constexpr int kLanes = kDim / 8;
  const long first = (long)blockIdx.x * kThreads + (threadIdx.x & ~31);
  const int hint = warp_find_sequence(r.cu_rows, r.n_seq, (int)min(first / kLanes / c.n_kv_head, (long)r.n_rows));
  const long t = (long)blockIdx.x * kThreads + threadIdx.x;
  if (t == 0 && __ldg(r.cu_rows + r.n_seq) > r.n_rows) report(status, kBadRows);
  const int sub = (int)(t % kLanes);
  const long item = t / kLanes;
  const long row = item / c.n_kv_head;
  const int head = (int)(item - row * c.n_kv_head);
  const long at = locate(c, r, row, head, hint, sub == 0 ? status : nullptr);
  if (at < 0) return;
  T* const dst_k = k + row * k_stride + (long)head * kDim + sub * 8;
  T* const dst_v = v + row * v_stride + (long)head * kDim + sub * 8;
  if (kFormat == WF_CACHE_PATH) {
    const Raw8<T> a = reinterpret_cast<const Raw8<T>*>(c.k)[at * kLanes + sub];
    const Raw8<T> b = reinterpret_cast<const Raw8<T>*>(c.v)[at * kLanes + sub];
    *reinterpret_cast<Raw8<T>*>(dst_k) = a;
    *reinterpret_cast<Raw8<T>*>(dst_v) = b;
  } else {
    const uint2 a = reinterpret_cast<const uint2*>(c.k)[at * kLanes + sub];
    const uint2 b = reinterpret_cast<const uint2*>(c.v)[at * kLanes + sub];
    const float sa = __bfloat162float(c.k_scale[at]), sb = __bfloat162float(c.v_scale[at]);
    float x[8];
    dequantise<kFormat>(a, sa, x);
    store8(dst_k, x);
    dequantise<kFormat>(b, sb, x);
    store8(dst_v, x);
  }
}

template <typename T, int kFormat, int kDim>
cudaError_t write_or_read(bool write, const CacheView& c, const RowsView& r, void* k, long ks, void* v, long vs, int* status,
                          cudaStream_t s) {
  const long threads = (long)r.n_rows * c.n_kv_head * (kDim / 8);
  const long blocks = (threads + kThreads - 1) / kThreads;
  const dim3 grid((unsigned)blocks);
  if (write)
    return launch_dependent(cache_write_kernel<T, kFormat, kDim>, grid, dim3(kThreads), 0, s, 1, false, c, r, (const T*)k, ks,
                            (const T*)v, vs, status);
  return launch_dependent(cache_read_kernel<T, kFormat, kDim>, grid, dim3(kThreads), 0, s, 1, false, c, r, (T*)k, ks, (T*)v, vs, status);
}

template <typename T>
cudaError_t by_format(bool write, const CacheView& c, const RowsView& r, int d, int format, void* k, long ks, void* v, long vs,
                      int* status, cudaStream_t s) {
  if (d == 64) {
    if (format == WF_CACHE_PATH) return write_or_read<T, WF_CACHE_PATH, 64>(write, c, r, k, ks, v, vs, status, s);
    if (format == WF_CACHE_E4M3) return write_or_read<T, WF_CACHE_E4M3, 64>(write, c, r, k, ks, v, vs, status, s);
    return write_or_read<T, WF_CACHE_INT8, 64>(write, c, r, k, ks, v, vs, status, s);
  }
  if (format == WF_CACHE_PATH) return write_or_read<T, WF_CACHE_PATH, 128>(write, c, r, k, ks, v, vs, status, s);
  if (format == WF_CACHE_E4M3) return write_or_read<T, WF_CACHE_E4M3, 128>(write, c, r, k, ks, v, vs, status, s);
  return write_or_read<T, WF_CACHE_INT8, 128>(write, c, r, k, ks, v, vs, status, s);
}

}  // namespace

cudaError_t launch_cache_write(const CacheView& c, const RowsView& r, int d_head, int dtype, int format, const void* k,
                               long k_stride, const void* v, long v_stride, int* status, cudaStream_t s) {
  return dtype == WF_BF16
             ? by_format<__nv_bfloat16>(true, c, r, d_head, format, (void*)k, k_stride, (void*)v, v_stride, status, s)
             : by_format<float>(true, c, r, d_head, format, (void*)k, k_stride, (void*)v, v_stride, status, s);
}
cudaError_t launch_cache_read(const CacheView& c, const RowsView& r, int d_head, int dtype, int format, void* k,
                              long k_stride, void* v, long v_stride, int* status, cudaStream_t s) {
  return dtype == WF_BF16 ? by_format<__nv_bfloat16>(false, c, r, d_head, format, k, k_stride, v, v_stride, status, s)
                          : by_format<float>(false, c, r, d_head, format, k, k_stride, v, v_stride, status, s);
}

}  // namespace wf
