// Paged key/value cache of the decoder: quantised as it is written, and read back.
//
// A vector (one position, one head, keys or values; d_head = 64 or 128 elements) is handled by
// d_head / 8 neighbouring lanes with 8 elements each, so its absolute maximum is a shuffle reduction
// and its codes leave as one 8-byte store per lane.  A warp takes four (d_head 128: two) consecutive rows and one to four
// heads of them, so that the codes of neighbouring positions, and their two-byte scales, leave side by side (heads lie whole runs
// of positions apart), and the search for a row's sequence and page is paid once for its keys and values.
// Bound by memory: d_head (esz + 1) + 2 bytes per vector, once.  35 M bfloat16 elements a side to e4m3 and back: 47 + 39 us, 4.9 TB/s, the
// rest being addresses and conversions between the loads; 9,062 float32 rows of 8 heads of 128 to int8 and back: 43 us, 4.3 TB/s.
#include <type_traits>

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

// Where a row lives in the cache: index of its first head's vector among all vectors of a side, or -1 (padding rows, bad tables).
// Reports what is wrong with the row's start and page; the prefix sums are checked_sums' to report.
__device__ __forceinline__ long locate(const CacheView& c, const RowsView& r, long row, int seq_hint, int* status) {
  if (row >= r.n_rows) return -1;
  int seq = seq_hint;
  while (seq + 1 < r.n_seq && __ldg(r.cu_rows + seq + 1) <= row) ++seq;
  const int first = __ldg(r.cu_rows + seq), next = __ldg(r.cu_rows + seq + 1);
  if (row < first || row >= next || first < 0) return -1;  // padding, or sums that do not fit
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
  return (((long)page * c.n_kv_head) << c.page_shift) + (pos & ((1L << c.page_shift) - 1));
}

// What a lane works on: one row, heads head .. head + kSteps - 1 (below n_kv_head).
struct Share {
  long row, at;  // at: vector of the row's head 0; < 0: nothing to do
  int head;
};
// The search for a row's sequence looks at a few prefix sums only.  All of them are checked by blocks of their own behind the others of
// a launch, a pair each thread.  (In the other blocks it cost: by all threads in front of the search 84.5 -> 86 us for 35 M elements a
// side with the read, between the search and the loads 5.4 -> 5.9 us for 70 rows, after the loads 84.5 -> 96 us.)
__host__ __device__ __forceinline__ unsigned checking_blocks(const RowsView& r) { return (unsigned)(r.n_seq - 1) / kThreads + 1; }
// Whether the block is one of those; it has done its work then.
__device__ __forceinline__ bool checked_sums(const RowsView& r, int* status) {
  const unsigned first = gridDim.x - checking_blocks(r);
  if (blockIdx.x < first) return false;
  const long i = (long)(blockIdx.x - first) * kThreads + threadIdx.x;
  if (i < r.n_seq) {
    const int lo = __ldg(r.cu_rows + i), hi = __ldg(r.cu_rows + i + 1);
    if (lo < 0 || hi < lo || hi > r.n_rows) report(status, kBadRows);
  }
  return true;
}
template <int kLanes, int kSteps>
__device__ __forceinline__ Share share_of(const CacheView& c, const RowsView& r, int n_chunks, int* status) {
  constexpr int kGroups = 32 / kLanes;
  const int lane = threadIdx.x & 31;
  const long w = ((long)blockIdx.x * kThreads + threadIdx.x) >> 5;
  Share s;
  const long block = (long)((unsigned long)w / (unsigned)n_chunks);
  s.head = (int)(w - block * n_chunks) * kSteps;
  const long row0 = block * kGroups;
  s.row = row0 + lane / kLanes;
  const int hint = warp_find_sequence(r.cu_rows, r.n_seq, (int)min(row0, (long)r.n_rows));
  s.at = locate(c, r, s.row, hint, lane % kLanes == 0 ? status : nullptr);  // the lanes of one vector agree
  return s;
}

template <typename T, int kFormat, int kDim, int kSteps>
__global__ void __launch_bounds__(kThreads) cache_write_kernel(CacheView c, RowsView r, const T* __restrict__ k, long k_stride,
                                                               const T* __restrict__ v, long v_stride, int n_chunks, int* status) {
  constexpr int kLanes = kDim / 8;
  const int sub = (threadIdx.x & 31) % kLanes;
  if (checked_sums(r, status)) return;
  const Share s = share_of<kLanes, kSteps>(c, r, n_chunks, status);
  if (s.at < 0) return;
  const T* from_k = k + s.row * k_stride + sub * 8;
  const T* from_v = v + s.row * v_stride + sub * 8;
  Raw8<T> raw[kSteps][2];
#pragma unroll
  for (int u = 0; u < kSteps; ++u) {
    const int head = s.head + u;
    if (head < c.n_kv_head) {
      load8(from_k + head * kDim, raw[u][0]);
      load8(from_v + head * kDim, raw[u][1]);
    }
  }
  const unsigned group = ((kLanes == 16 ? 0xffffu : 0xffu)) << (threadIdx.x & 31 & ~(kLanes - 1));
#pragma unroll
  for (int u = 0; u < kSteps; ++u) {
    const int head = s.head + u;
    if (head >= c.n_kv_head) break;
    const long at = s.at + ((long)head << c.page_shift);
#pragma unroll
    for (int side = 0; side < 2; ++side) {
      void* out = side == 0 ? c.k : c.v;
      if (kFormat == WF_CACHE_PATH) {
        reinterpret_cast<Raw8<T>*>(out)[at * kLanes + sub] = raw[u][side];
      } else {
        float x[8];
        unpack(raw[u][side], x);
        uint32_t top = 0;
#pragma unroll
        for (int i = 0; i < 8; ++i) top = max(top, __float_as_uint(x[i]) & 0x7fffffffu);
#pragma unroll
        for (int o = kLanes / 2; o > 0; o >>= 1) top = max(top, __shfl_xor_sync(group, top, o));
        const float scale = scale_of<kFormat>(top);
        uint2 codes = make_uint2(0, 0);
        if (top < 0x7f800000u) codes = kFormat == WF_CACHE_E4M3 ? quantise_e4m3(x, scale) : quantise_int8(x, scale);
        reinterpret_cast<uint2*>(out)[at * kLanes + sub] = codes;
        if (sub == 0) (side == 0 ? c.k_scale : c.v_scale)[at] = __float2bfloat16_rn(scale);  // exact: a bfloat16 already
      }
    }
  }
}

template <typename T, int kFormat, int kDim, int kSteps>
__global__ void __launch_bounds__(kThreads) cache_read_kernel(CacheView c, RowsView r, T* __restrict__ k, long k_stride,
                                                              T* __restrict__ v, long v_stride, int n_chunks, int* status) {
  constexpr int kLanes = kDim / 8;
  const int sub = (threadIdx.x & 31) % kLanes;
  if (checked_sums(r, status)) return;
  const Share s = share_of<kLanes, kSteps>(c, r, n_chunks, status);
  if (s.at < 0) return;
  T* to_k = k + s.row * k_stride + sub * 8;
  T* to_v = v + s.row * v_stride + sub * 8;
  using Raw = std::conditional_t<kFormat == WF_CACHE_PATH, Raw8<T>, uint2>;
  Raw raw[kSteps][2];
  float scale[kSteps][2];
#pragma unroll
  for (int u = 0; u < kSteps; ++u) {
    const int head = s.head + u;
    if (head < c.n_kv_head) {
      const long at = s.at + ((long)head << c.page_shift);
      raw[u][0] = reinterpret_cast<const Raw*>(c.k)[at * kLanes + sub];
      raw[u][1] = reinterpret_cast<const Raw*>(c.v)[at * kLanes + sub];
      if (kFormat != WF_CACHE_PATH) scale[u][0] = __bfloat162float(c.k_scale[at]), scale[u][1] = __bfloat162float(c.v_scale[at]);
    }
  }
#pragma unroll
  for (int u = 0; u < kSteps; ++u) {
    const int head = s.head + u;
    if (head >= c.n_kv_head) break;
#pragma unroll
    for (int side = 0; side < 2; ++side) {
      T* to = (side == 0 ? to_k : to_v) + head * kDim;
      if constexpr (kFormat == WF_CACHE_PATH) {
        *reinterpret_cast<Raw8<T>*>(to) = raw[u][side];
      } else {
        float x[8];
        dequantise<kFormat>(raw[u][side], scale[u][side], x);
        store8(to, x);
      }
    }
  }
}

template <typename T, int kFormat, int kDim, int kSteps>
cudaError_t write_or_read_steps(bool write, const CacheView& c, const RowsView& r, void* k, long ks, void* v, long vs, int* status,
                          cudaStream_t s) {
  constexpr int kGroups = 32 / (kDim / 8);
  const int n_chunks = (c.n_kv_head + kSteps - 1) / kSteps;
  const long warps = ((long)r.n_rows + kGroups - 1) / kGroups * n_chunks;
  const dim3 grid((unsigned)((warps * 32 + kThreads - 1) / kThreads) + checking_blocks(r));
  if (write)
    return launch_dependent(cache_write_kernel<T, kFormat, kDim, kSteps>, grid, dim3(kThreads), 0, s, 1, false, c, r, (const T*)k, ks,
                            (const T*)v, vs, n_chunks, status);
  return launch_dependent(cache_read_kernel<T, kFormat, kDim, kSteps>, grid, dim3(kThreads), 0, s, 1, false, c, r, (T*)k, ks, (T*)v, vs,
                          n_chunks, status);
}

template <typename T, int kFormat, int kDim>
cudaError_t write_or_read(bool write, const CacheView& c, const RowsView& r, void* k, long ks, void* v, long vs, int* status,
                          cudaStream_t s) {
  // Several heads per group of lanes pay once a large call of 16-bit rows leaves the SMs with threads enough either way: 35 M elements
  // a side with one / two / four of them are written in 59 / 51 / 47 us and read back in 47 / 39 / 42 us; float32 rows have as many
  // bytes in flight with one.
  if (sizeof(T) == 2 && (long)r.n_rows * c.n_kv_head * (kDim / 8) >= 1L << 20)
    return write ? write_or_read_steps<T, kFormat, kDim, 4>(true, c, r, k, ks, v, vs, status, s)
                 : write_or_read_steps<T, kFormat, kDim, 2>(false, c, r, k, ks, v, vs, status, s);
  return write_or_read_steps<T, kFormat, kDim, 1>(write, c, r, k, ks, v, vs, status, s);
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
