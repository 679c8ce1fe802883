// Attention of drafted tokens or beams over the paged cache.
//
// The query rows of one key/value head -- (row i, head of the group) pairs, i major -- form tiles; a block
// takes one tile of one sequence over one split of its positions and keeps the running maximum m, the sum l
// and the unnormalised output of every row:
//   m' = max(m, max_j s_j),  l' = l e^(m - m') + sum_j e^(s_j - m'),  o' = o e^(m - m') + sum_j e^(s_j - m') v_j.
// Splits are joined by a second kernel in split order, so results do not depend on scheduling.
#include <algorithm>
#include <cstdlib>

#include "wf_tree_attention.cuh"

namespace wf {

namespace {

// 16 bytes of stored elements as float32.
template <typename T, int kFormat>
struct Codes {
  static constexpr int kElems = kFormat == WF_CACHE_PATH ? 16 / (int)sizeof(T) : 16;
  static __device__ __forceinline__ void unpack(uint4 r, float s, float (&x)[kElems]) {
    const uint32_t w[4] = {r.x, r.y, r.z, r.w};
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      if constexpr (kFormat == WF_CACHE_PATH && sizeof(T) == 4) {
        x[i] = __uint_as_float(w[i]);
      } else if constexpr (kFormat == WF_CACHE_PATH) {
        x[2 * i] = __uint_as_float(w[i] << 16);
        x[2 * i + 1] = __uint_as_float(w[i] & 0xffff0000u);
      } else if constexpr (kFormat == WF_CACHE_E4M3) {
#pragma unroll
        for (int j = 0; j < 2; ++j) {
          const __half2_raw h = __nv_cvt_fp8x2_to_halfraw2((__nv_fp8x2_storage_t)(w[i] >> (16 * j)), __NV_E4M3);
          const float2 f = __half22float2(*reinterpret_cast<const __half2*>(&h));
          x[4 * i + 2 * j] = f.x * s;
          x[4 * i + 2 * j + 1] = f.y * s;
        }
      } else {
#pragma unroll
        for (int j = 0; j < 4; ++j) x[4 * i + j] = (float)(int)(int8_t)(w[i] >> (8 * j)) * s;
      }
    }
  }
};

__device__ __forceinline__ float to_float(float x) { return x; }
__device__ __forceinline__ float to_float(__nv_bfloat16 x) { return __bfloat162float(x); }
__device__ __forceinline__ void put(float* p, float x) { *p = x; }
__device__ __forceinline__ void put(__nv_bfloat16* p, float x) { *p = __float2bfloat16_rn(x); }

// ---------------------------------------------------------------------------------------------
// float32 kernel: tiles of 8 rows and 64 positions, everything dequantised into shared memory.
constexpr int kSimtRows = 8, kSimtKeys = 64, kSimtThreads = 128;

template <int kDim>
constexpr size_t simt_smem() {
  return sizeof(float) * (kSimtKeys * (kDim + 4) + kSimtKeys * kDim + kSimtRows * kDim + kSimtRows * kSimtKeys + 3 * kSimtRows);
}

template <typename T, int kFormat, int kDim>
__global__ void __launch_bounds__(kSimtThreads) tree_attention_simt_kernel(const __grid_constant__ TreeAttnParams p) {
  extern __shared__ __align__(16) float smem[];
  float* Ks = smem;                             // [64][kDim + 4]
  float* Vs = Ks + kSimtKeys * (kDim + 4);      // [64][kDim]
  float* Qs = Vs + kSimtKeys * kDim;            // [8][kDim]
  float* Ps = Qs + kSimtRows * kDim;            // [8][64]
  float* row_m = Ps + kSimtRows * kSimtKeys;    // [8]
  float* row_l = row_m + kSimtRows;             // [8]
  float* row_a = row_l + kSimtRows;             // [8] factor of this tile's rescaling
  const int seq = blockIdx.z, kvh = blockIdx.y;
  const int split = blockIdx.x % p.n_splits, tile = blockIdx.x / p.n_splits;
  const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5;
  const Sequence s = load_sequence(p, seq, tid == 0 && blockIdx.x == 0 && kvh == 0);
  const int rows = min(s.n_rows, p.max_rows) * p.group;  // of this key/value head
  const int r0 = tile * kSimtRows;
  if (r0 >= rows) return;
  const int begin = split * p.chunk, end = min(s.len, begin + p.chunk);
  if (split > 0 && begin >= s.len) return;

  const T* q = reinterpret_cast<const T*>(p.q);
  for (int i = tid; i < kSimtRows * kDim; i += kSimtThreads) {
    const int r = r0 + i / kDim;
    Qs[i] = r < rows ? to_float(q[(long)(s.first_row + r / p.group) * p.q_stride + (long)(kvh * p.group + r % p.group) * kDim + i % kDim]) : 0.f;
  }
  if (tid < kSimtRows) row_m[tid] = -INFINITY, row_l[tid] = 0.f;
  constexpr int kOut = kSimtRows * kDim / kSimtThreads;  // rows a thread accumulates (one channel)
  const int ch = tid % kDim, out_r0 = (tid / kDim) * kOut;
  float acc[kOut];
#pragma unroll
  for (int i = 0; i < kOut; ++i) acc[i] = 0.f;

  constexpr int kElems = Codes<T, kFormat>::kElems;
  constexpr int kVecs = kDim / kElems;
  for (int k0 = begin; k0 < end; k0 += kSimtKeys) {
    __syncthreads();
    for (int i = tid; i < kSimtKeys * kVecs; i += kSimtThreads) {
      const int key = i / kVecs, u = i % kVecs, pos = k0 + key;
      float xk[kElems], xv[kElems];
      const int page = pos < end ? page_of(p, seq, pos) : -1;
      if (page >= 0) {
        const long at = (((long)page * p.cache.n_kv_head + kvh) << p.cache.page_shift) + (pos & ((1 << p.cache.page_shift) - 1));
        const float sk = kFormat == WF_CACHE_PATH ? 1.f : __bfloat162float(p.cache.k_scale[at]);
        const float sv = kFormat == WF_CACHE_PATH ? 1.f : __bfloat162float(p.cache.v_scale[at]);
        Codes<T, kFormat>::unpack(reinterpret_cast<const uint4*>(p.cache.k)[at * kVecs + u], sk, xk);
        Codes<T, kFormat>::unpack(reinterpret_cast<const uint4*>(p.cache.v)[at * kVecs + u], sv, xv);
      } else {
#pragma unroll
        for (int e = 0; e < kElems; ++e) xk[e] = xv[e] = 0.f;
      }
      if (u == 0) Ks[key * (kDim + 4) + kDim] = page >= 0 ? 1.f : 0.f;  // in the padding: whether the position exists
#pragma unroll
      for (int e = 0; e < kElems; e += 4) {
        *reinterpret_cast<float4*>(Ks + key * (kDim + 4) + u * kElems + e) = make_float4(xk[e], xk[e + 1], xk[e + 2], xk[e + 3]);
        *reinterpret_cast<float4*>(Vs + key * kDim + u * kElems + e) = make_float4(xv[e], xv[e + 1], xv[e + 2], xv[e + 3]);
      }
    }
    __syncthreads();
    {  // scores: a thread has one position and four rows
      const int key = tid & 63, rr = (tid >> 6) * 4;
      float sc[4] = {0.f, 0.f, 0.f, 0.f};
#pragma unroll 4
      for (int c = 0; c < kDim; c += 4) {
        const float4 k4 = *reinterpret_cast<const float4*>(Ks + key * (kDim + 4) + c);
#pragma unroll
        for (int i = 0; i < 4; ++i) {
          const float4 q4 = *reinterpret_cast<const float4*>(Qs + (rr + i) * kDim + c);
          sc[i] = fmaf(q4.x, k4.x, sc[i]);
          sc[i] = fmaf(q4.y, k4.y, sc[i]);
          sc[i] = fmaf(q4.z, k4.z, sc[i]);
          sc[i] = fmaf(q4.w, k4.w, sc[i]);
        }
      }
      const int pos = k0 + key;
      const bool there = pos < end && Ks[key * (kDim + 4) + kDim] != 0.f;
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        const int r = r0 + rr + i;
        const bool see = there && r < rows && (pos < s.start || sees_tail(p, s, r / p.group, pos - s.start));
        Ps[(rr + i) * kSimtKeys + key] = see ? sc[i] * p.scale : -INFINITY;
      }
    }
    __syncthreads();
#pragma unroll
    for (int i = 0; i < 2; ++i) {  // softmax: a warp has two rows
      const int r = warp * 2 + i;
      const float a = Ps[r * kSimtKeys + lane], b = Ps[r * kSimtKeys + lane + 32];
      float mx = fmaxf(a, b);
      bool nan = a != a || b != b;  // a NaN score that the row sees makes the row NaN
#pragma unroll
      for (int o = 16; o > 0; o >>= 1) mx = fmaxf(mx, __shfl_xor_sync(0xffffffffu, mx, o));
      if (__any_sync(0xffffffffu, nan)) mx = __int_as_float(0x7fc00000);
      const float m_old = row_m[r];
      const float m_new = (m_old != m_old || mx != mx) ? __int_as_float(0x7fc00000) : fmaxf(m_old, mx);
      const float base = m_new == -INFINITY ? 0.f : m_new;
      const float pa = expf(a - base), pb = expf(b - base);
      float sum = pa + pb;
#pragma unroll
      for (int o = 16; o > 0; o >>= 1) sum += __shfl_xor_sync(0xffffffffu, sum, o);
      Ps[r * kSimtKeys + lane] = pa;
      Ps[r * kSimtKeys + lane + 32] = pb;
      if (lane == 0) {
        const float f = expf(m_old - base);
        row_a[r] = f;
        row_l[r] = row_l[r] * f + sum;
        row_m[r] = m_new;
      }
    }
    __syncthreads();
#pragma unroll
    for (int i = 0; i < kOut; ++i) acc[i] *= row_a[out_r0 + i];
    // positions that a row does not see have p = 0; only among the batch's own rows does that differ from
    // row to row, and there a value that is not finite must not reach them
    const bool guard = k0 + kSimtKeys > s.start;
    for (int key = 0; key < kSimtKeys; key += 4) {
      float v[4];
#pragma unroll
      for (int j = 0; j < 4; ++j) v[j] = Vs[(key + j) * kDim + ch];
#pragma unroll
      for (int i = 0; i < kOut; ++i) {
        const float4 pr = *reinterpret_cast<const float4*>(Ps + (out_r0 + i) * kSimtKeys + key);
        const float pj[4] = {pr.x, pr.y, pr.z, pr.w};
#pragma unroll
        for (int j = 0; j < 4; ++j)
          if (!guard || pj[j] != 0.f) acc[i] = fmaf(pj[j], v[j], acc[i]);
      }
    }
  }
  __syncthreads();
#pragma unroll
  for (int i = 0; i < kOut; ++i) {
    const int r = r0 + out_r0 + i;
    if (r >= rows) continue;
    const long row = s.first_row + r / p.group;
    const int head = kvh * p.group + r % p.group;
    const float l = row_l[out_r0 + i], m = row_m[out_r0 + i];
    if (p.n_splits > 1) {
      const long at = (row * p.n_head + head) * p.n_splits + split;
      p.part_o[at * kDim + ch] = acc[i];
      if (ch == 0) p.part_ml[at] = make_float2(m, l);
    } else {
      put(reinterpret_cast<T*>(p.out) + row * p.out_stride + (long)head * kDim + ch, l == 0.f ? 0.f : acc[i] / l);
      if (ch == 0 && p.lse) p.lse[row * p.n_head + head] = l == 0.f ? -INFINITY : m + logf(l);
    }
  }
}

// Joins the splits of a row: one block per (row, head), one thread per channel.
template <typename T, int kDim>
__global__ void __launch_bounds__(kDim) tree_attention_join_kernel(const __grid_constant__ TreeAttnParams p) {
  const int row = blockIdx.x, head = blockIdx.y, ch = threadIdx.x;
  const int seq = warp_find_sequence(p.rows.cu_rows, p.rows.n_seq, row);
  const Sequence s = load_sequence(p, seq, false);
  if (row < s.first_row || row - s.first_row >= min(s.n_rows, p.max_rows)) return;
  const int n = max(1, (s.len + p.chunk - 1) / p.chunk);
  const long at = ((long)row * p.n_head + head) * p.n_splits;
  float m = -INFINITY;
  bool nan = false;
  for (int i = 0; i < n; ++i) {
    const float mi = p.part_ml[at + i].x;
    nan |= mi != mi;
    m = fmaxf(m, mi);
  }
  if (nan) m = __int_as_float(0x7fc00000);
  const float base = m == -INFINITY ? 0.f : m;
  float l = 0.f, o = 0.f;
  for (int i = 0; i < n; ++i) {
    const float2 ml = p.part_ml[at + i];
    const float f = expf(ml.x - base);
    l += ml.y * f;
    const float x = p.part_o[(at + i) * kDim + ch];
    if (ml.y != 0.f) o += x * f;
  }
  put(reinterpret_cast<T*>(p.out) + (long)row * p.out_stride + (long)head * kDim + ch, l == 0.f ? 0.f : o / l);
  if (ch == 0 && p.lse) p.lse[(long)row * p.n_head + head] = l == 0.f ? -INFINITY : m + logf(l);
}

template <typename T, int kFormat, int kDim>
cudaError_t launch_simt(const TreeAttnParams& p, cudaStream_t s) {
  const int tiles = (int)(((long)p.max_rows * p.group + kSimtRows - 1) / kSimtRows);
  const dim3 grid((unsigned)(tiles * p.n_splits), (unsigned)p.cache.n_kv_head, (unsigned)p.rows.n_seq);
  auto kernel = tree_attention_simt_kernel<T, kFormat, kDim>;
  cudaError_t e = cudaFuncSetAttribute(kernel, cudaFuncAttributeMaxDynamicSharedMemorySize, (int)simt_smem<kDim>());
  if (e == cudaSuccess) e = launch_dependent(kernel, grid, dim3(kSimtThreads), simt_smem<kDim>(), s, 1, false, p);
  return e;
}

constexpr int kWideRows = 32;  // more rows of a key/value head than this go to the kernel with 128-row tiles

// Rows of one tile of the kernel for few rows.
int tc_rows(int d_head, long rows) { return rows <= 8 ? 8 : rows <= 16 || d_head == 128 ? 16 : 32; }

template <typename T, int kDim>
cudaError_t launch_format(const TreeAttnParams& p, int format, cudaStream_t s) {
  cudaError_t e;
  if constexpr (sizeof(T) == 2)
    e = p.unit_warps == 0 ? launch_tree_attention_wide(p, kDim, format, s)
                          : launch_tree_attention_tc(p, kDim, format, tc_rows(kDim, (long)p.max_rows * p.group), s);
  else if (format == WF_CACHE_PATH) e = launch_simt<T, WF_CACHE_PATH, kDim>(p, s);
  else if (format == WF_CACHE_E4M3) e = launch_simt<T, WF_CACHE_E4M3, kDim>(p, s);
  else e = launch_simt<T, WF_CACHE_INT8, kDim>(p, s);
  if (e == cudaSuccess && p.n_splits > 1)
    e = launch_dependent(tree_attention_join_kernel<T, kDim>, dim3((unsigned)p.rows.n_rows, (unsigned)p.n_head), dim3(kDim), 0, s, 1, false, p);
  return e;
}

}  // namespace

TreeAttnPlan plan_tree_attention(int dtype, int d_head, int n_head, int n_kv_head, int n_seq, int n_rows, int max_rows, int max_len,
                                 int num_sms) {
  TreeAttnPlan plan{};
  const long rows = (long)max_rows * (n_head / n_kv_head);
  const bool wide = dtype == WF_BF16 && rows > kWideRows;
  const int tile = wide ? 128 : dtype == WF_BF16 ? tc_rows(d_head, rows) : kSimtRows;
  const long tiles = (rows + tile - 1) / tile;
  const long units = tiles * n_kv_head * n_seq;
  if (wide) {
    const long splits = getenv("XC") ? ((long)max_len + atoi(getenv("XC")) - 1) / atoi(getenv("XC")) : std::max(1L, std::min((4L * num_sms + units - 1) / units, ((long)max_len + 511) / 512));
    plan.unit_warps = 0;
    plan.chunk = (int)(((long)max_len + splits * 64 - 1) / (splits * 64) * 64);
  } else if (dtype == WF_BF16) {
    // Warps that the registers let reside: 16, 12 or 8 per SM.  A unit is shared by as few warps as fill them (each one has
    // a start and an end to pay for), and cut into splits, all of one wave, where four are not enough.
    const long resident = (long)num_sms * (tile == 8 ? 16 : tile == 16 && d_head == 64 ? 12 : 8);
    plan.unit_warps = getenv("XW") ? atoi(getenv("XW")) : 4;
    const long splits = std::max(1L, std::min(resident / (4 * units), ((long)max_len + 255) / 256));
    plan.chunk = (int)(((long)max_len + splits * 64 - 1) / (splits * 64) * 64);
  } else {
    // as many splits as fill the SMs four times over, of at least 256 positions each
    const long splits = std::max(1L, std::min((4L * num_sms + units - 1) / units, ((long)max_len + 255) / 256));
    plan.unit_warps = 4;
    plan.chunk = (int)(((long)max_len + splits * kSimtKeys - 1) / (splits * kSimtKeys) * kSimtKeys);
  }
  if (plan.chunk < 64) plan.chunk = 64;
  plan.n_splits = (int)std::max(1L, ((long)max_len + plan.chunk - 1) / plan.chunk);
  plan.bytes = plan.n_splits > 1 ? (size_t)n_rows * n_head * plan.n_splits * (d_head * sizeof(float) + sizeof(float2)) : 0;
  return plan;
}

cudaError_t launch_tree_attention(const TreeAttnParams& p, int d_head, int dtype, int format, cudaStream_t s) {
  if (dtype == WF_BF16) return d_head == 64 ? launch_format<__nv_bfloat16, 64>(p, format, s) : launch_format<__nv_bfloat16, 128>(p, format, s);
  return d_head == 64 ? launch_format<float, 64>(p, format, s) : launch_format<float, 128>(p, format, s);
}

}  // namespace wf
