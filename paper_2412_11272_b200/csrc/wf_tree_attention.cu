// Attention of drafted tokens or beams over the paged cache.
//
// The query rows of one key/value head -- (row i, head of the group) pairs, i major -- form tiles; a block
// takes one tile of one sequence over one split of its positions and keeps the running maximum m, the sum l
// and the unnormalised output of every row:
//   m' = max(m, max_j s_j),  l' = l e^(m - m') + sum_j e^(s_j - m'),  o' = o e^(m - m') + sum_j e^(s_j - m') v_j.
// Splits are joined by a second kernel in split order, so results do not depend on scheduling.
#include <algorithm>
#include <type_traits>

#include "wf_ptx.cuh"
#include "wf_tree_attention.cuh"

namespace wf {

namespace {

// 16 bytes of stored elements as float32 (float32 path).
template <int kFormat>
struct Codes {
  static constexpr int kElems = kFormat == WF_CACHE_PATH ? 4 : 16;
  static __device__ __forceinline__ void unpack(uint4 r, float s, float (&x)[kElems]) {
    const uint32_t w[4] = {r.x, r.y, r.z, r.w};
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      if constexpr (kFormat == WF_CACHE_PATH) {
        x[i] = __uint_as_float(w[i]);
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

__device__ __forceinline__ void put(float* p, float x) { *p = x; }
__device__ __forceinline__ void put(__nv_bfloat16* p, float x) { *p = __float2bfloat16_rn(x); }

// ---------------------------------------------------------------------------------------------
// float32 path: 8 or 16 query rows and 64 positions a step, dequantised into shared memory; the next step's 16-byte
// pieces wait in registers meanwhile.  Products in float32 on the FMA pipe, whose rate (and shared memory's: a thread reads
// one key piece per 2 or 4 query rows) is the bound for more than a few rows; a softmax row belongs to a warp.
// 8 sequences of 301 .. 1508 positions, 6 heads of 64 channels, 3 .. 8 rows: 22 us with the join, 23.5 MB (1.07 TB/s).
constexpr int kSimtKeys = 64, kSimtThreads = 256;

template <int kDim, int kRows>
constexpr size_t simt_smem() {
  return sizeof(float) * (kSimtKeys * (kDim + 4) + kSimtKeys * kDim + kRows * kDim + kRows * kSimtKeys + 3 * kRows + 2);
}

template <int kFormat, int kDim, int kRows>
__global__ void __launch_bounds__(kSimtThreads, 2) tree_attention_simt_kernel(const __grid_constant__ TreeAttnParams p) {
  extern __shared__ __align__(16) float smem[];
  float* Ks = smem;                             // [64][kDim + 4]
  float* Vs = Ks + kSimtKeys * (kDim + 4);      // [64][kDim]
  float* Qs = Vs + kSimtKeys * kDim;            // [rows][kDim]
  float* Ps = Qs + kRows * kDim;                // [rows][64]
  float* row_m = Ps + kRows * kSimtKeys;        // [rows]
  float* row_l = row_m + kRows;                 // [rows]
  float* row_a = row_l + kRows;                 // [rows] factor of this step's rescaling
  unsigned* exists = reinterpret_cast<unsigned*>(row_a + kRows);  // [2] bits: the position has a page
  const int seq = blockIdx.z, kvh = blockIdx.y;
  const int split = blockIdx.x % p.n_splits, tile = blockIdx.x / p.n_splits;
  const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5;
  const Sequence s = load_sequence(p, seq, tid == 0 && blockIdx.x == 0 && kvh == 0);
  const int rows = min(s.n_rows, p.max_rows) * p.group;  // of this key/value head
  const int r0 = tile * kRows;
  if (r0 >= rows) return;
  const int begin = split * p.chunk, end = min(s.len, begin + p.chunk);
  if (split > 0 && begin >= s.len) return;

  constexpr int kElems = Codes<kFormat>::kElems, kPieces = kDim / kElems;
  constexpr int kEach = kSimtKeys * kPieces / kSimtThreads;  // pieces of a thread per step
  constexpr bool kQuant = kFormat != WF_CACHE_PATH;
  uint4 kraw[kEach], vraw[kEach];
  unsigned short kscale[kEach], vscale[kEach];
  bool there[kEach];
  int page_at[kEach];  // pages are looked up a step before what lies in them is loaded
  auto look_up = [&](int k0) {
#pragma unroll
    for (int i = 0; i < kEach; ++i) {
      const int pos = k0 + (i * kSimtThreads + tid) / kPieces;
      page_at[i] = pos < end ? __ldg(p.rows.page_table + (long)seq * p.rows.table_stride + (pos >> p.cache.page_shift)) : -1;
    }
  };
  auto load = [&](int k0) {
#pragma unroll
    for (int i = 0; i < kEach; ++i) {
      const int u = i * kSimtThreads + tid, pos = k0 + u / kPieces, page = page_at[i];
      there[i] = page >= 0 && page < p.cache.n_pages;
      if (pos < end && !there[i]) report(p.status, kBadPage);
      kraw[i] = vraw[i] = make_uint4(0, 0, 0, 0);
      kscale[i] = vscale[i] = 0;
      if (there[i]) {
        const long at = (((long)page * p.cache.n_kv_head + kvh) << p.cache.page_shift) + (pos & ((1 << p.cache.page_shift) - 1));
        kraw[i] = __ldcs(reinterpret_cast<const uint4*>(p.cache.k) + at * kPieces + u % kPieces);
        vraw[i] = __ldcs(reinterpret_cast<const uint4*>(p.cache.v) + at * kPieces + u % kPieces);
        if constexpr (kQuant) {
          kscale[i] = __ldg(reinterpret_cast<const unsigned short*>(p.cache.k_scale) + at);
          vscale[i] = __ldg(reinterpret_cast<const unsigned short*>(p.cache.v_scale) + at);
        }
      }
    }
    look_up(k0 + kSimtKeys);
  };
  if (begin < end) {
    look_up(begin);
    load(begin);
  }
  const float* q = reinterpret_cast<const float*>(p.q);
  for (int i = tid; i < kRows * kDim / 4; i += kSimtThreads) {
    const int r = r0 + i / (kDim / 4), row = r / p.group;
    reinterpret_cast<float4*>(Qs)[i] =
        r < rows ? __ldg(reinterpret_cast<const float4*>(q + (long)(s.first_row + row) * p.q_stride + (long)(kvh * p.group + r - row * p.group) * kDim) + i % (kDim / 4))
                 : make_float4(0.f, 0.f, 0.f, 0.f);
  }
  if (tid < kRows) row_m[tid] = -INFINITY, row_l[tid] = 0.f;
  constexpr int kOut = kRows * kDim / kSimtThreads;  // rows a thread accumulates (one channel)
  const int ch = tid % kDim, out_r0 = (tid / kDim) * kOut;
  float acc[kOut];
#pragma unroll
  for (int i = 0; i < kOut; ++i) acc[i] = 0.f;

  for (int k0 = begin; k0 < end; k0 += kSimtKeys) {
    __syncthreads();
    if (tid < 2) exists[tid] = 0;
    __syncthreads();
#pragma unroll
    for (int i = 0; i < kEach; ++i) {
      const int u = i * kSimtThreads + tid, key = u / kPieces, c = u % kPieces * kElems;
      float xk[kElems], xv[kElems];
      Codes<kFormat>::unpack(kraw[i], __uint_as_float((uint32_t)kscale[i] << 16), xk);
      Codes<kFormat>::unpack(vraw[i], __uint_as_float((uint32_t)vscale[i] << 16), xv);
#pragma unroll
      for (int e = 0; e < kElems; e += 4) {
        *reinterpret_cast<float4*>(Ks + key * (kDim + 4) + c + e) = make_float4(xk[e], xk[e + 1], xk[e + 2], xk[e + 3]);
        *reinterpret_cast<float4*>(Vs + key * kDim + c + e) = make_float4(xv[e], xv[e + 1], xv[e + 2], xv[e + 3]);
      }
      if (there[i] && c == 0) atomicOr(&exists[key >> 5], 1u << (key & 31));
    }
    __syncthreads();
    if (k0 + kSimtKeys < end) load(k0 + kSimtKeys);
    {  // scores: a thread has one position and a quarter of the rows
      constexpr int kEachRow = kRows / 4;
      const int key = tid & 63, rr = (tid >> 6) * kEachRow;
      float sc[kEachRow];
#pragma unroll
      for (int i = 0; i < kEachRow; ++i) sc[i] = 0.f;
#pragma unroll 8
      for (int c = 0; c < kDim; c += 4) {
        const float4 k4 = *reinterpret_cast<const float4*>(Ks + key * (kDim + 4) + c);
#pragma unroll
        for (int i = 0; i < kEachRow; ++i) {
          const float4 q4 = *reinterpret_cast<const float4*>(Qs + (rr + i) * kDim + c);
          sc[i] = fmaf(q4.x, k4.x, sc[i]);
          sc[i] = fmaf(q4.y, k4.y, sc[i]);
          sc[i] = fmaf(q4.z, k4.z, sc[i]);
          sc[i] = fmaf(q4.w, k4.w, sc[i]);
        }
      }
      const int pos = k0 + key;
      const bool have = (exists[key >> 5] >> (key & 31)) & 1;
#pragma unroll
      for (int i = 0; i < kEachRow; ++i) {
        const int r = r0 + rr + i;
        const bool see = have && r < rows && (pos < s.start || sees_tail(p, s, r / p.group, pos - s.start));
        Ps[(rr + i) * kSimtKeys + key] = see ? sc[i] * p.scale : -INFINITY;
      }
    }
    __syncthreads();
#pragma unroll
    for (int i = 0; i < kRows / 8; ++i) {  // softmax: a warp has one row or two
      const int r = warp * (kRows / 8) + i;
      const float a = Ps[r * kSimtKeys + lane], b = Ps[r * kSimtKeys + lane + 32];
      float mx = fmaxf(a, b);
      const bool nan = a != a || b != b;  // a NaN score that the row sees makes the row NaN
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
      __syncwarp();
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
    auto accumulate = [&](auto guard_tag) {
      constexpr bool kGuard = decltype(guard_tag)::value;
#pragma unroll 4
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
            if (!kGuard || pj[j] != 0.f) acc[i] = fmaf(pj[j], v[j], acc[i]);
        }
      }
    };
    if (k0 + kSimtKeys > s.start) accumulate(std::true_type{});
    else accumulate(std::false_type{});
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
      reinterpret_cast<float*>(p.out)[row * p.out_stride + (long)head * kDim + ch] = l == 0.f ? 0.f : acc[i] / l;
      if (ch == 0 && p.lse) p.lse[row * p.n_head + head] = l == 0.f ? -INFINITY : m + logf(l);
    }
  }
}

// Joins the splits of a row: one block per (row, head).  The splits' weights e^(m_i - m) first, all at once, then a sum over
// the splits by groups of kDim threads, whose parts are added in group order.  Bound by latency (the partial sums are in the L2):
// with many splits 256 threads (139 splits of 64 channels: 30 -> 13 us with the kernel before it), with few one group, as there
// are many rows then (5 splits, 12,800 rows and heads: 124 -> 107 us with the kernel before it).
template <typename T, int kDim, int kJoinThreads>
__global__ void __launch_bounds__(kJoinThreads) tree_attention_join_kernel(const __grid_constant__ TreeAttnParams p) {
  extern __shared__ __align__(16) float weight[];  // [n_splits]
  __shared__ float red_m[kJoinThreads / 32], red_l[kJoinThreads / 32], part[kJoinThreads];
  constexpr int kGroups = kJoinThreads / kDim;
  const int row = blockIdx.x, head = blockIdx.y, tid = threadIdx.x, ch = tid % kDim, group = tid / kDim;
  ptx::griddep_wait();  // the partial sums are the kernel's before this one
  const int seq = warp_find_sequence(p.rows.cu_rows, p.rows.n_seq, row);
  const Sequence s = load_sequence(p, seq, false);
  if (row < s.first_row || row - s.first_row >= min(s.n_rows, p.max_rows)) return;
  const int n = max(1, (s.len + p.chunk - 1) / p.chunk);
  const long at = ((long)row * p.n_head + head) * p.n_splits;
  float m = -INFINITY;
  bool nan = false;
  for (int i = tid; i < n; i += kJoinThreads) {
    const float mi = p.part_ml[at + i].x;
    nan |= mi != mi;
    m = fmaxf(m, mi);
  }
#pragma unroll
  for (int o = 16; o > 0; o >>= 1) m = fmaxf(m, __shfl_xor_sync(0xffffffffu, m, o));
  if (__any_sync(0xffffffffu, nan)) m = __int_as_float(0x7fc00000);
  if (tid % 32 == 0) red_m[tid / 32] = m;
  __syncthreads();
#pragma unroll
  for (int w = 0; w < kJoinThreads / 32; ++w) m = (m != m || red_m[w] != red_m[w]) ? __int_as_float(0x7fc00000) : fmaxf(m, red_m[w]);
  const float base = m == -INFINITY ? 0.f : m;
  float l = 0.f;
  for (int i = tid; i < n; i += kJoinThreads) {
    const float2 ml = p.part_ml[at + i];
    const float f = expf(ml.x - base);
    weight[i] = ml.y != 0.f ? f : 0.f;
    l += ml.y * f;
  }
#pragma unroll
  for (int o = 16; o > 0; o >>= 1) l += __shfl_xor_sync(0xffffffffu, l, o);
  if (tid % 32 == 0) red_l[tid / 32] = l;
  __syncthreads();
  l = 0.f;
#pragma unroll
  for (int w = 0; w < kJoinThreads / 32; ++w) l += red_l[w];
  float o = 0.f;
#pragma unroll 8
  for (int i = group; i < n; i += kGroups) {
    const float f = weight[i], x = p.part_o[(at + i) * kDim + ch];
    if (f != 0.f) o = fmaf(x, f, o);
  }
  part[tid] = o;
  __syncthreads();
  if (group != 0) return;
  o = part[ch];
#pragma unroll
  for (int w = 1; w < kGroups; ++w) o += part[w * kDim + ch];
  put(reinterpret_cast<T*>(p.out) + (long)row * p.out_stride + (long)head * kDim + ch, l == 0.f ? 0.f : o / l);
  if (ch == 0 && p.lse) p.lse[(long)row * p.n_head + head] = l == 0.f ? -INFINITY : m + logf(l);
}

template <int kFormat, int kDim, int kRows>
cudaError_t launch_simt_rows(const TreeAttnParams& p, cudaStream_t s) {
  const int tiles = (int)(((long)p.max_rows * p.group + kRows - 1) / kRows);
  const dim3 grid((unsigned)(tiles * p.n_splits), (unsigned)p.cache.n_kv_head, (unsigned)p.rows.n_seq);
  auto kernel = tree_attention_simt_kernel<kFormat, kDim, kRows>;
  constexpr size_t smem = simt_smem<kDim, kRows>();
  cudaError_t e = cudaFuncSetAttribute(kernel, cudaFuncAttributeMaxDynamicSharedMemorySize, (int)smem);
  if (e == cudaSuccess) e = launch_dependent(kernel, grid, dim3(kSimtThreads), smem, s, 1, false, p);
  return e;
}
int simt_rows(long rows) { return rows <= 8 ? 8 : 16; }
template <int kFormat, int kDim>
cudaError_t launch_simt(const TreeAttnParams& p, cudaStream_t s) {
  return simt_rows((long)p.max_rows * p.group) == 8 ? launch_simt_rows<kFormat, kDim, 8>(p, s) : launch_simt_rows<kFormat, kDim, 16>(p, s);
}

// More rows of a key/value head than fit one tile of the kernel for few rows go to the kernel with 128-row tiles.  Measured, that kernel /
// the one for few rows in us: 8 sequences of 1000 positions, 8 heads of 64 channels, e4m3: 24 rows 17.4 / 16.2, 40 rows 18.7 / 22.7,
// 100 rows 24 / 28; 32 sequences of 300 positions, 128 channels, int8: 12 rows 16.8 / 13.3, 24 rows 16.8 / 24.2, 40 rows 18.8 / 36, 160 rows
// 41 / 125.
int wide_rows(int d_head) { return d_head == 64 ? 32 : 16; }

// Rows of one tile of the kernel for few rows.
int tc_rows(int d_head, long rows) { return rows <= 8 ? 8 : rows <= 16 || d_head == 128 ? 16 : 32; }

template <typename T, int kDim>
cudaError_t launch_format(const TreeAttnParams& p, int format, cudaStream_t s) {
  cudaError_t e;
  if constexpr (sizeof(T) == 2)
    e = p.unit_warps == 0 ? launch_tree_attention_wide(p, kDim, format, s)
                          : launch_tree_attention_tc(p, kDim, format, tc_rows(kDim, (long)p.max_rows * p.group), s);
  else
    e = format == WF_CACHE_PATH   ? launch_simt<WF_CACHE_PATH, kDim>(p, s)
        : format == WF_CACHE_E4M3 ? launch_simt<WF_CACHE_E4M3, kDim>(p, s)
                                  : launch_simt<WF_CACHE_INT8, kDim>(p, s);
  if (e == cudaSuccess && p.n_splits > 1)
    e = launch_dependent(p.n_splits > 16 ? tree_attention_join_kernel<T, kDim, 256> : tree_attention_join_kernel<T, kDim, kDim>,
                         dim3((unsigned)p.rows.n_rows, (unsigned)p.n_head), dim3(p.n_splits > 16 ? 256 : kDim), p.n_splits * sizeof(float), s, 1,
                         true, p);
  return e;
}

}  // namespace

TreeAttnPlan plan_tree_attention(int dtype, int d_head, int n_head, int n_kv_head, int n_seq, int n_rows, int max_rows, int max_len,
                                 int num_sms) {
  TreeAttnPlan plan{};
  const long rows = (long)max_rows * (n_head / n_kv_head);
  const bool wide = dtype == WF_BF16 && rows > wide_rows(d_head);
  const int tile = wide ? 128 : dtype == WF_BF16 ? tc_rows(d_head, rows) : simt_rows(rows);
  const long tiles = (rows + tile - 1) / tile;
  const long units = tiles * n_kv_head * n_seq;
  if (wide) {
    // two blocks of an SM; sequences differ in length, so more blocks than fit at once even the load out, as long as a
    // block's start (7 us of its 35 at 768 positions) stays small.  Splits of at least 256 / 768 positions, or none, measured in us: 448
    // positions, 20 heads, 448 rows 28 / 19 / 19; 2 x 100 rows, 20 heads, 800 .. 1500 positions 22 / 25 / 31; 64 rows, 8 heads, 1500
    // positions 16 / 28 / 44 (few tiles would gain from shorter ones); 16 x 48 rows, 32 / 8 heads, 100 .. 4096 positions 184 / 184 / 167.
    const long splits = std::max(1L, std::min((8L * num_sms + units - 1) / units, ((long)max_len + 767) / 768));
    plan.unit_warps = 0;
    plan.chunk = (int)(((long)max_len + splits * 64 - 1) / (splits * 64) * 64);
  } else if (dtype == WF_BF16) {
    // Warps taken to reside on an SM, by tile: 16, 12 or 8 (the launch bounds let 20, 12 and 8; shared memory 12 in 8-row tiles of
    // unquantised caches of 128 channels).  A unit is shared by as few warps as fill them (each one has a start and an end to pay for).
    // Four / two / one warp a unit, measured in us: single tokens of 320 sequences, 20 heads of 64 channels, e4m3, up to 219 positions
    // (6400 units) 47 / 41 / 34, of 640 sequences 90 / 75 / 58, 160 sequences of up to 448 positions, 32 heads of 128 84 / 86 / 94;
    // 900 x 5 rows, 32 / 8 heads of 64, 50 .. 300 positions 276 / 186 / 143.
    // And cut into splits, all of one wave, where four are not enough, of at least 256 positions: 64 / 256 / 1024, measured in us: one
    // token of one sequence, 1000 positions, 8 heads of 128, bfloat16 7.5 / 10.4 / 19; 5000 positions of one head 8.1 / 8.2 / 13; 448
    // positions, 20 heads 8.5 / 7.7 / 6.9.
    const long resident = (long)num_sms * (tile == 8 ? 16 : tile == 16 && d_head == 64 ? 12 : 8);
    plan.unit_warps = units >= 4 * resident ? 1 : units >= 2 * resident ? 2 : 4;
    const long splits = std::max(1L, std::min(resident / (4 * units), ((long)max_len + 255) / 256));
    plan.chunk = (int)(((long)max_len + splits * 64 - 1) / (splits * 64) * 64);
  } else {
    // as many splits as fit the SMs at two blocks each, of at least 128 positions
    const long splits = std::max(1L, std::min(2L * num_sms / units, ((long)max_len + 127) / 128));
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
