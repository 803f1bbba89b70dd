// Block tables of a step, and the writer and reader of the 4-bit key-value cache.
#include "lt_kv4.cuh"

namespace lt {
namespace {

// ---------------------------------------------------------------------------------------------
// Block tables, slot map and positions of a step from the requests' lengths.
//
// Two prefix sums over the requests say where each one's tokens and fresh pages begin; the tokens and pages are then dealt out
// evenly over the CTAs, whichever requests they belong to.  Every CTA takes the sums itself (64 requests are one load per thread),
// so that one launch does it all and no CTA waits for another; a fresh page's number is read from the free list, by its rank, where
// it is needed.  Launch latency bounds it:
// 8 us a call through the binding, 64 requests with one token each as well as 701 with 359 K.
// ---------------------------------------------------------------------------------------------
constexpr int kTabThreads = 1024;

struct TableParams {
  const int32_t* context_len;
  const int32_t* new_len;
  const int32_t* free_pages;
  int n_free;
  int B, max_pages, T;
  int32_t* page_table;
  int32_t* total_len;
  int32_t* query_start;
  int32_t* slot_map;
  int32_t* position;
  int32_t* status;
};

// Exclusive sums of two counts over the CTA's threads; returns the totals.
__device__ __forceinline__ void scan2(long long& a, long long& b, long long& sum_a, long long& sum_b, long long (*warp_sums)[2]) {
  const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
  long long ia = a, ib = b;
#pragma unroll
  for (int d = 1; d < 32; d <<= 1) {
    const long long ta = __shfl_up_sync(0xffffffffu, ia, d), tb = __shfl_up_sync(0xffffffffu, ib, d);
    if (lane >= d) {
      ia += ta;
      ib += tb;
    }
  }
  if (lane == 31) {
    warp_sums[warp][0] = ia;
    warp_sums[warp][1] = ib;
  }
  __syncthreads();
  long long wa = warp_sums[lane][0], wb = warp_sums[lane][1];
  const long long own_a = wa, own_b = wb;
#pragma unroll
  for (int d = 1; d < 32; d <<= 1) {
    const long long ta = __shfl_up_sync(0xffffffffu, wa, d), tb = __shfl_up_sync(0xffffffffu, wb, d);
    if (lane >= d) {
      wa += ta;
      wb += tb;
    }
  }
  sum_a = __shfl_sync(0xffffffffu, wa, 31);
  sum_b = __shfl_sync(0xffffffffu, wb, 31);
  a = ia - a + __shfl_sync(0xffffffffu, wa - own_a, warp);
  b = ib - b + __shfl_sync(0xffffffffu, wb - own_b, warp);
  __syncthreads();
}

// The last i in [0, n) with first[i] <= x (first[0] <= x, ascending).
__device__ __forceinline__ int last_not_above(const long long* first, int n, long long x) {
  int lo = 0, hi = n;
  while (hi - lo > 1) {
    const int mid = (lo + hi) >> 1;
    if (first[mid] <= x) lo = mid; else hi = mid;
  }
  return lo;
}

__global__ void __launch_bounds__(kTabThreads) page_tables_kernel(const TableParams p) {
  chain_wait();
  __shared__ long long warp_sums[32][2];
  __shared__ long long s_start[kTabThreads + 1], s_first[kTabThreads + 1];
  __shared__ int s_ctx[kTabThreads], s_old[kTabThreads];
  const int tid = threadIdx.x;
  long long tokens = 0, pages = 0;  // of the requests before this chunk
  int bad = 0;
  for (int base = 0; base < p.B; base += kTabThreads) {
    const int b = base + tid;
    long long ctx = 0, add = 0, need = 0;
    int old = 0;
    if (b < p.B) {
      ctx = p.context_len[b];
      add = p.new_len[b];
      if (ctx < 0 || add < 0) bad = 1;
      ctx = ctx < 0 ? 0 : ctx;
      add = add < 0 ? 0 : add;
      const long long pages_old = (ctx + kPageKeys - 1) / kPageKeys;
      long long pages_all = (ctx + add + kPageKeys - 1) / kPageKeys;
      if (pages_all > p.max_pages) bad = 1;
      pages_all = pages_all > p.max_pages ? p.max_pages : pages_all;
      old = static_cast<int>(pages_old > p.max_pages ? p.max_pages : pages_old);
      need = pages_all - old;
    }
    long long start = add, first = need, sum_tokens, sum_pages;
    scan2(start, first, sum_tokens, sum_pages, warp_sums);
    s_start[tid] = tokens + start;
    s_first[tid] = pages + first;
    s_ctx[tid] = static_cast<int>(ctx);
    s_old[tid] = old;
    const int n = p.B - base < kTabThreads ? p.B - base : kTabThreads;
    if (blockIdx.x == 0 && b < p.B) {
      const long long at = tokens + start, total = ctx + add;
      p.query_start[b] = static_cast<int32_t>(at > p.T ? p.T : at);
      p.total_len[b] = static_cast<int32_t>(total > 0x7fffffff ? 0x7fffffff : total);
    }
    __syncthreads();
    // the chunk's fresh pages
    for (long long r = pages + static_cast<long long>(blockIdx.x) * kTabThreads + tid; r < pages + sum_pages;
         r += static_cast<long long>(gridDim.x) * kTabThreads) {
      const int i = last_not_above(s_first, n, r);
      p.page_table[static_cast<long long>(base + i) * p.max_pages + s_old[i] + (r - s_first[i])] = r < p.n_free ? p.free_pages[r] : -1;
    }
    // its tokens
    const long long end = tokens + sum_tokens < p.T ? tokens + sum_tokens : p.T;
    for (long long t = tokens + static_cast<long long>(blockIdx.x) * kTabThreads + tid; t < end;
         t += static_cast<long long>(gridDim.x) * kTabThreads) {
      const int i = last_not_above(s_start, n, t);
      const long long pos = s_ctx[i] + (t - s_start[i]), page = pos / kPageKeys;
      long long at = -1;
      if (page < s_old[i]) {
        at = p.page_table[static_cast<long long>(base + i) * p.max_pages + page];
      } else if (page < p.max_pages) {
        const long long r = s_first[i] + (page - s_old[i]);
        if (r < p.n_free) at = p.free_pages[r];
      }
      at = at < 0 ? -1 : at * kPageKeys + pos % kPageKeys;
      p.slot_map[t] = static_cast<int32_t>(at > 0x7fffffff ? -1 : at);
      p.position[t] = static_cast<int32_t>(pos > 0x7fffffff ? 0x7fffffff : pos);
    }
    tokens += sum_tokens;
    pages += sum_pages;
    __syncthreads();
  }
  // the rest of a padded batch
  for (long long t = tokens + static_cast<long long>(blockIdx.x) * kTabThreads + tid; t < p.T;
       t += static_cast<long long>(gridDim.x) * kTabThreads) {
    p.slot_map[t] = -1;
    p.position[t] = -1;
  }
  if (blockIdx.x != 0) return;
  bad = __syncthreads_or(bad);
  if (tid == 0) {
    p.query_start[p.B] = static_cast<int32_t>(tokens > p.T ? p.T : tokens);
    const long long missing = pages > p.n_free ? pages - p.n_free : 0;
    p.status[0] = bad != 0 || missing > 0 || tokens > p.T ? LT_STATUS_SHORT : 0;
    p.status[1] = static_cast<int32_t>(tokens > 0x7fffffff ? 0x7fffffff : tokens);
    p.status[2] = static_cast<int32_t>(pages - missing);
    p.status[3] = static_cast<int32_t>(missing > 0x7fffffff ? 0x7fffffff : missing);
  }
  if (tid >= 4 && tid < 8) p.status[tid] = 0;
}

// ---------------------------------------------------------------------------------------------
// Writer.  A thread takes 8 consecutive elements (one or two 16-byte loads), four threads share a group: two shuffles give its largest
// magnitude.  16 threads (D = 128) hold a head's keys and the 16 beside them its values, so a warp writes whole rows.  HBM bound:
// it reads 2 Hkv D elements a token and writes 9 / 16 byte for each.
// ---------------------------------------------------------------------------------------------
constexpr int kCacheThreads = 256;

template <typename In>
struct Vec8 {
  uint4 raw[sizeof(In) / 2];
};
__device__ __forceinline__ void unpack8(const Vec8<__nv_bfloat16>& v, float (&x)[8]) {
  const uint32_t w[4] = {v.raw[0].x, v.raw[0].y, v.raw[0].z, v.raw[0].w};
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    x[2 * i] = __uint_as_float(w[i] << 16);
    x[2 * i + 1] = __uint_as_float(w[i] & 0xffff0000u);
  }
}
__device__ __forceinline__ void unpack8(const Vec8<float>& v, float (&x)[8]) {
#pragma unroll
  for (int i = 0; i < 2; ++i) {
    x[4 * i] = __uint_as_float(v.raw[i].x);
    x[4 * i + 1] = __uint_as_float(v.raw[i].y);
    x[4 * i + 2] = __uint_as_float(v.raw[i].z);
    x[4 * i + 3] = __uint_as_float(v.raw[i].w);
  }
}

struct AppendParams {
  const void* k;
  const void* v;
  long long k_stride, v_stride;  // elements from one token's row to the next
  const int32_t* slot_map;
  int T, Hkv;
  uint8_t* pool;
  long long pool_rows;
};

template <typename In, int D>
__global__ void __launch_bounds__(kCacheThreads) append_kernel(const AppendParams p) {
  chain_wait();
  constexpr int kPer = D / 4;       // threads of one (token, head): keys and values, 8 elements each
  constexpr int kRow = kv4_row_bytes(D);
  const long long items = static_cast<long long>(p.T) * p.Hkv;
  const int sub = threadIdx.x % kPer;
  const bool is_v = sub >= kPer / 2;
  const int e = (sub % (kPer / 2)) * 8;  // first element
  constexpr int kAhead = 4;              // loads in flight per thread
  const long long step = static_cast<long long>(gridDim.x) * (kCacheThreads / kPer);
  // (whole warps stay in the loop: the shuffles below name all lanes)
  const long long first = static_cast<long long>(blockIdx.x) * (kCacheThreads / kPer) + threadIdx.x / kPer;
  for (long long base = first - threadIdx.x / kPer; base < items; base += step * kAhead) {
    Vec8<In> x[kAhead];
    long long slot[kAhead];
    int head[kAhead];
#pragma unroll
    for (int a = 0; a < kAhead; ++a) {
      const long long item = base + a * step + threadIdx.x / kPer;
      slot[a] = -1;
      head[a] = 0;
#pragma unroll
      for (int i = 0; i < static_cast<int>(sizeof(In) / 2); ++i) x[a].raw[i] = make_uint4(0, 0, 0, 0);
      if (item < items) {
        const long long t = item / p.Hkv;
        head[a] = static_cast<int>(item - t * p.Hkv);
        slot[a] = p.slot_map[t];
        const In* src = is_v ? static_cast<const In*>(p.v) + t * p.v_stride : static_cast<const In*>(p.k) + t * p.k_stride;
        const uint4* at = reinterpret_cast<const uint4*>(src + head[a] * D + e);
#pragma unroll
        for (int i = 0; i < static_cast<int>(sizeof(In) / 2); ++i) x[a].raw[i] = __ldg(at + i);
      }
    }
#pragma unroll
    for (int a = 0; a < kAhead; ++a) {
      float f[8];
      unpack8(x[a], f);
      float amax = 0.f;
#pragma unroll
      for (int i = 0; i < 8; ++i) amax = fmaxf(amax, fabsf(f[i]));
      amax = fmaxf(amax, __shfl_xor_sync(0xffffffffu, amax, 1));
      amax = fmaxf(amax, __shfl_xor_sync(0xffffffffu, amax, 2));
      const __half scale = kv4_scale(amax);
      const float s = __half2float(scale), inv = s > 0.f ? 1.f / s : 0.f;
      uint32_t codes = 0;
#pragma unroll
      for (int i = 0; i < 8; ++i) codes |= kv4_code(f[i], s, inv) << (4 * i);
      if (slot[a] < 0 || slot[a] >= p.pool_rows) continue;
      uint8_t* row = p.pool + (((slot[a] / kPageKeys) * p.Hkv + head[a]) * kPageKeys + slot[a] % kPageKeys) * kRow;
      *reinterpret_cast<uint32_t*>(row + sub * 4) = codes;
      if ((sub & 3) == 0) *reinterpret_cast<__half*>(row + D + (sub / 4) * 2) = scale;
    }
  }
}

// ---------------------------------------------------------------------------------------------
// Reader: the values that the cache holds, in the caller's type (rounded once); zeros where there is no slot.
// ---------------------------------------------------------------------------------------------
struct ReadParams {
  const uint8_t* pool;
  long long pool_rows;
  const int32_t* slots;
  int n, Hkv;
  void* k_out;
  void* v_out;
};

__device__ __forceinline__ void store8(__nv_bfloat16* at, const float (&x)[8]) {
  uint32_t w[4];
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    const __nv_bfloat162 h = __floats2bfloat162_rn(x[2 * i], x[2 * i + 1]);
    w[i] = *reinterpret_cast<const uint32_t*>(&h);
  }
  *reinterpret_cast<uint4*>(at) = make_uint4(w[0], w[1], w[2], w[3]);
}
__device__ __forceinline__ void store8(float* at, const float (&x)[8]) {
  reinterpret_cast<float4*>(at)[0] = make_float4(x[0], x[1], x[2], x[3]);
  reinterpret_cast<float4*>(at)[1] = make_float4(x[4], x[5], x[6], x[7]);
}

template <typename Out, int D>
__global__ void __launch_bounds__(kCacheThreads) read_kernel(const ReadParams p) {
  chain_wait();
  constexpr int kPer = D / 4;
  constexpr int kRow = kv4_row_bytes(D);
  const long long items = static_cast<long long>(p.n) * p.Hkv;
  const int sub = threadIdx.x % kPer;
  const int e = (sub % (kPer / 2)) * 8;
  Out* out = static_cast<Out*>(sub >= kPer / 2 ? p.v_out : p.k_out);
  constexpr int kAhead = 4;
  const long long step = static_cast<long long>(gridDim.x) * (kCacheThreads / kPer);
  for (long long base = static_cast<long long>(blockIdx.x) * (kCacheThreads / kPer) + threadIdx.x / kPer; base < items;
       base += step * kAhead) {
    uint32_t codes[kAhead];
    __half scale[kAhead];
#pragma unroll
    for (int a = 0; a < kAhead; ++a) {
      const long long item = base + a * step;
      codes[a] = 0x88888888u;
      scale[a] = __ushort_as_half(0);
      if (item < items) {
        const long long t = item / p.Hkv, slot = p.slots[t];
        if (slot >= 0 && slot < p.pool_rows) {
          const uint8_t* row = p.pool + (((slot / kPageKeys) * p.Hkv + (item - t * p.Hkv)) * kPageKeys + slot % kPageKeys) * kRow;
          codes[a] = *reinterpret_cast<const uint32_t*>(row + sub * 4);
          scale[a] = *reinterpret_cast<const __half*>(row + D + (sub / 4) * 2);
        }
      }
    }
#pragma unroll
    for (int a = 0; a < kAhead; ++a) {
      const long long item = base + a * step;
      if (item >= items) break;
      const float s = __half2float(scale[a]);
      float x[8];
#pragma unroll
      for (int i = 0; i < 8; ++i) x[i] = static_cast<float>(static_cast<int>((codes[a] >> (4 * i)) & 15u) - 8) * s;
      store8(out + item * D + e, x);
    }
  }
}

inline int cache_grid(long long items, int per_cta) {
  const long long want = (items + per_cta - 1) / per_cta, most = 8ll * sm_count();
  return static_cast<int>(want < most ? want : most);
}

}  // namespace

cudaError_t launch_page_tables(const int32_t* context_len, const int32_t* new_len, const int32_t* free_pages, int n_free, int B,
                               int max_pages, int T, int32_t* page_table, int32_t* total_len, int32_t* query_start,
                               int32_t* slot_map, int32_t* position, int32_t* status, cudaStream_t stream) {
  const TableParams p{context_len, new_len, free_pages, n_free, B, max_pages, T, page_table, total_len, query_start, slot_map, position, status};
  // one token per thread and pass: more tokens than the device has threads are taken in several
  const int want = (T + kTabThreads - 1) / kTabThreads, most = sm_count();
  return launch_chained(page_tables_kernel, dim3(want < 1 ? 1 : (want < most ? want : most)), dim3(kTabThreads), 0, stream, 1, p);
}

cudaError_t launch_kv4_append(int dtype, const void* k, const void* v, long long k_stride, long long v_stride,
                              const int32_t* slot_map, int T, int Hkv, int D, void* pool, long long pool_pages,
                              cudaStream_t stream) {
  const AppendParams p{k, v, k_stride, v_stride, slot_map, T, Hkv, static_cast<uint8_t*>(pool), pool_pages * kPageKeys};
  const int grid = cache_grid(static_cast<long long>(T) * Hkv, kCacheThreads / (D / 4));
  auto go = [&](auto kernel) { return launch_chained(kernel, dim3(grid), dim3(kCacheThreads), 0, stream, 1, p); };
  if (dtype == LT_DTYPE_F32) return D == 64 ? go(append_kernel<float, 64>) : go(append_kernel<float, 128>);
  return D == 64 ? go(append_kernel<__nv_bfloat16, 64>) : go(append_kernel<__nv_bfloat16, 128>);
}

cudaError_t launch_kv4_read(int dtype, const void* pool, long long pool_pages, const int32_t* slots, int n, int Hkv, int D,
                            void* k_out, void* v_out, cudaStream_t stream) {
  const ReadParams p{static_cast<const uint8_t*>(pool), pool_pages * kPageKeys, slots, n, Hkv, k_out, v_out};
  const int grid = cache_grid(static_cast<long long>(n) * Hkv, kCacheThreads / (D / 4));
  auto go = [&](auto kernel) { return launch_chained(kernel, dim3(grid), dim3(kCacheThreads), 0, stream, 1, p); };
  if (dtype == LT_DTYPE_F32) return D == 64 ? go(read_kernel<float, 64>) : go(read_kernel<float, 128>);
  return D == 64 ? go(read_kernel<__nv_bfloat16, 64>) : go(read_kernel<__nv_bfloat16, 128>);
}

}  // namespace lt
