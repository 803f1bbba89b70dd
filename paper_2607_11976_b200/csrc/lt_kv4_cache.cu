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
// it is needed.  Launch latency bounds it: 4 us of GPU time for 64 requests with one token each, 8 for 701 with 359 K tokens; a call
// through the binding takes 7 either way.
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
// magnitude.  16 threads (D = 128) hold a head's keys and the 16 beside them its values, so a warp writes whole rows.  It reads
// 2 Hkv D elements a token and writes 9 / 16 byte for each; instructions bound it, not HBM.  Quantising alone took 16 an element
// (65,536 tokens of 8 heads of 128: 200 us), so ordinary groups of bf16 take a shorter way of 6: the quotient by a reciprocal and one
// correction, the nibble from the bits of a sum that rounds.  With walking, addresses, shuffles and stores the kernel still executes 19 an
// element (80 M warp instructions for 134 M elements): 98 us, 3.5 TB/s, 0.74 of the issue slots.
// ---------------------------------------------------------------------------------------------
constexpr int kCacheThreads = 256;
constexpr int kCacheAhead = 4;  // loads in flight per thread

// A thread's place in the row of (token, head) items, kept up by additions.
struct ItemWalk {
  long long t;
  int h;
  __device__ __forceinline__ ItemWalk(long long item, int heads) : t(item / heads), h(static_cast<int>(item - t * heads)) {}
  __device__ __forceinline__ void add(long long dt, int dh, int heads) {
    t += dt;
    h += dh;
    if (h >= heads) {
      h -= heads;
      ++t;
    }
  }
};

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
// Largest magnitude's bits; a NaN counts above infinity here.
__device__ __forceinline__ uint32_t top_bits(const Vec8<__nv_bfloat16>& v) {
  const uint32_t k = 0x7fff7fffu;
  const uint32_t m = __vmaxu2(__vmaxu2(v.raw[0].x & k, v.raw[0].y & k), __vmaxu2(v.raw[0].z & k, v.raw[0].w & k));
  return max(m & 0xffffu, m >> 16) << 16;
}
__device__ __forceinline__ uint32_t top_bits(const Vec8<float>& v) {
  uint32_t m = 0;
#pragma unroll
  for (int i = 0; i < 2; ++i)
    m = max(m, max(max(v.raw[i].x & 0x7fffffffu, v.raw[i].y & 0x7fffffffu), max(v.raw[i].z & 0x7fffffffu, v.raw[i].w & 0x7fffffffu)));
  return m;
}

// Eight codes of ordinary bf16 values: the scale is a normal fp16 number and not cut off at its maximum, so |x / s| < 7.1.  x and s have 8
// significant bits: x / s is a tie between two integers exactly, or off by 2^-8 of itself or more.  q + (x - q s) inv is the quotient
// rounded once, so a tie is met exactly; 1.5 * 2^23 + 8 + q then rounds to the nearest integer, ties to even, and has code = 8 + n in its
// lowest bits.  The constant's bits, shifted along, sum up to another constant.
__device__ __forceinline__ uint32_t ordinary_codes(const float (&x)[8], float s, float inv) {
  uint32_t sum = 0;
#pragma unroll
  for (int i = 7; i >= 0; --i) {
    const float q = x[i] * inv, exact = __fmaf_rn(__fmaf_rn(-q, s, x[i]), inv, q);
    sum = (sum << 4) + __float_as_uint(exact + 12582920.f);
  }
  constexpr uint32_t kBits = 0x4B400000u;  // 1.5 * 2^23; its copies from the third on fall out at the top, but for their lowest bits
  constexpr uint32_t kAll = kBits + (kBits << 4) + (kBits << 8) + (kBits << 12) + (kBits << 16) + (kBits << 20) + (kBits << 24) + (kBits << 28);
  return sum - kAll;
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
  constexpr int kPer = D / 4;  // threads of one (token, head): keys and values, 8 elements each
  constexpr int kRow = kv4_row_bytes(D), kItems = kCacheThreads / kPer;
  const int sub = threadIdx.x % kPer;
  const bool is_v = sub >= kPer / 2;
  const int e = (sub % (kPer / 2)) * 8;  // first element
  const In* src = is_v ? static_cast<const In*>(p.v) : static_cast<const In*>(p.k);
  const long long stride = is_v ? p.v_stride : p.k_stride;
  const int step = gridDim.x * kItems, dt = step / p.Hkv, dh = step - dt * p.Hkv;
  ItemWalk at(blockIdx.x * kItems + threadIdx.x / kPer, p.Hkv);
  // (whole warps stay in the loop, the shuffles below name all lanes: it runs as long as the CTA's first item is there)
  ItemWalk lead(blockIdx.x * kItems, p.Hkv);
  while (lead.t < p.T) {
    Vec8<In> x[kCacheAhead];
    int slot[kCacheAhead], head[kCacheAhead];
#pragma unroll
    for (int a = 0; a < kCacheAhead; ++a) {
      slot[a] = -1;
      head[a] = at.h;
#pragma unroll
      for (int i = 0; i < static_cast<int>(sizeof(In) / 2); ++i) x[a].raw[i] = make_uint4(0, 0, 0, 0);
      if (at.t < p.T) {
        slot[a] = p.slot_map[at.t];
        const uint4* from = reinterpret_cast<const uint4*>(src + at.t * stride + at.h * D + e);
#pragma unroll
        for (int i = 0; i < static_cast<int>(sizeof(In) / 2); ++i) x[a].raw[i] = __ldg(from + i);
      }
      at.add(dt, dh, p.Hkv);
      lead.add(dt, dh, p.Hkv);
    }
#pragma unroll
    for (int a = 0; a < kCacheAhead; ++a) {
      uint32_t top = top_bits(x[a]);
      top = max(top, __shfl_xor_sync(0xffffffffu, top, 1));
      top = max(top, __shfl_xor_sync(0xffffffffu, top, 2));
      float f[8];
      unpack8(x[a], f);
      __half scale = kv4_scale(__uint_as_float(top));
      const float s = __half2float(scale);
      uint32_t codes = 0;
      if (sizeof(In) == 2 && top <= 0x46600000u && s >= 0x1p-14f) {  // (14336 = 7 * 2048)
        codes = ordinary_codes(f, s, __fdividef(1.f, s));
      } else {
        float amax = 0.f;  // without the NaN
#pragma unroll
        for (int i = 0; i < 8; ++i) amax = fmaxf(amax, fabsf(f[i]));
        const unsigned quad = 0xfu << (threadIdx.x & 28);  // (a group's four threads take the same way)
        amax = fmaxf(amax, __shfl_xor_sync(quad, amax, 1));
        amax = fmaxf(amax, __shfl_xor_sync(quad, amax, 2));
        scale = kv4_scale(amax);
        const float t = __half2float(scale), inv = t > 0.f ? 1.f / t : 0.f;
#pragma unroll
        for (int i = 0; i < 8; ++i) codes |= kv4_code(f[i], t, inv) << (4 * i);
      }
      if (slot[a] < 0 || slot[a] >= p.pool_rows) continue;
      uint8_t* row = p.pool + ((static_cast<long long>(slot[a] / kPageKeys) * p.Hkv + head[a]) * kPageKeys + slot[a] % kPageKeys) * kRow;
      *reinterpret_cast<uint32_t*>(row + sub * 4) = codes;
      if ((sub & 3) == 0) *reinterpret_cast<__half*>(row + D + (sub / 4) * 2) = scale;
    }
  }
}

// ---------------------------------------------------------------------------------------------
// Reader: the values that the cache holds, in the caller's type (rounded once); zeros where there is no slot.  A code with a constant
// or-ed into an exponent is 128 + u (bf16 pairs: one more subtraction and the product, exact up to its rounding) or 2^23 + u (fp32).
// 65,536 slots of 8 heads of 128 to bf16: 70 us, 4.9 TB/s.
// ---------------------------------------------------------------------------------------------
struct ReadParams {
  const uint8_t* pool;
  long long pool_rows;
  const int32_t* slots;
  int n, Hkv;
  void* k_out;
  void* v_out;
};

__device__ __forceinline__ uint32_t bf16x2_fma(uint32_t a, uint32_t b, uint32_t c) {
  uint32_t d;
  asm("fma.rn.bf16x2 %0, %1, %2, %3;" : "=r"(d) : "r"(a), "r"(b), "r"(c));
  return d;
}
__device__ __forceinline__ void store8(__nv_bfloat16* at, uint32_t codes, __half scale) {
  const uint32_t s = __bfloat16_as_ushort(__float2bfloat16_rn(__half2float(scale))), s2 = s | (s << 16);  // (8 bits: exact)
  uint32_t w[4];
#pragma unroll
  for (int i = 0; i < 4; ++i) {  // elements i and i + 4
    const uint32_t v = bf16x2_fma(((codes >> (4 * i)) & 0x000F000Fu) | 0x43004300u, 0x3F803F80u, 0xC308C308u);  // 128 + u - 136
    w[i] = bf16x2_fma(v, s2, 0x80008000u);                                                                     // v s - 0
  }
  *reinterpret_cast<uint4*>(at) = make_uint4(__byte_perm(w[0], w[1], 0x5410), __byte_perm(w[2], w[3], 0x5410), __byte_perm(w[0], w[1], 0x7632),
                                             __byte_perm(w[2], w[3], 0x7632));
}
__device__ __forceinline__ void store8(float* at, uint32_t codes, __half scale) {
  const float s = __half2float(scale);
  float x[8];
#pragma unroll
  for (int i = 0; i < 8; ++i) x[i] = (__uint_as_float(((codes >> (4 * i)) & 15u) | 0x4B000000u) - 8388616.f) * s;
  reinterpret_cast<float4*>(at)[0] = make_float4(x[0], x[1], x[2], x[3]);
  reinterpret_cast<float4*>(at)[1] = make_float4(x[4], x[5], x[6], x[7]);
}

template <typename Out, int D>
__global__ void __launch_bounds__(kCacheThreads) read_kernel(const ReadParams p) {
  chain_wait();
  constexpr int kPer = D / 4;
  constexpr int kRow = kv4_row_bytes(D), kItems = kCacheThreads / kPer;
  const int sub = threadIdx.x % kPer;
  const int e = (sub % (kPer / 2)) * 8;
  Out* out = static_cast<Out*>(sub >= kPer / 2 ? p.v_out : p.k_out);
  const int step = gridDim.x * kItems, dt = step / p.Hkv, dh = step - dt * p.Hkv;
  ItemWalk at(blockIdx.x * kItems + threadIdx.x / kPer, p.Hkv);
  while (at.t < p.n) {
    uint32_t codes[kCacheAhead];
    __half scale[kCacheAhead];
    Out* to[kCacheAhead];
    int slot[kCacheAhead];
    ItemWalk place = at;
#pragma unroll
    for (int a = 0; a < kCacheAhead; ++a) {
      slot[a] = place.t < p.n ? p.slots[place.t] : -1;
      place.add(dt, dh, p.Hkv);
    }
#pragma unroll
    for (int a = 0; a < kCacheAhead; ++a) {
      codes[a] = 0x88888888u;
      scale[a] = __ushort_as_half(0);
      to[a] = at.t < p.n ? out + (at.t * p.Hkv + at.h) * D + e : nullptr;
      if (slot[a] >= 0 && slot[a] < p.pool_rows) {
        const uint8_t* row = p.pool + ((static_cast<long long>(slot[a] / kPageKeys) * p.Hkv + at.h) * kPageKeys + slot[a] % kPageKeys) * kRow;
        codes[a] = *reinterpret_cast<const uint32_t*>(row + sub * 4);
        scale[a] = *reinterpret_cast<const __half*>(row + D + (sub / 4) * 2);
      }
      at.add(dt, dh, p.Hkv);
    }
#pragma unroll
    for (int a = 0; a < kCacheAhead; ++a)
      if (to[a] != nullptr) store8(to[a], codes[a], scale[a]);
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
