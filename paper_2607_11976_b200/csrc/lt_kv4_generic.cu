// Attention over the 4-bit cache in fp32 throughout: the path of fp32 queries, and the plain reading of the method.
#include "lt_kv4.cuh"

namespace lt {
namespace {

constexpr int kGenWarps = 8;

__device__ __forceinline__ float to_float(float x) { return x; }
__device__ __forceinline__ float to_float(__nv_bfloat16 x) { return __bfloat162float(x); }
__device__ __forceinline__ void store_out(float* at, float x) { *at = x; }
__device__ __forceinline__ void store_out(__nv_bfloat16* at, float x) { *at = __float2bfloat16_rn(x); }

// The request of a token: the last b with query_start[b] <= t that has tokens at t; -1 behind the last request.
__device__ __forceinline__ int request_of(const Kv4AttnParams& p, int t) {
  if (t >= p.query_start[p.B]) return -1;
  int lo = 0, hi = p.B;
  while (hi - lo > 1) {
    const int mid = (lo + hi) >> 1;
    if (p.query_start[mid] <= t) lo = mid; else hi = mid;
  }
  return lo;
}

// ---------------------------------------------------------------------------------------------
// One CTA per (token, query head).  A warp takes 32 keys at a time: lane i scores key i (its codes come as 16-byte loads, the query
// lies in shared memory), the running maximum and sum are the warp's, and for the products with the values each lane holds D / 32
// elements.  The warps' results are joined at the end.  Instruction bound (5 instructions per element): fp32 queries have no tensor
// path, and a bf16 query takes it only on request.
// ---------------------------------------------------------------------------------------------
template <typename In, int D, bool kTopk>
__global__ void __launch_bounds__(kGenWarps * 32) attention_generic_kernel(const Kv4AttnParams p) {
  chain_wait();
  constexpr int kRow = kv4_row_bytes(D), kGroups = D / kKvGroup, kPer = D / 32;
  __shared__ float s_q[D];
  __shared__ float s_o[kGenWarps][D];
  __shared__ float s_m[kGenWarps], s_l[kGenWarps];
  const int t = blockIdx.x, h = blockIdx.y, kvh = h / p.group;
  if (t == 0 && h == 0 && threadIdx.x < sizeof(Control) / 4) reinterpret_cast<int*>(p.ctl)[threadIdx.x] = 0;
  const int b = request_of(p, t);
  if (b < 0) return;
  const Kv4Request r = kv4_request(p, b);
  const int rows = r.n * p.group;
  if (!kTopk && (rows < p.min_rows || rows > p.max_rows)) return;
  const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5;
  const In* q = static_cast<const In*>(p.q) + t * p.q_stride + static_cast<long long>(h) * D;
  for (int d = tid; d < D; d += kGenWarps * 32) s_q[d] = to_float(q[d]) * p.scale;
  __syncthreads();
  const long long last = static_cast<long long>(r.ctx) + (t - r.first);  // the token's own position
  const long long reach = static_cast<long long>(p.max_pages) * kPageKeys;
  const long long n = kTopk ? p.topk : (last + 1 < reach ? last + 1 : reach);
  const int32_t* table = p.page_table + static_cast<long long>(b) * p.max_pages;
  float m = -INFINITY, l = 0.f, o[kPer];
#pragma unroll
  for (int i = 0; i < kPer; ++i) o[i] = 0.f;
  for (long long base = static_cast<long long>(warp) * 32; base < n; base += kGenWarps * 32) {
    long long pos = base + lane;
    bool sees = pos < n;
    if (kTopk) {
      pos = sees ? p.idx[static_cast<long long>(t) * p.topk + pos] : -1;
      sees = pos >= 0 && pos <= last && pos < reach;
    }
    const long long page = sees ? table[pos / kPageKeys] : -1;
    sees = page >= 0 && page < p.pool_pages;
    const uint8_t* row = p.pool + (sees ? ((page * p.Hkv + kvh) * kPageKeys + pos % kPageKeys) * kRow : 0);
    float s = -INFINITY;
    if (sees) {
      s = 0.f;
#pragma unroll
      for (int g = 0; g < kGroups; ++g) {
        float part = 0.f;
#pragma unroll
        for (int w = 0; w < 4; ++w) {
          const uint32_t c = *reinterpret_cast<const uint32_t*>(row + g * 16 + w * 4);
#pragma unroll
          for (int i = 0; i < 8; ++i)
            part = __fmaf_rn(s_q[g * 32 + w * 8 + i], static_cast<float>(static_cast<int>((c >> (4 * i)) & 15u) - 8), part);
        }
        s = __fmaf_rn(part, __half2float(*reinterpret_cast<const __half*>(row + D + g * 2)), s);
      }
    }
    float top = s;
#pragma unroll
    for (int d = 16; d > 0; d >>= 1) top = fmaxf(top, __shfl_xor_sync(0xffffffffu, top, d));
    if (top == -INFINITY) continue;  // (uniform: nothing to see here)
    const float m_new = fmaxf(m, top), back = expf(m - m_new), e = expf(s - m_new);
    m = m_new;
    l = l * back + e;
#pragma unroll
    for (int i = 0; i < kPer; ++i) o[i] *= back;
    const long long off = row - p.pool;
    for (unsigned live = __ballot_sync(0xffffffffu, sees); live != 0; live &= live - 1) {
      const int j = __ffs(live) - 1;
      const float ej = __shfl_sync(0xffffffffu, e, j);
      const uint8_t* rj = p.pool + __shfl_sync(0xffffffffu, off, j);
      const float es = ej * __half2float(*reinterpret_cast<const __half*>(rj + D + 2 * (kGroups + lane * kPer / kKvGroup)));
      uint32_t c;
      if constexpr (kPer == 4)
        c = *reinterpret_cast<const uint16_t*>(rj + D / 2 + lane * 2);
      else
        c = rj[D / 2 + lane];
#pragma unroll
      for (int i = 0; i < kPer; ++i) o[i] = __fmaf_rn(es, static_cast<float>(static_cast<int>((c >> (4 * i)) & 15u) - 8), o[i]);
    }
  }
#pragma unroll
  for (int d = 16; d > 0; d >>= 1) l += __shfl_xor_sync(0xffffffffu, l, d);
#pragma unroll
  for (int i = 0; i < kPer; ++i) s_o[warp][lane * kPer + i] = o[i];
  if (lane == 0) {
    s_m[warp] = m;
    s_l[warp] = l;
  }
  __syncthreads();
  float top = -INFINITY, sum = 0.f;
#pragma unroll
  for (int w = 0; w < kGenWarps; ++w) top = fmaxf(top, s_m[w]);
  if (top > -INFINITY) {
#pragma unroll
    for (int w = 0; w < kGenWarps; ++w) sum += s_l[w] * expf(s_m[w] - top);
  }
  In* out = static_cast<In*>(p.out) + (static_cast<long long>(t) * p.Hq + h) * D;
  for (int d = tid; d < D; d += kGenWarps * 32) {
    float x = 0.f;
    if (sum > 0.f) {
#pragma unroll
      for (int w = 0; w < kGenWarps; ++w) x += s_o[w][d] * expf(s_m[w] - top);
      x /= sum;
    }
    store_out(out + d, x);
  }
  if (tid == 0 && p.lse != nullptr) p.lse[static_cast<long long>(t) * p.Hq + h] = sum > 0.f ? top + logf(sum) : -INFINITY;
}

}  // namespace

cudaError_t launch_kv4_attention_generic(int dtype, int D, const Kv4AttnParams& p, cudaStream_t stream) {
  const dim3 grid(p.T, p.Hq);
  auto go = [&](auto kernel) { return launch_chained(kernel, grid, dim3(kGenWarps * 32), 0, stream, 1, p); };
  if (dtype == LT_DTYPE_F32) {
    if (p.idx != nullptr) return D == 64 ? go(attention_generic_kernel<float, 64, true>) : go(attention_generic_kernel<float, 128, true>);
    return D == 64 ? go(attention_generic_kernel<float, 64, false>) : go(attention_generic_kernel<float, 128, false>);
  }
  if (p.idx != nullptr)
    return D == 64 ? go(attention_generic_kernel<__nv_bfloat16, 64, true>) : go(attention_generic_kernel<__nv_bfloat16, 128, true>);
  return D == 64 ? go(attention_generic_kernel<__nv_bfloat16, 64, false>) : go(attention_generic_kernel<__nv_bfloat16, 128, false>);
}

}  // namespace lt
