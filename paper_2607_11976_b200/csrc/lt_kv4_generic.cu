// Attention over the 4-bit cache in fp32 throughout: the path of fp32 queries, and the plain reading of the method.
#include <float.h>

#include "lt_kv4.cuh"

namespace lt {
namespace {

constexpr int kGenWarps = 16;

__device__ __forceinline__ float to_float(float x) { return x; }
__device__ __forceinline__ float to_float(__nv_bfloat16 x) { return __bfloat162float(x); }
__device__ __forceinline__ void store_out(float* at, float x) { *at = x; }
__device__ __forceinline__ void store_out(__nv_bfloat16* at, float x) { *at = __float2bfloat16_rn(x); }

// The request of a token: the last b with query_start[b] <= t that has tokens at t; -1 outside of all.
__device__ __forceinline__ int request_of(const Kv4AttnParams& p, int t) {
  const Kv4Rows rows = kv4_rows(p);
  if (t < rows.first || t >= rows.end) return -1;
  int lo = 0, hi = p.B;
  while (hi - lo > 1) {
    const int mid = (lo + hi) >> 1;
    if (p.query_start[mid] <= t) lo = mid; else hi = mid;
  }
  return lo;
}

// ---------------------------------------------------------------------------------------------
// One CTA per token and kHeads query heads of one key-value head.  A warp takes 32 keys at a time: lane i scores key i for all heads (its
// codes come as wide loads and are unpacked once, the queries lie in shared memory), the running maxima and sums are the warp's, and for
// the products with the values each lane holds D / 32 elements.  The warps' results are joined at the end.  Instruction bound: 16 words of
// codes take 24 instructions each, and 8 more for every head.  fp32 queries have no tensor path, and a bf16 query takes this one only on
// request.
// ---------------------------------------------------------------------------------------------
template <int kRow>
__device__ __forceinline__ uint4 load16(const uint8_t* at) {  // (rows of 64-element heads are only 8-byte aligned)
  if constexpr (kRow % 16 == 0) return __ldg(reinterpret_cast<const uint4*>(at));
  const uint2 a = __ldg(reinterpret_cast<const uint2*>(at)), b = __ldg(reinterpret_cast<const uint2*>(at) + 1);
  return make_uint4(a.x, a.y, b.x, b.y);
}
// nibble i of w, less 8
__device__ __forceinline__ float code_value(uint32_t w, int i) { return __uint_as_float(((w >> (4 * i)) & 15u) | 0x4B000000u) - 8388616.f; }

template <typename In, int D, int kHeads, bool kTopk>
__global__ void __launch_bounds__(kGenWarps * 32) attention_generic_kernel(const Kv4AttnParams p) {
  chain_wait();
  constexpr int kRow = kv4_row_bytes(D), kGroups = D / kKvGroup, kPer = D / 32;
  __shared__ __align__(16) float s_q[kHeads][D];
  __shared__ float s_o[kGenWarps][kHeads][D];
  __shared__ float s_m[kGenWarps][kHeads], s_l[kGenWarps][kHeads];
  const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5;
  const int blocks = (p.group + kHeads - 1) / kHeads;  // of a key-value head
  const int t = blockIdx.x, kvh = blockIdx.y / blocks, h0 = (blockIdx.y - kvh * blocks) * kHeads, n_heads = min(kHeads, p.group - h0);
  if (t == 0 && blockIdx.y == 0 && tid < static_cast<int>(sizeof(Control) / 4)) reinterpret_cast<int*>(p.ctl)[tid] = 0;
  const int b = request_of(p, t);
  if (b < 0) return;
  const Kv4Request r = kv4_request(p, b);
  const In* q = static_cast<const In*>(p.q) + t * p.q_stride + (static_cast<long long>(kvh) * p.group + h0) * D;
  for (int i = tid; i < kHeads * D; i += kGenWarps * 32) {
    const float x = i / D < n_heads ? to_float(q[i]) * p.scale : 0.f;
    s_q[i / D][i % D] = isinf(x) ? copysignf(FLT_MAX, x) : x;  // (so that a key element of zero leaves zero)
  }
  __syncthreads();
  const long long last = static_cast<long long>(r.ctx) + (t - r.first);  // the token's own position
  const long long reach = static_cast<long long>(p.max_pages) * kPageKeys;
  const long long n = kTopk ? p.topk : (last + 1 < reach ? last + 1 : reach);
  const int32_t* table = p.page_table + static_cast<long long>(b) * p.max_pages;
  float m[kHeads], l[kHeads], o[kHeads][kPer];
#pragma unroll
  for (int h = 0; h < kHeads; ++h) {
    m[h] = -INFINITY;
    l[h] = 0.f;
#pragma unroll
    for (int i = 0; i < kPer; ++i) o[h][i] = 0.f;
  }
  for (long long base = static_cast<long long>(warp) * 32; base < n; base += kGenWarps * 32) {
    long long pos = base + lane;
    bool sees = pos < n;
    if (kTopk) {
      pos = sees ? p.idx[static_cast<long long>(t) * p.topk + pos] : -1;
      sees = pos >= 0 && pos <= last && pos < reach;
    }
    const long long page = sees ? table[pos / kPageKeys] : -1;
    sees = page >= 0 && page < p.pool_pages;
    const unsigned seen = __ballot_sync(0xffffffffu, sees);
    if (seen == 0) continue;
    const uint8_t* row = p.pool + (sees ? ((page * p.Hkv + kvh) * kPageKeys + pos % kPageKeys) * kRow : 0);
    float s[kHeads];
#pragma unroll
    for (int h = 0; h < kHeads; ++h) s[h] = 0.f;
    uint4 codes[kGroups];
    __half scale[kGroups];
#pragma unroll
    for (int g = 0; g < kGroups; ++g) {
      codes[g] = load16<kRow>(row + g * 16);
      scale[g] = *reinterpret_cast<const __half*>(row + D + g * 2);
    }
#pragma unroll
    for (int g = 0; g < kGroups; ++g) {
      const uint32_t w[4] = {codes[g].x, codes[g].y, codes[g].z, codes[g].w};
      float part[kHeads];
#pragma unroll
      for (int h = 0; h < kHeads; ++h) part[h] = 0.f;
#pragma unroll
      for (int j = 0; j < 4; ++j) {
        float c[8];
#pragma unroll
        for (int i = 0; i < 8; ++i) c[i] = code_value(w[j], i);
#pragma unroll
        for (int h = 0; h < kHeads; ++h) {
          const float4 a = *reinterpret_cast<const float4*>(&s_q[h][g * 32 + j * 8]), e = *reinterpret_cast<const float4*>(&s_q[h][g * 32 + j * 8 + 4]);
          part[h] = __fmaf_rn(a.x, c[0], part[h]);
          part[h] = __fmaf_rn(a.y, c[1], part[h]);
          part[h] = __fmaf_rn(a.z, c[2], part[h]);
          part[h] = __fmaf_rn(a.w, c[3], part[h]);
          part[h] = __fmaf_rn(e.x, c[4], part[h]);
          part[h] = __fmaf_rn(e.y, c[5], part[h]);
          part[h] = __fmaf_rn(e.z, c[6], part[h]);
          part[h] = __fmaf_rn(e.w, c[7], part[h]);
        }
      }
#pragma unroll
      for (int h = 0; h < kHeads; ++h) s[h] = __fmaf_rn(part[h], __half2float(scale[g]), s[h]);
    }
    float e[kHeads];
#pragma unroll
    for (int h = 0; h < kHeads; ++h) {
      if (!sees) s[h] = -INFINITY;
      float top = s[h];
#pragma unroll
      for (int d = 16; d > 0; d >>= 1) top = fmaxf(top, __shfl_xor_sync(0xffffffffu, top, d));
      const float m_new = fmaxf(m[h], top), back = expf(m[h] - m_new);
      e[h] = expf(s[h] - m_new);
      m[h] = m_new;
      l[h] = l[h] * back + e[h];
#pragma unroll
      for (int i = 0; i < kPer; ++i) o[h][i] *= back;
    }
    const long long off = row - p.pool;
#pragma unroll 8
    for (int j = 0; j < 32; ++j) {  // (no branch, so that the loads of several keys are under way)
      const uint8_t* rj = p.pool + __shfl_sync(0xffffffffu, off, j);
      const __half sj = *reinterpret_cast<const __half*>(rj + D + 2 * (kGroups + lane * kPer / kKvGroup));
      const float vs = (seen >> j) & 1u ? __half2float(sj) : 0.f;  // (a key that is not there points at some row)
      uint32_t c;
      if constexpr (kPer == 4)
        c = *reinterpret_cast<const uint16_t*>(rj + D / 2 + lane * 2);
      else
        c = rj[D / 2 + lane];
      float v[kPer];
#pragma unroll
      for (int i = 0; i < kPer; ++i) v[i] = code_value(c, i) * vs;
#pragma unroll
      for (int h = 0; h < kHeads; ++h) {
        const float ej = __shfl_sync(0xffffffffu, e[h], j);
#pragma unroll
        for (int i = 0; i < kPer; ++i) o[h][i] = __fmaf_rn(ej, v[i], o[h][i]);
      }
    }
  }
#pragma unroll
  for (int h = 0; h < kHeads; ++h) {
#pragma unroll
    for (int d = 16; d > 0; d >>= 1) l[h] += __shfl_xor_sync(0xffffffffu, l[h], d);
#pragma unroll
    for (int i = 0; i < kPer; ++i) s_o[warp][h][lane * kPer + i] = o[h][i];
    if (lane == 0) {
      s_m[warp][h] = m[h];
      s_l[warp][h] = l[h];
    }
  }
  __syncthreads();
  for (int i = tid; i < n_heads * D; i += kGenWarps * 32) {
    const int h = i / D, d = i - h * D;
    float top = -INFINITY, sum = 0.f, x = 0.f;
#pragma unroll
    for (int w = 0; w < kGenWarps; ++w) top = fmaxf(top, s_m[w][h]);
    if (top > -INFINITY) {
#pragma unroll
      for (int w = 0; w < kGenWarps; ++w) {
        const float f = expf(s_m[w][h] - top);
        sum += s_l[w][h] * f;
        x += s_o[w][h][d] * f;
      }
    }
    const long long head = static_cast<long long>(t) * p.Hq + kvh * p.group + h0 + h;
    store_out(static_cast<In*>(p.out) + head * D + d, sum > 0.f ? x / sum : 0.f);
    if (d == 0 && p.lse != nullptr) p.lse[head] = sum > 0.f ? top + logf(sum) : -INFINITY;
  }
}

template <typename In, int D, bool kTopk>
cudaError_t launch_generic(const Kv4AttnParams& p, cudaStream_t stream) {
  // 4 heads to a CTA share the unpacked codes; few tokens take 2, for twice the CTAs (16 tokens of 16 heads over 1000 to 2000 keys: 4
  // heads 36 us, 2 heads 27 us)
  auto go = [&](auto kernel, int heads) {
    return launch_chained(kernel, dim3(p.T, p.Hkv * ((p.group + heads - 1) / heads)), dim3(kGenWarps * 32), 0, stream, 1, p);
  };
  if (static_cast<long long>(p.T) * p.Hkv * ((p.group + 3) / 4) >= 2ll * sm_count()) return go(attention_generic_kernel<In, D, 4, kTopk>, 4);
  return go(attention_generic_kernel<In, D, 2, kTopk>, 2);
}

}  // namespace

cudaError_t launch_kv4_attention_generic(int dtype, int D, const Kv4AttnParams& p, cudaStream_t stream) {
  if (dtype == LT_DTYPE_F32) {
    if (p.idx != nullptr) return D == 64 ? launch_generic<float, 64, true>(p, stream) : launch_generic<float, 128, true>(p, stream);
    return D == 64 ? launch_generic<float, 64, false>(p, stream) : launch_generic<float, 128, false>(p, stream);
  }
  if (p.idx != nullptr) return D == 64 ? launch_generic<__nv_bfloat16, 64, true>(p, stream) : launch_generic<__nv_bfloat16, 128, true>(p, stream);
  return D == 64 ? launch_generic<__nv_bfloat16, 64, false>(p, stream) : launch_generic<__nv_bfloat16, 128, false>(p, stream);
}

}  // namespace lt
