// What the tensor-core attention kernels over the 4-bit cache share: arithmetic on codes, the running softmax, results and parts.
#pragma once

#include <type_traits>

#include "lt_kv4.cuh"

namespace lt {
namespace {

constexpr float kLog2e = 1.4426950408889634f, kLn2 = 0.6931471805599453f;
// Probabilities are held times 2^11, relative to a maximum that is only raised when a score has passed it by 4 powers of two (raising
// it multiplies all sums, and for 8 heads some score passes the exact maximum in every third unit): at most 2^15, and no less
// than 2^-35 of the largest in fp16.
constexpr float kPShift = 11.f, kPSlack = 4.f;
constexpr float kNothing = 2e38f;  // shift of a row that has seen nothing: beyond all others, which are under 2^126
// What a row's scores are worth in powers of two (query scaling, scale, log2 e), within bounds that keep products with the scores finite
// and masked ones at -inf.  At the lower bound all scores are under 2^-60, which no weight shows.
constexpr float kLeastWorth = 0x1p-100f;
// That worth for a row whose queries were multiplied by 2^(142 - e): 2^(e - 142) |scale| log2(e) gain, gain a power of two from 1 to 2^24.
// The first product can leave fp32's range: where it falls below, the result is under kLeastWorth (a scale of zero too), where it passes
// it, beyond `most`.
__device__ __forceinline__ float worth_of(int e, float scale, float gain, float most) {
  const float down = __uint_as_float(static_cast<uint32_t>(e - 15) << 23) * fabsf(scale);
  return fminf(fmaxf(down * (gain * kLog2e), kLeastWorth), most);
}
// What is added to a score top * worth for it to become kPShift, and the score up to which that stays: rounded down, so that no
// probability passes 2^15 however coarse fp32 is at that size.  (At 2^28 the largest then comes out as 2^-5 to 2^11.)
__device__ __forceinline__ float shift_of(float top, float worth) { return __fmaf_rd(-top, worth, kPShift); }
__device__ __forceinline__ float bar_of(float top, float worth) { return __fadd_rd(top, kPSlack / worth); }

// ---- arithmetic -------------------------------------------------------------------------------
__device__ __forceinline__ float ex2(float x) {
  float y;
  asm("ex2.approx.ftz.f32 %0, %1;" : "=f"(y) : "f"(x));
  return y;
}
__device__ __forceinline__ uint32_t hfma2(uint32_t a, uint32_t b, uint32_t c) {
  uint32_t d;
  asm("fma.rn.f16x2 %0, %1, %2, %3;" : "=r"(d) : "r"(a), "r"(b), "r"(c));
  return d;
}
__device__ __forceinline__ uint32_t hmul2(uint32_t a, uint32_t b) {
  uint32_t d;
  asm("mul.rn.f16x2 %0, %1, %2;" : "=r"(d) : "r"(a), "r"(b));
  return d;
}
__device__ __forceinline__ uint32_t hadd2(uint32_t a, uint32_t b) {
  uint32_t d;
  asm("add.rn.f16x2 %0, %1, %2;" : "=r"(d) : "r"(a), "r"(b));
  return d;
}
// A constant that stays in a register: instructions take one immediate, and the ones below would need two.
__device__ __forceinline__ uint32_t held(uint32_t x) {
  uint32_t r;
  asm("mov.b32 %0, %1;" : "=r"(r) : "r"(x));
  return r;
}
struct ValueConstants {
  uint32_t k1024, k16, inv16, minus72;
  __device__ __forceinline__ ValueConstants() : k1024(held(0x64006400u)), k16(held(0x4C004C00u)), inv16(held(0x2C002C00u)), minus72(held(0xD480D480u)) {}
};
__device__ __forceinline__ uint32_t and_or(uint32_t w, uint32_t mask, uint32_t c) {
  uint32_t d;
  asm("lop3.b32 %0, %1, %2, %3, 0xEA;" : "=r"(d) : "r"(w), "r"(mask), "r"(c));
  return d;
}
// Nibble i of each half of w as the fp16 pair (u - 8) s; minus24s = -24 s.  Exact for the scales that the writer leaves (lt_kv4.cuh).
template <int i>
__device__ __forceinline__ uint32_t f16_values(uint32_t w, uint32_t s, uint32_t minus24s, const ValueConstants& k) {
  if constexpr (i == 0)
    return hmul2(hadd2(and_or(w, 0x000F000Fu, k.k1024), 0xE408E408u), s);  // 1024 + u - 1032
  else if constexpr (i == 1)
    return hmul2(hfma2(and_or(w, 0x00F000F0u, k.k1024), k.inv16, k.minus72), s);  // (1024 + 16 u) / 16 - 72
  else
    return hfma2(and_or(w >> (4 * i - 6), 0x03C003C0u, k.k16), s, minus24s);  // 16 + u
}
__device__ __forceinline__ uint32_t half2_bits(float lo, float hi) {
  const __half2 h = __floats2half2_rn(lo, hi);
  return *reinterpret_cast<const uint32_t*>(&h);
}
__device__ __forceinline__ uint32_t bf162_bits(float lo, float hi) {
  const __nv_bfloat162 h = __floats2bfloat162_rn(lo, hi);
  return *reinterpret_cast<const uint32_t*>(&h);
}
// Quotient of counts that nearly always fit into 32 bits.
__device__ __forceinline__ long long quotient(long long a, long long b) {
  if (((a | b) >> 32) == 0) return static_cast<uint32_t>(a) / static_cast<uint32_t>(b);
  return a / b;
}

// Exclusive sum over the CTA's threads, and the total.
template <int kWarps>
__device__ __forceinline__ long long block_scan(long long v, long long& total, long long* warp_sums) {
  const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
  long long inc = v;
#pragma unroll
  for (int d = 1; d < 32; d <<= 1) {
    const long long x = __shfl_up_sync(0xffffffffu, inc, d);
    if (lane >= d) inc += x;
  }
  if (lane == 31) warp_sums[warp] = inc;
  __syncthreads();
  long long before = 0;
  total = 0;
#pragma unroll
  for (int w = 0; w < kWarps; ++w) {
    const long long x = warp_sums[w];
    before += w < warp ? x : 0;
    total += x;
  }
  __syncthreads();
  return before + inc - v;
}

// ---- requests, by a warp: 32 at a look ----------------------------------------------------------------
// (One request after the other, a warp waits for memory at each: 4 requests among 4096 empty slots took 820 us instead of 130.)
// The last request that begins at or before the row.
__device__ __forceinline__ int request_of_row(const Kv4AttnParams& p, int row) {
  const int lane = threadIdx.x & 31;
  int a = 0, n = p.B;
  while (n > 1) {
    const int step = (n + 31) / 32, i = lane * step;
    const unsigned le = __ballot_sync(0xffffffffu, i < n && p.query_start[a + i] <= row);
    const int hit = (31 - __clz(le | 1u)) * step;
    a += hit;
    n = n - hit < step ? n - hit : step;
  }
  return a;
}
// The same, known to be b or one behind it.
__device__ __forceinline__ int request_of_row_from(const Kv4AttnParams& p, int b, int row) {
  while (true) {
    const int i = b + 1 + (threadIdx.x & 31);
    const unsigned le = __ballot_sync(0xffffffffu, i < p.B && p.query_start[i] <= row);
    if (le != 0xffffffffu) return b + __popc(le);
    b += 32;
  }
}
// The first request from b on that `takes_part`; B if there is none.
template <typename F>
__device__ __forceinline__ int next_request(const Kv4AttnParams& p, int b, F takes_part) {
  for (; b < p.B; b += 32) {
    const int i = b + (threadIdx.x & 31);
    const unsigned some = __ballot_sync(0xffffffffu, i < p.B && takes_part(kv4_request(p, i < p.B ? i : b)));
    if (some != 0) return b + __ffs(some) - 1;
  }
  return p.B;
}

// ---- results ----------------------------------------------------------------------------------
// Row r of an item's request (dense) or token (selected): where its query and result are.
__device__ __forceinline__ void row_place(const Kv4AttnParams& p, int first, int kvh, int r, int& token, int& head) {
  const int j = r / p.group;
  token = first + j;
  head = kvh * p.group + (r - j * p.group);
}

// 4 joined elements of a row and its sum: out, and lse once per row.
template <int D>
__device__ __forceinline__ void write_row4(const Kv4AttnParams& p, int token, int head, int d, const float4& o, float m, float l) {
  const float inv = l > 0.f ? __fdividef(1.f, l) : 0.f;
  __nv_bfloat16* at = static_cast<__nv_bfloat16*>(p.out) + (static_cast<long long>(token) * p.Hq + head) * D + d;
  *reinterpret_cast<uint2*>(at) = make_uint2(bf162_bits(o.x * inv, o.y * inv), bf162_bits(o.z * inv, o.w * inv));
  if (d == 0 && p.lse != nullptr)
    p.lse[static_cast<long long>(token) * p.Hq + head] = l > 0.f ? (m - kPShift + log2f(l)) * kLn2 : -INFINITY;
}

// (o, m, l) and another part of the same row: sums relative to the larger maximum.
__device__ __forceinline__ void join(float4& o, float& m, float& l, const float4& x, float pm, float pl) {
  const float mm = fmaxf(m, pm), a = m == -INFINITY ? 0.f : ex2(m - mm), b = pm == -INFINITY ? 0.f : ex2(pm - mm);
  o = make_float4(o.x * a + x.x * b, o.y * a + x.y * b, o.z * a + x.z * b, o.w * a + x.w * b);
  l = l * a + pl * b;
  m = mm;
}

// ---- the parts of an item that several CTAs share --------------------------------------------------
// A piece of an item: which rows, and whether it holds the item's first and last unit.
struct PartDesc {
  int b, kvh, rt, flags;
};
constexpr int kValid = 1, kBegins = 2, kEnds = 4;
struct CtaDesc {
  PartDesc part[2];  // [0] an item that began before this CTA's run, [1] one that begins in it and does not end
  int status;        // LT_STATUS_* bits
  int pad[7];
};
// Scratch of a call, one kernel pair after the other.
struct SplitBuffers {
  CtaDesc* desc;  // [grid]
  float* cta;     // [grid][2] parts of kRows rows
  float* warp;    // [grid][warps] parts: the first, incomplete item of a warp that goes on to others (few-row kernel)
  Control* ctl;   // the call's status block
};
// Floats of a part: o[kRows][D], m[kRows] (powers of two), l[kRows].
__host__ __device__ constexpr int part_floats(int rows, int D) { return rows * (D + 2); }

// Items that span CTAs: the CTAs (c, *) join the one that begins in run c with the pieces of the runs behind it.  Items of few rows span
// many CTAs: there the 8 warps of a CTA share out the pieces of 32 groups of 4 elements, 4 of them under way each, and are joined in
// turn.  Items of many rows span few: there each warp has elements of its own, and a CTA several turns (a CTA for every 32 groups of
// elements took 50 us to launch: 1024 x 2048 positions 323 instead of 270 us).
constexpr int kJoinWarps = 8;
template <int D, int kRows, bool kTopk>
__global__ void __launch_bounds__(kJoinWarps * 32) attention_join_kernel(const Kv4AttnParams p, const SplitBuffers sb, int n_ctas, bool keep_status) {
  constexpr int kFloats = part_floats(kRows, D), kThreads = kJoinWarps * 32, kJoinGroups = kRows <= 16 ? kJoinWarps : 1;
  __shared__ int s_status, s_end;
  __shared__ float4 s_o[kJoinGroups][32];
  __shared__ float s_m[kJoinGroups][32], s_l[kJoinGroups][32];
  chain_wait();
  if (blockIdx.x == 0 && blockIdx.y == 0) {  // the call's status: what its CTAs left
    if (threadIdx.x == 0) s_status = keep_status ? sb.ctl->status : 0;
    __syncthreads();
    for (int c = threadIdx.x; c < n_ctas; c += kThreads)
      if (sb.desc[c].status != 0) atomicOr(&s_status, sb.desc[c].status);
    __syncthreads();
    if (threadIdx.x < sizeof(Control) / 4) reinterpret_cast<int*>(sb.ctl)[threadIdx.x] = threadIdx.x == 0 ? s_status : 0;
  }
  const PartDesc run = sb.desc[blockIdx.x].part[1];
  if (!(run.flags & kValid)) return;
  // up to the first CTA whose piece ends it (a run without units has no piece)
  if (threadIdx.x == 0) s_end = n_ctas;
  __syncthreads();
  for (int base = blockIdx.x + 1; base < n_ctas; base += kThreads) {
    const int c = base + threadIdx.x;
    if (c < n_ctas && (sb.desc[c].part[0].flags & kEnds)) atomicMin(&s_end, c);
    __syncthreads();
    const int end = s_end;
    __syncthreads();
    if (end < n_ctas) break;
  }
  const int n_more = (s_end < n_ctas ? s_end + 1 : n_ctas) - (blockIdx.x + 1);
  int first = run.b, rows = p.group;
  if constexpr (!kTopk) {
    const Kv4Request r = kv4_request(p, run.b);
    first = r.first;
    rows = r.n * p.group;
  }
  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31, group = kJoinGroups > 1 ? warp : 0;
  constexpr int kPerCta = kJoinGroups > 1 ? 32 : kThreads;
  for (int v = blockIdx.y * kPerCta + threadIdx.x % kPerCta; v < kRows * D / 4; v += gridDim.y * kPerCta) {
    const int n = v * 4 / D, d = v * 4 % D, r = run.rt * kRows + n;
    float4 o = make_float4(0.f, 0.f, 0.f, 0.f);
    float m = -INFINITY, l = 0.f;
    constexpr int kAhead = 4;  // pieces under way at once
    // piece 0 is CTA c's own, piece i the one of CTA c + i
    for (int i0 = group; i0 <= n_more; i0 += kAhead * kJoinGroups) {
      float4 x[kAhead];
      float pm[kAhead], pl[kAhead];
#pragma unroll
      for (int i = 0; i < kAhead; ++i) {
        const int at = i0 + i * kJoinGroups, c = blockIdx.x + at;
        x[i] = make_float4(0.f, 0.f, 0.f, 0.f);
        pm[i] = -INFINITY;
        pl[i] = 0.f;
        if (at <= n_more && r < rows && (at == 0 || (sb.desc[c].part[0].flags & kValid))) {
          const float* part = sb.cta + (static_cast<long long>(c) * 2 + (at == 0 ? 1 : 0)) * kFloats;
          x[i] = *reinterpret_cast<const float4*>(part + n * D + d);
          pm[i] = part[kRows * D + n];
          pl[i] = part[kRows * D + kRows + n];
        }
      }
#pragma unroll
      for (int i = 0; i < kAhead; ++i) join(o, m, l, x[i], pm[i], pl[i]);
    }
    if constexpr (kJoinGroups > 1) {  // (one turn only: the grid covers the item)
      s_o[group][lane] = o;
      s_m[group][lane] = m;
      s_l[group][lane] = l;
      __syncthreads();
      if (group != 0) return;
      const int groups = n_more + 1 < kJoinGroups ? n_more + 1 : kJoinGroups;
      for (int g = 1; g < groups; ++g) join(o, m, l, s_o[g][lane], s_m[g][lane], s_l[g][lane]);
    }
    if (r >= rows) continue;
    int token, head;
    row_place(p, first, run.kvh, r, token, head);
    write_row4<D>(p, token, head, d, o, m, l);
  }
}
template <int D, int kRows, bool kTopk>
inline cudaError_t launch_join(const Kv4AttnParams& p, const SplitBuffers& sb, int n_ctas, bool keep_status, cudaStream_t stream) {
  return launch_chained(attention_join_kernel<D, kRows, kTopk>, dim3(n_ctas, kRows <= 16 ? kRows * D / 128 : 8), dim3(kJoinWarps * 32), 0, stream, 1,
                        p, sb, n_ctas, keep_status);
}

}  // namespace
}  // namespace lt
