// The 4-bit key-value cache: its rows, and what the kernels that write and read them share.
//
// A page holds kPageKeys tokens.  For every (page, key-value head) the pool has 64 rows, one per token, of D + D / 8 bytes:
//   D / 2 bytes   key codes, element 2 i in the low half of byte i and 2 i + 1 in the high one
//   D / 2 bytes   value codes
//   D / 32 fp16   key scales, one per group of 32 elements
//   D / 32 fp16   value scales
// A code u stands for (u - 8) * scale, u = 1 .. 15.  Keys and values of a token lie side by side (144 bytes of one head of 128: a
// row that is picked by itself costs five 32-byte sectors), and 32 rows in a row are one run of memory.
//
// The scale is the group's largest magnitude / 7 rounded to bf16, held in fp16, at most 2048.  Its 8 significant bits keep
// 24 * scale exact in fp16, so that a value comes out of its code with one fp16x2 FMA, (16 + u) * scale - 24 * scale: 16 + u is a code
// with a constant or-ed into its exponent, no conversion.  Values are exact in fp16 too, subnormal scales included: |u - 8| <= 8 takes
// 3 more bits at most.  (A scale of more bits that something else put into the pool has its 24-fold and its values rounded.)
#pragma once

#include <cuda_bf16.h>
#include <cuda_fp16.h>
#include <cuda_runtime.h>
#include <stdint.h>

#include "lt_host.h"

namespace lt {

constexpr int kKvGroup = LT_KV4_GROUP;
constexpr float kKvMaxScale = 2048.f;

__host__ __device__ constexpr int kv4_row_bytes(int D) { return D + D / 8; }

// Scale of a group from its largest magnitude (both roundings to nearest even).
__device__ __forceinline__ __half kv4_scale(float amax) {
  // amax / 7, correctly rounded: a product with 1 / 7 and a correction by its remainder, as in Markstein's division (IBM J. Res. Dev. 34, 1990).
  // The product is up to 1.15 steps off, more than his theorem allows in general; for this divisor all 2^23 significands were gone through
  // (a power of two changes nothing): the remainder amax - 7 q is exact, and q + r / 7 rounds to the quotient every time.  (An infinite amax
  // stays as it is; quotients below the normal range become scales of zero.)
  const float seventh = 1.f / 7.f, q = amax * seventh, r = __fmaf_rn(q, -7.f, amax);
  const float s = __bfloat162float(__float2bfloat16_rn(amax < INFINITY ? __fmaf_rn(r, seventh, q) : amax));
  return __float2half_rn(fminf(s, kKvMaxScale));
}

// Code of x: the integer nearest to x / s, ties to even, within [-7, 7], plus 8.  The quotient is only guessed (inv = 1 / s, any
// rounding); the remainder x - n s, which one FMA gives exactly, decides.  NaN counts as 0.
__device__ __forceinline__ uint32_t kv4_code(float x, float s, float inv) {
  if (!(s > 0.f) || x != x) return 8u;
  float n = rintf(fminf(fmaxf(x * inv, -7.f), 7.f));
  const float r2 = 2.f * __fmaf_rn(-n, s, x);
  const bool odd = (static_cast<int>(n) & 1) != 0;
  if (r2 > s || (r2 == s && odd)) n += 1.f;
  if (r2 < -s || (r2 == -s && odd)) n -= 1.f;
  return static_cast<uint32_t>(static_cast<int>(fminf(fmaxf(n, -7.f), 7.f)) + 8);
}

}  // namespace lt

// ---------------------------------------------------------------------------------------------
// What the attention kernels are given.
// ---------------------------------------------------------------------------------------------
namespace lt {

struct Kv4AttnParams {
  const void* q;             // [T][q_stride]: Hq heads of D
  long long q_stride;        // elements from one token's row to the next
  const uint8_t* pool;
  long long pool_pages;
  const int32_t* page_table; // [B][max_pages]
  int max_pages;
  const int32_t* query_start;  // [B + 1]
  const int32_t* context_len;  // [B]
  const int32_t* idx;          // [T][topk] positions, or null: all positions up to the token's own
  int topk;
  int B, T, Hq, Hkv, group;    // group = Hq / Hkv
  float scale;
  void* out;                 // [T][Hq][D]
  float* lse;                // [T][Hq] or null
  Control* ctl;              // the call's status block
  unsigned int wait_limit_us;  // bound of every device-side wait
  int min_rows, max_rows;    // requests with min_rows .. max_rows (token, head of the group) rows are this kernel's
};

// Tokens of request b: [first, first + n), clipped to the batch; ctx clipped to the table's reach, beyond which nothing is seen (so that
// positions stay under 2^31: the reach and T are under 2^30 and 2^24).
struct Kv4Request {
  int first, n, ctx;
};
__device__ __forceinline__ Kv4Request kv4_request(const Kv4AttnParams& p, int b) {
  int a = p.query_start[b], e = p.query_start[b + 1], c = p.context_len[b];
  a = a < 0 ? 0 : (a > p.T ? p.T : a);
  e = e < a ? a : (e > p.T ? p.T : e);
  const int reach = p.max_pages * kPageKeys;
  return {a, e - a, c < 0 ? 0 : (c < reach ? c : reach)};
}
// Rows of the batch that belong to requests: [first, end).
struct Kv4Rows {
  int first, end;
};
__device__ __forceinline__ Kv4Rows kv4_rows(const Kv4AttnParams& p) {
  int a = p.query_start[0], e = p.query_start[p.B];
  a = a < 0 ? 0 : (a > p.T ? p.T : a);
  return {a, e < a ? a : (e > p.T ? p.T : e)};
}

}  // namespace lt
