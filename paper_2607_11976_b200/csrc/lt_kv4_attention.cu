// Attention of few rows per key-value head (decoding, drafted tokens, the indexer's selections) over the 4-bit cache.
//
// For a tile of rows n (query heads of one key-value head, and tokens) and the keys s that they see:
//     y[n][s] = scale log2(e) q[n] . k[s],   p = 2^(y - m),   o[n] = sum_s p v[s] / sum_s p
// in one pass with the running maximum m.  The cache is read once and is what bounds this (144 bytes per key and head of 128);
// everything else has to fit beside it: at 6.5 TB/s an SM gets a key and head every 6 clocks, in which it has to unpack 256 codes.
//
// So the codes never leave the registers.  Both products are computed transposed, keys (then value elements) as the 16 rows of an
// m16n8k16 product and the query rows as its 8 columns: a group of 8 heads wastes nothing, and the cached operand, which is the one
// that has to be unpacked, lies in the lanes as it comes out of memory.  (The tensor memory's route would write the unpacked tile
// to shared memory and read it back, 8 clocks per key and head.)
//   S^T = K Q^T: lane (g, t) holds keys g and g + 8, of each group of 32 elements the 8 of code word t.  Codes become the bf16 numbers
//     16 + u by or-ing an exponent; the accumulators start at -24 sum q, so that they end at sum q (u - 8), exact products in fp32,
//     and the scale of (key, group) multiplies that in fp32.
//   P^T: the accumulators, in fp16, turned by movmatrix.  p is held times 2^15, so that fp16 reaches down to 2^-39 of the largest.
//   O^T = V^T P^T: lane (g, t) holds elements 16 g .. 16 g + 15 of keys 2 t, 2 t + 1, 2 t + 8, 2 t + 9: one scale group, words that pair up
//     by two byte permutations; (16 + u) s - 24 s is one FMA on fp16 pairs.
//
// Work is dealt out in units of 32 keys: all units of all (request, key-value head, row tile) items in a row are cut into equal
// runs, one per warp, whatever the lengths.  A warp has its own ring of cp.async stages and waits for nobody.  Items that it
// sees whole it writes out itself; the parts of others are joined first within the CTA, then, where an item spans CTAs, by a
// second kernel.  Runs are a matter of the lengths alone, so results do not vary.
#include <type_traits>

#include "lt_kv4.cuh"

namespace lt {
namespace {

constexpr int kUnit = 32;          // keys of a unit
constexpr float kLog2e = 1.4426950408889634f, kLn2 = 0.6931471805599453f;
constexpr float kPShift = 15.f;    // probabilities are held times 2^15

template <int D, int NT>
struct Shape {
  static constexpr int kRow = kv4_row_bytes(D);
  static constexpr int kGroups = D / kKvGroup;
  static constexpr int kRows = 8 * NT;       // query rows of an item
  static constexpr int kTilesD = D / 16;     // 16-row tiles of O^T
  static constexpr int kWarps = NT == 1 ? 16 : 12;
  static constexpr int kThreads = kWarps * 32;
  static constexpr int kStages = 3;
  static constexpr int kUnitBytes = kUnit * kRow;
  static constexpr int kPartFloats = kRows * (D + 2);  // a part: o[kRows][D], m[kRows], l[kRows]
  static constexpr int kRingBytes = kStages * kUnitBytes;
  static constexpr int kPartInRing = kPartFloats * 4 <= kRingBytes;
  static constexpr size_t kSmem = static_cast<size_t>(kWarps) * kRingBytes;
  static_assert(kPartInRing, "a warp leaves its last part in its ring");
};

// A piece of an item: which rows, and whether it holds the item's first and last unit.
struct PartDesc {
  int b, kvh, rt, flags;
};
constexpr int kValid = 1, kBegins = 2, kEnds = 4;
struct CtaDesc {
  PartDesc part[2];  // [0] an item that began before this CTA's run, [1] one that begins in it and does not end
};

// ---- PTX ------------------------------------------------------------------------------------
__device__ __forceinline__ float ex2(float x) {
  float y;
  asm("ex2.approx.ftz.f32 %0, %1;" : "=f"(y) : "f"(x));
  return y;
}
__device__ __forceinline__ void mma_bf16(float (&c)[4], uint32_t a0, uint32_t a1, uint32_t a2, uint32_t a3, uint32_t b0, uint32_t b1) {
  asm("mma.sync.aligned.m16n8k16.row.col.f32.bf16.bf16.f32 {%0, %1, %2, %3}, {%4, %5, %6, %7}, {%8, %9}, {%0, %1, %2, %3};"
      : "+f"(c[0]), "+f"(c[1]), "+f"(c[2]), "+f"(c[3])
      : "r"(a0), "r"(a1), "r"(a2), "r"(a3), "r"(b0), "r"(b1));
}
__device__ __forceinline__ void mma_f16(float (&c)[4], uint32_t a0, uint32_t a1, uint32_t a2, uint32_t a3, uint32_t b0, uint32_t b1) {
  asm("mma.sync.aligned.m16n8k16.row.col.f32.f16.f16.f32 {%0, %1, %2, %3}, {%4, %5, %6, %7}, {%8, %9}, {%0, %1, %2, %3};"
      : "+f"(c[0]), "+f"(c[1]), "+f"(c[2]), "+f"(c[3])
      : "r"(a0), "r"(a1), "r"(a2), "r"(a3), "r"(b0), "r"(b1));
}
__device__ __forceinline__ uint32_t transposed(uint32_t a) {
  uint32_t d;
  asm volatile("movmatrix.sync.aligned.m8n8.trans.b16 %0, %1;" : "=r"(d) : "r"(a));
  return d;
}
template <int kBytes>
__device__ __forceinline__ void cp_async(uint32_t dst, const void* src) {
  if constexpr (kBytes == 16)
    asm volatile("cp.async.cg.shared.global [%0], [%1], 16;" ::"r"(dst), "l"(src) : "memory");
  else
    asm volatile("cp.async.ca.shared.global [%0], [%1], %2;" ::"r"(dst), "l"(src), "n"(kBytes) : "memory");
}
__device__ __forceinline__ void cp_commit() { asm volatile("cp.async.commit_group;" ::: "memory"); }
template <int kPending>
__device__ __forceinline__ void cp_wait() {
  asm volatile("cp.async.wait_group %0;" ::"n"(kPending) : "memory");
}

// Nibble i of each half of w as the bf16 pair 16 + u / as the fp16 pair 16 + u.
template <int i>
__device__ __forceinline__ uint32_t bf16_codes(uint32_t w) {
  const uint32_t x = i == 0 ? w << 3 : w >> (4 * i - 3);
  return (x & 0x00780078u) | 0x41804180u;
}
template <int i>
__device__ __forceinline__ uint32_t f16_codes(uint32_t w) {
  const uint32_t x = i < 2 ? w << (6 - 4 * i) : w >> (4 * i - 6);
  return (x & 0x03C003C0u) | 0x4C004C00u;
}
__device__ __forceinline__ uint32_t hfma2(uint32_t a, uint32_t b, uint32_t c) {
  uint32_t d;
  asm("fma.rn.f16x2 %0, %1, %2, %3;" : "=r"(d) : "r"(a), "r"(b), "r"(c));
  return d;
}
__device__ __forceinline__ uint32_t half2_bits(float lo, float hi) {
  const __half2 h = __floats2half2_rn(lo, hi);
  return *reinterpret_cast<const uint32_t*>(&h);
}
__device__ __forceinline__ uint32_t bf162_bits(float lo, float hi) {
  const __nv_bfloat162 h = __floats2bfloat162_rn(lo, hi);
  return *reinterpret_cast<const uint32_t*>(&h);
}

// ---- items ----------------------------------------------------------------------------------
template <int D, int NT>
struct RequestWork {
  Kv4Request r;
  int units, tiles;  // units of 32 keys, row tiles; 0 units: nothing to do
  __device__ __forceinline__ long long load(const Kv4AttnParams& p, int b) {
    r = kv4_request(p, b);
    const long long rows = static_cast<long long>(r.n) * p.group;
    units = tiles = 0;
    if (rows < p.min_rows || rows > p.max_rows) return 0;
    const long long keys = static_cast<long long>(r.ctx) + r.n, reach = static_cast<long long>(p.max_pages) * kPageKeys;
    units = static_cast<int>(((keys < reach ? keys : reach) + kUnit - 1) / kUnit);
    tiles = static_cast<int>((rows + Shape<D, NT>::kRows - 1) / Shape<D, NT>::kRows);
    return static_cast<long long>(units) * tiles * p.Hkv;
  }
};

// Where a warp stands in the row of all units.  Dense form: b is the request; selected form: b is the token.
template <int D, int NT, bool kTopk>
struct Cursor {
  RequestWork<D, NT> w;
  int b, kvh, rt, unit;
  __device__ __forceinline__ void start(const Kv4AttnParams& p, int b_, long long off) {
    b = b_;
    if constexpr (kTopk) {
      w.units = (p.topk + kUnit - 1) / kUnit;
      w.tiles = (p.group + Shape<D, NT>::kRows - 1) / Shape<D, NT>::kRows;
    } else {
      w.load(p, b);
    }
    const long long item = off / w.units;
    unit = static_cast<int>(off - item * w.units);
    kvh = static_cast<int>(item / w.tiles);
    rt = static_cast<int>(item - static_cast<long long>(kvh) * w.tiles);
  }
  // To the next item (there has to be one).
  __device__ __forceinline__ void next_item(const Kv4AttnParams& p) {
    unit = 0;
    if (++rt < w.tiles) return;
    rt = 0;
    if (++kvh < p.Hkv) return;
    kvh = 0;
    ++b;
    if constexpr (!kTopk)
      while (b < p.B && w.load(p, b) == 0) ++b;
  }
  __device__ __forceinline__ void next(const Kv4AttnParams& p, bool more) {
    if (++unit == w.units && more) next_item(p);
  }
};

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

struct SplitBuffers {
  CtaDesc* desc;   // [grid]
  float* cta;      // [grid][2][kPartFloats]
  float* warp;     // [grid * kWarps][kPartFloats]: the first, incomplete item of a warp that goes on to others
};

// ---------------------------------------------------------------------------------------------
template <int D, int NT, bool kTopk>
__global__ void __launch_bounds__(Shape<D, NT>::kThreads, 1) attention_rows_kernel(const Kv4AttnParams p, const SplitBuffers sb) {
  using S = Shape<D, NT>;
  extern __shared__ __align__(128) uint8_t smem[];
  __shared__ long long s_first[S::kThreads], s_sums[S::kWarps];
  __shared__ PartDesc s_part[S::kWarps][2];
  __shared__ unsigned s_seen[S::kWarps][S::kStages];
  const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5, g = lane >> 2, t = lane & 3;
  chain_wait();

  // ---- this warp's run [lo, hi) of all units, and where it begins --------------------------------
  const long long gw = static_cast<long long>(blockIdx.x) * S::kWarps + warp, n_warps = static_cast<long long>(gridDim.x) * S::kWarps;
  long long total = 0, lo, hi;
  Cursor<D, NT, kTopk> at;
  if constexpr (kTopk) {
    int end = p.query_start[p.B];
    end = end < 0 ? 0 : (end > p.T ? p.T : end);
    const int units = (p.topk + kUnit - 1) / kUnit, tiles = (p.group + S::kRows - 1) / S::kRows;
    const long long per = static_cast<long long>(units) * tiles * p.Hkv;
    total = per * end;
    lo = total * gw / n_warps;
    hi = total * (gw + 1) / n_warps;
    if (lo < hi) at.start(p, static_cast<int>(lo / per), lo % per);
  } else {
    RequestWork<D, NT> w;
    if (p.B > S::kThreads) {  // the total needs a pass of its own
      long long sum = 0;
      for (int b = tid; b < p.B; b += S::kThreads) sum += w.load(p, b);
      block_scan<S::kWarps>(sum, total, s_sums);
    }
    long long before = 0;
    lo = hi = 0;
    for (int base = 0; base < p.B; base += S::kThreads) {
      const long long mine = base + tid < p.B ? w.load(p, base + tid) : 0;
      long long sum;
      s_first[tid] = before + block_scan<S::kWarps>(mine, sum, s_sums);
      __syncthreads();
      if (p.B <= S::kThreads) total = sum;
      lo = total * gw / n_warps;
      hi = total * (gw + 1) / n_warps;
      if (lo < hi && lo >= before && lo < before + sum) {
        int a = 0, e = S::kThreads;  // the last request that begins at or before lo is one with units
        while (e - a > 1) {
          const int mid = (a + e) >> 1;
          if (s_first[mid] <= lo) a = mid; else e = mid;
        }
        at.start(p, base + a, lo - s_first[a]);
      }
      before += sum;
      __syncthreads();
    }
  }

  // ---- fetching -------------------------------------------------------------------------------
  uint8_t* ring = smem + static_cast<size_t>(warp) * S::kRingBytes;
  const uint32_t ring_addr = static_cast<uint32_t>(__cvta_generic_to_shared(ring));
  const long long page_bytes = static_cast<long long>(p.Hkv) * kPageKeys * S::kRow;
  Cursor<D, NT, kTopk> ahead = at;
  long long fetched = lo;
  int fetch_stage = 0;
  // dense: the request's pages, 32 at a time
  int pages = -1, pages_at = -1;
  // selected: the indices of the unit after the next one, the page numbers of the next one
  Cursor<D, NT, kTopk> idx_at = at;   // unit whose indices are loaded next
  long long idx_loaded = lo;
  int idx_far = -1;                   // loaded indices of the unit behind `slot_next`'s
  int near_pos = -1, near_page = -1;  // the next unit to fetch: position and page of this lane's key
  int req_b = 0, req_token = -1;
  Kv4Request req{0, 0, 0};

  auto load_indices = [&]() {
    idx_far = -1;
    if (idx_loaded < hi) {
      const int i = idx_at.unit * kUnit + lane;
      if (i < p.topk) idx_far = p.idx[static_cast<long long>(idx_at.b) * p.topk + i];
      ++idx_loaded;
      idx_at.next(p, true);
    }
  };
  // page numbers for the indices of `token`'s unit
  auto load_pages = [&](int token, bool any) {
    near_pos = near_page = -1;
    if (!any) return;
    if (token != req_token) {
      // 32 requests at a look: the last one that begins at or before the token
      if (req_token < 0) {
        int a = 0, n = p.B;
        while (n > 1) {
          const int step = (n + 31) / 32, i = lane * step;
          const unsigned le = __ballot_sync(0xffffffffu, i < n && p.query_start[a + i] <= token);
          const int hit = (31 - __clz(le | 1u)) * step;
          a += hit;
          n = n - hit < step ? n - hit : step;
        }
        req_b = a;
      } else {
        while (req_b + 1 < p.B && p.query_start[req_b + 1] <= token) ++req_b;
      }
      req = kv4_request(p, req_b);
      req_token = token;
    }
    const int pos = idx_far;
    const long long last = static_cast<long long>(req.ctx) + (token - req.first);
    if (pos >= 0 && pos <= last && pos / kPageKeys < p.max_pages) {
      near_pos = pos;
      near_page = p.page_table[static_cast<long long>(req_b) * p.max_pages + pos / kPageKeys];
    }
  };
  Cursor<D, NT, kTopk> page_at = at;  // unit whose page numbers are loaded next
  long long pages_loaded = lo;
  auto step_pages = [&]() {
    load_pages(page_at.b, pages_loaded < hi);
    if (pages_loaded < hi) {
      ++pages_loaded;
      page_at.next(p, true);
    }
  };
  if constexpr (kTopk) {
    load_indices();
    step_pages();
    load_indices();
  }

  auto fetch = [&]() {
    if (fetched < hi) {
      const uint32_t dst = ring_addr + fetch_stage * S::kUnitBytes;
      if constexpr (kTopk) {
        const bool sees = near_page >= 0 && near_page < p.pool_pages;
        const unsigned seen = __ballot_sync(0xffffffffu, sees);
        if (lane == 0) s_seen[warp][fetch_stage] = seen;
        const int slot = sees ? near_page * kPageKeys + near_pos % kPageKeys : -1;
        const uint8_t* head = p.pool + static_cast<long long>(ahead.kvh) * kPageKeys * S::kRow;
        constexpr int kPiece = S::kRow % 16 == 0 ? 16 : 8, kPieces = S::kRow / kPiece;
#pragma unroll
        for (int i = 0; i < kPieces; ++i) {
          const int n = i * 32 + lane, key = n / kPieces, part = n - key * kPieces;
          const int s = __shfl_sync(0xffffffffu, slot, key);
          if (s >= 0)
            cp_async<kPiece>(dst + key * S::kRow + part * kPiece,
                             head + static_cast<long long>(s / kPageKeys) * page_bytes + (s % kPageKeys) * S::kRow + part * kPiece);
        }
        step_pages();
        load_indices();
      } else {
        const int page_no = ahead.unit / 2;
        if (ahead.unit == 0 || pages_at < 0 || page_no - pages_at >= 32) {
          pages_at = page_no;
          pages = page_no + lane < p.max_pages ? p.page_table[static_cast<long long>(ahead.b) * p.max_pages + page_no + lane] : -1;
        }
        const int page = __shfl_sync(0xffffffffu, pages, page_no - pages_at);
        const bool sees = page >= 0 && page < p.pool_pages;
        if (lane == 0) s_seen[warp][fetch_stage] = sees ? 0xffffffffu : 0u;
        if (sees) {
          const uint8_t* src = p.pool + page * page_bytes + (static_cast<long long>(ahead.kvh) * kPageKeys + (ahead.unit & 1) * kUnit) * S::kRow;
#pragma unroll
          for (int i = 0; i < (S::kUnitBytes / 16 + 31) / 32; ++i) {
            const int n = i * 32 + lane;
            if (S::kUnitBytes / 16 % 32 == 0 || n < S::kUnitBytes / 16) cp_async<16>(dst + n * 16, src + n * 16);
          }
        }
      }
      ++fetched;
      if (fetched < hi) ahead.next(p, true);
      fetch_stage = fetch_stage + 1 == S::kStages ? 0 : fetch_stage + 1;
    }
    cp_commit();
  };
#pragma unroll
  for (int i = 0; i < S::kStages - 1; ++i) fetch();

  // ---- the run ----------------------------------------------------------------------------------
  if (lane < 2) s_part[warp][lane] = PartDesc{0, 0, 0, 0};
  int stage = 0;
  for (long long u = lo; u < hi;) {
    // an item, or the part of it that is in the run
    const long long left = hi - u;
    const int unit0 = at.unit, unit1 = at.w.units - unit0 <= left ? at.w.units : static_cast<int>(unit0 + left);
    const int first = kTopk ? at.b : at.w.r.first;
    const int rows = kTopk ? p.group : at.w.r.n * p.group;
    const int row0 = at.rt * S::kRows;
    // queries as the column operand, and -24 sum q of each group of 32
    uint32_t bq[NT][S::kGroups][2][2];
    float off[NT][S::kGroups][2];
#pragma unroll
    for (int nt = 0; nt < NT; ++nt) {
      const int r = row0 + nt * 8 + g;
      uint4 x[S::kGroups];
#pragma unroll
      for (int gi = 0; gi < S::kGroups; ++gi) x[gi] = make_uint4(0, 0, 0, 0);
      if (r < rows) {
        int token, head;
        row_place(p, first, at.kvh, r, token, head);
        const uint4* src = reinterpret_cast<const uint4*>(static_cast<const __nv_bfloat16*>(p.q) + token * p.q_stride + static_cast<long long>(head) * D);
#pragma unroll
        for (int gi = 0; gi < S::kGroups; ++gi) x[gi] = __ldg(src + gi * 4 + t);
      }
#pragma unroll
      for (int gi = 0; gi < S::kGroups; ++gi) {
        // elements i and i + 4 of the word side by side, as the codes come
        bq[nt][gi][0][0] = __byte_perm(x[gi].x, x[gi].z, 0x5410);
        bq[nt][gi][0][1] = __byte_perm(x[gi].x, x[gi].z, 0x7632);
        bq[nt][gi][1][0] = __byte_perm(x[gi].y, x[gi].w, 0x5410);
        bq[nt][gi][1][1] = __byte_perm(x[gi].y, x[gi].w, 0x7632);
        const uint32_t w[4] = {x[gi].x, x[gi].y, x[gi].z, x[gi].w};
        float sum = 0.f;
#pragma unroll
        for (int i = 0; i < 4; ++i) sum += __uint_as_float(w[i] << 16) + __uint_as_float(w[i] & 0xffff0000u);
        sum += __shfl_xor_sync(0xffffffffu, sum, 1);
        sum += __shfl_xor_sync(0xffffffffu, sum, 2);
        off[nt][gi][0] = -24.f * __shfl_sync(0xffffffffu, sum, 8 * t);
        off[nt][gi][1] = -24.f * __shfl_sync(0xffffffffu, sum, 8 * t + 4);
      }
    }
    // how far each column sees (dense form)
    int limit[NT][2], least = 0x7fffffff, most = -1;
    if constexpr (!kTopk) {
#pragma unroll
      for (int nt = 0; nt < NT; ++nt)
#pragma unroll
        for (int c = 0; c < 2; ++c) {
          const int r = row0 + nt * 8 + 2 * t + c;
          limit[nt][c] = at.w.r.ctx + (r < rows ? r : rows - 1) / p.group;
        }
      least = at.w.r.ctx + row0 / p.group;
      most = at.w.r.ctx + ((row0 + S::kRows < rows ? row0 + S::kRows : rows) - 1) / p.group;
    }
    float o[S::kTilesD][NT][4], m[NT][2], l[NT][2];
#pragma unroll
    for (int nt = 0; nt < NT; ++nt) {
      m[nt][0] = m[nt][1] = -INFINITY;
      l[nt][0] = l[nt][1] = 0.f;
#pragma unroll
      for (int j = 0; j < S::kTilesD; ++j)
#pragma unroll
        for (int c = 0; c < 4; ++c) o[j][nt][c] = 0.f;
    }
    const float to_log2 = p.scale * kLog2e;

    for (int unit = unit0; unit < unit1; ++unit, ++u) {
      cp_wait<S::kStages - 2>();
      __syncwarp();  // this unit has come, for all lanes, and all are through with the one before, whose stage is filled again
      fetch();
      const uint8_t* st = ring + stage * S::kUnitBytes;
      const unsigned seen = s_seen[warp][stage];
      const bool whole = seen == 0xffffffffu && (kTopk || unit * kUnit + kUnit - 1 <= least);
      float y[2][NT][4];
#pragma unroll
      for (int blk = 0; blk < 2; ++blk) {
        const uint8_t* k0 = st + (blk * 16 + g) * S::kRow;
        const uint8_t* k1 = k0 + 8 * S::kRow;
        __half ks0[S::kGroups], ks1[S::kGroups];
#pragma unroll
        for (int gi = 0; gi < S::kGroups; gi += 2) {
          *reinterpret_cast<uint32_t*>(&ks0[gi]) = *reinterpret_cast<const uint32_t*>(k0 + D + gi * 2);
          *reinterpret_cast<uint32_t*>(&ks1[gi]) = *reinterpret_cast<const uint32_t*>(k1 + D + gi * 2);
        }
#pragma unroll
        for (int nt = 0; nt < NT; ++nt)
#pragma unroll
          for (int c = 0; c < 4; ++c) y[blk][nt][c] = 0.f;
#pragma unroll
        for (int gi = 0; gi < S::kGroups; ++gi) {
          const uint32_t w0 = *reinterpret_cast<const uint32_t*>(k0 + gi * 16 + t * 4);
          const uint32_t w1 = *reinterpret_cast<const uint32_t*>(k1 + gi * 16 + t * 4);
          const uint32_t a00 = bf16_codes<0>(w0), a01 = bf16_codes<0>(w1), a02 = bf16_codes<1>(w0), a03 = bf16_codes<1>(w1);
          const uint32_t a10 = bf16_codes<2>(w0), a11 = bf16_codes<2>(w1), a12 = bf16_codes<3>(w0), a13 = bf16_codes<3>(w1);
          const float s0 = __half2float(ks0[gi]) * to_log2, s1 = __half2float(ks1[gi]) * to_log2;
#pragma unroll
          for (int nt = 0; nt < NT; ++nt) {
            float acc[4] = {off[nt][gi][0], off[nt][gi][1], off[nt][gi][0], off[nt][gi][1]};
            mma_bf16(acc, a00, a01, a02, a03, bq[nt][gi][0][0], bq[nt][gi][0][1]);
            mma_bf16(acc, a10, a11, a12, a13, bq[nt][gi][1][0], bq[nt][gi][1][1]);
            y[blk][nt][0] = __fmaf_rn(acc[0], s0, y[blk][nt][0]);
            y[blk][nt][1] = __fmaf_rn(acc[1], s0, y[blk][nt][1]);
            y[blk][nt][2] = __fmaf_rn(acc[2], s1, y[blk][nt][2]);
            y[blk][nt][3] = __fmaf_rn(acc[3], s1, y[blk][nt][3]);
          }
        }
      }
      unsigned live = seen;  // keys that some row of the tile sees: all others' values are taken as zero, whatever lies there
      if (!whole) {
        if constexpr (!kTopk) {
          const int n = most - unit * kUnit + 1;
          live = n <= 0 ? 0u : (n >= 32 ? live : live & ((1u << n) - 1u));
        }
#pragma unroll
        for (int blk = 0; blk < 2; ++blk)
#pragma unroll
          for (int nt = 0; nt < NT; ++nt)
#pragma unroll
            for (int c = 0; c < 4; ++c) {
              const int s = blk * 16 + g + (c >= 2 ? 8 : 0);
              bool ok = (live >> s) & 1u;
              if constexpr (!kTopk) ok = ok && unit * kUnit + s <= limit[nt][c & 1];
              if (!ok) y[blk][nt][c] = -INFINITY;
            }
      }
      // the running maximum, only where some lane has a larger one
      bool grows = false;
      float top[NT][2];
#pragma unroll
      for (int nt = 0; nt < NT; ++nt)
#pragma unroll
        for (int c = 0; c < 2; ++c) {
          top[nt][c] = fmaxf(fmaxf(y[0][nt][c], y[0][nt][c + 2]), fmaxf(y[1][nt][c], y[1][nt][c + 2]));
          grows = grows || top[nt][c] > m[nt][c];
        }
      if (__any_sync(0xffffffffu, grows)) {
#pragma unroll
        for (int nt = 0; nt < NT; ++nt)
#pragma unroll
          for (int c = 0; c < 2; ++c) {
            float x = fmaxf(top[nt][c], m[nt][c]);
            x = fmaxf(x, __shfl_xor_sync(0xffffffffu, x, 4));
            x = fmaxf(x, __shfl_xor_sync(0xffffffffu, x, 8));
            x = fmaxf(x, __shfl_xor_sync(0xffffffffu, x, 16));
            const float back = m[nt][c] == -INFINITY ? 0.f : ex2(m[nt][c] - x);
            m[nt][c] = x;
            l[nt][c] *= back;
#pragma unroll
            for (int j = 0; j < S::kTilesD; ++j) {
              o[j][nt][c] *= back;
              o[j][nt][c + 2] *= back;
            }
          }
      }
      uint32_t bp[2][NT][2];
#pragma unroll
      for (int nt = 0; nt < NT; ++nt) {
        const float m0 = m[nt][0] == -INFINITY ? 0.f : m[nt][0] - kPShift, m1 = m[nt][1] == -INFINITY ? 0.f : m[nt][1] - kPShift;
#pragma unroll
        for (int blk = 0; blk < 2; ++blk) {
          const float p0 = ex2(y[blk][nt][0] - m0), p1 = ex2(y[blk][nt][1] - m1);
          const float p2 = ex2(y[blk][nt][2] - m0), p3 = ex2(y[blk][nt][3] - m1);
          l[nt][0] += p0 + p2;
          l[nt][1] += p1 + p3;
          bp[blk][nt][0] = transposed(half2_bits(p0, p1));
          bp[blk][nt][1] = transposed(half2_bits(p2, p3));
        }
      }
      constexpr int kWords = D / 64;  // code words of a lane's D / 8 value elements
#pragma unroll
      for (int blk = 0; blk < 2; ++blk) {
        const int key = blk * 16 + 2 * t;
        const uint8_t* v0 = st + key * S::kRow + D / 2 + g * (D / 16);
        const uint8_t* sc = st + key * S::kRow + D + D / 16 + (g * (D / 8) / kKvGroup) * 2;
        uint32_t s2[2], c2[2];
#pragma unroll
        for (int h = 0; h < 2; ++h) {
          uint32_t a = *reinterpret_cast<const uint16_t*>(sc + h * 8 * S::kRow), b = *reinterpret_cast<const uint16_t*>(sc + (h * 8 + 1) * S::kRow);
          if (!whole) {
            if (!((live >> (key + h * 8)) & 1u)) a = 0;
            if (!((live >> (key + h * 8 + 1)) & 1u)) b = 0;
          }
          s2[h] = a | (b << 16);
          c2[h] = hfma2(s2[h], 0xCE00CE00u, 0u);  // -24 s, exact
        }
        uint32_t lo16[2][kWords], hi16[2][kWords];
#pragma unroll
        for (int h = 0; h < 2; ++h) {
          uint32_t a[kWords], b[kWords];
          const uint8_t* va = v0 + h * 8 * S::kRow;
          if constexpr (kWords == 2) {
            const uint2 x = *reinterpret_cast<const uint2*>(va), z = *reinterpret_cast<const uint2*>(va + S::kRow);
            a[0] = x.x;
            a[1] = x.y;
            b[0] = z.x;
            b[1] = z.y;
          } else {
            a[0] = *reinterpret_cast<const uint32_t*>(va);
            b[0] = *reinterpret_cast<const uint32_t*>(va + S::kRow);
          }
#pragma unroll
          for (int x = 0; x < kWords; ++x) {
            lo16[h][x] = __byte_perm(a[x], b[x], 0x5410);
            hi16[h][x] = __byte_perm(a[x], b[x], 0x7632);
          }
        }
        auto value = [&](int h, int x, auto e) {  // element e of word x, keys 2 t and 2 t + 1 (+ 8 h)
          constexpr int kE = decltype(e)::value;
          return hfma2(f16_codes<kE % 4>(kE < 4 ? lo16[h][x] : hi16[h][x]), s2[h], c2[h]);
        };
        auto tile = [&](auto j) {
          constexpr int kJ = decltype(j)::value;
          // rows g and g + 8 of the tile: of D = 128 the same element of the two words, of D = 64 elements j and j + 4 of the one
          constexpr int kE1 = kWords == 2 ? kJ : kJ + 4, kX1 = kWords - 1;
          const uint32_t a0 = value(0, 0, std::integral_constant<int, kJ>{}), a1 = value(0, kX1, std::integral_constant<int, kE1>{});
          const uint32_t a2 = value(1, 0, std::integral_constant<int, kJ>{}), a3 = value(1, kX1, std::integral_constant<int, kE1>{});
#pragma unroll
          for (int nt = 0; nt < NT; ++nt) mma_f16(o[kJ][nt], a0, a1, a2, a3, bp[blk][nt][0], bp[blk][nt][1]);
        };
        tile(std::integral_constant<int, 0>{});
        tile(std::integral_constant<int, 1>{});
        tile(std::integral_constant<int, 2>{});
        tile(std::integral_constant<int, 3>{});
        if constexpr (S::kTilesD == 8) {
          tile(std::integral_constant<int, 4>{});
          tile(std::integral_constant<int, 5>{});
          tile(std::integral_constant<int, 6>{});
          tile(std::integral_constant<int, 7>{});
        }
      }
      stage = stage + 1 == S::kStages ? 0 : stage + 1;
    }

    // ---- the item's end, or the run's -----------------------------------------------------------
#pragma unroll
    for (int nt = 0; nt < NT; ++nt)
#pragma unroll
      for (int c = 0; c < 2; ++c) {
        l[nt][c] += __shfl_xor_sync(0xffffffffu, l[nt][c], 4);
        l[nt][c] += __shfl_xor_sync(0xffffffffu, l[nt][c], 8);
        l[nt][c] += __shfl_xor_sync(0xffffffffu, l[nt][c], 16);
      }
    const int flags = kValid | (unit0 == 0 ? kBegins : 0) | (unit1 == at.w.units ? kEnds : 0);
    const bool complete = flags == (kValid | kBegins | kEnds), last_segment = u >= hi;
    float* part = nullptr;
    if (!complete) {
      if (last_segment) cp_wait<0>();  // (nothing of the ring is under way any more)
      part = last_segment ? reinterpret_cast<float*>(ring) : sb.warp + gw * S::kPartFloats;
      if (lane == 0) s_part[warp][last_segment ? 1 : 0] = PartDesc{at.b, at.kvh, at.rt, flags};
      __syncwarp();
    }
    constexpr int kPer = D / 8;  // consecutive elements of a row that a lane holds
#pragma unroll
    for (int nt = 0; nt < NT; ++nt)
#pragma unroll
      for (int c = 0; c < 2; ++c) {
        const int n = nt * 8 + 2 * t + c, r = row0 + n;
        float x[kPer];
#pragma unroll
        for (int j = 0; j < S::kTilesD; ++j) {
          x[j] = o[j][nt][c];
          x[kPer / 2 + j] = o[j][nt][c + 2];
        }
        if (complete) {
          if (r < rows) {
            int token, head;
            row_place(p, first, at.kvh, r, token, head);
#pragma unroll
            for (int i = 0; i < kPer; i += 4)
              write_row4<D>(p, token, head, g * kPer + i, make_float4(x[i], x[i + 1], x[i + 2], x[i + 3]), m[nt][c], l[nt][c]);
          }
        } else {
#pragma unroll
          for (int i = 0; i < kPer; i += 4)
            *reinterpret_cast<float4*>(part + n * D + g * kPer + i) = make_float4(x[i], x[i + 1], x[i + 2], x[i + 3]);
          if (g == 0) {
            part[S::kRows * D + n] = m[nt][c];
            part[S::kRows * D + S::kRows + n] = l[nt][c];
          }
        }
      }
    if (!last_segment) at.next_item(p);
  }

  // ---- parts of the CTA's warps, joined in the order of their units ------------------------------
  __syncthreads();
  CtaDesc* desc = sb.desc + blockIdx.x;
  if (tid < 2) {
    // which items are left open: the first part's if it does not begin here, the last one's if it does not end
    PartDesc open{0, 0, 0, 0};
    PartDesc run{0, 0, 0, 0};
    for (int i = 0; i < 2 * S::kWarps; ++i) {
      const PartDesc d = s_part[i >> 1][i & 1];
      if (!(d.flags & kValid)) continue;
      const bool same = (run.flags & kValid) && !(run.flags & kEnds) && d.b == run.b && d.kvh == run.kvh && d.rt == run.rt;
      if (same) run.flags |= d.flags & kEnds; else run = d;
      const bool begins = run.flags & kBegins, ends = run.flags & kEnds;
      if (tid == 0 ? !begins : (begins && !ends)) open = run;
      if (tid == 1 && begins && ends) open.flags = 0;
    }
    desc->part[tid] = open;
  }
  for (int v = tid; v < S::kRows * D / 4; v += S::kThreads) {
    const int n = v * 4 / D, d = v * 4 % D;
    PartDesc run{0, 0, 0, 0};
    float4 o = make_float4(0.f, 0.f, 0.f, 0.f);
    float m = -INFINITY, l = 0.f;
    for (int i = 0; i < 2 * S::kWarps; ++i) {
      const PartDesc pd = s_part[i >> 1][i & 1];
      if (!(pd.flags & kValid)) continue;
      if (pd.flags & kBegins || !(run.flags & kValid)) {
        run = pd;
        o = make_float4(0.f, 0.f, 0.f, 0.f);
        m = -INFINITY;
        l = 0.f;
      } else {
        run.flags |= pd.flags & kEnds;
      }
      const float* part = i & 1 ? reinterpret_cast<const float*>(smem + static_cast<size_t>(i >> 1) * S::kRingBytes)
                                : sb.warp + (static_cast<long long>(blockIdx.x) * S::kWarps + (i >> 1)) * S::kPartFloats;
      const float4 x = *reinterpret_cast<const float4*>(part + n * D + d);
      const float pm = part[S::kRows * D + n], pl = part[S::kRows * D + S::kRows + n];
      const float mm = fmaxf(m, pm), a = m == -INFINITY ? 0.f : ex2(m - mm), b = pm == -INFINITY ? 0.f : ex2(pm - mm);
      o = make_float4(o.x * a + x.x * b, o.y * a + x.y * b, o.z * a + x.z * b, o.w * a + x.w * b);
      l = l * a + pl * b;
      m = mm;
      const bool begins = run.flags & kBegins, ends = run.flags & kEnds;
      // does the item go on in a later part of this CTA?
      bool more = false;
      if (!ends)
        for (int k = i + 1; k < 2 * S::kWarps && !more; ++k) more = s_part[k >> 1][k & 1].flags & kValid;
      if (more) continue;
      if (begins && ends) {
        int first = run.b, rows = p.group;
        if constexpr (!kTopk) {
          const Kv4Request r = kv4_request(p, run.b);
          first = r.first;
          rows = r.n * p.group;
        }
        const int r = run.rt * S::kRows + n;
        if (r < rows) {
          int token, head;
          row_place(p, first, run.kvh, r, token, head);
          write_row4<D>(p, token, head, d, o, m, l);
        }
      } else {
        float* to = sb.cta + (static_cast<long long>(blockIdx.x) * 2 + (begins ? 1 : 0)) * S::kPartFloats;
        *reinterpret_cast<float4*>(to + n * D + d) = o;
        if (d == 0) {
          to[S::kRows * D + n] = m;
          to[S::kRows * D + S::kRows + n] = l;
        }
      }
      run.flags = 0;
    }
  }
}

// Items that span CTAs: CTA c joins the one that begins in run c with the pieces of the runs behind it.
template <int D, int NT, bool kTopk>
__global__ void __launch_bounds__(256) attention_join_kernel(const Kv4AttnParams p, const SplitBuffers sb, int n_ctas) {
  using S = Shape<D, NT>;
  chain_wait();
  const PartDesc run = sb.desc[blockIdx.x].part[1];
  if (!(run.flags & kValid)) return;
  int first = run.b, rows = p.group;
  if constexpr (!kTopk) {
    const Kv4Request r = kv4_request(p, run.b);
    first = r.first;
    rows = r.n * p.group;
  }
  for (int v = blockIdx.y * 256 + threadIdx.x; v < S::kRows * D / 4; v += gridDim.y * 256) {
    const int n = v * 4 / D, d = v * 4 % D, r = run.rt * S::kRows + n;
    if (r >= rows) continue;
    const float* part = sb.cta + (static_cast<long long>(blockIdx.x) * 2 + 1) * S::kPartFloats;
    float4 o = *reinterpret_cast<const float4*>(part + n * D + d);
    float m = part[S::kRows * D + n], l = part[S::kRows * D + S::kRows + n];
    for (int c = blockIdx.x + 1; c < n_ctas; ++c) {
      const int flags = sb.desc[c].part[0].flags;
      if (!(flags & kValid)) continue;  // (a run without units)
      part = sb.cta + static_cast<long long>(c) * 2 * S::kPartFloats;
      const float4 x = *reinterpret_cast<const float4*>(part + n * D + d);
      const float pm = part[S::kRows * D + n], pl = part[S::kRows * D + S::kRows + n];
      const float mm = fmaxf(m, pm), a = m == -INFINITY ? 0.f : ex2(m - mm), b = pm == -INFINITY ? 0.f : ex2(pm - mm);
      o = make_float4(o.x * a + x.x * b, o.y * a + x.y * b, o.z * a + x.z * b, o.w * a + x.w * b);
      l = l * a + pl * b;
      m = mm;
      if (flags & kEnds) break;
    }
    int token, head;
    row_place(p, first, run.kvh, r, token, head);
    write_row4<D>(p, token, head, d, o, m, l);
  }
}

template <int D, int NT>
size_t split_bytes(int grid) {
  using S = Shape<D, NT>;
  return static_cast<size_t>(grid) * (sizeof(CtaDesc) + (2 + S::kWarps) * S::kPartFloats * sizeof(float));
}

template <int D, int NT, bool kTopk>
cudaError_t launch_rows(const Kv4AttnParams& p, void* scratch, int grid, cudaStream_t stream) {
  using S = Shape<D, NT>;
  static std::atomic<unsigned long long> allowed{0};
  const cudaError_t e = allow_smem(reinterpret_cast<const void*>(attention_rows_kernel<D, NT, kTopk>), allowed);
  if (e != cudaSuccess) return e;
  SplitBuffers sb;
  sb.cta = static_cast<float*>(scratch);
  sb.warp = sb.cta + static_cast<size_t>(grid) * 2 * S::kPartFloats;
  sb.desc = reinterpret_cast<CtaDesc*>(sb.warp + static_cast<size_t>(grid) * S::kWarps * S::kPartFloats);
  const cudaError_t r = launch_chained(attention_rows_kernel<D, NT, kTopk>, dim3(grid), dim3(S::kThreads), S::kSmem, stream, 1, p, sb);
  if (r != cudaSuccess) return r;
  return launch_chained(attention_join_kernel<D, NT, kTopk>, dim3(grid, (S::kRows * D / 4 + 255) / 256), dim3(256), 0, stream, 1, p, sb, grid);
}

}  // namespace

size_t kv4_rows_scratch_bytes(int D) {
  const int grid = sm_count();
  const size_t a = D == 64 ? split_bytes<64, 1>(grid) : split_bytes<128, 1>(grid);
  const size_t b = D == 64 ? split_bytes<64, 2>(grid) : split_bytes<128, 2>(grid);
  return a > b ? a : b;
}

cudaError_t launch_kv4_attention_rows(int D, long long most_rows, const Kv4AttnParams& p, void* scratch, int grid, cudaStream_t stream) {
  const bool wide = most_rows > 8;
  if (p.idx != nullptr) {
    if (D == 64) return wide ? launch_rows<64, 2, true>(p, scratch, grid, stream) : launch_rows<64, 1, true>(p, scratch, grid, stream);
    return wide ? launch_rows<128, 2, true>(p, scratch, grid, stream) : launch_rows<128, 1, true>(p, scratch, grid, stream);
  }
  if (D == 64) return wide ? launch_rows<64, 2, false>(p, scratch, grid, stream) : launch_rows<64, 1, false>(p, scratch, grid, stream);
  return wide ? launch_rows<128, 2, false>(p, scratch, grid, stream) : launch_rows<128, 1, false>(p, scratch, grid, stream);
}

}  // namespace lt
