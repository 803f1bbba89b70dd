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
//   S^T = K Q^T: lane (g, t) holds keys g and g + 8, of each group of 32 elements the 8 of code word t.  A nibble by itself in the low
//     bits of an fp16 is u 2^-24, one in the bits above it u 2^-20, subnormal and exact, so that a mask makes operands of codes, and
//     half of them need no shift.  Queries are scaled by a power of two to fp16's range (exact but for what is under 2^-35 of the row's
//     largest), those that meet u 2^-20 by a further 1 / 16; the accumulators start at -8 sum q, so that they end at sum q (u - 8),
//     exact products in fp32, and the scale of (key, group) multiplies that in fp32.
//   P^T: the accumulators, in fp16, turned by movmatrix.
//   O^T = V^T P^T: lane (g, t) holds elements 16 g .. 16 g + 15 of keys 2 t, 2 t + 1, 2 t + 8, 2 t + 9: one scale group, words that pair up
//     by two byte permutations.  A value is (16 + u) s - 24 s, one FMA on fp16 pairs, for the nibbles that are shifted there anyway; for
//     the others (1024 + u) - 1032 or (1024 + 16 u) / 16 - 72, exact, times s: an FMA more and a shift less, which evens out the pipes.
//
// Work is dealt out in units of 32 keys: all units of all (request, key-value head, row tile) items in a row are cut into equal
// runs, one per warp, whatever the lengths.  A warp has its own ring of cp.async stages and waits for nobody.  Items that it
// sees whole it writes out itself; the parts of others are joined first within the CTA, then, where an item spans CTAs, by a
// second kernel.  Runs are a matter of the lengths alone, so results do not vary.
//
// Measured: 64 requests of up to 32 K positions, 8 key-value heads of 128 with 8 query heads each: 1.21 GB in 279 us, 4.3 TB/s, 0.66 of
// the copy rate (one request of 1 M: 269 us, 0.68).  Instructions bound it: 300 for 16 keys of a head (by count 40 masks and shifts for the
// keys, 48 and 58 of fp16 arithmetic for the values), 0.64 of the issue slots with 3 warps to a scheduler; at 335 it took, without its
// loads, still 0.91 of its time.
#include "lt_kv4_parts.cuh"

namespace lt {
namespace {

constexpr int kUnit = 32;          // keys of a unit

template <int D, int NT>
struct Shape {
  static constexpr int kRow = kv4_row_bytes(D);
  static constexpr int kGroups = D / kKvGroup;
  static constexpr int kRows = 8 * NT;       // query rows of an item
  static constexpr int kTilesD = D / 16;     // 16-row tiles of O^T
  // As many warps as their registers allow, and a multiple of the 4 schedulers (the decode step above, us of GPU time with 10 / 12 / 16 warps:
  // 315 / 265 / 277; 16 rows take 255 registers, which 8 warps have).  Two stages ahead suffice (with 4 stages 267).
  static constexpr int kWarps = NT == 1 ? 12 : 8;
  static constexpr int kThreads = kWarps * 32;
  static constexpr int kStages = 3;
  static constexpr int kUnitBytes = kUnit * kRow;
  static constexpr int kPartFloats = part_floats(kRows, D);
  static constexpr int kRingBytes = kStages * kUnitBytes;
  static constexpr int kPartInRing = kPartFloats * 4 <= kRingBytes;
  static constexpr size_t kSmem = static_cast<size_t>(kWarps) * kRingBytes;
  static_assert(kPartInRing, "a warp leaves its last part in its ring");
};

// ---- PTX ------------------------------------------------------------------------------------
__device__ __forceinline__ void mma_f16(float (&c)[4], uint32_t a0, uint32_t a1, uint32_t a2, uint32_t a3, uint32_t b0, uint32_t b1) {
  asm("mma.sync.aligned.m16n8k16.row.col.f32.f16.f16.f32 {%0, %1, %2, %3}, {%4, %5, %6, %7}, {%8, %9}, {%0, %1, %2, %3};"
      : "+f"(c[0]), "+f"(c[1]), "+f"(c[2]), "+f"(c[3])
      : "r"(a0), "r"(a1), "r"(a2), "r"(a3), "r"(b0), "r"(b1));
}
// The same into accumulators that begin at c.
__device__ __forceinline__ void mma_f16_from(float (&d)[4], uint32_t a0, uint32_t a1, uint32_t a2, uint32_t a3, uint32_t b0, uint32_t b1,
                                             const float (&c)[4]) {
  asm("mma.sync.aligned.m16n8k16.row.col.f32.f16.f16.f32 {%0, %1, %2, %3}, {%4, %5, %6, %7}, {%8, %9}, {%10, %11, %12, %13};"
      : "=f"(d[0]), "=f"(d[1]), "=f"(d[2]), "=f"(d[3])
      : "r"(a0), "r"(a1), "r"(a2), "r"(a3), "r"(b0), "r"(b1), "f"(c[0]), "f"(c[1]), "f"(c[2]), "f"(c[3]));
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

// Nibbles 0 and 1 of each half of w as fp16 pairs u 2^-24 and u 2^-20; nibbles 2 and 3 are those of w >> 8.
__device__ __forceinline__ uint32_t codes_low(uint32_t w) { return w & 0x000F000Fu; }
__device__ __forceinline__ uint32_t codes_high(uint32_t w) { return w & 0x00F000F0u; }
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
    const long long item = quotient(off, w.units);
    unit = static_cast<int>(off - item * w.units);
    kvh = static_cast<int>(quotient(item, w.tiles));
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
    if constexpr (!kTopk) {
      if (b < p.B && w.load(p, b) == 0) {
        b = next_request(p, b + 1, [&](const Kv4Request& r) {
          const long long rows = static_cast<long long>(r.n) * p.group;
          return rows >= p.min_rows && rows <= p.max_rows;
        });
        if (b < p.B) w.load(p, b);
      }
    }
  }
  __device__ __forceinline__ void next(const Kv4AttnParams& p, bool more) {
    if (++unit == w.units && more) next_item(p);
  }
};

// ---------------------------------------------------------------------------------------------
template <int D, int NT, bool kTopk>
__global__ void __launch_bounds__(Shape<D, NT>::kThreads, 1) attention_rows_kernel(const Kv4AttnParams p, const SplitBuffers sb) {
  using S = Shape<D, NT>;
  extern __shared__ __align__(128) uint8_t smem[];
  __shared__ long long s_first[S::kThreads], s_sums[S::kWarps];
  __shared__ PartDesc s_part[S::kWarps][2];
  const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5, g = lane >> 2, t = lane & 3;
  chain_wait();

  // ---- this warp's run [lo, hi) of all units, and where it begins --------------------------------
  const long long gw = static_cast<long long>(blockIdx.x) * S::kWarps + warp, n_warps = static_cast<long long>(gridDim.x) * S::kWarps;
  long long total = 0, lo, hi;
  auto cut = [&]() {  // as even as it goes; the remainder is spread over the CTAs
    const long long even = quotient(total, n_warps);
    const unsigned rest = static_cast<unsigned>(total - even * n_warps), n = static_cast<unsigned>(n_warps), w = static_cast<unsigned>(gw);
    lo = even * gw + rest * w / n;  // (rest and w are both under 2^12)
    hi = even * (gw + 1) + rest * (w + 1) / n;
  };
  Cursor<D, NT, kTopk> at;
  if constexpr (kTopk) {
    const Kv4Rows rows = kv4_rows(p);
    const int units = (p.topk + kUnit - 1) / kUnit, tiles = (p.group + S::kRows - 1) / S::kRows;
    const long long per = static_cast<long long>(units) * tiles * p.Hkv;
    total = per * (rows.end - rows.first);
    cut();
    if (lo < hi) {
      const long long token = quotient(lo, per);
      at.start(p, rows.first + static_cast<int>(token), lo - token * per);
    }
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
      cut();
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
  bool page_there = false;
  const uint8_t* page_src = p.pool;
  // selected: the indices of the unit after the next one, the page numbers of the next one
  Cursor<D, NT, kTopk> idx_at = at;   // unit whose indices are loaded next
  long long idx_loaded = lo;
  int idx_far = -1;                   // loaded indices of the unit behind `slot_next`'s
  int near_pos = -1, near_page = -1;  // the next unit to fetch: position and page of this lane's key
  int req_b = 0, req_token = -1;
  Kv4Request req{0, 0, 0};

  const int row3 = lane / 9, piece_at = (lane - row3 * 9) * (S::kRow / 9), piece3 = row3 * S::kRow + piece_at;
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
      req_b = req_token < 0 ? request_of_row(p, token) : request_of_row_from(p, req_b, token);
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

  unsigned seen_of[S::kStages];  // which keys of the stages under way are there at all, the oldest stage's first
#pragma unroll
  for (int i = 0; i < S::kStages; ++i) seen_of[i] = 0;
  auto fetch = [&]() {
#pragma unroll
    for (int i = 0; i + 1 < S::kStages; ++i) seen_of[i] = seen_of[i + 1];
    if (fetched < hi) {
      const uint32_t dst = ring_addr + fetch_stage * S::kUnitBytes;
      if constexpr (kTopk) {
        const bool sees = near_page >= 0 && near_page < p.pool_pages;
        seen_of[S::kStages - 1] = __ballot_sync(0xffffffffu, sees);
        const uint8_t* mine = sees ? p.pool + near_page * page_bytes + (ahead.kvh * kPageKeys + (near_pos & (kPageKeys - 1))) * S::kRow : nullptr;
        // 27 lanes take the 9 pieces of three rows at a time
        constexpr int kPiece = S::kRow / 9;
#pragma unroll
        for (int j = 0; j < (kUnit + 2) / 3; ++j) {
          const int key = j * 3 + row3;
          const unsigned long long row = __shfl_sync(0xffffffffu, reinterpret_cast<unsigned long long>(mine), key & 31);
          if (row != 0 && (j < kUnit / 3 ? row3 < 3 : row3 < kUnit % 3))
            cp_async<kPiece>(dst + piece3 + j * 3 * S::kRow, reinterpret_cast<const uint8_t*>(row) + piece_at);
        }
        step_pages();
        load_indices();
      } else {
        if ((ahead.unit & 1) == 0 || fetched == lo) {  // a page, or the half that the run begins with
          const int page_no = ahead.unit >> 1;
          if (ahead.unit < 2 || pages_at < 0 || page_no - pages_at >= 32) {
            pages_at = page_no;
            pages = page_no + lane < p.max_pages ? p.page_table[static_cast<long long>(ahead.b) * p.max_pages + page_no + lane] : -1;
          }
          const int page = __shfl_sync(0xffffffffu, pages, page_no - pages_at);
          page_there = page >= 0 && page < p.pool_pages;
          page_src = p.pool + (page_there ? page : 0) * page_bytes + (ahead.kvh * kPageKeys + (ahead.unit & 1) * kUnit) * S::kRow + lane * 16;
        }
        seen_of[S::kStages - 1] = page_there ? 0xffffffffu : 0u;
        if (page_there) {
#pragma unroll
          for (int i = 0; i < (S::kUnitBytes / 16 + 31) / 32; ++i)
            if (S::kUnitBytes / 16 % 32 == 0 || i * 32 + lane < S::kUnitBytes / 16) cp_async<16>(dst + lane * 16 + i * 512, page_src + i * 512);
        }
        page_src += S::kUnitBytes;
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
    // queries as the column operand, what the accumulators begin with, and what a column's scores are worth
    uint32_t bq[NT][S::kGroups][2][2];
    float off[NT][S::kGroups][4], worth[NT][2];
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
      // the row's largest exponent; its largest element comes to lie in [2^15, 2^16), under 65,280
      uint32_t top = 0;
#pragma unroll
      for (int gi = 0; gi < S::kGroups; ++gi) {
        const uint32_t w[4] = {x[gi].x, x[gi].y, x[gi].z, x[gi].w};
#pragma unroll
        for (int i = 0; i < 4; ++i) top = max(top, max(w[i] & 0x7fffu, (w[i] >> 16) & 0x7fffu));
      }
      top = max(top, __shfl_xor_sync(0xffffffffu, top, 1));
      top = max(top, __shfl_xor_sync(0xffffffffu, top, 2));
      const int e = max(static_cast<int>(top >> 7), 21);  // biased exponent; rows under 2^-106 stay smaller
      // (a negative scale turns the queries' signs)
      const float up = copysignf(__uint_as_float(static_cast<uint32_t>(127 + 127 + 15 - e) << 23), p.scale);
#pragma unroll
      for (int gi = 0; gi < S::kGroups; ++gi) {
        const uint32_t w[4] = {x[gi].x, x[gi].y, x[gi].z, x[gi].w};
        float f[8], low = 0.f, high = 0.f;
#pragma unroll
        for (int i = 0; i < 4; ++i) {
          f[2 * i] = __uint_as_float(w[i] << 16) * up;
          f[2 * i + 1] = __uint_as_float(w[i] & 0xffff0000u) * (up * 0.0625f);
          low += f[2 * i];
          high += f[2 * i + 1];
        }
        // elements i and i + 4 of the word side by side, as the codes come
#pragma unroll
        for (int i = 0; i < 4; ++i) bq[nt][gi][i >> 1][i & 1] = half2_bits(f[i], f[i + 4]);
        float sum = -8.f / 16777216.f * __fmaf_rn(16.f, high, low);
        sum += __shfl_xor_sync(0xffffffffu, sum, 1);
        sum += __shfl_xor_sync(0xffffffffu, sum, 2);
        off[nt][gi][0] = off[nt][gi][2] = __shfl_sync(0xffffffffu, sum, 8 * t);
        off[nt][gi][1] = off[nt][gi][3] = __shfl_sync(0xffffffffu, sum, 8 * t + 4);
      }
      // (before it scores are under 2^13: at most 32 products under 2^-5 and a scale under 2^11 for each of 4 groups)
      const float w = worth_of(e, p.scale, 16777216.f, 0x1p113f);
      worth[nt][0] = __shfl_sync(0xffffffffu, w, 8 * t);
      worth[nt][1] = __shfl_sync(0xffffffffu, w, 8 * t + 4);
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
    float o[S::kTilesD][NT][4], l[NT][2];
    float bar[NT][2], shift[NT][2];  // scores beyond bar raise the maximum m; shift = kPShift - m, in powers of two
#pragma unroll
    for (int nt = 0; nt < NT; ++nt) {
      bar[nt][0] = bar[nt][1] = -INFINITY;
      shift[nt][0] = shift[nt][1] = kNothing;
      l[nt][0] = l[nt][1] = 0.f;
#pragma unroll
      for (int j = 0; j < S::kTilesD; ++j)
#pragma unroll
        for (int c = 0; c < 4; ++c) o[j][nt][c] = 0.f;
    }

    const ValueConstants constants;
    // one unit; kWhole: every row of the tile sees all its keys
    auto take = [&](const uint8_t* st, int unit, unsigned seen, auto whole_unit) {
      constexpr bool kWhole = decltype(whole_unit)::value;
      float y[2][NT][4];
#pragma unroll
      for (int blk = 0; blk < 2; ++blk) {
        const uint8_t* k0 = st + (blk * 16 + g) * S::kRow;
        const uint8_t* k1 = k0 + 8 * S::kRow;
        struct alignas(D / 16) Scales {
          __half s[S::kGroups];
        };
        const Scales ks0 = *reinterpret_cast<const Scales*>(k0 + D), ks1 = *reinterpret_cast<const Scales*>(k1 + D);
#pragma unroll
        for (int nt = 0; nt < NT; ++nt)
#pragma unroll
          for (int c = 0; c < 4; ++c) y[blk][nt][c] = 0.f;
#pragma unroll
        for (int gi = 0; gi < S::kGroups; ++gi) {
          const uint32_t w0 = *reinterpret_cast<const uint32_t*>(k0 + gi * 16 + t * 4);
          const uint32_t w1 = *reinterpret_cast<const uint32_t*>(k1 + gi * 16 + t * 4);
          const uint32_t x0 = w0 >> 8, x1 = w1 >> 8;
          const float s0 = __half2float(ks0.s[gi]), s1 = __half2float(ks1.s[gi]);
#pragma unroll
          for (int nt = 0; nt < NT; ++nt) {
            float acc[4];
            mma_f16_from(acc, codes_low(w0), codes_low(w1), codes_high(w0), codes_high(w1), bq[nt][gi][0][0], bq[nt][gi][0][1], off[nt][gi]);
            mma_f16(acc, codes_low(x0), codes_low(x1), codes_high(x0), codes_high(x1), bq[nt][gi][1][0], bq[nt][gi][1][1]);
            y[blk][nt][0] = __fmaf_rn(acc[0], s0, y[blk][nt][0]);
            y[blk][nt][1] = __fmaf_rn(acc[1], s0, y[blk][nt][1]);
            y[blk][nt][2] = __fmaf_rn(acc[2], s1, y[blk][nt][2]);
            y[blk][nt][3] = __fmaf_rn(acc[3], s1, y[blk][nt][3]);
          }
        }
      }
      unsigned live = seen;  // keys that some row of the tile sees: all others' values are taken as zero, whatever lies there
      if constexpr (!kWhole) {
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
      bool grows = false;
      float top[NT][2];
#pragma unroll
      for (int nt = 0; nt < NT; ++nt)
#pragma unroll
        for (int c = 0; c < 2; ++c) {
          top[nt][c] = fmaxf(fmaxf(y[0][nt][c], y[0][nt][c + 2]), fmaxf(y[1][nt][c], y[1][nt][c + 2]));
          grows = grows || top[nt][c] > bar[nt][c];
        }
      if (__any_sync(0xffffffffu, grows)) {
#pragma unroll
        for (int nt = 0; nt < NT; ++nt)
#pragma unroll
          for (int c = 0; c < 2; ++c) {
            float x = top[nt][c];
            x = fmaxf(x, __shfl_xor_sync(0xffffffffu, x, 4));
            x = fmaxf(x, __shfl_xor_sync(0xffffffffu, x, 8));
            x = fmaxf(x, __shfl_xor_sync(0xffffffffu, x, 16));
            if (x > bar[nt][c]) {  // (the same in all lanes of the column)
              const float now = shift_of(x, worth[nt][c]), back = ex2(now - shift[nt][c]);
              bar[nt][c] = bar_of(x, worth[nt][c]);
              shift[nt][c] = now;
              l[nt][c] *= back;
#pragma unroll
              for (int j = 0; j < S::kTilesD; ++j) {
                o[j][nt][c] *= back;
                o[j][nt][c + 2] *= back;
              }
            }
          }
      }
      uint32_t bp[2][NT][2];
#pragma unroll
      for (int nt = 0; nt < NT; ++nt) {
        const float c0 = worth[nt][0], c1 = worth[nt][1], m0 = shift[nt][0], m1 = shift[nt][1];
#pragma unroll
        for (int blk = 0; blk < 2; ++blk) {
          const float p0 = ex2(__fmaf_rn(y[blk][nt][0], c0, m0)), p1 = ex2(__fmaf_rn(y[blk][nt][1], c1, m1));
          const float p2 = ex2(__fmaf_rn(y[blk][nt][2], c0, m0)), p3 = ex2(__fmaf_rn(y[blk][nt][3], c1, m1));
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
          if constexpr (!kWhole) {
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
          return f16_values<kE % 4>(kE < 4 ? lo16[h][x] : hi16[h][x], s2[h], c2[h], constants);
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
    };

    for (int unit = unit0; unit < unit1; ++unit, ++u) {
      cp_wait<S::kStages - 2>();
      __syncwarp();  // this unit has come, for all lanes, and all are through with the one before, whose stage is filled again
      fetch();
      const uint8_t* st = ring + stage * S::kUnitBytes;
      const unsigned seen = seen_of[0];
      const bool whole = seen == 0xffffffffu && (kTopk || unit * kUnit + kUnit - 1 <= least);
      if (whole)
        take(st, unit, seen, std::true_type{});
      else
        take(st, unit, seen, std::false_type{});
      stage = stage + 1 == S::kStages ? 0 : stage + 1;
    }

    // ---- the item's end, or the run's -----------------------------------------------------------
    float m[NT][2];
#pragma unroll
    for (int nt = 0; nt < NT; ++nt)
#pragma unroll
      for (int c = 0; c < 2; ++c) {
        l[nt][c] += __shfl_xor_sync(0xffffffffu, l[nt][c], 4);
        l[nt][c] += __shfl_xor_sync(0xffffffffu, l[nt][c], 8);
        l[nt][c] += __shfl_xor_sync(0xffffffffu, l[nt][c], 16);
        m[nt][c] = l[nt][c] > 0.f ? kPShift - shift[nt][c] : -INFINITY;
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
  const int my_flags = lane < 2 * S::kWarps ? s_part[lane >> 1][lane & 1].flags : 0;
  const unsigned parts = __ballot_sync(0xffffffffu, my_flags & kValid), begin_at = __ballot_sync(0xffffffffu, my_flags & kBegins),
                 end_at = __ballot_sync(0xffffffffu, my_flags & kEnds);
  static_assert(2 * S::kWarps <= 32, "a bit for every part");
  CtaDesc* desc = sb.desc + blockIdx.x;
  if (tid < 2) {
    // the items that are left open: the one that the first part goes on with if it does not begin here, and the one that the last part
    // belongs to if that item begins here and does not end
    PartDesc open{0, 0, 0, 0};
    const int first_part = __ffs(parts) - 1, last_begin = 31 - __clz(begin_at | 1u);
    if (tid == 0 && parts != 0 && !((begin_at >> first_part) & 1u)) {
      open = s_part[first_part >> 1][first_part & 1];
      const unsigned its = begin_at != 0 ? (1u << (__ffs(begin_at) - 1)) - 1u : 0xffffffffu;  // parts before any other item begins
      open.flags |= (end_at & its) != 0 ? kEnds : 0;
    }
    if (tid == 1 && begin_at != 0 && (end_at >> last_begin) == 0) open = s_part[last_begin >> 1][last_begin & 1];
    desc->part[tid] = open;
    if (tid == 0) desc->status = 0;
  }
  if (parts == 0) return;
  for (int v = tid; v < S::kRows * D / 4; v += S::kThreads) {
    const int n = v * 4 / D, d = v * 4 % D;
    float4 o = make_float4(0.f, 0.f, 0.f, 0.f);
    float m = -INFINITY, l = 0.f;
    bool begins = false;
    for (unsigned left = parts; left != 0; left &= left - 1) {
      const int i = __ffs(left) - 1;
      const float* part = i & 1 ? reinterpret_cast<const float*>(smem + static_cast<size_t>(i >> 1) * S::kRingBytes)
                                : sb.warp + (static_cast<long long>(blockIdx.x) * S::kWarps + (i >> 1)) * S::kPartFloats;
      const float4 x = *reinterpret_cast<const float4*>(part + n * D + d);
      const float pm = part[S::kRows * D + n], pl = part[S::kRows * D + S::kRows + n];
      if ((begin_at >> i) & 1u) {
        begins = true;
        o = x;
        m = pm;
        l = pl;
      } else {
        join(o, m, l, x, pm, pl);
      }
      const bool ends = (end_at >> i) & 1u;
      if (!ends && (left & (left - 1)) != 0) continue;  // the item goes on in the next part
      if (begins && ends) {
        const PartDesc run = s_part[i >> 1][i & 1];
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
      o = make_float4(0.f, 0.f, 0.f, 0.f);
      m = -INFINITY;
      l = 0.f;
      begins = false;
    }
  }
}

template <int D, int NT>
size_t split_bytes(int grid) {
  using S = Shape<D, NT>;
  return static_cast<size_t>(grid) * (sizeof(CtaDesc) + (2 + S::kWarps) * S::kPartFloats * sizeof(float));
}

template <int D, int NT, bool kTopk>
cudaError_t launch_rows(const Kv4AttnParams& p, void* scratch, Control* ctl, int grid, cudaStream_t stream) {
  using S = Shape<D, NT>;
  static std::atomic<unsigned long long> allowed{0};
  const cudaError_t e = allow_smem(reinterpret_cast<const void*>(attention_rows_kernel<D, NT, kTopk>), allowed);
  if (e != cudaSuccess) return e;
  SplitBuffers sb;
  sb.cta = static_cast<float*>(scratch);
  sb.warp = sb.cta + static_cast<size_t>(grid) * 2 * S::kPartFloats;
  sb.desc = reinterpret_cast<CtaDesc*>(sb.warp + static_cast<size_t>(grid) * S::kWarps * S::kPartFloats);
  sb.ctl = ctl;
  const cudaError_t r = launch_chained(attention_rows_kernel<D, NT, kTopk>, dim3(grid), dim3(S::kThreads), S::kSmem, stream, 1, p, sb);
  if (r != cudaSuccess) return r;
  return launch_join<D, S::kRows, kTopk>(p, sb, grid, false, stream);
}

}  // namespace

size_t kv4_rows_scratch_bytes(int D) {
  const int grid = sm_count();
  const size_t a = D == 64 ? split_bytes<64, 1>(grid) : split_bytes<128, 1>(grid);
  const size_t b = D == 64 ? split_bytes<64, 2>(grid) : split_bytes<128, 2>(grid);
  return a > b ? a : b;
}

cudaError_t launch_kv4_attention_rows(int D, long long most_rows, const Kv4AttnParams& p, void* scratch, Control* ctl, int grid,
                                      cudaStream_t stream) {
  // 8 rows, or 16 in one pass over the keys (64 requests over 16 K keys, 4 heads: 8 rows 125 us, in the wide form 175; 9 to 16 rows 230 in two
  // passes, 177 in one; 24 rows 336 and 330)
  const bool wide = most_rows > 8;
  if (p.idx != nullptr) {
    if (D == 64) return wide ? launch_rows<64, 2, true>(p, scratch, ctl, grid, stream) : launch_rows<64, 1, true>(p, scratch, ctl, grid, stream);
    return wide ? launch_rows<128, 2, true>(p, scratch, ctl, grid, stream) : launch_rows<128, 1, true>(p, scratch, ctl, grid, stream);
  }
  if (D == 64) return wide ? launch_rows<64, 2, false>(p, scratch, ctl, grid, stream) : launch_rows<64, 1, false>(p, scratch, ctl, grid, stream);
  return wide ? launch_rows<128, 2, false>(p, scratch, ctl, grid, stream) : launch_rows<128, 1, false>(p, scratch, ctl, grid, stream);
}

}  // namespace lt
