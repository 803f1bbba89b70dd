// Attention of many rows per key-value head (prefill chunks, or many heads on one key-value head) over the 4-bit cache: tcgen05.
//
// An item is up to kTiles tiles of 128 rows (query heads of one key-value head, and tokens) of a request; a CTA takes its keys 128 at a
// time, or 64 where it has one tile.  Roles, a warp or more each, that meet at mbarriers only:
//   rows      where the tile's 128 cache rows are (pages, or the indexer's positions), and their copy into a ring of 32 rows a stage
//   keys      codes from the ring -> fp16 (code - 8) scale, exact -> shared memory [key][element], 128-byte swizzle
//   values    the same, transposed: [element][key]
//   products  one thread: S = Q K^T into tensor memory, O += P V with P as the tensor-memory operand
//   softmax   a warpgroup per tile, a thread per row: maximum, exponentials, P (fp16) back over S
// Each tile's chain (S, softmax, P V) is serial; two tiles per CTA, or two CTAs of one tile per SM, keep the tensor cores and the
// exponential units at it in turn, and two tiles share the unpacked keys and values.  128 keys x 128 rows are 1024 clocks of tensor core
// (8192 bf16 flops a clock) and 1024 of exponentials (16 a clock): the two bound this together.  The roles' loops are kept short on purpose:
// with everything unrolled the warps of an SM waited for instructions most of the time (a chunk of 2048 over 30 K: 2.5 ms, loops 1.8).
//
// Measured: that chunk (32 query heads on 4 key-value heads of 128) 1.35 ms, 795 TFLOP/s, 0.49 of the measured bf16 burst: tensor cores at
// work 0.38 of the clocks, exponentials 0.38, issue slots 0.45; what is left is each tile's chain, 3.3 thousand clocks of softmax and 2.1 until
// its next scores.  1024 tokens of 64 heads over 2048 positions of one key-value head 268 us, bound by unpacking and by the same chain.
//
// Column c = 8 m + i of a key tile is key 8 m + (m + i) % 8: then 8 neighbouring rows of the ring, and the 8 columns of a 16-byte
// piece of the transposed values, are read and written in different banks.  Elements are paired as the codes come, (i, i + 4) of every
// eight, in the queries too.  Queries are scaled by a power of two to fp16's range.  The work of all items, in units
// of the keys taken at a time and a cost per item, is cut evenly over the CTAs; items that span CTAs are joined by a second kernel (lt_kv4_parts.cuh).
#include "lt_kv4_parts.cuh"
#include "lt_ptx.cuh"

namespace lt {
namespace {

constexpr int kTileRows = 128;
constexpr int kStep = 32;       // rows of a stage of the ring
constexpr int kKnown = 1024;    // requests whose work is kept from the first look to the second
constexpr int kSeenStages = 4;  // tiles whose visible keys are noted at once

template <int D, int kTiles>
struct Cfg {
  static constexpr int kRow = kv4_row_bytes(D);
  static constexpr int kRows = kTiles * kTileRows;
  // Two tiles share 128 unpacked keys at a time, and one's product runs beside the other's softmax.  A single tile takes 64 keys and has
  // S twice, so that its own next scores are there when a softmax ends.
  static constexpr int kKeys = 64 * kTiles, kBufs = kTiles == 2 ? 1 : 2, kChunks = kKeys / 32;
  static constexpr int kStages = 2;  // of unpacked keys, and of values
  static constexpr int kSoftmaxWarps = 4 * kTiles, kKeyWarp = kSoftmaxWarps, kValueWarp = kKeyWarp + 2, kMmaWarp = kValueWarp + 2,
                       kRowWarp = kMmaWarp + 1, kWarps = kRowWarp + 1, kThreads = kWarps * 32;
  static constexpr int kQueryBytes = kTileRows * D * 2, kTileBytes = kKeys * D * 2;  // queries; keys or values of one tile
  static constexpr int kRing = kTiles == 2 ? 6 : 3, kStepBytes = kStep * kRow;
  static constexpr size_t kSmem = 1024 + static_cast<size_t>(kQueryBytes) * kTiles + kTileBytes * 2 * kStages + kRing * kStepBytes;
  static constexpr int kCtasPerSm = kTiles == 2 ? 1 : 2;
  static constexpr int kTmemCols = 256 * kTiles;  // S / P: 128 columns a tile (kBufs times kKeys), O: D (128 are taken)
};

struct Shared {
  uint64_t k_full[2], k_empty[2], v_full[2], v_empty[2], s_full[2][2], p_full[2][2], o_done[2][2], q_full[2], ring_full[6], ring_empty[6],
      seen_full[kSeenStages], seen_empty[kSeenStages], drained;
  unsigned there[kSeenStages][4];  // a bit per key of the tile
  int abort_flag[2], drain_flag[2];  // [1]: limit of a wait in microseconds (lt_ptx.cuh)
  uint32_t tmem;
  long long sums[16];
  // where the CTA's run begins
  long long lo, hi;
  int b, kvh, rt, unit;
};

// Items of a request (dense form): row tiles of kRows rows, each with the units of kKeys keys that its last row sees.
template <int kRows, int kKeys>
__device__ __forceinline__ int item_units(const Kv4AttnParams& p, const Kv4Request& r, int rt) {
  const long long rows = static_cast<long long>(r.n) * p.group, end = static_cast<long long>(rt + 1) * kRows;
  const int last = static_cast<int>(((end < rows ? end : rows) - 1) / p.group);
  const long long keys = static_cast<long long>(r.ctx) + last + 1, reach = static_cast<long long>(p.max_pages) * kPageKeys;
  return static_cast<int>(((keys < reach ? keys : reach) + kKeys - 1) / kKeys);
}
template <int kRows>
__device__ __forceinline__ int request_tiles(const Kv4AttnParams& p, const Kv4Request& r) {
  const long long rows = static_cast<long long>(r.n) * p.group;
  return rows < p.min_rows || rows > p.max_rows ? 0 : static_cast<int>((rows + kRows - 1) / kRows);
}
// Units of one key-value head of a request, summed by a warp.
template <int kRows, int kKeys>
__device__ __forceinline__ long long request_units(const Kv4AttnParams& p, const Kv4Request& r, int tiles) {
  long long sum = 0;
  for (int rt = threadIdx.x & 31; rt < tiles; rt += 32) sum += item_units<kRows, kKeys>(p, r, rt);
#pragma unroll
  for (int d = 16; d > 0; d >>= 1) sum += __shfl_xor_sync(0xffffffffu, sum, d);
  return sum;
}

// Units of one head of request b (zero where there is none) and its tiles, for the requests of a warp's lanes.
template <int kRows, int kKeys>
__device__ __forceinline__ long long units_of_lanes(const Kv4AttnParams& p, int b, int& tiles) {
  constexpr int kFew = 4;  // tiles that a lane goes through by itself
  Kv4Request r{0, 0, 0};
  tiles = 0;
  if (b < p.B) {
    r = kv4_request(p, b);
    tiles = request_tiles<kRows>(p, r);
  }
  long long per = 0;
  if (tiles <= kFew)
    for (int rt = 0; rt < tiles; ++rt) per += item_units<kRows, kKeys>(p, r, rt);
  for (unsigned many = __ballot_sync(0xffffffffu, tiles > kFew); many != 0; many &= many - 1) {
    const int j = __ffs(many) - 1;
    const Kv4Request x{__shfl_sync(0xffffffffu, r.first, j), __shfl_sync(0xffffffffu, r.n, j), __shfl_sync(0xffffffffu, r.ctx, j)};
    const long long sum = request_units<kRows, kKeys>(p, x, __shfl_sync(0xffffffffu, tiles, j));
    if ((threadIdx.x & 31) == j) per = sum;
  }
  return per;
}

// The first request from b on that has tiles; out of line, so that the roles' loops stay together (2048 tokens over 30 K: 1430 us with
// it in each role, 1340).
__device__ __noinline__ int next_tiled_request(const int32_t* query_start, const int32_t* context_len, int B, int T, int group, int min_rows,
                                               int max_rows, int b) {
  Kv4AttnParams p{};
  p.query_start = query_start;
  p.context_len = context_len;
  p.max_pages = 1;  // (lengths do not matter here)
  p.B = B;
  p.T = T;
  p.group = group;
  p.min_rows = min_rows;
  p.max_rows = max_rows;
  return next_request(p, b, [&](const Kv4Request& x) { return request_tiles<kTileRows>(p, x) > 0; });
}

// Where a role stands: every role walks through the CTA's run by itself.
template <int D, int kTiles, bool kTopk>
struct Walk {
  static constexpr int kRows = Cfg<D, kTiles>::kRows, kKeys = Cfg<D, kTiles>::kKeys;
  int b, kvh, rt, unit, units, tiles;
  long long left;
  Kv4Request r;
  __device__ __forceinline__ void open(const Kv4AttnParams& p, const Shared& sh) {
    b = sh.b;
    kvh = sh.kvh;
    rt = sh.rt;
    unit = sh.unit;
    left = sh.hi - sh.lo;
    if (left > 0) request(p);
  }
  __device__ __forceinline__ void request(const Kv4AttnParams& p) {
    if constexpr (kTopk) {
      tiles = (p.group + kRows - 1) / kRows;
      units = (p.topk + kKeys - 1) / kKeys;
      r = Kv4Request{b, 1, 0};
    } else {
      r = kv4_request(p, b);
      tiles = request_tiles<kRows>(p, r);
      units = tiles > 0 ? item_units<kRows, kKeys>(p, r, rt) : 0;
    }
  }
  // the item's units that are in the run: unit .. end() - 1
  __device__ __forceinline__ int end() const { return units - unit <= left ? units : static_cast<int>(unit + left); }
  __device__ __forceinline__ bool next(const Kv4AttnParams& p) {  // to the next item; false at the run's end
    left -= end() - unit;
    if (left <= 0) return false;
    unit = 0;
    if (++rt < tiles) {
      if constexpr (!kTopk) units = item_units<kRows, kKeys>(p, r, rt);
      return true;
    }
    rt = 0;
    if (++kvh < p.Hkv) {
      if constexpr (!kTopk) units = item_units<kRows, kKeys>(p, r, 0);
      return true;
    }
    kvh = 0;
    ++b;
    if constexpr (!kTopk) {
      b = next_tiled_request(p.query_start, p.context_len, p.B, p.T, p.group, p.min_rows, p.max_rows, b);
      if (b >= p.B) {
        left = 0;
        return false;
      }
    }
    request(p);
    return true;
  }
};

// A ring of barriers: the stage of the next use and its phase.
template <int kN>
struct Turn {
  int i = 0;
  uint32_t phase = 0;
  __device__ __forceinline__ void next() {
    if (++i == kN) {
      i = 0;
      phase ^= 1;
    }
  }
};

__device__ __forceinline__ void tmem_ld16(uint32_t taddr, uint32_t (&v)[16]) {
  asm volatile(
      "tcgen05.ld.sync.aligned.32x32b.x16.b32 {%0, %1, %2, %3, %4, %5, %6, %7, %8, %9, %10, %11, %12, %13, %14, %15}, [%16];"
      : "=r"(v[0]), "=r"(v[1]), "=r"(v[2]), "=r"(v[3]), "=r"(v[4]), "=r"(v[5]), "=r"(v[6]), "=r"(v[7]), "=r"(v[8]), "=r"(v[9]), "=r"(v[10]),
        "=r"(v[11]), "=r"(v[12]), "=r"(v[13]), "=r"(v[14]), "=r"(v[15])
      : "r"(taddr)
      : "memory");
}
// The wait names the registers, so that no use of them moves above it.
__device__ __forceinline__ void tmem_ld16_wait(uint32_t (&v)[16]) {
  asm volatile("tcgen05.wait::ld.sync.aligned;"
               : "+r"(v[0]), "+r"(v[1]), "+r"(v[2]), "+r"(v[3]), "+r"(v[4]), "+r"(v[5]), "+r"(v[6]), "+r"(v[7]), "+r"(v[8]), "+r"(v[9]),
                 "+r"(v[10]), "+r"(v[11]), "+r"(v[12]), "+r"(v[13]), "+r"(v[14]), "+r"(v[15])
               :
               : "memory");
}
__device__ __forceinline__ void tmem_st8(uint32_t taddr, const uint32_t (&v)[8]) {
  asm volatile("tcgen05.st.sync.aligned.32x32b.x8.b32 [%0], {%1, %2, %3, %4, %5, %6, %7, %8};" ::"r"(taddr), "r"(v[0]), "r"(v[1]), "r"(v[2]),
               "r"(v[3]), "r"(v[4]), "r"(v[5]), "r"(v[6]), "r"(v[7])
               : "memory");
}
__device__ __forceinline__ void tmem_st32(uint32_t taddr, const uint32_t (&v)[32]) {
  asm volatile(
      "tcgen05.st.sync.aligned.32x32b.x32.b32 [%0], {%1, %2, %3, %4, %5, %6, %7, %8, %9, %10, %11, %12, %13, %14, %15, %16, "
      "%17, %18, %19, %20, %21, %22, %23, %24, %25, %26, %27, %28, %29, %30, %31, %32};" ::"r"(taddr),
      "r"(v[0]), "r"(v[1]), "r"(v[2]), "r"(v[3]), "r"(v[4]), "r"(v[5]), "r"(v[6]), "r"(v[7]), "r"(v[8]), "r"(v[9]), "r"(v[10]), "r"(v[11]),
      "r"(v[12]), "r"(v[13]), "r"(v[14]), "r"(v[15]), "r"(v[16]), "r"(v[17]), "r"(v[18]), "r"(v[19]), "r"(v[20]), "r"(v[21]), "r"(v[22]),
      "r"(v[23]), "r"(v[24]), "r"(v[25]), "r"(v[26]), "r"(v[27]), "r"(v[28]), "r"(v[29]), "r"(v[30]), "r"(v[31])
      : "memory");
}
__device__ __forceinline__ unsigned long long pack2(float a, float b) {
  unsigned long long x;
  asm("mov.b64 %0, {%1, %2};" : "=l"(x) : "f"(a), "f"(b));
  return x;
}
__device__ __forceinline__ void unpack2(unsigned long long x, float& a, float& b) { asm("mov.b64 {%0, %1}, %2;" : "=f"(a), "=f"(b) : "l"(x)); }
__device__ __forceinline__ unsigned long long fma2(unsigned long long a, unsigned long long b, unsigned long long c) {
  unsigned long long d;
  asm("fma.rn.f32x2 %0, %1, %2, %3;" : "=l"(d) : "l"(a), "l"(b), "l"(c));
  return d;
}
__device__ __forceinline__ unsigned long long add2(unsigned long long a, unsigned long long b) {
  unsigned long long d;
  asm("add.rn.f32x2 %0, %1, %2;" : "=l"(d) : "l"(a), "l"(b));
  return d;
}
__device__ __forceinline__ void tmem_st_wait() { asm volatile("tcgen05.wait::st.sync.aligned;" ::: "memory"); }
// Bounded wait, as ptx::mbar_wait, of a role with nothing else to do: the warp is suspended for up to 20 us at a time.  (Ten warps of
// an SM polling at will took 40 % of its issue slots.)
__device__ __forceinline__ bool long_wait(uint32_t bar, uint32_t parity, volatile int* abort_flag) {
  uint64_t t0 = 0;
  while (true) {
    uint32_t done;
    asm volatile(
        "{\n"
        ".reg .pred p;\n"
        "mbarrier.try_wait.parity.shared::cta.b64 p, [%1], %2, %3;\n"
        "selp.u32 %0, 1, 0, p;\n"
        "}\n"
        : "=r"(done)
        : "r"(bar), "r"(parity), "r"(20000u)
        : "memory");
    if (done) return true;
    if (*abort_flag) return false;
    const uint64_t now = ptx::globaltimer_ns();
    if (t0 == 0) {
      t0 = now;
    } else if (now - t0 > static_cast<uint64_t>(static_cast<uint32_t>(abort_flag[1])) * 1000ull) {
      *abort_flag = 1;
      return false;
    }
  }
}

// Products and their signals are issued by one lane, the same every time, from code that all lanes run: operands then live in uniform
// registers.  (With one lane in a branch of its own each product cost some 110 clocks to issue.)
// D[tmem] (+)= A[smem] * B[smem]^T
__device__ __forceinline__ void mma_from_smem(uint32_t d_tmem, uint64_t a_desc, uint64_t b_desc, uint32_t idesc, uint32_t accumulate) {
  asm volatile(
      "{\n"
      ".reg .pred p, e;\n"
      "setp.ne.b32 p, %4, 0;\n"
      "elect.sync _|e, 0xffffffff;\n"
      "@e tcgen05.mma.cta_group::1.kind::f16 [%0], %1, %2, %3, p;\n"
      "}\n" ::"r"(d_tmem),
      "l"(a_desc), "l"(b_desc), "r"(idesc), "r"(accumulate)
      : "memory");
}
// D[tmem] (+)= A[tmem] * B[smem]^T
__device__ __forceinline__ void mma_from_tmem(uint32_t d_tmem, uint32_t a_tmem, uint64_t b_desc, uint32_t idesc, uint32_t accumulate) {
  asm volatile(
      "{\n"
      ".reg .pred p, e;\n"
      "setp.ne.b32 p, %4, 0;\n"
      "elect.sync _|e, 0xffffffff;\n"
      "@e tcgen05.mma.cta_group::1.kind::f16 [%0], [%1], %2, %3, p;\n"
      "}\n" ::"r"(d_tmem),
      "r"(a_tmem), "l"(b_desc), "r"(idesc), "r"(accumulate)
      : "memory");
}
__device__ __forceinline__ void commit(uint32_t bar) {
  asm volatile(
      "{\n"
      ".reg .pred e;\n"
      "elect.sync _|e, 0xffffffff;\n"
      "@e tcgen05.commit.cta_group::1.mbarrier::arrive::one.shared::cluster.b64 [%0];\n"
      "}\n" ::"r"(bar)
      : "memory");
}
// fp32 accumulator, both operands fp16 and K-major, M = 128
__host__ __device__ constexpr uint32_t f16_idesc(int n) {
  return (1u << 4) | (static_cast<uint32_t>(n >> 3) << 17) | (static_cast<uint32_t>(128 >> 4) << 24);
}

// Byte of 16-byte piece `piece` (of 8) of row `r` in a tile of 128-byte rows with the 128-byte swizzle.
__device__ __forceinline__ uint32_t swizzled(int r, int piece) { return static_cast<uint32_t>(r * 128 + ((piece ^ (r & 7)) << 4)); }
__device__ __forceinline__ void sts128(uint32_t at, uint32_t a, uint32_t b, uint32_t c, uint32_t d) {
  asm volatile("st.shared.v4.b32 [%0], {%1, %2, %3, %4};" ::"r"(at), "r"(a), "r"(b), "r"(c), "r"(d) : "memory");
}
// `bytes` (a multiple of 16, both addresses too) to shared memory; the barrier counts them.
__device__ __forceinline__ void bulk_load(uint32_t dst, const void* src, uint32_t bytes, uint32_t bar) {
  asm volatile("cp.async.bulk.shared::cluster.global.mbarrier::complete_tx::bytes [%0], [%1], %2, [%3];" ::"r"(dst), "l"(src), "r"(bytes), "r"(bar)
               : "memory");
}
// kBytes to shared memory, or as many zeros.
template <int kBytes>
__device__ __forceinline__ void cp_async_or_zero(uint32_t dst, const void* src, bool there) {
  const int n = there ? kBytes : 0;
  if constexpr (kBytes == 16)
    asm volatile("cp.async.cg.shared.global [%0], [%1], 16, %2;" ::"r"(dst), "l"(src), "r"(n) : "memory");
  else
    asm volatile("cp.async.ca.shared.global [%0], [%1], %3, %2;" ::"r"(dst), "l"(src), "r"(n), "n"(kBytes) : "memory");
}
// The barrier gets this thread's arrival once its cp.async copies so far are there.
__device__ __forceinline__ void cp_async_arrive(uint32_t bar) {
  asm volatile("cp.async.mbarrier.arrive.noinc.shared::cta.b64 [%0];" ::"r"(bar) : "memory");
}
__device__ __forceinline__ uint32_t lds32(uint32_t at) {
  uint32_t x;
  asm volatile("ld.shared.b32 %0, [%1];" : "=r"(x) : "r"(at) : "memory");
  return x;
}
__device__ __forceinline__ uint32_t lds16(uint32_t at) {
  unsigned short x;
  asm volatile("ld.shared.u16 %0, [%1];" : "=h"(x) : "r"(at) : "memory");
  return x;
}
// 16 bytes of a ring row: rows of 64-element heads are only 8-byte aligned.
template <int kRow>
__device__ __forceinline__ uint4 lds_codes(uint32_t at) {
  uint4 x;
  if constexpr (kRow % 16 == 0) {
    asm volatile("ld.shared.v4.b32 {%0, %1, %2, %3}, [%4];" : "=r"(x.x), "=r"(x.y), "=r"(x.z), "=r"(x.w) : "r"(at) : "memory");
  } else {
    asm volatile("ld.shared.v2.b32 {%0, %1}, [%2];" : "=r"(x.x), "=r"(x.y) : "r"(at) : "memory");
    asm volatile("ld.shared.v2.b32 {%0, %1}, [%2];" : "=r"(x.z), "=r"(x.w) : "r"(at + 8) : "memory");
  }
  return x;
}

// A warp's rows of O times a factor each.  (Out of line it cost 5 %.)
template <int D>
__device__ __forceinline__ void scale_rows(uint32_t t_o, float back) {
#pragma unroll 1
  for (int chunk = 0; chunk < D / 32; ++chunk) {
    uint32_t v[32];
    ptx::tmem_ld32(t_o + chunk * 32, v);
    ptx::tmem_ld_wait(v);
#pragma unroll
    for (int i = 0; i < 32; ++i) v[i] = __float_as_uint(__uint_as_float(v[i]) * back);
    tmem_st32(t_o + chunk * 32, v);
  }
}

// ---------------------------------------------------------------------------------------------
template <int D, int kTiles, bool kTopk>
__global__ void __launch_bounds__(Cfg<D, kTiles>::kThreads, Cfg<D, kTiles>::kCtasPerSm)
attention_tiles_kernel(const Kv4AttnParams p, const SplitBuffers sb) {
  using C = Cfg<D, kTiles>;
  extern __shared__ uint8_t smem_raw[];
  __shared__ Shared sh;
  // (from a shuffle: the roles' branches, and with them the products' operands, are then known to be the same for a whole warp)
  const int tid = threadIdx.x, lane = tid & 31, warp = __shfl_sync(0xffffffffu, tid >> 5, 0);
  const uint32_t base = (ptx::smem_u32(smem_raw) + 1023u) & ~1023u;
  const uint32_t s_q = base, s_k = s_q + kTiles * C::kQueryBytes, s_v = s_k + C::kStages * C::kTileBytes, s_ring = s_v + C::kStages * C::kTileBytes;
  auto bar = [&](uint64_t& b) { return ptx::smem_u32(&b); };
  constexpr int kKeys = C::kKeys;
  constexpr uint32_t kHalfQ = kTileRows * 128, kHalfK = kKeys * 128, kHalfV = D * 128;  // bytes of 64 elements of the rows
  constexpr int kUnpackers = 64;

  if (tid == 0) {
    for (int i = 0; i < C::kStages; ++i) {
      ptx::mbar_init(bar(sh.k_full[i]), kUnpackers);
      ptx::mbar_init(bar(sh.k_empty[i]), 1);
      ptx::mbar_init(bar(sh.v_full[i]), kUnpackers);
      ptx::mbar_init(bar(sh.v_empty[i]), 1);
    }
    for (int i = 0; i < 2; ++i) {
      for (int j = 0; j < 2; ++j) {
        ptx::mbar_init(bar(sh.s_full[i][j]), 1);
        ptx::mbar_init(bar(sh.p_full[i][j]), kTileRows);
        ptx::mbar_init(bar(sh.o_done[i][j]), 1);
      }
      ptx::mbar_init(bar(sh.q_full[i]), kTileRows);
    }
    for (int i = 0; i < C::kRing; ++i) {
      ptx::mbar_init(bar(sh.ring_full[i]), 32);
      ptx::mbar_init(bar(sh.ring_empty[i]), 2 * kUnpackers);
    }
    for (int i = 0; i < kSeenStages; ++i) {
      ptx::mbar_init(bar(sh.seen_full[i]), 1);
      ptx::mbar_init(bar(sh.seen_empty[i]), C::kRows);
    }
    sh.abort_flag[0] = 0;
    sh.abort_flag[1] = static_cast<int>(p.wait_limit_us);
    ptx::mbar_init(bar(sh.drained), 1);
    sh.drain_flag[0] = 0;
    sh.drain_flag[1] = 100000;
    sh.lo = sh.hi = 0;
    ptx::fence_mbar_init();
  }
  if (warp == C::kMmaWarp) {
    ptx::tmem_alloc(ptx::smem_u32(&sh.tmem), C::kTmemCols);
    ptx::tmem_relinquish();
  }
  __syncthreads();
  ptx::tc_fence_after();
  const uint32_t tmem = sh.tmem;
  volatile int* gave_up = sh.abort_flag;
  chain_wait();

  // ---- the CTA's run of all units, and where it begins ----------------------------------------------
  {
    auto cut = [&](long long total, long long& lo, long long& hi) {
      const long long even = quotient(total, gridDim.x);
      const unsigned rest = static_cast<unsigned>(total - even * gridDim.x);
      lo = even * blockIdx.x + rest * blockIdx.x / gridDim.x;
      hi = even * (blockIdx.x + 1) + rest * (blockIdx.x + 1) / gridDim.x;
    };
    if constexpr (kTopk) {
      if (tid == 0) {
        const Kv4Rows rows = kv4_rows(p);
        const int units = (p.topk + kKeys - 1) / kKeys, tiles = (p.group + C::kRows - 1) / C::kRows;
        const long long per = static_cast<long long>(units) * tiles * p.Hkv;
        long long lo, hi;
        cut(per * (rows.end - rows.first), lo, hi);
        sh.lo = lo;
        sh.hi = hi;
        if (lo < hi) {
          long long off = lo;
          const long long token = quotient(off, per);
          sh.b = rows.first + static_cast<int>(token);
          off -= per * token;
          const long long item = quotient(off, units);
          sh.unit = static_cast<int>(off - item * units);
          sh.kvh = static_cast<int>(quotient(item, tiles));
          sh.rt = static_cast<int>(item - static_cast<long long>(sh.kvh) * tiles);
        }
      }
    } else {
      // An item costs its units and, for its queries and results, as much as kItemCost more: runs are cut evenly in that measure.  (By units
      // alone a run of short items, a prompt's first chunk, took 1.7 times the average: a mixed batch 256 us instead of 176.)
      constexpr int kItemCost = 256 / kKeys;
      // the total: 32 requests per warp and turn; what a head of the first ones takes is kept, where the first keys will come
      static_assert(kKnown * 12 <= C::kStages * C::kTileBytes, "room for the known requests");
      long long* known_units = reinterpret_cast<long long*>(smem_raw + (s_k - ptx::smem_u32(smem_raw)));
      int* known_tiles = reinterpret_cast<int*>(known_units + kKnown);
      long long sum = 0;
      for (int b0 = warp * 32; b0 < p.B; b0 += C::kWarps * 32) {
        int tiles;
        const long long per = units_of_lanes<C::kRows, kKeys>(p, b0 + lane, tiles);
        if (b0 + lane < kKnown) {
          known_units[b0 + lane] = per;
          known_tiles[b0 + lane] = tiles;
        }
        sum += (per + tiles * kItemCost) * p.Hkv;
      }
#pragma unroll
      for (int d = 16; d > 0; d >>= 1) sum += __shfl_xor_sync(0xffffffffu, sum, d);
      if (lane == 0) sh.sums[warp] = sum;
      __syncthreads();
      if (warp < 2) {  // where the run begins, and where the next one does
        long long total = 0, lo, hi;
        for (int w = 0; w < C::kWarps; ++w) total += sh.sums[w];
        cut(total, lo, hi);
        const long long x = warp == 0 ? lo : hi;
        long long before = 0, units_before = 0, per = 0;
        int b = p.B, tiles = 0;
        for (int b0 = 0; b0 < p.B; b0 += 32) {
          int my_tiles;
          long long mine;
          if (b0 + 32 <= kKnown) {
            mine = known_units[b0 + lane];
            my_tiles = known_tiles[b0 + lane];
          } else {
            mine = units_of_lanes<C::kRows, kKeys>(p, b0 + lane, my_tiles);
          }
          const long long cost = (mine + my_tiles * kItemCost) * p.Hkv;
          long long costs = cost, units = mine * p.Hkv;  // up to and with this lane's
#pragma unroll 1
          for (int d = 1; d < 32; d <<= 1) {
            const long long c = __shfl_up_sync(0xffffffffu, costs, d), u = __shfl_up_sync(0xffffffffu, units, d);
            if (lane >= d) {
              costs += c;
              units += u;
            }
          }
          const unsigned beyond = __ballot_sync(0xffffffffu, x < before + costs);
          const int j = beyond != 0 ? __ffs(beyond) - 1 : 31;
          if (beyond != 0) {
            b = b0 + j;
            per = __shfl_sync(0xffffffffu, mine, j);
            tiles = __shfl_sync(0xffffffffu, my_tiles, j);
            before += __shfl_sync(0xffffffffu, costs - cost, j);
            units_before += __shfl_sync(0xffffffffu, units - mine * p.Hkv, j);
            break;
          }
          before += __shfl_sync(0xffffffffu, costs, j);
          units_before += __shfl_sync(0xffffffffu, units, j);
        }
        int kvh = 0, my_rt = 0, my_unit = 0;
        bool here = b == p.B && lane == 0;  // (the end of all runs)
        if (b < p.B) {
          const Kv4Request r = kv4_request(p, b);
          const long long head = per + tiles * kItemCost;
          kvh = static_cast<int>(quotient(x - before, head));
          units_before += per * kvh;
          const long long off = x - before - head * kvh;
          long long passed = 0;  // cost of the tiles before, 32 tiles at a look
          for (int rt0 = 0; rt0 < tiles; rt0 += 32) {
            const int rt = rt0 + lane, units = rt < tiles ? item_units<C::kRows, kKeys>(p, r, rt) : 0;
            const int mine = rt < tiles ? units + kItemCost : 0;
            int inc = mine;
#pragma unroll
            for (int d = 1; d < 32; d <<= 1) {
              const int v = __shfl_up_sync(0xffffffffu, inc, d);
              if (lane >= d) inc += v;
            }
            const long long first = passed + inc - mine;
            here = off >= first && off < first + mine;
            if (here) {
              my_rt = rt;
              my_unit = off - first > kItemCost ? static_cast<int>(off - first) - kItemCost : 0;
              units_before += first - static_cast<long long>(rt) * kItemCost + my_unit;
            }
            if (__any_sync(0xffffffffu, here)) break;
            passed += __shfl_sync(0xffffffffu, inc, 31);
          }
        }
        if (here) {
          if (warp == 0) {
            sh.lo = units_before;
            sh.b = b;
            sh.kvh = kvh;
            sh.rt = my_rt;
            sh.unit = my_unit;
          } else {
            sh.hi = units_before;
          }
        }
      }
    }
    __syncthreads();
  }
  Walk<D, kTiles, kTopk> at;
  at.open(p, sh);
  const bool any = sh.hi > sh.lo;
  if (tid == 0) {
    CtaDesc* desc = sb.desc + blockIdx.x;
    desc->part[0].flags = desc->part[1].flags = 0;
  }
  __syncthreads();

  if (warp < C::kSoftmaxWarps) {
    if (any) {
    // ---- softmax ---------------------------------------------------------------------------------------
    const int tt = warp >> 2, r128 = (warp & 3) * 32 + lane;
    const uint32_t lanes = static_cast<uint32_t>((warp & 3) * 32) << 16;
    const uint32_t t_s = tmem + lanes + tt * 128, t_o = tmem + lanes + kTiles * 128 + tt * 128;
    Turn<kSeenStages> seen;
    uint32_t s_phase[2] = {0, 0}, o_uses[2] = {0, 0};  // (o_uses: parity of the products that were asked for from a buffer)
    int buf = 0;
    bool more = true, ok = true;
    while (more) {
      // the row's query, its largest element in [2^15, 2^16), elements paired as the codes are
      const int rows = kTopk ? p.group : at.r.n * p.group, r0 = at.rt * C::kRows + tt * kTileRows, r = r0 + r128;
      int token = 0, head = 0;
      float worth = 1.f;
      // (a tile without rows takes no part; a warp without any keeps step and computes nothing)
      const bool tile_there = r0 < rows, warp_there = r0 + (warp & 3) * 32 < rows;
      if (tile_there) {
        const uint32_t to = s_q + tt * C::kQueryBytes;
        const uint4* src = nullptr;
        if (r < rows) {
          row_place(p, at.r.first, at.kvh, r, token, head);
          src = reinterpret_cast<const uint4*>(static_cast<const __nv_bfloat16*>(p.q) + token * p.q_stride + static_cast<long long>(head) * D);
        }
        uint32_t top = 0;
        if (src != nullptr) {
#pragma unroll 4
          for (int i = 0; i < D / 8; ++i) {
            const uint4 x = __ldg(src + i);
            const uint32_t w[4] = {x.x, x.y, x.z, x.w};
#pragma unroll
            for (int j = 0; j < 4; ++j) top = max(top, max(w[j] & 0x7fffu, (w[j] >> 16) & 0x7fffu));
          }
        }
        const int e = max(static_cast<int>(top >> 7), 21);
        const float up = copysignf(__uint_as_float(static_cast<uint32_t>(127 + 127 + 15 - e) << 23), p.scale);
        // (before it scores are under 2^37: 128 products of 2^16 and 2^14 at most)
        worth = worth_of(e, p.scale, 1.f, 0x1p89f);
#pragma unroll 4
        for (int i = 0; i < D / 8; ++i) {
          uint4 x = make_uint4(0, 0, 0, 0);
          if (src != nullptr) x = __ldg(src + i);
          const uint32_t w[4] = {x.x, x.y, x.z, x.w};
          float f[8];
#pragma unroll
          for (int j = 0; j < 4; ++j) {
            f[2 * j] = __uint_as_float(w[j] << 16) * up;
            f[2 * j + 1] = __uint_as_float(w[j] & 0xffff0000u) * up;
          }
          sts128(to + (i >> 3) * kHalfQ + swizzled(r128, i & 7), half2_bits(f[0], f[4]), half2_bits(f[1], f[5]), half2_bits(f[2], f[6]),
                 half2_bits(f[3], f[7]));
        }
        ptx::fence_proxy_async();
        ptx::tc_fence_before();  // (the item before has been read from tensor memory)
        ptx::mbar_arrive(bar(sh.q_full[tt]));
      }
      // how far the row, and the tile's first row, see (dense form)
      const long long limit = static_cast<long long>(at.r.ctx) + (r < rows ? r : rows - 1) / p.group;
      const long long least = static_cast<long long>(at.r.ctx) + (r0 < rows ? r0 : rows - 1) / p.group;
      float worth_bar = -INFINITY, shift = kNothing, l = 0.f;
      const int unit0 = at.unit, unit1 = at.end();
      for (int unit = unit0; unit < unit1 && ok; ++unit) {
        ok = long_wait(bar(sh.seen_full[seen.i]), seen.phase, gave_up);
        if (!__all_sync(0xffffffffu, ok)) {  // (a warp goes on, or gives up, as one)
          ok = false;
          break;
        }
        unsigned there[C::kChunks], all = 0xffffffffu;
#pragma unroll
        for (int i = 0; i < C::kChunks; ++i) {
          there[i] = sh.there[seen.i][i];
          all &= there[i];
        }
        ptx::mbar_arrive(bar(sh.seen_empty[seen.i]));
        seen.next();
        if (!tile_there) continue;
        const bool whole = all == 0xffffffffu && (kTopk || static_cast<long long>(unit) * kKeys + kKeys - 1 <= least);
        ok = long_wait(bar(sh.s_full[tt][buf]), s_phase[buf], gave_up);
        s_phase[buf] ^= 1;
        if (!__all_sync(0xffffffffu, ok)) {
          ok = false;
          break;
        }
        const uint32_t t_sb = t_s + buf * kKeys;
        if (!warp_there) {
          ptx::mbar_arrive(bar(sh.p_full[tt][buf]));
          if (C::kBufs == 1) ptx::mbar_arrive(bar(sh.p_full[tt][1]));
          o_uses[buf] ^= 1;
          if (C::kBufs == 2) buf ^= 1;
          continue;
        }
        ptx::tc_fence_after();
        // S is read twice, 32 columns at a time: short loops, and few registers
        auto hide = [&](uint32_t (&v)[16], int c16) {  // column 8 m + i is key 8 m + (m + i) % 8
          const long long left = limit - (static_cast<long long>(unit) * kKeys + c16 * 16);
          unsigned sees = there[0];
#pragma unroll
          for (int i = 1; i < C::kChunks; ++i) sees = c16 / 2 == i ? there[i] : sees;
          sees >>= (c16 & 1) * 16;
          if constexpr (!kTopk) sees = left >= 15 ? sees : left < 0 ? 0u : sees & (0xffffu >> (15 - static_cast<int>(left)));
#pragma unroll
          for (int i = 0; i < 16; ++i) {
            const int key = (i & 8) + ((c16 * 2 + (i >> 3) + i) & 7);
            if (!((sees >> key) & 1u)) v[i] = 0xff800000u;
          }
        };
        constexpr int kN = C::kKeys / 16;
        uint32_t x[16], y[16];
        float tops[2] = {-INFINITY, -INFINITY};
        auto raise = [&](const uint32_t (&v)[16]) {
#pragma unroll
          for (int i = 0; i < 16; i += 4) {
            tops[0] = fmaxf(fmaxf(__uint_as_float(v[i]), __uint_as_float(v[i + 1])), tops[0]);
            tops[1] = fmaxf(fmaxf(__uint_as_float(v[i + 2]), __uint_as_float(v[i + 3])), tops[1]);
          }
        };
        // (loops of their own for units that are seen whole: a test in the loop became selects that ran every time)
        auto first_reading = [&](auto whole_unit) {
          constexpr bool kWhole = decltype(whole_unit)::value;
#pragma unroll 1
          for (int c = 0; c < kN; c += 2) {
            tmem_ld16(t_sb + c * 16, x);
            tmem_ld16(t_sb + c * 16 + 16, y);
            tmem_ld16_wait(x);
            tmem_ld16_wait(y);
            if constexpr (!kWhole) hide(x, c);
            if constexpr (!kWhole) hide(y, c + 1);
            raise(x);
            raise(y);
          }
        };
        if (__builtin_expect(whole, 1))
          first_reading(std::true_type{});
        else
          first_reading(std::false_type{});
        const float top = fmaxf(tops[0], tops[1]);
        const bool grows = top > worth_bar;
        if (__builtin_expect(__any_sync(0xffffffffu, grows), 0)) {
          float back = 1.f;
          if (grows) {
            const float now = shift_of(top, worth);
            back = ex2(now - shift);
            worth_bar = bar_of(top, worth);
            shift = now;
            l *= back;
          }
          if (unit > unit0) {  // what there is of O, once the product before is through
            const int before = C::kBufs == 2 ? buf ^ 1 : 0;
            ok = long_wait(bar(sh.o_done[tt][before]), o_uses[before] ^ 1, gave_up);
            if (!__all_sync(0xffffffffu, ok)) {
              ok = false;
              break;
            }
            ptx::tc_fence_after();
            scale_rows<D>(t_o, back);
          }
        }
        // p = 2^(worth s + shift), two at a time where the pipes allow
        const unsigned long long worth2 = pack2(worth, worth), shift2 = pack2(shift, shift);
        unsigned long long sum = 0;
        auto exponentials = [&](const uint32_t (&v)[16], int c) {
          uint32_t h[8];
#pragma unroll
          for (int i = 0; i < 8; ++i) {
            const unsigned long long e = fma2(pack2(__uint_as_float(v[2 * i]), __uint_as_float(v[2 * i + 1])), worth2, shift2);
            float a, b;
            unpack2(e, a, b);
            a = ex2(a);
            b = ex2(b);
            sum = add2(sum, pack2(a, b));
            h[i] = half2_bits(a, b);
          }
          tmem_st8(t_sb + c * 8, h);
        };
        auto second_reading = [&](auto whole_unit) {
          constexpr bool kWhole = decltype(whole_unit)::value;
#pragma unroll 1
          for (int c = 0; c < kN; c += 2) {
            tmem_ld16(t_sb + c * 16, x);
            tmem_ld16(t_sb + c * 16 + 16, y);
            tmem_ld16_wait(x);
            tmem_ld16_wait(y);
            if constexpr (!kWhole) hide(x, c);
            if constexpr (!kWhole) hide(y, c + 1);
            exponentials(x, c);
            exponentials(y, c + 1);
            if ((c & 3) == 2) {  // 64 keys: their product may begin
              tmem_st_wait();
              ptx::tc_fence_before();
              ptx::mbar_arrive(bar(sh.p_full[tt][C::kBufs == 2 ? buf : c >> 2]));
            }
          }
        };
        if (__builtin_expect(whole, 1))
          second_reading(std::true_type{});
        else
          second_reading(std::false_type{});
        float sum0, sum1;
        unpack2(sum, sum0, sum1);
        l += sum0 + sum1;
        o_uses[buf] ^= 1;
        if (C::kBufs == 2) buf ^= 1;
      }
      if (!ok) break;
      // the item's end, or the run's
      if (tile_there)
        for (int i = 0; i < C::kBufs; ++i) ok = ok && long_wait(bar(sh.o_done[tt][i]), o_uses[i] ^ 1, gave_up);
      if (!__all_sync(0xffffffffu, ok)) {
        ok = false;
        break;
      }
      ptx::tc_fence_after();
      const bool begins = unit0 == 0, ends = unit1 == at.units;
      const float m = l > 0.f ? kPShift - shift : -INFINITY;
      float* part = sb.cta + (static_cast<long long>(blockIdx.x) * 2 + (begins ? 1 : 0)) * part_floats(C::kRows, D);
      const int n = tt * kTileRows + r128;
#pragma unroll 1
      for (int chunk = 0; warp_there && chunk < D / 32; ++chunk) {
        uint32_t v[32];
        ptx::tmem_ld32(t_o + chunk * 32, v);
        ptx::tmem_ld_wait(v);
        if (begins && ends) {
          if (r < rows) {
            const float inv = l > 0.f ? __fdividef(1.f, l) : 0.f;
            uint4* to = reinterpret_cast<uint4*>(static_cast<__nv_bfloat16*>(p.out) + (static_cast<long long>(token) * p.Hq + head) * D + chunk * 32);
#pragma unroll
            for (int i = 0; i < 4; ++i) {
              uint32_t h[4];
#pragma unroll
              for (int j = 0; j < 4; ++j)
                h[j] = bf162_bits(__uint_as_float(v[i * 8 + j * 2]) * inv, __uint_as_float(v[i * 8 + j * 2 + 1]) * inv);
              to[i] = make_uint4(h[0], h[1], h[2], h[3]);
            }
          }
        } else {
#pragma unroll
          for (int i = 0; i < 8; ++i)
            *reinterpret_cast<uint4*>(part + n * D + chunk * 32 + i * 4) = make_uint4(v[i * 4], v[i * 4 + 1], v[i * 4 + 2], v[i * 4 + 3]);
        }
      }
      if (begins && ends) {
        if (r < rows && p.lse != nullptr)
          p.lse[static_cast<long long>(token) * p.Hq + head] = l > 0.f ? (m - kPShift + log2f(l)) * kLn2 : -INFINITY;
      } else {
        if (warp_there) {
          part[C::kRows * D + n] = m;
          part[C::kRows * D + C::kRows + n] = l;
        }
        if (tid == 0)
          sb.desc[blockIdx.x].part[begins ? 1 : 0] = PartDesc{at.b, at.kvh, at.rt, kValid | (begins ? kBegins : 0) | (ends ? kEnds : 0)};
      }
      more = at.next(p);
    }
    }
  } else if (warp < C::kMmaWarp) {
    if (any && warp < C::kValueWarp) {
    // ---- keys: lane = group * 8 + x handles that group of 8 neighbouring keys; D = 64 has two groups, and half of the lanes take the
    // next eight ------------------------------------------------------------------------------------------
    constexpr int kGroups = D / kKvGroup, kOctets = 4 / kGroups;  // octets of keys a warp takes at once
    const int x = lane & 7, gi = (lane >> 3) % kGroups, o0 = (warp - C::kKeyWarp) * kOctets + (lane >> 3) / kGroups;
    const ValueConstants constants;
    Turn<C::kRing> ring;
    Turn<C::kStages> k;
    bool ok = true;
    for (long long left = sh.hi - sh.lo; left > 0 && ok; --left) {
      ok = long_wait(bar(sh.k_empty[k.i]), k.phase ^ 1, gave_up);
      const uint32_t to = s_k + k.i * C::kTileBytes + (gi >> 1) * kHalfK;
#pragma unroll 1
      for (int step = 0; step < kKeys / kStep && ok; ++step) {
        ok = long_wait(bar(sh.ring_full[ring.i]), ring.phase, gave_up);
#pragma unroll 1
        for (int o = o0; o < kStep / 8; o += 2 * kOctets) {
          const uint32_t from = s_ring + ring.i * C::kStepBytes + (o * 8 + x) * C::kRow;
          const int m = step * (kStep / 8) + o, c = m * 8 + ((x - m) & 7);  // column of key 8 m + x
          const uint4 codes = lds_codes<C::kRow>(from + gi * 16);
          const uint32_t scale = lds16(from + D + gi * 2), s2 = scale | (scale << 16), c2 = hfma2(s2, 0xCE00CE00u, 0u);  // -24 s
          const uint32_t w[4] = {codes.x, codes.y, codes.z, codes.w};
#pragma unroll
          for (int j = 0; j < 4; ++j)
            sts128(to + swizzled(c, (gi & 1) * 4 + j), f16_values<0>(w[j], s2, c2, constants), f16_values<1>(w[j], s2, c2, constants),
                   f16_values<2>(w[j], s2, c2, constants), f16_values<3>(w[j], s2, c2, constants));
        }
        ptx::mbar_arrive(bar(sh.ring_empty[ring.i]));
        ring.next();
      }
      ptx::fence_proxy_async();
      ptx::mbar_arrive(bar(sh.k_full[k.i]));
      k.next();
    }
    } else if (any) {
    // ---- values: a lane handles a code word of the 8 keys of a piece (4 pieces a step); of D = 128 each warp takes half of the words, of
    // D = 64 every other step -----------------------------------------------------------------------------
    const int v_warp = warp - C::kValueWarp, word = (lane >> 2) + (D == 128 ? v_warp * 8 : 0);
    const ValueConstants constants;
    Turn<C::kRing> ring;
    Turn<C::kStages> v;
    bool ok = true;
    for (long long left = sh.hi - sh.lo; left > 0 && ok; --left) {
      ok = long_wait(bar(sh.v_empty[v.i]), v.phase ^ 1, gave_up);
#pragma unroll 1
      for (int step = 0; step < kKeys / kStep && ok; ++step) {
        ok = long_wait(bar(sh.ring_full[ring.i]), ring.phase, gave_up);
        if (D == 128 || (step & 1) == v_warp) {
          const int m = step * (kStep / 8) + (lane & 3);
          const uint32_t from = s_ring + ring.i * C::kStepBytes + (lane & 3) * 8 * C::kRow;
          uint32_t lo16[4], hi16[4], s2[4], c2[4];
#pragma unroll
          for (int q = 0; q < 4; ++q) {  // columns 2 q and 2 q + 1 of the piece
            const uint32_t r0 = from + ((m + 2 * q) & 7) * C::kRow, r1 = from + ((m + 2 * q + 1) & 7) * C::kRow;
            const uint32_t a = lds32(r0 + D / 2 + word * 4), b = lds32(r1 + D / 2 + word * 4);
            s2[q] = lds16(r0 + D + D / 16 + (word >> 2) * 2) | (lds16(r1 + D + D / 16 + (word >> 2) * 2) << 16);
            c2[q] = hfma2(s2[q], 0xCE00CE00u, 0u);
            lo16[q] = __byte_perm(a, b, 0x5410);
            hi16[q] = __byte_perm(a, b, 0x7632);
          }
          const uint32_t to = s_v + v.i * C::kTileBytes + (m >> 3) * kHalfV + word * 8 * 128;
          auto put = [&](auto e) {
            constexpr int kE = decltype(e)::value;
            const uint32_t(&src)[4] = kE < 4 ? lo16 : hi16;
            sts128(to + swizzled(kE, m & 7), f16_values<kE % 4>(src[0], s2[0], c2[0], constants),
                   f16_values<kE % 4>(src[1], s2[1], c2[1], constants), f16_values<kE % 4>(src[2], s2[2], c2[2], constants),
                   f16_values<kE % 4>(src[3], s2[3], c2[3], constants));
          };
          put(std::integral_constant<int, 0>{});
          put(std::integral_constant<int, 1>{});
          put(std::integral_constant<int, 2>{});
          put(std::integral_constant<int, 3>{});
          put(std::integral_constant<int, 4>{});
          put(std::integral_constant<int, 5>{});
          put(std::integral_constant<int, 6>{});
          put(std::integral_constant<int, 7>{});
        }
        ptx::mbar_arrive(bar(sh.ring_empty[ring.i]));
        ring.next();
      }
      ptx::fence_proxy_async();
      ptx::mbar_arrive(bar(sh.v_full[v.i]));
      v.next();
    }
    }
  } else {
    if (any && warp == C::kRowWarp) {
    // ---- rows: a lane has a key of each step; the next tile's positions and pages are looked up while this one's are copied -----------
    Turn<C::kRing> ring;
    Turn<kSeenStages> seen;
    int req_b = -1;
    long long last = 0;  // the last position that any row of the item sees
    const int32_t* table = p.page_table;
    auto item = [&]() {
      Kv4Request r = at.r;
      int b = at.b;
      if constexpr (kTopk) {
        b = req_b = req_b < 0 ? request_of_row(p, at.b) : request_of_row_from(p, req_b, at.b);
        r = kv4_request(p, b);
        last = static_cast<long long>(r.ctx) + (at.b - r.first);
      } else {
        const long long rows = static_cast<long long>(r.n) * p.group, end = static_cast<long long>(at.rt + 1) * C::kRows;
        last = r.ctx + ((end < rows ? end : rows) - 1) / p.group;
      }
      table = p.page_table + static_cast<long long>(b) * p.max_pages;
    };
    constexpr int kSteps = kKeys / kStep;
    int page[kSteps], in_page[kSteps], kvh = 0;
    int idx[kSteps];  // the indexer's positions of the unit whose pages are looked up next
    Walk<D, kTiles, kTopk> idx_at = at;
    long long idx_left = sh.hi - sh.lo;
    auto load_indices = [&]() {
#pragma unroll
      for (int i = 0; i < kSteps; ++i) idx[i] = -1;
      if (kTopk && idx_left > 0) {
#pragma unroll
        for (int i = 0; i < kSteps; ++i) {
          const int x = idx_at.unit * kKeys + i * kStep + lane;
          if (x < p.topk) idx[i] = p.idx[static_cast<long long>(idx_at.b) * p.topk + x];
        }
        if (--idx_left > 0 && ++idx_at.unit == idx_at.units) {
          idx_at.left = idx_left + 1;  // (Walk counts the units from where it stands)
          idx_at.unit = idx_at.units - 1;
          idx_at.next(p);
        }
      }
    };
    auto look_up = [&](int unit) {  // page numbers (loads under way), and the rows within the pages
      kvh = at.kvh;
#pragma unroll
      for (int i = 0; i < kSteps; ++i) {
        // (units end at the table's reach, under 2^31 positions)
        const int pos = kTopk ? idx[i] : static_cast<int>(static_cast<long long>(unit) * kKeys + i * kStep + lane);
        page[i] = pos >= 0 && pos <= last && pos / kPageKeys < p.max_pages ? table[pos / kPageKeys] : -1;
        in_page[i] = pos & (kPageKeys - 1);
      }
      load_indices();
    };
    const long long page_bytes = static_cast<long long>(p.Hkv) * kPageKeys * C::kRow;
    item();
    int unit = at.unit, end = at.end(), issued = 0;
    load_indices();
    look_up(unit);
    bool ok = true;
    for (long long left = sh.hi - sh.lo; left > 0 && ok; --left) {
      const uint8_t* row[kSteps];
      unsigned there[kSteps];
#pragma unroll
      for (int i = 0; i < kSteps; ++i) {
        const bool sees = page[i] >= 0 && page[i] < p.pool_pages;
        there[i] = __ballot_sync(0xffffffffu, sees);
        row[i] = sees ? p.pool + page[i] * page_bytes + (kvh * kPageKeys + in_page[i]) * C::kRow : nullptr;
      }
      if (left > 1) {
        if (++unit == end) {
          at.next(p);
          item();
          unit = at.unit;
          end = at.end();
        }
        look_up(unit);
      }
      ok = long_wait(bar(sh.seen_empty[seen.i]), seen.phase ^ 1, gave_up);
      if (lane == 0 && ok) {
#pragma unroll
        for (int i = 0; i < kSteps; ++i) sh.there[seen.i][i] = there[i];
        ptx::mbar_arrive(bar(sh.seen_full[seen.i]));
      }
      seen.next();
#pragma unroll
      for (int i = 0; i < kSteps; ++i) {
        ok = ok && long_wait(bar(sh.ring_empty[ring.i]), ring.phase ^ 1, gave_up);
        if (!__all_sync(0xffffffffu, ok)) {
          ok = false;
          break;
        }
        const uint32_t to = s_ring + ring.i * C::kStepBytes, full = bar(sh.ring_full[ring.i]);
        if (!kTopk && there[i] == 0xffffffffu) {  // half a page in one piece
          if (lane == 0) {
            ptx::mbar_arrive_expect_tx(full, C::kStepBytes);
            bulk_load(to, row[i], C::kStepBytes, full);
          } else {
            ptx::mbar_arrive(full);
          }
        } else {
          // 9 pieces a row, neighbouring lanes on neighbouring pieces; rows that are not there become codes and scales of zero.  (A bulk copy
          // per row, issued lane by lane, took 80 clocks each: 1024 x 2048 positions 355 us)
          constexpr int kPiece = C::kRow / 9;
#pragma unroll
          for (int j = 0; j < 9; ++j) {
            const int n = j * 32 + lane, key = n / 9, piece = n - key * 9;
            const uint8_t* src = reinterpret_cast<const uint8_t*>(__shfl_sync(0xffffffffu, reinterpret_cast<unsigned long long>(row[i]), key));
            cp_async_or_zero<kPiece>(to + n * kPiece, src != nullptr ? src + piece * kPiece : p.pool, src != nullptr);
          }
          cp_async_arrive(full);
        }
        ring.next();
        ++issued;
      }
    }
    // no copy is under way when the CTA ends, also where a role gave up
    for (int i = 0; i < C::kRing; ++i) {
      const int n = (issued - i + C::kRing - 1) / C::kRing;  // uses of stage i
      if (issued > i) long_wait(bar(sh.ring_full[i]), static_cast<uint32_t>((n - 1) & 1), sh.drain_flag);
    }
    } else if (any && warp == C::kMmaWarp) {
    // ---- products --------------------------------------------------------------------------------------
    {
      Turn<C::kStages> k, v;
      uint32_t q_phase[2] = {0, 0}, o_phase[2][2] = {{0, 0}, {0, 0}}, p_phase[2][2] = {{0, 0}, {0, 0}};
      auto wait = [&](uint64_t& b, uint32_t phase) { return __all_sync(0xffffffffu, long_wait(bar(b), phase, gave_up)) != 0; };
      auto scores = [&](int tt, int buf) {
#pragma unroll
        for (int s = 0; s < D / 16; ++s)
          mma_from_smem(tmem + tt * 128 + buf * kKeys, ptx::make_smem_desc_sw128(s_q + tt * C::kQueryBytes + (s >> 2) * kHalfQ + (s & 3) * 32),
                        ptx::make_smem_desc_sw128(s_k + k.i * C::kTileBytes + (s >> 2) * kHalfK + (s & 3) * 32), f16_idesc(kKeys), s > 0);
        commit(bar(sh.s_full[tt][buf]));
      };
      auto values = [&](int tt, int col, int half, bool more) {  // 64 keys
#pragma unroll
        for (int s = 0; s < 4; ++s)
          mma_from_tmem(tmem + kTiles * 128 + tt * 128, tmem + tt * 128 + col + s * 8,
                        ptx::make_smem_desc_sw128(s_v + v.i * C::kTileBytes + half * kHalfV + s * 32), f16_idesc(D), more || s > 0);
      };
      bool more = true, ok = true;
      int buf = 0;
      while (more && ok) {
        const int n = at.end() - at.unit;
        // (a second tile without rows is left out)
        const int nt = kTiles == 2 && !kTopk && static_cast<long long>(at.r.n) * p.group <= at.rt * C::kRows + kTileRows ? 1 : kTiles;
        for (int tt = 0; tt < nt; ++tt) {
          ok = ok && wait(sh.q_full[tt], q_phase[tt]);
          q_phase[tt] ^= 1;
        }
        if constexpr (kTiles == 2) {
          ok = ok && wait(sh.k_full[k.i], k.phase);
          if (!ok) break;
          ptx::tc_fence_after();
          for (int tt = 0; tt < nt; ++tt) scores(tt, 0);
          commit(bar(sh.k_empty[k.i]));
          k.next();
          for (int j = 0; j < n && ok; ++j) {
            const bool ahead = j + 1 < n;
            ok = wait(sh.v_full[v.i], v.phase);
            for (int tt = 0; tt < nt && ok; ++tt) {
              for (int half = 0; half < 2 && ok; ++half) {
                ok = wait(sh.p_full[tt][half], p_phase[tt][half]);
                p_phase[tt][half] ^= 1;
                if (!ok) break;
                ptx::tc_fence_after();
                values(tt, half * 32, half, j > 0 || half > 0);
              }
              if (!ok) break;
              commit(bar(sh.o_done[tt][0]));
              // (before the wait for the next keys: unpacking them takes the ring along, and with it the next values)
              if (tt == nt - 1) commit(bar(sh.v_empty[v.i]));
              if (ahead) {  // S lies where P does: P has to be read first
                if (tt == 0) ok = wait(sh.k_full[k.i], k.phase);
                ok = ok && wait(sh.o_done[tt][0], o_phase[tt][0]);
                if (!ok) break;
                ptx::tc_fence_after();
                scores(tt, 0);
              }
              o_phase[tt][0] ^= 1;
            }
            if (!ok) break;
            v.next();
            if (ahead) {
              commit(bar(sh.k_empty[k.i]));
              k.next();
            }
          }
        } else {
          for (int j = 0; j < n + 2 && ok; ++j) {  // scores of unit j, product with the values of unit j - 2; both have the same buffer
            if (j >= 2) {
              ok = wait(sh.v_full[v.i], v.phase) && wait(sh.p_full[0][buf], p_phase[0][buf]);
              p_phase[0][buf] ^= 1;
              if (!ok) break;
              ptx::tc_fence_after();
              values(0, buf * kKeys, 0, j > 2);
              commit(bar(sh.o_done[0][buf]));
              commit(bar(sh.v_empty[v.i]));  // (before the wait for the next keys, as above)
              v.next();
            }
            if (j < n) {
              ok = wait(sh.k_full[k.i], k.phase);
              if (j >= 2) ok = ok && wait(sh.o_done[0][buf], o_phase[0][buf]);
              if (!ok) break;
              ptx::tc_fence_after();
              scores(0, buf);
              commit(bar(sh.k_empty[k.i]));
              k.next();
            }
            if (j >= 2) o_phase[0][buf] ^= 1;
            buf ^= 1;
          }
          // (two turns more than units: buf is the next unit's)
        }
        more = ok && at.next(p);
      }
    }
    }
  }

  __syncthreads();
  if (warp == C::kMmaWarp) {
    // every product and every signal of theirs is through before the memory goes, also where a role gave up
    commit(bar(sh.drained));
    long_wait(bar(sh.drained), 0, sh.drain_flag);
    __syncwarp();
    ptx::tmem_dealloc(tmem, C::kTmemCols);
  }
  if (tid == 0) sb.desc[blockIdx.x].status = sh.abort_flag[0] ? LT_STATUS_TIMEOUT : 0;
}

template <int D, int kTiles, bool kTopk>
cudaError_t launch_tiles(const Kv4AttnParams& p, void* scratch, Control* ctl, int sms, bool keep_status, cudaStream_t stream) {
  using C = Cfg<D, kTiles>;
  static std::atomic<unsigned long long> allowed{0};
  const cudaError_t e = allow_smem(reinterpret_cast<const void*>(attention_tiles_kernel<D, kTiles, kTopk>), allowed);
  if (e != cudaSuccess) return e;
  const int grid = sms * C::kCtasPerSm;
  SplitBuffers sb;
  sb.cta = static_cast<float*>(scratch);
  sb.warp = nullptr;
  sb.desc = reinterpret_cast<CtaDesc*>(sb.cta + static_cast<size_t>(grid) * 2 * part_floats(C::kRows, D));
  sb.ctl = ctl;
  const cudaError_t r = launch_chained(attention_tiles_kernel<D, kTiles, kTopk>, dim3(grid), dim3(C::kThreads), C::kSmem, stream, 1, p, sb);
  if (r != cudaSuccess) return r;
  return launch_join<D, C::kRows, kTopk>(p, sb, grid, keep_status, stream);
}

}  // namespace

// 256 rows and 128 rows twice as often take the same
size_t kv4_tiles_scratch_bytes(int D) {
  return static_cast<size_t>(sm_count()) * 2 * (sizeof(CtaDesc) + 2 * part_floats(kTileRows, D) * sizeof(float));
}

cudaError_t launch_kv4_attention_tiles(int D, bool pairs, const Kv4AttnParams& p, void* scratch, Control* ctl, int sms, bool keep_status,
                                       cudaStream_t stream) {
  if (p.idx != nullptr)
    return D == 64 ? launch_tiles<64, 1, true>(p, scratch, ctl, sms, keep_status, stream)
                   : launch_tiles<128, 1, true>(p, scratch, ctl, sms, keep_status, stream);
  if (pairs)
    return D == 64 ? launch_tiles<64, 2, false>(p, scratch, ctl, sms, keep_status, stream)
                   : launch_tiles<128, 2, false>(p, scratch, ctl, sms, keep_status, stream);
  return D == 64 ? launch_tiles<64, 1, false>(p, scratch, ctl, sms, keep_status, stream)
                 : launch_tiles<128, 1, false>(p, scratch, ctl, sms, keep_status, stream);
}

}  // namespace lt
