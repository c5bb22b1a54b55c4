// Attention over the 4-bit paged cache for many queries of a sequence (prompts and their chunks; see attend.cu for the formula).
//
// Rows are queries times the heads of a group, 256 to an item as two tiles of 128; keys come in tiles of 128.  Roles of the warps:
//   loader     copies units of 16 cached tokens into a ring of key and value stages
//   decoders   codes -> fp16 tiles in shared memory in the layout of the matrix instruction, values transposed
//   issuer     tcgen05.mma: S = Q K^T into tensor memory, O += P V with P read from tensor memory
//   softmax    a warpgroup for each row tile, a thread for each row: S -> P in place, running maximum and sum
// While one row tile's weights are made the tensor cores work on the other.  Maxima are raised only when they have grown by
// more than 8 (in powers of 2), so that O is seldom touched between products.  The order of a sum over d is free: K and Q are stored
// as the pairs (n, n + 4) in which codes are decoded, V's rows in the order that stores them without bank conflicts.
// The tiles of all items are dealt to the CTAs in equal runs; items that were cut are joined by the CTA that arrives last, those
// of many parts in groups first.
//
// What bounds it: a step of 256 rows and 128 keys takes 2900 to 3600 clocks.  Its products alone, with the operands as they lie, take
// 2460 (2048 at the nominal rate; Q K^T with both operands in shared memory reads 128 bytes a clock, all that there is), its
// exponentials 2048 on the special-function units, and the softmax and decoding instructions 1400 of a scheduler's slots.  Two
// chunks of 2048 queries over 6144 tokens, 64 heads of 128: 504 us, 989 TFLOP/s, of which the row tiles' starts and ends are
// about 70 us.  Left out because they were slower (2 x 32768 tokens, 256 queries each, 339 us now): a quarter of the
// exponentials as polynomials on the FMA pipe 408 against 369, two threads to a row 436 against 369.
#include "attend_common.cuh"
#include "mma_warp.cuh"

namespace tempo {

namespace {

constexpr int kThreads = 512;                         // four warpgroups: loader, issuer and decoders; decoders; softmax; softmax
constexpr int kKeys = 128, kRowTile = 128, kRows = 2 * kRowTile;
static_assert(kRows == kAttendManyRows, "the workspace is sized for it");
constexpr int kDecoders = 6;                          // warps 2 to 7

template <int D>
struct ManySmem {
  static constexpr int kTileBytes = kKeys * D * 2;                       // fp16 keys, values, or one row tile of queries
  static constexpr int kStageBytes = kKeys / kUnit * CacheUnit<D>::kBytes;
  static constexpr int kStages = 3;
  static constexpr int kQ = 0, kK = 2 * kTileBytes, kV = 4 * kTileBytes, kCodes = 6 * kTileBytes;
  static constexpr int kBefore = kCodes + kStages * kStageBytes;
  static int bytes(int B) { return kBefore + (B + 1) * 4 + 1024; }       // the tiles start on 1024 bytes
  static_assert(kBefore + (kAttendMaxB + 1) * 4 + 1024 + 512 <= 227 * 1024, "shared memory of one SM");
};

struct Bars {
  uint64_t code_full[3], code_empty[3], k_full[2], k_empty[2], v_full[2], v_empty[2];
  uint64_t s_full[2], p_ready[2][2], q_full[2], o_done[2], o_free[2];   // of each row tile (P in two halves of 64 keys)
  uint64_t joined;                                                      // all softmax warps
};

// A CTA's run as pieces of items, the same in every role.
template <class Tiles>
struct Pieces {
  using Item = typename Tiles::Item;
  Item it;
  int x, end;
  bool first;
  const int* before;
  __device__ __forceinline__ Pieces(const Item& it_, int begin, int end_, const int* before_)
      : it(it_), x(begin), end(end_), first(true), before(before_) {}
  __device__ __forceinline__ bool next(const AttendParams& p) {
    if (!first) {
      x = it.begin + it.tiles;
      if (x < end) Tiles::next_item(p, before, it);
    }
    first = false;
    return x < end;
  }
  __device__ __forceinline__ int tile0() const { return x - it.begin; }
  __device__ __forceinline__ int steps() const { return min(it.begin + it.tiles, end) - x; }
  __device__ __forceinline__ bool two(int group) const { return it.n * group - it.row0 > kRowTile; }
};

constexpr int kLeast = 4, kSnap = 3;

// Where run r begins, and in which item: its equal share of the tiles, or the border of an item that is near.  So an item [b, e) is cut
// at the equal shares in (b + kSnap, e - kSnap), and nowhere else.
template <class Tiles>
__device__ __forceinline__ int snapped(const AttendParams& p, const int* before, const Runs& runs, int r, int n_runs, int total, typename Tiles::Item& it) {
  const int x = r >= n_runs ? total : runs.begin(r);
  if (x == total) return total;
  it = Tiles::item_at(p, before, x);
  if (x - it.begin <= kSnap) return it.begin;
  if (it.begin + it.tiles - x > kSnap) return x;
  if (it.begin + it.tiles < total) Tiles::next_item(p, before, it);
  else it.begin += it.tiles;
  return it.begin;
}

// Instruction descriptor of kind::f16 with fp16 operands (0 at bits 7 and 10), 32-bit sums, both K-major, 128 rows, N columns.
template <int N>
constexpr uint32_t kIdesc = (1u << 4) | (static_cast<uint32_t>(N >> 3) << 17) | (static_cast<uint32_t>(kRowTile >> 4) << 24);

__device__ __forceinline__ void mma_ss(uint32_t leader, uint32_t d, uint32_t a_lo, uint32_t b_lo, uint32_t idesc, uint32_t accumulate) {
  warp_mma_bf16(leader, d, a_lo, b_lo, idesc, accumulate);               // kind::f16: the types are the descriptor's
}
// A from tensor memory.
__device__ __forceinline__ void mma_ts(uint32_t leader, uint32_t d, uint32_t a, uint32_t b_lo, uint32_t idesc, uint32_t accumulate) {
  asm volatile(
      "{\n\t.reg .pred p, l;\n\t.reg .b64 db;\n\t"
      "setp.ne.b32 p, %4, 0;\n\tsetp.ne.b32 l, %6, 0;\n\t"
      "mov.b64 db, {%2, %5};\n\t"
      "@l tcgen05.mma.cta_group::1.kind::f16 [%0], [%1], db, %3, p;\n\t}"
      ::"r"(d), "r"(a), "r"(b_lo), "r"(idesc), "r"(accumulate), "r"(kDescHi), "r"(leader) : "memory");
}
__device__ __forceinline__ void tmem_st32(uint32_t taddr, const uint32_t (&r)[32]) {
  asm volatile(
      "tcgen05.st.sync.aligned.32x32b.x32.b32 [%0], "
      "{%1, %2, %3, %4, %5, %6, %7, %8, %9, %10, %11, %12, %13, %14, %15, %16, "
      "%17, %18, %19, %20, %21, %22, %23, %24, %25, %26, %27, %28, %29, %30, %31, %32};"
      ::"r"(taddr), "r"(r[0]), "r"(r[1]), "r"(r[2]), "r"(r[3]), "r"(r[4]), "r"(r[5]), "r"(r[6]), "r"(r[7]),
        "r"(r[8]), "r"(r[9]), "r"(r[10]), "r"(r[11]), "r"(r[12]), "r"(r[13]), "r"(r[14]), "r"(r[15]),
        "r"(r[16]), "r"(r[17]), "r"(r[18]), "r"(r[19]), "r"(r[20]), "r"(r[21]), "r"(r[22]), "r"(r[23]),
        "r"(r[24]), "r"(r[25]), "r"(r[26]), "r"(r[27]), "r"(r[28]), "r"(r[29]), "r"(r[30]), "r"(r[31])
      : "memory");
}
__device__ __forceinline__ void tmem_st1(uint32_t taddr, uint32_t v) {
  asm volatile("tcgen05.st.sync.aligned.32x32b.x1.b32 [%0], {%1};" ::"r"(taddr), "r"(v) : "memory");
}
__device__ __forceinline__ void tmem_wait_st() { asm volatile("tcgen05.wait::st.sync.aligned;" ::: "memory"); }

__device__ __forceinline__ float max3(float a, float b, float c) {
  float r;
  asm("max.f32 %0, %1, %2, %3;" : "=f"(r) : "f"(a), "f"(b), "f"(c));
  return r;
}
// (a, b) * f + (m, m)
__device__ __forceinline__ void fma_pair(float& a, float& b, float f, float m) {
  asm("{\n\t.reg .b64 x, y, z;\n\tmov.b64 x, {%0, %1};\n\tmov.b64 y, {%2, %2};\n\tmov.b64 z, {%3, %3};\n\t"
      "fma.rn.f32x2 x, x, y, z;\n\tmov.b64 {%0, %1}, x;\n\t}" : "+f"(a), "+f"(b) : "f"(f), "f"(m));
}
__device__ __forceinline__ void add_pair(float& a, float& b, float c, float d) {
  asm("{\n\t.reg .b64 x, y;\n\tmov.b64 x, {%0, %1};\n\tmov.b64 y, {%2, %3};\n\t"
      "add.rn.f32x2 x, x, y;\n\tmov.b64 {%0, %1}, x;\n\t}" : "+f"(a), "+f"(b) : "f"(c), "f"(d));
}

// Row `row` of a K-major tile in the 128-byte swizzle: blocks of 64 numbers, each of `rows` rows of 128 bytes.
__device__ __forceinline__ uint32_t chunk_at(uint32_t base, int rows, int row, int block, int chunk) {
  return base + block * rows * 128 + row * 128 + ((chunk ^ (row & 7)) << 4);
}

// ---- decoders -----------------------------------------------------------------------------------------
// Keys of one stage.  A lane takes 32 neighbouring elements of a key: one group, four words, four 16-byte stores.
template <int D>
__device__ __forceinline__ void decode_keys(const Decode& dc, const uint8_t* stage, uint8_t* tile, uint32_t absent, int warp) {
  using U = CacheUnit<D>;
  constexpr int kParts = D / 32, kPer = 32 / kParts;                     // lanes to a key, keys to a warp
  const int lane = threadIdx.x & 31, j = lane % kParts, at = lane / kParts;
  // Key task * kPer + at is in row at % 8 of its eight whatever the task: the swizzle is the lane's own.  The second block's lanes
  // store in another order, so that no bank is met twice.
  const bool turn = D == 128 && (j & 2) != 0;
  uint8_t* to[4];
#pragma unroll
  for (int i = 0; i < 4; ++i)
    to[i] = tile + j / 2 * kKeys * 128 + at * 128 + (((4 * (j & 1) + (turn ? i ^ 2 : i)) ^ (at & 7)) << 4);
#pragma unroll 1
  for (int task = warp; task < kKeys / kPer; task += kDecoders) {
    const int key = task * kPer + at;
    const uint8_t* unit = stage + key / kUnit * U::kBytes;
    const uint4 u = *reinterpret_cast<const uint4*>(unit + key % kUnit * U::kKeyRow + j * 16);
    uint32_t params = *reinterpret_cast<const uint16_t*>(unit + U::kCodes + key % kUnit * U::kKeyParams + j * 2) * 0x10001u;
    if (absent != 0 && (absent >> (key / kUnit) & 1)) params |= kMarked * 0x10001u;
    uint32_t s, b;
    group_params(params, s, b);
    const uint32_t w[4] = {turn ? u.z : u.x, turn ? u.w : u.y, turn ? u.x : u.z, turn ? u.y : u.w};
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      uint32_t v[4];
      decode8(dc, w[i], s, b, v);
      *reinterpret_cast<uint4*>(to[i] + task * (kPer * 128)) = make_uint4(v[0], v[1], v[2], v[3]);
    }
  }
}

// Values of one stage, transposed: a lane takes two words (8 elements) of four pairs of tokens and stores, for each element, its
// eight tokens.  Element 8 x + 4 e + n is row 64 (x / 8) + 8 (4 e + n) + x % 8 of the tile: no bank twice in a store, and 64
// neighbouring rows are 64 neighbouring elements.  `left`: tokens that exist from the tile's first on; `edge`: some row does not see all.
template <int D>
__device__ __forceinline__ void decode_values(const Decode& dc, uint8_t* stage, uint8_t* tile, int left, bool edge, int warp) {
  using U = CacheUnit<D>;
  constexpr int kX = D / 8, kPer = 32 / kX;                              // lanes to eight tokens, eights of tokens to a warp
  const int lane = threadIdx.x & 31, x = lane % kX;
#pragma unroll 1
  for (int task = warp; task < kKeys / 8 / kPer; task += kDecoders) {
    const int eight = task * kPer + lane / kX;
    const uint8_t* unit = stage + eight / 2 * U::kBytes + (eight & 1) * 4 * U::kPairRow + x * 8;
    uint8_t* eight_params = stage + eight / 2 * U::kBytes + U::kCodes + (eight & 1) * 4 * U::kPairParams;
    const uint8_t* unit_params = eight_params + x / 4 * 4;
    if (edge) {                                                          // a word of byte pairs to each lane, which all read
      uint32_t* w = reinterpret_cast<uint32_t*>(eight_params) + x;
      *w = edge_params(*w, left - (8 * eight + 2 * (x / (D / 32))));
      __syncwarp();
    }
    uint32_t v[4][2][4];
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      const uint2 w = *reinterpret_cast<const uint2*>(unit + i * U::kPairRow);
      uint32_t s, b;
      group_params(*reinterpret_cast<const uint32_t*>(unit_params + i * U::kPairParams), s, b);
      decode8(dc, w.x, s, b, v[i][0]);
      decode8(dc, w.y, s, b, v[i][1]);
    }
    uint8_t* to = tile + eight / 8 * D * 128 + (x / 8 * 64 + x % 8) * 128 + (((eight ^ x) & 7) << 4);
#pragma unroll
    for (int n = 0; n < 4; ++n)
#pragma unroll
      for (int e = 0; e < 2; ++e)
        *reinterpret_cast<uint4*>(to + (4 * e + n) * 1024) = make_uint4(v[0][e][n], v[1][e][n], v[2][e][n], v[3][e][n]);
  }
}

// ---- softmax ------------------------------------------------------------------------------------------
struct Row {
  float f;                   // a score is f times the sum of products
  int limit;                 // last token the row sees
  bool in;
  __nv_bfloat16* out;
};

// 32 bytes in one access: with a row to a thread every access meets 32 lines, and their number is what it costs.
__device__ __forceinline__ void load32(const void* src, uint32_t (&v)[8]) {
  asm volatile("ld.global.v8.b32 {%0, %1, %2, %3, %4, %5, %6, %7}, [%8];"
               : "=r"(v[0]), "=r"(v[1]), "=r"(v[2]), "=r"(v[3]), "=r"(v[4]), "=r"(v[5]), "=r"(v[6]), "=r"(v[7]) : "l"(src));
}
__device__ __forceinline__ void store32(void* dst, const uint32_t (&v)[8]) {
  asm volatile("st.global.v8.b32 [%0], {%1, %2, %3, %4, %5, %6, %7, %8};"
               ::"l"(dst), "r"(v[0]), "r"(v[1]), "r"(v[2]), "r"(v[3]), "r"(v[4]), "r"(v[5]), "r"(v[6]), "r"(v[7]) : "memory");
}

// This thread's row of queries into its row tile, as fp16 in the order of the decoded keys.
template <int D, class Item>
__device__ __forceinline__ Row load_row(const AttendParams& p, const Item& it, int r, uint32_t tile, int row_in_tile) {
  Row o;
  const int row = it.row0 + r, qi = row / p.group, head = it.h * p.group + row - qi * p.group;
  o.in = row < it.n * p.group;
  o.limit = o.in ? it.len - it.n + qi : it.len - 1;
  o.out = p.out + static_cast<size_t>(it.q0 + qi) * p.ld_out + static_cast<size_t>(head) * p.hd_out;
  const __nv_bfloat16* src = p.q + static_cast<size_t>(it.q0 + qi) * p.ld_q + static_cast<size_t>(head) * p.hd_q;
  uint32_t u[D / 16][8];
#pragma unroll
  for (int c = 0; c < D / 16; ++c) {
    if (o.in && p.wide) {
      load32(src + 16 * c, u[c]);
    } else {
      const uint4 zero = make_uint4(0, 0, 0, 0);
      const uint4 a = o.in ? __ldg(reinterpret_cast<const uint4*>(src) + 2 * c) : zero, b = o.in ? __ldg(reinterpret_cast<const uint4*>(src) + 2 * c + 1) : zero;
      u[c][0] = a.x; u[c][1] = a.y; u[c][2] = a.z; u[c][3] = a.w; u[c][4] = b.x; u[c][5] = b.y; u[c][6] = b.z; u[c][7] = b.w;
    }
  }
  uint32_t most = 0;                                   // the largest magnitudes as integers: infinities and NaN come out on top
#pragma unroll
  for (int c = 0; c < D / 16; ++c)
#pragma unroll
    for (int i = 0; i < 8; ++i) most = __vmaxu2(most, u[c][i] & 0x7fff7fffu);
  most = max(most & 0xffffu, most >> 16);
  float up;
  row_factors(__uint_as_float(most << 16), most >= 0x7f80u, p.scale_log2, up, o.f);
#pragma unroll
  for (int c = 0; c < D / 8; ++c) {
    float x[8];
#pragma unroll
    for (int i = 0; i < 8; ++i) {
      const uint32_t v = u[c / 2][4 * (c & 1) + i / 2];
      x[i] = __uint_as_float((i & 1) ? (v & 0xffff0000u) : (v << 16)) * up;
    }
    uint32_t h[4];
#pragma unroll
    for (int n = 0; n < 4; ++n) h[n] = as_u32(__floats2half2_rn(x[n], x[n + 4]));
    st_shared_v4(chunk_at(tile, kRowTile, row_in_tile, c / 8, c % 8), make_uint4(h[0], h[1], h[2], h[3]));
  }
  return o;
}

// Columns [64 y, 64 y + 64) of O in the row's elements 64 y on: column 8 (4 e + n) + x is element 8 x + 4 e + n of them.
__device__ __forceinline__ void store_half(const Row& r, int y, const float (&o)[64], float k, bool wide) {
  if (!r.in) return;
#pragma unroll
  for (int x = 0; x < 8; x += 2) {
    uint32_t v[8];
#pragma unroll
    for (int i = 0; i < 8; ++i) {
      const __nv_bfloat162 h = __floats2bfloat162_rn(o[16 * (i % 4) + x + i / 4] * k, o[16 * (i % 4) + 8 + x + i / 4] * k);
      v[i] = *reinterpret_cast<const uint32_t*>(&h);
    }
    if (wide) {
      store32(r.out + 64 * y + 8 * x, v);
    } else {
      reinterpret_cast<uint4*>(r.out)[8 * y + x] = make_uint4(v[0], v[1], v[2], v[3]);
      reinterpret_cast<uint4*>(r.out)[8 * y + x + 1] = make_uint4(v[4], v[5], v[6], v[7]);
    }
  }
}

// A row of O times k, in tensor memory.
template <int D>
__device__ __forceinline__ void rescale(uint32_t o_at, float k) {
#pragma unroll 1
  for (int b = 0; b < D / 32; ++b) {
    uint32_t o[32];
    tmem_ld32(o_at + 32 * b, o);
    tmem_wait_ld();
#pragma unroll
    for (int v = 0; v < 32; ++v) o[v] = __float_as_uint(__uint_as_float(o[v]) * k);
    tmem_st32(o_at + 32 * b, o);
  }
  tmem_wait_st();
}
template <int D>
__device__ __noinline__ void rescale_far(uint32_t o_at, float k) { rescale<D>(o_at, k); }

template <int D, bool PADDED>
__global__ void __launch_bounds__(kThreads, 1) attend_many_kernel(const __grid_constant__ AttendParams p) {
  extern __shared__ uint8_t smem_raw[];
  using Tiles = Cut<kRows, kKeys, PADDED>;
  using Item = typename Tiles::Item;
  using S = ManySmem<D>;
  using U = CacheUnit<D>;
  __shared__ Bars bars;
  __shared__ uint32_t s_tmem;
  __shared__ int abort_flag, s_last, warp_sum[kThreads / 32];
  __shared__ uint32_t s_absent[S::kStages];
  const uint32_t raw = smem_u32(smem_raw), pad = (1024 - (raw & 1023)) & 1023;
  uint8_t* smem = smem_raw + pad;
  const uint32_t base = raw + pad;
  int* before = reinterpret_cast<int*>(smem + S::kBefore);
  const int tid = threadIdx.x, warp = tid >> 5, lane = tid & 31;
  const auto bar = [&](uint64_t& b) { return smem_u32(&b); };

  pdl_trigger();
  if (warp == 1) {
    asm volatile("tcgen05.alloc.cta_group::1.sync.aligned.shared::cta.b32 [%0], %1;" ::"r"(smem_u32(&s_tmem)), "r"(kTmemCols) : "memory");
    asm volatile("tcgen05.relinquish_alloc_permit.cta_group::1.sync.aligned;" ::: "memory");
  }
  if (tid == 0) {
    abort_flag = 0;
    for (int i = 0; i < S::kStages; ++i) { mbar_init(bar(bars.code_full[i]), 1); mbar_init(bar(bars.code_empty[i]), kDecoders); }
    for (int i = 0; i < 2; ++i) {
      mbar_init(bar(bars.k_full[i]), kDecoders); mbar_init(bar(bars.k_empty[i]), 1);
      mbar_init(bar(bars.v_full[i]), kDecoders); mbar_init(bar(bars.v_empty[i]), 1);
      mbar_init(bar(bars.s_full[i]), 1); mbar_init(bar(bars.p_ready[i][0]), 4); mbar_init(bar(bars.p_ready[i][1]), 4); mbar_init(bar(bars.q_full[i]), 4);
      mbar_init(bar(bars.o_done[i]), 1); mbar_init(bar(bars.o_free[i]), 4);
    }
    mbar_init(bar(bars.joined), 8);
    asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
  }
  pdl_wait();
  tc_fence_before();
  const int total = Tiles::template count_tiles<kThreads / 32>(p, before, warp_sum, false);      // also orders what is set up above
  tc_fence_after();
  const uint32_t tmem = s_tmem;

  // Runs of kLeast tiles and more, and none that leaves a part of kSnap tiles or less of an item: writing and joining the parts of an
  // item takes as long as six tiles.
  const int n_runs = min(max(total / kLeast, 1), static_cast<int>(gridDim.x));
  const bool works = total > 0 && static_cast<int>(blockIdx.x) < n_runs;
  if (works) {
    const Runs runs(total, n_runs);
    Item start, behind;                                // the items that the run begins in, and that the next one begins in
    const int begin = snapped<Tiles>(p, before, runs, blockIdx.x, n_runs, total, start), end = snapped<Tiles>(p, before, runs, blockIdx.x + 1, n_runs, total, behind);
    volatile int* abort_at = &abort_flag;
    const auto wait = [&](uint64_t& b, uint32_t parity) { return mbar_wait_warp(smem_u32(&b), parity, abort_at, p.wait_ns); };
    // The softmax waits for scores and joins as long as a call may take: while items have one row tile its second warpgroup has nothing to
    // do until the next item, or until a cut one is joined, and that is the whole run of the first one.  The roles that feed it, and the
    // issuer for its weights, wait within the ordinary limit at every tile: where anything stalls, one of theirs ends and ends these.
    const auto wait_softmax = [&](uint64_t& b, uint32_t parity) { return mbar_wait_warp(smem_u32(&b), parity, abort_at, p.idle_ns); };

    // 512 threads of 128 registers at launch: 256 of 64 and 256 of 192
    if (warp < 8) {
    asm volatile("setmaxnreg.dec.sync.aligned.u32 64;");
    Pieces<Tiles> pc(start, begin, end, before);
    if (warp == 0) {
      // ---- loader: keys, then values of each tile; lanes 0 to 7 a unit each
      const size_t head_bytes = static_cast<size_t>(p.page_size / kUnit) * U::kBytes;
      int stage = 0;
      uint32_t phase = 0;
      bool fine = true;
      while (fine && pc.next(p)) {
        for (int i = 0; fine && i < pc.steps(); ++i) {
          const int t = (pc.tile0() + i) * kKeys + lane * kUnit;
          const bool wanted = lane < kKeys / kUnit && t < pc.it.len;
          int page = 0;
          if (wanted) page = p.page_table[static_cast<size_t>(pc.it.b) * p.max_pages + (t >> p.page_shift)];
          const bool there = static_cast<unsigned>(page) < static_cast<unsigned>(p.n_pages);
          const uint32_t want = __ballot_sync(0xffffffffu, wanted), gone = __ballot_sync(0xffffffffu, wanted && !there);
          if (gone != 0 && lane == 0) atomicOr(p.status, TEMPO_STATUS_BAD_INDEX);
          const uint8_t* src = p.cache + (static_cast<size_t>(there ? page : 0) * p.Hkv + pc.it.h) * 2 * head_bytes +
                               ((t & (p.page_size - 1)) / kUnit) * U::kBytes;
#pragma unroll
          for (int kv = 0; kv < 2; ++kv) {
            fine = wait(bars.code_empty[stage], phase ^ 1);
            if (!fine) break;
            if (lane == 0) {
              s_absent[stage] = gone;
              mbar_arrive_expect_tx(bar(bars.code_full[stage]), __popc(want) * U::kBytes);
            }
            __syncwarp();
            if (wanted) bulk_load(base + S::kCodes + stage * S::kStageBytes + lane * U::kBytes, src + kv * head_bytes, U::kBytes, bar(bars.code_full[stage]));
            if (++stage == S::kStages) { stage = 0; phase ^= 1; }
          }
        }
      }
      if (!fine) {                                     // what was requested arrives before the memory goes
        volatile int none = 0;
        for (int st = 0; st < S::kStages; ++st) mbar_wait_warp(bar(bars.code_full[st]), phase ^ (st < stage ? 0u : 1u), &none, p.wait_ns);
      }
    } else if (warp == 1) {
      // ---- issuer: a warp whose loops are uniform (see mma_warp.cuh)
      const uint32_t leader = elect_one();
      constexpr uint32_t kQk = kIdesc<kKeys>, kPv = kIdesc<D>;
      const uint32_t tm = warp_uniform(tmem);
      const auto product_qk = [&](uint32_t x, uint32_t buf) {
        const uint32_t s_at = tm + x * kKeys, q = base + S::kQ + x * S::kTileBytes, k0 = base + S::kK + buf * S::kTileBytes;
#pragma unroll
        for (int k = 0; k < D / 16; ++k) {
          const uint32_t at = (k / 4) * kKeys * 128 + (k % 4) * 32;
          mma_ss(leader, s_at, desc_lo_sw128(q + at), desc_lo_sw128(k0 + at), kQk, k > 0);
        }
        warp_commit(leader, bar(bars.s_full[x]));
      };
      int buf = 0, done0 = 0, done1 = 0, seen0 = 0, seen1 = 0;           // steps and items of each row tile
      uint32_t turn = 0;                                                 // of the two buffers
      bool fine = true;
      while (fine && warp_uniform(pc.next(p))) {
        const int steps = warp_uniform(pc.steps());
        const bool two = warp_uniform(pc.two(p.group)) != 0;
        fine = wait(bars.k_full[buf], turn) && wait(bars.q_full[0], seen0 & 1);
        if (!fine) break;
        tc_fence_after();
        product_qk(0, buf);
        if (two) {
          fine = wait(bars.q_full[1], seen1 & 1);
          if (!fine) break;
          tc_fence_after();
          product_qk(1, buf);
        }
        warp_commit(leader, bar(bars.k_empty[buf]));
#pragma unroll 1
        for (int i = 0; i < steps; ++i) {
          const int next = buf ^ 1;
          const uint32_t next_turn = turn ^ (buf == 1 ? 1u : 0u);
          fine = wait(bars.v_full[buf], turn);
          if (!fine) break;
#pragma unroll 1
          for (int x = 0; x < (two ? 2 : 1); ++x) {
            const uint32_t ready = (x == 0 ? done0++ : done1++) & 1;
            fine = wait(bars.p_ready[x][0], ready) && (i > 0 || wait(bars.o_free[x], ((x == 0 ? seen0 : seen1) & 1) ^ 1));
            if (!fine) break;
            tc_fence_after();
            const uint32_t o_at = tm + 2 * kKeys + x * D, s_at = tm + x * kKeys, v0 = base + S::kV + buf * S::kTileBytes;
            const uint32_t add = i > 0 ? 1u : 0u;
#pragma unroll
            for (int k = 0; k < 4; ++k) mma_ts(leader, o_at, s_at + k * 8, desc_lo_sw128(v0 + k * 32), kPv, k > 0 ? 1u : add);
            fine = wait(bars.p_ready[x][1], ready);
            if (!fine) break;
            tc_fence_after();
#pragma unroll
            for (int k = 0; k < 4; ++k) mma_ts(leader, o_at, s_at + 32 + k * 8, desc_lo_sw128(v0 + D * 128 + k * 32), kPv, 1u);
            const bool last = x == (two ? 1 : 0);
            if (i == steps - 1) warp_commit(leader, bar(bars.o_done[x]));
            if (last) warp_commit(leader, bar(bars.v_empty[buf]));
            if (i + 1 < steps) {
              if (x == 0) {
                fine = wait(bars.k_full[next], next_turn);
                if (!fine) break;
                tc_fence_after();
              }
              product_qk(x, next);
              if (last) warp_commit(leader, bar(bars.k_empty[next]));
            }
          }
          if (!fine) break;
          buf = next;
          turn = next_turn;
        }
        ++seen0;
        if (two) ++seen1;
      }
    } else {
      // ---- decoders
      const Decode dc;
      int stage = 0, t = 0;
      uint32_t phase = 0;
      bool fine = true;
      while (fine && pc.next(p)) {
        const int steps = pc.steps(), least = pc.it.len - pc.it.n + pc.it.row0 / p.group;   // the last token that every row sees
        for (int i = 0; fine && i < steps; ++i, ++t) {
          const int buf = t & 1, k0 = (pc.tile0() + i) * kKeys;
#pragma unroll
          for (int kv = 0; kv < 2; ++kv) {
            fine = wait(kv == 0 ? bars.k_empty[buf] : bars.v_empty[buf], (t >> 1 & 1) ^ 1) && wait(bars.code_full[stage], phase);
            if (!fine) break;
            uint8_t* codes = smem + S::kCodes + stage * S::kStageBytes;
            if (kv == 0) decode_keys<D>(dc, codes, smem + S::kK + buf * S::kTileBytes, s_absent[stage], warp - 2);
            else decode_values<D>(dc, codes, smem + S::kV + buf * S::kTileBytes, pc.it.len - k0, k0 + kKeys - 1 > least, warp - 2);
            fence_async_smem();
            __syncwarp();
            if (lane == 0) {
              mbar_arrive(bar(kv == 0 ? bars.k_full[buf] : bars.v_full[buf]));
              mbar_arrive(bar(bars.code_empty[stage]));
            }
            if (++stage == S::kStages) { stage = 0; phase ^= 1; }
          }
        }
      }
    }
    } else {
      asm volatile("setmaxnreg.inc.sync.aligned.u32 192;");
      Pieces<Tiles> pc(start, begin, end, before);
      // ---- softmax: warpgroup x on row tile x, thread by row
      const int x = (warp - 8) >> 2, row = (warp & 3) * 32 + lane, r = x * kRowTile + row;
      const uint32_t lanes = static_cast<uint32_t>((warp & 3) * 32) << 16;
      const uint32_t s_at = tmem + lanes + x * kKeys, o_at = tmem + lanes + 2 * kKeys + x * D;
      const uint32_t q_tile = base + S::kQ + x * S::kTileBytes;
      int done = 0, seen = 0;
      uint32_t joins = 0;
      const auto sync_softmax = [&]() {                // a barrier of the softmax warps whose wait ends like any other
        __syncwarp();
        if (lane == 0) mbar_arrive(bar(bars.joined));
        return wait_softmax(bars.joined, joins++ & 1);
      };
      bool fine = true;
      Row mine;
      const auto load = [&](const Pieces<Tiles>& c) {
        if (x == 1 && !c.two(p.group)) return;
        mine = load_row<D>(p, c.it, r, q_tile, row);
        fence_async_smem();
        __syncwarp();
        if (lane == 0) mbar_arrive(bar(bars.q_full[x]));
      };
      bool more = pc.next(p);
      if (more) load(pc);
      while (more && fine) {
        const Item it = pc.it;
        const int steps = pc.steps(), tile0 = pc.tile0();
        const bool active = x == 0 || pc.two(p.group);
        float m = -INFINITY, l[2][2] = {{0.0f, 0.0f}, {0.0f, 0.0f}};
        const Row cur = mine;
        const auto ready = [&](int h) {                // P's columns 32 h to 32 h + 31, where S's first ones were
          tmem_wait_st();
          tc_fence_before();
          __syncwarp();
          if (lane == 0) mbar_arrive(bar(bars.p_ready[x][h]));
        };
        if (active) {
          bool far = false;                            // far_scores of some row of the warp, from step i on
          int i = 0;
          for (; i < steps; ++i) {
            fine = wait_softmax(bars.s_full[x], done & 1);
            if (!fine) break;
            ++done;
            tc_fence_after();
            const int k0 = (tile0 + i) * kKeys;
            const int see = cur.limit - k0;
            const bool masked = __any_sync(0xffffffffu, see < kKeys - 1);
            uint32_t c[4][32];
#pragma unroll
            for (int b = 0; b < 4; ++b) tmem_ld32(s_at + 32 * b, c[b]);
            tmem_wait_ld();
            if (masked) {
#pragma unroll
              for (int v = 0; v < 128; ++v)
                if (v > see) c[v / 32][v % 32] = 0xff800000u;
            }
            float tops[4] = {-INFINITY, -INFINITY, -INFINITY, -INFINITY};
#pragma unroll
            for (int v = 0; v < 128; v += 2) tops[v / 2 % 4] = max3(tops[v / 2 % 4], __uint_as_float(c[v / 32][v % 32]), __uint_as_float(c[v / 32][v % 32 + 1]));
            float top = fmaxf(max3(tops[0], tops[1], tops[2]), tops[3]);
            top *= cur.f;
            if (__any_sync(0xffffffffu, top > m + kSlack)) {
              const float to = top > m + kSlack ? top : m;
              const float k = to == m ? 1.0f : exp2_fast(m - to);
              m = to;
              l[0][0] *= k; l[0][1] *= k; l[1][0] *= k; l[1][1] *= k;
              if (i > 0) rescale<D>(o_at, k);          // S of this step is there: the products into O before it are done
              far = __any_sync(0xffffffffu, far_scores(m));
              if (far) break;
            }
            const float less = m == -INFINITY ? 0.0f : kBias - m;
#pragma unroll
            for (int h = 0; h < 2; ++h) {              // from S's columns 64 h to 64 h + 63
              uint32_t w[32];
#pragma unroll
              for (int v = 0; v < 32; ++v) {
                float a = __uint_as_float(c[2 * h + v / 16][v % 16 * 2]), b = __uint_as_float(c[2 * h + v / 16][v % 16 * 2 + 1]);
                fma_pair(a, b, cur.f, less);
                a = exp2_fast(a);
                b = exp2_fast(b);
                add_pair(l[v & 1][0], l[v & 1][1], a, b);
                w[v] = as_u32(__floats2half2_rn(a, b));
              }
              tmem_st32(s_at + 32 * h, w);
              ready(h);
            }
          }
          // The rest of the piece where scores are far from zero: by quarters of S, each read again.  In a loop of its own, for the registers
          // of the other one: two chunks of 2048 over 6144 tokens take 502 us, with both ways in one loop 517, without this one 492.
          for (bool first = true; far && i < steps; ++i, first = false) {
            if (!first) {
              fine = wait_softmax(bars.s_full[x], done & 1);
              if (!fine) break;
              ++done;
              tc_fence_after();
            }
            const int see = cur.limit - (tile0 + i) * kKeys;
            const auto quarter = [&](int b, float (&sums)[32]) {
              uint32_t u[32];
              tmem_ld32(s_at + 32 * b, u);
              tmem_wait_ld();
#pragma unroll
              for (int v = 0; v < 32; ++v) sums[v] = 32 * b + v > see ? -INFINITY : __uint_as_float(u[v]);
            };
            float sums[32], top = -INFINITY;
#pragma unroll 1
            for (int b = 0; b < 4; ++b) {
              quarter(b, sums);
#pragma unroll
              for (int v = 0; v < 32; ++v) top = fmaxf(top, sums[v]);
            }
            top *= cur.f;
            if (__any_sync(0xffffffffu, top > m + kSlack)) {
              const float to = top > m + kSlack ? top : m, k = to == m ? 1.0f : exp2_fast(m - to);
              m = to;
              l[0][0] *= k; l[0][1] *= k; l[1][0] *= k; l[1][1] *= k;
              if (i > 0) rescale_far<D>(o_at, k);
            }
            const float less = m == -INFINITY ? 0.0f : kBias - m;
#pragma unroll 1
            for (int b = 0; b < 4; ++b) {
              quarter(b, sums);
#pragma unroll
              for (int v = 0; v < 32; v += 2) {
#pragma unroll
                for (int j = v; j < v + 2; ++j) {
                  sums[j] = exp2_fast(far_scores(m) ? from_far(sums[j], cur.f, m) + kBias : fmaf(sums[j], cur.f, less));
                  l[v / 2 & 1][j & 1] += sums[j];
                }
                tmem_st1(s_at + 16 * b + v / 2, as_u32(__floats2half2_rn(sums[v], sums[v + 1])));
              }
              if (b & 1) ready(b / 2);
            }
          }
          if (!fine) break;
        }
        more = pc.next(p);
        if (more) load(pc);                            // the next item's queries: every product with these is done

        const float sum = (l[0][0] + l[0][1]) + (l[1][0] + l[1][1]);
        const int first = runs.of(it.begin + kSnap), ctas = max(0, runs.of(it.begin + it.tiles - kSnap - 1) - first) + 1;
        // A cut item's parts go to the workspace, four columns of a row to a 16-byte line of 256 rows; the CTA that arrives last adds
        // them up in their order.
        const auto part_of = [&](int cta) { return static_cast<size_t>(cta) * 2 + (cta == first ? 1 : 0); };
        float4* parts = reinterpret_cast<float4*>(p.part);
        float2* stats = reinterpret_cast<float2*>(p.stats);
        if (active) {
          fine = wait(bars.o_done[x], seen & 1);
          if (!fine) break;
          tc_fence_after();
          const float k = sum == 0.0f ? 0.0f : 1.0f / sum;
          const size_t at = part_of(blockIdx.x);
          if (ctas > 1) __stcg(stats + at * kRows + r, make_float2(m, sum));
#pragma unroll 1
          for (int y = 0; y < D / 64; ++y) {
            uint32_t v[2][32];
            tmem_ld32(o_at + 64 * y, v[0]);
            tmem_ld32(o_at + 64 * y + 32, v[1]);
            tmem_wait_ld();
            if (y == D / 64 - 1) {
              tc_fence_before();
              __syncwarp();
              if (lane == 0) mbar_arrive(bar(bars.o_free[x]));
            }
            float o[64];
#pragma unroll
            for (int i = 0; i < 64; ++i) o[i] = __uint_as_float(v[i / 32][i % 32]);
            if (ctas == 1) {
              store_half(cur, y, o, k, p.wide);
            } else {
#pragma unroll
              for (int q = 0; q < 16; ++q)
                __stcg(parts + (at * (D / 4) + 16 * y + q) * kRows + r, make_float4(o[4 * q], o[4 * q + 1], o[4 * q + 2], o[4 * q + 3]));
            }
          }
          ++seen;
        }
        if (ctas == 1) continue;
        // Of many parts, groups first, each by its own last CTA: a CTA reads 64 bytes a clock at best, 2000 clocks for a part of two row
        // tiles.  18 parts (16 queries over 16384 tokens, 64 heads on 8) 49 -> 43 us, 37 (64 queries over 65536, 16 heads of 64 on 2) 65 ->
        // 56; 6 or 7 are joined sooner at once (300 queries over 5000 tokens 49 against 53).
        int group = ctas;
        if (ctas > 12)
          for (group = 4; group * group < ctas;) ++group;
        const int lead = (static_cast<int>(blockIdx.x) - first) / group * group;
#pragma unroll 1
        for (int level = 0; level < 2; ++level) {
          const int from = first + (level == 0 ? lead : 0), stride = level == 0 ? 1 : group;
          const int count = level == 0 ? min(group, ctas - lead) : (ctas + group - 1) / group;
          const bool ends = level == 1 || group == ctas;
          __threadfence();
          fine = sync_softmax();
          if (!fine) break;
          if (tid == kThreads - 1) {
            unsigned* counter = ends ? p.counters + first : p.groups + part_of(from);
            const bool last = atomicAdd(counter, 1u) == static_cast<unsigned>(count) - 1u;
            if (last) *counter = 0;
            s_last = last;
          }
          fine = sync_softmax();
          if (!fine) break;
          const bool go = s_last != 0;
          if (go && active) {
            __threadfence();
            float top = -INFINITY, all = 0.0f;
            for (int c = 0; c < count; ++c) top = fmaxf(top, __ldcg(stats + part_of(from + c * stride) * kRows + r).x);
            const float ref = top == -INFINITY ? 0.0f : top;
            for (int c = 0; c < count; ++c) {
              const float2 st = __ldcg(stats + part_of(from + c * stride) * kRows + r);
              all += st.y * exp2_fast(st.x - ref);
            }
#pragma unroll 1
            for (int y = 0; y < D / 64; ++y) {
              float o[64];
#pragma unroll
              for (int i = 0; i < 64; ++i) o[i] = 0.0f;
#pragma unroll 1
              for (int c = 0; c < count; ++c) {
                const size_t at = part_of(from + c * stride);
                const float k = exp2_fast(__ldcg(stats + at * kRows + r).x - ref);
                float4 v[16];
#pragma unroll
                for (int q = 0; q < 16; ++q) v[q] = __ldcg(parts + (at * (D / 4) + 16 * y + q) * kRows + r);
#pragma unroll
                for (int q = 0; q < 16; ++q) {
                  o[4 * q] += v[q].x * k; o[4 * q + 1] += v[q].y * k; o[4 * q + 2] += v[q].z * k; o[4 * q + 3] += v[q].w * k;
                }
              }
              if (ends) {
                store_half(cur, y, o, all == 0.0f ? 0.0f : 1.0f / all, p.wide);
              } else {                                 // in the place of the group's first part, whose elements are this thread's
#pragma unroll
                for (int q = 0; q < 16; ++q)
                  __stcg(parts + (part_of(from) * (D / 4) + 16 * y + q) * kRows + r, make_float4(o[4 * q], o[4 * q + 1], o[4 * q + 2], o[4 * q + 3]));
              }
            }
            if (!ends) __stcg(stats + part_of(from) * kRows + r, make_float2(top, all));
          }
          fine = sync_softmax();                       // s_last is read before it is written again
          if (!fine || !go || ends) break;
        }
      }
    }
  }

  tc_fence_before();
  __syncthreads();
  if (abort_flag) {
    if (tid == 0) atomicOr(p.status, static_cast<uint32_t>(TEMPO_STATUS_TIMEOUT));
    for (int i = 0; i < 50; ++i) __nanosleep(1000);    // products in flight drain
  }
  if (warp == 1) {
    tc_fence_after();
    __syncwarp();
    asm volatile("tcgen05.dealloc.cta_group::1.sync.aligned.b32 %0, %1;" ::"r"(tmem), "r"(kTmemCols) : "memory");
  }
}

// The warps' split of registers draws on those that the block was launched with: with fewer of them it would wait for good.
template <int D, bool PADDED>
bool registers_suffice() {
  cudaFuncAttributes a;
  return cudaFuncGetAttributes(&a, attend_many_kernel<D, PADDED>) == cudaSuccess && a.numRegs * kThreads >= 256 * 64 + 256 * 192;
}

template <int D, bool PADDED>
cudaError_t launch_as(const AttendParams& p, int num_sms, cudaStream_t stream) {
  static const bool fits = registers_suffice<D, PADDED>();
  if (!fits) return cudaErrorInvalidConfiguration;
  static std::atomic<unsigned long long> done{0};
  const cudaError_t e = smem_limit_once(attend_many_kernel<D, PADDED>, ManySmem<D>::bytes(kAttendMaxB), done);
  if (e != cudaSuccess) return e;
  return launch_pdl(attend_many_kernel<D, PADDED>, dim3(num_sms), dim3(kThreads), ManySmem<D>::bytes(p.B), stream, p);
}

}  // namespace

cudaError_t launch_attend_many(const AttendParams& p, int D, int num_sms, cudaStream_t stream) {
  if (p.n_valid == nullptr) return D == 64 ? launch_as<64, false>(p, num_sms, stream) : launch_as<128, false>(p, num_sms, stream);
  return D == 64 ? launch_as<64, true>(p, num_sms, stream) : launch_as<128, true>(p, num_sms, stream);
}

}  // namespace tempo
