// Attention over the 4-bit paged cache (tempo_attend).
//
//   out[i, h] = sum_t p[t] V[t] / sum_t p[t],  p[t] = exp(scale <q, K[t]> - m),  t <= the query's own position
//
// A key head's queries (the heads of its group, and the new tokens of the sequence) are the rows of one item, 16 rows to an item;
// each cached byte is read once for all of them.  One pass over the tokens with the running maximum and sum.
//
// Bound by the cache's bytes, which one SM takes in at 23 bytes a clock: that leaves 2.8 instruction slots of a lane for each
// cached element.  So codes go from shared memory to registers and are decoded there into the B operands of the
// matrix instruction (m16n8k16, 32-bit sums), at 11 instructions for 8 elements; a decoded copy in shared memory for the
// tensor-memory form of the instruction would move 2 bytes per element in and 2 out, 184 bytes a clock where the SM has 128.
// The order of a sum over d or t is free, so that a lane's 16-byte load is what it needs: of keys 32 neighbouring elements
// (one group: one scale) of one token, of values 16 neighbouring elements of two tokens side by side in a word's halves.
//
// Work is dealt in tiles of 32 tokens: the tiles of all items in one row, cut into equal runs, one for each warp of the
// launch, whatever the lengths.  A warp streams its run through a ring of its own (bulk copies, one barrier per stage) and
// waits for nobody; parts of items that were cut are joined in shared memory after the CTA's last tile, and across CTAs by the one
// that arrives last, in a fixed order.
#include "attend_common.cuh"

namespace tempo {

namespace {

constexpr int kWarps = 8, kTile = 64, kUnits = kTile / kUnit, kRows = 16;

using Tiles = Cut<kRows, kTile>;
using Item = Tiles::Item;

struct Part {                 // a cut item's share of one warp
  Item item;
  int valid;
};

template <int D>
struct AttendSmem {
  static constexpr int kStageBytes = 2 * kUnits * CacheUnit<D>::kBytes;   // keys and values of each unit
  static constexpr int kStages = D == 64 ? 4 : 2;
  static constexpr int kRing = kWarps * kStages * kStageBytes;
  static constexpr int kPart = kRows * D * 4 + kRows * 8;            // O, then (m, l) of each row
  static constexpr int kBars = kRing, kParts = kBars + kWarps * kStages * 8;
  static constexpr int kRecords = kParts + kWarps * kPart;
  static constexpr int kBefore = kRecords + kWarps * 2 * static_cast<int>(sizeof(Part));
  static_assert(kRing >= kWarps * kPart, "the second parts take the ring's place");
  static_assert(kRing >= kAttendMaxSms * kRows * 4 + kRows * 4, "so do the weights of a join");
  static int bytes(int B) { return kBefore + (B + 1) * 4; }
};

__device__ __forceinline__ void mma_f16(float (&c)[4], const uint32_t (&a)[4], uint32_t b0, uint32_t b1) {
  asm("mma.sync.aligned.m16n8k16.row.col.f32.f16.f16.f32 {%0, %1, %2, %3}, {%4, %5, %6, %7}, {%8, %9}, {%0, %1, %2, %3};"
      : "+f"(c[0]), "+f"(c[1]), "+f"(c[2]), "+f"(c[3]) : "r"(a[0]), "r"(a[1]), "r"(a[2]), "r"(a[3]), "r"(b0), "r"(b1));
}
template <int W>
__device__ __forceinline__ void load_words(const uint8_t* a, uint32_t (&v)[W]) {
  if constexpr (W == 4) {
    const uint4 u = *reinterpret_cast<const uint4*>(a);
    v[0] = u.x; v[1] = u.y; v[2] = u.z; v[3] = u.w;
  } else {
    const uint2 u = *reinterpret_cast<const uint2*>(a);
    v[0] = u.x; v[1] = u.y;
  }
}

// Float4 number q (of D / 4) of a row in a part: rotated so that the eight lanes of a store's phase meet eight bank groups.
__device__ __forceinline__ int part_at(int row, int q) { return q ^ ((((row & 1) << 2) | ((q >> 3) & 3)) & 7); }

// A warp's running state of one item.
template <int D>
struct Running {
  static constexpr int kN = D / 8;                   // 8-column tiles of O
  uint32_t q[D / 16][4];                             // A operands: rows lane / 4 and + 8
  float f[2];                                        // score = f * (sum of products), in units of log2; above zero
  int limit[2], least;                               // last token that each row sees; the least over the 16 rows
  float m[2];
  float l[4];                                        // the sums of the weights, one more column of O: rows in l[0] and l[2]
  float o[kN][4];
};

template <int D>
__device__ __forceinline__ void begin_item(const AttendParams& p, const Item& it, Running<D>& s) {
  constexpr int W = D / 32;                          // 8-element words of a lane
  const int lane = threadIdx.x & 31, j = lane & 3;
  const int rows = it.n * p.group;
#pragma unroll
  for (int half = 0; half < 2; ++half) {
    const int row = it.row0 + lane / 4 + 8 * half;
    const bool in = row < rows;
    const int qi = row / p.group, head = it.h * p.group + row % p.group;
    s.limit[half] = in ? it.len - it.n + qi : it.len - 1;
    float x[W][8];
    float top = 0.0f;
    bool odd = false;
    const __nv_bfloat16* src = p.q + static_cast<size_t>(it.q0 + (in ? qi : 0)) * p.ld_q + static_cast<size_t>(in ? head : 0) * p.hd_q + j * (D / 4);
#pragma unroll
    for (int w = 0; w < W; ++w) {
      const uint4 u = in ? __ldg(reinterpret_cast<const uint4*>(src) + w) : make_uint4(0, 0, 0, 0);
      const uint32_t v[4] = {u.x, u.y, u.z, u.w};
#pragma unroll
      for (int i = 0; i < 8; ++i) {
        x[w][i] = __uint_as_float((i & 1) ? (v[i / 2] & 0xffff0000u) : (v[i / 2] << 16));
        top = fmaxf(top, fabsf(x[w][i]));
        odd = odd || !isfinite(x[w][i]);
      }
    }
#pragma unroll
    for (int d = 1; d <= 2; d *= 2) {
      top = fmaxf(top, __shfl_xor_sync(0xffffffffu, top, d));
      odd = __shfl_xor_sync(0xffffffffu, static_cast<int>(odd), d) != 0 || odd;
    }
    float up;
    row_factors(top, odd, p.scale_log2, up, s.f[half]);
#pragma unroll
    for (int w = 0; w < W; ++w)
#pragma unroll
      for (int u = 0; u < 2; ++u) {                  // the pairs (n, n + 4) of decode8, two to a matrix instruction
        s.q[2 * w + u][half] = as_u32(__floats2half2_rn(x[w][2 * u] * up, x[w][2 * u + 4] * up));
        s.q[2 * w + u][half + 2] = as_u32(__floats2half2_rn(x[w][2 * u + 1] * up, x[w][2 * u + 5] * up));
      }
    s.m[half] = -INFINITY;
  }
  s.least = it.len - it.n + it.row0 / p.group;
  s.l[0] = s.l[1] = s.l[2] = s.l[3] = 0.0f;
#pragma unroll
  for (int i = 0; i < Running<D>::kN; ++i) { s.o[i][0] = s.o[i][1] = s.o[i][2] = s.o[i][3] = 0.0f; }
}

// One tile: tokens [t0, t0 + 64) of the item at `stage`.  `absent`: bits of its units whose page is not in the cache.
template <int D>
__device__ __forceinline__ void run_tile(Running<D>& s, const uint8_t* stage, int t0, int len, uint32_t absent) {
  using U = CacheUnit<D>;
  constexpr int W = D / 32, kCols = kTile / 8;
  const int lane = threadIdx.x & 31, g = lane / 4, j = lane & 3;
  float c[kCols][4];
#pragma unroll
  for (int k = 0; k < kUnits; ++k) {                 // scores of unit k: two chains of matrix instructions side by side
    const uint8_t* unit = stage + k * 2 * U::kBytes;
    uint32_t w[2][W], sc[2], b[2];
#pragma unroll
    for (int x = 0; x < 2; ++x) {
      c[2 * k + x][0] = c[2 * k + x][1] = c[2 * k + x][2] = c[2 * k + x][3] = 0.0f;
      const int at = x * 8 + g;
      load_words<W>(unit + at * U::kKeyRow + j * (D / 8), w[x]);
      group_params(*reinterpret_cast<const uint16_t*>(unit + U::kCodes + at * U::kKeyParams + (D == 128 ? j : j / 2) * 2) * 0x10001u, sc[x], b[x]);
    }
#pragma unroll
    for (int y = 0; y < W; ++y) {
      uint32_t v[2][4];
#pragma unroll
      for (int x = 0; x < 2; ++x) decode8(w[x][y], sc[x], b[x], v[x]);
#pragma unroll
      for (int u = 0; u < 2; ++u)
#pragma unroll
        for (int x = 0; x < 2; ++x) mma_f16(c[2 * k + x], s.q[2 * y + u], v[x][2 * u], v[x][2 * u + 1]);
    }
  }
  if (absent != 0) {
#pragma unroll
    for (int i = 0; i < kCols; ++i)
      if (absent >> (i / 2) & 1) c[i][0] = c[i][1] = c[i][2] = c[i][3] = __uint_as_float(0x7fc00000u);
  }
  if (t0 + kTile - 1 > s.least) {
#pragma unroll
    for (int i = 0; i < kCols; ++i)
#pragma unroll
      for (int x = 0; x < 4; ++x)
        if (t0 + 8 * i + 2 * j + (x & 1) > s.limit[x / 2]) c[i][x] = -INFINITY;
  }
  float top[2] = {-INFINITY, -INFINITY};
#pragma unroll
  for (int r = 0; r < 2; ++r) {
#pragma unroll
    for (int i = 0; i < kCols; ++i) top[r] = fmaxf(top[r], fmaxf(c[i][2 * r], c[i][2 * r + 1]));
    top[r] = fmaxf(top[r], __shfl_xor_sync(0xffffffffu, top[r], 1));
    top[r] = fmaxf(top[r], __shfl_xor_sync(0xffffffffu, top[r], 2));
    top[r] *= s.f[r];
  }
  // a maximum that has grown little stays: weights up to 2^15 are in fp16's range, and O is left alone
  if (__any_sync(0xffffffffu, top[0] > s.m[0] + kSlack || top[1] > s.m[1] + kSlack)) {
#pragma unroll
    for (int r = 0; r < 2; ++r) {
      const float m = top[r] > s.m[r] + kSlack ? top[r] : s.m[r];
      const float k = m == s.m[r] ? 1.0f : exp2_fast(s.m[r] - m);
      s.m[r] = m;
      s.l[2 * r] *= k;
#pragma unroll
      for (int i = 0; i < Running<D>::kN; ++i) { s.o[i][2 * r] *= k; s.o[i][2 * r + 1] *= k; }
    }
  }
  uint32_t a[kUnits][4];
#pragma unroll
  for (int r = 0; r < 2; ++r) {
    const float m = s.m[r] == -INFINITY ? 0.0f : kBias - s.m[r];
#pragma unroll
    for (int i = 0; i < kCols; ++i)
      a[i / 2][(i & 1) * 2 + r] =
          as_u32(__floats2half2_rn(exp2_fast(fmaf(c[i][2 * r], s.f[r], m)), exp2_fast(fmaf(c[i][2 * r + 1], s.f[r], m))));
  }
#pragma unroll
  for (int k = 0; k < kUnits; ++k) {                 // unit k: tokens 16 k + 2 j, + 1 and 16 k + 8 + 2 j, + 1
    const uint8_t* unit = stage + (k * 2 + 1) * U::kBytes;
    uint32_t w[2][W], sc[2], b[2];
#pragma unroll
    for (int x = 0; x < 2; ++x) {
      const int pair = 4 * x + j;
      load_words<W>(unit + pair * U::kPairRow + g * (D / 8), w[x]);
      uint32_t params = *reinterpret_cast<const uint32_t*>(unit + U::kCodes + pair * U::kPairParams + (D == 128 ? g / 2 : g / 4) * 4);
      const int left = len - (t0 + 16 * k + 2 * pair);           // tokens of the pair that exist: what lies behind may be anything
      if (left < 2) params &= left == 1 ? 0xffffu : 0u;
      group_params(params, sc[x], b[x]);
    }
    mma_f16(s.l, a[k], 0x3c003c00u, 0x3c003c00u);    // times 1: the sum is that of the weights as they meet V
#pragma unroll
    for (int y = 0; y < W; ++y) {
      uint32_t v0[4], v1[4];
      decode8(w[0][y], sc[0], b[0], v0);
      decode8(w[1][y], sc[1], b[1], v1);
#pragma unroll
      for (int n = 0; n < 4; ++n) mma_f16(s.o[4 * y + n], a[k], v0[n], v1[n]);
    }
  }
}

__device__ __forceinline__ __nv_bfloat16* out_row(const AttendParams& p, const Item& it, int row) {
  const int r = it.row0 + row;
  return p.out + static_cast<size_t>(it.q0 + r / p.group) * p.ld_out + static_cast<size_t>(it.h * p.group + r % p.group) * p.hd_out;
}

// A whole item's result from the registers.  Lane (g, j) has, of the rows g and g + 8, the elements j D/4 to (j+1) D/4 - 1: O tile i
// holds element i of each of the eight runs of D / 8.
template <int D>
__device__ __forceinline__ void store_item(const AttendParams& p, const Item& it, Running<D>& s) {
  const int lane = threadIdx.x & 31, g = lane / 4, j = lane & 3;
#pragma unroll
  for (int r = 0; r < 2; ++r) {
    if (it.row0 + g + 8 * r >= it.n * p.group) continue;
    const float k = s.l[2 * r] == 0.0f ? 0.0f : 1.0f / s.l[2 * r];
    uint4* dst = reinterpret_cast<uint4*>(out_row(p, it, g + 8 * r) + j * (D / 4));
#pragma unroll
    for (int y = 0; y < 2; ++y)
#pragma unroll
      for (int i = 0; i < Running<D>::kN; i += 8) {
        uint32_t v[4];
#pragma unroll
        for (int x = 0; x < 4; ++x) {
          const __nv_bfloat162 h = __floats2bfloat162_rn(s.o[i + 2 * x][2 * r + y] * k, s.o[i + 2 * x + 1][2 * r + y] * k);
          v[x] = *reinterpret_cast<const uint32_t*>(&h);
        }
        dst[(y * Running<D>::kN + i) / 8] = make_uint4(v[0], v[1], v[2], v[3]);
      }
  }
}

template <int D>
__device__ __forceinline__ void keep_part(Running<D>& s, uint8_t* part) {
  const int lane = threadIdx.x & 31, g = lane / 4, j = lane & 3;
  float4* o = reinterpret_cast<float4*>(part);
  float2* stat = reinterpret_cast<float2*>(part + kRows * D * 4);
#pragma unroll
  for (int r = 0; r < 2; ++r) {
    const int row = g + 8 * r;
    if (j == 0) stat[row] = make_float2(s.m[r], s.l[2 * r]);
#pragma unroll
    for (int y = 0; y < 2; ++y)
#pragma unroll
      for (int i = 0; i < Running<D>::kN; i += 4) {
        const int q = j * (D / 16) + (y * Running<D>::kN + i) / 4;
        o[row * (D / 4) + part_at(row, q)] =
            make_float4(s.o[i][2 * r + y], s.o[i + 1][2 * r + y], s.o[i + 2][2 * r + y], s.o[i + 3][2 * r + y]);
      }
  }
}

__device__ __forceinline__ void store4(__nv_bfloat16* dst, float4 v, float k) {
  const __nv_bfloat162 a = __floats2bfloat162_rn(v.x * k, v.y * k), b = __floats2bfloat162_rn(v.z * k, v.w * k);
  *reinterpret_cast<uint2*>(dst) = make_uint2(*reinterpret_cast<const uint32_t*>(&a), *reinterpret_cast<const uint32_t*>(&b));
}

struct Segment {              // neighbouring parts of one item in this CTA
  int first, more;            // record of the first part, and how many warps follow with their first parts
  int slot, cta0, ctas;       // -1: the item is whole; else where its part goes, and the CTAs that share the item
  int last;                   // this CTA is the last of them to arrive
};

template <int D>
__global__ void __launch_bounds__(kWarps * 32, 1) attend_kernel(const __grid_constant__ AttendParams p) {
  extern __shared__ __align__(128) uint8_t smem[];
  using S = AttendSmem<D>;
  using U = CacheUnit<D>;
  __shared__ int warp_sum[kWarps];
  __shared__ Segment segments[kWarps + 1];
  __shared__ int n_segments, abort_flag;
  int* before = reinterpret_cast<int*>(smem + S::kBefore);
  Part* records = reinterpret_cast<Part*>(smem + S::kRecords);
  const int tid = threadIdx.x, warp = tid >> 5, lane = tid & 31;
  const uint32_t bars = smem_u32(smem + S::kBars) + warp * S::kStages * 8;
  const uint8_t* ring = smem + warp * S::kStages * S::kStageBytes;

  pdl_trigger();
  if (lane < S::kStages) mbar_init(bars + 8 * lane, 1);
  if (tid == 0) { abort_flag = 0; n_segments = 0; }
  if (lane < 2) records[2 * warp + lane].valid = 0;
  asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
  pdl_wait();

  const int total = Tiles::count_tiles<kWarps>(p, before, warp_sum, blockIdx.x == 0);
  if (total == 0) return;

  const int n_runs = min(total, static_cast<int>(gridDim.x) * kWarps);
  const Runs runs(total, n_runs);
  const int run0 = blockIdx.x * kWarps;
  if (run0 >= n_runs) return;
  const int cta_begin = runs.begin(run0), cta_end = runs.begin(min(run0 + kWarps, n_runs));

  if (run0 + warp < n_runs) {
    const int begin = runs.begin(run0 + warp), end = runs.begin(run0 + warp + 1);
    Item it = Tiles::item_at(p, before, begin);
    Item ahead = it;                                 // the item of the next tile to be requested
    int asked = begin;
    uint32_t absent_bits = 0;                        // four bits per stage
    // Lanes 0 to 7 each fetch one unit's keys or values.  The page numbers are read one request ahead.
    const int my_unit = lane >> 1;
    const size_t head_bytes = static_cast<size_t>(p.page_size / kUnit) * U::kBytes;
    const auto look = [&](int tile) {                // tile of the item `ahead`
      const int t = tile * kTile + my_unit * kUnit;
      return lane < 2 * kUnits && t < ahead.len ? p.page_table[static_cast<size_t>(ahead.b) * p.max_pages + (t >> p.page_shift)] : -1;
    };
    int page = look(asked - ahead.begin);
    const auto request = [&](int stage) {
      const int tile = asked - ahead.begin, t = tile * kTile + my_unit * kUnit;
      const bool wanted = lane < 2 * kUnits && t < ahead.len;
      const bool there = static_cast<unsigned>(page) < static_cast<unsigned>(p.n_pages);
      const uint8_t* src = p.cache + ((static_cast<size_t>(there ? page : 0) * p.Hkv + ahead.h) * 2 + (lane & 1)) * head_bytes +
                           ((t & (p.page_size - 1)) / kUnit) * U::kBytes;
      const uint32_t want = __ballot_sync(0xffffffffu, wanted), gone = __ballot_sync(0xffffffffu, wanted && !there);
      if (gone != 0 || absent_bits != 0) {
        const uint32_t bits = (gone & 1u) | (gone >> 1 & 2u) | (gone >> 2 & 4u) | (gone >> 3 & 8u);
        absent_bits = (absent_bits & ~(15u << (4 * stage))) | bits << (4 * stage);
        if (gone != 0 && lane == 0) atomicOr(p.status, TEMPO_STATUS_BAD_INDEX);
      }
      if (lane == 0) mbar_arrive_expect_tx(bars + 8 * stage, __popc(want) * U::kBytes);
      __syncwarp();
      if (wanted) bulk_load(smem_u32(ring + stage * S::kStageBytes + lane * U::kBytes), src, U::kBytes, bars + 8 * stage);
      if (++asked < end) {
        if (asked == ahead.begin + ahead.tiles) Tiles::next_item(p, ahead);
        page = look(asked - ahead.begin);
      }
    };
#pragma unroll 1
    for (int st = 0; st < S::kStages && asked < end; ++st) request(st);

    Running<D> s;
    begin_item<D>(p, it, s);
    int x = begin, stage = 0;
    uint32_t phase = 0;
    bool fine = true, late = false;
#pragma unroll 1
    while (true) {
      fine = __all_sync(0xffffffffu, mbar_wait(bars + 8 * stage, phase, &abort_flag, p.wait_ns));
      if (!fine) break;
      run_tile<D>(s, ring + stage * S::kStageBytes, (x - it.begin) * kTile, it.len, absent_bits >> (4 * stage) & 15u);
      __syncwarp();
      if (asked < end) request(stage);
      ++x;
      if (x == it.begin + it.tiles || x == end) {
        if (it.begin >= begin && x == it.begin + it.tiles) {
          store_item<D>(p, it, s);
        } else {
          // The run's first item keeps its part beside the ring.  A last one that is another waits until every warp of the CTA
          // has left the ring, and takes its place.
          const int at = it.begin <= begin ? 0 : 1;
          if (lane == 0) { records[2 * warp + at].item = it; records[2 * warp + at].valid = 1; }
          late = at == 1;
          if (!late) keep_part<D>(s, smem + S::kParts + warp * S::kPart);
        }
        if (x == end) break;
        Tiles::next_item(p, it);
        begin_item<D>(p, it, s);
      }
      if (++stage == S::kStages) { stage = 0; phase ^= 1; }
    }
    if (!fine) {                                     // let what was requested arrive before the memory goes
      if (lane == 0) atomicOr(p.status, TEMPO_STATUS_TIMEOUT);
      volatile int none = 0;
      for (int st = 0; st < S::kStages; ++st) mbar_wait(bars + 8 * st, phase ^ (st < stage ? 1u : 0u), &none, p.wait_ns);
    }
    __syncthreads();
    if (late) keep_part<D>(s, smem + warp * S::kPart);
  } else {
    __syncthreads();
  }
  __syncthreads();

  // Which parts belong together: those of neighbouring warps with one item.
  if (warp == 0) {
    const int w = lane >> 1;
    bool leads = w < kWarps && records[lane].valid != 0;
    int more = 0;
    if (leads) {
      const int begin = records[lane].item.begin;
      const auto same = [&](int r) { return records[r].valid != 0 && records[r].item.begin == begin; };
      if ((lane & 1) == 0 && w > 0 && (same(lane - 1) || same(lane - 2))) leads = false;
      while (leads && w + 1 + more < kWarps && same(2 * (w + 1 + more))) ++more;
    }
    const uint32_t all = __ballot_sync(0xffffffffu, leads);
    if (leads) {
      const Item& it = records[lane].item;
      Segment& g = segments[__popc(all & ((1u << lane) - 1u))];
      g.first = lane;
      g.more = more;
      g.slot = it.begin >= cta_begin && it.begin + it.tiles <= cta_end ? -1 : it.begin <= cta_begin ? 0 : 1;
      g.cta0 = runs.of(it.begin) / kWarps;
      g.ctas = runs.of(it.begin + it.tiles - 1) / kWarps - g.cta0 + 1;
    }
    if (lane == 0) n_segments = __popc(all);
  }
  __syncthreads();

  constexpr int kQuads = kRows * D / 4;
  const int segs = n_segments;
  for (int task = tid; task < segs * kQuads; task += kWarps * 32) {
    const Segment& g = segments[task / kQuads];
    const int row = task % kQuads / (D / 4), q = task % (D / 4);
    const int w0 = g.first >> 1;
    const auto part = [&](int i) -> const uint8_t* {
      return (i == 0 && (g.first & 1)) ? smem + w0 * S::kPart : smem + S::kParts + (w0 + i) * S::kPart;
    };
    float m = -INFINITY;
    for (int i = 0; i <= g.more; ++i) m = fmaxf(m, reinterpret_cast<const float2*>(part(i) + kRows * D * 4)[row].x);
    const float ref = m == -INFINITY ? 0.0f : m;
    float l = 0.0f;
    float4 o = make_float4(0.0f, 0.0f, 0.0f, 0.0f);
    for (int i = 0; i <= g.more; ++i) {
      const float2 st = reinterpret_cast<const float2*>(part(i) + kRows * D * 4)[row];
      const float4 v = reinterpret_cast<const float4*>(part(i))[row * (D / 4) + part_at(row, q)];
      const float k = exp2_fast(st.x - ref);
      l += st.y * k;
      o.x += v.x * k; o.y += v.y * k; o.z += v.z * k; o.w += v.w * k;
    }
    if (g.slot < 0) {
      const Item& it = records[g.first].item;
      if (it.row0 + row < it.n * p.group) store4(out_row(p, it, row) + 4 * q, o, l == 0.0f ? 0.0f : 1.0f / l);
    } else {
      const size_t at = (static_cast<size_t>(blockIdx.x) * 2 + g.slot) * kRows + row;
      __stcg(reinterpret_cast<float4*>(p.part + at * D) + q, o);
      if (q == 0) __stcg(reinterpret_cast<float2*>(p.stats) + at, make_float2(m, l));
    }
  }
  __threadfence();
  __syncthreads();
  if (tid < segs && segments[tid].slot >= 0) {
    Segment& g = segments[tid];
    g.last = atomicAdd(p.counters + g.cta0, 1u) == static_cast<unsigned>(g.ctas) - 1u;
    if (g.last) p.counters[g.cta0] = 0;
  }
  __syncthreads();

  // Items shared with other CTAs, by the last of them: the parts in the order of the CTAs, whoever it is.
  float* weights = reinterpret_cast<float*>(smem);
  for (int i = 0; i < segs; ++i) {
    const Segment g = segments[i];
    if (g.slot < 0 || !g.last) continue;
    __threadfence();
    const Item it = records[g.first].item;
    const int begin0 = runs.begin(g.cta0 * kWarps);
    const auto row_at = [&](int c, int row) {
      return (static_cast<size_t>(g.cta0 + c) * 2 + (c == 0 && it.begin > begin0 ? 1 : 0)) * kRows + row;
    };
    for (int row = warp; row < kRows; row += kWarps) {
      float m = -INFINITY;
      for (int c = lane; c < g.ctas; c += 32) m = fmaxf(m, __ldcg(reinterpret_cast<const float2*>(p.stats) + row_at(c, row)).x);
#pragma unroll
      for (int d = 16; d > 0; d /= 2) m = fmaxf(m, __shfl_xor_sync(0xffffffffu, m, d));
      const float ref = m == -INFINITY ? 0.0f : m;
      float l = 0.0f;
      for (int c = lane; c < g.ctas; c += 32) {
        const float2 st = __ldcg(reinterpret_cast<const float2*>(p.stats) + row_at(c, row));
        const float k = exp2_fast(st.x - ref);
        weights[c * kRows + row] = k;
        l += st.y * k;
      }
#pragma unroll
      for (int d = 16; d > 0; d /= 2) l += __shfl_xor_sync(0xffffffffu, l, d);
      if (lane == 0) weights[kAttendMaxSms * kRows + row] = l;
    }
    __syncthreads();
    for (int task = tid; task < kQuads; task += kWarps * 32) {
      const int row = task / (D / 4), q = task % (D / 4);
      float4 o = make_float4(0.0f, 0.0f, 0.0f, 0.0f);
#pragma unroll 8
      for (int c = 0; c < g.ctas; ++c) {
        const float4 v = __ldcg(reinterpret_cast<const float4*>(p.part + row_at(c, row) * D) + q);
        const float k = weights[c * kRows + row];
        o.x += v.x * k; o.y += v.y * k; o.z += v.z * k; o.w += v.w * k;
      }
      const float l = weights[kAttendMaxSms * kRows + row];
      if (it.row0 + row < it.n * p.group) store4(out_row(p, it, row) + 4 * q, o, l == 0.0f ? 0.0f : 1.0f / l);
    }
    __syncthreads();
  }
}

template <int D>
cudaError_t launch_attend_as(const AttendParams& p, int num_sms, cudaStream_t stream) {
  using S = AttendSmem<D>;
  static_assert(S::kBefore + (kAttendMaxB + 1) * 4 + 1024 <= 227 * 1024, "shared memory of one SM");
  static std::atomic<unsigned long long> done{0};
  const cudaError_t e = smem_limit_once(attend_kernel<D>, S::bytes(kAttendMaxB), done);
  if (e != cudaSuccess) return e;
  return launch_pdl(attend_kernel<D>, dim3(num_sms), dim3(kWarps * 32), S::bytes(p.B), stream, p);
}

}  // namespace

AttendLayout attend_layout(int D) {
  const auto round = [](size_t v) { return (v + 255) / 256 * 256; };
  AttendLayout L;
  L.off_counters = 0;
  L.off_stats = round(kAttendMaxSms * sizeof(unsigned int));
  L.off_out = L.off_stats + round(static_cast<size_t>(kAttendMaxSms) * 2 * kAttendManyRows * 8);
  L.total = L.off_out + static_cast<size_t>(kAttendMaxSms) * 2 * kAttendManyRows * D * 4;
  return L;
}

// Sequences of up to kFewRows rows are this kernel's, longer ones the other's.
constexpr int kFewRows = 64;

cudaError_t launch_attend(AttendParams p, int max_q, int D, int num_sms, cudaStream_t stream) {
  const bool many = static_cast<int64_t>(max_q) * p.group > kFewRows;
  p.rows_above = 0;
  p.rows_most = many ? kFewRows : INT32_MAX;         // without the other kernel this one takes whatever comes
  cudaError_t e = D == 64 ? launch_attend_as<64>(p, num_sms, stream) : launch_attend_as<128>(p, num_sms, stream);
  if (e != cudaSuccess || !many) return e;
  p.rows_above = kFewRows;
  p.rows_most = INT32_MAX;
  return launch_attend_many(p, D, num_sms, stream);
}

}  // namespace tempo
