// Attention over the 4-bit paged cache (tempo_attend) for few queries of a sequence; attend_many.cu has the other kernel.
//
//   out[i, h] = sum_t p[t] V[t] / sum_t p[t],  p[t] = exp(scale <q, K[t]> - m),  t <= the query's own position
//
// A key head's queries (the heads of its group, and the new tokens of the sequence) are the rows of an item, 8 or 16 of them; a
// cached byte is read once for all.  One pass over the tokens with the running maximum and sum; 32-bit statistics, weights rounded
// to fp16 where they meet V (their sum is that of the rounded ones).
//
// An SM takes in the cache at 23 bytes a clock, which leaves 2.8 instruction slots of a lane for an element.  So codes go from
// shared memory to registers and are decoded there into operands of the matrix instruction (m16n8k16, 32-bit sums) at 11
// instructions for 8 elements; a decoded copy in shared memory for tcgen05 would move 2 bytes of an element in and 2 out, 184 bytes
// a clock where the SM has 128.  Keys and values are the 16-row operand, so that 8 queries cost half the products of 16.  The order
// of a sum over d or t is free: a lane's 16-byte load is what it needs, of keys 32 neighbouring elements (one group: one scale) of a
// token, of values 16 neighbouring elements of two tokens side by side in a word's halves.
// What bounds it: 64 sequences of up to 8192 tokens (16 rows; 193 MB) take 64.9 us, 45 % of a copy's rate, of which about 12 are
// start and end; 16 tokens of a head cost a scheduler 321 instructions in 670 clocks, 119 of them on the pipe of logic, 127 on the one
// of fp16 sums, 34 matrix instructions of 8 clocks: with its two warps it waits for results half of the time.  2 sequences of 131072
// (4 rows; 245 MB) 57.7 us, 65 %: 286 instructions, 17 matrix instructions, in 440 clocks of a scheduler's three warps, of which this mix
// of instructions alone takes 370.  One sequence of 1500: 9.9 us, a chain of latencies (tiles counted 1, queries and first page 2, one
// tile 2.5, merges 1, arrival and join 2.5 us).
//
// Work is dealt in tiles of 64 tokens: the tiles of all items in one row, cut into equal runs, one for each warp of the launch,
// whatever the lengths.  A warp streams its run through a tile of shared memory of its own (16-byte asynchronous copies: a bulk copy
// costs the warp that issues it 200 to 400 clocks, a tenth of a tile) and waits for nobody; parts of items that were cut are joined in
// shared memory after the CTA's last tile, and across CTAs by the one that arrives last, in a fixed order.
#include <algorithm>

#include "attend_common.cuh"

namespace tempo {

namespace {

// The kernel's form for items of 8 NR rows.  Warps: as many as have their registers without a spill, which would go to L2 (shared memory
// leaves no L1): 16 rows and 12 warps took 88 us where 8 take 64 (64 x 8192); 8 rows and 12 warps 57, 16 warps 61, 8 warps 61
// (2 x 131072), for D = 64 16 warps 22.5 and 12 warps 27 (37 x 2999).
template <int D_, int NR_, bool PADDED>
struct Few {
  static constexpr int D = D_, NR = NR_, kRows = 8 * NR;
  static constexpr int kWarps = NR == 2 ? 8 : D == 128 ? 12 : 16, kTile = 64, kUnits = kTile / kUnit;
  using Tiles = Cut<kRows, kTile, PADDED>;
  using Item = typename Tiles::Item;
  static constexpr int kStageBytes = 2 * kUnits * CacheUnit<D>::kBytes;   // the keys of its units, then the values
  static constexpr int kRing = kWarps * kStageBytes;
  static constexpr int kPart = kRows * D * 4 + kRows * 8;            // O, then (m, l) of each row
  static constexpr int kParts = kRing;
  static constexpr int kBefore = kParts + kWarps * kPart;
  static_assert(kRing >= kWarps * kPart, "the second parts take the ring's place");
  static int bytes(int B) { return kBefore + (B + 1) * 4; }
};

__device__ __forceinline__ void mma_f16(float (&c)[4], uint32_t a0, uint32_t a1, uint32_t a2, uint32_t a3, uint32_t b0, uint32_t b1) {
  asm("mma.sync.aligned.m16n8k16.row.col.f32.f16.f16.f32 {%0, %1, %2, %3}, {%4, %5, %6, %7}, {%8, %9}, {%0, %1, %2, %3};"
      : "+f"(c[0]), "+f"(c[1]), "+f"(c[2]), "+f"(c[3]) : "r"(a0), "r"(a1), "r"(a2), "r"(a3), "r"(b0), "r"(b1));
}
// An 8 x 8 matrix of 16-bit numbers, two neighbours of row lane / 4 in each lane, transposed.
__device__ __forceinline__ uint32_t transpose8(uint32_t v) {
  uint32_t r;
  asm("movmatrix.sync.aligned.m8n8.trans.b16 %0, %1;" : "=r"(r) : "r"(v));
  return r;
}
__device__ __forceinline__ void copy_async_16(uint32_t dst, const void* src) {
  asm volatile("cp.async.cg.shared.global [%0], [%1], 16;" ::"r"(dst), "l"(src) : "memory");
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
__device__ __forceinline__ int part_at(int row, int q) { return q ^ (row >> 1 & 3); }

// A warp's running state of one item.  Lane (g, j) = (lane / 4, lane % 4) keeps the rows 2 j and 2 j + 1 of each eight.
template <class F>
struct Running {
  static constexpr int kN = F::D / 16;               // products with 16 elements of a value row
  uint32_t q[F::NR][F::D / 16][2];                   // B operands of the scores: row g, elements j D/4 to (j+1) D/4 - 1
  float f[F::NR][2];                                 // score = f * (sum of products), in units of log2; above zero
  int limit[F::NR][2], least;                        // last token that each row sees; the least over all rows
  float m[F::NR][2];
  bool far;                                          // far_scores of some row of the warp
  float l[F::NR][4];                                 // sums of the weights: rows in [0] and [1]
  float o[F::NR][kN][4];                             // elements g D/8 + 2 i (in [0], [1]) and + 2 i + 1 (in [2], [3])
};

// A lane's share of an item's queries, as they are: of row g of each eight the elements j D/4 to (j+1) D/4 - 1.
template <class F>
__device__ __forceinline__ void load_queries(const AttendParams& p, const typename F::Item& it, uint4 (&u)[F::NR][F::D / 32]) {
  const int lane = threadIdx.x & 31, g = lane / 4, j = lane & 3;
#pragma unroll
  for (int r = 0; r < F::NR; ++r) {
    const int row = it.row0 + 8 * r + g;
    const bool in = row < it.n * p.group;
    const int qi = in ? row / p.group : 0, head = in ? it.h * p.group + row - qi * p.group : 0;
    const __nv_bfloat16* src = p.q + static_cast<size_t>(it.q0 + qi) * p.ld_q + static_cast<size_t>(head) * p.hd_q + j * (F::D / 4);
#pragma unroll
    for (int w = 0; w < F::D / 32; ++w) u[r][w] = in ? __ldg(reinterpret_cast<const uint4*>(src) + w) : make_uint4(0, 0, 0, 0);
  }
}

template <class F>
__device__ __forceinline__ void begin_item(const AttendParams& p, const typename F::Item& it, const uint4 (&u)[F::NR][F::D / 32], Running<F>& s) {
  constexpr int W = F::D / 32;                       // 8-element words of a lane
  const int lane = threadIdx.x & 31, j = lane & 3;
#pragma unroll
  for (int r = 0; r < F::NR; ++r) {
    float x[W][8];
    float top = 0.0f;
    bool odd = false;
#pragma unroll
    for (int w = 0; w < W; ++w) {
      const uint32_t v[4] = {u[r][w].x, u[r][w].y, u[r][w].z, u[r][w].w};
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
    float up, f;
    row_factors(top, odd, p.scale_log2, up, f);
#pragma unroll
    for (int w = 0; w < W; ++w)
#pragma unroll
      for (int y = 0; y < 2; ++y) {                  // the pairs (n, n + 4) of decode8, two to a matrix instruction
        s.q[r][2 * w + y][0] = as_u32(__floats2half2_rn(x[w][2 * y] * up, x[w][2 * y + 4] * up));
        s.q[r][2 * w + y][1] = as_u32(__floats2half2_rn(x[w][2 * y + 1] * up, x[w][2 * y + 5] * up));
      }
#pragma unroll
    for (int y = 0; y < 2; ++y) {
      s.f[r][y] = __shfl_sync(0xffffffffu, f, (2 * j + y) * 4);
      const int mine = it.row0 + 8 * r + 2 * j + y;
      s.limit[r][y] = it.len - it.n + min(mine / p.group, it.n - 1);
      s.m[r][y] = -INFINITY;
    }
    s.l[r][0] = s.l[r][1] = s.l[r][2] = s.l[r][3] = 0.0f;
#pragma unroll
    for (int i = 0; i < Running<F>::kN; ++i) { s.o[r][i][0] = s.o[r][i][1] = s.o[r][i][2] = s.o[r][i][3] = 0.0f; }
  }
  s.least = it.len - it.n + it.row0 / p.group;
  s.far = false;
}

// One tile is the tokens [t0, t0 + kTile) of the item, its keys and its values at `stage`.  Here its scores: c[k][r], of the tokens
// 16 k + g (in [0], [1]) and 16 k + 8 + g, rows 2 j and 2 j + 1 of eight r.  `absent`: bits of its units whose page is not in the cache.
template <class F>
__device__ __forceinline__ void run_keys(const Running<F>& s, const Decode& dc, const uint8_t* stage, int t0, uint32_t absent,
                                         float (&c)[F::kUnits][F::NR][4]) {
  using U = CacheUnit<F::D>;
  constexpr int D = F::D, W = D / 32, NR = F::NR;
  const int lane = threadIdx.x & 31, g = lane / 4, j = lane & 3;
#pragma unroll
  for (int k0 = 0; k0 < F::kUnits; k0 += 2) {        // two units side by side
    uint32_t w[2][2][W], sc[2][2], b[2][2];
#pragma unroll
    for (int k = 0; k < 2; ++k) {
      const uint8_t* unit = stage + (k0 + k) * U::kBytes;
#pragma unroll
      for (int x = 0; x < 2; ++x) {
        const int at = x * 8 + g;
        load_words<W>(unit + at * U::kKeyRow + j * (D / 8), w[k][x]);
        group_params(*reinterpret_cast<const uint16_t*>(unit + U::kCodes + at * U::kKeyParams + (D == 128 ? j : j / 2) * 2) * 0x10001u,
                     sc[k][x], b[k][x]);
      }
#pragma unroll
      for (int r = 0; r < NR; ++r) c[k0 + k][r][0] = c[k0 + k][r][1] = c[k0 + k][r][2] = c[k0 + k][r][3] = 0.0f;
    }
#pragma unroll
    for (int y = 0; y < W; ++y)
#pragma unroll
      for (int k = 0; k < 2; ++k) {
        uint32_t v[2][4];
#pragma unroll
        for (int x = 0; x < 2; ++x) decode8(dc, w[k][x][y], sc[k][x], b[k][x], v[x]);
#pragma unroll
        for (int u = 0; u < 2; ++u)
#pragma unroll
          for (int r = 0; r < NR; ++r)
            mma_f16(c[k0 + k][r], v[0][2 * u], v[1][2 * u], v[0][2 * u + 1], v[1][2 * u + 1], s.q[r][2 * y + u][0], s.q[r][2 * y + u][1]);
      }
  }
  if (absent != 0) {
#pragma unroll
    for (int k = 0; k < F::kUnits; ++k)
      if (absent >> k & 1) {
#pragma unroll
        for (int r = 0; r < NR; ++r) c[k][r][0] = c[k][r][1] = c[k][r][2] = c[k][r][3] = __uint_as_float(0x7fc00000u);
      }
  }
  if (t0 + F::kTile - 1 > s.least) {
#pragma unroll
    for (int k = 0; k < F::kUnits; ++k)
#pragma unroll
      for (int r = 0; r < NR; ++r)
#pragma unroll
        for (int x = 0; x < 4; ++x)
          if (t0 + 16 * k + 8 * (x / 2) + g > s.limit[r][x & 1]) c[k][r][x] = -INFINITY;
  }
}

// Scores to weights, as the B operands of the output: w8[k][r] of row g, tokens 2 j, + 1 and 8 + 2 j, + 1 of unit k.
template <class F>
__device__ __forceinline__ void run_weights(Running<F>& s, float (&c)[F::kUnits][F::NR][4], uint32_t (&w8)[F::kUnits][F::NR][2]) {
  constexpr int NR = F::NR;
  bool raise = false;
  float top[NR][2];
#pragma unroll
  for (int r = 0; r < NR; ++r)
#pragma unroll
    for (int y = 0; y < 2; ++y) {
      float t = fmaxf(c[0][r][y], c[0][r][y + 2]);
#pragma unroll
      for (int k = 1; k < F::kUnits; ++k) t = fmaxf(t, fmaxf(c[k][r][y], c[k][r][y + 2]));
      top[r][y] = t * s.f[r][y];
      raise = raise || top[r][y] > s.m[r][y] + kSlack;
    }
  // A maximum that has grown little stays: weights up to 2^15 are in fp16's range, and O is left alone.
  if (__any_sync(0xffffffffu, raise)) {
    bool far = false;
#pragma unroll
    for (int r = 0; r < NR; ++r)
#pragma unroll
      for (int y = 0; y < 2; ++y) {
        float t = top[r][y];
#pragma unroll
        for (int d = 4; d < 32; d *= 2) t = fmaxf(t, __shfl_xor_sync(0xffffffffu, t, d));
        const float m = t > s.m[r][y] + kSlack ? t : s.m[r][y];
        const float k = m == s.m[r][y] ? 1.0f : exp2_fast(s.m[r][y] - m);
        s.m[r][y] = m;
        far = far || far_scores(m);
        s.l[r][y] *= k;
#pragma unroll
        for (int i = 0; i < Running<F>::kN; ++i) { s.o[r][i][y] *= k; s.o[r][i][y + 2] *= k; }
      }
    s.far = __any_sync(0xffffffffu, far);
  }
  float f[NR][2], less[NR][2];
#pragma unroll
  for (int r = 0; r < NR; ++r)
#pragma unroll
    for (int y = 0; y < 2; ++y) { f[r][y] = s.f[r][y]; less[r][y] = s.m[r][y] == -INFINITY ? 0.0f : kBias - s.m[r][y]; }
  if (s.far) {
#pragma unroll
    for (int r = 0; r < NR; ++r)
#pragma unroll
      for (int y = 0; y < 2; ++y)
        if (far_scores(s.m[r][y])) {
#pragma unroll
          for (int k = 0; k < F::kUnits; ++k)
#pragma unroll
            for (int x = y; x < 4; x += 2) c[k][r][x] = from_far(c[k][r][x], f[r][y], s.m[r][y]);
          f[r][y] = 1.0f;
          less[r][y] = kBias;
        }
  }
#pragma unroll
  for (int r = 0; r < NR; ++r)
#pragma unroll
    for (int k = 0; k < F::kUnits; ++k)
#pragma unroll
      for (int x = 0; x < 2; ++x)
        w8[k][r][x] = transpose8(as_u32(__floats2half2_rn(exp2_fast(fmaf(c[k][r][2 * x], f[r][0], less[r][0])),
                                                          exp2_fast(fmaf(c[k][r][2 * x + 1], f[r][1], less[r][1])))));
}

// Values of a tile of which some row does not see all, before they are decoded.
template <class F>
__device__ __forceinline__ void mend_values(uint8_t* stage, int t0, int len) {
  using U = CacheUnit<F::D>;
  constexpr int kWords = U::kParams / 4, kPair = U::kPairParams / 4;     // of a unit, of two tokens
#pragma unroll
  for (int k = 0; k < F::kUnits; ++k)
#pragma unroll
    for (int i = threadIdx.x & 31; i < kWords; i += 32) {
      uint32_t* w = reinterpret_cast<uint32_t*>(stage + k * U::kBytes + U::kCodes) + i;
      *w = edge_params(*w, len - (t0 + 16 * k + 2 * (i / kPair)));
    }
  __syncwarp();
}

template <class F>
__device__ __forceinline__ void run_values(Running<F>& s, const Decode& dc, const uint8_t* stage, const uint32_t (&w8)[F::kUnits][F::NR][2]) {
  using U = CacheUnit<F::D>;
  constexpr int D = F::D, W = D / 32, NR = F::NR;
  const int lane = threadIdx.x & 31, g = lane / 4, j = lane & 3;
#pragma unroll
  for (int k = 0; k < F::kUnits; ++k) {
    const uint8_t* unit = stage + k * U::kBytes;
    uint32_t w[2][W], sc[2], b[2];
#pragma unroll
    for (int x = 0; x < 2; ++x) {                    // tokens 16 k + 2 pair, + 1
      const int pair = 4 * x + j;
      load_words<W>(unit + pair * U::kPairRow + g * (D / 8), w[x]);
      group_params(*reinterpret_cast<const uint32_t*>(unit + U::kCodes + pair * U::kPairParams + (D == 128 ? g / 2 : g / 4) * 4), sc[x], b[x]);
    }
#pragma unroll
    for (int r = 0; r < NR; ++r)                     // times 1: the sum is that of the weights as they meet V
      mma_f16(s.l[r], 0x3c003c00u, 0x3c003c00u, 0x3c003c00u, 0x3c003c00u, w8[k][r][0], w8[k][r][1]);
#pragma unroll
    for (int y = 0; y < W; ++y) {
      uint32_t v0[4], v1[4];
      decode8(dc, w[0][y], sc[0], b[0], v0);
      decode8(dc, w[1][y], sc[1], b[1], v1);
#pragma unroll
      for (int h = 0; h < 2; ++h)
#pragma unroll
        for (int r = 0; r < NR; ++r)
          mma_f16(s.o[r][2 * y + h], v0[2 * h], v0[2 * h + 1], v1[2 * h], v1[2 * h + 1], w8[k][r][0], w8[k][r][1]);
    }
  }
}

template <class Item>
__device__ __forceinline__ __nv_bfloat16* out_row(const AttendParams& p, const Item& it, int row) {
  const int r = it.row0 + row;
  return p.out + static_cast<size_t>(it.q0 + r / p.group) * p.ld_out + static_cast<size_t>(it.h * p.group + r % p.group) * p.hd_out;
}

// A whole item's result from the registers: of its rows a lane has the elements g D/8 to (g+1) D/8 - 1.
template <class F>
__device__ __forceinline__ void store_item(const AttendParams& p, const typename F::Item& it, Running<F>& s) {
  const int lane = threadIdx.x & 31, g = lane / 4, j = lane & 3;
#pragma unroll
  for (int r = 0; r < F::NR; ++r)
#pragma unroll
    for (int y = 0; y < 2; ++y) {
      const int row = 8 * r + 2 * j + y;
      if (it.row0 + row >= it.n * p.group) continue;
      const float k = s.l[r][y] == 0.0f ? 0.0f : 1.0f / s.l[r][y];
      uint4* dst = reinterpret_cast<uint4*>(out_row(p, it, row) + g * (F::D / 8));
#pragma unroll
      for (int i = 0; i < Running<F>::kN; i += 4) {
        uint32_t v[4];
#pragma unroll
        for (int x = 0; x < 4; ++x) {
          const __nv_bfloat162 h = __floats2bfloat162_rn(s.o[r][i + x][y] * k, s.o[r][i + x][y + 2] * k);
          v[x] = *reinterpret_cast<const uint32_t*>(&h);
        }
        dst[i / 4] = make_uint4(v[0], v[1], v[2], v[3]);
      }
    }
}

template <class F>
__device__ __forceinline__ void keep_part(Running<F>& s, uint8_t* part) {
  const int lane = threadIdx.x & 31, g = lane / 4, j = lane & 3;
  float4* o = reinterpret_cast<float4*>(part);
  float2* stat = reinterpret_cast<float2*>(part + F::kRows * F::D * 4);
#pragma unroll
  for (int r = 0; r < F::NR; ++r)
#pragma unroll
    for (int y = 0; y < 2; ++y) {
      const int row = 8 * r + 2 * j + y;
      if (g == 0) stat[row] = make_float2(s.m[r][y], s.l[r][y]);
#pragma unroll
      for (int i = 0; i < Running<F>::kN; i += 2)
        o[row * (F::D / 4) + part_at(row, g * (F::D / 32) + i / 2)] =
            make_float4(s.o[r][i][y], s.o[r][i][y + 2], s.o[r][i + 1][y], s.o[r][i + 1][y + 2]);
    }
}

__device__ __forceinline__ void store4(__nv_bfloat16* dst, float4 v, float k) {
  const __nv_bfloat162 a = __floats2bfloat162_rn(v.x * k, v.y * k), b = __floats2bfloat162_rn(v.z * k, v.w * k);
  *reinterpret_cast<uint2*>(dst) = make_uint2(*reinterpret_cast<const uint32_t*>(&a), *reinterpret_cast<const uint32_t*>(&b));
}

// Parts of an item one after the other: their sums under the common maximum, for eight elements of a row as two quads.
struct Merged {
  float m = -INFINITY, l = 0.0f;
  float4 o[2] = {make_float4(0.0f, 0.0f, 0.0f, 0.0f), make_float4(0.0f, 0.0f, 0.0f, 0.0f)};
  __device__ __forceinline__ float factor() const { return l == 0.0f ? 0.0f : 1.0f / l; }
};
// `stat(i)` and `quad(i, y)` read part i's (m, l) of the row and quad y; BATCH parts' loads are in flight together.
template <int BATCH, typename Stat, typename Quad>
__device__ __forceinline__ Merged merge(int n, Stat stat, Quad quad) {
  Merged r;
  for (int i0 = 0; i0 < n; i0 += BATCH) {
    float2 st[BATCH];
    float4 v[BATCH][2];
#pragma unroll
    for (int i = 0; i < BATCH; ++i)
      if (i0 + i < n) { st[i] = stat(i0 + i); v[i][0] = quad(i0 + i, 0); v[i][1] = quad(i0 + i, 1); }
    float m = r.m;
#pragma unroll
    for (int i = 0; i < BATCH; ++i)
      if (i0 + i < n) m = fmaxf(m, st[i].x);
    const float ref = m == -INFINITY ? 0.0f : m, before = exp2_fast(r.m - ref);
    r.m = m;
    r.l *= before;
#pragma unroll
    for (int y = 0; y < 2; ++y) { r.o[y].x *= before; r.o[y].y *= before; r.o[y].z *= before; r.o[y].w *= before; }
#pragma unroll
    for (int i = 0; i < BATCH; ++i)
      if (i0 + i < n) {
        const float k = exp2_fast(st[i].x - ref);
        r.l += st[i].y * k;
#pragma unroll
        for (int y = 0; y < 2; ++y) {
          r.o[y].x += v[i][y].x * k; r.o[y].y += v[i][y].y * k; r.o[y].z += v[i][y].z * k; r.o[y].w += v[i][y].w * k;
        }
      }
  }
  return r;
}

template <class Item>
struct Segment {              // neighbouring parts of one item in this CTA
  Item item;
  int warp, late, more;       // the first part is that warp's (its late one or its first), then the first parts of so many warps behind it
  int slot, cta0, ctas;       // -1: the item is whole; else where its part goes, and the CTAs that share the item
  int last;                   // this CTA is the last of them to arrive
};

template <class F>
__global__ void __launch_bounds__(F::kWarps * 32, 1) attend_kernel(const __grid_constant__ AttendParams p) {
  extern __shared__ __align__(128) uint8_t smem[];
  using Item = typename F::Item;
  using Tiles = typename F::Tiles;
  using U = CacheUnit<F::D>;
  constexpr int D = F::D, kWarps = F::kWarps, kRows = F::kRows, kTile = F::kTile, kUnits = F::kUnits;
  __shared__ int warp_sum[kWarps];
  __shared__ Segment<Item> segments[kWarps + 1];
  __shared__ int n_segments;
  int* before = reinterpret_cast<int*>(smem + F::kBefore);
  const int tid = threadIdx.x, warp = tid >> 5, lane = tid & 31;
  uint8_t* ring = smem + warp * F::kStageBytes;

  pdl_trigger();
  if (tid == 0) n_segments = 0;
  pdl_wait();

  const int total = Tiles::template count_tiles<kWarps>(p, before, warp_sum, blockIdx.x == 0);
  if (total == 0) return;

  // Few tiles go to more CTAs of fewer warps: a warp alone on its scheduler is three times as fast.
  const int warps = min(kWarps, max(4, (total + static_cast<int>(gridDim.x) - 1) / static_cast<int>(gridDim.x)));
  const int n_runs = min(total, static_cast<int>(gridDim.x) * warps);
  const Runs runs(total, n_runs);
  const int run0 = blockIdx.x * warps;
  if (run0 >= n_runs) return;

  if (warp < warps && run0 + warp < n_runs) {
    const int begin = runs.begin(run0 + warp), end = runs.begin(run0 + warp + 1);
    Item it = Tiles::item_at(p, before, begin);

    // What is requested next.  A tile's units lie in runs of `together` in one page; a lane keeps the number (through the whole
    // cache, in 32 bits) of one run's first key unit.  Page numbers are read one tile ahead.
    Item ahead = it;
    int asked = begin, unit, units;                  // the run's first unit in the sequence, and how many the sequence has
    int left;                                        // units from the requested tile's first on
    const int32_t* pages;
    uint32_t head, number, absent;                   // absent: units of the requested tile whose page is not in the cache
    const int unit_shift = p.page_shift - 4, unit_mask = (1 << unit_shift) - 1;
    const int together = min(kUnits, 1 << unit_shift), n_parts = kUnits / together, shift_together = min(unit_shift, 2);
    static_assert(kUnits == 4, "log2 of the largest run");
    const uint32_t page_units = static_cast<uint32_t>(p.Hkv) << (unit_shift + 1);
    const size_t to_values = static_cast<size_t>(1 << unit_shift) * U::kBytes;
    const auto enter = [&]() {
      unit = (asked - ahead.begin) * kUnits + (lane & (n_parts - 1)) * together;
      units = (ahead.len + kUnit - 1) / kUnit;
      pages = p.page_table + static_cast<size_t>(ahead.b) * p.max_pages;
      head = static_cast<uint32_t>(ahead.h * 2) << unit_shift;
    };
    const auto look = [&]() { return unit < units ? pages[unit >> unit_shift] : 0; };
    enter();
    int page = look();
    const auto locate = [&]() {                      // the tile `asked`, and a look at the next
      asm volatile("" : "+r"(page));                 // nothing is computed from it, and so waited for, before this point
      const bool there = static_cast<unsigned>(page) < static_cast<unsigned>(p.n_pages);
      const uint32_t gone = __ballot_sync(0xffffffffu, !there);
      number = (there ? static_cast<uint32_t>(page) : 0u) * page_units + head + (unit & unit_mask);
      left = units - __shfl_sync(0xffffffffu, unit, 0);
      absent = 0;
      if (gone != 0) {
#pragma unroll
        for (int k = 0; k < kUnits; ++k) absent |= (gone >> (k / together) & 1u) << k;
        if (lane == 0) atomicOr(p.status, TEMPO_STATUS_BAD_INDEX);
      }
      unit += kUnits;
      if (++asked < end) {
        if (asked == ahead.begin + ahead.tiles) {
          Tiles::next_item(p, before, ahead);
          enter();
        }
        page = look();
      }
    };
    const auto request = [&](int kv) {               // keys or values of the tile that was located
      constexpr int kRun = kUnits * U::kBytes;
      const uint32_t dst = smem_u32(ring) + kv * kRun + lane * 16;
      const uint8_t* from = p.cache + kv * to_values;
      if (n_parts == 1) {                            // units of the page behind the sequence's last come along
        const uint8_t* src = from + static_cast<size_t>(number) * U::kBytes + lane * 16;
#pragma unroll
        for (int at = 0; at < kRun; at += 512)
          if (at + 512 <= kRun || at + lane * 16 < kRun) copy_async_16(dst + at, src + at);
      } else {
#pragma unroll
        for (int at = 0; at < kRun; at += 512) {
          const int k = (at + lane * 16) / U::kBytes;                    // the unit of this lane's 16 bytes
          const uint32_t first = __shfl_sync(0xffffffffu, number, k >> shift_together) + (k & (together - 1));
          if (k < left && k < kUnits) copy_async_16(dst + at, from + static_cast<size_t>(first) * U::kBytes + (at + lane * 16 - k * U::kBytes));
        }
      }
    };

    // A tile's keys make room for the next one's as soon as its scores are there, its values when its output is: either load has
    // the other half's work to hide behind.
    const Decode dc;
    Running<F> s;
    uint4 raw[F::NR][D / 32];
    load_queries<F>(p, it, raw);                     // asked for before the cache, so as not to queue behind it
    locate();
    request(0);
    cp_async_commit();
    request(1);
    cp_async_commit();
    begin_item<F>(p, it, raw, s);
    int x = begin;
    bool late = false;
#pragma unroll 1
    while (true) {
      const int t0 = (x - it.begin) * kTile;
      const bool more = asked < end;
      float c[kUnits][F::NR][4];
      uint32_t w8[kUnits][F::NR][2];
      cp_async_wait<1>();
      __syncwarp();
      run_keys<F>(s, dc, ring, t0, absent, c);
      __syncwarp();
      if (more) {
        locate();
        request(0);
      }
      cp_async_commit();
      run_weights<F>(s, c, w8);
      cp_async_wait<1>();
      __syncwarp();
      if (t0 + kTile - 1 > s.least) mend_values<F>(ring + kUnits * U::kBytes, t0, it.len);
      run_values<F>(s, dc, ring + kUnits * U::kBytes, w8);
      __syncwarp();
      if (more) request(1);
      cp_async_commit();
      ++x;
      if (x == it.begin + it.tiles || x == end) {
        if (it.begin >= begin && x == it.begin + it.tiles) {
          store_item<F>(p, it, s);
        } else {
          // The run's first item keeps its part beside the ring.  A last one that is another waits until every warp of the CTA
          // has left the ring, and takes its place.
          late = it.begin > begin;
          if (!late) keep_part<F>(s, smem + F::kParts + warp * F::kPart);
          if (lane == 0 && (it.begin >= begin || warp == 0)) {           // the first of the item's parts in this CTA
            const int cta_begin = runs.begin(run0), cta_end = runs.begin(min(run0 + warps, n_runs));
            const int from = runs.of(it.begin), to = runs.of(it.begin + it.tiles - 1);
            Segment<Item>& g = segments[atomicAdd(&n_segments, 1)];
            g.item = it;
            g.warp = warp;
            g.late = late;
            g.more = min(to, run0 + warps - 1) - (run0 + warp);
            g.slot = it.begin >= cta_begin && it.begin + it.tiles <= cta_end ? -1 : it.begin <= cta_begin ? 0 : 1;
            g.cta0 = from / warps;
            g.ctas = to / warps - g.cta0 + 1;
          }
        }
        if (x == end) break;
        Tiles::next_item(p, before, it);
        load_queries<F>(p, it, raw);
        begin_item<F>(p, it, raw, s);
      }
    }
    __syncthreads();
    if (late) keep_part<F>(s, smem + warp * F::kPart);
  } else {
    __syncthreads();
  }
  __syncthreads();

  // Two quads of a row, q and q + D / 8, to a thread.
  constexpr int kTasks = kRows * D / 8, kStats = kRows * D * 4;
  const int segs = n_segments;
  for (int task = tid; task < segs * kTasks; task += kWarps * 32) {
    const Segment<Item>& g = segments[task / kTasks];
    const int row = task % kTasks / (D / 8), q = task % (D / 8);
    const uint8_t* kept = smem + F::kParts + g.warp * F::kPart;
    const uint8_t* first = g.late ? smem + g.warp * F::kPart : kept;
    const auto part = [&](int i) { return i == 0 ? first : kept + i * F::kPart; };
    const Merged r = merge<2>(
        g.more + 1, [&](int i) { return reinterpret_cast<const float2*>(part(i) + kStats)[row]; },
        [&](int i, int y) { return reinterpret_cast<const float4*>(part(i))[row * (D / 4) + part_at(row, q + y * (D / 8))]; });
    if (g.slot < 0) {
      if (g.item.row0 + row < g.item.n * p.group) {
        __nv_bfloat16* dst = out_row(p, g.item, row) + 4 * q;
        store4(dst, r.o[0], r.factor());
        store4(dst + D / 2, r.o[1], r.factor());
      }
    } else {
      const size_t at = (static_cast<size_t>(blockIdx.x) * 2 + g.slot) * kRows + row;
      __stcg(reinterpret_cast<float4*>(p.part + at * D) + q, r.o[0]);
      __stcg(reinterpret_cast<float4*>(p.part + at * D) + q + D / 8, r.o[1]);
      if (q == 0) __stcg(reinterpret_cast<float2*>(p.stats) + at, make_float2(r.m, r.l));
    }
  }
  __threadfence();
  __syncthreads();
  if (tid < segs && segments[tid].slot >= 0) {
    Segment<Item>& g = segments[tid];
    g.last = atomicAdd(p.counters + g.cta0, 1u) == static_cast<unsigned>(g.ctas) - 1u;
    if (g.last) p.counters[g.cta0] = 0;
  }
  __syncthreads();

  // Items shared with other CTAs, by the last of them: the parts in the order of the CTAs, whoever it is.
  for (int i = 0; i < segs; ++i) {
    const Segment<Item>& g = segments[i];
    if (g.slot < 0 || !g.last) continue;
    __threadfence();
    const int begin0 = g.item.begin > runs.begin(g.cta0 * warps) ? 1 : 0;
    for (int task = tid; task < kTasks; task += kWarps * 32) {
      const int row = task / (D / 8), q = task % (D / 8);
      const auto at = [&](int c) { return (static_cast<size_t>(g.cta0 + c) * 2 + (c == 0 ? begin0 : 0)) * kRows + row; };
      const Merged r = merge<8>(
          g.ctas, [&](int c) { return __ldcg(reinterpret_cast<const float2*>(p.stats) + at(c)); },
          [&](int c, int y) { return __ldcg(reinterpret_cast<const float4*>(p.part + at(c) * D) + q + y * (D / 8)); });
      if (g.item.row0 + row < g.item.n * p.group) {
        __nv_bfloat16* dst = out_row(p, g.item, row) + 4 * q;
        store4(dst, r.o[0], r.factor());
        store4(dst + D / 2, r.o[1], r.factor());
      }
    }
  }
}

template <int D, int NR, bool PADDED>
cudaError_t launch_attend_as(const AttendParams& p, int num_sms, cudaStream_t stream) {
  using F = Few<D, NR, PADDED>;
  static_assert(F::kBefore + (kAttendMaxB + 1) * 4 + 1024 <= 227 * 1024, "shared memory of one SM");
  static std::atomic<unsigned long long> done{0};
  const cudaError_t e = smem_limit_once(attend_kernel<F>, F::bytes(kAttendMaxB), done);
  if (e != cudaSuccess) return e;
  return launch_pdl(attend_kernel<F>, dim3(num_sms), dim3(F::kWarps * 32), F::bytes(p.B), stream, p);
}

// Items of 8 rows where no sequence has more: half the products of items of 16, and registers for 12 warps (16 with D = 64) instead of 8.
template <int D, bool PADDED>
cudaError_t launch_attend_as(const AttendParams& p, int64_t rows, int num_sms, cudaStream_t stream) {
  return rows <= 8 ? launch_attend_as<D, 1, PADDED>(p, num_sms, stream) : launch_attend_as<D, 2, PADDED>(p, num_sms, stream);
}
template <int D>
cudaError_t launch_attend_as(const AttendParams& p, int64_t rows, int num_sms, cudaStream_t stream) {
  return p.n_valid == nullptr ? launch_attend_as<D, false>(p, rows, num_sms, stream) : launch_attend_as<D, true>(p, rows, num_sms, stream);
}

}  // namespace

AttendLayout attend_layout(int D) {
  const auto round = [](size_t v) { return (v + 255) / 256 * 256; };
  AttendLayout L;
  L.off_counters = 0;
  L.off_groups = round(kAttendMaxSms * sizeof(unsigned int));
  L.off_stats = L.off_groups + round(kAttendMaxSms * 2 * sizeof(unsigned int));
  L.off_out = L.off_stats + round(static_cast<size_t>(kAttendMaxSms) * 2 * kAttendManyRows * 8);
  L.total = L.off_out + static_cast<size_t>(kAttendMaxSms) * 2 * kAttendManyRows * D * 4;
  return L;
}

// Sequences of up to kFewRows rows are this kernel's, longer ones the other's.  128 keys of a head take this one 1300 clocks of an SM
// for each 16 rows and the other 4000 for any number up to 128.
// That counts where every SM has work.  Where there is little, the other one's items of 256 rows leave most SMs idle and its start and
// end cost 12 us: up to kFewPairs pairs of a row and a token in all, were every token of the batch in a sequence as long as this one,
// they are this kernel's too.  Both sides at 64 heads or fewer, this one first: 128 queries over 128 tokens (0.5 M pairs) 12 and 39 us,
// 3 x 40 over 700 (1.3 M) 15 and 29, 2 x 64 over 200 (1.6 M) 19 and 39, 2 x 5 over 9000 (2.9 M) 16 and 28, 100 over 2000 (3.2 M) 26
// and 30; 512 over 512 (8.4 M) 37 and 36, 8 x 16 over 2000 (16 M) 41 and 31, 300 over 5000 (32 M) 97 and 49.
constexpr int kFewRows = 48;
constexpr int64_t kFewPairs = 4 << 20;

cudaError_t launch_attend(AttendParams p, int max_q, int D, int num_sms, cudaStream_t stream) {
  const int64_t rows = static_cast<int64_t>(max_q) * p.group, heads = static_cast<int64_t>(p.group) * p.Hkv;
  const int64_t longest = static_cast<int64_t>(p.max_pages) << p.page_shift;
  p.rows_few = kFewRows;
  p.len_few = static_cast<int>(kFewPairs / std::max<int64_t>(p.T * heads, 1));
  const bool many = rows > kFewRows && longest > p.len_few;
  if (!many) p.len_few = INT32_MAX;                    // without the other kernel this one takes whatever comes
  const cudaError_t e = D == 64 ? launch_attend_as<64>(p, rows, num_sms, stream) : launch_attend_as<128>(p, rows, num_sms, stream);
  return e != cudaSuccess || !many ? e : launch_attend_many(p, D, num_sms, stream);
}

}  // namespace tempo
