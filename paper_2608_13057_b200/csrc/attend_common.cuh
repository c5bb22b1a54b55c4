// What the attention kernels share: how work is cut into items and tiles, and how it is dealt.
//
// A key head's queries (the heads of its group, and the new tokens of the sequence) are rows; kRows of them are an item.  An item
// has one tile for each kTile tokens that its last row sees.  The tiles of all items stand in one row, which is cut into runs of
// equal length whatever the lengths of the sequences.
#pragma once

#include "cache.cuh"
#include "ffn_common.cuh"

namespace tempo {

// PADDED: with n_valid, in kernels of their own (in the others its lines cost a prompt 1 to 2 %).
template <int ROWS, int TILE, bool PADDED>
struct Cut {
  static constexpr int kRows = ROWS, kTile = TILE;
  static constexpr bool kMany = ROWS == kAttendManyRows;

  struct Item {                 // rows [row0, row0 + kRows) of a sequence and key head, and its tiles
    int begin, tiles;           // number of its first tile in the launch
    int b, h, row0;
    int len, q0, n;             // tokens in the cache, first query row and queries of the sequence
  };

  // A sequence; one that is the other kernel's has no queries here.  Rows from n_valid on are not there, nor are the tokens that they
  // stand for: its other queries see what they see with them.
  static __device__ __forceinline__ void span_of(const AttendParams& p, int b, int& len, int& q0, int& n, bool tell = false) {
    const int given = p.lens[b];
    len = min(max(given, 0), p.max_pages << p.page_shift);
    int from = b, to = b + 1;
    if (p.q_start != nullptr) { from = p.q_start[b]; to = p.q_start[b + 1]; }
    q0 = min(max(from, 0), p.T);
    n = max(min(max(to, 0), p.T) - q0, 0);
    if (tell && (len != given || q0 != from || q0 + n != to)) atomicOr(p.status, TEMPO_STATUS_BAD_INDEX);
    if constexpr (PADDED) {
      const int cut = min(max(q0 + n - max(*p.n_valid, 0), 0), n);
      n -= cut;
      len = max(len - cut, 0);
    }
    if ((n * p.group <= p.rows_few || len <= p.len_few) == kMany) n = 0;
  }

  // Tiles are numbered in 32 bits: a sequence whose bound of them would not leave room for B like it is not taken.
  static __device__ __forceinline__ bool too_many(const AttendParams& p, int len, int n) {
    const float tiles = (static_cast<float>(n * p.group) / kRows + 1.0f) * (static_cast<float>(len) / kTile + 1.0f) * p.Hkv;
    if (n == 0 || tiles * p.B <= 1e9f) return false;
    atomicOr(p.status, TEMPO_STATUS_CAPACITY);
    return true;
  }

  // Tiles that the rows [row0, row0 + kRows) see: at least one, so that rows without a token are written too.
  static __device__ __forceinline__ int tiles_of(int len, int n, int group, int row0) {
    const int last = min(row0 + kRows, n * group) - 1;
    const int seen = len - n + last / group + 1;
    return max(1, (seen + kTile - 1) / kTile);
  }

  // The item of tile x.  before[b]: tiles before sequence b.
  static __device__ __forceinline__ Item item_at(const AttendParams& p, const int* before, int x) {
    int lo = 0, hi = p.B - 1;
    while (lo < hi) {                                  // the last sequence with before[b] <= x: the one that has tile x
      const int mid = (lo + hi + 1) >> 1;
      if (before[mid] <= x) lo = mid; else hi = mid - 1;
    }
    Item it;
    it.b = lo;
    span_of(p, lo, it.len, it.q0, it.n);
    const int per_head = (before[lo + 1] - before[lo]) / p.Hkv;
    int rest = x - before[lo];
    it.h = rest / per_head;
    rest -= it.h * per_head;
    it.row0 = 0;
    for (;;) {
      it.tiles = tiles_of(it.len, it.n, p.group, it.row0);
      if (rest < it.tiles) break;
      rest -= it.tiles;
      it.row0 += kRows;
    }
    it.begin = x - rest;
    return it;
  }

  // The one behind it (there is one: the caller has a tile left).
  static __device__ __forceinline__ void next_item(const AttendParams& p, const int* before, Item& it) {
    it.begin += it.tiles;
    it.row0 += kRows;
    if (it.row0 >= it.n * p.group) {
      it.row0 = 0;
      if (++it.h == p.Hkv) {
        it.h = 0;
        do ++it.b; while (before[it.b + 1] == before[it.b]);
        span_of(p, it.b, it.len, it.q0, it.n);
      }
    }
    it.tiles = tiles_of(it.len, it.n, p.group, it.row0);
  }

  // before[0] to before[B], by a whole CTA of WARPS warps; returns before[B].
  template <int WARPS>
  static __device__ __forceinline__ int count_tiles(const AttendParams& p, int* before, int* warp_sum, bool tell) {
    const int tid = threadIdx.x, warp = tid >> 5, lane = tid & 31;
    if (kRows > 16 && p.B <= WARPS) {                  // few long sequences: a warp to each
      if (warp < p.B) {
        int len, q0, n, mine = 0;
        span_of(p, warp, len, q0, n, tell);
        if (too_many(p, len, n)) n = 0;
        for (int row0 = lane * kRows; row0 < n * p.group; row0 += 32 * kRows) mine += tiles_of(len, n, p.group, row0);
#pragma unroll
        for (int d = 16; d > 0; d /= 2) mine += __shfl_xor_sync(0xffffffffu, mine, d);
        if (lane == 0) warp_sum[warp] = mine * p.Hkv;
      }
      __syncthreads();
      int total = 0;
      for (int b = 0; b < p.B; ++b) {
        if (tid == b) before[b] = total;
        total += warp_sum[b];
      }
      if (tid == 0) before[p.B] = total;
      __syncthreads();
      return total;
    }
    int total = 0;
    for (int b0 = 0; b0 < p.B; b0 += WARPS * 32) {
      const int b = b0 + tid;
      int mine = 0;
      if (b < p.B) {
        int len, q0, n;
        span_of(p, b, len, q0, n, tell);
        if (too_many(p, len, n)) n = 0;
        // tiles_of for each row0; the last row's query, (row0 + kRows - 1) / group, is carried along
        const int step = kRows / p.group, over = kRows - step * p.group;
        int query = (kRows - 1) / p.group, rest = kRows - 1 - query * p.group;
        for (int row0 = 0; row0 < n * p.group; row0 += kRows) {
          mine += max(1, (len - n + min(query, n - 1) + kTile) / kTile);
          query += step;
          rest += over;
          if (rest >= p.group) { rest -= p.group; ++query; }
        }
        mine *= p.Hkv;
      }
      int run = mine;
#pragma unroll
      for (int d = 1; d < 32; d *= 2) {
        const int up = __shfl_up_sync(0xffffffffu, run, d);
        if (lane >= d) run += up;
      }
      if (lane == 31) warp_sum[warp] = run;
      __syncthreads();
      int base = total;
#pragma unroll
      for (int w = 0; w < WARPS; ++w) {
        const int v = warp_sum[w];
        if (w < warp) base += v;
        total += v;
      }
      if (b < p.B) before[b + 1] = base + run;
      if (b == 0) before[0] = 0;
      __syncthreads();
    }
    return total;
  }
};

// Runs of equal length: the first `longer` of them have one tile more.
struct Runs {
  int quota, longer;
  __device__ __forceinline__ Runs(int total, int runs) : quota(total / runs), longer(total - total / runs * runs) {}
  __device__ __forceinline__ int begin(int r) const { return r * quota + min(r, longer); }
  __device__ __forceinline__ int of(int x) const {
    return x < longer * (quota + 1) ? x / (quota + 1) : longer + (x - longer * (quota + 1)) / quota;
  }
};

__device__ __forceinline__ float exp2_fast(float x) {
  float y;
  asm("ex2.approx.ftz.f32 %0, %1;" : "=f"(y) : "f"(x));
  return y;
}

constexpr float kBias = 7.0f, kSlack = 8.0f;      // weights are 2^(x - m + 7); m is raised once x exceeds it by more than 8

// A weight's exponent is fma(sum, f, 7 - m), with one rounding.  m itself is rounded, to a multiple of 1 from 2^23 on: then the exact
// product may lie so far above or below it that every weight of the row overflows or vanishes.  From 2^22 on products are rounded as m
// was, before m is taken off them.
__device__ __forceinline__ bool far_scores(float m) { return fabsf(m) >= 0x1p22f && m != -INFINITY; }
__device__ __forceinline__ float from_far(float sum, float f, float m) { return __fsub_rn(__fmul_rn(sum, f), m); }

// A row of queries times a power of two (and the scale's sign), its largest element in [256, 512): fp16 holds 2^-33 of it.
// `up`: that factor; `f`: a score is f times the sum of products, in units of log2; f is above zero, and at most 2^96, with which no score
// overflows (a sum is below 2^30) and any two that differ are too far apart for both to count.
__device__ __forceinline__ void row_factors(float top, bool odd, float scale_log2, float& up, float& f) {
  const int e = top > 0.0f ? min(max(static_cast<int>(__float_as_uint(top) >> 23) - 127 - 8, -110), 119) : 0;
  up = odd ? __uint_as_float(0x7fc00000u)
           : __uint_as_float((static_cast<uint32_t>(127 - e) << 23) | (__float_as_uint(scale_log2) & 0x80000000u));
  f = fminf(fmaxf(__uint_as_float(static_cast<uint32_t>(127 + e) << 23) * fabsf(scale_log2), 1.2e-38f), 0x1p96f);
}

}  // namespace tempo
