// The router: logits = x * Wr^T on the tensor cores, scores, the k best experts of every token and their weights, one
// kernel.
//
// A cluster of S CTAs owns a tile of up to 128 tokens (64 for more than 256 experts, so that the tile's logits fit into
// shared memory) and splits the reduction over d between its CTAs: with few tokens that spreads the router's weights
// over S SMs, with many tokens it brings the number of CTAs up to the number of SMs.  Per CTA: a ring of TMA tiles
// (tokens x 64 and experts x 64 bf16 values, 128-byte swizzle), tcgen05.mma.kind::f16 (M 128, N = experts) into tensor
// memory, the partial logits to shared memory; then the CTAs share the tile's tokens out, and a warp sums its tokens' S
// partials in rank order (the same bits every time) over distributed shared memory and picks their experts: every lane
// holds up to 16 logits as order-preserving integer keys whose low bits carry the expert, sorted in the lane; rounds of a
// warp-wide integer maximum take the k best and two more, and only where two of those are closer than the bits that
// the expert took are they put in order by their full values.  Ties go to the lowest index.  Logits, scores and
// weights stay in 32 bits, and every step that decides between experts is rounded singly.
//
// S: few tokens take a split as wide as a cluster goes (16 where the device runs such clusters), since the weights' way
// from memory to one SM is the time; many tokens take the split that fills the SMs.  What bounds it, as measured: one
// token of d 4096, 128 experts 5.5 us, of which a launch alone is 2.3, the rest a chain of latencies (tiles, tensor cores,
// cluster barrier, 8 rounds); 8192 tokens of d 7168, 256 experts 40 us, 18.6 by the operations at the library rate: the
// main loop runs at 85 % of it per SM on 128 of 148 SMs (24 us: tiles of 128 tokens come in whole numbers), the sum and the
// choice (integer instructions of all warps) take the rest.
//
// A logit that is not finite counts as minus infinity: it is chosen after every finite one, with weight 0.
#include "mma_warp.cuh"

namespace tempo {

constexpr int kRouteThreads = 512;
constexpr int kRouteMaxStages = 8;
constexpr int kRouteRing = 200 * 1024;

__device__ __forceinline__ uint32_t cluster_rank() {
  uint32_t r;
  asm volatile("mov.u32 %0, %%cluster_ctarank;" : "=r"(r));
  return r;
}
__device__ __forceinline__ uint32_t map_peer(uint32_t addr, uint32_t rank) {
  uint32_t r;
  asm volatile("mapa.shared::cluster.u32 %0, %1, %2;" : "=r"(r) : "r"(addr), "r"(rank));
  return r;
}
__device__ __forceinline__ float ld_peer(uint32_t addr) {
  float v;
  asm volatile("ld.shared::cluster.f32 %0, [%1];" : "=f"(v) : "r"(addr));
  return v;
}
__device__ __forceinline__ float4 ld_peer4(uint32_t addr) {
  float4 v;
  asm volatile("ld.shared::cluster.v4.f32 {%0, %1, %2, %3}, [%4];" : "=f"(v.x), "=f"(v.y), "=f"(v.z), "=f"(v.w) : "r"(addr));
  return v;
}
// Larger floats have larger keys, never 0 or 1 (-0 before +0: callers add +0, or a bias, so that the two tie).
__device__ __forceinline__ uint32_t order_key(float v) {
  const uint32_t u = __float_as_uint(v);
  return u ^ (static_cast<uint32_t>(static_cast<int>(u) >> 31) | 0x80000000u);
}
constexpr uint32_t kLeastFinite = 0x00800000u;           // key of the lowest finite value (that of -inf is the one below)
__device__ __forceinline__ float from_key(uint32_t k) {
  return __uint_as_float(k ^ ((k >> 31) != 0 ? 0x80000000u : 0xffffffffu));
}
// Expert of a lane's j-th logit: four neighbours per 16-byte load, 128 to a warp.
__device__ __forceinline__ int expert_of(int j, int lane) { return 128 * (j >> 2) + 4 * lane + (j & 3); }
// Rounded step by step, without contraction: the choice among biased scores must not depend on how the compiler fuses.
__device__ __forceinline__ float sigmoid_rn(float l) { return __fdiv_rn(1.f, __fadd_rn(1.f, expf(-l))); }

// Descending order of a lane's J keys (J = 4, 8, 16: odd-even merge network, 5, 19 or 63 exchanges).
template <int J>
__device__ __forceinline__ void sort_keys(uint32_t (&v)[J]) {
#pragma unroll
  for (int w = 1; w < J; w *= 2)
#pragma unroll
    for (int q = w; q >= 1; q /= 2)
#pragma unroll
      for (int j = q % w; j + q < J; j += 2 * q)
#pragma unroll
        for (int i = 0; i < q; ++i)
          if (j + i + q < J && (j + i) / (2 * w) == (j + i + q) / (2 * w)) {
            const uint32_t a = v[j + i], b = v[j + i + q];
            v[j + i] = max(a, b);
            v[j + i + q] = min(a, b);
          }
}

__device__ __forceinline__ float exact_score(const RouteParams& p, float l, float mx, float sum) {
  return p.sigmoid ? sigmoid_rn(l) : __fdiv_rn(expf(l - mx), sum);
}
__device__ __forceinline__ float warp_sum(float v) {
#pragma unroll
  for (int o = 16; o > 0; o >>= 1) v += __shfl_xor_sync(0xffffffffu, v, o);
  return v;
}
// Renormalised sigmoid weights of logits below -41, before the division, and their sum: there 1 / (1 + exp(-l)) is exp(l) to
// 2^-59 of itself; below -87 it has no normal 32-bit value, while its quotient by the sum has one, that of exp(l - m), m the
// largest logit chosen.  Not inlined: in the loop over tokens it costs every call 0.05 to 0.08 us (one token of 128 experts).
__device__ __noinline__ float2 small_scores(float l, bool on) {
  const uint32_t m = __reduce_max_sync(0xffffffffu, on ? order_key(l) : 0u);
  const float w = on ? expf(l - from_key(m)) : 0.f;
  return make_float2(w, warp_sum(w));
}
// The logit of expert `id` (every lane asks for its own), from the lane that holds it; an index into the registers would
// put them into local memory.
template <int J>
__device__ __forceinline__ float lane_logit(const float (&l)[J], int id) {
  float r = 0.f;
#pragma unroll
  for (int j = 0; j < J; ++j) {
    const float v = __shfl_sync(0xffffffffu, l[j], (id >> 2) & 31);
    if (j == ((id >> 7) << 2 | (id & 3))) r = v;
  }
  return r;
}
// Whether two candidates' keys (both of finite scores, a >= b) may stand in the wrong order.  Without a bias the scores are
// the logits and only the cut bits are open; a biased score is off by less than 2^-19 of its terms, which are below 1 + |a|.
__device__ __forceinline__ bool too_near(const RouteParams& p, uint32_t a, uint32_t b, uint32_t mask) {
  const float fa = from_key(a & ~mask), fb = from_key(b & ~mask);
  return (a & ~mask) - (b & ~mask) <= mask + 1u || (p.bias != nullptr && fa - fb <= 0x1p-17f * (1.f + fabsf(fa)));
}
// The exact choice among all experts: k rounds of a warp-wide maximum on exact keys, ties to the lowest expert.  Lane s < k
// gets the s-th, and whether its score is finite.
template <int J>
__device__ __forceinline__ void choose_exact(const RouteParams& p, const float (&l)[J], const float (&bias)[J], float mx, float sum,
                                             int lane, int& my_id, bool& my_fine) {
  uint32_t key[J];
#pragma unroll
  for (int j = 0; j < J; ++j) {
    float v = l[j];
    if (p.bias != nullptr && isfinite(v)) v = __fadd_rn(exact_score(p, v, mx, sum), bias[j]);   // bias -inf: taken out
    key[j] = expert_of(j, lane) >= p.E ? 0u : isfinite(v) ? order_key(v + 0.f) : 1u;
  }
#pragma unroll 1
  for (int s = 0; s < p.k; ++s) {
    uint32_t best = key[0];
#pragma unroll
    for (int j = 1; j < J; ++j) best = max(best, key[j]);
    const uint32_t top = __reduce_max_sync(0xffffffffu, best);
    int jj = J;
#pragma unroll
    for (int j = J - 1; j >= 0; --j)
      if (key[j] == top) jj = j;
    const uint32_t mine = best == top ? static_cast<uint32_t>(expert_of(jj, lane)) : 0xffffffffu;
    const uint32_t e = __reduce_min_sync(0xffffffffu, mine);
    if (lane == s) { my_id = static_cast<int>(e); my_fine = top > 1; }
    const int gone = mine == e ? jj : J;
#pragma unroll
    for (int j = 0; j < J; ++j)
      if (j == gone) key[j] = 0;
  }
}

// Sum of a token's partial logits over the cluster's CTAs, in rank order.
template <int JJ>
__device__ __forceinline__ void gather(const RouteParams& p, uint32_t row_addr, int lane, float (&l)[4 * JJ]) {
#pragma unroll
  for (int j = 0; j < 4 * JJ; ++j) l[j] = 0.f;
  // kAhead CTAs' partials are requested before any is added
  constexpr int kAhead = JJ == 1 ? 8 : JJ == 2 ? 4 : 2;
#pragma unroll 1
  for (int q0 = 0; q0 < p.splits; q0 += kAhead) {
    float4 v[kAhead][JJ];
#pragma unroll
    for (int q = 0; q < kAhead; ++q)
      if (q0 + q < p.splits) {
        const uint32_t peer = map_peer(row_addr, q0 + q);
#pragma unroll
        for (int j = 0; j < JJ; ++j) v[q][j] = ld_peer4(peer + 4u * min(128 * j + 4 * lane, p.E16 - 4));
      }
#pragma unroll
    for (int q = 0; q < kAhead; ++q)
      if (q0 + q < p.splits) {
#pragma unroll
        for (int j = 0; j < JJ; ++j) {
          l[4 * j] += v[q][j].x; l[4 * j + 1] += v[q][j].y;
          l[4 * j + 2] += v[q][j].z; l[4 * j + 3] += v[q][j].w;
        }
      }
  }
}

// One warp, NR tokens at once (the chains of dependent steps overlap): J logits of each per lane.
//
// Candidates, a few more than k, are found on keys that carry the expert: the upper bits of the order-preserving key of the
// score, the lower bits count the experts down.  A lane sorts its keys once; a round is then a warp-wide maximum of the
// lanes' first keys, and the winner moves its list up.  The upper bits leave out the score's last 7 to 9 bits, and a biased
// score comes from the fast exponential and division.  Where neighbours among the first k + 1 are nearer than that can be
// off, the candidates are ordered again by exact keys, a lane each (one or two tokens in 100 on normal logits); where even the
// last candidate is that near to the k-th, or a logit is not finite, all experts are.
template <int J, int NR>
__device__ __forceinline__ void pick(const RouteParams& p, const int (&t)[NR], const bool (&on)[NR], const float (&l)[NR][J],
                                     const float (&bias)[J], int lane) {
  constexpr int kBits = J == 4 ? 7 : J == 8 ? 8 : 9;
  constexpr uint32_t kMask = (1u << kBits) - 1u;
  // Softmax: the row's maximum and sum, where a weight or a biased key needs them (renormalised weights without a bias
  // do not: the sum cancels, and the first expert chosen has the maximum).
  const bool whole = !p.sigmoid && (!p.renormalise || p.bias != nullptr);
  const int m = min(p.k + 2, 32);
  bool bad[NR];
  float mx[NR], sum[NR];
  uint32_t key[NR][J], mine[NR];                         // mine, lane s: the s-th candidate
#pragma unroll
  for (int n = 0; n < NR; ++n) {
    float zero = 0.f;                                    // stays 0 while every logit is finite
#pragma unroll
    for (int j = 0; j < J; ++j) zero = fmaf(l[n][j], 0.f, zero);
    bad[n] = __any_sync(0xffffffffu, zero != 0.f);       // NaN != 0
    mx[n] = 0.f;
    sum[n] = 1.f;
    mine[n] = 0;
    if (whole) {
      uint32_t top = 0;
#pragma unroll
      for (int j = 0; j < J; ++j)
        if (expert_of(j, lane) < p.E && isfinite(l[n][j])) top = max(top, order_key(l[n][j]));
      top = __reduce_max_sync(0xffffffffu, top);
      mx[n] = top == 0 ? 0.f : from_key(top);
      float v = 0.f;
#pragma unroll
      for (int j = 0; j < J; ++j)
        if (expert_of(j, lane) < p.E && isfinite(l[n][j])) v += expf(l[n][j] - mx[n]);
      v = warp_sum(v);
      sum[n] = v > 0.f ? v : 1.f;
    }
    const float inv_sum = 1.f / sum[n];
#pragma unroll
    for (int j = 0; j < J; ++j) {
      float v = l[n][j];
      if (p.bias != nullptr) v = p.sigmoid ? __fdividef(1.f, 1.f + __expf(-v)) : __expf(v - mx[n]) * inv_sum;
      key[n][j] = (order_key(v + bias[j]) & ~kMask) | (kMask - static_cast<uint32_t>(expert_of(j, lane)));
    }
    sort_keys<J>(key[n]);
  }
#pragma unroll 1
  for (int s = 0; s < m; ++s) {
    uint32_t top[NR];
#pragma unroll
    for (int n = 0; n < NR; ++n) top[n] = __reduce_max_sync(0xffffffffu, key[n][0]);
#pragma unroll
    for (int n = 0; n < NR; ++n) {
      if (lane == s) mine[n] = top[n];
      const bool won = key[n][0] == top[n];              // keys differ, except the zeros of lists that have run out
#pragma unroll
      for (int j = 0; j + 1 < J; ++j) key[n][j] = won ? key[n][j + 1] : key[n][j];
      key[n][J - 1] = won ? 0u : key[n][J - 1];
    }
  }
#pragma unroll
  for (int n = 0; n < NR; ++n) {
    if (bad[n] && lane == 0) atomicOr(p.status, static_cast<uint32_t>(TEMPO_STATUS_BAD_LOGIT));
    int id = static_cast<int>(kMask - (mine[n] & kMask));
    bool fine = mine[n] >= kLeastFinite;                 // finite logit, finite bias
    const uint32_t below = __shfl_down_sync(0xffffffffu, mine[n], 1);
    const bool near = __any_sync(0xffffffffu, lane < p.k && lane + 1 < m && below >= kLeastFinite && too_near(p, mine[n], below, kMask));
    float el = lane_logit<J>(l[n], id);
    if (near || bad[n] || p.k == 32) {                   // 32 choices leave no lane for the first left out
      const uint32_t kth = __shfl_sync(0xffffffffu, mine[n], p.k - 1), last = __shfl_sync(0xffffffffu, mine[n], m - 1);
      if (!bad[n] && m > p.k && (last < kLeastFinite || !too_near(p, kth, last, kMask))) {
        uint32_t exact = 0;
        if (id < p.E && lane < m) {
          float v = el;
          if (p.bias != nullptr) {
            const float b = __ldg(p.bias + id);
            v = isfinite(b) ? __fadd_rn(exact_score(p, v, mx[n], sum[n]), b) : b;
          }
          exact = isfinite(v) ? order_key(v + 0.f) : 1u;
        }
        int rank = 0;
        for (int s = 0; s < m; ++s) {
          const uint32_t o = __shfl_sync(0xffffffffu, exact, s);
          const int oid = __shfl_sync(0xffffffffu, id, s);
          rank += o > exact || (o == exact && oid < id) ? 1 : 0;
        }
        const uint32_t self = static_cast<uint32_t>(id) | (exact > 1u ? 0x80000000u : 0u);
        uint32_t got = 0;
        for (int s = 0; s < m; ++s) {
          const int r = __shfl_sync(0xffffffffu, rank, s);
          const uint32_t v = __shfl_sync(0xffffffffu, self, s);
          if (r == lane) got = v;
        }
        id = static_cast<int>(got & 0x7fffffffu);
        fine = (got >> 31) != 0;
      } else {
        choose_exact<J>(p, l[n], bias, mx[n], sum[n], lane, id, fine);
      }
      el = lane_logit<J>(l[n], id);
    }
    const float top_l = whole ? mx[n] : __shfl_sync(0xffffffffu, el, 0);
    float w = 0.f;
    if (lane < p.k && fine) w = exact_score(p, el, top_l, sum[n]);
    if (p.renormalise) {
      float v = warp_sum(w);
      if (p.sigmoid && v < 0x1p-60f) {                   // (the same in every lane)
        const float2 r = small_scores(el, lane < p.k && fine);
        w = r.x;
        v = r.y;
      }
      w = v > 0.f ? __fdiv_rn(w, v) : 0.f;
    }
    if (lane < p.k && on[n]) {
      p.ids[static_cast<size_t>(t[n]) * p.k + lane] = id;
      p.w[static_cast<size_t>(t[n]) * p.k + lane] = w * p.scale;
    }
  }
}

template <int JJ, int NR>
__global__ void __launch_bounds__(kRouteThreads, 1)
route_kernel(const __grid_constant__ CUtensorMap tmX, const __grid_constant__ CUtensorMap tmW, const RouteParams p) {
  extern __shared__ uint8_t smem_raw[];
  __shared__ __align__(8) uint64_t s_full[kRouteMaxStages];
  __shared__ __align__(8) uint64_t s_empty[kRouteMaxStages];
  __shared__ __align__(8) uint64_t s_acc;
  __shared__ uint32_t s_tmem_base;
  __shared__ int s_abort_storage;
  volatile int* s_abort = &s_abort_storage;
  const int tid = threadIdx.x, warp = tid >> 5, lane = tid & 31;
  const uint32_t smem_base = (smem_u32(smem_raw) + 1023u) & ~1023u;
  const uint32_t rank = cluster_rank();
  const int S = p.splits, tile = blockIdx.x / S, t0 = tile * p.tile_rows;
  pdl_trigger();
  if (tid == 0) {
    for (int s = 0; s < p.stages; ++s) { mbar_init(smem_u32(&s_full[s]), 1); mbar_init(smem_u32(&s_empty[s]), 1); }
    mbar_init(smem_u32(&s_acc), 1);
    s_abort_storage = 0;
    asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
    asm volatile("prefetch.tensormap [%0];" ::"l"(reinterpret_cast<uint64_t>(&tmX)) : "memory");
    asm volatile("prefetch.tensormap [%0];" ::"l"(reinterpret_cast<uint64_t>(&tmW)) : "memory");
  }
  if (warp == 1) {
    asm volatile("tcgen05.alloc.cta_group::1.sync.aligned.shared::cta.b32 [%0], %1;" ::"r"(smem_u32(&s_tmem_base)),
                 "r"(p.tmem_cols) : "memory");
    asm volatile("tcgen05.relinquish_alloc_permit.cta_group::1.sync.aligned;" ::: "memory");
  }
  tc_fence_before();
  __syncthreads();
  tc_fence_after();
  const uint32_t tmem_base = s_tmem_base;
  pdl_wait();
  int nv = p.T;
  if (p.n_valid != nullptr) nv = max(0, min(*p.n_valid, p.T));
  const int live = max(0, min(p.tile_rows, nv - t0));   // the same in every CTA of the cluster
  const int kb0 = static_cast<int>(rank) * p.Kb / S, kb1 = (static_cast<int>(rank) + 1) * p.Kb / S;
  const bool work = live > 0 && kb1 > kb0;
  if (work && warp == 0) {
    // The ring is empty at first: one lane per stage issues its loads (one thread takes 0.2 us per block).
    auto load = [&](int kb, uint32_t stage) {
      const uint32_t full = smem_u32(&s_full[stage]), sX = smem_base + stage * p.stage_bytes, sW = sX + kABytes;
      mbar_arrive_expect_tx(full, p.x_box * 128 + p.w_boxes * p.w_box * 128);
      tma_load_2d(sX, &tmX, full, kb * kBlockK, t0);
      for (int c = 0; c < p.w_boxes; ++c) tma_load_2d(sW + c * p.w_box * 128, &tmW, full, kb * kBlockK, c * p.w_box);
    };
    if (lane < p.stages && kb0 + lane < kb1) load(kb0 + lane, lane);
    __syncwarp();
    if (lane == 0) {
      uint32_t stage = 0, phase = 0;
      for (int kb = kb0 + p.stages; kb < kb1; ++kb) {
        if (!mbar_wait(smem_u32(&s_empty[stage]), phase, s_abort, kDefaultWaitNs)) break;
        load(kb, stage);
        if (++stage == static_cast<uint32_t>(p.stages)) { stage = 0; phase ^= 1u; }
      }
    }
  } else if (work && warp == 1) {
    const uint32_t leader = elect_one();
    const uint32_t full0 = smem_u32(s_full), empty0 = smem_u32(s_empty), desc0 = desc_lo_sw128(smem_base), desc_step = p.stage_bytes >> 4;
    uint32_t stage = 0, phase = 0, accumulate = 0;
    bool ok = true;
    for (int kb = kb0; kb < kb1; ++kb) {
      if (!mbar_wait_warp(full0 + 8 * stage, phase, s_abort, kDefaultWaitNs)) { ok = false; break; }
      tc_fence_after();
      const uint32_t da = desc0 + stage * desc_step;
      uint32_t db = da + (kABytes >> 4), acc = tmem_base;
      for (int c = 0; c < p.w_boxes; ++c) {
        const int n = min(p.w_box, p.E16 - c * p.w_box);
        const uint32_t idesc = (1u << 4) | (1u << 7) | (1u << 10) | (static_cast<uint32_t>(n >> 3) << 17) |
                               (static_cast<uint32_t>(kTileM >> 4) << 24);
#pragma unroll
        for (int ks = 0; ks < 4; ++ks) warp_mma_bf16(leader, acc, da + 2 * ks, db + 2 * ks, idesc, ks == 0 ? accumulate : 1u);
        db += (p.w_box * 128) >> 4;
        acc += p.w_box;
      }
      accumulate = 1;
      warp_commit(leader, empty0 + 8 * stage);
      if (++stage == static_cast<uint32_t>(p.stages)) { stage = 0; phase ^= 1u; }
    }
    if (ok) warp_commit(leader, smem_u32(&s_acc));
  }
  __syncwarp();
  // Partial logits to shared memory: lane = token row of the warp's quadrant; 16-byte stores at a pitch of 4 words more than
  // a multiple of 32 touch every bank once per eight lanes, and so do the reads along a row.  The ring is free: every MMA
  // that read it has completed.
  float* logits = reinterpret_cast<float*>(smem_raw + (smem_base - smem_u32(smem_raw)));
  const uint32_t logits_addr = smem_u32(logits);
  const int pitch = p.pitch;
  constexpr int J = 4 * JJ, kWarps = kRouteThreads / 32;
  bool have = work;
  if (work) {
    have = __all_sync(0xffffffffu, mbar_wait(smem_u32(&s_acc), 0, s_abort, kDefaultWaitNs));
    tc_fence_after();
  }
  float bias[J];
#pragma unroll
  for (int j = 0; j < J; ++j) {
    const int e = 128 * (j / 4) + 4 * lane + j % 4;
    const float b = p.bias != nullptr && e < p.E ? __ldg(p.bias + e) : 0.f;
    bias[j] = e < p.E && isfinite(b) ? b : -INFINITY;    // a bias that is not finite takes its expert out, as one that is not there
  }
  if ((warp & 3) * 32 < live) {
    const int row = (warp & 3) * 32 + lane;
    for (int c = (warp >> 2) * 16; c < p.E16; c += 16 * (kRouteThreads / 128)) {
      uint32_t v[16];
      if (have) {
        asm volatile(
            "tcgen05.ld.sync.aligned.32x32b.x16.b32 {%0, %1, %2, %3, %4, %5, %6, %7, %8, %9, %10, %11, %12, %13, %14, %15}, [%16];"
            : "=r"(v[0]), "=r"(v[1]), "=r"(v[2]), "=r"(v[3]), "=r"(v[4]), "=r"(v[5]), "=r"(v[6]), "=r"(v[7]), "=r"(v[8]),
              "=r"(v[9]), "=r"(v[10]), "=r"(v[11]), "=r"(v[12]), "=r"(v[13]), "=r"(v[14]), "=r"(v[15])
            : "r"(tmem_base + (static_cast<uint32_t>((warp & 3) * 32) << 16) + c) : "memory");
        tmem_wait_ld();
      } else {
#pragma unroll
        for (int i = 0; i < 16; ++i) v[i] = 0;
      }
      if (row < live) {
#pragma unroll
        for (int i = 0; i < 16; i += 4)
          st_shared_v4(logits_addr + 4u * (row * pitch + c + i), make_uint4(v[i], v[i + 1], v[i + 2], v[i + 3]));
      }
    }
  }
  __syncwarp();
  asm volatile("barrier.cluster.arrive.release.aligned;\n\tbarrier.cluster.wait.acquire.aligned;" ::: "memory");
  // The tokens are dealt to the cluster's CTAs and their warps, NR at a time.
  const int step = S * kWarps;
  for (int r0 = static_cast<int>(rank) + S * warp; r0 < p.tile_rows && t0 + r0 < p.T; r0 += NR * step) {
    int t[NR];
    bool on[NR];
    float l[NR][J];
#pragma unroll
    for (int n = 0; n < NR; ++n) {
      const int r = r0 + n * step;
      t[n] = t0 + r;
      on[n] = r < live;
      if (!on[n] && r < p.tile_rows && t[n] < p.T && lane < p.k) {       // a padding row
        p.ids[static_cast<size_t>(t[n]) * p.k + lane] = -1;
        p.w[static_cast<size_t>(t[n]) * p.k + lane] = 0.f;
      }
    }
    if (!on[0]) continue;                                // rows beyond it are padding too
#pragma unroll
    for (int n = 0; n < NR; ++n)                         // a row that is not there repeats the first
      gather<JJ>(p, logits_addr + 4u * static_cast<uint32_t>((on[n] ? r0 + n * step : r0) * pitch), lane, l[n]);
    pick<J, NR>(p, t, on, l, bias, lane);
  }
  // nobody leaves while a peer may still read its logits
  __syncwarp();
  asm volatile("barrier.cluster.arrive.relaxed.aligned;\n\tbarrier.cluster.wait.aligned;" ::: "memory");
  if (*s_abort) {
    if (tid == 0) atomicOr(p.status, static_cast<uint32_t>(TEMPO_STATUS_TIMEOUT));
    for (int i = 0; i < 50; ++i) __nanosleep(1000);      // let copies and MMAs in flight drain
  }
  tc_fence_before();
  __syncthreads();
  if (warp == 1) {
    tc_fence_after();
    asm volatile("tcgen05.dealloc.cta_group::1.sync.aligned.b32 %0, %1;" ::"r"(tmem_base), "r"(p.tmem_cols) : "memory");
  }
}

constexpr int kRouteSmem = 226 * 1024;      // the most a launch asks for

template <int JJ, int NR>
static cudaError_t launch_route_t(const CUtensorMap& tmX, const CUtensorMap& tmW, const RouteParams& p, int ctas,
                                  size_t smem, cudaStream_t stream) {
  static std::atomic<unsigned long long> smem_set{0};
  cudaError_t e = smem_limit_once(route_kernel<JJ, NR>, kRouteSmem, smem_set);
  if (e != cudaSuccess) return e;
  if (p.splits > 8) {
    static std::atomic<unsigned long long> wide_set{0};
    int dev = 0;
    e = cudaGetDevice(&dev);
    if (e != cudaSuccess) return e;
    const unsigned long long bit = dev >= 0 && dev < 64 ? 1ull << dev : 0ull;
    if (bit == 0 || !(wide_set.load(std::memory_order_acquire) & bit)) {
      e = cudaFuncSetAttribute(route_kernel<JJ, NR>, cudaFuncAttributeNonPortableClusterSizeAllowed, 1);
      if (e != cudaSuccess) return e;
      if (bit != 0) wide_set.fetch_or(bit, std::memory_order_release);
    }
  }
  cudaLaunchConfig_t cfg = {};
  cfg.gridDim = dim3(ctas);
  cfg.blockDim = dim3(kRouteThreads);
  cfg.dynamicSmemBytes = smem;
  cfg.stream = stream;
  cudaLaunchAttribute attr[2];
  attr[0].id = cudaLaunchAttributeProgrammaticStreamSerialization;
  attr[0].val.programmaticStreamSerializationAllowed = 1;
  attr[1].id = cudaLaunchAttributeClusterDimension;
  attr[1].val.clusterDim.x = p.splits;
  attr[1].val.clusterDim.y = attr[1].val.clusterDim.z = 1;
  cfg.attrs = attr;
  cfg.numAttrs = 2;
  return cudaLaunchKernelEx(&cfg, route_kernel<JJ, NR>, tmX, tmW, p);
}

// Clusters of 16 CTAs (one per SM) that this device runs at once; 0 where it refuses them.  Asked once per device.
static int wide_clusters() {
  static std::atomic<int> cached[64];                   // 0: not asked yet, else the answer + 1
  int dev = 0;
  if (cudaGetDevice(&dev) != cudaSuccess || dev < 0 || dev >= 64) return 0;
  const int known = cached[dev].load(std::memory_order_acquire);
  if (known != 0) return known - 1;
  int n = 0;
  if (cudaFuncSetAttribute(route_kernel<1, 1>, cudaFuncAttributeMaxDynamicSharedMemorySize, kRouteSmem) != cudaSuccess ||
      cudaFuncSetAttribute(route_kernel<1, 1>, cudaFuncAttributeNonPortableClusterSizeAllowed, 1) != cudaSuccess) {
    (void)cudaGetLastError();
  } else {
    cudaLaunchConfig_t cfg = {};
    cfg.gridDim = dim3(16);
    cfg.blockDim = dim3(kRouteThreads);
    cfg.dynamicSmemBytes = kRouteSmem;
    cudaLaunchAttribute attr[1];
    attr[0].id = cudaLaunchAttributeClusterDimension;
    attr[0].val.clusterDim.x = 16;
    attr[0].val.clusterDim.y = attr[0].val.clusterDim.z = 1;
    cfg.attrs = attr;
    cfg.numAttrs = 1;
    if (cudaOccupancyMaxActiveClusters(&n, route_kernel<1, 1>, &cfg) != cudaSuccess) {
      (void)cudaGetLastError();                          // a refused query must not poison the next launch
      n = 0;
    }
  }
  cached[dev].store(n + 1, std::memory_order_release);
  return n;
}

RoutePlan route_plan(int T, int E, int d, int num_sms) {
  RoutePlan r;
  r.E16 = (E + 15) / 16 * 16;
  const int Kb = d / 64;
  r.tile_rows = E <= 256 ? 128 : 64;
  r.x_box = min(r.tile_rows, (T + 7) / 8 * 8);
  r.w_box = min(r.E16, 256);
  r.w_boxes = (r.E16 + 255) / 256;
  r.stage_bytes = kABytes + r.w_boxes * r.w_box * 128;
  r.stages = min(kRouteMaxStages, kRouteRing / r.stage_bytes);
  const int tiles = (T + r.tile_rows - 1) / r.tile_rows;
  r.splits = 1;
  while (r.splits < 8 && 2 * r.splits * tiles <= num_sms && 2 * r.splits <= Kb) r.splits *= 2;
  if (r.splits == 8 && Kb >= 32 && tiles <= wide_clusters()) r.splits = 16;
  r.ctas = tiles * r.splits;
  return r;
}

cudaError_t launch_route(const CUtensorMap& tmX, const CUtensorMap& tmW, RouteParams p, const RoutePlan& r, cudaStream_t stream) {
  p.E16 = r.E16;
  p.tile_rows = r.tile_rows;
  p.x_box = r.x_box;
  p.w_box = r.w_box;
  p.w_boxes = r.w_boxes;
  p.stage_bytes = r.stage_bytes;
  p.stages = r.stages;
  p.splits = r.splits;
  p.pitch = (r.E16 + 31) / 32 * 32 + 4;
  p.tmem_cols = 32;
  while (p.tmem_cols < r.E16) p.tmem_cols *= 2;
  const size_t ring = static_cast<size_t>(r.stages) * r.stage_bytes;
  const size_t table = static_cast<size_t>(r.tile_rows) * p.pitch * 4;
  const size_t smem = (ring > table ? ring : table) + 1024;
  // two tokens per warp at a time where every warp has at least two (16 logits per lane leave no registers for it)
  const bool two = min(r.tile_rows, p.T) / r.splits >= 2 * (kRouteThreads / 32);
  if (p.E <= 128) return two ? launch_route_t<1, 2>(tmX, tmW, p, r.ctas, smem, stream) : launch_route_t<1, 1>(tmX, tmW, p, r.ctas, smem, stream);
  if (p.E <= 256) return two ? launch_route_t<2, 2>(tmX, tmW, p, r.ctas, smem, stream) : launch_route_t<2, 1>(tmX, tmW, p, r.ctas, smem, stream);
  return launch_route_t<4, 1>(tmX, tmW, p, r.ctas, smem, stream);
}

}  // namespace tempo
