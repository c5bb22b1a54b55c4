// The router: logits = x * Wr^T on the tensor cores, scores, the k best experts of every token and their weights, one
// kernel.
//
// A cluster of S CTAs owns a tile of up to 128 tokens (64 for more than 256 experts, so that the tile's logits fit into
// shared memory) and splits the reduction over d between its CTAs: with few tokens that spreads the router's weights
// over S SMs, with many tokens it brings the number of CTAs up to the number of SMs.  Per CTA: a ring of TMA tiles
// (tokens x 64 and experts x 64 bf16 values, 128-byte swizzle), tcgen05.mma.kind::f16 (M 128, N = experts) into tensor
// memory, the partial logits to shared memory; then the CTAs share the tile's tokens out, and a warp sums a token's S
// partials in rank order (the same bits every time) over distributed shared memory and picks its experts:
// every lane holds E/32 logits, k rounds of a warp-wide maximum on order-preserving integer keys take the best left and
// break ties towards the lowest index.  Logits, scores and weights stay in 32 bits.
//
// A logit that is not finite counts as minus infinity: it is chosen after every finite one, with weight 0.
#include "mma_warp.cuh"

namespace tempo {

constexpr int kRouteThreads = 256;
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
  asm volatile("ld.shared::cluster.f32 %0, [%1];" : "=f"(v) : "r"(addr) : "memory");
  return v;
}
// Larger floats have larger keys; finite values only, never 0 or 1.
__device__ __forceinline__ uint32_t order_key(float v) {
  const uint32_t u = __float_as_uint(v + 0.f);           // -0 and +0 tie
  return u ^ ((u >> 31) != 0 ? 0xffffffffu : 0x80000000u);
}
// Rounded step by step, without contraction: the choice among biased scores must not depend on how the compiler fuses.
__device__ __forceinline__ float sigmoid_rn(float l) { return __fdiv_rn(1.f, __fadd_rn(1.f, expf(-l))); }

struct RouteRow {
  const RouteParams* p;
  float mx, sum;
  __device__ float score(float l) const {
    if (!isfinite(l)) return 0.f;
    return p->sigmoid ? sigmoid_rn(l) : __fdiv_rn(expf(l - mx), sum);
  }
};

// One warp, one token: J logits per lane (expert lane + 32 j).
template <int J>
__device__ __forceinline__ void pick(const RouteParams& p, int t, const float (&l)[J], int lane) {
  RouteRow row{&p, 0.f, 1.f};
  bool bad = false;
#pragma unroll
  for (int j = 0; j < J; ++j) bad |= lane + 32 * j < p.E && !isfinite(l[j]);
  if (__any_sync(0xffffffffu, bad) && lane == 0) atomicOr(p.status, static_cast<uint32_t>(TEMPO_STATUS_BAD_LOGIT));
  if (!p.sigmoid) {
    uint32_t m = 0;
#pragma unroll
    for (int j = 0; j < J; ++j)
      if (lane + 32 * j < p.E && isfinite(l[j])) m = max(m, order_key(l[j]));
    m = __reduce_max_sync(0xffffffffu, m);
    row.mx = m == 0 ? 0.f : __uint_as_float(m ^ ((m >> 31) != 0 ? 0x80000000u : 0xffffffffu));
    float s = 0.f;
#pragma unroll
    for (int j = 0; j < J; ++j)
      if (lane + 32 * j < p.E && isfinite(l[j])) s += expf(l[j] - row.mx);
#pragma unroll
    for (int o = 16; o > 0; o >>= 1) s += __shfl_xor_sync(0xffffffffu, s, o);
    row.sum = s > 0.f ? s : 1.f;
  }
  uint32_t key[J];
#pragma unroll
  for (int j = 0; j < J; ++j) {
    const int e = lane + 32 * j;
    key[j] = 0;
    if (e < p.E) {
      float v = l[j];
      if (p.bias != nullptr) v = isfinite(v) ? __fadd_rn(row.score(v), __ldg(p.bias + e)) : v;
      key[j] = isfinite(v) ? order_key(v) : 1u;
    }
  }
  int my_id = 0;
  float my_l = 0.f;
  for (int s = 0; s < p.k; ++s) {
    uint32_t best = 0;
    int bj = 0;
    float bl = 0.f;
#pragma unroll
    for (int j = 0; j < J; ++j)
      if (key[j] > best) { best = key[j]; bj = j; bl = l[j]; }
    const uint32_t top = __reduce_max_sync(0xffffffffu, best);
    const uint32_t e = __reduce_min_sync(0xffffffffu, best == top ? static_cast<uint32_t>(lane + 32 * bj) : 0xffffffffu);
    const float el = __shfl_sync(0xffffffffu, bl, static_cast<int>(e & 31u));
    if (lane == s) { my_id = static_cast<int>(e); my_l = el; }
    if (static_cast<uint32_t>(lane) == (e & 31u)) {
#pragma unroll
      for (int j = 0; j < J; ++j)
        if (j == static_cast<int>(e >> 5)) key[j] = 0;
    }
  }
  float w = 0.f;
  if (lane < p.k) {
    w = row.score(my_l);
    if (p.bias != nullptr && !isfinite(__ldg(p.bias + my_id))) w = 0.f;   // an expert that the bias takes out
  }
  if (p.renormalise) {
    float s = w;
#pragma unroll
    for (int o = 16; o > 0; o >>= 1) s += __shfl_xor_sync(0xffffffffu, s, o);
    w = s > 0.f ? __fdiv_rn(w, s) : 0.f;
  }
  if (lane < p.k) {
    p.ids[static_cast<size_t>(t) * p.k + lane] = my_id;
    p.w[static_cast<size_t>(t) * p.k + lane] = w * p.scale;
  }
}

template <int J>
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
  if (work && warp == 0 && lane == 0) {
    uint32_t stage = 0, phase = 0;
    for (int kb = kb0; kb < kb1; ++kb) {
      if (!mbar_wait(smem_u32(&s_empty[stage]), phase ^ 1u, s_abort, kDefaultWaitNs)) break;
      const uint32_t full = smem_u32(&s_full[stage]), sX = smem_base + stage * p.stage_bytes, sW = sX + kABytes;
      mbar_arrive_expect_tx(full, p.x_box * 128 + p.w_boxes * p.w_box * 128);
      tma_load_2d(sX, &tmX, full, kb * kBlockK, t0);
      for (int c = 0; c < p.w_boxes; ++c) tma_load_2d(sW + c * p.w_box * 128, &tmW, full, kb * kBlockK, c * p.w_box);
      if (++stage == static_cast<uint32_t>(p.stages)) { stage = 0; phase ^= 1u; }
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
  // Partial logits to shared memory: lane = token row of the warp's quadrant, so a column of 32 rows is one
  // conflict-free store (the pitch is odd).  The ring is free: every MMA that read it has completed.
  float* logits = reinterpret_cast<float*>(smem_raw + (smem_base - smem_u32(smem_raw)));
  const int pitch = p.E16 + 1;
  const int row = (warp & 3) * 32 + lane;
  bool have = work;
  if (work) {
    have = __all_sync(0xffffffffu, mbar_wait(smem_u32(&s_acc), 0, s_abort, kDefaultWaitNs));
    tc_fence_after();
  }
  if ((warp & 3) * 32 < live) {
    for (int c = (warp >> 2) * 16; c < p.E16; c += 32) {
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
        for (int i = 0; i < 16; ++i) logits[row * pitch + c + i] = __uint_as_float(v[i]);
      }
    }
  }
  __syncwarp();
  asm volatile("barrier.cluster.arrive.release.aligned;\n\tbarrier.cluster.wait.acquire.aligned;" ::: "memory");
  // The tile's tokens are dealt to the cluster's CTAs and their warps.
  const uint32_t logits_addr = smem_u32(logits);
  for (int r = static_cast<int>(rank) + S * warp; r < p.tile_rows && t0 + r < p.T; r += S * (kRouteThreads / 32)) {
    if (r >= live) {                                     // a padding row
      if (lane < p.k) {
        p.ids[static_cast<size_t>(t0 + r) * p.k + lane] = -1;
        p.w[static_cast<size_t>(t0 + r) * p.k + lane] = 0.f;
      }
      continue;
    }
    float l[J];
#pragma unroll
    for (int j = 0; j < J; ++j) l[j] = 0.f;
    for (int q = 0; q < S; ++q) {
      const uint32_t src = map_peer(logits_addr, q) + static_cast<uint32_t>(r * pitch + lane) * 4u;
#pragma unroll
      for (int j = 0; j < J; ++j)
        if (lane + 32 * j < p.E) l[j] += ld_peer(src + 128u * j);
    }
    pick<J>(p, t0 + r, l, lane);
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

template <int J>
static cudaError_t launch_route_t(const CUtensorMap& tmX, const CUtensorMap& tmW, const RouteParams& p, int ctas,
                                  size_t smem, cudaStream_t stream) {
  static std::atomic<unsigned long long> smem_set{0};
  cudaError_t e = smem_limit_once(route_kernel<J>, 227 * 1024 - 1024, smem_set);
  if (e != cudaSuccess) return e;
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
  return cudaLaunchKernelEx(&cfg, route_kernel<J>, tmX, tmW, p);
}

RoutePlan route_plan(int T, int E, int d, int num_sms) {
  RoutePlan r;
  r.E16 = (E + 15) / 16 * 16;
  r.tile_rows = E <= 256 ? 128 : 64;
  r.x_box = min(r.tile_rows, (T + 7) / 8 * 8);
  r.w_box = min(r.E16, 256);
  r.w_boxes = (r.E16 + 255) / 256;
  r.stage_bytes = kABytes + r.w_boxes * r.w_box * 128;
  r.stages = min(kRouteMaxStages, kRouteRing / r.stage_bytes);
  const int tiles = (T + r.tile_rows - 1) / r.tile_rows, Kb = d / 64;
  r.splits = 1;
  while (r.splits < 8 && 2 * r.splits * tiles <= num_sms && 2 * r.splits <= Kb) r.splits *= 2;
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
  p.tmem_cols = 32;
  while (p.tmem_cols < r.E16) p.tmem_cols *= 2;
  const size_t ring = static_cast<size_t>(r.stages) * r.stage_bytes;
  const size_t table = static_cast<size_t>(r.tile_rows) * (r.E16 + 1) * 4;
  const size_t smem = (ring > table ? ring : table) + 1024;
  const int J = (p.E + 31) / 32;
  if (J <= 1) return launch_route_t<1>(tmX, tmW, p, r.ctas, smem, stream);
  if (J <= 2) return launch_route_t<2>(tmX, tmW, p, r.ctas, smem, stream);
  if (J <= 4) return launch_route_t<4>(tmX, tmW, p, r.ctas, smem, stream);
  if (J <= 8) return launch_route_t<8>(tmX, tmW, p, r.ctas, smem, stream);
  return launch_route_t<16>(tmX, tmW, p, r.ctas, smem, stream);
}

}  // namespace tempo
