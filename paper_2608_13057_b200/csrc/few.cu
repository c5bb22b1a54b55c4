// The experts of an MoE layer for a few tokens, one persistent kernel:
//   out[t] = sum_s w[t,s] * W2_e (silu(Wg_e x_t) (.) (Wu_e x_t)),  e = ids[t,s], experts of this rank only.
//
// With a few tokens the layer is bound by the bytes of the chosen experts' weights (3 d f per expert), so everything
// here serves one weight stream that starts early, never stops and is the same length on every SM:
//   - The weights are the M side of the tensor-core product and the tokens the N side: a 32 KB tile of the packed blob
//     (256 weight rows x 128 bytes of K, already in the shared-memory image) is the A operand of two M 128
//     instructions, and N is the number of token columns, a multiple of 16.  No row of a tile is padding.
//   - The blocks (tiles of 32 KB) of all chosen experts' gate/up matrices are dealt to the CTAs as equal contiguous
//     runs, whatever expert or column block they belong to; a gate/up column block that spans CTAs is summed by the CTA
//     that has its first block (that one ends its run there, so it is the last thing it does), from the others' 32-bit
//     partial sums in the workspace, in the order of the runs.  The down matrices are dealt in the same way.
//   - With enough blocks the experts are taken in two halves (gate/up 1, gate/up 2, down 1, down 2): while one half's H
//     is summed and published the other half's weights stream, and the ring goes on with down weights all the same
//     (one token of 8 experts, 4096 x 1536: 34.0 us in halves, 35.6 us without).
//   - Activations enter as two terms, not as one 8-bit code.  fp8 weights: a bf16 value has 8 significant bits, an e4m3 value 4, so
//     x = 2^eps (q1 + q2 / 16) with two e4m3 terms is x itself for everything within 2^-13 of the block's largest value
//     (and within 2^-22 of that value below), and each token takes two columns whose block scales differ by 2^4; the
//     two sums are added in 32 bits.  H is split the same way: 8 bits like a bf16 rounding, with 0.4 of its mean error.  The
//     output is 0.0018 of its norm from 64 bits, of which its own rounding to bf16 alone is 0.0016 to 0.0017.
//     bf16 weights: x as it is, H as two bf16 terms (16 bits).
// A value of H that is not finite (bf16 weights: beyond bf16's range), and with fp8 weights one of x, becomes a NaN: its
// token's output is NaN, no other token's.  With bf16 weights an x that is not finite makes H so.
//
// What bounds it: the weight stream.  Measured, each against the chosen weights' bytes at the rate of a plain copy: one
// token of 8 experts, d 4096, f 1536, fp8: 31.8 us against 23.1; 64 tokens over 16 experts of the same: 55.3 against
// 46.2 (305 MB read from memory for 302 MB of weights); 11 tokens over 41 experts, d 2048, f 1408, bf16: 106.7 against
// 110.3 (a stream that only reads runs above the copy's rate).  What stays above the stream, about 9 us, is latency: the
// expert lists and the first tiles, 4 us; the last half's H, about 2 us beside the down weights; the sum over experts, 3 us.
// With few bytes that latency is all there is: 11.4 us for 5 tokens at d 256, f 512.
//
// Phases of a CTA (one per SM, 384 threads): warps 4-11 write their share of the x operand image to the workspace while
// warps 0-3 build the expert lists; warp 0 streams weight tiles, warp 2 token tiles (they wait for the image, then for
// H), warp 1 issues the MMAs, warps 4-11 drain the accumulators: gate/up partials or H, then down partials; at the end
// the CTAs that worked on a 256-column block of the output share its weighted sum out among them.  Nothing is summed
// with atomics, so results do not depend on timing.
//
// Counters in the workspace come in two sets: a launch counts in one and zeroes the other for the next launch; which
// one is told by a count, modulo twice the grid, that every CTA bumps once as it leaves.  Every wait is bounded (FewParams::wait_ns).
#include <cuda_fp16.h>

#include "mma_warp.cuh"

namespace tempo {

constexpr int kFewThreads = 384;
constexpr int kFewRing = 8;                 // most stages
constexpr int kFewBudget = 222 * 1024;      // dynamic shared memory: ring, then the lists
// Weight tiles of a CTA on their way at a time: 96 KB per SM cover the memory's latency at its full rate; 2 leave gaps, and
// with 4 the CTAs that a line is shared by drift apart (both slower on every size measured).
constexpr uint32_t kFewFlight = 3;
// Fewest blocks of a gate/up line that are worth a CTA of their own (2, 4 and 16 were slower where a phase has few blocks,
// and make no difference where it has many).
constexpr int kFewRun = 8;
// Token columns that an epilogue group takes at a time.  8 would serve many tokens on one expert (64: 34.5 us, not 35.6), but
// their registers cost every other size 0.2 to 0.5 us.
constexpr int kFewBatch = 4;
constexpr int kFewHalf = 8;                 // fewest gate/up blocks per CTA of a half

// ---- small helpers --------------------------------------------------------------------------------
__device__ __forceinline__ void bar_sync(int id, int n) { asm volatile("bar.sync %0, %1;" ::"r"(id), "r"(n) : "memory"); }
// Adds to a counter after everything this thread has seen written (a barrier before it makes that the CTA's writes).
__device__ __forceinline__ void add_release(int32_t* p, int v) {
  asm volatile("red.release.gpu.global.add.s32 [%0], %1;" ::"l"(p), "r"(v) : "memory");
}
__device__ __forceinline__ void bar_arrive(int id, int n) { asm volatile("bar.arrive %0, %1;" ::"r"(id), "r"(n) : "memory"); }
// Barrier of n threads that tells every one of them whether `ok` held in all.
__device__ __forceinline__ bool bar_all(int id, int n, bool ok) {
  uint32_t r;
  asm volatile(
      "{\n\t.reg .pred p, q;\n\t"
      "setp.ne.u32 p, %3, 0;\n\t"
      "barrier.cta.red.and.pred q, %1, %2, p;\n\t"
      "selp.u32 %0, 1, 0, q;\n\t}"
      : "=r"(r) : "r"(id), "r"(n), "r"(ok ? 1u : 0u) : "memory");
  return r != 0;
}
__device__ __forceinline__ void tmem_ld1(uint32_t taddr, uint32_t& r) {
  asm volatile("tcgen05.ld.sync.aligned.32x32b.x1.b32 {%0}, [%1];" : "=r"(r) : "r"(taddr) : "memory");
}
__device__ __forceinline__ void tmem_ld4(uint32_t taddr, uint32_t (&r)[4]) {
  asm volatile("tcgen05.ld.sync.aligned.32x32b.x4.b32 {%0, %1, %2, %3}, [%4];"
               : "=r"(r[0]), "=r"(r[1]), "=r"(r[2]), "=r"(r[3]) : "r"(taddr) : "memory");
}
__device__ __forceinline__ bool few_poll(const int32_t* flag, int want, volatile int* abort_flag, unsigned long long limit_ns) {
  unsigned long long t0 = 0;
  for (uint32_t it = 0; ld_acquire(flag) < want; ++it) {
    if ((it & 63u) == 63u) {
      if (*abort_flag) return false;
      const unsigned long long now = global_timer_ns();
      if (t0 == 0) t0 = now;
      else if (now - t0 > limit_ns) { *abort_flag = 1; return false; }
    }
  }
  return true;
}

// Run of CTA c when B blocks are dealt to C CTAs, and the CTA that block b falls to (products below 2^32, checked on
// the host).
__device__ __forceinline__ uint32_t run_begin(uint32_t c, uint32_t C, uint32_t B) { return c * B / C; }
__device__ __forceinline__ uint32_t run_owner(uint32_t b, uint32_t C, uint32_t B) { return ((b + 1) * C - 1) / B; }

// One of the four phases of a launch: gate/up of the first half of the active experts, of the second half, then down of
// the first and of the second.  While a half's H is being summed and published the other half's weights stream.
struct FewPhase {
  int a0, an;                              // its active experts
  uint32_t B, C;                           // blocks, CTAs that they are dealt to
  uint32_t b, e;                           // this CTA's run
  int line, kb0, q, r;                     // where the run begins: line, K-block in it, line / inner, line % inner
};
__device__ __forceinline__ void few_phase(FewPhase& f, const FewParams& p, int ph, int A, uint32_t ctas, uint32_t cta) {
  // two halves where each of them keeps every CTA busy
  const int A1 = static_cast<uint32_t>(A) * p.NT1 * p.Kb1 >= 2u * kFewHalf * ctas && A >= 2 ? (A + 1) / 2 : A;
  f.a0 = (ph & 1) ? A1 : 0;
  f.an = (ph & 1) ? A - A1 : A1;
  const bool down = ph >= 2;
  const uint32_t Kb = down ? p.Kb2 : p.Kb1, inner = down ? f.an : p.NT1;
  const uint32_t lines = static_cast<uint32_t>(f.an) * (down ? p.NT2 : p.NT1);
  f.B = lines * Kb;
  // Short phases are dealt to fewer CTAs.  Gate/up: a line is cut only into runs of kFewRun blocks or more (a cut costs
  // an exchange of partial sums).  Down: into at most kFewSplit partial sums, i.e. a third of a line per CTA.
  f.C = down ? 3u * lines : max(lines, f.B / kFewRun);
  f.C = max(1u, min(f.C, min(ctas, f.B)));
  f.b = cta < f.C ? run_begin(cta, f.C, f.B) : 0u;
  f.e = cta < f.C ? run_begin(cta + 1, f.C, f.B) : 0u;
  f.line = f.kb0 = f.q = f.r = 0;
  if (f.e > f.b) {
    f.line = static_cast<int>(f.b / Kb);
    f.kb0 = static_cast<int>(f.b - f.line * Kb);
    f.q = f.line / static_cast<int>(inner);
    f.r = f.line % static_cast<int>(inner);
  }
}
// Segments of a CTA's run: the parts of lines (one expert's column block, Kb blocks long) that it covers.  Lines are
// a * NT1 + nt (gate/up) or nt * an + a (down), a counted within the phase.
struct FewIter {
  int left, Kb, inner, a0, q, r;
  bool down;
  int a, nt, kb0, kb1, line;               // the segment
  __device__ FewIter(const FewParams& p, const FewPhase& f, bool down_) {
    down = down_;
    left = static_cast<int>(f.e - f.b);
    Kb = down ? p.Kb2 : p.Kb1;
    inner = down ? f.an : p.NT1;
    a0 = f.a0; q = f.q; r = f.r - 1; line = f.line - 1;
    kb1 = f.kb0;
  }
  __device__ bool next() {
    if (left <= 0) return false;
    kb0 = kb1 == Kb ? 0 : kb1;             // only the run's first segment may begin inside its line
    kb1 = min(Kb, kb0 + left);
    left -= kb1 - kb0;
    ++line;
    if (++r == inner) { r = 0; ++q; }
    a = a0 + (down ? r : q);
    nt = down ? q : r;
    return true;
  }
};

// Block exponent of the two-term split: 2^eps * 448 covers the block, and eps - 4 is still a valid scale.
__device__ __forceinline__ int split_exponent(float amax) { return max(pow2_scale_exponent(amax), -122); }
// (v, v') -> two e4m3 codes of the first and of the second term; a value that is not finite gives NaN codes.
__device__ __forceinline__ void split_e4m3(float a, float b, float inv, uint32_t& q1, uint32_t& q2) {
  a *= inv;
  b *= inv;
  q1 = cvt_e4m3x2(a, b);
  uint32_t h;                                                   // the codes as two f16 values (exact)
  asm("cvt.rn.f16x2.e4m3x2 %0, %1;" : "=r"(h) : "h"(static_cast<uint16_t>(q1)));
  const __half2 hh = *reinterpret_cast<const __half2*>(&h);
  q2 = cvt_e4m3x2((a - __low2float(hh)) * 16.f, (b - __high2float(hh)) * 16.f);
  if (!isfinite(a)) { q1 |= 0x7fu; }
  if (!isfinite(b)) { q1 |= 0x7f00u; }
}

__device__ __forceinline__ uint32_t few_idesc_fp8(int n, int sf_id) {     // weights: A (scale id = K-block % 4), tokens: B (id 0)
  return (static_cast<uint32_t>(n >> 3) << 17) | (1u << 23) | (static_cast<uint32_t>(kTileM >> 4) << 24) |
         (static_cast<uint32_t>(sf_id) << 29);
}
__device__ __forceinline__ uint32_t few_idesc_bf16(int n) {
  return (1u << 4) | (1u << 7) | (1u << 10) | (static_cast<uint32_t>(n >> 3) << 17) | (static_cast<uint32_t>(kTileM >> 4) << 24);
}

struct FewLists {                          // in dynamic shared memory behind the ring
  unsigned long long* mask;                // [G]  tokens of each instance slot, bit t
  uint16_t* act;                           // [A]  instance slot of the a-th active expert (ascending)
  uint16_t* off;                           // [A+1] (token, expert) pairs before it
  uint16_t* hrow;                          // [A]  operand rows of H before it
  int16_t* s2a;                            // [G]  inverse of act
  int16_t* pa;                             // [T*k] slot of each pair, -1: none on this rank; then see below
  int16_t* pu;                             // [T*k] its row of the down partials
  uint8_t* tok;                            // [T*k] token of each row of the down partials (by expert, then token)
  float* w;                                // [T*k] routing weights
  int16_t* first;                          // [E]  first replica column of every expert (-1: not a slot)
  uint8_t* split;                          // [2][A] partial sums per expert of the column block being reduced
};
__host__ __device__ inline size_t few_list_bytes(int G, int P, int E) {
  const size_t A = G < P ? G : P;
  return static_cast<size_t>(G) * 8 + (2 * (A + 1) + 7) / 8 * 8 * 3 + (2 * static_cast<size_t>(G) + 7) / 8 * 8 +
         (2 * static_cast<size_t>(P) + 7) / 8 * 8 * 2 + (4 * static_cast<size_t>(P) + 7) / 8 * 8 + (static_cast<size_t>(P) + 7) / 8 * 8 + (2 * static_cast<size_t>(E) + 7) / 8 * 8 + (2 * A + 7) / 8 * 8;
}

template <bool kBf16>
__global__ void __launch_bounds__(kFewThreads, 1) few_kernel(const FewParams p) {
  extern __shared__ uint8_t smem_raw[];
  __shared__ __align__(16) uint64_t s_bars[3 * kFewRing];
  uint64_t *s_full = s_bars, *s_tok = s_bars + kFewRing, *s_empty = s_bars + 2 * kFewRing;   // weight tile, token tile landed; free
  __shared__ __align__(8) uint64_t s_acc_full[2];
  __shared__ __align__(8) uint64_t s_acc_empty[2];
  __shared__ uint32_t s_tmem_base;
  __shared__ int s_abort_storage, s_A;
  __shared__ FewPhase s_phase[4];
  __shared__ int s_local[kFewMaxT];        // pairs on this rank of each token
  __shared__ uint32_t s_amax[2][2][4][kFewBatch];  // [batch parity][group][warp][token]
  volatile int* s_abort = &s_abort_storage;

  const int tid = threadIdx.x, warp = tid >> 5, lane = tid & 31;
  const uint32_t smem_base = (smem_u32(smem_raw) + 1023u) & ~1023u;
  const uint32_t C = gridDim.x, cta = blockIdx.x;
  const int T = p.T, k = p.k, G = p.G, P = T * k, A_cap = min(G, P);
  constexpr int kTerms = kBf16 ? 1 : 2;    // columns per token of the gate/up product
  FewLists L;
  {
    uint8_t* q = smem_raw + (smem_base - smem_u32(smem_raw)) + p.stages * p.stage_bytes;
    const size_t act_bytes = ((static_cast<size_t>(A_cap) + 1) * 2 + 7) / 8 * 8;
    L.mask = reinterpret_cast<unsigned long long*>(q); q += static_cast<size_t>(G) * 8;
    L.act = reinterpret_cast<uint16_t*>(q); q += act_bytes;
    L.off = reinterpret_cast<uint16_t*>(q); q += act_bytes;
    L.hrow = reinterpret_cast<uint16_t*>(q); q += act_bytes;
    L.s2a = reinterpret_cast<int16_t*>(q); q += (static_cast<size_t>(G) * 2 + 7) / 8 * 8;
    L.pa = reinterpret_cast<int16_t*>(q); q += (static_cast<size_t>(P) * 2 + 7) / 8 * 8;
    L.pu = reinterpret_cast<int16_t*>(q); q += (static_cast<size_t>(P) * 2 + 7) / 8 * 8;
    L.w = reinterpret_cast<float*>(q); q += (static_cast<size_t>(P) * 4 + 7) / 8 * 8;
    L.tok = q; q += (static_cast<size_t>(P) + 7) / 8 * 8;
    L.first = reinterpret_cast<int16_t*>(q); q += (static_cast<size_t>(p.E) * 2 + 7) / 8 * 8;
    L.split = q;
  }
  pdl_trigger();
  // prologue that needs nothing from the previous kernel
  if (tid == 0) {
    for (int s = 0; s < p.stages; ++s) {
      mbar_init(smem_u32(&s_full[s]), 1);
      mbar_init(smem_u32(&s_tok[s]), 1);
      mbar_init(smem_u32(&s_empty[s]), 1);
    }
    for (int s = 0; s < 2; ++s) { mbar_init(smem_u32(&s_acc_full[s]), 1); mbar_init(smem_u32(&s_acc_empty[s]), 8); }
    s_abort_storage = 0;
    asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
  }
  if (warp == 1) {
    asm volatile("tcgen05.alloc.cta_group::1.sync.aligned.shared::cta.b32 [%0], %1;" ::"r"(smem_u32(&s_tmem_base)),
                 "r"(kTmemCols) : "memory");
    asm volatile("tcgen05.relinquish_alloc_permit.cta_group::1.sync.aligned;" ::: "memory");
  }
  for (int i = tid; i < G; i += kFewThreads) L.mask[i] = 0ull;
  tc_fence_before();
  __syncthreads();
  tc_fence_after();
  const uint32_t tmem_base = s_tmem_base;
  pdl_wait();
  const uint32_t left = *reinterpret_cast<volatile const uint32_t*>(p.leave);
  const int n_valid = p.n_valid != nullptr ? *p.n_valid : T;
  // The first pairs and the replica map's first column are requested before anything waits for what was just read: one
  // memory latency for all of it.
  int id[4];
  float w[4];
  if (warp < 4) {
#pragma unroll
    for (int j = 0; j < 4; ++j) {
      id[j] = tid + 128 * j < P ? p.ids[tid + 128 * j] : 0;
      w[j] = tid + 128 * j < P ? p.w[tid + 128 * j] : 0.f;
    }
#pragma unroll 4
    for (int e = tid; e < p.E; e += 128) {
      const int v = p.replica_map[e * p.R];
      L.first[e] = static_cast<int16_t>(v >= 0 && v < G ? v : -1);
    }
  }
  const int nv = max(0, min(n_valid, T));
  // CTAs count modulo 2 C as they leave: a launch finds the count in [0, C) or in [C, 2 C), with those of its own CTAs
  // that have left already
  int32_t* cnt = p.counters + (left >= C ? p.counter_ints : 0);
  int32_t* cnt_next = p.counters + (left >= C ? 0 : p.counter_ints);
  // h_done: 32 ints per half; part_done: [half][CTA], the partial sums of that CTA's first segment are in the workspace
  int32_t *x_done = cnt, *h_done = cnt + 32, *y_cnt = cnt + 96, *part_done = cnt + 96 + p.NT2;
  const int T8 = (T + 7) & ~7;
  const int R1 = kBf16 ? (T + 15) & ~15 : 2 * T8;                   // operand rows of x: MMA columns of gate/up
  const uint32_t x_block = R1 * 128 + (kBf16 ? 0 : 512);           // one K-block of the x image, scale atom behind it
  const int units = p.Kb1 * nv;
  const int x_want = min(static_cast<int>(C), (units + 7) / 8);

  if (warp < 4) {
    // ---- expert lists (128 threads) ----------------------------------------------------------------
    bar_sync(1, 128);
    bool bad = false;
    for (int i0 = tid; i0 < P; i0 += 512) {
#pragma unroll
      for (int j = 0; j < 4; ++j) {
        const int i = i0 + 128 * j;
        if (i >= P) break;
        const bool live = i < nv * k;
        if (i0 >= 512) {
          id[j] = p.ids[i];
          w[j] = p.w[i];
        }
        const bool good = id[j] >= 0 && id[j] < p.E;
        bad |= live && !good;
        int v = live && good ? L.first[id[j]] : -1;
        for (int r = 1; r < p.R && v < 0 && live && good; ++r) {     // else the first replica on this rank
          const int u = p.replica_map[id[j] * p.R + r];
          if (u < G) v = u;
        }
        L.pa[i] = static_cast<int16_t>(v < 0 ? -1 : v);
        L.w[i] = w[j];
        if (v >= 0) {                                                // the union of bits: no order
          const int t = i / k;
          atomicOr(reinterpret_cast<uint32_t*>(&L.mask[v]) + (t >> 5), 1u << (t & 31));   // (low word first)
        }
      }
    }
    if (bad && cta == 0) atomicOr(p.status, static_cast<uint32_t>(TEMPO_STATUS_BAD_ID));
    bar_sync(1, 128);
    if (warp == 0) {
      // 128 slots per turn, four neighbours to a lane; experts, pairs and operand rows before a slot in one 64-bit scan
      unsigned long long before = 0;                                // 16 bits each: experts, pairs, rows
      for (int base = 0; base < G; base += 128) {
        unsigned long long n4[4], sum = 0;
#pragma unroll
        for (int q = 0; q < 4; ++q) {
          const int i = base + 4 * lane + q, n = i < G ? __popcll(L.mask[i]) : 0;
          n4[q] = n == 0 ? 0ull : 1ull | static_cast<unsigned long long>(n) << 16 | static_cast<unsigned long long>(2 * ((n + 7) & ~7)) << 32;
          sum += n4[q];
        }
        unsigned long long incl = sum;
#pragma unroll
        for (int o = 1; o < 32; o <<= 1) {
          const unsigned long long u = __shfl_up_sync(0xffffffffu, incl, o);
          if (lane >= o) incl += u;
        }
        unsigned long long at = before + incl - sum;
#pragma unroll
        for (int q = 0; q < 4; ++q) {
          if (n4[q] != 0) {
            const int a = static_cast<int>(at & 0xffff), i = base + 4 * lane + q;
            L.act[a] = static_cast<uint16_t>(i);
            L.off[a] = static_cast<uint16_t>(at >> 16);
            L.hrow[a] = static_cast<uint16_t>(at >> 32);
            L.s2a[i] = static_cast<int16_t>(a);
          }
          at += n4[q];
        }
        before += __shfl_sync(0xffffffffu, incl, 31);
      }
      if (lane == 0) { s_A = static_cast<int>(before & 0xffff); L.off[before & 0xffff] = static_cast<uint16_t>(before >> 16); }
    } else if (warp == 1) {                                         // the runs need the number of experts only
      int n = 0;
      for (int base = 0; base < G; base += 32) n += __popc(__ballot_sync(0xffffffffu, base + lane < G && L.mask[base + lane] != 0ull));
      if (lane < 4) few_phase(s_phase[lane], p, lane, n, C, cta);
    }
    bar_sync(1, 128);
    bar_arrive(2, kFewThreads);                                     // the lists, for the epilogue warps
  } else {
    // ---- this CTA's share of the x operand image: one (K-block, token) per warp and turn --------------
    for (int u = static_cast<int>(cta) * 8 + warp - 4; u < units; u += static_cast<int>(C) * 8) {
      const int kb = u / nv, t = u - kb * nv;
      uint8_t* blk = p.x_img + static_cast<size_t>(kb) * x_block;
      if constexpr (kBf16) {
        const uint32_t v = *reinterpret_cast<const uint32_t*>(p.x + static_cast<size_t>(t) * p.d + kb * 64 + lane * 2);
        *reinterpret_cast<uint32_t*>(blk + t * 128 + (((lane >> 2) ^ (t & 7)) << 4) + (lane & 3) * 4) = v;
      } else {
        const uint2 v = *reinterpret_cast<const uint2*>(p.x + static_cast<size_t>(t) * p.d + kb * 128 + lane * 4);
        uint32_t m = max(max(v.x & 0x7fffu, (v.x >> 16) & 0x7fffu), max(v.y & 0x7fffu, (v.y >> 16) & 0x7fffu));
        m = __reduce_max_sync(0xffffffffu, m);                      // bits of a bf16 magnitude order like its value
        const int eps = split_exponent(__uint_as_float(m << 16));
        const float inv = pow2_neg(eps);
        uint32_t a1, a2, b1, b2;
        split_e4m3(__uint_as_float(v.x << 16), __uint_as_float(v.x & 0xffff0000u), inv, a1, a2);
        split_e4m3(__uint_as_float(v.y << 16), __uint_as_float(v.y & 0xffff0000u), inv, b1, b2);
        const int r1 = t, r2 = T8 + t;
        const int at = (lane >> 2), in = (lane & 3) * 4;
        *reinterpret_cast<uint32_t*>(blk + r1 * 128 + ((at ^ (r1 & 7)) << 4) + in) = a1 | (b1 << 16);
        *reinterpret_cast<uint32_t*>(blk + r2 * 128 + ((at ^ (r2 & 7)) << 4) + in) = a2 | (b2 << 16);
        if (lane < 2) {                                             // scale byte: word of the row, byte 0
          const int r = lane == 0 ? r1 : r2;
          blk[R1 * 128 + (r & 31) * 16 + (r >> 5) * 4] = static_cast<uint8_t>(eps + 127 - 4 * lane);
        }
      }
    }
    bar_sync(3, 256);
    if (tid == 128 && static_cast<int>(cta) < x_want) add_release(x_done, 1);
    for (int i = static_cast<int>(cta) * 256 + tid - 128; i < p.counter_ints; i += static_cast<int>(C) * 256) cnt_next[i] = 0;
    bar_sync(2, kFewThreads);
  }
  const int A = s_A;

  if (warp == 0) {
    // ---- weight producer ---------------------------------------------------------------------------
    if (lane == 0) {
      uint32_t stage = 0, phase = 0;
      uint32_t old_stage = 0, old_phase = 0, issued = 0;            // the block kFewFlight before the next one
      bool ok = true;
#pragma unroll 1
      for (int ph = 0; ph < 4; ++ph) {
        const bool down = ph >= 2;
        FewIter s(p, s_phase[ph], down);
        const int NT = down ? p.NT2 : p.NT1, Kb = down ? p.Kb2 : p.Kb1, J = down ? p.J2 : p.J1;
        const uint8_t* wt = down ? p.w2 : p.w13;
        const uint8_t* sf = down ? p.sf2 : p.sf13;
        while (ok && s.next()) {
          const size_t tile = static_cast<size_t>(L.act[s.a]) * NT + s.nt;
          const uint8_t* src = wt + tile * Kb * kBBytes;
          const uint8_t* sf_src = sf + tile * J * kSfbBytes;
#pragma unroll 1
          for (int kb = s.kb0; kb < s.kb1; ++kb) {
            if (!mbar_wait(smem_u32(&s_empty[stage]), phase ^ 1u, s_abort, p.wait_ns)) { ok = false; break; }
            if (issued++ >= kFewFlight) {
              if (!mbar_wait(smem_u32(&s_full[old_stage]), old_phase, s_abort, p.wait_ns)) { ok = false; break; }
              if (++old_stage == static_cast<uint32_t>(p.stages)) { old_stage = 0; old_phase ^= 1u; }
            }
            const uint32_t full = smem_u32(&s_full[stage]), sA = smem_base + stage * p.stage_bytes;
            const bool with_sf = !kBf16 && ((kb & 3) == 0 || kb == s.kb0);
            mbar_arrive_expect_tx(full, kBBytes + (with_sf ? kSfbBytes : 0));
            bulk_load_stream(sA, src + static_cast<size_t>(kb) * kBBytes, kBBytes, full);
            if (with_sf) bulk_load(sA + kBBytes, sf_src + static_cast<size_t>(kb >> 2) * kSfbBytes, kSfbBytes, full);
            if (++stage == static_cast<uint32_t>(p.stages)) { stage = 0; phase ^= 1u; }
          }
        }
      }
    }
  } else if (warp == 2) {
    // ---- token producer: x image, then H image -------------------------------------------------------
    if (lane == 0) {
      uint32_t stage = 0, phase = 0;
      bool ok = true;
#pragma unroll 1
      for (int ph = 0; ph < 4; ++ph) {
        FewIter s(p, s_phase[ph], ph >= 2);
        if (s.left <= 0) continue;
        ok = ok && few_poll(ph < 2 ? x_done : h_done + 32 * (ph - 2), ph < 2 ? x_want : s_phase[ph].an * p.NT1, s_abort, p.wait_ns);
        asm volatile("fence.proxy.async;" ::: "memory");            // ordinary stores before the bulk copies below
        while (ok && s.next()) {
          uint32_t bytes = x_block;
          const uint8_t* src = p.x_img;
          if (ph >= 2) {
            const int rows = 2 * ((L.off[s.a + 1] - L.off[s.a] + 7) & ~7);
            bytes = rows * 128 + (kBf16 ? 0 : 512);
            src = p.h_img + static_cast<size_t>(p.Kb2) * (static_cast<size_t>(L.hrow[s.a]) * 128 + (kBf16 ? 0 : 512) * static_cast<size_t>(s.a));
          }
#pragma unroll 1
          for (int kb = s.kb0; kb < s.kb1; ++kb) {
            if (!mbar_wait(smem_u32(&s_empty[stage]), phase ^ 1u, s_abort, p.wait_ns)) { ok = false; break; }
            const uint32_t full = smem_u32(&s_tok[stage]);
            mbar_arrive_expect_tx(full, bytes);
            bulk_load(smem_base + stage * p.stage_bytes + kBBytes + kSfbBytes, src + static_cast<size_t>(kb) * bytes, bytes, full);
            if (++stage == static_cast<uint32_t>(p.stages)) { stage = 0; phase ^= 1u; }
          }
        }
      }
    }
  } else if (warp == 1) {
    // ---- MMA issuer ------------------------------------------------------------------------------------
    const uint32_t leader = elect_one();
    const uint32_t bars = smem_u32(s_bars), desc0 = desc_lo_sw128(smem_base), desc_step = p.stage_bytes >> 4;
    uint32_t sf_slot = tmem_base + kSfCol0, tok_slot = tmem_base + kSfCol0 + 16u;        // two of each, used in turn
    uint32_t stage = 0, phase = 0, n_seg = 0;
    bool ok = true;
#pragma unroll 1
    for (int ph = 0; ph < 4 && ok; ++ph) {
      FewIter s(p, s_phase[ph], ph >= 2);
      while (ok && warp_uniform(s.next()) != 0) {
        const int N = warp_uniform(ph < 2 ? R1 : 2 * ((L.off[s.a + 1] - L.off[s.a] + 7) & ~7));
        const int kb0 = warp_uniform(s.kb0), kb1 = warp_uniform(s.kb1);
        const uint32_t slot = p.slots == 2 ? n_seg & 1u : 0u, use = p.slots == 2 ? n_seg >> 1 : n_seg;
        ++n_seg;
        if (!mbar_wait_warp(smem_u32(&s_acc_empty[slot]), (use & 1u) ^ 1u, s_abort, p.wait_ns)) { ok = false; break; }
        tc_fence_after();
        const uint32_t acc = tmem_base + slot * 128u, acc2 = acc + N;
        const uint32_t idesc0 = kBf16 ? few_idesc_bf16(N) : few_idesc_fp8(N, 0);
        uint32_t accumulate = 0;
#pragma unroll 1
        for (int kb = kb0; kb < kb1; ++kb) {
          if (!mbar_wait_warp(bars + 8 * stage, phase, s_abort, p.wait_ns) ||
              !mbar_wait_warp(bars + 8 * (kFewRing + stage), phase, s_abort, p.wait_ns)) { ok = false; break; }
          tc_fence_after();
          const uint32_t da = desc0 + stage * desc_step, db = da + ((kBBytes + kSfbBytes) >> 4), da2 = da + ((kTileM * 128) >> 4);
          if constexpr (kBf16) {
#pragma unroll
            for (int ks = 0; ks < 4; ++ks) warp_mma_bf16(leader, acc, da + 2 * ks, db + 2 * ks, idesc0, ks == 0 ? accumulate : 1u);
#pragma unroll
            for (int ks = 0; ks < 4; ++ks) warp_mma_bf16(leader, acc2, da2 + 2 * ks, db + 2 * ks, idesc0, ks == 0 ? accumulate : 1u);
          } else {
            const uint32_t sSF = smem_base + stage * p.stage_bytes + kBBytes;
            if ((kb & 3) == 0 || accumulate == 0) {
              sf_slot ^= 8u;
              warp_cp_sf(leader, sf_slot, sSF);
              warp_cp_sf(leader, sf_slot + 4, sSF + 512);
            }
            tok_slot ^= 4u;
            warp_cp_sf(leader, tok_slot, sSF + kSfbBytes + N * 128);
            const uint32_t idesc = idesc0 | static_cast<uint32_t>(kb & 3) << 29;
#pragma unroll
            for (int ks = 0; ks < 4; ++ks)
              warp_mma_fp8(leader, acc, da + 2 * ks, db + 2 * ks, idesc, sf_slot, tok_slot, ks == 0 ? accumulate : 1u);
#pragma unroll
            for (int ks = 0; ks < 4; ++ks)
              warp_mma_fp8(leader, acc2, da2 + 2 * ks, db + 2 * ks, idesc, sf_slot + 4, tok_slot, ks == 0 ? accumulate : 1u);
          }
          accumulate = 1;
          warp_commit(leader, bars + 8 * (2 * kFewRing + stage));
          if (++stage == static_cast<uint32_t>(p.stages)) { stage = 0; phase ^= 1u; }
        }
        if (ok) warp_commit(leader, smem_u32(&s_acc_full[slot]));
      }
    }
  } else if (warp >= 4) {
    // ---- epilogue: two groups of four warps; a thread owns row `row` of both 128-row halves of a tile ------
    const int g = (warp - 4) >> 2, quad = warp & 3, row = quad * 32 + lane, et = tid - 128;
    const uint32_t lanes = static_cast<uint32_t>(quad * 32) << 16;
    uint32_t n_seg = 0, par = 0;
    bool ok = true;
    if (et < T) {                                                   // a token's pairs on this rank, packed to the front
      const int t = et;
      int n = 0;
      for (int q = 0; q < k; ++q) {
        const int sl = L.pa[t * k + q];
        if (sl < 0) continue;
        const int a = L.s2a[sl], u = L.off[a] + __popcll(L.mask[sl] & ((1ull << t) - 1ull));
        L.pa[t * k + n] = static_cast<int16_t>(a);                  // active expert, row of its partials, weight
        L.pu[t * k + n] = static_cast<int16_t>(u);
        L.w[t * k + n] = L.w[t * k + q];
        L.tok[u] = static_cast<uint8_t>(t);
        ++n;
      }
      s_local[t] = n;
    }
    // ---- gate/up.  The CTA with a line's first block finishes it: its part of the line is the last of its run, while
    // the other parts are the first segments of the runs after it, done long before except in runs of one line.  So nobody
    // waits in a circle, and mostly not at all.
#pragma unroll 1
    for (int ph = 0; ph < 2; ++ph) {
      const FewPhase& f = s_phase[ph];
      FewIter s(p, f, false);
      while (ok && s.next()) {
        const uint32_t slot = p.slots == 2 ? n_seg & 1u : 0u, use = p.slots == 2 ? n_seg >> 1 : n_seg;
        ++n_seg;
        const int last = s.kb0 == 0 && s.kb1 < p.Kb1 ? static_cast<int>(run_owner(s.line * p.Kb1 + p.Kb1 - 1, f.C, f.B)) : static_cast<int>(cta);
        bool seen = mbar_wait(smem_u32(&s_acc_full[slot]), use & 1u, s_abort, p.wait_ns);
        for (int c = static_cast<int>(cta) + 1 + et; c <= last; c += 256)
          seen = seen && few_poll(part_done + ph * C + c, 1, s_abort, p.wait_ns);
        ok = bar_all(3, 256, seen);
        if (!ok) break;
        tc_fence_after();
        const uint32_t acc = tmem_base + slot * 128u + lanes;
        const int u0 = L.off[s.a], n_col = L.off[s.a + 1] - u0, C8 = (n_col + 7) & ~7;
        uint8_t* himg = p.h_img + static_cast<size_t>(p.Kb2) * (static_cast<size_t>(L.hrow[s.a]) * 128 + (kBf16 ? 0 : 512) * static_cast<size_t>(s.a));
        float* mine = p.gu_part + (static_cast<size_t>(ph) * C + cta) * T * 256 + row;     // [token column][half][row]
#pragma unroll 1
        for (int c0 = g * kFewBatch; c0 < n_col; c0 += 2 * kFewBatch) {
          uint32_t v[kFewBatch][2][kTerms];
#pragma unroll
          for (int i = 0; i < kFewBatch; ++i) {
            const uint32_t t = L.tok[u0 + min(c0 + i, n_col - 1)];
#pragma unroll
            for (int h = 0; h < 2; ++h)
#pragma unroll
              for (int j = 0; j < kTerms; ++j) tmem_ld1(acc + h * R1 + j * T8 + t, v[i][h][j]);
          }
          tmem_wait_ld();
          float gu[kFewBatch][2];
#pragma unroll
          for (int i = 0; i < kFewBatch; ++i)
#pragma unroll
            for (int h = 0; h < 2; ++h) {
              gu[i][h] = __uint_as_float(v[i][h][0]);
              if constexpr (kTerms == 2) gu[i][h] += __uint_as_float(v[i][h][1]);
            }
          if (s.kb0 > 0) {                                          // another CTA's line: hand the partial sums over
#pragma unroll
            for (int i = 0; i < kFewBatch; ++i)
              if (c0 + i < n_col) {
                __stcg(mine + (c0 + i) * 256, gu[i][0]);
                __stcg(mine + (c0 + i) * 256 + 128, gu[i][1]);
              }
            continue;
          }
          for (int ca = static_cast<int>(cta) + 1; ca <= last; ca += 3) {   // the other parts, three in flight, in the order of the runs
            float v3[3][kFewBatch][2];
#pragma unroll
            for (int m = 0; m < 3; ++m) {
              const float* src = p.gu_part + (static_cast<size_t>(ph) * C + min(ca + m, last)) * T * 256 + row;
#pragma unroll
              for (int i = 0; i < kFewBatch; ++i) {
                const bool on = ca + m <= last && c0 + i < n_col;
                v3[m][i][0] = on ? __ldcg(src + (c0 + i) * 256) : 0.f;
                v3[m][i][1] = on ? __ldcg(src + (c0 + i) * 256 + 128) : 0.f;
              }
            }
#pragma unroll
            for (int m = 0; m < 3; ++m)
#pragma unroll
              for (int i = 0; i < kFewBatch; ++i) {
                gu[i][0] += v3[m][i][0];
                gu[i][1] += v3[m][i][1];
              }
          }
          // H of this (expert, 128-column block): SwiGLU, the two-term split, straight into the operand image
#pragma unroll
          for (int i = 0; i < kFewBatch; ++i) gu[i][0] = __fdividef(gu[i][0], 1.f + __expf(-gu[i][0])) * gu[i][1];
          if constexpr (kBf16) {
            uint8_t* blk = himg + static_cast<size_t>(s.nt * 2 + (row >> 6)) * (2 * C8 * 128);
            const int ii = row & 63;
#pragma unroll
            for (int i = 0; i < kFewBatch; ++i)
              if (c0 + i < n_col) {
                const int col = c0 + i, r2 = C8 + col;
                // beyond bf16's range: NaN, as the other form's codes (an infinite first term alone would give an infinite output)
                __nv_bfloat16 hi = __float2bfloat16_rn(gu[i][0]);
                const float hf = __bfloat162float(hi);
                if (!isfinite(hf)) hi = __ushort_as_bfloat16(0x7fff);
                const __nv_bfloat16 lo = __float2bfloat16_rn(isfinite(hf) ? gu[i][0] - hf : 0.f);
                *reinterpret_cast<__nv_bfloat16*>(blk + col * 128 + (((ii >> 3) ^ (col & 7)) << 4) + (ii & 7) * 2) = hi;
                *reinterpret_cast<__nv_bfloat16*>(blk + r2 * 128 + (((ii >> 3) ^ (r2 & 7)) << 4) + (ii & 7) * 2) = lo;
              }
          } else {
#pragma unroll
            for (int i = 0; i < kFewBatch; ++i) {
              const uint32_t m = __reduce_max_sync(0xffffffffu, __float_as_uint(gu[i][0]) & 0x7fffffffu);
              if (lane == i) s_amax[par][g][quad][i] = m;
            }
            bar_sync(4 + g, 128);
            uint8_t* blk = himg + static_cast<size_t>(s.nt) * (2 * C8 * 128 + 512);
#pragma unroll
            for (int i = 0; i < kFewBatch; ++i)
              if (c0 + i < n_col) {
                const uint32_t m = max(max(s_amax[par][g][0][i], s_amax[par][g][1][i]), max(s_amax[par][g][2][i], s_amax[par][g][3][i]));
                const int eps = split_exponent(__uint_as_float(m));
                uint32_t q1, q2;
                split_e4m3(gu[i][0], 0.f, pow2_neg(eps), q1, q2);
                const int col = c0 + i, r2 = C8 + col;
                blk[col * 128 + (((row >> 4) ^ (col & 7)) << 4) + (row & 15)] = static_cast<uint8_t>(q1);
                blk[r2 * 128 + (((row >> 4) ^ (r2 & 7)) << 4) + (row & 15)] = static_cast<uint8_t>(q2);
                if (row < 2) {
                  const int r = row == 0 ? col : r2;
                  blk[2 * C8 * 128 + (r & 31) * 16 + (r >> 5) * 4] = static_cast<uint8_t>(eps + 127 - 4 * row);
                }
              }
            par ^= 1u;
          }
        }
        tc_fence_before();
        __syncwarp();
        if (lane == 0) mbar_arrive(smem_u32(&s_acc_empty[slot]));
        bar_sync(3, 256);
        if (et == 0) add_release(s.kb0 > 0 ? part_done + ph * C + cta : h_done + 32 * ph, 1);   // the partial sums, or H
      }
    }
    // ---- down: partial sums of (256 output columns, expert), one row of Y per (token, expert) pair -----------
    int pend_nt = -1, pend = 0;                                     // blocks of column block pend_nt not yet published
#pragma unroll 1
    for (int ph = 2; ph < 4; ++ph) {
      const FewPhase& f = s_phase[ph];
      FewIter s(p, f, true);
      while (ok && s.next()) {
        if (s.nt != pend_nt && pend > 0) {
          bar_sync(3, 256);
          if (et == 0) add_release(y_cnt + pend_nt, pend);
          pend = 0;
        }
        const uint32_t slot = p.slots == 2 ? n_seg & 1u : 0u, use = p.slots == 2 ? n_seg >> 1 : n_seg;
        ++n_seg;
        const int j = static_cast<int>(cta - run_owner(s.line * p.Kb2, f.C, f.B));
        ok = bar_all(3, 256, mbar_wait(smem_u32(&s_acc_full[slot]), use & 1u, s_abort, p.wait_ns));
        if (!ok) break;
        tc_fence_after();
        const int u0 = L.off[s.a], n_col = L.off[s.a + 1] - u0, C8 = (n_col + 7) & ~7;
        const uint32_t acc = tmem_base + slot * 128u + lanes + g * (2 * C8);
        const int n = s.nt * 256 + g * 128 + row;
        float* dst = p.y_part + (static_cast<size_t>(j) * P + u0) * p.d + n;
#pragma unroll 1
        for (int c0 = 0; c0 < n_col; c0 += kFewBatch) {
          uint32_t v0[kFewBatch], v1[kFewBatch];
          tmem_ld4(acc + c0, v0);
          tmem_ld4(acc + C8 + c0, v1);
          tmem_wait_ld();
          if (n < p.d) {
#pragma unroll
            for (int i = 0; i < kFewBatch; ++i)
              if (c0 + i < n_col)
                __stcg(dst + static_cast<size_t>(c0 + i) * p.d, __uint_as_float(v0[i]) + __uint_as_float(v1[i]));
          }
        }
        tc_fence_before();
        __syncwarp();
        if (lane == 0) mbar_arrive(smem_u32(&s_acc_empty[slot]));
        pend_nt = s.nt;
        pend += s.kb1 - s.kb0;
      }
    }
    if (pend > 0) {
      bar_sync(3, 256);
      if (et == 0) add_release(y_cnt + pend_nt, pend);
    }
    // ---- weighted sums: the CTAs of a column block share its (token, 4 columns) items --------------------------
    if (A == 0) {
      uint4* out = reinterpret_cast<uint4*>(p.out);
      for (size_t i = static_cast<size_t>(cta) * 256 + et; i < static_cast<size_t>(T) * p.d / 8; i += static_cast<size_t>(C) * 256)
        out[i] = make_uint4(0, 0, 0, 0);
    } else if (ok) {
      const FewPhase &f0 = s_phase[2], &f = s_phase[3].an > 0 ? s_phase[3] : s_phase[2];   // f: the last phase that has work
      const uint32_t per_nt = static_cast<uint32_t>(f.an) * p.Kb2;
      const int nt_lo = static_cast<int>(f.b / per_nt), nt_hi = f.e > f.b ? static_cast<int>((f.e - 1) / per_nt) : nt_lo - 1;
      const size_t part_pitch = static_cast<size_t>(P) * p.d;
      for (int nt0 = nt_lo; nt0 <= nt_hi; nt0 += 2) {               // (almost every CTA has one or two column blocks)
        // What the wait does not need is computed before it: partials per expert, and this CTA's share of each block's
        // (token, 4 columns) items.
        const int two = min(2, nt_hi - nt0 + 1);
        for (int i = et; i < two * A; i += 256) {
          const int m = i >= A ? 1 : 0, a = i - m * A, nt = nt0 + m;
          const FewPhase& h = a < f0.an ? f0 : f;
          const uint32_t b = (static_cast<uint32_t>(nt) * h.an + a - h.a0) * p.Kb2;
          L.split[i] = static_cast<uint8_t>(run_owner(b + p.Kb2 - 1, h.C, h.B) - run_owner(b, h.C, h.B) + 1);
        }
        int from[2], n_item[2];
#pragma unroll
        for (int m = 0; m < 2; ++m) {
          const uint32_t c_lo = run_owner((nt0 + m) * per_nt, f.C, f.B), c_hi = run_owner((nt0 + m + 1) * per_nt - 1, f.C, f.B);
          const uint32_t parts = c_hi - c_lo + 1, me = cta - c_lo;
          from[m] = m < two ? static_cast<int>(run_begin(me, parts, T * 64)) : 0;
          n_item[m] = m < two ? static_cast<int>(run_begin(me + 1, parts, T * 64)) - from[m] : 0;
        }
        bool seen = true;
        if (et < two) seen = few_poll(y_cnt + nt0 + et, A * p.Kb2, s_abort, p.wait_ns);
        ok = bar_all(3, 256, seen);
        if (!ok) break;
        // With few items four lanes share one (lane q takes the token's pairs q, q + 4, ..., then the four sums are added in
        // a fixed tree); two pairs' partials are in flight.
        const int items = n_item[0] + n_item[1];
        const int lanes_per = items * 4 <= 512 ? 4 : 1, q = et & (lanes_per - 1), groups = 256 / lanes_per;
        for (int i0 = 0; i0 < items; i0 += groups) {                // the same number of turns for every lane of a warp
          const int i = i0 + et / lanes_per;
          const int m = i >= n_item[0] ? 1 : 0, it = (m ? i - n_item[0] + from[1] : i + from[0]);
          const int t = it >> 6, col = (nt0 + m) * 256 + (it & 63) * 4;
          const bool on = i < items && col < p.d;
          const uint8_t* split = L.split + m * A;
          const int n_pair = on ? s_local[t] : 0;
          float4 acc = make_float4(0.f, 0.f, 0.f, 0.f);
#pragma unroll 1
          for (int s = q; s < n_pair; s += 2 * lanes_per) {
            float4 v[2][kFewSplit];
            float w[2];
#pragma unroll
            for (int h = 0; h < 2; ++h) {
              const int at = t * k + min(s + h * lanes_per, n_pair - 1);
              const int n = s + h * lanes_per < n_pair ? split[L.pa[at]] : 0;
              w[h] = L.w[at];
              const float* src = p.y_part + static_cast<size_t>(L.pu[at]) * p.d + col;
#pragma unroll
              for (int j = 0; j < kFewSplit; ++j)
                v[h][j] = n > j ? __ldcg(reinterpret_cast<const float4*>(src + j * part_pitch)) : make_float4(0.f, 0.f, 0.f, 0.f);
              if (n == 0) w[h] = 0.f;
            }
#pragma unroll
            for (int h = 0; h < 2; ++h) {
              acc.x = fmaf(w[h], v[h][0].x + v[h][1].x + v[h][2].x + v[h][3].x, acc.x);
              acc.y = fmaf(w[h], v[h][0].y + v[h][1].y + v[h][2].y + v[h][3].y, acc.y);
              acc.z = fmaf(w[h], v[h][0].z + v[h][1].z + v[h][2].z + v[h][3].z, acc.z);
              acc.w = fmaf(w[h], v[h][0].w + v[h][1].w + v[h][2].w + v[h][3].w, acc.w);
            }
          }
          for (int o = 1; o < lanes_per; o <<= 1) {
            acc.x += __shfl_xor_sync(0xffffffffu, acc.x, o);
            acc.y += __shfl_xor_sync(0xffffffffu, acc.y, o);
            acc.z += __shfl_xor_sync(0xffffffffu, acc.z, o);
            acc.w += __shfl_xor_sync(0xffffffffu, acc.w, o);
          }
          if (on && q == 0) {
            const __nv_bfloat162 lo = __floats2bfloat162_rn(acc.x, acc.y), hi = __floats2bfloat162_rn(acc.z, acc.w);
            *reinterpret_cast<uint2*>(p.out + static_cast<size_t>(t) * p.d + col) =
                make_uint2(*reinterpret_cast<const uint32_t*>(&lo), *reinterpret_cast<const uint32_t*>(&hi));
          }
        }
        if (nt0 + 2 <= nt_hi) bar_sync(3, 256);                     // before the table is written again
      }
    }
  }

  __syncwarp();
  tc_fence_before();
  __syncthreads();
  if (tid == 0) atomicInc(p.leave, 2 * C - 1);
  if (*s_abort) {
    if (tid == 0) atomicOr(p.status, static_cast<uint32_t>(TEMPO_STATUS_TIMEOUT));
    for (int i = 0; i < 50; ++i) __nanosleep(1000);      // let copies and MMAs in flight drain
  }
  if (warp == 1) {
    tc_fence_after();
    __syncwarp();
    asm volatile("tcgen05.dealloc.cta_group::1.sync.aligned.b32 %0, %1;" ::"r"(tmem_base), "r"(kTmemCols) : "memory");
  }
}

// ---- host ---------------------------------------------------------------------------------------------
static size_t align256(size_t v) { return (v + 255) & ~static_cast<size_t>(255); }

FewLayout few_layout(int T, int k, int G, int d, int f, int num_sms) {
  FewLayout L;
  const size_t P = static_cast<size_t>(T) * k, A = P < static_cast<size_t>(G) ? P : static_cast<size_t>(G);
  const int NT2 = (d + 255) / 256;
  // the widest of both weight types: rows of 128 bytes per K-block of 64 (bf16) or 128 (fp8) values
  const size_t T16 = (static_cast<size_t>(T) + 15) / 16 * 16;
  L.counter_ints = 96 + NT2 + 2 * num_sms;
  L.off_leave = 0;
  L.off_counters = 256;
  L.off_x = align256(L.off_counters + 2 * sizeof(int32_t) * static_cast<size_t>(L.counter_ints));
  L.off_h = align256(L.off_x + static_cast<size_t>(d / 64) * T16 * 128 + static_cast<size_t>(d / 128) * 512);
  const size_t h_rows = 2 * (P + 7 * A);                 // every expert's columns rounded up to 8, two terms
  L.off_gu = align256(L.off_h + static_cast<size_t>(f / 64) * (h_rows * 128 + 512 * A));
  L.off_y = align256(L.off_gu + static_cast<size_t>(num_sms) * 2 * T * 256 * 4);
  L.total = align256(L.off_y + static_cast<size_t>(kFewSplit) * P * d * 4);
  return L;
}

template <bool kBf16>
static cudaError_t launch_few_t(FewParams p, int num_sms, cudaStream_t stream) {
  static std::atomic<unsigned long long> smem_set{0};
  const int T8 = (p.T + 7) & ~7, T16 = (p.T + 15) & ~15;
  // columns: gate/up R1 (all tokens), down twice the tokens of an expert rounded up to 8
  const int rows = kBf16 ? max(T16, 2 * T8) : 2 * T8;
  p.stage_bytes = (kBBytes + kSfbBytes + rows * 128 + 512 + 1023) / 1024 * 1024;
  p.slots = rows <= 64 ? 2 : 1;
  const size_t lists = few_list_bytes(p.G, p.T * p.k, p.E);
  p.stages = min(kFewRing, static_cast<int>((kFewBudget - 1024 - lists) / p.stage_bytes));
  const size_t smem = 1024 + static_cast<size_t>(p.stages) * p.stage_bytes + lists;
  cudaError_t e = smem_limit_once(few_kernel<kBf16>, kFewBudget, smem_set);
  if (e != cudaSuccess) return e;
  return launch_pdl(few_kernel<kBf16>, dim3(num_sms), dim3(kFewThreads), smem, stream, p);
}

cudaError_t launch_few(const FewParams& p, bool bf16, int num_sms, cudaStream_t stream) {
  return bf16 ? launch_few_t<true>(p, num_sms, stream) : launch_few_t<false>(p, num_sms, stream);
}

}  // namespace tempo
