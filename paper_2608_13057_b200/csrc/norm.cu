// The norms around a block.  A row of the residual stream is held in a CTA's registers from its first load to its last store
// (one row per CTA, or several one after the other with the next in flight), so every operand is read once and every result
// written once:
//   tempo_norm_in    x  = norm(r) * w + b
//   tempo_norm_out   r' = r_scale * r + y_scale * g (.) (norm(y) * post_w + post_b),  x' = norm(r') * next_w + next_b
// norm(v) = v / sqrt(mean(v^2) + eps), or the same of v - mean(v).  The mean and the mean square are two sums over
// the row, each a shuffle tree in a warp and a fixed-order sum over the warps (32-bit, the same bits every time); the
// centred square sum is taken after the mean from the registers, not as a difference of two large sums.
// x' is taken from the 32-bit r', not from its rounding to the stream's type.
// Bound by the bytes: 8192 x 7168 with a gate per channel reads y and r and writes r' and x', 470 MB, in 79.7 us, 90 % of a
// copy's rate in long runs (two copies of the same bytes take 78.3 us); one row is the latency of a launch and a load, 2.4 us.
// Rows of bf16 at odd addresses go through shared memory on their way in and out, and that staging is what bounds them (49
// instructions a column and thread, 60 % of the issue slots, four to six barriers a row): 4096 x 5001 in 50 us of 25.  Short rows
// in batches are bound by what each row's CTA of one or two warps does before and behind its loads: 8192 x 512 in 7.9 us of 5.1.
// Which kernel a shape gets, and the figures behind that, stand at the launcher below.
#include "tempo_kernels.cuh"

namespace tempo {

// Loads of VEC elements into floats; the streams are read once, so they do not stay in L1 beside the weights.
template <int VEC>
__device__ __forceinline__ void load_bf16_stream(const __nv_bfloat16* p, uint32_t (&u)[(VEC + 1) / 2]) {
  if constexpr (VEC == 8) {
    asm volatile("ld.global.L1::no_allocate.v4.b32 {%0, %1, %2, %3}, [%4];"
                 : "=r"(u[0]), "=r"(u[1]), "=r"(u[2]), "=r"(u[3]) : "l"(p));
  } else if constexpr (VEC == 4) {
    asm volatile("ld.global.L1::no_allocate.v2.b32 {%0, %1}, [%2];" : "=r"(u[0]), "=r"(u[1]) : "l"(p));
  } else if constexpr (VEC == 2) {
    asm volatile("ld.global.L1::no_allocate.b32 %0, [%1];" : "=r"(u[0]) : "l"(p));
  } else {
    u[0] = *reinterpret_cast<const uint16_t*>(p);
  }
}

// The first n bytes of 16, the rest zero.
__device__ __forceinline__ void copy16_part(void* dst, const void* src, uint32_t n) {
  asm volatile("cp.async.cg.shared.global [%0], [%1], 16, %2;" ::"r"(smem_u32(dst)), "l"(src), "r"(n) : "memory");
}
__device__ __forceinline__ void copy16(void* dst, const void* src) {
  asm volatile("cp.async.cg.shared.global [%0], [%1], 16;" ::"r"(smem_u32(dst)), "l"(src) : "memory");
}

template <int VEC>
__device__ __forceinline__ void widen(const uint32_t (&u)[(VEC + 1) / 2], float (&v)[VEC]) {
#pragma unroll
  for (int i = 0; i < VEC; ++i)
    v[i] = __uint_as_float((i & 1) ? (u[i / 2] & 0xffff0000u) : (u[i / 2] << 16));
}

template <int VEC>
__device__ __forceinline__ void load_f32(const float* p, float (&v)[VEC]) {
  if constexpr (VEC >= 4) {
#pragma unroll
    for (int i = 0; i < VEC; i += 4) {
      const float4 q = __ldg(reinterpret_cast<const float4*>(p + i));
      v[i] = q.x; v[i + 1] = q.y; v[i + 2] = q.z; v[i + 3] = q.w;
    }
  } else if constexpr (VEC == 2) {
    const float2 q = __ldg(reinterpret_cast<const float2*>(p));
    v[0] = q.x; v[1] = q.y;
  } else {
    v[0] = __ldg(p);
  }
}

template <int VEC>
__device__ __forceinline__ void load_f32_stream(const float* p, float (&v)[VEC]) {
  if constexpr (VEC >= 4) {
#pragma unroll
    for (int i = 0; i < VEC; i += 4)
      asm volatile("ld.global.L1::no_allocate.v4.f32 {%0, %1, %2, %3}, [%4];"
                   : "=f"(v[i]), "=f"(v[i + 1]), "=f"(v[i + 2]), "=f"(v[i + 3]) : "l"(p + i));
  } else if constexpr (VEC == 2) {
    asm volatile("ld.global.L1::no_allocate.v2.f32 {%0, %1}, [%2];" : "=f"(v[0]), "=f"(v[1]) : "l"(p));
  } else {
    v[0] = *p;
  }
}

// Weights, biases, gates: bf16 or f32 (the same for the whole launch), kept in L1 across the rows of an SM.
template <int VEC>
__device__ __forceinline__ void load_param(const void* base, size_t at, int is_f32, float (&v)[VEC]) {
  if (is_f32) {
    load_f32<VEC>(static_cast<const float*>(base) + at, v);
  } else {
    const __nv_bfloat16* p = static_cast<const __nv_bfloat16*>(base) + at;
    uint32_t u[(VEC + 1) / 2];
    if constexpr (VEC == 8) {
      const uint4 q = __ldg(reinterpret_cast<const uint4*>(p));
      u[0] = q.x; u[1] = q.y; u[2] = q.z; u[3] = q.w;
    } else if constexpr (VEC == 4) {
      const uint2 q = __ldg(reinterpret_cast<const uint2*>(p));
      u[0] = q.x; u[1] = q.y;
    } else if constexpr (VEC == 2) {
      u[0] = __ldg(reinterpret_cast<const uint32_t*>(p));
    } else {
      u[0] = __ldg(reinterpret_cast<const uint16_t*>(p));
    }
    widen<VEC>(u, v);
  }
}

template <int VEC>
__device__ __forceinline__ void store_bf16(__nv_bfloat16* p, const float (&v)[VEC]) {
  if constexpr (VEC == 1) {
    *p = __float2bfloat16_rn(v[0]);
  } else {
    uint32_t u[VEC / 2];
#pragma unroll
    for (int i = 0; i < VEC / 2; ++i) {
      const __nv_bfloat162 b = __floats2bfloat162_rn(v[2 * i], v[2 * i + 1]);
      u[i] = *reinterpret_cast<const uint32_t*>(&b);
    }
    if constexpr (VEC == 8) __stcs(reinterpret_cast<uint4*>(p), make_uint4(u[0], u[1], u[2], u[3]));
    else if constexpr (VEC == 4) __stcs(reinterpret_cast<uint2*>(p), make_uint2(u[0], u[1]));
    else __stcs(reinterpret_cast<uint32_t*>(p), u[0]);
  }
}

template <int VEC>
__device__ __forceinline__ void store_f32(float* p, const float (&v)[VEC]) {
  if constexpr (VEC >= 4) {
#pragma unroll
    for (int i = 0; i < VEC; i += 4) __stcs(reinterpret_cast<float4*>(p + i), make_float4(v[i], v[i + 1], v[i + 2], v[i + 3]));
  } else if constexpr (VEC == 2) {
    __stcs(reinterpret_cast<float2*>(p), make_float2(v[0], v[1]));
  } else {
    *p = v[0];
  }
}

// Sum over the CTA, the same bits in every thread.  `slot` alternates, so one barrier per sum is enough: a warp can only
// overwrite a slot's words after the barrier of the sum in between, which every reader of those words has passed.
__device__ __forceinline__ float cta_sum(float v, float (&s_part)[2][32], int slot, int warps) {
#pragma unroll
  for (int o = 16; o > 0; o >>= 1) v += __shfl_xor_sync(0xffffffffu, v, o);
  if (warps == 1) return v;
  if ((threadIdx.x & 31) == 0) s_part[slot][threadIdx.x >> 5] = v;
  __syncthreads();
  float t = (threadIdx.x & 31) < warps ? s_part[slot][threadIdx.x & 31] : 0.f;
#pragma unroll
  for (int o = 16; o > 0; o >>= 1) t += __shfl_xor_sync(0xffffffffu, t, o);
  return t;
}

// Two 32-bit operations per instruction: with bf16 operands a row costs more instructions than bytes, so the arithmetic is
// done on pairs (the issue slots, not HBM, bounded the scalar form: 35 instructions an element, 0.65 issued per clock).
__device__ __forceinline__ float2 mul2(float2 a, float2 b) {
  float2 r;
  asm("{\n\t.reg .b64 a, b, r;\n\tmov.b64 a, {%2, %3};\n\tmov.b64 b, {%4, %5};\n\tmul.rn.f32x2 r, a, b;\n\tmov.b64 {%0, %1}, r;\n\t}"
      : "=f"(r.x), "=f"(r.y) : "f"(a.x), "f"(a.y), "f"(b.x), "f"(b.y));
  return r;
}
__device__ __forceinline__ float2 add2(float2 a, float2 b) {
  float2 r;
  asm("{\n\t.reg .b64 a, b, r;\n\tmov.b64 a, {%2, %3};\n\tmov.b64 b, {%4, %5};\n\tadd.rn.f32x2 r, a, b;\n\tmov.b64 {%0, %1}, r;\n\t}"
      : "=f"(r.x), "=f"(r.y) : "f"(a.x), "f"(a.y), "f"(b.x), "f"(b.y));
  return r;
}
__device__ __forceinline__ float2 fma2(float2 a, float2 b, float2 c) {
  float2 r;
  asm("{\n\t.reg .b64 a, b, c, r;\n\tmov.b64 a, {%2, %3};\n\tmov.b64 b, {%4, %5};\n\tmov.b64 c, {%6, %7};\n\t"
      "fma.rn.f32x2 r, a, b, c;\n\tmov.b64 {%0, %1}, r;\n\t}"
      : "=f"(r.x), "=f"(r.y) : "f"(a.x), "f"(a.y), "f"(b.x), "f"(b.y), "f"(c.x), "f"(c.y));
  return r;
}
// A thread's values of a row: CH chunks of VEC neighbours, as pairs.  kSplit (rows that no vector divides or aligns, where they do
// not go through shared memory): a
// chunk is two single elements, blockDim.x columns apart, so that a warp still reads neighbours; the second may lie beyond the
// row when the first does not.
template <int VEC, int CH>
struct RowVals { float2 v[CH][VEC / 2]; };
template <int CH>
struct Cols {
  int col[CH];
  bool on[CH], on2[CH];      // first, second element of a split chunk inside the row
  int n[CH];                 // elements of a chunk inside the row (at most VEC)
  int nt;                    // distance of a split chunk's elements
};
template <int VEC, int CH, bool kSplit, bool kFull>
__device__ __forceinline__ void set_cols(Cols<CH>& k, int d) {
  k.nt = static_cast<int>(blockDim.x);
#pragma unroll
  for (int c = 0; c < CH; ++c) {
    k.col[c] = kSplit ? 2 * c * k.nt + static_cast<int>(threadIdx.x) : (c * k.nt + static_cast<int>(threadIdx.x)) * VEC;
    k.on[c] = kFull || k.col[c] < d;
    k.on2[c] = kSplit ? k.col[c] + k.nt < d : k.on[c];
    k.n[c] = max(0, min(VEC, d - k.col[c]));
  }
}
template <int VEC>
__device__ __forceinline__ void to_pairs(const float (&f)[VEC], float2 (&v)[VEC / 2]) {
#pragma unroll
  for (int i = 0; i < VEC / 2; ++i) v[i] = make_float2(f[2 * i], f[2 * i + 1]);
}
template <int VEC, bool kSplit>
__device__ __forceinline__ void load_bf16_chunk(const __nv_bfloat16* p, uint32_t (&u)[VEC / 2], int nt, bool on2) {
  if constexpr (kSplit) {
    const uint16_t* q = reinterpret_cast<const uint16_t*>(p);
    u[0] = q[0] | (on2 ? static_cast<uint32_t>(q[nt]) << 16 : 0u);
  } else {
    load_bf16_stream<VEC>(p, u);
  }
}
template <int VEC, bool kSplit>
__device__ __forceinline__ void load_f32_chunk(const float* p, float (&f)[VEC], int nt, bool on2) {
  if constexpr (kSplit) {
    f[0] = p[0];
    f[1] = on2 ? p[nt] : 0.f;
  } else {
    load_f32_stream<VEC>(p, f);
  }
}
template <int VEC, bool kSplit>
__device__ __forceinline__ void store_bf16_chunk(__nv_bfloat16* p, const float2 (&v)[VEC / 2], int nt, bool on2) {
  if constexpr (kSplit) {
    p[0] = __float2bfloat16_rn(v[0].x);
    if (on2) p[nt] = __float2bfloat16_rn(v[0].y);
  } else {
    float f[VEC];
#pragma unroll
    for (int i = 0; i < VEC / 2; ++i) { f[2 * i] = v[i].x; f[2 * i + 1] = v[i].y; }
    store_bf16<VEC>(p, f);
  }
}
template <int VEC, bool kSplit>
__device__ __forceinline__ void store_f32_chunk(float* p, const float2 (&v)[VEC / 2], int nt, bool on2) {
  if constexpr (kSplit) {
    p[0] = v[0].x;
    if (on2) p[nt] = v[0].y;
  } else {
    float f[VEC];
#pragma unroll
    for (int i = 0; i < VEC / 2; ++i) { f[2 * i] = v[i].x; f[2 * i + 1] = v[i].y; }
    store_f32<VEC>(p, f);
  }
}

// ---- rows at any alignment (kShift) ---------------------------------------------------------------
// A row that starts h elements (0 to 7) past a 16-byte boundary: its granule g (16 aligned bytes) holds the columns 8 g - h to
// 8 g - h + 7, so a thread's eight columns lie in two granules, and a granule's in the columns of two threads.
__device__ __forceinline__ int row_shift(const __nv_bfloat16* row) { return static_cast<int>(reinterpret_cast<uintptr_t>(row) >> 1) & 7; }

// u[c] = eight elements from element `off` (0 to 7, the same for the CTA) of the 16-byte words first + c * nt and the next one
// on; a word before `base` is not needed and not read.
template <int CH, int K>
__device__ __forceinline__ void windows_at(const uint4* base, const uint4* first, int nt, uint32_t sh, uint32_t (&u)[CH][4]) {
#pragma unroll
  for (int c = 0; c < CH; ++c) {
    const uint4* q = first + c * nt;
    const uint4 lo = *(c == 0 && q < base ? base : q), hi = q[1];
    const uint32_t w[8] = {lo.x, lo.y, lo.z, lo.w, hi.x, hi.y, hi.z, hi.w};
#pragma unroll
    for (int i = 0; i < 4; ++i) u[c][i] = __funnelshift_r(w[K + i], w[K + i + 1], sh);
  }
}
template <int CH>
__device__ __forceinline__ void windows(const uint4* base, int first, int nt, int off, uint32_t (&u)[CH][4]) {
  const uint4* q = base + first;
  const uint32_t sh = (off & 1) * 16;
  switch (off >> 1) {
    case 0:
      if (off == 0) {
#pragma unroll
        for (int c = 0; c < CH; ++c) {
          const uint4 w = q[c * nt];
          u[c][0] = w.x; u[c][1] = w.y; u[c][2] = w.z; u[c][3] = w.w;
        }
      } else {
        windows_at<CH, 0>(base, q, nt, sh, u);
      }
      break;
    case 1: windows_at<CH, 1>(base, q, nt, sh, u); break;
    case 2: windows_at<CH, 2>(base, q, nt, sh, u); break;
    default: windows_at<CH, 3>(base, q, nt, sh, u);
  }
}
// A thread's columns of a row whose granules are in shared memory, zero beyond the row.
template <int CH>
__device__ __forceinline__ void load_shifted(const uint4* granules, int h, const Cols<CH>& k, uint32_t (&u)[CH][4]) {
  windows<CH>(granules, threadIdx.x, k.nt, h, u);
#pragma unroll
  for (int c = 0; c < CH; ++c)
    if (k.n[c] < 8) {
#pragma unroll
      for (int i = 0; i < 4; ++i) u[c][i] = 2 * i + 1 < k.n[c] ? u[c][i] : 2 * i < k.n[c] ? u[c][i] & 0xffffu : 0u;
    }
}
// A thread's columns to shared memory, rounded, where store_shifted takes them from.
template <int CH>
__device__ __forceinline__ void stage_row(uint4* stage, const Cols<CH>& k, const RowVals<8, CH>& a) {
#pragma unroll
  for (int c = 0; c < CH; ++c) {
    uint32_t u[4];
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      const __nv_bfloat162 b = __floats2bfloat162_rn(a.v[c][i].x, a.v[c][i].y);
      u[i] = *reinterpret_cast<const uint32_t*>(&b);
    }
    stage[c * k.nt + threadIdx.x] = make_uint4(u[0], u[1], u[2], u[3]);
  }
}
// Writes a staged row (after a barrier): whole granules, and the row's two edges by element.
template <int CH>
__device__ __forceinline__ void store_shifted(__nv_bfloat16* row, const uint4* stage, const Cols<CH>& k, int d) {
  const int h = row_shift(row), tid = threadIdx.x;
  uint32_t u[CH][4];
  windows<CH>(stage, tid - (h > 0), k.nt, (8 - h) & 7, u);
#pragma unroll
  for (int c = 0; c < CH; ++c) {
    const int a = k.col[c] - h;                         // the granule's first column
    if (a >= 0 && a + 8 <= d) {
      __stcs(reinterpret_cast<uint4*>(row + a), make_uint4(u[c][0], u[c][1], u[c][2], u[c][3]));
    } else if (a < d) {
      uint16_t* q = reinterpret_cast<uint16_t*>(row) + a;
#pragma unroll
      for (int i = 0; i < 8; ++i)
        if (a + i >= 0 && a + i < d) q[i] = static_cast<uint16_t>(u[c][i / 2] >> (16 * (i & 1)));
    }
  }
  if (tid < h) {                                        // the granule behind the last thread's
    const int col = 8 * CH * k.nt - h + tid;
    if (col < d) reinterpret_cast<uint16_t*>(row)[col] = reinterpret_cast<const uint16_t*>(stage)[col];
  }
}
// Eight neighbours of a parameter, n of them inside the row; `vec`: they can be read in 16-byte loads.
__device__ __forceinline__ void load_param_part(const void* base, size_t at, int is_f32, bool vec, int n, float (&v)[8]) {
  if (vec && n == 8) {
    load_param<8>(base, at, is_f32, v);
  } else {
#pragma unroll
    for (int i = 0; i < 8; ++i) {
      float f[1] = {0.f};
      if (i < n) load_param<1>(base, at + i, is_f32, f);
      v[i] = f[0];
    }
  }
}

// v -> normed in place, without weights and without the final factor, which is returned: 1 / sqrt(mean square + eps).
// Values beyond the row are zero and stay so; kFull: there are none.
template <int VEC, int CH, bool kSplit, bool kFull, bool kShift>
__device__ __forceinline__ float norm_row(RowVals<VEC, CH>& a, const Cols<CH>& k, int layer, float inv_d, float eps,
                                          float (&s_part)[2][32], int& slot) {
  const int warps = k.nt >> 5;
  if (layer) {
    float2 s = make_float2(0.f, 0.f);
#pragma unroll
    for (int c = 0; c < CH; ++c)
#pragma unroll
      for (int i = 0; i < VEC / 2; ++i) s = add2(s, a.v[c][i]);
    const float mean = cta_sum(s.x + s.y, s_part, slot, warps) * inv_d;
    slot ^= 1;
#pragma unroll
    for (int c = 0; c < CH; ++c)
      if (kFull || k.on[c]) {
        const float2 m = make_float2(-mean, !kSplit || k.on2[c] ? -mean : 0.f);
#pragma unroll
        for (int i = 0; i < VEC / 2; ++i) a.v[c][i] = add2(a.v[c][i], m);
        if (kShift && k.n[c] < VEC) {
#pragma unroll
          for (int i = 0; i < VEC / 2; ++i) {
            if (2 * i >= k.n[c]) a.v[c][i].x = 0.f;
            if (2 * i + 1 >= k.n[c]) a.v[c][i].y = 0.f;
          }
        }
      }
  }
  float2 q = make_float2(0.f, 0.f);
#pragma unroll
  for (int c = 0; c < CH; ++c)
#pragma unroll
    for (int i = 0; i < VEC / 2; ++i) q = fma2(a.v[c][i], a.v[c][i], q);
  const float ms = cta_sum(q.x + q.y, s_part, slot, warps) * inv_d;
  slot ^= 1;
  return 1.f / sqrtf(ms + eps);
}

// v *= the parameter, or += it.
template <int VEC, int CH, bool kSplit, bool kFull, bool kShift, bool kAdd>
__device__ __forceinline__ void apply_param(RowVals<VEC, CH>& a, const void* base, size_t at, int is_f32, const Cols<CH>& k,
                                            [[maybe_unused]] bool vec) {
#pragma unroll
  for (int c = 0; c < CH; ++c) {
    if (!kFull && !k.on[c]) continue;
    float f[VEC];
    float2 w[VEC / 2];
    if constexpr (kSplit) {
      float f0[1], f1[1] = {0.f};
      load_param<1>(base, at + k.col[c], is_f32, f0);
      if (k.on2[c]) load_param<1>(base, at + k.col[c] + k.nt, is_f32, f1);
      f[0] = f0[0];
      f[1] = f1[0];
    } else if constexpr (kShift) {
      load_param_part(base, at + k.col[c], is_f32, vec, k.n[c], f);
    } else {
      load_param<VEC>(base, at + k.col[c], is_f32, f);
    }
    to_pairs<VEC>(f, w);
#pragma unroll
    for (int i = 0; i < VEC / 2; ++i) a.v[c][i] = kAdd ? add2(a.v[c][i], w[i]) : mul2(a.v[c][i], w[i]);
  }
}
template <int VEC, int CH, bool kFull>
__device__ __forceinline__ void apply_fold(RowVals<VEC, CH>& a, const float4* fold, const Cols<CH>& k) {
  static_assert(VEC == 2 || VEC == 4 || VEC == 8, "");
#pragma unroll
  for (int c = 0; c < CH; ++c) {
    if (!kFull && !k.on[c]) continue;
#pragma unroll
    for (int h = 0; h < VEC / 4; ++h) {
      const float4 w = fold[(2 * c + h) * k.nt];
      a.v[c][2 * h] = mul2(a.v[c][2 * h], make_float2(w.x, w.y));
      a.v[c][2 * h + 1] = mul2(a.v[c][2 * h + 1], make_float2(w.z, w.w));
    }
  }
}
template <int VEC, int CH>
__device__ __forceinline__ void scale_row(RowVals<VEC, CH>& a, float f) {
#pragma unroll
  for (int c = 0; c < CH; ++c)
#pragma unroll
    for (int i = 0; i < VEC / 2; ++i) a.v[c][i] = mul2(a.v[c][i], make_float2(f, f));
}

// Everything between a row's loads and its stores.  yu: the block's output (kOut); ru or r: the stream; zero beyond the row.
// kFold: the parameter that follows the first norm, the same for every row, comes from `fold` in 32 bits (this thread's words:
// [chunk][pair of float4][thread]): post_w, times a gate per channel, or next_w in the norm before a block.
template <int VEC, int CH, bool kSplit, bool kF32, bool kOut, bool kFull, bool kFold = false, bool kShift = false>
__device__ __forceinline__ void finish_row(const NormParams& p, size_t row, const Cols<CH>& k, const uint32_t (&yu)[CH][VEC / 2],
                                           const uint32_t (&ru)[CH][VEC / 2], RowVals<VEC, CH>& r, float (&s_part)[2][32], int& slot,
                                           const float4* fold = nullptr, [[maybe_unused]] uint4* stage_r = nullptr,
                                           [[maybe_unused]] uint4* stage_x = nullptr) {
  const float inv_d = 1.f / static_cast<float>(p.d);
  RowVals<VEC, CH> a;
  float f[VEC];
  if constexpr (kOut) {
    float ys = p.y_scale;
#pragma unroll
    for (int c = 0; c < CH; ++c) {
      widen<VEC>(yu[c], f);
      to_pairs<VEC>(f, a.v[c]);
    }
    if constexpr (kFold) {
      ys *= norm_row<VEC, CH, kSplit, kFull, kShift>(a, k, p.layer, inv_d, p.eps, s_part, slot);
      apply_fold<VEC, CH, kFull>(a, fold, k);
    } else if (p.post_w != nullptr) {
      const float inv = norm_row<VEC, CH, kSplit, kFull, kShift>(a, k, p.layer, inv_d, p.eps, s_part, slot);
      apply_param<VEC, CH, kSplit, kFull, kShift, false>(a, p.post_w, 0, p.param_f32, k, p.param_vec);
      if (p.post_b != nullptr) {
        scale_row<VEC, CH>(a, inv);
        apply_param<VEC, CH, kSplit, kFull, kShift, true>(a, p.post_b, 0, p.param_f32, k, p.param_vec);
      } else {
        ys *= inv;
      }
    }
    if (p.gate != nullptr) {
      if (p.gate_col == 0) {                            // one gate for the row
        float g1[1];
        load_param<1>(p.gate, row * p.gate_row, p.gate_f32, g1);
        ys *= g1[0];
      } else if (kFold) {                               // in the folded parameter
      } else if (p.gate_vec) {
        apply_param<VEC, CH, kSplit, kFull, kShift, false>(a, p.gate, row * p.gate_row, p.gate_f32, k, true);
      } else {                                          // columns at a pitch of their own
#pragma unroll
        for (int c = 0; c < CH; ++c) {
          if (!kFull && !k.on[c]) continue;
#pragma unroll
          for (int i = 0; i < VEC; ++i) {
            if ((kSplit && i == 1 && !k.on2[c]) || (kShift && i >= k.n[c])) continue;
            float g1[1];
            load_param<1>(p.gate, row * p.gate_row + static_cast<size_t>(k.col[c] + (kSplit ? i * k.nt : i)) * p.gate_col, p.gate_f32, g1);
            (i & 1 ? a.v[c][i / 2].y : a.v[c][i / 2].x) *= g1[0];
          }
        }
      }
    }
#pragma unroll
    for (int c = 0; c < CH; ++c) {
      if constexpr (!kF32) {
        widen<VEC>(ru[c], f);
        to_pairs<VEC>(f, r.v[c]);
      }
#pragma unroll
      for (int i = 0; i < VEC / 2; ++i)
        a.v[c][i] = fma2(a.v[c][i], make_float2(ys, ys), mul2(r.v[c][i], make_float2(p.r_scale, p.r_scale)));
      if (!kShift && (kFull || k.on[c])) {
        if constexpr (kF32) store_f32_chunk<VEC, kSplit>(static_cast<float*>(p.r_out) + row * p.ld_r_out + k.col[c], a.v[c], k.nt, k.on2[c]);
        else store_bf16_chunk<VEC, kSplit>(static_cast<__nv_bfloat16*>(p.r_out) + row * p.ld_r_out + k.col[c], a.v[c], k.nt, k.on2[c]);
      }
    }
    if constexpr (kShift) {
      if (p.post_w == nullptr || k.nt == 32) __syncthreads();   // every thread has read y: its words take r'
      stage_row<CH>(stage_r, k, a);
      if (p.x == nullptr || k.nt == 32) __syncthreads();
      if (p.x == nullptr) store_shifted<CH>(static_cast<__nv_bfloat16*>(p.r_out) + row * p.ld_r_out, stage_r, k, p.d);
    }
    if (p.x == nullptr) return;
  } else {
#pragma unroll
    for (int c = 0; c < CH; ++c) {
      if constexpr (kF32) {
#pragma unroll
        for (int i = 0; i < VEC / 2; ++i) a.v[c][i] = r.v[c][i];
      } else {
        widen<VEC>(ru[c], f);
        to_pairs<VEC>(f, a.v[c]);
      }
    }
  }
  const float inv = norm_row<VEC, CH, kSplit, kFull, kShift>(a, k, p.layer, inv_d, p.eps, s_part, slot);
  // a barrier (in the sum) lies behind: r' is staged, and every thread has read r
  if constexpr (kShift && kOut) store_shifted<CH>(static_cast<__nv_bfloat16*>(p.r_out) + row * p.ld_r_out, stage_r, k, p.d);
  if constexpr (kFold && !kOut) apply_fold<VEC, CH, kFull>(a, fold, k);
  else apply_param<VEC, CH, kSplit, kFull, kShift, false>(a, p.next_w, 0, p.param_f32, k, p.param_vec);
  scale_row<VEC, CH>(a, inv);
  if (p.next_b != nullptr) apply_param<VEC, CH, kSplit, kFull, kShift, true>(a, p.next_b, 0, p.param_f32, k, p.param_vec);
  if constexpr (kShift) {
    if (k.nt == 32) __syncwarp();
    stage_row<CH>(stage_x, k, a);
    __syncthreads();
    store_shifted<CH>(p.x + row * p.ld_x, stage_x, k, p.d);
  } else {
#pragma unroll
    for (int c = 0; c < CH; ++c)
      if (kFull || k.on[c]) store_bf16_chunk<VEC, kSplit>(p.x + row * p.ld_x + k.col[c], a.v[c], k.nt, k.on2[c]);
  }
}

// One row per CTA.  kOut: the norm after a block (p.y), else the norm before one.  kF32: the residual stream is f32.
template <int VEC, int CH, bool kSplit, bool kF32, bool kOut, bool kFull>
__global__ void __launch_bounds__(VEC * CH >= 32 ? 512 : 1024) norm_kernel(const NormParams p) {
  __shared__ float s_part[2][32];
  const int t = blockIdx.x;
  pdl_trigger();
  pdl_wait();
  if (p.n_valid != nullptr && t >= *p.n_valid) return;
  Cols<CH> k;
  set_cols<VEC, CH, kSplit, kFull>(k, p.d);
  const size_t row = static_cast<size_t>(t);
  uint32_t yu[CH][VEC / 2], ru[CH][VEC / 2];
  RowVals<VEC, CH> r;
#pragma unroll
  for (int c = 0; c < CH; ++c) {
    float rf[VEC];
#pragma unroll
    for (int i = 0; i < VEC; ++i) rf[i] = 0.f;
#pragma unroll
    for (int i = 0; i < VEC / 2; ++i) yu[c][i] = ru[c][i] = 0u;
    if (kFull || k.on[c]) {
      if constexpr (kOut) load_bf16_chunk<VEC, kSplit>(p.y + row * p.ld_y + k.col[c], yu[c], k.nt, k.on2[c]);
      if constexpr (kF32) load_f32_chunk<VEC, kSplit>(static_cast<const float*>(p.r) + row * p.ld_r + k.col[c], rf, k.nt, k.on2[c]);
      else load_bf16_chunk<VEC, kSplit>(static_cast<const __nv_bfloat16*>(p.r) + row * p.ld_r + k.col[c], ru[c], k.nt, k.on2[c]);
    }
    if constexpr (kF32) to_pairs<VEC>(rf, r.v[c]);
  }
  int slot = 0;
  finish_row<VEC, CH, kSplit, kF32, kOut, kFull>(p, row, k, yu, ru, r, s_part, slot);
}

// Several rows per CTA (bf16 stream, VEC = 8): the next row is on its way while this one is summed and written.  Every
// thread copies its own columns of the next row to its own words of shared memory (cp.async, 16 bytes each) and reads only
// those back, so the copies need no barrier; two buffers.  64 registers: two CTAs of 448 threads to an SM at d = 7168, where
// the compiler's own choice leaves one.
// kFold: the parameter after the first norm (see finish_row) is kept in shared memory in 32 bits, each thread its own columns:
// fewer loads and conversions per row (8192 rows of 7168 with an f32 gate per channel: 79 us against 87; 4096 of 4096: 23
// against 29).
template <int CH, bool kOut, bool kFull, bool kFold>
__global__ void __maxnreg__(64) norm_rows_kernel(const NormParams p) {
  extern __shared__ uint4 s_row[];                      // [buffer][y, r][chunk][thread], then the folded parameters
  __shared__ float s_part[2][32];
  constexpr int VEC = 8, kR = kOut ? 1 : 0, kStreams = kR + 1;
  pdl_trigger();
  pdl_wait();
  int rows = p.T;
  if (p.n_valid != nullptr) rows = max(0, min(*p.n_valid, p.T));
  Cols<CH> k;
  set_cols<VEC, CH, false, kFull>(k, p.d);
  const int nt = k.nt, tid = threadIdx.x;
  auto fetch = [&](int t, int buf) {
    if (t < rows) {
      const size_t row = static_cast<size_t>(t);
#pragma unroll
      for (int c = 0; c < CH; ++c) {
        if (!kFull && !k.on[c]) continue;
        uint4* dst = s_row + (buf * kStreams * CH + c) * nt + tid;
        if constexpr (kOut) copy16(dst, p.y + row * p.ld_y + k.col[c]);
        copy16(dst + kR * CH * nt, static_cast<const __nv_bfloat16*>(p.r) + row * p.ld_r + k.col[c]);
      }
    }
    asm volatile("cp.async.commit_group;" ::: "memory");
  };
  int slot = 0, buf = 0;
  fetch(blockIdx.x, 0);
  float4* fold = reinterpret_cast<float4*>(s_row + 2 * kStreams * CH * nt) + tid;
  if constexpr (kFold) {
#pragma unroll
    for (int c = 0; c < CH; ++c) {
      if (!kFull && !k.on[c]) continue;
      float w[VEC], g[VEC];
      load_param<VEC>(kOut ? p.post_w : p.next_w, k.col[c], p.param_f32, w);
#pragma unroll
      for (int i = 0; i < VEC; ++i) g[i] = 1.f;
      if (kOut && p.gate != nullptr && p.gate_col != 0) load_param<VEC>(p.gate, k.col[c], p.gate_f32, g);
#pragma unroll
      for (int h = 0; h < 2; ++h)
        fold[(2 * c + h) * nt] = make_float4(w[4 * h] * g[4 * h], w[4 * h + 1] * g[4 * h + 1], w[4 * h + 2] * g[4 * h + 2], w[4 * h + 3] * g[4 * h + 3]);
    }
  }
  for (int t = blockIdx.x; t < rows; t += gridDim.x, buf ^= 1) {
    fetch(t + gridDim.x, buf ^ 1);
    asm volatile("cp.async.wait_group 1;" ::: "memory");
    uint32_t yu[CH][4], ru[CH][4];
    RowVals<VEC, CH> r;
#pragma unroll
    for (int c = 0; c < CH; ++c) {
      const uint4* src = s_row + (buf * kStreams * CH + c) * nt + tid;
      uint4 a = make_uint4(0, 0, 0, 0), b = a;
      if (kFull || k.on[c]) {
        if constexpr (kOut) a = src[0];
        b = src[kR * CH * nt];
      }
      yu[c][0] = a.x; yu[c][1] = a.y; yu[c][2] = a.z; yu[c][3] = a.w;
      ru[c][0] = b.x; ru[c][1] = b.y; ru[c][2] = b.z; ru[c][3] = b.w;
    }
    finish_row<VEC, CH, false, false, kOut, kFull, kFold>(p, static_cast<size_t>(t), k, yu, ru, r, s_part, slot, fold);
  }
}

// Rows of bf16 at any pitch, width and alignment.  As norm_rows_kernel, but a row is copied as the 16-byte granules that it
// has in memory; a thread's eight columns come from two of them, and the results go back through the same shared memory and out
// in whole granules, single elements at the row's two edges alone (two more barriers per row).
template <int CH, bool kOut, bool kFold>
__global__ void __maxnreg__(64) norm_shift_kernel(const NormParams p) {
  extern __shared__ uint4 s_row[];                      // [buffer][y, r][granule], then the folded parameters
  __shared__ float s_part[2][32];
  constexpr int kR = kOut ? 1 : 0, kStreams = kR + 1;
  pdl_trigger();
  pdl_wait();
  int rows = p.T;
  if (p.n_valid != nullptr) rows = max(0, min(*p.n_valid, p.T));
  Cols<CH> k;
  set_cols<8, CH, false, false>(k, p.d);
  const int nt = k.nt, tid = threadIdx.x, pitch = CH * nt + 1;
  auto fetch_row = [&](const __nv_bfloat16* base, size_t ld, int t, uint4* dst) {
    const size_t at = static_cast<size_t>(t) * ld;
    const __nv_bfloat16* row = base + at;
    const int h = row_shift(row);
#pragma unroll
    for (int c = 0; c <= CH; ++c) {
      const int g = c * nt + tid, a = 8 * g - h;        // granule, its first column
      if ((c == CH && tid > 0) || a >= p.d) continue;
      // The columns before the row's first are the end of the row before, or what lies between the two; the granule
      // that begins before the first row of all is read by element.
      if (a >= 0 || at >= static_cast<size_t>(h)) {
        copy16_part(dst + g, row + a, static_cast<uint32_t>(min(16, 2 * (p.d - a))));
      } else {
        uint16_t* e = reinterpret_cast<uint16_t*>(dst + g);
        for (int i = h; i < min(8, h + p.d); ++i) e[i] = reinterpret_cast<const uint16_t*>(row)[i - h];
      }
    }
  };
  auto fetch = [&](int t, int buf) {
    if (t < rows) {
      if constexpr (kOut) fetch_row(p.y, p.ld_y, t, s_row + buf * kStreams * pitch);
      fetch_row(static_cast<const __nv_bfloat16*>(p.r), p.ld_r, t, s_row + (buf * kStreams + kR) * pitch);
    }
    asm volatile("cp.async.commit_group;" ::: "memory");
  };
  int slot = 0, buf = 0;
  fetch(blockIdx.x, 0);
  float4* fold = reinterpret_cast<float4*>(s_row + 2 * kStreams * pitch) + tid;
  if constexpr (kFold) {
#pragma unroll
    for (int c = 0; c < CH; ++c) {
      if (!k.on[c]) continue;
      float w[8], g[8];
      load_param_part(kOut ? p.post_w : p.next_w, k.col[c], p.param_f32, p.param_vec, k.n[c], w);
#pragma unroll
      for (int i = 0; i < 8; ++i) g[i] = 1.f;
      if (kOut && p.gate != nullptr && p.gate_col != 0) load_param_part(p.gate, k.col[c], p.gate_f32, p.gate_vec, k.n[c], g);
#pragma unroll
      for (int h = 0; h < 2; ++h)
        fold[(2 * c + h) * nt] = make_float4(w[4 * h] * g[4 * h], w[4 * h + 1] * g[4 * h + 1], w[4 * h + 2] * g[4 * h + 2], w[4 * h + 3] * g[4 * h + 3]);
    }
  }
  for (int t = blockIdx.x; t < rows; t += gridDim.x, buf ^= 1) {
    asm volatile("cp.async.wait_group 0;" ::: "memory");
    __syncthreads();                                    // every thread's copies of row t are here, and row t - grid was read
    fetch(t + gridDim.x, buf ^ 1);
    uint32_t yu[CH][4], ru[CH][4];
    RowVals<8, CH> r;
    const size_t row = static_cast<size_t>(t);
    uint4* in_y = s_row + buf * kStreams * pitch;
    uint4* in_r = in_y + kR * pitch;
    if constexpr (kOut) load_shifted<CH>(in_y, row_shift(p.y + row * p.ld_y), k, yu);
    load_shifted<CH>(in_r, row_shift(static_cast<const __nv_bfloat16*>(p.r) + row * p.ld_r), k, ru);
    finish_row<8, CH, false, false, kOut, false, kFold, true>(p, row, k, yu, ru, r, s_part, slot, fold, in_y, in_r);
  }
}

template <int VEC, int CH, bool kSplit, bool kF32, bool kOut>
static cudaError_t launch_norm_o(const NormParams& p, cudaStream_t stream) {
  const int threads = ((p.d + VEC * CH - 1) / (VEC * CH) + 31) / 32 * 32;
  if (VEC == 8 && p.d == VEC * CH * threads)
    return launch_pdl(norm_kernel<VEC, CH, kSplit, kF32, kOut, VEC == 8>, dim3(p.T), dim3(threads), 0, stream, p);
  return launch_pdl(norm_kernel<VEC, CH, kSplit, kF32, kOut, false>, dim3(p.T), dim3(threads), 0, stream, p);
}

// Whether the norm after a block has one parameter between its first norm and the sum: post_w, alone or with a gate per token
// or per channel.
static bool folds(const NormParams& p) {
  return p.post_w != nullptr && p.post_b == nullptr &&
         (p.gate == nullptr || p.gate_col == 0 || (p.gate_row == 0 && (p.shift ? p.gate_col == 1 : p.gate_vec != 0)));
}

template <int CH, bool kOut, bool kFull, bool kFold>
static cudaError_t launch_rows_f(const NormParams& p, int threads, int num_sms, cudaStream_t stream) {
  static std::atomic<unsigned long long> smem_set{0};
  const int smem = (2 * (kOut ? 2 : 1) + (kFold ? 2 : 0)) * CH * threads * 16;
  cudaError_t e = smem_limit_once(norm_rows_kernel<CH, kOut, kFull, kFold>, 200 * 1024, smem_set);
  if (e != cudaSuccess) return e;
  const int per_sm = max(1, min(min(32, 65536 / (64 * threads)), 224 * 1024 / (smem + 1280)));   // CTAs that are resident
  return launch_pdl(norm_rows_kernel<CH, kOut, kFull, kFold>, dim3(min(p.T, per_sm * num_sms)), dim3(threads), smem, stream, p);
}
template <int CH, bool kFull>
static cudaError_t launch_rows_t(const NormParams& p, int threads, int num_sms, cudaStream_t stream) {
  if (p.y == nullptr) return launch_rows_f<CH, false, kFull, true>(p, threads, num_sms, stream);
  return folds(p) ? launch_rows_f<CH, true, kFull, true>(p, threads, num_sms, stream) : launch_rows_f<CH, true, kFull, false>(p, threads, num_sms, stream);
}
template <int CH>
static cudaError_t launch_rows(const NormParams& p, int num_sms, cudaStream_t stream) {
  const int threads = ((p.d + 8 * CH - 1) / (8 * CH) + 31) / 32 * 32;
  return p.d == 8 * CH * threads ? launch_rows_t<CH, true>(p, threads, num_sms, stream) : launch_rows_t<CH, false>(p, threads, num_sms, stream);
}

template <int CH, bool kOut, bool kFold>
static cudaError_t launch_shift_f(const NormParams& p, int num_sms, cudaStream_t stream) {
  static std::atomic<unsigned long long> smem_set{0};
  const int threads = ((p.d + 8 * CH - 1) / (8 * CH) + 31) / 32 * 32;
  const int smem = (2 * (kOut ? 2 : 1) * (CH * threads + 1) + (kFold ? 2 * CH * threads : 0)) * 16;
  cudaError_t e = smem_limit_once(norm_shift_kernel<CH, kOut, kFold>, 200 * 1024, smem_set);
  if (e != cudaSuccess) return e;
  const int per_sm = max(1, min(min(32, 65536 / (64 * threads)), 224 * 1024 / (smem + 1280)));   // CTAs that are resident
  return launch_pdl(norm_shift_kernel<CH, kOut, kFold>, dim3(min(p.T, per_sm * num_sms)), dim3(threads), smem, stream, p);
}
template <int CH>
static cudaError_t launch_shift(const NormParams& p, int num_sms, cudaStream_t stream) {
  if (p.y == nullptr) return launch_shift_f<CH, false, true>(p, num_sms, stream);
  return folds(p) ? launch_shift_f<CH, true, true>(p, num_sms, stream) : launch_shift_f<CH, true, false>(p, num_sms, stream);
}

template <int VEC, int CH, bool kSplit>
static cudaError_t launch_norm_f32(const NormParams& p, cudaStream_t stream) {
  return p.y ? launch_norm_o<VEC, CH, kSplit, true, true>(p, stream) : launch_norm_o<VEC, CH, kSplit, true, false>(p, stream);
}
template <int VEC, int CH, bool kSplit = false>
static cudaError_t launch_norm_t(const NormParams& p, cudaStream_t stream) {
  if (p.stream_f32) return launch_norm_f32<VEC, CH, kSplit>(p, stream);
  return p.y ? launch_norm_o<VEC, CH, kSplit, false, true>(p, stream) : launch_norm_o<VEC, CH, kSplit, false, false>(p, stream);
}

// Rows of bf16 that only loads of one or two elements fit: through shared memory in 16-byte pieces (8192 rows of 7168 at a pitch
// of 7171: 117 us, element by element 383; 4096 of 5001 50 against 101, of 5002 50 against 59; one row of 4001 4.1 against
// 4.4), not rows so short that most of a warp idles (3000 of 257: 7.3 against 6.5; 8192 of 511: 17.5 against 19.0).
// Four elements at a time keep their own loads (4096 of 5004: 38.4 us, through shared memory 50).
bool norm_shifts(const NormParams& p, int vec) { return !p.stream_f32 && vec <= 2 && p.d >= 384; }

// vec: the widest load that every pointer and pitch allows (8, 4, 2 or 1 elements).
//   Fewer than two rows per SM: one chunk per thread, the shortest chain (one row of 4096: 2.4 us with one, 2.6 with two, 3.2
//   with four; 203 rows 3.9, 4.3, 5.4), unless two CTAs of that many threads do not fit an SM and there are more rows than SMs
//   (290 rows of 7168: 5.4 us with one, 4.0 with two).
//   More: the kernel with several rows per CTA where the parameter folds (4096 rows of 4096 23.3 us against 28.9, before a block
//   12.7 against 14.6), or a CTA gets few rows or wide ones (600 rows of 7168: 7.6 us against 10.9, 8192 rows 87 against 102); else
//   one row per CTA, whose CTAs' phases mix (8192 rows of 2048, two parameters after the first norm: 24.1 us against 25.7),
//   and below d = 1024, unless the columns fill whole warps and leave no thread idle (multiples of 512; 8192 rows of 512: 7.9 us
//   against 9.7; of 1000: 18.0 against 15.1).
//   An f32 stream has half as many elements to its bytes and needs the registers: one row per CTA, four chunks (8192 rows of
//   7168: 123 us against 161).
//   p.shift: one chunk per thread for few or short rows (515 rows of 1021: 3.3 us against 3.7, after a block 5.6 against 7.0),
//   two for the rest (8192 rows of 1021 10.7 us against 14.8; 4096 of 2048 at a pitch of 2051 20.4 against 22.9).
cudaError_t launch_norm(const NormParams& p, int vec, int num_sms, cudaStream_t stream) {
  if (vec == 8) {
    if (p.T < 2 * num_sms)
      return p.d > 8192 || (p.T > num_sms && p.d > 4096) ? launch_norm_t<8, 2>(p, stream) : launch_norm_t<8, 1>(p, stream);
    if (!p.stream_f32 && (p.d >= 1024 || p.d % 512 == 0) && (p.d > 4096 || p.T < 10 * num_sms || p.y == nullptr || folds(p))) return launch_rows<2>(p, num_sms, stream);
    if (p.d > 4096 || (p.stream_f32 && p.d > 2048)) return launch_norm_t<8, 4>(p, stream);
    return p.d > 512 ? launch_norm_t<8, 2>(p, stream) : launch_norm_t<8, 1>(p, stream);
  }
  if (p.shift) {
    if (p.d > 8192 || (p.T > num_sms && p.d > 1024) || (p.T > 10 * num_sms && p.d > 512)) return launch_shift<2>(p, num_sms, stream);
    return launch_shift<1>(p, num_sms, stream);
  }
  if (vec == 4) {
    if (p.d <= 4096) return launch_norm_t<4, 1>(p, stream);
    return launch_norm_t<4, 4>(p, stream);
  }
  if (p.d <= 4096) return vec == 2 ? launch_norm_t<2, 2>(p, stream) : launch_norm_t<2, 2, true>(p, stream);
  return vec == 2 ? launch_norm_f32<2, 8, false>(p, stream) : launch_norm_f32<2, 8, true>(p, stream);
}

}  // namespace tempo
