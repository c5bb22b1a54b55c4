// The norms around a block.  One row of the residual stream per CTA, held in registers from the first load to the last
// store, so every operand is read once and every result written once:
//   tempo_norm_in    x  = norm(r) * w + b
//   tempo_norm_out   r' = r_scale * r + y_scale * g (.) (norm(y) * post_w + post_b),  x' = norm(r') * next_w + next_b
// norm(v) = v / sqrt(mean(v^2) + eps), or the same of v - mean(v).  The mean and the mean square are two sums over
// the row, each a shuffle tree in a warp and a fixed-order sum over the warps (32-bit, the same bits every time); the
// centred square sum is taken after the mean from the registers, not as a difference of two large sums.
// x' is taken from the 32-bit r', not from its rounding to the stream's type.
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

// v (CH chunks of VEC values of this thread; those beyond the row are zero) -> normed in place, without weights.
template <int VEC, int CH>
__device__ __forceinline__ void norm_row(float (&v)[CH][VEC], const bool (&on)[CH], int layer, float inv_d, float eps,
                                         float (&s_part)[2][32], int& slot, int warps) {
  if (layer) {
    float s = 0.f;
#pragma unroll
    for (int c = 0; c < CH; ++c)
#pragma unroll
      for (int i = 0; i < VEC; ++i) s += v[c][i];
    const float mean = cta_sum(s, s_part, slot, warps) * inv_d;
    slot ^= 1;
#pragma unroll
    for (int c = 0; c < CH; ++c)
#pragma unroll
      for (int i = 0; i < VEC; ++i) v[c][i] = on[c] ? v[c][i] - mean : 0.f;
  }
  float q = 0.f;
#pragma unroll
  for (int c = 0; c < CH; ++c)
#pragma unroll
    for (int i = 0; i < VEC; ++i) q = fmaf(v[c][i], v[c][i], q);
  const float ms = cta_sum(q, s_part, slot, warps) * inv_d;
  slot ^= 1;
  const float r = 1.f / sqrtf(ms + eps);
#pragma unroll
  for (int c = 0; c < CH; ++c)
#pragma unroll
    for (int i = 0; i < VEC; ++i) v[c][i] *= r;
}

// kF32: the residual stream is f32.  p.y == NULL: the norm before a block.
template <int VEC, int CH, bool kF32>
__global__ void __launch_bounds__(VEC * CH >= 32 ? 512 : 1024) norm_kernel(const NormParams p) {
  __shared__ float s_part[2][32];
  const int t = blockIdx.x, nt = blockDim.x, warps = nt >> 5;
  pdl_trigger();
  pdl_wait();
  if (p.n_valid != nullptr && t >= *p.n_valid) return;
  const float inv_d = 1.f / static_cast<float>(p.d);
  int col[CH];
  bool on[CH];
#pragma unroll
  for (int c = 0; c < CH; ++c) {
    col[c] = (c * nt + static_cast<int>(threadIdx.x)) * VEC;
    on[c] = col[c] < p.d;                               // d is a multiple of VEC
  }
  const size_t row = static_cast<size_t>(t);
  uint32_t yu[CH][(VEC + 1) / 2], ru[CH][(VEC + 1) / 2];
  float v[CH][VEC], rf[CH][VEC];
  int slot = 0;
#pragma unroll
  for (int c = 0; c < CH; ++c) {
    if constexpr (kF32) {
#pragma unroll
      for (int i = 0; i < VEC; ++i) rf[c][i] = 0.f;
    }
#pragma unroll
    for (int i = 0; i < (VEC + 1) / 2; ++i) yu[c][i] = ru[c][i] = 0u;
    if (!on[c]) continue;
    if (p.y != nullptr) load_bf16_stream<VEC>(p.y + row * p.ld_y + col[c], yu[c]);
    if constexpr (kF32) load_f32_stream<VEC>(static_cast<const float*>(p.r) + row * p.ld_r + col[c], rf[c]);
    else load_bf16_stream<VEC>(static_cast<const __nv_bfloat16*>(p.r) + row * p.ld_r + col[c], ru[c]);
  }
  if (p.y != nullptr) {
#pragma unroll
    for (int c = 0; c < CH; ++c) widen<VEC>(yu[c], v[c]);
    if (p.post_w != nullptr) norm_row<VEC, CH>(v, on, p.layer, inv_d, p.eps, s_part, slot, warps);
    float gt = 1.f;
    if (p.gate != nullptr && p.gate_col == 0) {         // one gate for the row
      float g1[1];
      load_param<1>(p.gate, row * p.gate_row, p.gate_f32, g1);
      gt = g1[0];
    }
    const float ys = p.y_scale * gt;
#pragma unroll
    for (int c = 0; c < CH; ++c) {
      if (!on[c]) continue;
      float w[VEC];
      if (p.post_w != nullptr) {
        load_param<VEC>(p.post_w, col[c], p.param_f32, w);
#pragma unroll
        for (int i = 0; i < VEC; ++i) v[c][i] *= w[i];
        if (p.post_b != nullptr) {
          load_param<VEC>(p.post_b, col[c], p.param_f32, w);
#pragma unroll
          for (int i = 0; i < VEC; ++i) v[c][i] += w[i];
        }
      }
      if (p.gate != nullptr && p.gate_col != 0) {
        if (p.gate_vec) {
          load_param<VEC>(p.gate, row * p.gate_row + col[c], p.gate_f32, w);
        } else {
#pragma unroll
          for (int i = 0; i < VEC; ++i) {
            float g1[1];
            load_param<1>(p.gate, row * p.gate_row + static_cast<size_t>(col[c] + i) * p.gate_col, p.gate_f32, g1);
            w[i] = g1[0];
          }
        }
#pragma unroll
        for (int i = 0; i < VEC; ++i) v[c][i] *= w[i];
      }
      if constexpr (!kF32) widen<VEC>(ru[c], rf[c]);
#pragma unroll
      for (int i = 0; i < VEC; ++i) v[c][i] = fmaf(ys, v[c][i], p.r_scale * rf[c][i]);
      if constexpr (kF32) store_f32<VEC>(static_cast<float*>(p.r_out) + row * p.ld_r_out + col[c], v[c]);
      else store_bf16<VEC>(static_cast<__nv_bfloat16*>(p.r_out) + row * p.ld_r_out + col[c], v[c]);
    }
    if (p.x == nullptr) return;
  } else {
#pragma unroll
    for (int c = 0; c < CH; ++c) {
      if constexpr (kF32) {
#pragma unroll
        for (int i = 0; i < VEC; ++i) v[c][i] = rf[c][i];
      } else {
        widen<VEC>(ru[c], v[c]);
      }
    }
  }
  norm_row<VEC, CH>(v, on, p.layer, inv_d, p.eps, s_part, slot, warps);
#pragma unroll
  for (int c = 0; c < CH; ++c) {
    if (!on[c]) continue;
    float w[VEC];
    load_param<VEC>(p.next_w, col[c], p.param_f32, w);
#pragma unroll
    for (int i = 0; i < VEC; ++i) v[c][i] *= w[i];
    if (p.next_b != nullptr) {
      load_param<VEC>(p.next_b, col[c], p.param_f32, w);
#pragma unroll
      for (int i = 0; i < VEC; ++i) v[c][i] += w[i];
    }
    store_bf16<VEC>(p.x + row * p.ld_x + col[c], v[c]);
  }
}

template <int VEC, int CH>
static cudaError_t launch_norm_t(const NormParams& p, cudaStream_t stream) {
  const int threads = ((p.d + VEC * CH - 1) / (VEC * CH) + 31) / 32 * 32;
  if (p.stream_f32) return launch_pdl(norm_kernel<VEC, CH, true>, dim3(p.T), dim3(threads), 0, stream, p);
  return launch_pdl(norm_kernel<VEC, CH, false>, dim3(p.T), dim3(threads), 0, stream, p);
}

// vec: the widest load that every pointer and pitch allows (8, 4, 2 or 1 elements).  Chunks per thread: one where the
// row count leaves SMs idle (latency), more where they are full.
cudaError_t launch_norm(const NormParams& p, int vec, int num_sms, cudaStream_t stream) {
  const bool full = p.T >= 2 * num_sms;
  if (vec == 8) {
    if (full && p.d > 2048) return launch_norm_t<8, 4>(p, stream);
    if (p.d > 8192 || (full && p.d > 512)) return launch_norm_t<8, 2>(p, stream);
    return launch_norm_t<8, 1>(p, stream);
  }
  if (vec == 4) {
    if (p.d <= 4096) return launch_norm_t<4, 1>(p, stream);
    return launch_norm_t<4, 4>(p, stream);
  }
  if (vec == 2) {
    if (p.d <= 4096) return launch_norm_t<2, 2>(p, stream);
    return launch_norm_t<2, 8>(p, stream);
  }
  if (p.d <= 4096) return launch_norm_t<1, 4>(p, stream);
  return launch_norm_t<1, 16>(p, stream);
}

}  // namespace tempo
