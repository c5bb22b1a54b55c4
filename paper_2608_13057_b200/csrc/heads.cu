// Norm and rotation of each head of queries and keys, the append of keys and values to the 4-bit paged cache, and the way back.
//   tempo_qk_rotate  x' = rot(norm(x) * w, position) for q and k
//   tempo_kv_append  the same for q; k' and v quantised into the cache in the same pass
//   tempo_kv_read    rows of the cache as fp16
// A head is held by D / 8 neighbouring lanes, eight elements each, so every operand is read once and every result written once.
// Queries: a lane has both elements of its pairs, so that nothing is exchanged but the sum of squares, and weights, cos and sin
// are multiplied once for all heads of a token that a group of lanes takes (one while there are few warps: latency; up to all).  Bound
// by the bytes for a prompt, 8192 tokens of 64 + 4 heads of 128 in 56.4 us, 78 % of a copy's rate; by one launch and one
// load-sum-load-store chain for a token, 2.0 us.  Rotations of other lengths than multiples of 8 and rows at odd addresses go element by
// element, the other ones through shared memory: 1200 tokens of 24 + 8 heads with 90 of 128 elements turned 13.4 us, all 128 7.5.
// Keys on their way into the cache: a code is the formula's in 64 bits also next to a border between two codes, whatever order a sum
// is taken in, so that a cache filled here equals one filled elsewhere.  They are computed in 32 bits with a bound of their error, and
// a warp in which any element lies within it of a border does all of its own again in 64.  4096 rows of 4 heads beside 64 heads of
// queries, appended and read back: 39.6 us; all in 64 bits 44.5 us.
#include "cache.cuh"

namespace tempo {

namespace {

__device__ __forceinline__ uint4 load8(const __nv_bfloat16* p, bool vec) {
  uint4 u;
  if (vec) {
    asm volatile("ld.global.L1::no_allocate.v4.b32 {%0, %1, %2, %3}, [%4];" : "=r"(u.x), "=r"(u.y), "=r"(u.z), "=r"(u.w) : "l"(p) : "memory");
  } else {
    const uint16_t* h = reinterpret_cast<const uint16_t*>(p);
    uint32_t v[4];
#pragma unroll
    for (int i = 0; i < 4; ++i) v[i] = h[2 * i] | (static_cast<uint32_t>(h[2 * i + 1]) << 16);
    u = make_uint4(v[0], v[1], v[2], v[3]);
  }
  return u;
}

__device__ __forceinline__ void store8(__nv_bfloat16* p, const float (&y)[8], bool vec) {
  uint32_t v[4];
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    const __nv_bfloat162 h = __floats2bfloat162_rn(y[2 * i], y[2 * i + 1]);
    v[i] = *reinterpret_cast<const uint32_t*>(&h);
  }
  if (vec) {
    *reinterpret_cast<uint4*>(p) = make_uint4(v[0], v[1], v[2], v[3]);
  } else {
    uint16_t* h = reinterpret_cast<uint16_t*>(p);
#pragma unroll
    for (int i = 0; i < 8; ++i) h[i] = static_cast<uint16_t>(v[i / 2] >> (16 * (i & 1)));
  }
}

__device__ __forceinline__ void widen8(uint4 u, float (&x)[8]) {
  const uint32_t v[4] = {u.x, u.y, u.z, u.w};
#pragma unroll
  for (int i = 0; i < 8; ++i) x[i] = __uint_as_float((i & 1) ? (v[i / 2] & 0xffff0000u) : (v[i / 2] << 16));
}

__device__ __forceinline__ void weights8(const void* w, int f32, bool vec, int e, float (&x)[8]) {
  if (f32) {
    const float* p = static_cast<const float*>(w) + e;
    if (vec) {
      const float4 a = __ldg(reinterpret_cast<const float4*>(p)), b = __ldg(reinterpret_cast<const float4*>(p) + 1);
      x[0] = a.x; x[1] = a.y; x[2] = a.z; x[3] = a.w; x[4] = b.x; x[5] = b.y; x[6] = b.z; x[7] = b.w;
    } else {
#pragma unroll
      for (int i = 0; i < 8; ++i) x[i] = __ldg(p + i);
    }
  } else {
    const __nv_bfloat16* p = static_cast<const __nv_bfloat16*>(w) + e;
    if (vec) {
      widen8(__ldg(reinterpret_cast<const uint4*>(p)), x);
    } else {
#pragma unroll
      for (int i = 0; i < 8; ++i) x[i] = __bfloat162float(p[i]);
    }
  }
}

__device__ __forceinline__ float weight1(const void* w, int f32, int e) {
  return f32 ? __ldg(static_cast<const float*>(w) + e) : __bfloat162float(static_cast<const __nv_bfloat16*>(w)[e]);
}

template <typename R>
__device__ __forceinline__ R inverse_root(R v);
template <>
__device__ __forceinline__ float inverse_root<float>(float v) { return rsqrtf(v); }
template <>
__device__ __forceinline__ double inverse_root<double>(double v) { return rsqrt(v); }

// A mean square (with eps) of 2^-100 to 2^101 is one that a sum in 32 bits gives: no square left their range, and what the products below
// may lose at either end of it is far below the result's last bit.
__device__ __forceinline__ bool in_range(float mean) { return __float_as_uint(mean) - (27u << 23) <= (200u << 23); }

// For a head of any size: x times a power of two that brings the head's largest element (or the root of eps) next to 1, and the inverse
// root of the mean square of that.  Returns the power.
template <int LPH>
__device__ __forceinline__ float scaled_root(const HeadsParams& p, float (&x)[8], float& r) {
  float top = 0.0f, ss = 0.0f;
#pragma unroll
  for (int i = 0; i < 8; ++i) top = fmaxf(top, fabsf(x[i]));
#pragma unroll
  for (int d = LPH / 2; d > 0; d /= 2) top = fmaxf(top, __shfl_xor_sync(0xffffffffu, top, d));
  const int e = min(max(static_cast<int>(__float_as_uint(fmaxf(top, sqrtf(p.eps))) >> 23) - 127, -126), 126);
  const float k = __uint_as_float(static_cast<uint32_t>(127 - e) << 23);
#pragma unroll
  for (int i = 0; i < 8; ++i) { x[i] *= k; ss = fmaf(x[i], x[i], ss); }
#pragma unroll
  for (int d = LPH / 2; d > 0; d /= 2) ss += __shfl_xor_sync(0xffffffffu, ss, d);
  r = rsqrtf(fmaf(ss, p.inverse_d, p.eps * k * k));
  return k;
}

// Warps per SM, with a head of each lane group to a warp, from which on a group takes four heads.
constexpr int kSpread = 64;
// Warps per SM that are kept when a group takes four heads again and again.
constexpr int kRounds = 16;

// One operand of the launch: queries or keys.
struct Operand {
  const __nv_bfloat16* x;
  size_t ld, hd;
  const void* w;
  bool vec;
};

struct Target {
  __nv_bfloat16* x;
  size_t ld, hd;
  bool vec;
};

__device__ __forceinline__ Operand operand_of(const HeadsParams& p, bool keys) {
  return keys ? Operand{p.k, p.ld_k, p.hd_k, p.k_w, p.k_vec} : Operand{p.q, p.ld_q, p.hd_q, p.q_w, p.q_vec};
}
__device__ __forceinline__ Target target_of(const HeadsParams& p, bool keys) {
  return keys ? Target{p.k_out, p.ld_k_out, p.hd_k_out, p.k_out_vec} : Target{p.q_out, p.ld_q_out, p.hd_q_out, p.q_out_vec};
}

// a * c + b * s, and what the two add up to without their signs into `amplitude`: angle tables need not be of unit length.
template <typename R>
__device__ __forceinline__ R turned_by(R a, R b, float s, float c, float& amplitude) {
  amplitude = fmaxf(amplitude, fmaf(fabsf(static_cast<float>(a)), fabsf(c), fabsf(static_cast<float>(b) * s)));
  return a * R(c) + b * R(s);
}

// A lane's eight elements of norm(x) * w turned by the row's angles, in R.  `e` is the lane's first element, beyond D for a
// lane without one; every lane of the warp takes part in the exchanges (`stage`: 32 places of the warp's own in shared memory).
// amplitude: the most that an element's two products add up to without their signs; infinite where the sum of squares is not one that
// 32 bits give, so that nothing is taken for near, and at least kLeast where an element that enters is not zero: its products may have
// vanished in 32 bits.
constexpr float kLeast = 1.2e-38f;
__device__ __forceinline__ float least_of(uint4 raw) { return ((raw.x | raw.y | raw.z | raw.w) & 0x7fff7fffu) != 0 ? kLeast : 0.0f; }
template <int LPH, typename R>
__device__ __forceinline__ void turned(const HeadsParams& p, const Operand& o, int e, bool live, const float* angles, uint4 raw, uint4* stage,
                                       R (&y)[8], float& amplitude) {
  const int lane = threadIdx.x & 31, half = p.rot / 2;
  const bool mine = live && e < p.D;
  float x[8], w[8];
  widen8(raw, x);
  R r = R(1);
  amplitude = least_of(raw);
  if (o.w != nullptr) {
    R ss = R(0);
#pragma unroll
    for (int i = 0; i < 8; ++i) ss += R(x[i]) * R(x[i]);
#pragma unroll
    for (int d = LPH / 2; d > 0; d /= 2) ss += __shfl_xor_sync(0xffffffffu, ss, d);
    const R mean = ss / R(p.D) + R(p.eps);
    r = inverse_root<R>(mean);
    if constexpr (sizeof(R) == 4) amplitude = in_range(mean) ? amplitude : INFINITY;
    if (mine) weights8(o.w, p.w_f32, p.w_vec, e, w);
  }
#pragma unroll
  for (int i = 0; i < 8; ++i) y[i] = o.w != nullptr ? R(x[i]) * r * R(w[i]) : R(x[i]);
#pragma unroll
  for (int i = 0; i < 8; ++i) amplitude = fmaxf(amplitude, fabsf(static_cast<float>(y[i])));
  if (p.rot == 0) return;

  if (p.interleaved) {
    if (!mine || e >= p.rot) return;
    float c[4], s[4];
    const float* t = angles + e / 2;
    if (p.rot_vec) {
      const float4 a = __ldg(reinterpret_cast<const float4*>(t)), b = __ldg(reinterpret_cast<const float4*>(t + half));
      c[0] = a.x; c[1] = a.y; c[2] = a.z; c[3] = a.w; s[0] = b.x; s[1] = b.y; s[2] = b.z; s[3] = b.w;
    } else {
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        const bool in = e + 2 * i < p.rot;
        c[i] = in ? __ldg(t + i) : 1.0f;
        s[i] = in ? __ldg(t + half + i) : 0.0f;
      }
    }
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      if (e + 2 * i >= p.rot) continue;                 // unturned elements pass as they are
      const R a = y[2 * i], b = y[2 * i + 1];
      y[2 * i] = turned_by(a, b, -s[i], c[i], amplitude);
      y[2 * i + 1] = turned_by(b, a, s[i], c[i], amplitude);
    }
    return;
  }

  if (p.rot_vec) {                                      // rot / 2 is a multiple of 8: the other elements are one lane's eight
    const bool turn = mine && e < p.rot, first = e < half;
    const int from = turn ? (first ? lane + half / 8 : lane - half / 8) : lane;
    uint4 u;
    u.x = __shfl_sync(0xffffffffu, raw.x, from);
    u.y = __shfl_sync(0xffffffffu, raw.y, from);
    u.z = __shfl_sync(0xffffffffu, raw.z, from);
    u.w = __shfl_sync(0xffffffffu, raw.w, from);
    if (!turn) return;
    widen8(u, x);
    amplitude = fmaxf(amplitude, least_of(u));
    const int eo = first ? e + half : e - half;
    if (o.w != nullptr) weights8(o.w, p.w_f32, p.w_vec, eo, w);
    const float4* t = reinterpret_cast<const float4*>(angles + (first ? e : eo));
    const float4* u4 = reinterpret_cast<const float4*>(angles + half + (first ? e : eo));
    float c[8], s[8];
#pragma unroll
    for (int i = 0; i < 2; ++i) {
      const float4 a = __ldg(t + i), b = __ldg(u4 + i);
      c[4 * i] = a.x; c[4 * i + 1] = a.y; c[4 * i + 2] = a.z; c[4 * i + 3] = a.w;
      s[4 * i] = b.x; s[4 * i + 1] = b.y; s[4 * i + 2] = b.z; s[4 * i + 3] = b.w;
    }
#pragma unroll
    for (int i = 0; i < 8; ++i) {
      const R other = o.w != nullptr ? R(x[i]) * r * R(w[i]) : R(x[i]);
      y[i] = turned_by(y[i], other, first ? -s[i] : s[i], c[i], amplitude);
    }
    return;
  }
  // Any even rot: the other elements one by one, through shared memory.
  stage[lane] = raw;
  __syncwarp();
  const __nv_bfloat16* head = reinterpret_cast<const __nv_bfloat16*>(stage + lane / LPH * LPH);
  if (mine) {
#pragma unroll
    for (int i = 0; i < 8; ++i) {
      if (e + i >= p.rot) continue;
      const bool first = e + i < half;
      const int eo = first ? e + i + half : e + i - half, a = first ? e + i : eo;
      const float xo = __bfloat162float(head[eo]);
      if (xo != 0.0f) amplitude = fmaxf(amplitude, kLeast);
      const R other = o.w != nullptr ? R(xo) * r * R(weight1(o.w, p.w_f32, eo)) : R(xo);
      const float s = __ldg(angles + half + a);
      y[i] = turned_by(y[i], other, first ? -s : s, __ldg(angles + a), amplitude);
    }
  }
  __syncwarp();
}

__device__ __forceinline__ const float* angles_of(const HeadsParams& p, int t, bool live) {
  if (p.rot == 0 || !live) return p.cos_sin;
  const int at = p.positions[t];
  const int in = min(max(at, 0), p.n_pos - 1);
  if (in != at) atomicOr(p.status, TEMPO_STATUS_BAD_INDEX);
  return p.cos_sin + static_cast<size_t>(in) * p.rot;
}

// Eight elements of a group that four neighbouring lanes share -> a word of eight codes, and the group's (s, 16 z) byte pair.
// Elements in 64 bits, as sums of two floats; a quotient's nearest integer comes from 32 bits and is set right by its remainder.
__device__ __forceinline__ uint32_t quantise8(const double (&y)[8], uint32_t& params) {
  double lo = 0.0, hi = 0.0;
#pragma unroll
  for (int i = 0; i < 8; ++i) { lo = y[i] < lo ? y[i] : lo; hi = y[i] > hi ? y[i] : hi; }
#pragma unroll
  for (int d = 1; d <= 2; d *= 2) {
    const double l = __shfl_xor_sync(0xffffffffu, lo, d), h = __shfl_xor_sync(0xffffffffu, hi, d);
    lo = l < lo ? l : lo;
    hi = h > hi ? h : hi;
  }
  const double range = hi - lo;
  params = 0;
  if (range == 0.0) return 0;
  float s = 768.0f;
  if (range <= 15.0 * 768.0) {
    // four significant bits, rounded up: a multiple of 2^(exponent - 3), at least of 2^-17; 32 bits may miss it by one
    const float step = static_cast<float>(range) * (1.0f / 15.0f);
    const int exponent = max(static_cast<int>(__float_as_uint(step) >> 23) - 127 - 3, -17);
    const float up = __uint_as_float(static_cast<uint32_t>(127 + exponent) << 23), down = __uint_as_float(static_cast<uint32_t>(127 - exponent) << 23);
    s = ceilf(step * down) * up;
    if (15.0 * static_cast<double>(s - up) >= range) s -= up;
    if (15.0 * static_cast<double>(s) < range) s += s >= 16.0f * up ? 2.0f * up : up;
  }
  const float inverse = 1.0f / s, h = 0.5f * s;
  const auto nearest = [&](double x) {
    const float a = static_cast<float>(x), b = static_cast<float>(x - static_cast<double>(a));
    const float k = (fminf(fmaxf(a * inverse, -1e5f), 1e5f) + 12582912.0f) - 12582912.0f;
    const float above = fmaf(-k, s, a) - h, below = fmaf(-k, s, a) + h;            // exact where it matters, next to a border
    const bool odd = (__float_as_uint(k + 12582912.0f) & 1u) != 0;
    if (above > -b || (above == -b && odd)) return k + 1.0f;
    if (below < -b || (below == -b && odd)) return k - 1.0f;
    return k;
  };
  const float z = fminf(nearest(-lo), 15.0f);
  params = (static_cast<uint32_t>(__half_as_ushort(__float2half(s))) >> 7) | (static_cast<uint32_t>(z) << 12);
  uint32_t word = 0;
#pragma unroll
  for (int i = 0; i < 8; ++i) {
    const float c = fminf(fmaxf(nearest(y[i]) + z, 0.0f), 15.0f);
    word |= (__float_as_uint(c + 8388608.0f) & 15u) << (4 * i);
  }
  return word;
}

// (a, b) * (c, d), and that plus (e, f)
__device__ __forceinline__ void mul_pair(float& a, float& b, float c, float d) {
  asm("{\n\t.reg .b64 x, y;\n\tmov.b64 x, {%0, %1};\n\tmov.b64 y, {%2, %3};\n\tmul.rn.f32x2 x, x, y;\n\tmov.b64 {%0, %1}, x;\n\t}"
      : "+f"(a), "+f"(b) : "f"(c), "f"(d));
}
__device__ __forceinline__ void fma_pair(float& a, float& b, float c, float d, float e, float f) {
  asm("{\n\t.reg .b64 x, y, z;\n\tmov.b64 x, {%0, %1};\n\tmov.b64 y, {%2, %3};\n\tmov.b64 z, {%4, %5};\n\t"
      "fma.rn.f32x2 x, x, y, z;\n\tmov.b64 {%0, %1}, x;\n\t}" : "+f"(a), "+f"(b) : "f"(c), "f"(d), "f"(e), "f"(f));
}

// Four elements of a row, or four weights.
__device__ __forceinline__ uint2 load4(const __nv_bfloat16* p) {
  uint2 u;
  asm volatile("ld.global.L1::no_allocate.v2.b32 {%0, %1}, [%2];" : "=r"(u.x), "=r"(u.y) : "l"(p) : "memory");
  return u;
}
__device__ __forceinline__ void widen4(uint2 u, float* x) {
  x[0] = __uint_as_float(u.x << 16); x[1] = __uint_as_float(u.x & 0xffff0000u);
  x[2] = __uint_as_float(u.y << 16); x[3] = __uint_as_float(u.y & 0xffff0000u);
}
__device__ __forceinline__ void weights4(const void* w, int f32, int e, float* x) {
  if (f32) {
    const float4 a = __ldg(reinterpret_cast<const float4*>(static_cast<const float*>(w) + e));
    x[0] = a.x; x[1] = a.y; x[2] = a.z; x[3] = a.w;
  } else {
    widen4(__ldg(reinterpret_cast<const uint2*>(static_cast<const __nv_bfloat16*>(w) + e)), x);
  }
}
__device__ __forceinline__ void store4(__nv_bfloat16* p, const float* y) {
  const __nv_bfloat162 a = __floats2bfloat162_rn(y[0], y[1]), b = __floats2bfloat162_rn(y[2], y[3]);
  *reinterpret_cast<uint2*>(p) = make_uint2(*reinterpret_cast<const uint32_t*>(&a), *reinterpret_cast<const uint32_t*>(&b));
}

// The same for any even rot and any alignment (see turn_heads): a lane has eight neighbouring elements, and where pairs are half a
// rotation apart their other elements come through shared memory.  FAR: those heads alone whose sums of squares are not in range, which
// the other form leaves as they are.  Returns whether the warp has any.
template <int LPH, int NH, bool FAR>
__device__ __forceinline__ bool turn_any(const HeadsParams& p, const Operand& o, const Target& out, int t, int h0, int H, int rounds, bool live,
                                         const float* angles, uint4* stage) {
  constexpr int HPW = 32 / LPH;
  const int lane = threadIdx.x & 31, e = lane % LPH * 8, half = p.rot / 2;
  const bool mine = live && e < p.D;
  uint4 raw[NH];
  const auto load = [&]() {
#pragma unroll
    for (int n = 0; n < NH; ++n) {
      const int h = h0 + n * HPW;
      raw[n] = mine && h < H ? load8(o.x + t * o.ld + h * o.hd + e, o.vec) : make_uint4(0, 0, 0, 0);
    }
  };
  load();
  float a[8], b[8];
  int others[8];                                        // below zero: the element does not turn
#pragma unroll
  for (int i = 0; i < 8; ++i) {
    const int at = e + i;
    const bool turns = mine && at < p.rot, first = p.interleaved ? (i & 1) == 0 : at < half;
    a[i] = mine && o.w != nullptr ? weight1(o.w, p.w_f32, at) : 1.0f;
    b[i] = 0.0f;
    others[i] = -1;
    if (turns) {
      const int pair = p.interleaved ? at / 2 : first ? at : at - half, other = p.interleaved ? at ^ 1 : first ? at + half : at - half;
      const float c = __ldg(angles + pair), s = __ldg(angles + half + pair);
      const float w = o.w != nullptr ? weight1(o.w, p.w_f32, other) : 1.0f;
      a[i] *= c;
      b[i] = first ? -w * s : w * s;
      others[i] = other;
    }
  }
  const __nv_bfloat16* head = reinterpret_cast<const __nv_bfloat16*>(stage + lane / LPH * LPH);
  bool left = false;
#pragma unroll 1
  for (int round = 0;; ++round) {
#pragma unroll
    for (int n = 0; n < NH; ++n) {
      float x[8], z[8];
      widen8(raw[n], x);
      float r = 1.0f, k = 1.0f;
      const int h = h0 + n * HPW;
      bool keep = mine && h < H;
      if (o.w != nullptr) {
        float ss = 0.0f;
#pragma unroll
        for (int i = 0; i < 8; ++i) ss = fmaf(x[i], x[i], ss);
#pragma unroll
        for (int d = LPH / 2; d > 0; d /= 2) ss += __shfl_xor_sync(0xffffffffu, ss, d);
        const float mean = fmaf(ss, p.inverse_d, p.eps);
        const bool far = !in_range(mean);
        left = left || (keep && far);
        keep = keep && far == FAR;
        if constexpr (FAR) k = scaled_root<LPH>(p, x, r);
        else r = rsqrtf(mean);
      }
      if (p.interleaved) {
#pragma unroll
        for (int i = 0; i < 8; ++i) z[i] = others[i] >= 0 ? x[i ^ 1] : 0.0f;
      } else {
        stage[lane] = raw[n];
        __syncwarp();
#pragma unroll
        for (int i = 0; i < 8; ++i) z[i] = others[i] >= 0 ? __bfloat162float(head[others[i]]) : 0.0f;
        __syncwarp();
        if constexpr (FAR) {
#pragma unroll
          for (int i = 0; i < 8; ++i) z[i] *= k;
        }
      }
#pragma unroll
      for (int i = 0; i < 8; ++i) x[i] = fmaf(x[i], a[i], z[i] * b[i]) * r;
      if (keep) store8(out.x + t * out.ld + h * out.hd + e, x, out.vec);
    }
    h0 += NH * HPW;
    if (round + 1 >= rounds) break;
    load();
  }
  return __any_sync(0xffffffffu, left);
}

// Heads whose sums of squares left the range of 32 bits, of `count` times HPW from h0 on.  A pass behind the others, which hardly a batch
// needs: 8192 tokens of 64 + 4 heads take 56.4 us with it and 55.2 without; 58.0 with a vote for each head on its way, 56.8 as a function
// that is called.
template <int LPH>
__device__ __forceinline__ void turn_far(const HeadsParams& p, bool keys, int t, int h0, int count, uint4* stage) {
  turn_any<LPH, 1, true>(p, operand_of(p, keys), target_of(p, keys), t, h0, keys ? p.Hkv : p.Hq, count, true, angles_of(p, t, true), stage);
}

// Heads of one token by one group of lanes, h0, h0 + HPW, ... below H, `rounds` times NH of them: NH heads' loads are in flight
// together, and weights, cos and sin are multiplied once for all.  A lane has two runs of four elements which turn with one another
// (half pairs: i and i + rot/2) or each in itself, so that nothing is exchanged but the sum of squares:
//   out[i] = r * (x[i] * a[i] + other[i] * b[i])
template <int LPH, int NH>
__device__ __forceinline__ bool turn_heads(const HeadsParams& p, const Operand& o, const Target& out, int t, int h0, int H, int rounds, bool live,
                                           uint4* stage) {
  constexpr int HPW = 32 / LPH;
  const int l = threadIdx.x % LPH, half = p.rot / 2;
  const float* angles = angles_of(p, t, live);
  if (!p.quads) return turn_any<LPH, NH, false>(p, o, out, t, h0, H, rounds, live, angles, stage);
  const bool mine = live && 8 * l < p.D;
  const bool turns = 8 * l < p.rot, apart = turns && !p.interleaved;
  const int e0 = apart ? 4 * l : 8 * l, e1 = apart ? half + 4 * l : 8 * l + 4;
  const __nv_bfloat16* src = o.x + t * o.ld + h0 * o.hd + e0;
  __nv_bfloat16* dst = out.x + t * out.ld + h0 * out.hd + e0;
  const int to = e1 - e0;
  bool left = false;
  uint2 raw[NH][2];
  const auto load = [&](int h) {
#pragma unroll
    for (int n = 0; n < NH; ++n) {
      const bool in = mine && h + n * HPW < H;
      raw[n][0] = in ? load4(src + n * HPW * o.hd) : make_uint2(0, 0);
      raw[n][1] = in ? load4(src + n * HPW * o.hd + to) : make_uint2(0, 0);
    }
  };
  load(h0);
  float a[8], b[8];
#pragma unroll
  for (int i = 0; i < 8; ++i) { a[i] = 1.0f; b[i] = 0.0f; }
  if (mine && o.w != nullptr) { weights4(o.w, p.w_f32, e0, a); weights4(o.w, p.w_f32, e1, a + 4); }
  if (mine && turns) {
    const float* at = angles + (apart ? e0 : 4 * l);
    const float4 c4 = __ldg(reinterpret_cast<const float4*>(at)), s4 = __ldg(reinterpret_cast<const float4*>(at + half));
    const float c[4] = {c4.x, c4.y, c4.z, c4.w}, s[4] = {s4.x, s4.y, s4.z, s4.w};
#pragma unroll
    for (int i = 0; i < 4; ++i) {                       // pair i: elements (i, 4 + i) of the lane's eight, or (2 i, 2 i + 1)
      const float x0 = p.interleaved ? a[2 * i] : a[i], x1 = p.interleaved ? a[2 * i + 1] : a[4 + i];
      b[i] = x0 * s[i];                                 // kept by pair until a is no longer needed
      b[4 + i] = -x1 * s[i];
    }
    float f[8];
#pragma unroll
    for (int i = 0; i < 8; ++i) f[i] = b[i];
#pragma unroll
    for (int i = 0; i < 8; ++i) a[i] *= p.interleaved ? c[i / 2] : c[i % 4];
#pragma unroll
    for (int i = 0; i < 8; ++i)                         // an element's other one: the pair's second for its first, and the reverse
      b[i] = p.interleaved ? ((i & 1) ? f[i / 2] : f[4 + i / 2]) : (i < 4 ? f[4 + i] : f[i - 4]);
  }
#pragma unroll 1
  for (int round = 0;; ++round) {
#pragma unroll
    for (int n = 0; n < NH; ++n) {
      float x[8];
      widen4(raw[n][0], x);
      widen4(raw[n][1], x + 4);
      float r = 1.0f;
      bool keep = mine && h0 + n * HPW < H;
      if (o.w != nullptr) {
        float s0 = x[0] * x[0], s1 = x[1] * x[1];
#pragma unroll
        for (int i = 2; i < 8; i += 2) {
          float q0 = x[i], q1 = x[i + 1];
          fma_pair(q0, q1, q0, q1, s0, s1);
          s0 = q0; s1 = q1;
        }
        float ss = s0 + s1;
#pragma unroll
        for (int d = LPH / 2; d > 0; d /= 2) ss += __shfl_xor_sync(0xffffffffu, ss, d);
        const float mean = fmaf(ss, p.inverse_d, p.eps);
        r = rsqrtf(mean);
        left = left || (keep && !in_range(mean));
        keep = keep && in_range(mean);
      }
      float y[8];
      if (turns) {
        if (p.interleaved) {
#pragma unroll
          for (int i = 0; i < 8; i += 2) {
            y[i] = x[i + 1]; y[i + 1] = x[i];
            mul_pair(y[i], y[i + 1], b[i], b[i + 1]);
          }
        } else {
#pragma unroll
          for (int i = 0; i < 8; i += 2) {
            y[i] = x[i ^ 4]; y[i + 1] = x[(i + 1) ^ 4];
            mul_pair(y[i], y[i + 1], b[i], b[i + 1]);
          }
        }
#pragma unroll
        for (int i = 0; i < 8; i += 2) {
          float z0 = x[i], z1 = x[i + 1];
          fma_pair(z0, z1, a[i], a[i + 1], y[i], y[i + 1]);
          y[i] = z0; y[i + 1] = z1;
        }
      } else {
#pragma unroll
        for (int i = 0; i < 8; i += 2) {
          y[i] = x[i]; y[i + 1] = x[i + 1];
          mul_pair(y[i], y[i + 1], a[i], a[i + 1]);
        }
      }
      if (o.w != nullptr) {
#pragma unroll
        for (int i = 0; i < 8; i += 2) mul_pair(y[i], y[i + 1], r, r);
      }
      if (keep) {
        store4(dst + n * HPW * out.hd, y);
        store4(dst + n * HPW * out.hd + to, y + 4);
      }
    }
    h0 += NH * HPW;
    if (round + 1 >= rounds) break;
    src += NH * HPW * o.hd;
    dst += NH * HPW * out.hd;
    load(h0);
  }
  return __any_sync(0xffffffffu, left);
}

// The same in 32 bits, for elements that are off by at most `off` (EXACT: not at all, as they came), with `sure`: whether no border
// was so near that the exact elements might have another scale, zero point or code.
template <bool EXACT>
__device__ __forceinline__ uint32_t quantise8_near(const float (&y)[8], float off, uint32_t& params, bool& sure) {
  float lo = 0.0f, hi = 0.0f;
#pragma unroll
  for (int i = 0; i < 8; ++i) { lo = fminf(lo, y[i]); hi = fmaxf(hi, y[i]); }
#pragma unroll
  for (int d = 1; d <= 2; d *= 2) {
    lo = fminf(lo, __shfl_xor_sync(0xffffffffu, lo, d));
    hi = fmaxf(hi, __shfl_xor_sync(0xffffffffu, hi, d));
  }
  const float range = hi - lo, step = range * (1.0f / 15.0f);
  const int exponent = max(static_cast<int>(__float_as_uint(step) >> 23) - 127 - 3, -17);
  const float up = __uint_as_float(static_cast<uint32_t>(127 + exponent) << 23), down = __uint_as_float(static_cast<uint32_t>(127 - exponent) << 23);
  float s = ceilf(step * down) * up;
  params = 0;
  if constexpr (EXACT) {                               // 15 s and the difference have few bits: compared as they are
    sure = range + lo == hi && hi - range == lo && range < 11000.0f;
    if (15.0f * (s - up) >= range) s -= up;
    if (15.0f * s < range) s += up;
  } else {
    const float doubt = 4.0f * off + 1e-6f * range;    // of the range: both ends, and a few roundings
    sure = range == 0.0f ? off == 0.0f : range < 15.0f * s - doubt && range > 15.0f * (s - up) + doubt && range < 11000.0f;
  }
  if (range == 0.0f || !sure) return 0;
  const float inverse = 1.0f / s;
  // a quotient is off by off / s and two roundings of at most 16
  const float border = 0.5f - off * inverse - 2.5e-6f;
  const auto nearest = [&](float x) {                  // |x / s| is at most 16
    const float q = x * inverse, k = (q + 12582912.0f) - 12582912.0f;
    if constexpr (!EXACT) sure = sure && fabsf(q - k) < border;
    if constexpr (EXACT) {
      const float rest = fmaf(-k, s, x), h = 0.5f * s;
      const bool odd = (__float_as_uint(k + 12582912.0f) & 1u) != 0;
      if (rest > h || (rest == h && odd)) return k + 1.0f;
      if (rest < -h || (rest == -h && odd)) return k - 1.0f;
    }
    return k;
  };
  const float z = fminf(nearest(-lo), 15.0f);
  params = (static_cast<uint32_t>(__half_as_ushort(__float2half(s))) >> 7) | (static_cast<uint32_t>(z) << 12);
  uint32_t word = 0;
#pragma unroll
  for (int i = 0; i < 8; ++i) {
    const float c = fminf(fmaxf(nearest(y[i]) + z, 0.0f), 15.0f);
    word |= (__float_as_uint(c + 8388608.0f) & 15u) << (4 * i);
  }
  return word;
}

template <int LPH, bool APPEND, int NH>
__global__ void __launch_bounds__(256, 4) heads_kernel(const __grid_constant__ HeadsParams p) {
  constexpr int HPW = 32 / LPH;                          // heads of a warp at a time
  __shared__ uint4 stages[8][32];
  uint4* stage = stages[threadIdx.x >> 5];
  pdl_trigger();
  pdl_wait();
  const int n = p.n_valid != nullptr ? min(max(*p.n_valid, 0), p.T) : p.T;
  const int lane = threadIdx.x & 31, e = (lane % LPH) * 8;
  // the keys, which take longest on their way into the cache, begin first
  const uint32_t k_blocks = p.k_blocks;
  const bool keys = blockIdx.x < k_blocks;
  const int H = keys ? p.Hkv : p.Hq;
  const int rounds = keys ? 1 : p.rounds, step = HPW * (APPEND && keys ? 1 : NH * rounds);
  const uint32_t chunks = (H + step - 1) / step;         // of a token's heads
  const uint32_t warp = (blockIdx.x - (keys ? 0u : k_blocks)) * 8 + (threadIdx.x >> 5);
  const uint32_t row = warp / chunks;
  const int h0 = static_cast<int>(warp - row * chunks) * step + lane / LPH;
  const bool in = row < static_cast<uint32_t>(n);
  const int t = in ? static_cast<int>(row) : 0;
  const Operand o = operand_of(p, keys);
  if (!APPEND || !keys) {
    if (turn_heads<LPH, NH>(p, o, target_of(p, keys), t, h0, H, rounds, in, stage)) turn_far<LPH>(p, keys, t, h0, NH * rounds, stage);
    return;
  }

  const bool live = in && h0 < H;
  const int h = h0 < H ? h0 : 0;
  const size_t at = t * o.ld + h * o.hd;
  const bool mine = live && e < p.D;
  const uint4 zero = make_uint4(0, 0, 0, 0);
  uint4 raw = mine ? load8(o.x + at + e, o.vec) : zero;
  const uint4 raw_v = mine ? load8(p.v + t * p.ld_v + h * p.hd_v + e, p.v_vec) : zero;
  const int slot = live ? p.slots[t] : -1;
  const float* angles = angles_of(p, t, live);
  float v[8];
  widen8(raw_v, v);
  uint32_t pk, pv, wk, wv;
  bool bad = false;
  {
    // In 32 bits first.  An element is off by less than 15 * 2^-24 of its amplitude: 4 of the inverse root, half of 13 of the sum of
    // squares under it, 4 of the products.
    float y[8], amplitude;
    turned<LPH, float>(p, o, e, live, angles, raw, stage, y, amplitude);
#pragma unroll
    for (int d = 1; d <= 2; d *= 2) amplitude = fmaxf(amplitude, __shfl_xor_sync(0xffffffffu, amplitude, d));
    bool sure_k, sure_v;
    wk = quantise8_near<false>(y, amplitude * 0x1p-20f, pk, sure_k);
    wv = quantise8_near<true>(v, 0.0f, pv, sure_v);
    bool fine = sure_k && sure_v;
#pragma unroll
    for (int i = 0; i < 8; ++i) fine = fine && isfinite(v[i]) && isfinite(y[i]);
    if (__any_sync(0xffffffffu, mine && !fine)) {
      // Some element of the warp is next to a border (one warp of 150) or not finite: all of them in 64 bits.
      double exact[8];
      turned<LPH, double>(p, o, e, live, angles, raw, stage, exact, amplitude);
#pragma unroll
      for (int i = 0; i < 8; ++i) {
        if (!isfinite(exact[i])) { exact[i] = 0.0; bad = true; }
        if (!isfinite(v[i])) { v[i] = 0.0f; bad = true; }
      }
      const uint32_t head_lanes = (LPH == 32 ? 0xffffffffu : ((1u << LPH) - 1u)) << (lane / LPH * LPH);
      bad = (__ballot_sync(0xffffffffu, bad) & head_lanes) != 0;
      wk = quantise8(exact, pk);
#pragma unroll
      for (int i = 0; i < 8; ++i) exact[i] = v[i];
      wv = quantise8(exact, pv);
    }
  }
  if (bad) pk |= kMarked;
  if (!live) return;
  if (slot < 0 || slot >= p.n_pages * p.page_size) {
    if (slot >= 0) atomicOr(p.status, TEMPO_STATUS_BAD_INDEX);
    return;
  }
  if (bad) atomicOr(p.status, TEMPO_STATUS_BAD_VALUE);
  if constexpr (APPEND) {
    using U = CacheUnit<LPH * 8>;
    const int page = slot / p.page_size, in_page = slot % p.page_size, in_unit = in_page % kUnit;
    uint8_t* uk = p.cache + unit_offset<LPH * 8>(page, h, 0, in_page, p.Hkv, p.page_size);
    uint8_t* uv = p.cache + unit_offset<LPH * 8>(page, h, 1, in_page, p.Hkv, p.page_size);
    *reinterpret_cast<uint32_t*>(uk + in_unit * U::kKeyRow + e / 2) = wk;
    uint16_t* pair = reinterpret_cast<uint16_t*>(uv + (in_unit / 2) * U::kPairRow + e) + (in_unit & 1);
    pair[0] = static_cast<uint16_t>(wv);
    pair[2] = static_cast<uint16_t>(wv >> 16);
    if (e % kGroup == 0) {
      *reinterpret_cast<uint16_t*>(uk + U::kCodes + in_unit * U::kKeyParams + e / kGroup * 2) = static_cast<uint16_t>(pk);
      *reinterpret_cast<uint16_t*>(uv + U::kCodes + (in_unit / 2) * U::kPairParams + e / kGroup * 4 + (in_unit & 1) * 2) =
          static_cast<uint16_t>(pv);
    }
  }
}

template <int D>
__global__ void __launch_bounds__(256) kv_read_kernel(const __grid_constant__ KvReadParams p) {
  constexpr int LPH = D / 8;
  using U = CacheUnit<D>;
  pdl_trigger();
  pdl_wait();
  const int64_t item = (static_cast<int64_t>(blockIdx.x) * blockDim.x + threadIdx.x) / LPH;
  const int e = (threadIdx.x % LPH) * 8;
  const int64_t i = item / p.Hkv;
  const int h = static_cast<int>(item - i * p.Hkv);
  if (i >= p.n) return;
  const int slot = p.slots[i];
  uint4 k = make_uint4(0, 0, 0, 0), v = k;
  if (slot >= 0 && slot < p.n_pages * p.page_size) {
    const int page = slot / p.page_size, in_page = slot % p.page_size, in_unit = in_page % kUnit;
    const uint8_t* uk = p.cache + unit_offset<D>(page, h, 0, in_page, p.Hkv, p.page_size);
    const uint8_t* uv = p.cache + unit_offset<D>(page, h, 1, in_page, p.Hkv, p.page_size);
    const uint16_t* pair = reinterpret_cast<const uint16_t*>(uv + (in_unit / 2) * U::kPairRow + e) + (in_unit & 1);
    const uint32_t words[2] = {*reinterpret_cast<const uint32_t*>(uk + in_unit * U::kKeyRow + e / 2),
                               pair[0] | (static_cast<uint32_t>(pair[2]) << 16)};
    const uint32_t params[2] = {
        *reinterpret_cast<const uint16_t*>(uk + U::kCodes + in_unit * U::kKeyParams + e / kGroup * 2),
        *reinterpret_cast<const uint16_t*>(uv + U::kCodes + (in_unit / 2) * U::kPairParams + e / kGroup * 4 + (in_unit & 1) * 2)};
    uint4* out[2] = {&k, &v};
#pragma unroll
    for (int j = 0; j < 2; ++j) {
      uint32_t s, b, pairs[4];
      group_params(params[j] * 0x10001u, s, b);
      decode8(Decode(), words[j], s, b, pairs);                    // codes (n, n + 4)
      *out[j] = make_uint4(__byte_perm(pairs[0], pairs[1], 0x5410), __byte_perm(pairs[2], pairs[3], 0x5410),
                           __byte_perm(pairs[0], pairs[1], 0x7632), __byte_perm(pairs[2], pairs[3], 0x7632));
    }
  } else if (slot >= 0) {
    atomicOr(p.status, TEMPO_STATUS_BAD_INDEX);
  }
  const size_t at = (static_cast<size_t>(i) * p.Hkv + h) * D + e;
  *reinterpret_cast<uint4*>(p.k + at) = k;
  *reinterpret_cast<uint4*>(p.v + at) = v;
}

template <int LPH, bool APPEND, int NH>
cudaError_t launch_heads_as(HeadsParams p, int rounds, cudaStream_t stream) {
  constexpr int HPW = 32 / LPH, kKeys = HPW * (APPEND ? 1 : NH);
  const int queries = HPW * NH * rounds;
  const int64_t k = (static_cast<int64_t>(p.T) * ((p.Hkv + kKeys - 1) / kKeys) + 7) / 8;
  const int64_t q = (static_cast<int64_t>(p.T) * ((p.Hq + queries - 1) / queries) + 7) / 8;
  if (k + q > 0x1fffffff) return cudaErrorInvalidValue;          // warps are numbered in 32 bits
  p.k_blocks = static_cast<uint32_t>(k);
  p.rounds = rounds;
  return launch_pdl(heads_kernel<LPH, APPEND, NH>, dim3(static_cast<unsigned>(k + q)), dim3(256), 0, stream, p);
}

// One head to a lane group while there are few warps, then four, then four again and again up to all of a token's.
template <int LPH, bool APPEND>
cudaError_t launch_heads_as(const HeadsParams& p, int num_sms, cudaStream_t stream) {
  constexpr int HPW = 32 / LPH;
  const int64_t warps = static_cast<int64_t>(p.T) * (static_cast<int64_t>(p.Hq) + p.Hkv) / HPW, few = static_cast<int64_t>(num_sms) * kSpread;
  if (warps <= few) return launch_heads_as<LPH, APPEND, 1>(p, 1, stream);
  const int most = max(1, (p.Hq + 4 * HPW - 1) / (4 * HPW));
  const int chunks = static_cast<int>(min(static_cast<int64_t>(most), (static_cast<int64_t>(num_sms) * kRounds + p.T - 1) / p.T));   // of a token
  return launch_heads_as<LPH, APPEND, 4>(p, (most + chunks - 1) / chunks, stream);
}

}  // namespace

cudaError_t launch_heads(const HeadsParams& p, bool append, int num_sms, cudaStream_t stream) {
  if (append) return p.D == 64 ? launch_heads_as<8, true>(p, num_sms, stream) : launch_heads_as<16, true>(p, num_sms, stream);
  if (p.D <= 64) return launch_heads_as<8, false>(p, num_sms, stream);
  if (p.D <= 128) return launch_heads_as<16, false>(p, num_sms, stream);
  return launch_heads_as<32, false>(p, num_sms, stream);
}

cudaError_t launch_kv_read(const KvReadParams& p, int D, cudaStream_t stream) {
  const int64_t blocks = (static_cast<int64_t>(p.n) * p.Hkv * (D / 8) + 255) / 256;
  if (blocks > 0x7fffffff) return cudaErrorInvalidValue;
  const dim3 grid(static_cast<unsigned>(blocks));
  return D == 64 ? launch_pdl(kv_read_kernel<64>, grid, dim3(256), 0, stream, p)
                 : launch_pdl(kv_read_kernel<128>, grid, dim3(256), 0, stream, p);
}

}  // namespace tempo
