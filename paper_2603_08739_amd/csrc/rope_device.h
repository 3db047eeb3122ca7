// rope_device.h - rotation of a head's elements and roundings to a cache's types, shared by
// the kernels that write rotated heads (the mathematics: k_rope.hip).
#pragma once

#include "kv_device.h"
#include "kv_paged.h"

namespace kv {
namespace rope {

typedef __bf16 bf16x8 __attribute__((ext_vector_type(8)));
typedef _Float16 f16x8 __attribute__((ext_vector_type(8)));
template <class V>
struct Elem;
template <>
struct Elem<bf16x8> {
  typedef __bf16 type;
  static constexpr float kMost = 0x1.fep127f;  // the largest number
};
template <>
struct Elem<f16x8> {
  typedef _Float16 type;
  static constexpr float kMost = 65504.0f;
};

template <class V>
__device__ __forceinline__ void unpack(const uint4& u, float* f) {
  const V v = __builtin_bit_cast(V, u);
#pragma unroll
  for (int i = 0; i < 8; ++i) f[i] = (float)v[i];
}

template <class V>
__device__ __forceinline__ uint4 pack(const float* f) {
  V v;
#pragma unroll
  for (int i = 0; i < 8; ++i) v[i] = (typename Elem<V>::type)f[i];
  return __builtin_bit_cast(uint4, v);
}

// To e4m3, nearest even; past the largest number, that number; NaN stays NaN.
__device__ __forceinline__ uint32_t pack_fp8x4(float a, float b, float c, float d) {
  auto cut = [](float x) { return fabsf(x) > 448.0f ? copysignf(448.0f, x) : x; };
  uint32_t u = __builtin_amdgcn_cvt_pk_fp8_f32(cut(a), cut(b), 0, false);
  return __builtin_amdgcn_cvt_pk_fp8_f32(cut(c), cut(d), u, true);
}

__device__ __forceinline__ uint2 pack_fp8(const float* f) {
  return make_uint2(pack_fp8x4(f[0], f[1], f[2], f[3]), pack_fp8x4(f[4], f[5], f[6], f[7]));
}

// Sine and cosine of p * turn turns.
__device__ __forceinline__ void turn_sincos(int32_t p, uint64_t turn, float& sn, float& cs) {
  const uint64_t t = (uint64_t)(int64_t)p * turn;
  const uint32_t hi = (uint32_t)(t >> 32);
  const uint32_t quarter = (hi + (1u << 29)) >> 30;               // nearest quarter turn
  const float x = (float)(int32_t)(hi - (quarter << 30)) * 1.4629180792671596e-9f;  // 2 pi / 2^32
  const float z = x * x;
  float s = fmaf(z, 2.7557319e-6f, -1.9841270e-4f);
  s = fmaf(z, s, 8.3333333e-3f);
  s = fmaf(z, s, -1.6666667e-1f);
  s = fmaf(x * z, s, x);
  float c = fmaf(z, -2.7557319e-7f, 2.4801587e-5f);
  c = fmaf(z, c, -1.3888889e-3f);
  c = fmaf(z, c, 4.1666667e-2f);
  c = fmaf(z, c, -0.5f);
  c = fmaf(z, c, 1.0f);
  const bool odd = quarter & 1;
  const float a = odd ? c : s, b = odd ? s : c;
  sn = (quarter & 2) ? -a : a;
  cs = ((quarter + 1) & 2) ? -b : b;
}

struct Turns {
  float sn[8], cs[8];
};

__device__ __forceinline__ void load_turns(Turns& t, const uint64_t* __restrict__ turn, int unit, int32_t p, float sign,
                                           float magnitude) {
#pragma unroll
  for (int i = 0; i < 8; ++i) {
    float s, c;
    turn_sincos(p, turn[unit * 8 + i], s, c);
    t.sn[i] = s * sign * magnitude;
    t.cs[i] = c * magnitude;
  }
}

// The elements of unit u of a head: chunks of 8 at lo and hi.
template <bool kHalf>
__device__ __forceinline__ void unit_at(int unit, int rot_dim, int& lo, int& hi) {
  if (kHalf && unit < rot_dim / 16) {
    lo = unit * 8;
    hi = lo + rot_dim / 2;
  } else {
    lo = unit * 16;
    hi = lo + 8;
  }
}

template <bool kHalf>
__device__ __forceinline__ void turn_unit(float* a, float* b, const Turns& t) {
  if (kHalf) {
#pragma unroll
    for (int i = 0; i < 8; ++i) {
      const float x = a[i], y = b[i];
      a[i] = fmaf(x, t.cs[i], -(y * t.sn[i]));
      b[i] = fmaf(x, t.sn[i], y * t.cs[i]);
    }
  } else {
#pragma unroll
    for (int i = 0; i < 8; ++i) {
      float* e = i < 4 ? a + 2 * i : b + 2 * (i - 4);
      const float x = e[0], y = e[1];
      e[0] = fmaf(x, t.cs[i], -(y * t.sn[i]));
      e[1] = fmaf(x, t.sn[i], y * t.cs[i]);
    }
  }
}

// A thread's elements of heads first .. end - 1 of a token.  Four heads are read before
// the first is written: the compiler may not move reads past writes, as y may be x.
template <class V, bool kHalf>
__device__ __forceinline__ void turn_heads(const uint16_t* x, int64_t xh, uint16_t* y, int64_t yh, uint32_t first,
                                           uint32_t end, int lo, int hi, bool turns, const Turns& t) {
  constexpr uint32_t kAhead = 4;
  for (uint32_t h = first; h < end; h += kAhead) {
    uint4 u[kAhead], w[kAhead];
#pragma unroll
    for (uint32_t i = 0; i < kAhead; ++i)
      if (h + i < end) {
        u[i] = *(const uint4*)(x + (h + i) * xh + lo);
        w[i] = *(const uint4*)(x + (h + i) * xh + hi);
      }
#pragma unroll
    for (uint32_t i = 0; i < kAhead; ++i)
      if (h + i < end) {
        if (turns) {
          float f[8], g[8];
          unpack<V>(u[i], f);
          unpack<V>(w[i], g);
          turn_unit<kHalf>(f, g, t);
          u[i] = pack<V>(f);
          w[i] = pack<V>(g);
        }
        *(uint4*)(y + (h + i) * yh + lo) = u[i];
        *(uint4*)(y + (h + i) * yh + hi) = w[i];
      }
  }
}

// Heads a thread walks over: more of them share its sines and cosines, but a
// step of few tokens needs the threads.  One per thread up to 2^18 units (four
// wavefronts on each SIMD of the chip), at most eight.
inline uint32_t heads_each_for(uint64_t units) {
  uint32_t n = 1;
  while (n < 8 && units / (n * 2) >= (1u << 18)) n *= 2;
  return n;
}

}  // namespace rope
}  // namespace kv
