// k_attn.hip - attention of a step's new tokens over a paged KV cache.
//
// For a request with c cached tokens, its new token t sees the keys j <= c + t
// within the window:  o_t = sum_j w_tj V_j,  w_tj = exp(s q_t.K_j - m_t) / l_t,
// one pass over the keys with the running maximum m and sum l in 32 bits.  The
// G query heads of a key/value head are rows of one matrix (row = t*G + head), so
// keys and values are read once for all of them.
//
// Both kernels work on transposed products: S^T = K Q^T, O^T = V^T P^T.  In the
// matrix instructions' result a lane then holds one query's column: its share of
// the row maximum and sum stays in the lane, rescaling O needs no broadcast, and
// P^T, the second product's right operand, is the first product's result converted
// in place.  For the key order of the two to agree, the rows of K are fed
// permuted: wherever a lane will hold results for several runs of 4 keys,
// it gets runs that follow one another in the cache, so that its V^T operand is a
// plain run of keys.
//
//   k_attn_tile   tiles of 128 rows (four wavefronts of 32), 64 keys at a time
//                 through LDS: chunks of prompts, bound by the matrix cores
//   k_attn_rows   up to 64 rows (single tokens): keys and values go from memory
//                 to registers, four wavefronts share the keys; bound by memory
//   k_attn_join   the pieces of tiles whose keys were cut
//
// A weight of 0 times a NaN or an infinity in a masked value would be NaN.  Where
// a tile holds masked keys, values are therefore looked at: non-finite ones are
// taken out of the product and added back only to the queries that see them.
#include "kv_device.h"
#include "kv_paged.h"

namespace kv {
namespace {

typedef __bf16 bf16x8 __attribute__((ext_vector_type(8)));
typedef __bf16 bf16x2 __attribute__((ext_vector_type(2)));
typedef _Float16 f16x8 __attribute__((ext_vector_type(8)));
typedef _Float16 f16x2 __attribute__((ext_vector_type(2)));
typedef float f32x16 __attribute__((ext_vector_type(16)));
typedef float f32x4 __attribute__((ext_vector_type(4)));

constexpr float kLog2e = 1.4426950408889634f;
constexpr float kLn2 = 0.6931471805599453f;

struct BF16 {
  static constexpr uint32_t kExp = 0x7f80u;  // exponent bits: all set = not finite
  static constexpr uint16_t kOne = 0x3f80u;
  static __device__ __forceinline__ f32x16 mfma32(const uint4& a, const uint4& b, const f32x16& c) {
    return __builtin_amdgcn_mfma_f32_32x32x16_bf16(__builtin_bit_cast(bf16x8, a), __builtin_bit_cast(bf16x8, b), c, 0, 0, 0);
  }
  static __device__ __forceinline__ f32x4 mfma16(const uint4& a, const uint4& b, const f32x4& c) {
    return __builtin_amdgcn_mfma_f32_16x16x32_bf16(__builtin_bit_cast(bf16x8, a), __builtin_bit_cast(bf16x8, b), c, 0, 0, 0);
  }
  static __device__ __forceinline__ uint32_t pack(float a, float b) {
    bf16x2 v;
    v[0] = (__bf16)a;
    v[1] = (__bf16)b;
    return __builtin_bit_cast(uint32_t, v);
  }
  // two 8-bit numbers (low or high half of u); exact, e4m3 fits in 16 bits
  template <bool kHigh>
  static __device__ __forceinline__ uint32_t widen(uint32_t u) {
    return __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(u, 1.0f, kHigh));
  }
};

struct F16 {
  static constexpr uint32_t kExp = 0x7c00u;
  static constexpr uint16_t kOne = 0x3c00u;
  static __device__ __forceinline__ f32x16 mfma32(const uint4& a, const uint4& b, const f32x16& c) {
    return __builtin_amdgcn_mfma_f32_32x32x16_f16(__builtin_bit_cast(f16x8, a), __builtin_bit_cast(f16x8, b), c, 0, 0, 0);
  }
  static __device__ __forceinline__ f32x4 mfma16(const uint4& a, const uint4& b, const f32x4& c) {
    return __builtin_amdgcn_mfma_f32_16x16x32_f16(__builtin_bit_cast(f16x8, a), __builtin_bit_cast(f16x8, b), c, 0, 0, 0);
  }
  static __device__ __forceinline__ uint32_t pack(float a, float b) {
    f16x2 v;
    v[0] = (_Float16)a;
    v[1] = (_Float16)b;
    return __builtin_bit_cast(uint32_t, v);
  }
  template <bool kHigh>
  static __device__ __forceinline__ uint32_t widen(uint32_t u) {
    return __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_f16_fp8(u, 1.0f, kHigh));
  }
};

// 8 numbers of 8 bits to 16 bits
template <class T>
__device__ __forceinline__ uint4 widen8(uint32_t a, uint32_t b) {
  return make_uint4(T::template widen<false>(a), T::template widen<true>(a), T::template widen<false>(b),
                    T::template widen<true>(b));
}

struct AttnArgs {
  const uint16_t* q;
  uint16_t* out;
  float* lse;
  int64_t qt, qh, ot, oh;
  const uint8_t *k, *v;
  int64_t k_block, v_block;  // bytes
  const float *k_scale, *v_scale;
  const int32_t* table;
  const WorkHeader* head;
  const PieceItem* items;
  const SplitTile* split;
  float *acc, *ml;
  float scale;
  uint32_t max_tokens, max_blocks, n_blocks, kv_heads, q_heads, group, window, shift;
};

// Both halves of the wave exchange a value (lane i with lane i ^ 32).
__device__ __forceinline__ float other_half(float x) {
  const uint32_t u = __builtin_bit_cast(uint32_t, x);
  const auto r = __builtin_amdgcn_permlane32_swap(u, u, false, false);
  return __builtin_bit_cast(float, lane_id() < 32 ? r[1] : r[0]);
}

// Masked values that are not finite (see the head of the file).  For one 16-bit
// operand register: the numbers that are not finite become 0.
template <class T>
__device__ __forceinline__ uint32_t not_finite(uint32_t u) {  // all ones in the halves that are not finite
  uint32_t m = 0;
  if ((u & T::kExp) == T::kExp) m |= 0xffffu;
  if (((u >> 16) & T::kExp) == T::kExp) m |= 0xffff0000u;
  return m;
}
template <class T>
__device__ __forceinline__ bool any_not_finite(const uint4& u) {
  return (not_finite<T>(u.x) | not_finite<T>(u.y) | not_finite<T>(u.z) | not_finite<T>(u.w)) != 0;
}
template <class T>
__device__ __forceinline__ uint4 finite_part(const uint4& u) {
  return make_uint4(u.x & ~not_finite<T>(u.x), u.y & ~not_finite<T>(u.y), u.z & ~not_finite<T>(u.z),
                    u.w & ~not_finite<T>(u.w));
}
// 1 where the number is an infinity of this sign or a NaN, else 0
template <class T>
__device__ __forceinline__ uint32_t marks(uint32_t u, bool negative) {
  uint32_t m = 0;
#pragma unroll
  for (int i = 0; i < 2; ++i) {
    const uint32_t h = (u >> (16 * i)) & 0xffffu;
    const bool bad = (h & T::kExp) == T::kExp;
    const bool nan = bad && (h & 0x7fffu) != T::kExp;
    if (nan || (bad && ((h >> 15) != 0) == negative)) m |= (uint32_t)T::kOne << (16 * i);
  }
  return m;
}
template <class T>
__device__ __forceinline__ uint4 marks(const uint4& u, bool negative) {
  return make_uint4(marks<T>(u.x, negative), marks<T>(u.y, negative), marks<T>(u.z, negative), marks<T>(u.w, negative));
}
// what sums of marks under the queries that see the keys add to the output
__device__ __forceinline__ float marked(float plus, float minus) {
  const float inf = __builtin_inff();
  return (plus > 0.0f ? inf : 0.0f) + (minus > 0.0f ? -inf : 0.0f);
}

// ---------------------------------------------------------------------------
// tiles of 128 rows
// ---------------------------------------------------------------------------
// LDS holds 64 keys of K ([64][D]) and V^T ([D][64]) in 16 bits, twice: the next
// keys are loaded to registers while the present ones are multiplied.  16-byte
// chunks are stored at chunk ^ row, or at chunk ^ row/2 where two rows of 128 bytes
// share the 64 banks (V^T, and K of 64 elements), so that the 16-byte reads of a
// column of rows fall on different banks.
template <int D>
__device__ __forceinline__ int k_chunk(int row, int c) {
  return D == 64 ? row * 8 + (c ^ ((row >> 1) & 7)) : row * (D / 8) + (c ^ (row & 15));
}
__device__ __forceinline__ int v_chunk(int row, int c) { return row * 8 + (c ^ ((row >> 1) & 7)); }

template <class T, int D, bool kFp8>
__global__ __launch_bounds__(256, D == 256 ? 1 : 2) void k_attn_tile(AttnArgs a) {
  constexpr int BK = 64, C = D / 8;
  constexpr int kKeep = BK * C / 256;  // chunks of K (and of V^T) a thread moves
  extern __shared__ uint4 lds[];       // [2][K 64*C | V^T D*8]
  const uint32_t item = blockIdx.x / a.kv_heads, head = blockIdx.x % a.kv_heads;
  if ((int)item >= a.head->n_items) return;
  const PieceItem it = a.items[item];
  const int tid = threadIdx.x, lane = tid & 63, wave = wave_id();
  const int col = lane & 31, half = lane >> 5;
  const uint32_t G = a.group;

  // this lane's query
  const int row = it.row0 + 32 * wave + col;
  const int safe_row = min(row, it.row_end - 1);
  const int token = safe_row / (int)G, gh = safe_row - token * (int)G;
  const int qpos = it.ctx + token;
  const bool wave_on = it.row0 + 32 * wave < it.row_end;
  uint4 qf[D / 16];
  {
    const uint16_t* p = a.q + (int64_t)(it.q_start + token) * a.qt + (int64_t)(head * G + gh) * a.qh + 8 * half;
#pragma unroll
    for (int s = 0; s < D / 16; ++s) qf[s] = *(const uint4*)(p + 16 * s);
  }
  // positions of the wave's first and last queries
  const int first_pos = it.ctx + (it.row0 + 32 * wave) / (int)G;
  const int last_pos = it.ctx + (min(it.row0 + 32 * wave + 32, it.row_end) - 1) / (int)G;
  const int window = a.window ? (int)a.window : 0x40000000;
  const float k_scale = kFp8 && a.k_scale ? a.k_scale[head] : 1.0f;
  const float c = a.scale * kLog2e * k_scale;

  f32x16 o[D / 32];
#pragma unroll
  for (int i = 0; i < D / 32; ++i) o[i] = f32x16{};
  float m = -__builtin_inff(), l = 0.0f;

  const int32_t* table = a.table + (uint64_t)it.req * a.max_blocks;
  const int bs_mask = (1 << a.shift) - 1;
  constexpr int kBytes = kFp8 ? 1 : 2;
  const int64_t k_head = (int64_t)head * D * kBytes << a.shift;
  uint4 kr[kKeep], vr[kKeep];
  uint64_t next_valid = 0;

  // loads 64 keys from `key` on to registers; keys without a block read block 0
  auto fetch = [&](int key) {
    {
      const int kk = key + lane;
      int page = -1;
      if (kk < it.key_end) page = table[kk >> a.shift];
      next_valid = __ballot(page >= 0 && page < (int)a.n_blocks);
    }
#pragma unroll
    for (int i = 0; i < kKeep; ++i) {
      const int chunk = tid + 256 * i;
      const int r = chunk / C, cc = chunk % C;
      const int kk = min(key + r, it.key_end - 1);
      int page = table[kk >> a.shift];
      if (page < 0 || page >= (int)a.n_blocks) page = 0;
      const uint8_t* p = a.k + page * a.k_block * kBytes + k_head + ((int64_t)(kk & bs_mask) * D + cc * 8) * kBytes;
      if (kFp8) {
        const uint2 u = *(const uint2*)p;
        kr[i].x = u.x, kr[i].y = u.y;
      } else {
        kr[i] = *(const uint4*)p;
      }
    }
    {
      const int kk = key + 8 * (tid & 7);
      // a run of 8 keys that begins past the last one reads the last one's run
      const int k8 = min(kk, (it.key_end - 1) & ~7);
      int page = table[k8 >> a.shift];
      if (page < 0 || page >= (int)a.n_blocks) page = 0;
      const uint8_t* p = a.v + page * a.v_block * kBytes + k_head + (k8 & bs_mask) * kBytes;
#pragma unroll
      for (int i = 0; i < kKeep; ++i) {
        const int d = (tid >> 3) + 32 * i;
        const uint8_t* q = p + ((int64_t)d * kBytes << a.shift);
        if (kFp8) {
          const uint2 u = *(const uint2*)q;
          vr[i].x = u.x, vr[i].y = u.y;
        } else {
          vr[i] = *(const uint4*)q;
        }
      }
    }
  };
  auto store = [&](int buf) {
    uint4* lk = lds + buf * (BK * C + D * 8);
    uint4* lv = lk + BK * C;
#pragma unroll
    for (int i = 0; i < kKeep; ++i) {
      const int chunk = tid + 256 * i;
      const uint4 u = kFp8 ? widen8<T>(kr[i].x, kr[i].y) : kr[i];
      lk[k_chunk<D>(chunk / C, chunk % C)] = u;
      const uint4 w = kFp8 ? widen8<T>(vr[i].x, vr[i].y) : vr[i];
      lv[v_chunk((tid >> 3) + 32 * i, tid & 7)] = w;
    }
  };

  fetch(it.key_begin);
  uint64_t valid = next_valid;
  store(0);
  __syncthreads();
  int buf = 0;
  for (int key = it.key_begin; key < it.key_end; key += BK) {
    const bool more = key + BK < it.key_end;
    if (more) fetch(key + BK);
    if (wave_on && key <= last_pos && key + BK > first_pos - window + 1) {
      const uint4* lk = lds + buf * (BK * C + D * 8);
      const uint4* lv = lk + BK * C;
      // S^T: lane holds keys 32*n + 16*(b/2) + 8*half + 4*(b%2) + i at s[n][4*b + i]
      f32x16 s[2];
      const int krow = (col & 19) | ((col & 4) << 1) | ((col & 8) >> 1);
#pragma unroll
      for (int n = 0; n < 2; ++n) {
        s[n] = f32x16{};
#pragma unroll
        for (int d = 0; d < D / 16; ++d)
          s[n] = T::mfma32(lk[k_chunk<D>(32 * n + krow, 2 * d + half)], qf[d], s[n]);
      }
      const bool edge = key + BK - 1 > first_pos || key <= last_pos - window || ~valid;
      uint32_t seen = ~0u;  // bit 16*n + e: this lane's query sees the key of s[n][e]
      if (edge) {
        seen = 0;
#pragma unroll
        for (int n = 0; n < 2; ++n)
#pragma unroll
          for (int e = 0; e < 16; ++e) {
            const int at = 32 * n + 16 * (e >> 3) + 8 * half + (e & 7);
            const int kk = key + at;
            const bool ok = kk <= qpos && kk > qpos - window && ((valid >> at) & 1);
            if (ok)
              seen |= 1u << (16 * n + e);
            else
              s[n][e] = -__builtin_inff();
          }
      }
      float top = -__builtin_inff();
#pragma unroll
      for (int n = 0; n < 2; ++n)
#pragma unroll
        for (int e = 0; e < 16; ++e) top = fmaxf(top, s[n][e]);
      top = fmaxf(top, other_half(top)) * c;
      const float m_new = fmaxf(m, top);
      const float sub = m_new == -__builtin_inff() ? 0.0f : m_new;
      const float alpha = __builtin_amdgcn_exp2f(m - sub);
      m = m_new;
      float sum = 0.0f;
      uint4 p[4];
#pragma unroll
      for (int n = 0; n < 2; ++n) {
#pragma unroll
        for (int e = 0; e < 16; ++e) {
          s[n][e] = __builtin_amdgcn_exp2f(fmaf(s[n][e], c, -sub));
          sum += s[n][e];
        }
#pragma unroll
        for (int h = 0; h < 2; ++h)
          p[2 * n + h] = make_uint4(T::pack(s[n][8 * h], s[n][8 * h + 1]), T::pack(s[n][8 * h + 2], s[n][8 * h + 3]),
                                    T::pack(s[n][8 * h + 4], s[n][8 * h + 5]), T::pack(s[n][8 * h + 6], s[n][8 * h + 7]));
      }
      l = l * alpha + sum;
#pragma unroll
      for (int i = 0; i < D / 32; ++i)
#pragma unroll
        for (int e = 0; e < 16; ++e) o[i][e] *= alpha;
      bool bad = false;
      if (edge) {
#pragma unroll 1
        for (int i = 0; i < D / 32; ++i)
#pragma unroll
          for (int kb = 0; kb < 4; ++kb) bad |= any_not_finite<T>(lv[v_chunk(32 * i + col, 2 * kb + half)]);
        bad = __any(bad);
      }
      if (!bad) {
#pragma unroll
        for (int i = 0; i < D / 32; ++i)
#pragma unroll
          for (int kb = 0; kb < 4; ++kb) o[i] = T::mfma32(lv[v_chunk(32 * i + col, 2 * kb + half)], p[kb], o[i]);
      } else {
        uint4 sees[4];
#pragma unroll
        for (int kb = 0; kb < 4; ++kb) {
          uint32_t u[4];
#pragma unroll
          for (int j = 0; j < 4; ++j) {
            const uint32_t bits = seen >> (8 * kb + 2 * j);
            u[j] = (bits & 1 ? (uint32_t)T::kOne : 0u) | (bits & 2 ? (uint32_t)T::kOne << 16 : 0u);
          }
          sees[kb] = make_uint4(u[0], u[1], u[2], u[3]);
        }
#pragma unroll
        for (int i = 0; i < D / 32; ++i) {
          f32x16 plus{}, minus{};
#pragma unroll
          for (int kb = 0; kb < 4; ++kb) {
            const uint4 v = lv[v_chunk(32 * i + col, 2 * kb + half)];
            o[i] = T::mfma32(finite_part<T>(v), p[kb], o[i]);
            plus = T::mfma32(marks<T>(v, false), sees[kb], plus);
            minus = T::mfma32(marks<T>(v, true), sees[kb], minus);
          }
#pragma unroll
          for (int e = 0; e < 16; ++e) o[i][e] += marked(plus[e], minus[e]);
        }
      }
    }
    if (more) {
      store(buf ^ 1);
      valid = next_valid;
    }
    __syncthreads();
    buf ^= 1;
  }

  l += other_half(l);
  if (row >= it.row_end) return;
  if (it.part >= 0) {
    const int64_t at = ((int64_t)it.part * a.kv_heads + head) * 128 + 32 * wave + col;
    float* acc = a.acc + at * D;
#pragma unroll
    for (int i = 0; i < D / 32; ++i)
#pragma unroll
      for (int b = 0; b < 4; ++b)
        *(float4*)(acc + 32 * i + 8 * b + 4 * half) =
            make_float4(o[i][4 * b], o[i][4 * b + 1], o[i][4 * b + 2], o[i][4 * b + 3]);
    if (half == 0) *(float2*)(a.ml + at * 2) = make_float2(m, l);
    return;
  }
  const float v_scale = kFp8 && a.v_scale ? a.v_scale[head] : 1.0f;
  const float inv = l > 0.0f || l != l ? v_scale / l : 0.0f;
  uint16_t* op = a.out + (int64_t)(it.q_start + token) * a.ot + (int64_t)(head * G + gh) * a.oh;
#pragma unroll
  for (int i = 0; i < D / 32; ++i)
#pragma unroll
    for (int b = 0; b < 4; ++b)
      *(uint2*)(op + 32 * i + 8 * b + 4 * half) = make_uint2(T::pack(o[i][4 * b] * inv, o[i][4 * b + 1] * inv),
                                                             T::pack(o[i][4 * b + 2] * inv, o[i][4 * b + 3] * inv));
  if (a.lse && half == 0)
    a.lse[(int64_t)(it.q_start + token) * a.q_heads + head * G + gh] = (m + __builtin_amdgcn_logf(l)) * kLn2;
}

// ---------------------------------------------------------------------------
// up to 64 rows
// ---------------------------------------------------------------------------
// A wavefront takes every fourth run of kKeys keys: 32 of a 16-bit cache, 64 of an
// 8-bit one, so that a lane's loads are 16 bytes in both.  With 16x16x32 products
// a lane group g of 16 lanes holds 4 rows of S^T; the rows of K are
// permuted so that over the run's blocks these are the keys kPer*g .. kPer*g +
// kPer - 1 (kPer = 8 or 16), which is also its run of V^T.  At the end the four
// wavefronts' results are joined through LDS.
template <class T, int D, bool kFp8, int NC>
__global__ __launch_bounds__(256) void k_attn_rows(AttnArgs a) {
  constexpr int kPer = kFp8 ? 16 : 8, kKeys = 4 * kPer, kBlocks = kKeys / 16, kSteps = kKeys / 32;
  constexpr int kLoadsK = D / 4 / kPer;  // 16-byte loads of a key row by a lane
  const uint32_t item = blockIdx.x / a.kv_heads, head = blockIdx.x % a.kv_heads;
  if ((int)item >= a.head->n_items) return;
  const PieceItem it = a.items[item];
  const int tid = threadIdx.x, lane = tid & 63, wave = wave_id();
  const int col = lane & 15, g = lane >> 4;
  const uint32_t G = a.group;
  const int rows = it.row_end;  // row0 is 0: one tile a request

  // Queries: operand step s covers the elements that the lane's key loads hold:
  // load x = elements 4*kPer*x + kPer*g + 0 .. kPer-1
  int qpos[NC];
  uint4 qf[NC][D / 32];
#pragma unroll
  for (int n = 0; n < NC; ++n) {
    const int r = min(16 * n + col, rows - 1);
    const int token = r / (int)G, gh = r - token * (int)G;
    qpos[n] = it.ctx + token;
    const uint16_t* p = a.q + (int64_t)(it.q_start + token) * a.qt + (int64_t)(head * G + gh) * a.qh + kPer * g;
#pragma unroll
    for (int s = 0; s < D / 32; ++s) {
      constexpr int kSub = kPer / 8;
      qf[n][s] = *(const uint4*)(p + 4 * kPer * (s / kSub) + 8 * (s % kSub));
    }
  }
  const int window = a.window ? (int)a.window : 0x40000000;
  const int first_pos = it.ctx, last_pos = it.ctx + (rows - 1) / (int)G;
  const float k_scale = kFp8 && a.k_scale ? a.k_scale[head] : 1.0f;
  const float c = a.scale * kLog2e * k_scale;

  f32x4 o[NC][D / 16];
  float m[NC], l[NC];
#pragma unroll
  for (int n = 0; n < NC; ++n) {
    m[n] = -__builtin_inff();
    l[n] = 0.0f;
#pragma unroll
    for (int i = 0; i < D / 16; ++i) o[n][i] = f32x4{};
  }

  const int32_t* table = a.table + (uint64_t)it.req * a.max_blocks;
  const int bs_mask = (1 << a.shift) - 1;
  constexpr int kBytes = kFp8 ? 1 : 2;
  const int64_t k_head = (int64_t)head * D * kBytes << a.shift;
  const int last_run = (it.key_end - 1) & ~(kPer - 1);
  // this lane's keys: rows of K from run kPer * (col / 4), V^T's run kPer * g
  const int k_run = kPer * (col >> 2), v_run = kPer * g;

  for (int key = it.key_begin + kKeys * wave; key < it.key_end; key += 4 * kKeys) {
    const int kk = min(key + k_run, last_run), kv = min(key + v_run, last_run);
    int k_page = table[kk >> a.shift], v_page = table[kv >> a.shift];
    const bool k_ok = k_page >= 0 && k_page < (int)a.n_blocks, v_ok = v_page >= 0 && v_page < (int)a.n_blocks;
    if (!k_ok) k_page = 0;
    if (!v_ok) v_page = 0;
    const uint8_t* kp = a.k + k_page * a.k_block * kBytes + k_head + ((int64_t)((kk & bs_mask) + (col & 3)) * D + kPer * g) * kBytes;
    const uint8_t* vp = a.v + v_page * a.v_block * kBytes + k_head + ((int64_t)(col << a.shift) + (kv & bs_mask)) * kBytes;
    uint4 kf[kBlocks][kLoadsK], vf[D / 16];
#pragma unroll
    for (int b = 0; b < kBlocks; ++b)
#pragma unroll
      for (int x = 0; x < kLoadsK; ++x) kf[b][x] = *(const uint4*)(kp + 4 * b * D * kBytes + 4 * kPer * x * kBytes);
#pragma unroll
    for (int i = 0; i < D / 16; ++i) vf[i] = *(const uint4*)(vp + ((int64_t)(16 * i * kBytes) << a.shift));

    const bool edge = key + kKeys - 1 > first_pos || key <= last_pos - window || __any(!v_ok);
#pragma unroll
    for (int n = 0; n < NC; ++n) {
      // s[b][i]: key v_run + 4*b + i of the run, query 16*n + col
      f32x4 s[kBlocks];
#pragma unroll
      for (int b = 0; b < kBlocks; ++b) {
        s[b] = f32x4{};
#pragma unroll
        for (int x = 0; x < kLoadsK; ++x) {
          if (kFp8) {
            s[b] = T::mfma16(widen8<T>(kf[b][x].x, kf[b][x].y), qf[n][2 * x], s[b]);
            s[b] = T::mfma16(widen8<T>(kf[b][x].z, kf[b][x].w), qf[n][2 * x + 1], s[b]);
          } else {
            s[b] = T::mfma16(kf[b][x], qf[n][x], s[b]);
          }
        }
      }
      uint32_t seen = ~0u;  // bit 4*b + i
      if (edge) {
        seen = 0;
#pragma unroll
        for (int b = 0; b < kBlocks; ++b)
#pragma unroll
          for (int i = 0; i < 4; ++i) {
            const int at = key + v_run + 4 * b + i;
            const bool ok = v_ok && at <= qpos[n] && at > qpos[n] - window && at < it.key_end;
            if (ok)
              seen |= 1u << (4 * b + i);
            else
              s[b][i] = -__builtin_inff();
          }
      }
      float top = -__builtin_inff();
#pragma unroll
      for (int b = 0; b < kBlocks; ++b)
#pragma unroll
        for (int i = 0; i < 4; ++i) top = fmaxf(top, s[b][i]);
      top = fmaxf(top, __shfl_xor(top, 16, 64));
      top = fmaxf(top, other_half(top)) * c;
      const float m_new = fmaxf(m[n], top);
      const float sub = m_new == -__builtin_inff() ? 0.0f : m_new;
      const float alpha = __builtin_amdgcn_exp2f(m[n] - sub);
      m[n] = m_new;
      float sum = 0.0f;
#pragma unroll
      for (int b = 0; b < kBlocks; ++b)
#pragma unroll
        for (int i = 0; i < 4; ++i) {
          s[b][i] = __builtin_amdgcn_exp2f(fmaf(s[b][i], c, -sub));
          sum += s[b][i];
        }
      uint4 p[kSteps];
#pragma unroll
      for (int e = 0; e < kSteps; ++e)
        p[e] = make_uint4(T::pack(s[2 * e][0], s[2 * e][1]), T::pack(s[2 * e][2], s[2 * e][3]),
                          T::pack(s[2 * e + 1][0], s[2 * e + 1][1]), T::pack(s[2 * e + 1][2], s[2 * e + 1][3]));
      l[n] = l[n] * alpha + sum;
      bool bad = false;
      if (edge) {
#pragma unroll
        for (int i = 0; i < D / 16; ++i) {
          if (kFp8) {
            bad |= any_not_finite<T>(widen8<T>(vf[i].x, vf[i].y)) || any_not_finite<T>(widen8<T>(vf[i].z, vf[i].w));
          } else {
            bad |= any_not_finite<T>(vf[i]);
          }
        }
        bad = __any(bad);
      }
#pragma unroll
      for (int i = 0; i < D / 16; ++i) {
        uint4 v[kSteps];
        if (kFp8) {
          v[0] = widen8<T>(vf[i].x, vf[i].y);
          v[kSteps - 1] = widen8<T>(vf[i].z, vf[i].w);
        } else {
          v[0] = vf[i];
        }
#pragma unroll
        for (int e = 0; e < 4; ++e) o[n][i][e] *= alpha;
        if (!bad) {
#pragma unroll
          for (int e = 0; e < kSteps; ++e) o[n][i] = T::mfma16(v[e], p[e], o[n][i]);
        } else {
          f32x4 plus{}, minus{};
#pragma unroll
          for (int e = 0; e < kSteps; ++e) {
            uint32_t u[4];
#pragma unroll
            for (int j = 0; j < 4; ++j) {
              const uint32_t bits = seen >> (8 * e + 2 * j);
              u[j] = (bits & 1 ? (uint32_t)T::kOne : 0u) | (bits & 2 ? (uint32_t)T::kOne << 16 : 0u);
            }
            const uint4 sees = make_uint4(u[0], u[1], u[2], u[3]);
            o[n][i] = T::mfma16(finite_part<T>(v[e]), p[e], o[n][i]);
            plus = T::mfma16(marks<T>(v[e], false), sees, plus);
            minus = T::mfma16(marks<T>(v[e], true), sees, minus);
          }
#pragma unroll
          for (int e = 0; e < 4; ++e) o[n][i][e] += marked(plus[e], minus[e]);
        }
      }
    }
  }

  // join the wavefronts
  constexpr int kPad = D + 4;
  extern __shared__ float flds[];  // [4][16 * NC][kPad], then [4][16 * NC][2]
  float* stat = flds + 4 * 16 * NC * kPad;
#pragma unroll
  for (int n = 0; n < NC; ++n) {
    l[n] += __shfl_xor(l[n], 16, 64);
    l[n] += other_half(l[n]);
    const int at = wave * 16 * NC + 16 * n + col;
#pragma unroll
    for (int i = 0; i < D / 16; ++i) *(f32x4*)(flds + at * kPad + 16 * i + 4 * g) = o[n][i];
    if (g == 0) {
      stat[2 * at] = m[n];
      stat[2 * at + 1] = l[n];
    }
  }
  __syncthreads();
  const float v_scale = kFp8 && a.v_scale ? a.v_scale[head] : 1.0f;
  constexpr int kQuads = D / 4;
  for (int x = tid; x < rows * kQuads; x += 256) {
    const int r = x / kQuads, q = x % kQuads;
    float top = -__builtin_inff();
#pragma unroll
    for (int w = 0; w < 4; ++w) top = fmaxf(top, stat[2 * (w * 16 * NC + r)]);
    const float sub = top == -__builtin_inff() ? 0.0f : top;
    f32x4 sum{};
    float total = 0.0f;
#pragma unroll
    for (int w = 0; w < 4; ++w) {
      const int at = w * 16 * NC + r;
      const float f = __builtin_amdgcn_exp2f(stat[2 * at] - sub);
      const f32x4 v = *(const f32x4*)(flds + at * kPad + 4 * q);
      total = fmaf(f, stat[2 * at + 1], total);
#pragma unroll
      for (int e = 0; e < 4; ++e) sum[e] = fmaf(f, v[e], sum[e]);
    }
    if (it.part >= 0) {
      const int64_t at = ((int64_t)it.part * a.kv_heads + head) * (16 * NC) + r;
      *(f32x4*)(a.acc + at * D + 4 * q) = sum;
      if (q == 0) *(float2*)(a.ml + at * 2) = make_float2(top, total);
      continue;
    }
    const int token = r / (int)G, gh = r - token * (int)G;
    const float inv = total > 0.0f || total != total ? v_scale / total : 0.0f;
    *(uint2*)(a.out + (int64_t)(it.q_start + token) * a.ot + (int64_t)(head * G + gh) * a.oh + 4 * q) =
        make_uint2(T::pack(sum[0] * inv, sum[1] * inv), T::pack(sum[2] * inv, sum[3] * inv));
    if (a.lse && q == 0)
      a.lse[(int64_t)(it.q_start + token) * a.q_heads + head * G + gh] = (top + __builtin_amdgcn_logf(total)) * kLn2;
  }
}

// Joins the pieces of a tile: rows of one (tile, head) by blockIdx, 4 elements
// a thread.
template <class T>
__global__ __launch_bounds__(256) void k_attn_join(AttnArgs a, uint32_t tile_rows, uint32_t dim, uint32_t fp8) {
  const uint32_t tile = blockIdx.x / a.kv_heads, head = blockIdx.x % a.kv_heads;
  if ((int)tile >= a.head->n_split) return;
  const SplitTile t = a.split[tile];
  const uint32_t quads = dim / 4;
  const float v_scale = fp8 && a.v_scale ? a.v_scale[head] : 1.0f;
  const uint32_t rows = (uint32_t)min((int)tile_rows, t.row_end - t.row0);
  for (uint32_t x = blockIdx.y * 256 + threadIdx.x; x < rows * quads; x += gridDim.y * 256) {
    const uint32_t r = x / quads, q = x % quads;
    float top = -__builtin_inff();
    for (int i = 0; i < t.n_parts; ++i)
      top = fmaxf(top, a.ml[(((int64_t)(t.first_part + i) * a.kv_heads + head) * tile_rows + r) * 2]);
    const float sub = top == -__builtin_inff() ? 0.0f : top;
    f32x4 sum{};
    float total = 0.0f;
    for (int i = 0; i < t.n_parts; ++i) {
      const int64_t at = ((int64_t)(t.first_part + i) * a.kv_heads + head) * tile_rows + r;
      const float2 ml = *(const float2*)(a.ml + at * 2);
      const float f = __builtin_amdgcn_exp2f(ml.x - sub);
      const f32x4 v = *(const f32x4*)(a.acc + at * dim + 4 * q);
      total = fmaf(f, ml.y, total);
#pragma unroll
      for (int e = 0; e < 4; ++e) sum[e] = fmaf(f, v[e], sum[e]);
    }
    const int row = t.row0 + (int)r;
    const int token = row / (int)a.group, gh = row - token * (int)a.group;
    const float inv = total > 0.0f || total != total ? v_scale / total : 0.0f;
    *(uint2*)(a.out + (int64_t)(t.q_start + token) * a.ot + (int64_t)(head * a.group + gh) * a.oh + 4 * q) =
        make_uint2(T::pack(sum[0] * inv, sum[1] * inv), T::pack(sum[2] * inv, sum[3] * inv));
    if (a.lse && q == 0)
      a.lse[(int64_t)(t.q_start + token) * a.q_heads + head * a.group + gh] =
          (top + __builtin_amdgcn_logf(total)) * kLn2;
  }
}

template <class T, int D, bool kFp8>
kv_status launch_tile(const AttnArgs& a, uint32_t grid, hipStream_t s) {
  const size_t lds = 2 * (64 * D + D * 64) * 2;
  static const hipError_t ready = hipFuncSetAttribute((const void*)k_attn_tile<T, D, kFp8>,
                                                      hipFuncAttributeMaxDynamicSharedMemorySize, (int)lds);
  KV_HIP(ready);
  hipLaunchKernelGGL((k_attn_tile<T, D, kFp8>), dim3(grid), dim3(256), lds, s, a);
  KV_HIP(hipGetLastError());
  return KV_OK;
}

template <class T, int D, bool kFp8, int NC>
kv_status launch_rows(const AttnArgs& a, uint32_t grid, hipStream_t s) {
  const size_t lds = 4 * 16 * NC * (D + 4 + 2) * sizeof(float);
  static const hipError_t ready = hipFuncSetAttribute((const void*)k_attn_rows<T, D, kFp8, NC>,
                                                      hipFuncAttributeMaxDynamicSharedMemorySize, (int)lds);
  KV_HIP(ready);
  hipLaunchKernelGGL((k_attn_rows<T, D, kFp8, NC>), dim3(grid), dim3(256), lds, s, a);
  KV_HIP(hipGetLastError());
  return KV_OK;
}

template <class T, int D, bool kFp8>
kv_status launch_one(const AttnArgs& a, uint32_t rows, uint32_t grid, hipStream_t s) {
  switch (rows) {
    case 16: return launch_rows<T, D, kFp8, 1>(a, grid, s);
    case 32: return launch_rows<T, D, kFp8, 2>(a, grid, s);
    case 64:
      if constexpr (D <= 128) return launch_rows<T, D, kFp8, 4>(a, grid, s);
      [[fallthrough]];
    default: return launch_tile<T, D, kFp8>(a, grid, s);
  }
}

template <class T, bool kFp8>
kv_status launch_dim(const AttnArgs& a, uint32_t dim, uint32_t rows, uint32_t grid, hipStream_t s) {
  switch (dim) {
    case 64: return launch_one<T, 64, kFp8>(a, rows, grid, s);
    case 128: return launch_one<T, 128, kFp8>(a, rows, grid, s);
    default: return launch_one<T, 256, kFp8>(a, rows, grid, s);
  }
}

}  // namespace

kv_status paged_attention(const kv_paged_batch& b, const WorkLayout& w, const kv_paged_cache& c, uint32_t dtype,
                          const kv_heads_view& q, const kv_heads_view& out, float* lse, float scale, hipStream_t s) {
  AttnArgs a{};
  a.q = (const uint16_t*)q.ptr, a.out = (uint16_t*)out.ptr, a.lse = lse;
  a.qt = q.token_stride, a.qh = q.head_stride, a.ot = out.token_stride, a.oh = out.head_stride;
  a.k = (const uint8_t*)c.k, a.v = (const uint8_t*)c.v;
  a.k_block = c.k_block_stride, a.v_block = c.v_block_stride;
  a.k_scale = c.k_scale, a.v_scale = c.v_scale;
  a.table = b.table;
  const uint8_t* at = (const uint8_t*)b.work;
  a.head = (const WorkHeader*)at;
  a.items = (const PieceItem*)(at + w.items);
  a.split = (const SplitTile*)(at + w.split);
  a.acc = (float*)((uint8_t*)b.work + w.acc), a.ml = (float*)((uint8_t*)b.work + w.ml);
  a.scale = scale;
  a.max_tokens = b.max_tokens, a.max_blocks = b.max_blocks, a.n_blocks = c.n_blocks;
  a.kv_heads = b.kv_heads, a.q_heads = b.q_heads, a.group = w.group, a.window = b.window;
  a.shift = (uint32_t)__builtin_ctz(b.block_size);
  const uint64_t grid = (uint64_t)w.max_items * b.kv_heads;
  if (grid > 0x7fffffffull) return fail(KV_ERR_UNSUPPORTED, "kv_paged_attention: too many tiles for one call");
  const bool fp8 = c.dtype == KV_DT_FP8;
  kv_status st;
  if (dtype == KV_DT_BF16)
    st = fp8 ? launch_dim<BF16, true>(a, b.head_dim, w.rows, (uint32_t)grid, s)
             : launch_dim<BF16, false>(a, b.head_dim, w.rows, (uint32_t)grid, s);
  else
    st = fp8 ? launch_dim<F16, true>(a, b.head_dim, w.rows, (uint32_t)grid, s)
             : launch_dim<F16, false>(a, b.head_dim, w.rows, (uint32_t)grid, s);
  if (st != KV_OK) return st;
  // no tile can be cut when the whole table is at most one piece long
  if ((uint64_t)b.max_blocks * b.block_size <= kMinUnits * kKeyUnit) return KV_OK;
  const dim3 join(w.max_split * b.kv_heads, w.rows < 128 ? 1 : 4);
  if (dtype == KV_DT_BF16)
    hipLaunchKernelGGL(k_attn_join<BF16>, join, dim3(256), 0, s, a, w.rows, b.head_dim, (uint32_t)fp8);
  else
    hipLaunchKernelGGL(k_attn_join<F16>, join, dim3(256), 0, s, a, w.rows, b.head_dim, (uint32_t)fp8);
  KV_HIP(hipGetLastError());
  return KV_OK;
}

}  // namespace kv
