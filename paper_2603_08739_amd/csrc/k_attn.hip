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
//   k_attn_join   the pieces of tiles of 128 rows whose keys were cut
//
// A weight of 0 times a NaN or an infinity in a masked value would be NaN.  Where
// a tile holds masked keys, values are therefore looked at: non-finite ones are
// taken out of the product and added back only to the queries that see them.
#include <atomic>

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
  static constexpr float kLift = 0.0f;
  static constexpr uint32_t kExp = 0x7f80u;  // exponent bits: all set = not finite
  static __device__ __forceinline__ float value(uint16_t u) { return (float)__builtin_bit_cast(__bf16, u); }
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
  // Weights are up to 2^6 at the running maximum: their small ones, of 24 bits below
  // 1 in all, then lose less.
  static constexpr float kLift = 6.0f;
  static constexpr uint32_t kExp = 0x7c00u;
  static __device__ __forceinline__ float value(uint16_t u) { return (float)__builtin_bit_cast(_Float16, u); }
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
  uint64_t sizes;
  const WorkHeader* head;
  const PieceItem* items;
  const SplitTile* split;
  uint32_t* done;
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

// Masked values that are not finite (see the head of the file).  Bits 15 and 31:
// whether the halves' exponents are all ones (adding one at the exponent's lowest
// bit then carries into the sign's place).
template <class T>
__device__ __forceinline__ uint32_t not_finite(uint32_t u) {
  constexpr uint32_t kExp = T::kExp, kLow = kExp & (~kExp + 1);
  return ((u & (kExp | kExp << 16)) + (kLow | kLow << 16)) & 0x80008000u;
}
template <class T>
__device__ __forceinline__ uint32_t not_finite(const uint4& u) {
  return not_finite<T>(u.x) | not_finite<T>(u.y) | not_finite<T>(u.z) | not_finite<T>(u.w);
}
// 0 in the place of what is not finite
template <class T>
__device__ __forceinline__ uint32_t finite_part(uint32_t u) {
  const uint32_t m = not_finite<T>(u);
  return u & ~(m | (m - (m >> 15)));
}
template <class T>
__device__ __forceinline__ uint4 finite_part(const uint4& u) {
  return make_uint4(finite_part<T>(u.x), finite_part<T>(u.y), finite_part<T>(u.z), finite_part<T>(u.w));
}
// one value of the cache, unscaled
template <class T, bool kFp8>
__device__ __forceinline__ float element(const uint8_t* p) {
  return T::value(kFp8 ? (uint16_t)T::template widen<false>(*p) : *(const uint16_t*)p);
}

// ---------------------------------------------------------------------------
// tiles of 128 rows
// ---------------------------------------------------------------------------
// 64 keys at a time in LDS, twice: the next ones arrive by loads that go from
// memory straight to LDS while the present ones are multiplied, with one barrier
// between.  Wavefront w fetches keys 16w .. 16w + 15, which lie in one block, so the
// block's number is looked up once for the whole wavefront and a lane's offset
// never changes.  K is kept by rows of D elements, V^T in four groups of 16 keys
// by rows of 16 keys; both in the cache's type, 8-bit values are widened after
// they are read.  16-byte chunks are stored exclusive-ored with bits of their row,
// so that the reads of a column of rows fall on different banks (the loads place
// lanes in order, so the lane picks the chunk of memory that belongs there).
//
// One prompt of 8,111 tokens after 256 cached ones, 32 query and 8 key/value heads of
// 128, bf16: 573 GFLOP over the keys that queries see in 557 to 619 us (cards
// differ), 0.93 to 1.03 PFLOP/s where a large matrix product does 1.3 to 1.4; on a card
// that has rested before each call 630, under a kernel trace up to 690.  The matrix
// cores are busy half of the time: the exponentials, conversions and masks take
// vector instructions, of which two wavefronts on a SIMD hide a part only.  The same
// prompt over an 8-bit cache: 579 us beside 571.  Heads of 64: 885 TFLOP/s, 8 bits the
// same; half of the products for each exponential.  Heads of 256: 685, 8 bits 770; one
// wavefront on a SIMD has the registers, so that nothing hides its softmax.  What was
// tried beside it and was no faster: the next scores worked out between the steps of
// the softmax (599 us for 577), LDS reads issued a step ahead (740, registers spilled),
// wavefront priorities (the same).
template <int D, int kBytes>
struct TileLds {
  static constexpr int kRowChunks = D * kBytes / 16;              // of a row of K
  static constexpr int kChunks = 64 * kRowChunks;                 // of K, and of V^T
  static constexpr int kLoads = kChunks / 256;                    // a lane's
  static constexpr int kShift = kRowChunks >= 16 ? 0 : kRowChunks == 8 ? 1 : 2;  // rows that share the banks: 2^kShift
  static constexpr int kMask = kRowChunks >= 16 ? 15 : kRowChunks - 1;
  static __device__ __forceinline__ int k_swap(int row) { return (row >> kShift) & kMask; }
  static __device__ __forceinline__ int k_at(int row, int chunk) { return row * kRowChunks + (chunk ^ k_swap(row)); }
  // V^T, element row d of key group g: 16-bit rows are two chunks
  static __device__ __forceinline__ int v_swap(int d) { return kBytes == 2 ? (d >> 3) & 1 : 0; }
  static __device__ __forceinline__ int v_at(int g, int d, int chunk) {
    return kBytes == 2 ? (g * D + d) * 2 + (chunk ^ v_swap(d)) : g * D + d;
  }
};

__device__ __forceinline__ void load_to_lds(const uint8_t* from, uint4* to) {
  __builtin_amdgcn_global_load_lds((const __attribute__((address_space(1))) void*)from,
                                   (__attribute__((address_space(3))) void*)to, 16, 0, 0);
}

// A NaN wins: it stays out of the running maximum and reaches the sum as a weight.
__device__ __forceinline__ float max2(float a, float b) { return __builtin_elementwise_maximum(a, b); }
__device__ __forceinline__ float max3(float a, float b, float c) { return max2(max2(a, b), c); }

// Partial results pass between workgroups of one kernel, whose second-level caches
// may differ: stores that go through to where all of them look, loads that look there.
__device__ __forceinline__ void put_pair(float* p, float x, float y) {
  const float2 v = make_float2(x, y);
  __hip_atomic_store((uint64_t*)p, __builtin_bit_cast(uint64_t, v), __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
}
__device__ __forceinline__ float2 get_pair(const float* p) {
  return __builtin_bit_cast(float2, __hip_atomic_load((const uint64_t*)p, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT));
}

// Rescaling is put off until a maximum rises by more than this (base 2): weights
// then reach 2^8, in float16 2^14, which their 16-bit types hold with the same relative
// rounding.
constexpr float kSlack = 8.0f;
// Or until the weights of 32 keys sum to more than this: none overflows.
constexpr float kWeights = 16384.0f;

template <class T, int D, bool kFp8>
__global__ __launch_bounds__(256, D == 256 ? 1 : D == 128 ? 2 : 4) void k_attn_tile(AttnArgs a) {
  constexpr int BK = 64, kBytes = kFp8 ? 1 : 2;
  typedef TileLds<D, kBytes> L;
  __shared__ uint4 k_lds0[L::kChunks], k_lds1[L::kChunks], v_lds0[L::kChunks], v_lds1[L::kChunks];
  __shared__ int mend;
  const uint32_t item = blockIdx.x / a.kv_heads, head = blockIdx.x % a.kv_heads;
  const PieceItem it = a.items[item];  // loaded whether there is one or not: one wait for both
  if ((int)item >= a.head->n_items || a.head->sizes != a.sizes) return;
  const int tid = threadIdx.x, lane = tid & 63, wave = wave_id();
  const int col = lane & 31, half = lane >> 5;
  const uint32_t G = a.group;

  // this lane's query
  int end_lane = lane;
  asm volatile("" : "+v"(end_lane));
  const int row = min(it.row0 + 32 * wave + col, it.row_end - 1);
  const int qpos = it.ctx + row / (int)G;
  const bool wave_on = it.row0 + 32 * wave < it.row_end;
  // Operand step s of the first product: elements 16*s + 8*half + 0..7 of a 16-bit
  // cache; of an 8-bit one, whose 16-byte chunk serves two steps, 32*(s/2) + 16*half
  // + 8*(s%2) + 0..7
  uint4 qf[D / 16];
  {
    const int token = row / (int)G, gh = row - token * (int)G;
    const uint16_t* p = a.q + (int64_t)(it.q_start + token) * a.qt + (int64_t)(head * G + gh) * a.qh;
#pragma unroll
    for (int s = 0; s < D / 16; ++s)
      qf[s] = *(const uint4*)(p + (kFp8 ? 32 * (s / 2) + 16 * half + 8 * (s % 2) : 16 * s + 8 * half));
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
  const uint8_t* k_base = a.k + ((int64_t)head * D * kBytes << a.shift);
  const uint8_t* v_base = a.v + ((int64_t)head * D * kBytes << a.shift);
  // this lane's places in a group of 16 keys
  uint32_t k_from[L::kLoads], v_from[L::kLoads];
#pragma unroll
  for (int i = 0; i < L::kLoads; ++i) {
    const int x = 64 * i + lane;  // chunk of the group
    const int r = x / L::kRowChunks;
    k_from[i] = (uint32_t)(r * L::kRowChunks + ((x % L::kRowChunks) ^ L::k_swap(16 * wave + r))) * 16;
    const int d = kBytes == 2 ? x / 2 : x;
    v_from[i] = (uint32_t)((d * kBytes) << a.shift) + (kBytes == 2 ? (uint32_t)((x & 1) ^ L::v_swap(d)) * 16 : 0u);
  }
  // A tile's four groups have one block each: lane i looks up that of group i % 4,
  // two tiles ahead.  Groups past the last key read its group again, missing blocks
  // block 0.
  auto there = [&](int page) { return page >= 0 && page < (int)a.n_blocks; };
  auto look_up = [&](int key) { return table[min(key + 16 * (lane & 3), it.key_end - 1) >> a.shift]; };
  auto fetch = [&](int key, int pages, uint4* lk, uint4* lv) {
    const int k16 = min(key + 16 * wave, (it.key_end - 1) & ~15);
    int page = __builtin_amdgcn_readlane(pages, wave);
    if (!there(page)) page = 0;
    const uint8_t* kp = k_base + page * a.k_block * kBytes + (int64_t)(k16 & bs_mask) * D * kBytes;
    const uint8_t* vp = v_base + page * a.v_block * kBytes + (k16 & bs_mask) * kBytes;
#pragma unroll
    for (int i = 0; i < L::kLoads; ++i) load_to_lds(kp + k_from[i], lk + (wave * L::kLoads + i) * 64);
#pragma unroll
    for (int i = 0; i < L::kLoads; ++i) load_to_lds(vp + v_from[i], lv + (wave * L::kLoads + i) * 64);
  };

  // The lane's results e = 0..15 of the first product's block n are keys 32*n + 16*(e/8)
  // + 8*half + e%8 (8 bits: 32*n + 16*half + e); the row of K that gives them:
  const int krow = kFp8 ? ((col & 4) << 2) | ((col & 24) >> 1) | (col & 3) : (col & 19) | ((col & 4) << 1) | ((col & 8) >> 1);
  auto v_frag = [&](const uint4* lv, int i, int kb) {
    if (kFp8) {
      const uint4 u = lv[L::v_at((kb & ~1) + half, 32 * i + col, 0)];
      return kb & 1 ? widen8<T>(u.z, u.w) : widen8<T>(u.x, u.y);
    }
    return lv[L::v_at(kb, 32 * i + col, half)];
  };

  // Values that are not finite leave V^T before anyone multiplies by it, where some
  // query masks a key of the group; `mend` says that one belonged to a key that
  // some query sees (a block's unused end, say, may hold anything).
  const int tile_first = it.ctx + it.row0 / (int)G, tile_last = it.ctx + (min(it.row0 + 128, it.row_end) - 1) / (int)G;
  auto clean = [&](int key, uint32_t groups, uint4* lv) {
    const int k16 = key + 16 * wave;
    const bool here = (groups >> wave) & 1;
    if (here && k16 + 15 <= tile_first && k16 > tile_last - window && k16 + 15 < it.key_end) return;
    uint32_t any = 0;
#pragma unroll
    for (int i = 0; i < L::kLoads; ++i) {
      const uint4 u = lv[(wave * L::kLoads + i) * 64 + lane];
      any |= kFp8 ? not_finite<T>(widen8<T>(u.x, u.y)) | not_finite<T>(widen8<T>(u.z, u.w)) : not_finite<T>(u);
    }
    if (!__any(any != 0)) return;
    bool seen = false;
#pragma unroll 1
    for (int i = 0; i < L::kLoads * 16 / kBytes; ++i) {
      const int chunk = (wave * L::kLoads + i / (16 / kBytes)) * 64 + lane, j = i % (16 / kBytes);
      uint8_t* e = (uint8_t*)(lv + chunk) + j * kBytes;
      if (__builtin_isfinite(element<T, kFp8>(e))) continue;
      if (kFp8)
        *e = 0;
      else
        *(uint16_t*)e = 0;
      // chunk 2*d + (half of the group ^ swap), or one chunk for the whole group
      const int x = chunk - wave * L::kLoads * 64;
      const int at = k16 + (kBytes == 2 ? 8 * ((x & 1) ^ L::v_swap(x >> 1)) : 0) + j;
      seen |= here && at <= tile_last && at > tile_first - window && at < it.key_end;
    }
    if (__any(seen)) mend = 1;
  };

  int pages = look_up(it.key_begin), next_pages = look_up(it.key_begin + BK);
  uint32_t valid = 0;  // groups of 16 keys that are there
  auto arrive = [&](int key, uint4* lv, uint4* next_k, uint4* next_v) __attribute__((always_inline)) {
    valid = (uint32_t)__ballot(there(pages) && key + 16 * (lane & 3) < it.key_end) & 15u;
    // This wavefront's loads to LDS have arrived.  They are counted with the loads
    // from memory, which the barrier itself does not wait for.
    asm volatile("s_waitcnt vmcnt(0)" ::: "memory");
    if (key < it.key_end) clean(key, valid, lv);
    __syncthreads();  // everybody's have, and nobody reads the other keys any more
    if (key + BK < it.key_end) fetch(key + BK, next_pages, next_k, next_v);
    pages = next_pages;
    next_pages = look_up(key + 2 * BK);
  };
  auto active = [&](int key) {
    return wave_on && key < it.key_end && key <= last_pos && key + BK > first_pos - window + 1;
  };
  auto multiply = [&](int key, const uint4* lk, const uint4* lv) __attribute__((always_inline)) {
    const bool edge = key + BK - 1 > first_pos || key <= last_pos - window || valid != 15;
    // Weights are taken from the maximum of the keys seen when it was last looked for
    // (at first, and again when a weight has grown past kWeights: their sum, at
    // hand anyway, says so; the tile is then done again).  Their rounding is relative,
    // so that costs no accuracy, and the maximum of every tile, 16 instructions
    // and a wait across lanes, is saved: a prompt of 8,111 tokens 601 -> 580 us.  Heads of
    // 256 have no registers to spare for the way back and look at every tile.
    constexpr bool kLazy = D <= 128;
    f32x16 s[2];
    uint4 p[4];
    bool look = !kLazy || __any(m == -__builtin_inff());
    for (;;) {
#pragma unroll
      for (int n = 0; n < 2; ++n) {
        s[n] = f32x16{};
        if (kFp8) {
#pragma unroll
          for (int d = 0; d < D / 32; ++d) {
            const uint4 u = lk[L::k_at(32 * n + krow, 2 * d + half)];
            s[n] = T::mfma32(widen8<T>(u.x, u.y), qf[2 * d], s[n]);
            s[n] = T::mfma32(widen8<T>(u.z, u.w), qf[2 * d + 1], s[n]);
          }
        } else {
#pragma unroll
          for (int d = 0; d < D / 16; ++d) s[n] = T::mfma32(lk[L::k_at(32 * n + krow, 2 * d + half)], qf[d], s[n]);
        }
      }
      if (edge) {
        constexpr int kRun = kFp8 ? 16 : 8;
        const int from = key + kRun * half, most = qpos - from, least = qpos - window - from;
#pragma unroll
        for (int n = 0; n < 2; ++n)
#pragma unroll
          for (int e = 0; e < 16; ++e) {
            const int at = 32 * n + (kFp8 ? e : 16 * (e >> 3) + (e & 7));  // + kRun * half: the key
            const bool here = (valid >> (2 * n + (kFp8 ? half : e >> 3))) & 1;
            s[n][e] = (here & (at <= most) & (at > least)) ? s[n][e] : -__builtin_inff();
          }
      }
      if (look) {
        float top = s[0][0];
#pragma unroll
        for (int n = 0; n < 2; ++n)
#pragma unroll
          for (int e = 0; e < 16; e += 2) top = max3(top, s[n][e], s[n][e + 1]);
        top = fmaf(max2(top, other_half(top)), c, -T::kLift);
        if (kLazy || __any(top > m + kSlack)) {
          const float m_new = fmaxf(m, top);
          const float alpha = m_new == -__builtin_inff() ? 1.0f : __builtin_amdgcn_exp2f(m - m_new);
          m = m_new;
          l *= alpha;
#pragma unroll
          for (int i = 0; i < D / 32; ++i)
#pragma unroll
            for (int e = 0; e < 16; ++e) o[i][e] *= alpha;
        }
      }
      const float sub = m == -__builtin_inff() ? 0.0f : m;
      float sum[4] = {0.0f, 0.0f, 0.0f, 0.0f};
#pragma unroll
      for (int n = 0; n < 2; ++n) {
#pragma unroll
        for (int e = 0; e < 16; ++e) {
          s[n][e] = __builtin_amdgcn_exp2f(fmaf(s[n][e], c, -sub));
          sum[e & 3] += s[n][e];
        }
#pragma unroll
        for (int h = 0; h < 2; ++h)
          p[2 * n + h] = make_uint4(T::pack(s[n][8 * h], s[n][8 * h + 1]), T::pack(s[n][8 * h + 2], s[n][8 * h + 3]),
                                    T::pack(s[n][8 * h + 4], s[n][8 * h + 5]), T::pack(s[n][8 * h + 6], s[n][8 * h + 7]));
      }
      const float all = (sum[0] + sum[1]) + (sum[2] + sum[3]);
      if (!kLazy || look || !__any(!(all <= kWeights))) {
        l += all;
        break;
      }
      look = true;
      // Heads of 64: the keys are read again; kept for this, they would take the
      // registers of a fourth wavefront on each SIMD (a prompt 344 -> 330 us; heads of 128
      // gain no wavefront, and lose 1 % by it).
      if (D == 64) asm volatile("" ::: "memory");
    }
#pragma unroll
    for (int i = 0; i < D / 32; ++i)
#pragma unroll
      for (int kb = 0; kb < 4; ++kb) o[i] = T::mfma32(v_frag(lv, i, kb), p[kb], o[i]);
  };

  if (tid == 0) mend = 0;
  fetch(it.key_begin, pages, k_lds0, v_lds0);
  __syncthreads();  // mend
  // two tiles a turn: their places in LDS are known to the compiler, which waits for
  // loads to LDS before any read that they might concern
  for (int key = it.key_begin; key < it.key_end; key += 2 * BK) {
    arrive(key, v_lds0, k_lds1, v_lds1);
    if (active(key)) multiply(key, k_lds0, v_lds0);
    arrive(key + BK, v_lds1, k_lds0, v_lds0);
    if (active(key + BK)) multiply(key + BK, k_lds1, v_lds1);
  }
  // What was taken out, added to what has been stored for this lane's query (an
  // infinity or a NaN decides its element whatever the scale).
  auto add_bad = [&](auto add) {
#pragma unroll 1
    for (int key = max(it.key_begin, qpos - window + 1); key < it.key_end && key <= qpos; ++key) {
      const int page = table[key >> a.shift];
      if (!there(page)) continue;
      const uint8_t* vp = v_base + page * a.v_block * kBytes + (key & bs_mask) * kBytes;
#pragma unroll 1
      for (int x = 0; x < D / 2; ++x) {
        const int d = 8 * (x >> 2) + 4 * half + (x & 3);
        const float v = element<T, kFp8>(vp + ((int64_t)(d * kBytes) << a.shift));
        if (!__builtin_isfinite(v)) add(d, v);
      }
    }
  };

  __syncthreads();
  const bool mended = mend != 0;
  l += other_half(l);
  // the query again, from a copy of the lane: kept through the loop, its numbers would
  // take registers
  const int last_row = it.row0 + 32 * wave + (end_lane & 31);
  if (last_row >= it.row_end) return;
  const int token = last_row / (int)G, gh = last_row - token * (int)G;
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
    if (mended) add_bad([&](int d, float v) { acc[d] += v; });
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
  if (mended) add_bad([&](int d, float v) { op[d] = (uint16_t)T::pack(T::value(op[d]) + v, 0.0f); });
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
//
// 64 chats of up to 16,000 tokens, 32 query and 8 key/value heads of 128, bf16: 618 MB
// of keys and values in 116 us, 5.3 TB/s, where a large read does 6.2.  8 contexts of up
// to 131,071 tokens, 64 query heads, 8-bit cache: 768 MB in 146 us, 5.3 TB/s.  A
// wavefront keeps two runs of keys and values in flight; a third wavefront on each
// SIMD has not the registers for that (172 us for 116; 8 bits 150 for 146).  One context of 501
// tokens: 7.3 us a call, where an empty launch takes 4.
template <class T, int D, bool kFp8, int NC>
__global__ __launch_bounds__(256, D * NC <= 128 ? 2 : 1) void k_attn_rows(AttnArgs a) {
  constexpr int kPer = kFp8 ? 16 : 8, kKeys = 4 * kPer, kBlocks = kKeys / 16, kSteps = kKeys / 32;
  constexpr int kLoadsK = D / 4 / kPer;  // 16-byte loads of a key row by a lane
  const uint32_t item = blockIdx.x / a.kv_heads, head = blockIdx.x % a.kv_heads;
  const PieceItem it = a.items[item];  // loaded whether there is one or not: one wait for both
  if ((int)item >= a.head->n_items || a.head->sizes != a.sizes) return;
  const int tid = threadIdx.x, lane = tid & 63, wave = wave_id();
  const int col = lane & 15, g = lane >> 4;
  const uint32_t G = a.group;
  const int rows = it.row_end;  // row0 is 0: one tile a request

  const int32_t* table = a.table + (uint64_t)it.req * a.max_blocks;
  const int bs_mask = (1 << a.shift) - 1;
  constexpr int kBytes = kFp8 ? 1 : 2;
  const int64_t k_head = (int64_t)head * D * kBytes << a.shift;
  const int last_run = (it.key_end - 1) & ~(kPer - 1);
  // this lane's keys: rows of K from run kPer * (col / 4), V^T's run kPer * g
  const int k_run = kPer * (col >> 2), v_run = kPer * g;
  const int window = a.window ? (int)a.window : 0x40000000;
  const int first_pos = it.ctx, last_pos = it.ctx + (rows - 1) / (int)G;

  // Blocks are looked up two runs ahead, keys and values loaded one ahead: keys as
  // soon as the first product has taken the present ones, values after the second.
  struct Pages {
    int k, v;
  };
  auto there = [&](int page) { return page >= 0 && page < (int)a.n_blocks; };
  auto look_up = [&](int key) {
    Pages p;
    p.k = table[min(key + k_run, last_run) >> a.shift];
    p.v = table[min(key + v_run, last_run) >> a.shift];
    return p;
  };
  uint4 kf[kBlocks][kLoadsK], vf[D / 16];
  auto load_k = [&](int key, int page) {
    const int kk = min(key + k_run, last_run);
    const uint8_t* kp = a.k + (there(page) ? page : 0) * a.k_block * kBytes + k_head +
                        ((int64_t)((kk & bs_mask) + (col & 3)) * D + kPer * g) * kBytes;
#pragma unroll
    for (int b = 0; b < kBlocks; ++b)
#pragma unroll
      for (int x = 0; x < kLoadsK; ++x) kf[b][x] = *(const uint4*)(kp + 4 * b * D * kBytes + 4 * kPer * x * kBytes);
  };
  auto load_v = [&](int key, int page) {
    const int kk = min(key + v_run, last_run);
    const uint8_t* vp = a.v + (there(page) ? page : 0) * a.v_block * kBytes + k_head +
                        (((int64_t)col << a.shift) + (kk & bs_mask)) * kBytes;
    const int64_t stride = (int64_t)(16 * kBytes) << a.shift;
#pragma unroll
    for (int i = 0; i < D / 16; ++i) vf[i] = *(const uint4*)(vp + i * stride);
  };
  const int first = it.key_begin + kKeys * wave;
  Pages now{-1, -1}, next{-1, -1};
  if (first < it.key_end) {
    now = look_up(first);
    next = look_up(first + 4 * kKeys);
    load_k(first, now.k);
    load_v(first, now.v);
  }

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
  bool mend = false;

#pragma unroll 1
  for (int key = first; key < it.key_end; key += 4 * kKeys) {
    const bool more = key + 4 * kKeys < it.key_end;
    const bool v_ok = there(now.v);
    const bool edge = key + kKeys - 1 > first_pos || key <= last_pos - window || __any(!v_ok);
    // s[n][b][i]: key v_run + 4*b + i of the run, query 16*n + col
    f32x4 s[NC][kBlocks];
#pragma unroll
    for (int b = 0; b < kBlocks; ++b) {
#pragma unroll
      for (int n = 0; n < NC; ++n) s[n][b] = f32x4{};
#pragma unroll
      for (int x = 0; x < kLoadsK; ++x) {
        const uint4 lo = kFp8 ? widen8<T>(kf[b][x].x, kf[b][x].y) : kf[b][x];
#pragma unroll
        for (int n = 0; n < NC; ++n) s[n][b] = T::mfma16(lo, qf[n][kFp8 ? 2 * x : x], s[n][b]);
        if (kFp8) {
          const uint4 hi = widen8<T>(kf[b][x].z, kf[b][x].w);
#pragma unroll
          for (int n = 0; n < NC; ++n) s[n][b] = T::mfma16(hi, qf[n][(2 * x + 1) % (D / 32)], s[n][b]);
        }
      }
    }
    if (more) load_k(key + 4 * kKeys, next.k);
    uint4 p[NC][kSteps];
#pragma unroll
    for (int n = 0; n < NC; ++n) {
      if (edge) {
        const int from = key + v_run;
#pragma unroll
        for (int b = 0; b < kBlocks; ++b)
#pragma unroll
          for (int i = 0; i < 4; ++i) {
            const int at = 4 * b + i;
            const bool ok = v_ok && at <= qpos[n] - from && at > qpos[n] - window - from && at < it.key_end - from;
            s[n][b][i] = ok ? s[n][b][i] : -__builtin_inff();
          }
      }
      float top = s[n][0][0];
#pragma unroll
      for (int b = 0; b < kBlocks; ++b) {
        top = max3(top, s[n][b][0], s[n][b][1]);
        top = max3(top, s[n][b][2], s[n][b][3]);
      }
      top = max2(top, __shfl_xor(top, 16, 64));
      top = fmaf(max2(top, other_half(top)), c, -T::kLift);
      if (__any(top > m[n] + kSlack)) {
        const float m_new = fmaxf(m[n], top);
        const float alpha = m_new == -__builtin_inff() ? 1.0f : __builtin_amdgcn_exp2f(m[n] - m_new);
        m[n] = m_new;
        l[n] *= alpha;
#pragma unroll
        for (int i = 0; i < D / 16; ++i)
#pragma unroll
          for (int e = 0; e < 4; ++e) o[n][i][e] *= alpha;
      }
      const float sub = m[n] == -__builtin_inff() ? 0.0f : m[n];
#pragma unroll
      for (int b = 0; b < kBlocks; ++b)
#pragma unroll
        for (int i = 0; i < 4; ++i) s[n][b][i] = __builtin_amdgcn_exp2f(fmaf(s[n][b][i], c, -sub));
#pragma unroll
      for (int b = 0; b < kBlocks; ++b) l[n] += (s[n][b][0] + s[n][b][1]) + (s[n][b][2] + s[n][b][3]);
#pragma unroll
      for (int e = 0; e < kSteps; ++e)
        p[n][e] = make_uint4(T::pack(s[n][2 * e][0], s[n][2 * e][1]), T::pack(s[n][2 * e][2], s[n][2 * e][3]),
                             T::pack(s[n][2 * e + 1][0], s[n][2 * e + 1][1]), T::pack(s[n][2 * e + 1][2], s[n][2 * e + 1][3]));
    }
    uint32_t any = 0;
#pragma unroll
    for (int i = 0; i < D / 16; ++i)
#pragma unroll
      for (int e = 0; e < kSteps; ++e) {
        uint4 v = kFp8 ? e ? widen8<T>(vf[i].z, vf[i].w) : widen8<T>(vf[i].x, vf[i].y) : vf[i];
        if (edge) {
          any |= not_finite<T>(v);
          v = finite_part<T>(v);
        }
#pragma unroll
        for (int n = 0; n < NC; ++n) o[n][i] = T::mfma16(v, p[n][e], o[n][i]);
        if (NC > 1 && e == kSteps - 1) __builtin_amdgcn_sched_barrier(0);
      }
    // Of a key that some query sees?  (A block's unused end may hold anything; a
    // run that only begins among the seen is looked at again below.)
    if (edge) mend = mend || __any(any != 0 && v_ok && key + v_run <= last_pos && key + v_run + kPer > first_pos - window + 1);
    if (more) load_v(key + 4 * kKeys, next.v);
    now = next;
    if (key + 8 * kKeys < it.key_end) next = look_up(key + 8 * kKeys);
  }

  // join the wavefronts
  constexpr int kPad = D + 4;
  extern __shared__ float flds[];  // [4][16 * NC][kPad], then [4][16 * NC][2]
  __shared__ int mends[4];
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
  if (lane == 0) mends[wave] = mend;
  __syncthreads();
  mend = mends[0] | mends[1] | mends[2] | mends[3];
  const float v_scale = kFp8 && a.v_scale ? a.v_scale[head] : 1.0f;
  constexpr int kQuads = D / 4;
  auto put_row = [&](int r, int q, const f32x4& sum, float top, float total) {
    const int token = r / (int)G, gh = r - token * (int)G;
    const float inv = total > 0.0f || total != total ? v_scale / total : 0.0f;
    *(uint2*)(a.out + (int64_t)(it.q_start + token) * a.ot + (int64_t)(head * G + gh) * a.oh + 4 * q) =
        make_uint2(T::pack(sum[0] * inv, sum[1] * inv), T::pack(sum[2] * inv, sum[3] * inv));
    if (a.lse && q == 0)
      a.lse[(int64_t)(it.q_start + token) * a.q_heads + head * G + gh] = (top + __builtin_amdgcn_logf(total)) * kLn2;
  };
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
    if (mend) {  // values that are not finite, left out where keys were masked, to the queries that see them
      const int pos = it.ctx + r / (int)G;
#pragma unroll 1
      for (int key = max(it.key_begin, pos - window + 1); key < it.key_end && key <= pos; ++key) {
        const int page = table[key >> a.shift];
        if (!there(page)) continue;
        const uint8_t* vp = a.v + page * a.v_block * kBytes + k_head + (((int64_t)(4 * q) << a.shift) + (key & bs_mask)) * kBytes;
#pragma unroll
        for (int e = 0; e < 4; ++e) {
          const float v = element<T, kFp8>(vp + ((int64_t)(e * kBytes) << a.shift));
          if (!__builtin_isfinite(v)) sum[e] += v;
        }
      }
    }
    if (it.part >= 0) {
      const int64_t at = ((int64_t)it.part * a.kv_heads + head) * (16 * NC) + r;
      put_pair(a.acc + at * D + 4 * q, sum[0], sum[1]);
      put_pair(a.acc + at * D + 4 * q + 2, sum[2], sum[3]);
      if (q == 0) put_pair(a.ml + at * 2, top, total);
      continue;
    }
    put_row(r, q, sum, top, total);
  }
  if (it.part < 0) return;

  // The last of the tile's workgroups joins its pieces, in their order.
  __shared__ int last;
  // Every wavefront waits until its own stores, which went through, are done.  (A
  // release and an acquire fence for the device would do it for plain stores, but they
  // write back and invalidate whole caches: single tokens of 64 chats took 290 us
  // with them, 130 without.)
  asm volatile("s_waitcnt vmcnt(0)" ::: "memory");
  __syncthreads();
  uint32_t* done = a.done + (uint32_t)it.split * a.kv_heads + head;
  if (tid == 0) last = __hip_atomic_fetch_add(done, 1u, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT) == (uint32_t)it.n_parts - 1;
  __syncthreads();
  if (!last) return;
  if (tid == 0) __hip_atomic_store(done, 0u, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
  const int64_t step = (int64_t)a.kv_heads * 16 * NC;
  const int64_t part0 = ((int64_t)it.first_part * a.kv_heads + head) * (16 * NC);
  constexpr int kBatch = NC == 1 ? 8 : 2;  // pieces read at a time
  float2 lo[kBatch], hi[kBatch];
  auto read = [&](int x, int i) {
    const float* acc = a.acc + (part0 + x / kQuads) * D + 4 * (x % kQuads);
#pragma unroll
    for (int j = 0; j < kBatch; ++j) {
      const float* p = acc + min(i + j, it.n_parts - 1) * step * D;
      lo[j] = get_pair(p);
      hi[j] = get_pair(p + 2);
    }
  };
  if (tid < rows * kQuads) read(tid, 0);  // on its way while the weights are worked out
  // the pieces' weights, in the memory of the wavefronts' results
  float* weight = flds;                      // [rows][kMaxParts]
  float* sums = flds + 16 * NC * kMaxParts;  // [rows][2]
  for (int x = tid; x < rows * 8; x += 256) {  // 8 lanes a row
    const int r = x / 8, j = x % 8;
    float2 st[kMaxParts / 8];
#pragma unroll
    for (int i = 0; i < kMaxParts / 8; ++i)
      if (8 * i < it.n_parts) st[i] = get_pair(a.ml + (part0 + r + min(8 * i + j, it.n_parts - 1) * step) * 2);
    float top = -__builtin_inff(), total = 0.0f;
#pragma unroll
    for (int i = 0; i < kMaxParts / 8; ++i)
      if (8 * i + j < it.n_parts) top = fmaxf(top, st[i].x);
#pragma unroll
    for (int d = 1; d < 8; d <<= 1) top = fmaxf(top, __shfl_xor(top, d, 8));
    const float sub = top == -__builtin_inff() ? 0.0f : top;
#pragma unroll
    for (int i = 0; i < kMaxParts / 8; ++i)
      if (8 * i + j < it.n_parts) {
        const float f = __builtin_amdgcn_exp2f(st[i].x - sub);
        weight[r * kMaxParts + 8 * i + j] = f;
        total = fmaf(f, st[i].y, total);
      }
#pragma unroll
    for (int d = 1; d < 8; d <<= 1) total += __shfl_xor(total, d, 8);
    if (j == 0) sums[2 * r] = top, sums[2 * r + 1] = total;
  }
  __syncthreads();
  for (int x = tid; x < rows * kQuads; x += 256) {
    const int r = x / kQuads;
    f32x4 sum{};
#pragma unroll 1
    for (int i = 0; i < it.n_parts; i += kBatch) {
      if (x != tid || i > 0) read(x, i);
#pragma unroll
      for (int j = 0; j < kBatch; ++j) {
        if (i + j >= it.n_parts) break;
        const float f = weight[r * kMaxParts + i + j];
        sum[0] = fmaf(f, lo[j].x, sum[0]);
        sum[1] = fmaf(f, lo[j].y, sum[1]);
        sum[2] = fmaf(f, hi[j].x, sum[2]);
        sum[3] = fmaf(f, hi[j].y, sum[3]);
      }
    }
    put_row(r, x % kQuads, sum, sums[2 * r], sums[2 * r + 1]);
  }
}

// Joins the pieces of tiles of 128 rows, 4 elements a thread.  A row of a tile and
// head takes dim / 4 threads; workgroups walk over the rows of all cut tiles.  Bound by
// latency: 5 us after the prompt above, 7 after 12 ragged chunks of up to 1,300
// tokens.  (Joining in the last workgroup of a tile, as with few rows, would leave
// 128 rows to one workgroup.)
template <class T>
__global__ __launch_bounds__(256) void k_attn_join(AttnArgs a, uint32_t dim, uint32_t fp8) {
  const uint32_t quads = dim / 4, each = 256 / quads;  // rows of a workgroup
  const uint32_t q = threadIdx.x % quads, chunks = 128 / each;
  if (a.head->sizes != a.sizes) return;
  const uint32_t total = (uint32_t)a.head->n_split * a.kv_heads * chunks;
  for (uint32_t w = blockIdx.x; w < total; w += gridDim.x) {
    const uint32_t r = w % chunks * each + threadIdx.x / quads, head = w / chunks % a.kv_heads;
    const SplitTile t = a.split[w / chunks / a.kv_heads];
    const int row = t.row0 + (int)r;
    if (row >= t.row_end) continue;
    const int64_t step = (int64_t)a.kv_heads * 128, at = ((int64_t)t.first_part * a.kv_heads + head) * 128 + r;
    const float* ml = a.ml + at * 2;
    const float* acc = a.acc + at * dim + 4 * q;
    float top = -__builtin_inff(), total_l = 0.0f;
    for (int i = 0; i < t.n_parts; ++i) top = fmaxf(top, ml[i * step * 2]);
    const float sub = top == -__builtin_inff() ? 0.0f : top;
    f32x4 sum{};
#pragma unroll 4
    for (int i = 0; i < t.n_parts; ++i) {
      const float2 st = *(const float2*)(ml + i * step * 2);
      const f32x4 v = *(const f32x4*)(acc + i * step * dim);
      const float f = __builtin_amdgcn_exp2f(st.x - sub);
      total_l = fmaf(f, st.y, total_l);
#pragma unroll
      for (int e = 0; e < 4; ++e) sum[e] = fmaf(f, v[e], sum[e]);
    }
    const int token = row / (int)a.group, gh = row - token * (int)a.group;
    const float v_scale = fp8 && a.v_scale ? a.v_scale[head] : 1.0f;
    const float inv = total_l > 0.0f || total_l != total_l ? v_scale / total_l : 0.0f;
    *(uint2*)(a.out + (int64_t)(t.q_start + token) * a.ot + (int64_t)(head * a.group + gh) * a.oh + 4 * q) =
        make_uint2(T::pack(sum[0] * inv, sum[1] * inv), T::pack(sum[2] * inv, sum[3] * inv));
    if (a.lse && q == 0)
      a.lse[(int64_t)(t.q_start + token) * a.q_heads + head * a.group + gh] =
          (top + __builtin_amdgcn_logf(total_l)) * kLn2;
  }
}

template <class T, int D, bool kFp8>
kv_status launch_tile(const AttnArgs& a, uint32_t grid, hipStream_t s) {
  hipLaunchKernelGGL((k_attn_tile<T, D, kFp8>), dim3(grid), dim3(256), 0, s, a);
  KV_HIP(hipGetLastError());
  return KV_OK;
}

template <class T, int D, bool kFp8, int NC>
kv_status launch_rows(const AttnArgs& a, uint32_t grid, hipStream_t s) {
  const size_t lds = 4 * 16 * NC * (D + 4 + 2) * sizeof(float);
  if (lds > 64 * 1024) {  // has to be allowed, once on each device
    static std::atomic<uint64_t> allowed{0};
    int dev = 0;
    KV_HIP(hipGetDevice(&dev));
    const uint64_t bit = 1ull << (dev & 63);
    if (!(allowed.load(std::memory_order_relaxed) & bit)) {
      KV_HIP(hipFuncSetAttribute((const void*)k_attn_rows<T, D, kFp8, NC>, hipFuncAttributeMaxDynamicSharedMemorySize,
                                 (int)lds));
      allowed.fetch_or(bit, std::memory_order_relaxed);
    }
  }
  hipLaunchKernelGGL((k_attn_rows<T, D, kFp8, NC>), dim3(grid), dim3(256), lds, s, a);
  KV_HIP(hipGetLastError());
  return KV_OK;
}

template <class T, int D, bool kFp8>
kv_status launch_one(const AttnArgs& a, uint32_t rows, uint32_t grid, hipStream_t s) {
  switch (rows) {
    case 16: return launch_rows<T, D, kFp8, 1>(a, grid, s);
    case 32:
      if constexpr (D <= 128) return launch_rows<T, D, kFp8, 2>(a, grid, s);
      break;
    case 64:
      if constexpr (D <= 64) return launch_rows<T, D, kFp8, 4>(a, grid, s);
      break;
    default: break;
  }
  return launch_tile<T, D, kFp8>(a, grid, s);
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
  a.sizes = work_sizes(b);
  a.head = (const WorkHeader*)at;
  a.items = (const PieceItem*)(at + w.items);
  a.split = (const SplitTile*)(at + w.split);
  a.done = (uint32_t*)((uint8_t*)b.work + w.done);
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
  // tiles of few rows are joined already, and none is cut when the whole table is
  // at most one piece long
  if (w.rows < 128) return KV_OK;
  if ((uint64_t)b.max_blocks * b.block_size <= kMinUnits * kKeyUnit) return KV_OK;
  const dim3 join(std::min<uint32_t>(w.max_split * b.kv_heads * 4, 4096));
  if (dtype == KV_DT_BF16)
    hipLaunchKernelGGL(k_attn_join<BF16>, join, dim3(256), 0, s, a, b.head_dim, (uint32_t)fp8);
  else
    hipLaunchKernelGGL(k_attn_join<F16>, join, dim3(256), 0, s, a, b.head_dim, (uint32_t)fp8);
  KV_HIP(hipGetLastError());
  return KV_OK;
}

}  // namespace kv
