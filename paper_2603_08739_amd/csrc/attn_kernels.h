// attn_kernels.h - the attention kernels over a paged KV cache and their launches, for
// every kind of cache; k_attn.hip and k_attn_block.hip each build their own.
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
#pragma once

#include <atomic>
#include <type_traits>

#include "kv_device.h"
#include "kv_paged.h"

namespace kv {
namespace attn {

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
  // Two whole numbers of 8 bits.  Exact: 8 significant bits, so that a float's upper half
  // is all of it.
  template <bool kHigh>
  static __device__ __forceinline__ uint32_t widen_i8(uint32_t u) {
    const float a = (float)(int8_t)(u >> (kHigh ? 16 : 0)), b = (float)(int8_t)(u >> (kHigh ? 24 : 8));
    return __builtin_amdgcn_perm(__builtin_bit_cast(uint32_t, b), __builtin_bit_cast(uint32_t, a), 0x07060302u);
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
  // A byte n + 128 below the upper byte of 1024 is 1024 + n + 128.
  template <bool kHigh>
  static __device__ __forceinline__ uint32_t widen_i8(uint32_t u) {
    const uint32_t v = __builtin_amdgcn_perm(0x64646464u, u ^ 0x80808080u, kHigh ? 0x04030402u : 0x04010400u);
    const f16x2 off = {(_Float16)1152.0f, (_Float16)1152.0f};
    return __builtin_bit_cast(uint32_t, __builtin_bit_cast(f16x2, v) - off);
  }
};

// What a cache holds.  By head: one scale for a head's keys, one for its values; by
// block: for each block of tokens and head.
enum Kind { kSixteen, kFp8Head, kFp8Block, kI8Block };

// 8 numbers of 8 bits to 16 bits
template <class T, Kind kKind>
__device__ __forceinline__ uint4 widen8(uint32_t a, uint32_t b) {
  if constexpr (kKind == kI8Block)
    return make_uint4(T::template widen_i8<false>(a), T::template widen_i8<true>(a), T::template widen_i8<false>(b),
                      T::template widen_i8<true>(b));
  else
    return make_uint4(T::template widen<false>(a), T::template widen<true>(a), T::template widen<false>(b),
                      T::template widen<true>(b));
}

// The type of weights and values in the second product: the queries', but with scales by
// block float16 whatever that is.  Its weights are rounded to 11 bits, not 8 (64 chats of
// bfloat16: off by 0.0017 of the result, as rounding the result alone is, for 0.0024), and whole numbers
// take fewer instructions to widen to it; what is held is exact in both, and the
// scales, which could leave its range, are taken relative to the largest seen.
template <class T, Kind kKind>
struct Weights {
  typedef std::conditional_t<(kKind >= kFp8Block), F16, T> type;
};

// Two results in the queries' type.  What a cache with scales by block holds may be more than the
// values that were written, and near the end of float16's range more than it holds: results past
// the range are its largest number there (NaN stays NaN), not infinities that nobody wrote.
template <class T, bool kByBlock>
__device__ __forceinline__ uint32_t pack_result(float a, float b) {
  const uint32_t u = T::pack(a, b);
  if constexpr (kByBlock && std::is_same_v<T, F16>) {
    const f16x2 most = {(_Float16)65504.0f, (_Float16)65504.0f};
    return __builtin_bit_cast(uint32_t, __builtin_elementwise_minimum(__builtin_elementwise_maximum(__builtin_bit_cast(f16x2, u), -most), most));
  }
  return u;
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

// ---- scales by block ----
// A scale of 0 (nothing but zeros is held) must not meet the -inf of a masked score.
__device__ __forceinline__ float score_factor(float c, float k) { return fmaxf(c * k, 1.17549435e-38f); }
// Units are powers of two, known by their exponent bits; 0: none yet.
__device__ __forceinline__ float unit_value(uint32_t e) { return __builtin_bit_cast(float, e << 23); }
__device__ __forceinline__ float unit_ratio(uint32_t from, uint32_t to) {  // from < to
  return __builtin_amdgcn_ldexpf(1.0f, (int)from - (int)to);
}
// A scale in units: below 2.  What is smaller than 2^-60 of the largest adds nothing to a
// sum in 32 bits; its logarithm and reciprocal stay finite.
__device__ __forceinline__ float in_units(float v, uint32_t e) { return fmaxf(__builtin_amdgcn_ldexpf(v, 127 - (int)e), 0x1p-60f); }

// The largest of every four lanes.
__device__ __forceinline__ uint32_t most_of_four(uint32_t x) {
  x = max(x, (uint32_t)__builtin_amdgcn_mov_dpp((int)x, 0xb1, 0xf, 0xf, true));  // lane ^ 1
  return max(x, (uint32_t)__builtin_amdgcn_mov_dpp((int)x, 0x4e, 0xf, 0xf, true));  // lane ^ 2
}

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
template <class T, bool k8>
__device__ __forceinline__ float element(const uint8_t* p) {
  return T::value(k8 ? (uint16_t)T::template widen<false>(*p) : *(const uint16_t*)p);
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
// differ), 0.93 to 1.03 PFLOP/s where a large matrix product does 1.15 to 1.35 (8,192
// and 16,384 squared on one card); on a card that has rested before each call 630,
// under a kernel trace up to 690.  The matrix cores are busy half of the time: the
// exponentials, conversions and masks take vector instructions, of which two
// wavefronts on a SIMD hide a part only.  The same prompt over an 8-bit cache: 579 us
// beside 571.  Heads of 64: 885 TFLOP/s, 8 bits the
// same; half of the products for each exponential.  Heads of 256: 685, 8 bits 770; one
// wavefront on a SIMD has the registers, so that nothing hides its softmax.  What was
// tried beside it and was no faster: the next scores worked out between the steps of
// the softmax (599 us for 577), LDS reads issued a step ahead (740, registers spilled),
// wavefront priorities (the same).
//
// With scales by block, 7,777 tokens after 300, 32 query and 8 key/value heads of 128, bfloat16
// over whole numbers: 534 GFLOP in 581 to 620 us, 0.86 to 0.92 PFLOP/s; 5,003 after 2,000,
// float16 over e4m3 in blocks of 64: 369 GFLOP in 404 to 424 us, 0.87 to 0.91.  In turn on one
// card, calls that follow one another, the first prompt over e4m3 with scales by head takes 528
// us, by block 563, whole numbers 581 (heads of 64: 304, 348, 354; 16 and 4 heads of 256: 707, 742,
// 948).  A wavefront's tile takes 300 vector instructions beside its 32 products, 27 of them for
// the scales; whole numbers 270, of which 80 widen its share; 16 bits 150.  The matrix cores are
// busy 42 % of the time (16 bits 49).
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

template <class T, int D, Kind kKind>
__global__ __launch_bounds__(256, D == 256 ? 1 : D == 128 ? 2 : kKind >= kFp8Block ? 3 : 4) void k_attn_tile(AttnArgs a) {
  constexpr bool k8 = kKind != kSixteen, kByBlock = kKind >= kFp8Block;
  constexpr bool kFinite = kKind == kI8Block;  // nothing held is anything else
  typedef typename Weights<T, kKind>::type P;
  // Whole numbers are widened on the way into LDS.  Heads of 256 have no registers for numbers that
  // wait for it (256 and 204 are in use): every wavefront widens all of a tile, which is what they
  // take beyond e4m3 (948 us for 742, see above).
  constexpr bool kStage = kKind == kI8Block && D <= 128;
  constexpr bool kNarrow = k8 && !kStage;                 // 8 bits in LDS
  constexpr int BK = 64, kBytes = k8 ? 1 : 2;
  typedef TileLds<D, kNarrow ? 1 : 2> L;
  __shared__ uint4 k_lds0[L::kChunks], k_lds1[L::kChunks], v_lds0[L::kChunks], v_lds1[L::kChunks];
  __shared__ int mend;
  __shared__ float scales[kByBlock ? 2 : 1][kByBlock ? 4 : 1][kByBlock ? 4 : 1][4];
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
      qf[s] = *(const uint4*)(p + (kNarrow ? 32 * (s / 2) + 16 * half + 8 * (s % 2) : 16 * s + 8 * half));
  }
  // positions of the wave's first and last queries
  const int first_pos = it.ctx + (it.row0 + 32 * wave) / (int)G;
  const int last_pos = it.ctx + (min(it.row0 + 32 * wave + 32, it.row_end) - 1) / (int)G;
  const int window = a.window ? (int)a.window : 0x40000000;
  const float k_scale = kKind == kFp8Head && a.k_scale ? a.k_scale[head] : 1.0f;
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
  constexpr int kLoads = kStage ? L::kLoads / 2 : L::kLoads;
  uint32_t k_from[kLoads], v_from[kLoads];
#pragma unroll
  for (int i = 0; i < kLoads; ++i) {
    const int x = 64 * i + lane;  // chunk of the group
    if constexpr (kStage) {
      k_from[i] = (uint32_t)x * 16;
      v_from[i] = (uint32_t)x << a.shift;
      continue;
    }
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
  [[maybe_unused]] uint4 k_here[kStage ? kLoads : 1], v_here[kStage ? kLoads : 1];
  auto fetch = [&](int key, int pages, uint4* lk, uint4* lv) {
    const int k16 = min(key + 16 * wave, (it.key_end - 1) & ~15);
    int page = __builtin_amdgcn_readlane(pages, wave);
    if (!there(page)) page = 0;
    const uint8_t* kp = k_base + page * a.k_block * kBytes + (int64_t)(k16 & bs_mask) * D * kBytes;
    const uint8_t* vp = v_base + page * a.v_block * kBytes + (k16 & bs_mask) * kBytes;
    if constexpr (kStage) {
#pragma unroll
      for (int i = 0; i < kLoads; ++i) k_here[i] = *(const uint4*)(kp + k_from[i]), v_here[i] = *(const uint4*)(vp + v_from[i]);
      return;
    }
#pragma unroll
    for (int i = 0; i < kLoads; ++i) load_to_lds(kp + k_from[i], lk + (wave * kLoads + i) * 64);
#pragma unroll
    for (int i = 0; i < kLoads; ++i) load_to_lds(vp + v_from[i], lv + (wave * kLoads + i) * 64);
  };
  // Whole numbers take two or three instructions for two to widen, and every wavefront reads all
  // of the tile: they are widened once, by the one that has loaded them.  (With loads of 8 bytes
  // its writes to LDS would not meet on banks, but the prompt took 860 us for the 830 that it did
  // before this ran beside the products.)
  [[maybe_unused]] auto put = [&](uint4* lk, uint4* lv) {
    constexpr int kRow = D / 16;  // chunks of 16 numbers of a key
#pragma unroll
    for (int i = 0; i < kLoads; ++i) {
      const int x = 64 * i + lane, r = 16 * wave + x / kRow, ch = 2 * (x % kRow);
      lk[L::k_at(r, ch)] = widen8<T, kKind>(k_here[i].x, k_here[i].y);
      lk[L::k_at(r, ch + 1)] = widen8<T, kKind>(k_here[i].z, k_here[i].w);
      lv[L::v_at(wave, x, 0)] = widen8<P, kKind>(v_here[i].x, v_here[i].y);
      lv[L::v_at(wave, x, 1)] = widen8<P, kKind>(v_here[i].z, v_here[i].w);
    }
  };

  // The lane's results e = 0..15 of the first product's block n are keys 32*n + 16*(e/8)
  // + 8*half + e%8 (8 bits: 32*n + 16*half + e); the row of K that gives them:
  const int krow = kNarrow ? ((col & 4) << 2) | ((col & 24) >> 1) | (col & 3) : (col & 19) | ((col & 4) << 1) | ((col & 8) >> 1);
  auto v_frag = [&](const uint4* lv, int i, int kb) {
    if (kNarrow) {
      const uint4 u = lv[L::v_at((kb & ~1) + half, 32 * i + col, 0)];
      return kb & 1 ? widen8<P, kKind>(u.z, u.w) : widen8<P, kKind>(u.x, u.y);
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
      any |= k8 ? not_finite<T>(widen8<T, kKind>(u.x, u.y)) | not_finite<T>(widen8<T, kKind>(u.z, u.w)) : not_finite<T>(u);
    }
    if (!__any(any != 0)) return;
    bool seen = false;
#pragma unroll 1
    for (int i = 0; i < L::kLoads * 16 / kBytes; ++i) {
      const int chunk = (wave * L::kLoads + i / (16 / kBytes)) * 64 + lane, j = i % (16 / kBytes);
      uint8_t* e = (uint8_t*)(lv + chunk) + j * kBytes;
      if (__builtin_isfinite(element<T, k8>(e))) continue;
      if (k8)
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

  // Scales by block.  Scores take the keys' in the factor of their exponent.  Weights are
  // multiplied by the values' on their way into the second product, relative to a power of
  // two that follows the largest seen (o counts in units of it), so that they stay in the range of
  // 16 bits; in the exponent again, where it costs nothing, and the sum of weights undoes it.
  // Lane i loads the scales of group i % 4 two tiles ahead; a group that no row of the tile
  // sees has none.  What comes of them goes through LDS a tile ahead, in a place for each
  // wavefront: kept in registers over the products, they would be too many.
  [[maybe_unused]] float k_next = 0.0f, v_next = 0.0f;
  // groups that some row sees begin at least at `least` and at most at min(key_end - 1, tile_last)
  [[maybe_unused]] int seen_from = 0;
  [[maybe_unused]] uint32_t seen_many = 0;
  if constexpr (kByBlock) {
    const int least = max(tile_first - window - 14, 0);
    seen_from = 16 * (lane & 3) - least;
    seen_many = (uint32_t)max(min(it.key_end - 1, tile_last) - least + 1, 0);
  }
  [[maybe_unused]] uint32_t unit = 0, unit_now = 0, unit_here = 0;  // the power's exponent bits: of the tile to come, of the present one, of o
  [[maybe_unused]] auto load_scales = [&](int page) {
    const uint64_t from = (uint64_t)((uint32_t)page < a.n_blocks ? (uint32_t)page : 0u) * a.kv_heads + head;
    k_next = a.k_scale[from], v_next = a.v_scale[from];
  };
  [[maybe_unused]] auto take_scales = [&](int key, int page, int turn) {
    const bool seen = (uint32_t)page < a.n_blocks && (uint32_t)(key + seen_from) < seen_many;
    const float v = seen ? v_next : 0.0f;
    unit = max(unit, (uint32_t)__builtin_amdgcn_readfirstlane((int)(most_of_four(__builtin_bit_cast(uint32_t, v) & 0x7fffffffu) >> 23)));
    const float l2 = __builtin_amdgcn_logf(in_units(v, unit));
    if (lane < 4) *(float4*)scales[kByBlock ? turn : 0][kByBlock ? wave : 0][kByBlock ? lane : 0] = make_float4(score_factor(c, k_next), l2, __builtin_amdgcn_exp2f(-l2), 0.0f);
  };
  int pages = look_up(it.key_begin), next_pages = look_up(it.key_begin + BK);
  [[maybe_unused]] int third_pages = 0;
  uint32_t valid = 0;  // groups of 16 keys that are there
  auto arrive = [&](int key, [[maybe_unused]] int turn, uint4* lv, uint4* next_k, uint4* next_v) __attribute__((always_inline)) {
    valid = (uint32_t)__ballot(there(pages) && key + 16 * (lane & 3) < it.key_end) & 15u;
    // This wavefront's loads to LDS have arrived.  They are counted with the loads
    // from memory, which the barrier itself does not wait for.
    if constexpr (!kStage) asm volatile("s_waitcnt vmcnt(0)" ::: "memory");
    if constexpr (!kFinite)
      if (key < it.key_end) clean(key, valid, lv);
    __syncthreads();  // everybody's have, and nobody reads the other keys any more
    if constexpr (kByBlock) {
      unit_now = unit;
      take_scales(key + BK, next_pages, turn ^ 1);
    }
    if constexpr (!kStage)
      if (key + BK < it.key_end) fetch(key + BK, next_pages, next_k, next_v);
    if constexpr (kByBlock) {
      load_scales(third_pages);
      pages = next_pages;
      next_pages = third_pages;
      third_pages = look_up(key + 3 * BK);
    } else {
      pages = next_pages;
      next_pages = look_up(key + 2 * BK);
    }
  };
  // Numbers that are widened are loaded two tiles ahead.  They go into LDS while the present
  // tile's second products run.  (`pages` and `next_pages` are those of the next tiles by then.)
  [[maybe_unused]] auto stage = [&](int key, uint4* next_k, uint4* next_v) __attribute__((always_inline)) {
    // (also past the end, where the last keys are read again: with loads that may or may not
    // have been sent, the compiler waits for all of them where it needs an earlier one)
    put(next_k, next_v);
    fetch(key + 2 * BK, next_pages, nullptr, nullptr);
  };
  auto active = [&](int key) {
    return wave_on && key < it.key_end && key <= last_pos && key + BK > first_pos - window + 1;
  };
  auto multiply = [&](int key, [[maybe_unused]] int turn, const uint4* lk, const uint4* lv) __attribute__((always_inline)) {
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
    if constexpr (kByBlock)
      if (unit_here != unit_now) {
        const float less = unit_ratio(unit_here, unit_now);
        unit_here = unit_now;
#pragma unroll
        for (int i = 0; i < D / 32; ++i)
#pragma unroll
          for (int x = 0; x < 16; ++x) o[i][x] *= less;
      }
    // Of the groups that hold this lane's keys 8h .. 8h + 7 of blocks n: factor, logarithm and
    // what undoes it.
    constexpr int kGroups = kNarrow ? 1 : 2;  // of a block n
    [[maybe_unused]] float factor[2][kGroups], log2v[2][kGroups], undo[2][kGroups];
    if constexpr (kByBlock) {
#pragma unroll
      for (int n = 0; n < 2; ++n)
#pragma unroll
        for (int h = 0; h < kGroups; ++h) {
          const float4 f = *(const float4*)scales[turn][wave][2 * n + (kNarrow ? half : h)];
          factor[n][h] = f.x, log2v[n][h] = f.y, undo[n][h] = f.z;
        }
    }
    bool look = !kLazy || __any(m == -__builtin_inff());
    for (;;) {
      if constexpr (kNarrow && kByBlock && D <= 128) {
        // both blocks in turn, all of their keys read ahead
        uint4 ahead[2][D / 32];
#pragma unroll
        for (int d = 0; d < D / 32; ++d)
#pragma unroll
          for (int n = 0; n < 2; ++n) ahead[n][d] = lk[L::k_at(32 * n + krow, 2 * d + half)];
        __builtin_amdgcn_sched_barrier(0);
        s[0] = s[1] = f32x16{};
#pragma unroll
        for (int d = 0; d < D / 32; ++d) {
#pragma unroll
          for (int n = 0; n < 2; ++n) s[n] = T::mfma32(widen8<T, kKind>(ahead[n][d].x, ahead[n][d].y), qf[2 * d], s[n]);
#pragma unroll
          for (int n = 0; n < 2; ++n) s[n] = T::mfma32(widen8<T, kKind>(ahead[n][d].z, ahead[n][d].w), qf[2 * d + 1], s[n]);
        }
      } else if constexpr (kStage) {
        // Both blocks in turn, their keys read a step ahead.  (Left to the compiler, which has not the
        // registers to read all of them ahead as in 16 bits, each product waited for its own.)
        uint4 ahead[2][2];
#pragma unroll
        for (int n = 0; n < 2; ++n) {
          s[n] = f32x16{};
          ahead[0][n] = lk[L::k_at(32 * n + krow, half)];
        }
#pragma unroll
        for (int d = 0; d < D / 16; ++d) {
          if (d + 1 < D / 16)
#pragma unroll
            for (int n = 0; n < 2; ++n) ahead[(d + 1) & 1][n] = lk[L::k_at(32 * n + krow, 2 * (d + 1) + half)];
#pragma unroll
          for (int n = 0; n < 2; ++n) s[n] = T::mfma32(ahead[d & 1][n], qf[d], s[n]);
          __builtin_amdgcn_sched_barrier(0);
        }
      }
#pragma unroll
      for (int n = 0; n < (kByBlock && D <= 128 ? 0 : 2); ++n) {
        s[n] = f32x16{};
        if (kNarrow) {
#pragma unroll
          for (int d = 0; d < D / 32; ++d) {
            const uint4 u = lk[L::k_at(32 * n + krow, 2 * d + half)];
            s[n] = T::mfma32(widen8<T, kKind>(u.x, u.y), qf[2 * d], s[n]);
            s[n] = T::mfma32(widen8<T, kKind>(u.z, u.w), qf[2 * d + 1], s[n]);
          }
        } else {
#pragma unroll
          for (int d = 0; d < D / 16; ++d) s[n] = T::mfma32(lk[L::k_at(32 * n + krow, 2 * d + half)], qf[d], s[n]);
        }
      }
      if (edge) {
        constexpr int kRun = kNarrow ? 16 : 8;
        const int from = key + kRun * half;
        int most = qpos - from, least = qpos - window - from;
        // (worked out ahead of this loop, the masks would take more scalar registers than there are)
        if constexpr (kByBlock) asm volatile("" : "+v"(most), "+v"(least));
#pragma unroll
        for (int n = 0; n < 2; ++n)
#pragma unroll
          for (int e = 0; e < 16; ++e) {
            const int at = 32 * n + (kNarrow ? e : 16 * (e >> 3) + (e & 7));  // + kRun * half: the key
            const bool here = (valid >> (2 * n + (kNarrow ? half : e >> 3))) & 1;
            s[n][e] = (here & (at <= most) & (at > least)) ? s[n][e] : -__builtin_inff();
          }
      }
      if (look) {
        float top = s[0][0];
        if constexpr (kByBlock) {
          top = -__builtin_inff();
#pragma unroll
          for (int n = 0; n < 2; ++n)
#pragma unroll
            for (int h = 0; h < kGroups; ++h) {
              float most = s[n][8 * h];
#pragma unroll
              for (int e = 0; e < (kNarrow ? 16 : 8); e += 2) most = max3(most, s[n][8 * h + e], s[n][8 * h + e + 1]);
              top = max2(top, most * factor[n][h]);
            }
          top = max2(top, other_half(top)) - P::kLift;
        } else {
#pragma unroll
          for (int n = 0; n < 2; ++n)
#pragma unroll
            for (int e = 0; e < 16; e += 2) top = max3(top, s[n][e], s[n][e + 1]);
          top = fmaf(max2(top, other_half(top)), c, -P::kLift);
        }
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
        float from = -sub, by = c;
        if constexpr (kByBlock) from = log2v[n][0] - sub, by = factor[n][0];
#pragma unroll
        for (int e = 0; e < 16; ++e) {
          if constexpr (kByBlock && !kNarrow)
            if (e == 8) from = log2v[n][1] - sub, by = factor[n][1];
          s[n][e] = __builtin_amdgcn_exp2f(fmaf(s[n][e], by, from));
          sum[!kByBlock ? e & 3 : kNarrow ? 2 * n + (e & 1) : 2 * n + (e >> 3)] += s[n][e];
        }
#pragma unroll
        for (int h = 0; h < 2; ++h)
          p[2 * n + h] = make_uint4(P::pack(s[n][8 * h], s[n][8 * h + 1]), P::pack(s[n][8 * h + 2], s[n][8 * h + 3]),
                                    P::pack(s[n][8 * h + 4], s[n][8 * h + 5]), P::pack(s[n][8 * h + 6], s[n][8 * h + 7]));
      }
      float all = (sum[0] + sum[1]) + (sum[2] + sum[3]);
      if constexpr (kByBlock && kNarrow) {
        all = fmaf(sum[2] + sum[3], undo[1][0], (sum[0] + sum[1]) * undo[0][0]);
      } else if constexpr (kByBlock) {
        all = sum[0] * undo[0][0];
#pragma unroll
        for (int x = 1; x < 4; ++x) all = fmaf(sum[x], undo[x >> 1][x & 1], all);
      }
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
      for (int kb = 0; kb < 4; ++kb) o[i] = P::mfma32(v_frag(lv, i, kb), p[kb], o[i]);
  };

  if (tid == 0) mend = 0;
  fetch(it.key_begin, pages, k_lds0, v_lds0);
  if constexpr (kByBlock) {
    load_scales(pages);
    if constexpr (kStage) put(k_lds0, v_lds0);
    take_scales(it.key_begin, pages, 0);
    // in the order in which the loop sends them: it waits for some of them only
    load_scales(next_pages);
    third_pages = look_up(it.key_begin + 2 * BK);
    if constexpr (kStage) fetch(it.key_begin + BK, next_pages, nullptr, nullptr);
  }
  __syncthreads();  // mend
  // two tiles a turn: their places in LDS are known to the compiler, which waits for
  // loads to LDS before any read that they might concern
  for (int key = it.key_begin; key < it.key_end; key += 2 * BK) {
    arrive(key, 0, v_lds0, k_lds1, v_lds1);
    if constexpr (kStage) stage(key, k_lds1, v_lds1);
    if (active(key)) multiply(key, 0, k_lds0, v_lds0);
    arrive(key + BK, 1, v_lds1, k_lds0, v_lds0);
    if constexpr (kStage) stage(key + BK, k_lds0, v_lds0);
    if (active(key + BK)) multiply(key + BK, 1, k_lds1, v_lds1);
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
        const float v = element<T, k8>(vp + ((int64_t)(d * kBytes) << a.shift));
        if (!__builtin_isfinite(v)) add(d, v);
      }
    }
  };

  __syncthreads();
  const bool mended = !kFinite && mend != 0;
  l += other_half(l);
  if constexpr (kByBlock) {
    const float one = unit_value(unit_here);
#pragma unroll
    for (int i = 0; i < D / 32; ++i)
#pragma unroll
      for (int e = 0; e < 16; ++e) o[i][e] *= one;
  }
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
  const float v_scale = kKind == kFp8Head && a.v_scale ? a.v_scale[head] : 1.0f;
  const float inv = l > 0.0f || l != l ? v_scale / l : 0.0f;
  uint16_t* op = a.out + (int64_t)(it.q_start + token) * a.ot + (int64_t)(head * G + gh) * a.oh;
#pragma unroll
  for (int i = 0; i < D / 32; ++i)
#pragma unroll
    for (int b = 0; b < 4; ++b)
      *(uint2*)(op + 32 * i + 8 * b + 4 * half) = make_uint2(pack_result<T, kByBlock>(o[i][4 * b] * inv, o[i][4 * b + 1] * inv),
                                                             pack_result<T, kByBlock>(o[i][4 * b + 2] * inv, o[i][4 * b + 3] * inv));
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
//
// With scales by block, 64 chats over up to 15,930 tokens, whole numbers: 417 MB in 84 us, 4.95
// TB/s; 8 contexts of up to 98,866, 64 query heads, e4m3: 627 MB in 120 us, 5.2 TB/s; the
// same with scales by head takes as long (131 us for 130 from cold caches).  Loads that
// go past the caches are not taken: 81 and 115 us, but 8 requests over one prefix of 60,000 tokens,
// whose blocks they share, 133 for 107.
template <class T, int D, Kind kKind, int NC>
__global__ __launch_bounds__(256, D * NC <= 128 ? 2 : 1) void k_attn_rows(AttnArgs a) {
  constexpr bool k8 = kKind != kSixteen, kByBlock = kKind >= kFp8Block;
  constexpr bool kFinite = kKind == kI8Block;  // nothing held is anything else
  typedef typename Weights<T, kKind>::type P;
  constexpr int kPer = k8 ? 16 : 8, kKeys = 4 * kPer, kBlocks = kKeys / 16, kSteps = kKeys / 32;
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
  constexpr int kBytes = k8 ? 1 : 2;
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
  // Scales by block of the run of V^T, whose keys are also those of the lane's scores: used
  // as in k_attn_tile.
  float k_by = 0.0f, v_by = 0.0f;
  uint32_t unit = 0;
  auto load_scales = [&](int page) {
    const uint64_t from = (uint64_t)((uint32_t)page < a.n_blocks ? (uint32_t)page : 0u) * a.kv_heads + head;
    k_by = a.k_scale[from], v_by = a.v_scale[from];
  };
  const int first = it.key_begin + kKeys * wave;
  Pages now{-1, -1}, next{-1, -1};
  if (first < it.key_end) {
    now = look_up(first);
    next = look_up(first + 4 * kKeys);
    load_k(first, now.k);
    if constexpr (kByBlock) load_scales(now.v);  // ahead of the values, which are waited for later
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
  const float k_scale = kKind == kFp8Head && a.k_scale ? a.k_scale[head] : 1.0f;
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
        const uint4 lo = k8 ? widen8<T, kKind>(kf[b][x].x, kf[b][x].y) : kf[b][x];
#pragma unroll
        for (int n = 0; n < NC; ++n) s[n][b] = T::mfma16(lo, qf[n][k8 ? 2 * x : x], s[n][b]);
        if (k8) {
          const uint4 hi = widen8<T, kKind>(kf[b][x].z, kf[b][x].w);
#pragma unroll
          for (int n = 0; n < NC; ++n) s[n][b] = T::mfma16(hi, qf[n][(2 * x + 1) % (D / 32)], s[n][b]);
        }
      }
    }
    if (more) load_k(key + 4 * kKeys, next.k);
    float cv = c, from = 0.0f, undo = 1.0f;
    if constexpr (kByBlock) {
      const bool seen = v_ok && key + v_run < it.key_end && key + v_run <= last_pos && key + v_run + kPer > first_pos - window + 1;
      const float v = seen ? v_by : 0.0f;
      float most = fabsf(v);
      most = fmaxf(most, __shfl_xor(most, 16, 64));
      most = fmaxf(most, other_half(most));
      const uint32_t e = __builtin_amdgcn_readfirstlane(__builtin_bit_cast(int, most)) >> 23;
      if (e > unit) {
        const float less = unit_ratio(unit, e);
        unit = e;
#pragma unroll
        for (int n = 0; n < NC; ++n)
#pragma unroll
          for (int i = 0; i < D / 16; ++i)
#pragma unroll
            for (int x = 0; x < 4; ++x) o[n][i][x] *= less;
      }
      cv = score_factor(c, k_by);
      from = __builtin_amdgcn_logf(in_units(v, unit));
      undo = __builtin_amdgcn_exp2f(-from);
    }
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
      if constexpr (kByBlock) top *= cv;
      top = max2(top, __shfl_xor(top, 16, 64));
      top = kByBlock ? max2(top, other_half(top)) - P::kLift : fmaf(max2(top, other_half(top)), c, -P::kLift);
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
        for (int i = 0; i < 4; ++i) s[n][b][i] = __builtin_amdgcn_exp2f(fmaf(s[n][b][i], cv, kByBlock ? from - sub : -sub));
      if constexpr (kByBlock) {
        float all = 0.0f;
#pragma unroll
        for (int b = 0; b < kBlocks; ++b) all += (s[n][b][0] + s[n][b][1]) + (s[n][b][2] + s[n][b][3]);
        l[n] = fmaf(all, undo, l[n]);
      } else {
#pragma unroll
        for (int b = 0; b < kBlocks; ++b) l[n] += (s[n][b][0] + s[n][b][1]) + (s[n][b][2] + s[n][b][3]);
      }
#pragma unroll
      for (int e = 0; e < kSteps; ++e)
        p[n][e] = make_uint4(P::pack(s[n][2 * e][0], s[n][2 * e][1]), P::pack(s[n][2 * e][2], s[n][2 * e][3]),
                             P::pack(s[n][2 * e + 1][0], s[n][2 * e + 1][1]), P::pack(s[n][2 * e + 1][2], s[n][2 * e + 1][3]));
    }
    uint32_t any = 0;
#pragma unroll
    for (int i = 0; i < D / 16; ++i)
#pragma unroll
      for (int e = 0; e < kSteps; ++e) {
        uint4 v = k8 ? e ? widen8<P, kKind>(vf[i].z, vf[i].w) : widen8<P, kKind>(vf[i].x, vf[i].y) : vf[i];
        if (!kFinite && edge) {
          any |= not_finite<P>(v);
          v = finite_part<P>(v);
        }
#pragma unroll
        for (int n = 0; n < NC; ++n) o[n][i] = P::mfma16(v, p[n][e], o[n][i]);
        if (NC > 1 && e == kSteps - 1) __builtin_amdgcn_sched_barrier(0);
      }
    // Of a key that some query sees?  (A block's unused end may hold anything; a
    // run that only begins among the seen is looked at again below.)
    if (!kFinite && edge) mend = mend || __any(any != 0 && v_ok && key + v_run <= last_pos && key + v_run + kPer > first_pos - window + 1);
    if constexpr (kByBlock)
      if (more) load_scales(next.v);
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
    if constexpr (kByBlock) {
      const float one = unit_value(unit);
#pragma unroll
      for (int i = 0; i < D / 16; ++i)
#pragma unroll
        for (int x = 0; x < 4; ++x) o[n][i][x] *= one;
    }
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
  const float v_scale = kKind == kFp8Head && a.v_scale ? a.v_scale[head] : 1.0f;
  constexpr int kQuads = D / 4;
  auto put_row = [&](int r, int q, const f32x4& sum, float top, float total) {
    const int token = r / (int)G, gh = r - token * (int)G;
    const float inv = total > 0.0f || total != total ? v_scale / total : 0.0f;
    *(uint2*)(a.out + (int64_t)(it.q_start + token) * a.ot + (int64_t)(head * G + gh) * a.oh + 4 * q) =
        make_uint2(pack_result<T, kByBlock>(sum[0] * inv, sum[1] * inv), pack_result<T, kByBlock>(sum[2] * inv, sum[3] * inv));
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
          const float v = element<T, k8>(vp + ((int64_t)(e * kBytes) << a.shift));
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
template <class T, bool kByBlock>
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
        make_uint2(pack_result<T, kByBlock>(sum[0] * inv, sum[1] * inv), pack_result<T, kByBlock>(sum[2] * inv, sum[3] * inv));
    if (a.lse && q == 0)
      a.lse[(int64_t)(t.q_start + token) * a.q_heads + head * a.group + gh] =
          (top + __builtin_amdgcn_logf(total_l)) * kLn2;
  }
}

template <class T, int D, Kind kKind>
kv_status launch_tile(const AttnArgs& a, uint32_t grid, hipStream_t s) {
  hipLaunchKernelGGL((k_attn_tile<T, D, kKind>), dim3(grid), dim3(256), 0, s, a);
  KV_HIP(hipGetLastError());
  return KV_OK;
}

template <class T, int D, Kind kKind, int NC>
kv_status launch_rows(const AttnArgs& a, uint32_t grid, hipStream_t s) {
  const size_t lds = 4 * 16 * NC * (D + 4 + 2) * sizeof(float);
  if (lds > 64 * 1024) {  // has to be allowed, once on each device
    static std::atomic<uint64_t> allowed{0};
    int dev = 0;
    KV_HIP(hipGetDevice(&dev));
    const uint64_t bit = 1ull << (dev & 63);
    if (!(allowed.load(std::memory_order_relaxed) & bit)) {
      KV_HIP(hipFuncSetAttribute((const void*)k_attn_rows<T, D, kKind, NC>, hipFuncAttributeMaxDynamicSharedMemorySize,
                                 (int)lds));
      allowed.fetch_or(bit, std::memory_order_relaxed);
    }
  }
  hipLaunchKernelGGL((k_attn_rows<T, D, kKind, NC>), dim3(grid), dim3(256), lds, s, a);
  KV_HIP(hipGetLastError());
  return KV_OK;
}

template <class T, int D, Kind kKind>
kv_status launch_one(const AttnArgs& a, uint32_t rows, uint32_t grid, hipStream_t s) {
  switch (rows) {
    case 16: return launch_rows<T, D, kKind, 1>(a, grid, s);
    case 32:
      if constexpr (D <= 128) return launch_rows<T, D, kKind, 2>(a, grid, s);
      break;
    case 64:
      if constexpr (D <= 64) return launch_rows<T, D, kKind, 4>(a, grid, s);
      break;
    default: break;
  }
  return launch_tile<T, D, kKind>(a, grid, s);
}

template <class T, Kind kKind>
kv_status launch_dim(const AttnArgs& a, uint32_t dim, uint32_t rows, uint32_t grid, hipStream_t s) {
  switch (dim) {
    case 64: return launch_one<T, 64, kKind>(a, rows, grid, s);
    case 128: return launch_one<T, 128, kKind>(a, rows, grid, s);
    default: return launch_one<T, 256, kKind>(a, rows, grid, s);
  }
}

}  // namespace attn
}  // namespace kv
