// k_rope.hip - rotary positions, and the write of a step's keys and values
// into a paged cache.
//
// A pair (a, b) of a head at position p turns by the angle p*f.  f is kept as a
// fraction of a turn in 64 fixed-point bits, so that p*f modulo a turn is one
// wrapping product without rounding.  What remains is the error of f itself, which
// is worked out in double: a few units of 2^-53 of at most 0.16 turns, less than
// 2^-22 turns at any 32-bit position (in 32-bit floating point p*f is off by 0.004
// radians at p = 131,072 already).  The sine and cosine of the remaining eighth of a
// turn are Taylor sums whose next term is below 2^-25.
//
// All of it is bound by memory traffic and, at a step's few tokens, by latency.
// A thread owns 16 elements of a head (8 pairs: two 16-byte loads and stores,
// in the half layout one from each half) of one token, works out the eight
// sines and cosines once and walks over heads with them.  8,191 tokens of 40 heads
// of 128 (168 MB read and written) take 36.5 us, 4.6 TB/s, where a large copy does
// 4.8; 64 tokens of 32 heads 6.0 us a call, which is the host's time, and 2.7 in a
// graph of 100 calls (caches warm).  The writes of a chunk's queries, keys and
// values (212 MB) take 51 us, 4.1 TB/s: V^T is written in runs of a block's tokens,
// 128 bytes where blocks have 64; into an 8-bit cache of blocks of 16 tokens 42 MB
// take 11.7 us.
#include "rope_device.h"

namespace kv {
using namespace rope;
namespace {

struct ApplyArgs {
  const uint64_t* turn;
  const uint16_t* x;
  uint16_t* y;
  int64_t xt, xh, yt, yh;
  const int32_t* pos;
  uint32_t n_tokens, n_heads, units, rot_dim, heads_each, groups;
  float sign, magnitude;
  int in_place;
};

// Threads: unit fastest, then groups of heads, then tokens: neighbours read and write
// neighbouring 16 bytes of a head.
template <class V, bool kHalf>
__global__ __launch_bounds__(256) void k_rope_apply(ApplyArgs a) {
  const uint64_t id = (uint64_t)blockIdx.x * 256 + threadIdx.x;
  const uint32_t unit = (uint32_t)(id % a.units);
  const uint64_t rest = id / a.units;
  const uint32_t group = (uint32_t)(rest % a.groups);
  const uint64_t token = rest / a.groups;
  if (token >= a.n_tokens) return;
  const bool turns = unit < a.rot_dim / 16;
  if (!turns && a.in_place) return;
  Turns t;
  if (turns) load_turns(t, a.turn, unit, a.pos[token], a.sign, a.magnitude);
  int lo, hi;
  unit_at<kHalf>(unit, a.rot_dim, lo, hi);
  const uint32_t end = min(a.n_heads, (group + 1) * a.heads_each);
  const uint16_t* x = a.x + (int64_t)token * a.xt;
  uint16_t* y = a.y + (int64_t)token * a.yt;
  turn_heads<V, kHalf>(x, a.xh, y, a.yh, group * a.heads_each, end, lo, hi, turns, t);
}

struct AppendArgs {
  const uint64_t* turn;
  const int32_t *pos, *q_start;
  const int64_t* slot;
  const uint16_t *q, *k, *v;
  uint16_t* q_out;
  int64_t qt, qh, ot, oh, kt, kh, vt, vh;
  void *kc, *vc;
  int64_t k_block, v_block;
  const float *k_scale, *v_scale;
  uint64_t slots;  // n_blocks * block_size
  uint32_t max_tokens, n_req, q_heads, kv_heads, dim, units, rot_dim, heads_each, q_groups, groups;
  uint32_t block_shift;
  uint32_t qk_blocks;  // workgroups of queries and keys; the rest take values
  float magnitude;
};

// Queries and keys: threads as in k_rope_apply, groups of query heads before
// groups of key heads.  Values: a workgroup turns 64 tokens by 64 elements of a head
// in LDS; then lanes are tokens, so that tokens in neighbouring places of a block are
// written side by side, whatever request and place they begin at.
template <class V, bool kHalf, bool kFp8>
__global__ __launch_bounds__(256) void k_append(AppendArgs a) {
  const uint32_t n_tokens = min((uint32_t)max(a.q_start[a.n_req], 0), a.max_tokens);
  const int64_t block_mask = (1 << a.block_shift) - 1;
  if (blockIdx.x < a.qk_blocks) {
    const uint64_t id = (uint64_t)blockIdx.x * 256 + threadIdx.x;
    const uint32_t unit = (uint32_t)(id % a.units);
    const uint64_t rest = id / a.units;
    const uint32_t group = (uint32_t)(rest % a.groups);
    const uint64_t token = rest / a.groups;
    if (token >= n_tokens) return;
    const bool turns = unit < a.rot_dim / 16;
    Turns t;
    if (turns) load_turns(t, a.turn, unit, a.pos[token], 1.0f, a.magnitude);
    int lo, hi;
    unit_at<kHalf>(unit, a.rot_dim, lo, hi);
    if (group < a.q_groups) {
      const uint32_t end = min(a.q_heads, (group + 1) * a.heads_each);
      const uint16_t* x = a.q + (int64_t)token * a.qt;
      uint16_t* y = a.q_out + (int64_t)token * a.ot;
      turn_heads<V, kHalf>(x, a.qh, y, a.oh, group * a.heads_each, end, lo, hi, turns, t);
      return;
    }
    const int64_t slot = a.slot[token];
    if (slot < 0 || (uint64_t)slot >= a.slots) return;
    const uint32_t first = (group - a.q_groups) * a.heads_each, end = min(a.kv_heads, first + a.heads_each);
    const uint16_t* x = a.k + (int64_t)token * a.kt;
    for (uint32_t h = first; h < end; ++h) {
      uint4 u = *(const uint4*)(x + h * a.kh + lo), w = *(const uint4*)(x + h * a.kh + hi);
      const int64_t at = (slot >> a.block_shift) * a.k_block +
                         (((int64_t)h << a.block_shift) + (slot & block_mask)) * a.dim;
      float f[8], g[8];
      if (turns || kFp8) {
        unpack<V>(u, f);
        unpack<V>(w, g);
        if (turns) turn_unit<kHalf>(f, g, t);
      }
      if (kFp8) {
        const float s = a.k_scale ? a.k_scale[h] : 1.0f;
#pragma unroll
        for (int i = 0; i < 8; ++i) f[i] = f[i] / s, g[i] = g[i] / s;
        *(uint2*)((uint8_t*)a.kc + at + lo) = pack_fp8(f);
        *(uint2*)((uint8_t*)a.kc + at + hi) = pack_fp8(g);
      } else {
        if (turns) {
          u = pack<V>(f);
          w = pack<V>(g);
        }
        *(uint4*)((uint16_t*)a.kc + at + lo) = u;
        *(uint4*)((uint16_t*)a.kc + at + hi) = w;
      }
    }
    return;
  }

  const uint32_t strips = a.dim / 64;
  const uint32_t id = blockIdx.x - a.qk_blocks, strip = id % strips, h = id / strips % a.kv_heads;
  const uint32_t t0 = id / strips / a.kv_heads * 64;
  __shared__ uint16_t tile[64][66];  // 33 words a row: a column's reads fall on different banks
#pragma unroll
  for (int i = 0; i < 2; ++i) {
    const uint32_t t = threadIdx.x / 8 + 32 * i, chunk = threadIdx.x % 8;
    if (t0 + t < n_tokens) {
      const uint4 u = *(const uint4*)(a.v + (int64_t)(t0 + t) * a.vt + h * a.vh + strip * 64 + chunk * 8);
      uint32_t* to = (uint32_t*)&tile[t][chunk * 8];
      to[0] = u.x, to[1] = u.y, to[2] = u.z, to[3] = u.w;
    }
  }
  const uint32_t lane = threadIdx.x % 64, wave = threadIdx.x / 64;
  const int64_t slot = t0 + lane < n_tokens ? a.slot[t0 + lane] : -1;
  __syncthreads();
  if (slot < 0 || (uint64_t)slot >= a.slots) return;
  const int64_t at = (slot >> a.block_shift) * a.v_block +
                     (((int64_t)h * a.dim + strip * 64 + wave * 16) << a.block_shift) + (slot & block_mask);
  const float s = kFp8 && a.v_scale ? a.v_scale[h] : 1.0f;
#pragma unroll
  for (int d = 0; d < 16; d += 2) {
    const uint32_t two = *(const uint32_t*)&tile[lane][wave * 16 + d];
    if (kFp8) {
      const V v = __builtin_bit_cast(V, make_uint4(two, 0, 0, 0));
      const uint32_t w = pack_fp8x4((float)v[0] / s, (float)v[1] / s, 0.0f, 0.0f);
      ((uint8_t*)a.vc)[at + ((int64_t)d << a.block_shift)] = (uint8_t)w;
      ((uint8_t*)a.vc)[at + ((int64_t)(d + 1) << a.block_shift)] = (uint8_t)(w >> 8);
    } else {
      ((uint16_t*)a.vc)[at + ((int64_t)d << a.block_shift)] = (uint16_t)two;
      ((uint16_t*)a.vc)[at + ((int64_t)(d + 1) << a.block_shift)] = (uint16_t)(two >> 16);
    }
  }
}

template <bool kHalf>
void launch_apply(const ApplyArgs& a, uint32_t dtype, uint32_t grid, hipStream_t s) {
  if (dtype == KV_DT_BF16)
    hipLaunchKernelGGL((k_rope_apply<bf16x8, kHalf>), dim3(grid), dim3(256), 0, s, a);
  else
    hipLaunchKernelGGL((k_rope_apply<f16x8, kHalf>), dim3(grid), dim3(256), 0, s, a);
}

template <class V>
void launch_append(const AppendArgs& a, bool half, bool fp8, uint32_t grid, hipStream_t s) {
  if (half && fp8) hipLaunchKernelGGL((k_append<V, true, true>), dim3(grid), dim3(256), 0, s, a);
  if (half && !fp8) hipLaunchKernelGGL((k_append<V, true, false>), dim3(grid), dim3(256), 0, s, a);
  if (!half && fp8) hipLaunchKernelGGL((k_append<V, false, true>), dim3(grid), dim3(256), 0, s, a);
  if (!half && !fp8) hipLaunchKernelGGL((k_append<V, false, false>), dim3(grid), dim3(256), 0, s, a);
}

}  // namespace

kv_status rope_apply(const RopeTable& r, uint32_t dtype, const kv_heads_view& x, const kv_heads_view& y,
                     const int32_t* pos, uint32_t n_tokens, uint32_t n_heads, uint32_t head_dim, bool backward,
                     hipStream_t s) {
  ApplyArgs a{};
  a.turn = r.turn;
  a.x = (const uint16_t*)x.ptr;
  a.y = (uint16_t*)y.ptr;
  a.xt = x.token_stride, a.xh = x.head_stride, a.yt = y.token_stride, a.yh = y.head_stride;
  a.pos = pos;
  a.n_tokens = n_tokens;
  a.n_heads = n_heads;
  a.units = head_dim / 16;
  a.rot_dim = r.rot_dim;
  a.heads_each = heads_each_for((uint64_t)n_tokens * n_heads * a.units);
  a.groups = (n_heads + a.heads_each - 1) / a.heads_each;
  a.sign = backward ? -1.0f : 1.0f;
  a.magnitude = r.magnitude;
  a.in_place = x.ptr == y.ptr && x.token_stride == y.token_stride && x.head_stride == y.head_stride;
  const uint64_t grid = ((uint64_t)n_tokens * a.groups * a.units + 255) / 256;
  if (grid > 0x7fffffffull) return fail(KV_ERR_UNSUPPORTED, "kv_rope_apply: too many heads for one call");
  if (r.layout == KV_ROPE_HALF)
    launch_apply<true>(a, dtype, (uint32_t)grid, s);
  else
    launch_apply<false>(a, dtype, (uint32_t)grid, s);
  KV_HIP(hipGetLastError());
  return KV_OK;
}

kv_status paged_append(const kv_paged_batch& b, const kv_paged_cache& c, const RopeTable* r, uint32_t dtype,
                       const kv_heads_view& q, const kv_heads_view& q_out, const kv_heads_view& k,
                       const kv_heads_view& v, hipStream_t s) {
  AppendArgs a{};
  a.turn = r ? r->turn : nullptr;
  a.rot_dim = r ? r->rot_dim : 0;
  a.magnitude = r ? r->magnitude : 1.0f;
  a.pos = b.pos, a.q_start = b.q_start, a.slot = b.slot;
  a.q = (const uint16_t*)q.ptr, a.k = (const uint16_t*)k.ptr, a.v = (const uint16_t*)v.ptr;
  a.q_out = (uint16_t*)q_out.ptr;
  a.qt = q.token_stride, a.qh = q.head_stride, a.ot = q_out.token_stride, a.oh = q_out.head_stride;
  a.kt = k.token_stride, a.kh = k.head_stride, a.vt = v.token_stride, a.vh = v.head_stride;
  a.kc = c.k, a.vc = c.v;
  a.k_block = c.k_block_stride, a.v_block = c.v_block_stride;
  a.k_scale = c.k_scale, a.v_scale = c.v_scale;
  a.slots = (uint64_t)c.n_blocks * b.block_size;
  a.max_tokens = b.max_tokens, a.n_req = b.n_req;
  a.q_heads = q.ptr ? b.q_heads : 0, a.kv_heads = b.kv_heads;
  a.dim = b.head_dim, a.units = b.head_dim / 16;
  a.heads_each = heads_each_for((uint64_t)b.max_tokens * (a.q_heads + b.kv_heads) * a.units);
  a.q_groups = (a.q_heads + a.heads_each - 1) / a.heads_each;
  a.groups = a.q_groups + (b.kv_heads + a.heads_each - 1) / a.heads_each;
  a.block_shift = (uint32_t)__builtin_ctz(b.block_size);
  const uint64_t qk = ((uint64_t)b.max_tokens * a.groups * a.units + 255) / 256;
  const uint64_t vv = ((uint64_t)b.max_tokens + 63) / 64 * b.kv_heads * (b.head_dim / 64);
  if (qk + vv > 0x7fffffffull) return fail(KV_ERR_UNSUPPORTED, "kv_paged_append: too many heads for one call");
  a.qk_blocks = (uint32_t)qk;
  const bool half = !r || r->layout == KV_ROPE_HALF, fp8 = c.dtype == KV_DT_FP8;
  if (dtype == KV_DT_BF16)
    launch_append<bf16x8>(a, half, fp8, (uint32_t)(qk + vv), s);
  else
    launch_append<f16x8>(a, half, fp8, (uint32_t)(qk + vv), s);
  KV_HIP(hipGetLastError());
  return KV_OK;
}

}  // namespace kv
