// k_block.hip - the write of a step's keys and values into a paged cache of 8 bits with a
// scale for each block of tokens and head, and the read of any paged cache into rows.
//
// A held number c of block b and head h stands for c * s[b][h].  With Q the type's
// largest number and x what a step puts into the block, need = max |x| / Q:
//   the block's first token is among them:  s = need
//   it goes on (a context ends inside it):  s = old * 2^n, the least n >= 0 with
//                                           need <= s; earlier numbers become
//                                           round(c * 2^-n)
// and c = round(x * (1 / s)).  Scales rise by whole powers of two, so that the
// earlier numbers' roundings add up to less than one unit whatever the number of rises
// (1/2 + 1/4 + ...), where scales that follow the maximum would add half a unit each time.
//
// Both kernels walk over runs: the tokens of one request in one block.  No two runs of a
// step write to one block, so there is no order among workgroups, and no atomics.
//
// Both are bound by memory, and small ones by a chain of round trips (what is known of the
// request, then its slot or block, then the elements, then the old scale).  Measured, with 32
// query and 8 key/value heads of 128:
//   the write of 11,675 prompt tokens (24 requests, blocks of 64, bfloat16 to whole numbers)
//   81 us from cold caches, 48 in a graph with warm ones; most of it are the queries, 191 MB,
//   the rest 72 MB (25 us alone); with the read of the blocks it touched 74 us a call, 340 MB at
//   4.6 TB/s, where a large copy does 5.2.  64 single tokens: 5.1 us in a graph of 100, 7 a call (host).
//   1,000 single tokens, keys and values of 8 heads: 17.7 us in a graph in blocks of 16, 48 in blocks of 64
//   (into 16-bit caches 12.7 and 15.1): a task has wavefronts for all of its block, whatever goes into it.
//   the read of 64 prefixes (135,457 tokens, blocks of 16, heads of 64, 417 MB) 80 us, 5.2 TB/s;
//   of 4 documents (202,264 tokens, blocks of 64, 1.24 GB) 219 us, 5.7 TB/s; of 3 chats (155
//   tokens) 3.6 us in a graph, 7 a call (host).
#include "rope_device.h"

namespace kv {
using namespace rope;
namespace {

// ---------------------------------------------------------------------------
// runs
// ---------------------------------------------------------------------------
// Request r has tokens start[r] .. start[r+1] - 1 of a packed batch, at positions
// from `at` on.  They fall into at most n / size + 2 blocks, so the places
// start[r] / size + 2 r  and on are its own; some stay empty.  A place finds its
// request by a search over r, 64 candidates at a time.  Where requests times the runs
// that one can have is about as many places (single tokens, one long prompt),
// those are used and nothing is searched.
struct Runs {
  const int32_t* start;  // [n_req + 1]
  uint32_t n_req, shift;
  uint32_t each;         // runs of a request, or 0: search
};

uint64_t plan_runs(Runs& r, const int32_t* start, uint32_t n_req, uint32_t block, uint64_t tokens, uint64_t most) {
  r.start = start, r.n_req = n_req, r.shift = (uint32_t)__builtin_ctz(block);
  const uint64_t found = tokens / block + 2ull * n_req;
  const uint64_t one = most <= 1 ? 1 : (most - 1) / block + 2;
  const bool direct = one * n_req <= 2 * found && one * n_req <= 0xffffffffull;
  r.each = direct ? (uint32_t)one : 0;
  return direct ? one * n_req : found;
}

struct Run {
  uint32_t req, run;        // the request, n_req: none; which of its runs
  int32_t start, end;       // its tokens
  int32_t length, first;    // kv_len, and the first position asked for (NULL: 0)
};

// The run of place u; the whole wavefront asks.  What is known of a request is loaded
// by the lane that has it as its candidate, all at once: a small step is one chain of such
// round trips.
__device__ __forceinline__ Run find_run(const Runs& runs, uint32_t u, const int32_t* length, const int32_t* first) {
  Run r;
  if (runs.each) {
    r.req = u / runs.each;
    r.run = u - r.req * runs.each;
    const uint32_t at = min(r.req, runs.n_req - 1);
    r.start = runs.start[at], r.end = runs.start[at + 1], r.length = length[at], r.first = first ? first[at] : 0;
    return r;
  }
  auto base = [&](int32_t start, uint32_t req) { return ((uint32_t)max(start, 0) >> runs.shift) + 2 * req; };
  uint32_t lo = 0, n = runs.n_req;
  while (n > 64) {
    const uint32_t step = (n + 63) / 64, at = lane_id() * step;
    const uint64_t below = __ballot(at < n && base(runs.start[lo + min(at, n - 1)], lo + at) <= u);
    const uint32_t i = (uint32_t)max((int)__popcll(below) - 1, 0) * step;
    lo += i;
    n = min(step, n - i);
  }
  const uint32_t at = lo + min(lane_id(), n - 1);
  const int32_t start = runs.start[at], end = runs.start[at + 1], len = length[at], from = first ? first[at] : 0;
  const uint64_t below = __ballot(lane_id() < n && base(start, at) <= u);
  const int i = max((int)__popcll(below) - 1, 0);
  r.start = __builtin_amdgcn_readlane(start, i), r.end = __builtin_amdgcn_readlane(end, i);
  r.length = __builtin_amdgcn_readlane(len, i), r.first = __builtin_amdgcn_readlane(from, i);
  // (a first row that is not 0 leaves the places before it to nobody)
  r.req = below ? lo + i : runs.n_req;
  r.run = u - base(r.start, lo + i);
  return r;
}

// ---------------------------------------------------------------------------
// the two held types
// ---------------------------------------------------------------------------
struct Fp8 {
  static constexpr float kMost = 448.0f;
  static __device__ __forceinline__ uint32_t pack4(float a, float b, float c, float d) { return pack_fp8x4(a, b, c, d); }
  template <int I>
  static __device__ __forceinline__ float value(uint32_t u) { return __builtin_amdgcn_cvt_f32_fp8((int)u, I); }
};
struct I8 {
  static constexpr float kMost = 127.0f;
  // nearest even: the low bits of a sum with 3 * 2^22 are the whole number
  static __device__ __forceinline__ uint32_t bits(float x) {
    x = x == x ? x : 0.0f;
    return __builtin_bit_cast(uint32_t, __builtin_amdgcn_fmed3f(x, -127.0f, 127.0f) + 12582912.0f);
  }
  static __device__ __forceinline__ uint32_t pack4(float a, float b, float c, float d) {
    const uint32_t lo = __builtin_amdgcn_perm(bits(b), bits(a), 0x0c0c0400u);
    const uint32_t hi = __builtin_amdgcn_perm(bits(d), bits(c), 0x04000c0cu);
    return lo | hi;
  }
  template <int I>
  static __device__ __forceinline__ float value(uint32_t u) { return (float)(int8_t)(u >> (8 * I)); }
};

template <class H>
__device__ __forceinline__ void values4(uint32_t u, float* f) {
  f[0] = H::template value<0>(u), f[1] = H::template value<1>(u), f[2] = H::template value<2>(u), f[3] = H::template value<3>(u);
}
// earlier numbers in a larger unit
template <class H>
__device__ __forceinline__ uint32_t shrink4(uint32_t u, float by) {
  float f[4];
  values4<H>(u, f);
  return H::pack4(f[0] * by, f[1] * by, f[2] * by, f[3] * by);
}

// byte (16 bits: half) i of the result's word j is byte j of word i
__device__ __forceinline__ void turn_bytes(uint32_t* u) {
  const uint32_t a = __builtin_amdgcn_perm(u[1], u[0], 0x05010400u), b = __builtin_amdgcn_perm(u[3], u[2], 0x05010400u);
  const uint32_t c = __builtin_amdgcn_perm(u[1], u[0], 0x07030602u), d = __builtin_amdgcn_perm(u[3], u[2], 0x07030602u);
  u[0] = __builtin_amdgcn_perm(b, a, 0x05040100u), u[1] = __builtin_amdgcn_perm(b, a, 0x07060302u);
  u[2] = __builtin_amdgcn_perm(d, c, 0x05040100u), u[3] = __builtin_amdgcn_perm(d, c, 0x07060302u);
}
__device__ __forceinline__ void turn_halves(uint32_t& a, uint32_t& b) {
  const uint32_t lo = __builtin_amdgcn_perm(b, a, 0x05040100u);
  b = __builtin_amdgcn_perm(b, a, 0x07060302u);
  a = lo;
}

// Infinities and NaN do not make a scale.
__device__ __forceinline__ float magnitude_of(float x) {
  const uint32_t u = __builtin_bit_cast(uint32_t, x) & 0x7fffffffu;
  return __builtin_bit_cast(float, u < 0x7f800000u ? u : 0u);
}

struct NewScale {
  float scale, inverse, shrink;  // shrink: of the earlier numbers
};
// `old`: the scale so far, 0 for a block that begins.  What no write has left there (NaN,
// infinities, negative and subnormal numbers) counts as 0.
__device__ __forceinline__ NewScale new_scale(float need, float old) {
  NewScale n;
  n.shrink = 1.0f;
  n.scale = need;
  if (old >= 0x1p-126f && old <= 3.402823466e38f) {
    const uint32_t a = __builtin_bit_cast(uint32_t, need), b = __builtin_bit_cast(uint32_t, old);
    int rise = 0;
    if (need > old) {
      rise = (int)(a >> 23) - (int)(b >> 23) + ((a & 0x7fffffu) > (b & 0x7fffffu) ? 1 : 0);
      n.shrink = __builtin_amdgcn_ldexpf(1.0f, -rise);
    }
    n.scale = __builtin_amdgcn_ldexpf(old, rise);
  } else if (need > 0.0f) {
    n.shrink = 0.0f;
  }
  // (any number does for zeros; infinities become the largest number with this one)
  n.inverse = n.scale > 0.0f ? 1.0f / n.scale : 0x1p-126f;
  return n;
}

// ---------------------------------------------------------------------------
// the write
// ---------------------------------------------------------------------------
struct BlockArgs {
  Runs runs;
  const uint64_t* turn;
  const int32_t *pos, *kv_len;
  const int64_t* slot;
  const uint16_t *q, *k, *v;
  uint16_t* q_out;
  int64_t qt, qh, ot, oh, kt, kh, vt, vh;
  uint8_t *kc, *vc;
  int64_t k_block, v_block;
  float *k_scale, *v_scale;
  uint64_t slots;  // n_blocks * block_size
  uint32_t max_tokens, q_heads, kv_heads, dim_shift, units, rot_dim, heads_each, q_groups;
  uint64_t run_share;   // share of workgroups that take runs, in 2^-32; the rest take queries
  uint32_t waves;       // of a task
  uint32_t tasks;       // runs by heads by keys or values
  float magnitude;
};

// A task is a run's keys of one head, or its values: a wavefront for up to 2,048 of
// a block's numbers, up to 16 of them together.  (A workgroup for a run's keys and values that
// reads them once for the scale and again for the numbers, and turns values byte by byte in LDS,
// takes 101 us for 81 of the prompts above, from cold caches.)  What goes into the block stays in
// registers from its largest magnitude to its rounding, so everything is read and written
// once.
//   keys     a lane has 16 elements of kItems tokens, turned
//   values   8 elements of 4 tokens, kItems / 2 times, turned to 4 tokens of 8
//            elements in registers; words that other tokens share are read first
template <class V, bool kHalf, class H, int kItems>
__global__ void __launch_bounds__(1024) k_append_block(BlockArgs a) {
  const uint32_t tid = threadIdx.x;
  // Workgroups of runs lie evenly among those of queries: a run is a chain of round trips, and what
  // queries read and write meanwhile hides it (the prompts above with their read 74 us; queries
  // first 78, runs first 81).
  const uint32_t run_block = (uint32_t)((uint64_t)blockIdx.x * a.run_share >> 32);
  const bool queries = (uint32_t)(((uint64_t)blockIdx.x + 1) * a.run_share >> 32) == run_block;
  if (queries) {  // as in k_append
    const uint32_t n_tokens = min((uint32_t)max(a.runs.start[a.runs.n_req], 0), a.max_tokens);
    const uint64_t id = (uint64_t)(blockIdx.x - run_block) * blockDim.x + tid;
    const uint32_t unit = (uint32_t)(id % a.units);
    const uint64_t rest = id / a.units;
    const uint32_t group = (uint32_t)(rest % a.q_groups);
    const uint64_t token = rest / a.q_groups;
    if (token >= n_tokens) return;
    const bool turns = unit < a.rot_dim / 16;
    Turns t;
    if (turns) load_turns(t, a.turn, unit, a.pos[token], 1.0f, a.magnitude);
    int lo, hi;
    unit_at<kHalf>(unit, a.rot_dim, lo, hi);
    turn_heads<V, kHalf>(a.q + (int64_t)token * a.qt, a.qh, a.q_out + (int64_t)token * a.ot, a.oh, group * a.heads_each,
                         min(a.q_heads, (group + 1) * a.heads_each), lo, hi, turns, t);
    return;
  }

  // All wavefronts of a task leave together or not at all: there is a barrier below.
  const bool alone = a.waves == 1;
  const uint32_t me = alone ? lane_id() : tid, threads = a.waves * 64;
  const uint32_t task = alone ? run_block * (blockDim.x / 64) + wave_id() : run_block;
  if (task >= a.tasks) return;
  const bool keys = !(task & 1);
  const uint32_t place = task / 2 / a.kv_heads, head = task / 2 - place * a.kv_heads;
  const Run r = find_run(a.runs, place, a.kv_len, nullptr);
  if (r.req >= a.runs.n_req) return;
  const uint32_t shift = a.runs.shift;
  const int64_t t0 = r.start, t1 = min((int64_t)r.end, (int64_t)a.max_tokens);
  if (t0 < 0 || t0 >= t1) return;
  // the run: n tokens from `token` on, in places `at` and on of their block
  const int64_t ctx = r.length - ((int64_t)r.end - t0);
  if (ctx < 0) return;
  const int64_t block0 = ((ctx >> shift) + r.run) << shift;
  const int64_t from = max(ctx, block0), to = min(ctx + (t1 - t0), block0 + (1ll << shift));
  if (from >= to) return;
  const uint32_t token = (uint32_t)(t0 + (from - ctx)), n = (uint32_t)(to - from), at = (uint32_t)(from - block0);
  const int64_t slot = a.slot[token];
  // (looked at when the elements are on their way)
  const bool there = slot >= 0 && (uint64_t)slot < a.slots;
  const int64_t page = there ? slot >> shift : 0;
  float* const scales = (keys ? a.k_scale : a.v_scale) + page * a.kv_heads + head;

  __shared__ uint32_t most[16];
  // the largest magnitude of the task's elements, and what it makes of the scale
  auto scale_of = [&](float mine, float old) {
    uint32_t u = (uint32_t)__builtin_amdgcn_readlane((int)wave_incl_max_u32(__builtin_bit_cast(uint32_t, mine)), 63);
    if (!alone) {
      if (lane_id() == 0) most[wave_id()] = u;
      __syncthreads();
      u = most[0];
      for (uint32_t w = 1; w < a.waves; ++w) u = max(u, most[w]);
    }
    // A need that is not 0 is no subnormal number: new_scale() reads exponents.
    const float x = __builtin_bit_cast(float, u) / H::kMost;
    const NewScale s = new_scale(x > 0.0f ? fmaxf(x, 0x1p-126f) : 0.0f, old);
    if (me == 0) *scales = s.scale;
    return s;
  };

  if (keys) {
    uint8_t* const kc = a.kc + page * a.k_block + ((int64_t)head << (shift + a.dim_shift));
    const uint32_t unit_shift = a.dim_shift - 4, unit = me & (a.units - 1);
    int lo, hi;
    unit_at<kHalf>(unit, a.rot_dim, lo, hi);
    const bool turns = unit < a.rot_dim / 16;
    const uint16_t* const k = a.k + (int64_t)token * a.kt + head * a.kh;
    float f[kItems][8], g[kItems][8];
    uint4 u[kItems], w[kItems];
    int32_t pos[kItems];
    // (units divide a task's threads: a lane's items are those of one unit)
#pragma unroll
    for (int i = 0; i < kItems; ++i) {
      const uint32_t t = (me + i * threads) >> unit_shift;
      u[i] = w[i] = make_uint4(0, 0, 0, 0);
      pos[i] = 0;
      if (t < n) {
        u[i] = *(const uint4*)(k + (int64_t)t * a.kt + lo);
        w[i] = *(const uint4*)(k + (int64_t)t * a.kt + hi);
        if (turns) pos[i] = a.pos[token + t];
      }
    }
    if (!there) return;
    const float old = at ? *scales : 0.0f;
    float mine = 0.0f;
#pragma unroll
    for (int i = 0; i < kItems; ++i) {
      unpack<V>(u[i], f[i]);
      unpack<V>(w[i], g[i]);
      if (turns && (me + i * threads) >> unit_shift < n) {
        Turns t;
        load_turns(t, a.turn, unit, pos[i], 1.0f, a.magnitude);
        turn_unit<kHalf>(f[i], g[i], t);
      }
#pragma unroll
      for (int e = 0; e < 8; ++e) mine = fmaxf(mine, fmaxf(magnitude_of(f[i][e]), magnitude_of(g[i][e])));
    }
    const NewScale s = scale_of(mine, old);
#pragma unroll
    for (int i = 0; i < kItems; ++i) {
      const uint32_t t = (me + i * threads) >> unit_shift;
      if (t >= n) continue;
#pragma unroll
      for (int e = 0; e < 8; ++e) f[i][e] *= s.inverse, g[i][e] *= s.inverse;
      uint8_t* row = kc + ((int64_t)(at + t) << a.dim_shift);
      *(uint2*)(row + lo) = make_uint2(H::pack4(f[i][0], f[i][1], f[i][2], f[i][3]), H::pack4(f[i][4], f[i][5], f[i][6], f[i][7]));
      *(uint2*)(row + hi) = make_uint2(H::pack4(g[i][0], g[i][1], g[i][2], g[i][3]), H::pack4(g[i][4], g[i][5], g[i][6], g[i][7]));
    }
    if (at && s.shrink != 1.0f)
      for (uint32_t i = me; i < at << (a.dim_shift - 4); i += threads) {
        uint4* p = (uint4*)kc + i;
        const uint4 x = *p;
        *p = make_uint4(shrink4<H>(x.x, s.shrink), shrink4<H>(x.y, s.shrink), shrink4<H>(x.z, s.shrink), shrink4<H>(x.w, s.shrink));
      }
    return;
  }

  uint8_t* const vc = a.vc + page * a.v_block + ((int64_t)head << (shift + a.dim_shift));
  const uint32_t chunk_shift = a.dim_shift - 3, d = (me & ((1u << chunk_shift) - 1)) * 8;
  const uint16_t* const v = a.v + (int64_t)token * a.vt + head * a.vh + d;
  constexpr int kWords = kItems / 2;
  uint4 x[kWords][4];
  uint32_t before[kWords][8];
  // places p .. p + 3 of the block; bytes of those that the run fills
  auto place_of = [&](int i) { return ((me + i * threads) >> chunk_shift) * 4; };
  auto bytes_in = [](int first, int last) {  // of places `first` to `last` - 1 of four
    const uint32_t below = last >= 4 ? 0xffffffffu : last > 0 ? (1u << (8 * last)) - 1 : 0u;
    return first <= 0 ? below : first >= 4 ? 0u : below & ~((1u << (8 * first)) - 1);
  };
#pragma unroll
  for (int i = 0; i < kWords; ++i) {
    const uint32_t p = place_of(i);
#pragma unroll
    for (int j = 0; j < 4; ++j) {
      x[i][j] = make_uint4(0, 0, 0, 0);
      if (p + j >= at && p + j < at + n) x[i][j] = *(const uint4*)(v + (int64_t)(p + j - at) * a.vt);
    }
  }
  if (!there) return;
  const float old = at ? *scales : 0.0f;
#pragma unroll
  for (int i = 0; i < kWords; ++i) {
    const uint32_t p = place_of(i);
    const uint32_t fills = bytes_in((int)at - (int)p, (int)(at + n) - (int)p);
#pragma unroll
    for (int e = 0; e < 8; ++e) before[i][e] = 0;
    if (fills && fills != 0xffffffffu)
#pragma unroll
      for (int e = 0; e < 8; ++e) before[i][e] = *(const uint32_t*)(vc + ((int64_t)(d + e) << shift) + p);
  }
  float mine = 0.0f;
#pragma unroll
  for (int i = 0; i < kWords; ++i)
#pragma unroll
    for (int j = 0; j < 4; ++j) {
      float f[8];
      unpack<V>(x[i][j], f);
#pragma unroll
      for (int e = 0; e < 8; ++e) mine = fmaxf(mine, magnitude_of(f[e]));
    }
  const NewScale s = scale_of(mine, old);
#pragma unroll
  for (int i = 0; i < kWords; ++i) {
    const uint32_t p = place_of(i);
    const uint32_t fills = bytes_in((int)at - (int)p, (int)(at + n) - (int)p);
    const uint32_t shrinks = s.shrink != 1.0f && p < 1u << shift ? bytes_in(0, (int)at - (int)p) : 0u;
    if (!fills && !shrinks) continue;
    uint8_t* const to_words = vc + ((int64_t)d << shift) + p;
    if (!fills)
#pragma unroll
      for (int e = 0; e < 8; ++e) before[i][e] = *(const uint32_t*)(to_words + ((int64_t)e << shift));
    uint32_t lo[4], hi[4];
#pragma unroll
    for (int j = 0; j < 4; ++j) {
      float f[8];
      unpack<V>(x[i][j], f);
#pragma unroll
      for (int e = 0; e < 8; ++e) f[e] *= s.inverse;
      lo[j] = H::pack4(f[0], f[1], f[2], f[3]);
      hi[j] = H::pack4(f[4], f[5], f[6], f[7]);
    }
    turn_bytes(lo);
    turn_bytes(hi);
#pragma unroll
    for (int e = 0; e < 8; ++e) {
      uint32_t* const word = (uint32_t*)(to_words + ((int64_t)e << shift));
      uint32_t u = e < 4 ? lo[e & 3] : hi[e & 3];
      if (fills != 0xffffffffu) {
        uint32_t b = before[i][e];
        if (shrinks) b = (shrink4<H>(b, s.shrink) & shrinks) | (b & ~shrinks);
        u = (u & fills) | (b & ~fills);
      }
      *word = u;
    }
  }
}

// ---------------------------------------------------------------------------
// the read
// ---------------------------------------------------------------------------
struct ReadArgs {
  Runs runs;
  const int32_t *first, *table, *kv_len;
  uint16_t *k, *v;
  int64_t kt, kh, vt, vh;
  const uint8_t *kc, *vc;
  int64_t k_block, v_block;  // bytes
  const float *k_scale, *v_scale;
  uint32_t max_rows, max_blocks, n_blocks, kv_heads, dim_shift;
  uint32_t each;      // wavefronts of a run's keys, and of its values
  uint32_t tasks;     // wavefronts in all
  uint32_t by_block;  // scales by block, or by head
};

// 16-bit caches: numbers are copied
struct Same {};
// so many words
template <int kWords>
struct Load {
  typedef uint4 type;
};
template <>
struct Load<2> {
  typedef uint2 type;
};
template <>
struct Load<1> {
  typedef uint32_t type;
};

// 4 numbers, times their scale, in 16 bits.  A value near the end of the type's range may be held
// as up to a unit more than it was: what is past the range becomes its largest number, as the
// write does with its own type's.  (NaN stays NaN.)  `past`: whether some scale of the wavefront's
// can bring that about (asked of every number, the documents above take 227 us for 219).
template <class V, class H>
__device__ __forceinline__ uint2 rows4(uint32_t u, float by, bool past) {
  typedef typename Elem<V>::type E;
  constexpr float kMost = Elem<V>::kMost;
  float f[4];
  values4<H>(u, f);
#pragma unroll
  for (int i = 0; i < 4; ++i) f[i] *= by;
  if (past)
#pragma unroll
    for (int i = 0; i < 4; ++i) f[i] = __builtin_elementwise_minimum(__builtin_elementwise_maximum(f[i], -kMost), kMost);
  uint16_t h[4];
#pragma unroll
  for (int i = 0; i < 4; ++i) h[i] = __builtin_bit_cast(uint16_t, (E)f[i]);
  return make_uint2(h[0] | (uint32_t)h[1] << 16, h[2] | (uint32_t)h[3] << 16);
}
template <class V, class H>
__device__ __forceinline__ bool may_pass(float by) {  // (whole numbers that a caller filled in may be -128)
  return fabsf(by) > Elem<V>::kMost / (H::kMost + 1.0f);
}

// Rows are written past the caches, which they would fill with what nobody reads twice (the
// prefixes above 80 us, with plain stores 86; the documents 219 and 239).
__device__ __forceinline__ void put_row(uint16_t* p, const uint4& w) {
  typedef uint32_t u32x4 __attribute__((ext_vector_type(4)));
  __builtin_nontemporal_store(__builtin_bit_cast(u32x4, w), (u32x4*)p);
}

// A wavefront reads 2 KB times kWords of a run's keys, or of its values, whatever heads these
// are: it shares nothing with others.  Keys go as they lie, 8 elements a load.  Of the values
// a lane takes 8 elements of as many tokens as kWords words hold, turns them in registers
// and writes 16 bytes of each token's row.  8 KB (the documents above 219 us, with 2 KB 273; the
// prefixes 80 and 81), and 2 where that leaves compute units without work (the chats 3.6 us in a
// graph, with 8 KB 6.3): see kFewTasks.
template <class V, class H, int kWords>
__global__ __launch_bounds__(256) void k_read(ReadArgs a) {
  constexpr int kBytes = __is_same(H, Same) ? 2 : 1;
  constexpr int kTokens = 4 * kWords / kBytes;  // of a lane's values
  constexpr uint32_t kTokenShift = __builtin_ctz(kTokens);
  const uint32_t lane = lane_id();
  const uint32_t task = blockIdx.x * 4 + wave_id();
  if (task >= a.tasks) return;
  const uint32_t place = task / (2 * a.each);
  uint32_t part = task - place * (2 * a.each);
  const Run r = find_run(a.runs, place, a.kv_len, a.first);
  if (r.req >= a.runs.n_req) return;
  const uint32_t shift = a.runs.shift;
  const int64_t t0 = r.start, t1 = min((int64_t)r.end, (int64_t)a.max_rows);
  if (t0 < 0 || t0 >= t1) return;
  const int64_t first = r.first;
  const int64_t column = (first >> shift) + r.run, block0 = column << shift;
  const int64_t from = max(first, block0), to = min(first + (t1 - t0), block0 + (1ll << shift));
  if (from >= to) return;
  // Places begin .. end - 1 of the block are rows, those before `have` are in the cache.
  const uint32_t begin = (uint32_t)(from - block0), end = (uint32_t)(to - block0);
  const int64_t row0 = t0 + (from - first) - begin;  // row of place 0
  int page = -1;
  if (column >= 0 && column < a.max_blocks) page = a.table[(uint64_t)r.req * a.max_blocks + column];
  const bool there = page >= 0 && page < (int)a.n_blocks;
  const uint32_t have = there ? (uint32_t)min(max((int64_t)r.length - block0, (int64_t)0), (int64_t)end) : 0;
  if (!there) page = 0;
  const bool keys = part < a.each;
  if (!keys) part -= a.each;
  const float* scales = keys ? a.k_scale : a.v_scale;
  auto scale_of = [&](uint32_t head) {
    if (kBytes == 2 || !scales) return 1.0f;
    return scales[(a.by_block ? (int64_t)page * a.kv_heads : 0) + head];
  };

  if (keys) {
    const uint8_t* kc = a.kc + page * a.k_block;
    constexpr int kSteps = 4 * kWords / kBytes;  // of 64 lanes by 8 elements
    const uint32_t chunk_shift = a.dim_shift - 3;
    typedef typename Load<2 * kBytes>::type U;
    U u[kSteps];
    float by[kSteps];
    auto item = [&](int i, uint32_t& t, uint32_t& head) {
      const uint32_t at = (part * kSteps + i) * 64 + lane;
      t = (at >> chunk_shift) & ((1u << shift) - 1), head = at >> (chunk_shift + shift);
      return at;
    };
#pragma unroll
    for (int i = 0; i < kSteps; ++i) {
      uint32_t t, head;
      const uint32_t at = item(i, t, head);
      u[i] = U{};
      by[i] = 1.0f;
      if (head < a.kv_heads && t >= begin && t < have) {
        u[i] = *(const U*)(kc + (int64_t)at * 8 * kBytes);
        by[i] = scale_of(head);
      }
    }
    bool past = false;
    if constexpr (kBytes == 1) {
#pragma unroll
      for (int i = 0; i < kSteps; ++i) past |= may_pass<V, H>(by[i]);
      past = __any(past);
    }
#pragma unroll
    for (int i = 0; i < kSteps; ++i) {
      uint32_t t, head;
      const uint32_t at = item(i, t, head);
      if (head >= a.kv_heads || t < begin || t >= end) continue;
      uint4 w;
      if constexpr (kBytes == 1) {
        const uint2 lo = rows4<V, H>(u[i].x, by[i], past), hi = rows4<V, H>(u[i].y, by[i], past);
        w = make_uint4(lo.x, lo.y, hi.x, hi.y);
      } else {
        w = u[i];
      }
      put_row(a.k + (row0 + t) * a.kt + head * a.kh + (at & ((1u << chunk_shift) - 1)) * 8, w);
    }
    return;
  }

  // values: item = (head, tokens, 8 elements), the elements first
  const uint32_t item = part * 64 + lane, chunk_shift = a.dim_shift - 3;
  const uint32_t d = (item & ((1u << chunk_shift) - 1)) * 8;
  const uint32_t t = (item >> chunk_shift << kTokenShift) & ((1u << shift) - 1);
  const uint32_t head = item >> (chunk_shift + shift - kTokenShift);
  if (head >= a.kv_heads || t + kTokens <= begin || t >= end) return;
  typedef typename Load<kWords>::type U;
  U u[8];
#pragma unroll
  for (int i = 0; i < 8; ++i) u[i] = U{};
  float by = 1.0f;
  if (t < have) {
    by = scale_of(head);
    const uint8_t* p = a.vc + page * a.v_block + (((((int64_t)head << a.dim_shift) + d) << shift) + t) * kBytes;
#pragma unroll
    for (int i = 0; i < 8; ++i) u[i] = *(const U*)(p + ((int64_t)(i * kBytes) << shift));
  }
  bool past = false;
  if constexpr (kBytes == 1) past = __any(may_pass<V, H>(by));
  uint16_t* out = a.v + (row0 + t) * a.vt + head * a.vh + d;
  auto put = [&](int i, const uint4& w) {
    const uint32_t at = t + i;
    if (at >= begin && at < end) put_row(out + i * a.vt, at < have ? w : make_uint4(0, 0, 0, 0));
  };
  auto word = [](const U& w, int i) {
    if constexpr (kWords == 1)
      return w;
    else
      return i == 0 ? w.x : i == 1 ? w.y : i == 2 ? w.z : w.w;
  };
#pragma unroll
  for (int w = 0; w < kWords; ++w) {  // a word of 4 tokens, or of 2
    uint32_t lo[4], hi[4];
#pragma unroll
    for (int i = 0; i < 4; ++i) lo[i] = word(u[i], w), hi[i] = word(u[4 + i], w);
    if constexpr (kBytes == 1) {
      turn_bytes(lo);
      turn_bytes(hi);
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        const uint2 x = rows4<V, H>(lo[i], by, past), y = rows4<V, H>(hi[i], by, past);
        put(4 * w + i, make_uint4(x.x, x.y, y.x, y.y));
      }
    } else {
      turn_halves(lo[0], lo[1]), turn_halves(lo[2], lo[3]), turn_halves(hi[0], hi[1]), turn_halves(hi[2], hi[3]);
      put(2 * w, make_uint4(lo[0], lo[2], hi[0], hi[2]));
      put(2 * w + 1, make_uint4(lo[1], lo[3], hi[1], hi[3]));
    }
  }
}

template <class V, class H>
void launch_append(const BlockArgs& a, bool half, bool more, uint32_t grid, uint32_t threads, hipStream_t s) {
  if (half && !more) hipLaunchKernelGGL((k_append_block<V, true, H, 2>), dim3(grid), dim3(threads), 0, s, a);
  if (half && more) hipLaunchKernelGGL((k_append_block<V, true, H, 4>), dim3(grid), dim3(threads), 0, s, a);
  if (!half && !more) hipLaunchKernelGGL((k_append_block<V, false, H, 2>), dim3(grid), dim3(threads), 0, s, a);
  if (!half && more) hipLaunchKernelGGL((k_append_block<V, false, H, 4>), dim3(grid), dim3(threads), 0, s, a);
}

// Fewer wavefronts than this, two for each SIMD of the chip, leave some without work.
constexpr uint64_t kFewTasks = 2048;

template <class V, class H>
void launch_read(const ReadArgs& a, bool few, uint32_t grid, hipStream_t s) {
  if (few)
    hipLaunchKernelGGL((k_read<V, H, 1>), dim3(grid), dim3(256), 0, s, a);
  else
    hipLaunchKernelGGL((k_read<V, H, 4>), dim3(grid), dim3(256), 0, s, a);
}

template <class V>
void launch_read(const ReadArgs& a, uint32_t kept, bool few, uint32_t grid, hipStream_t s) {
  if (kept == KV_DT_I8_BLOCK)
    launch_read<V, I8>(a, few, grid, s);
  else if (eight_bits(kept))
    launch_read<V, Fp8>(a, few, grid, s);
  else
    launch_read<V, Same>(a, few, grid, s);
}

}  // namespace

kv_status paged_append_block(const kv_paged_batch& b, const kv_paged_cache& c, const RopeTable* r, uint32_t dtype,
                             const kv_heads_view& q, const kv_heads_view& q_out, const kv_heads_view& k,
                             const kv_heads_view& v, hipStream_t s) {
  BlockArgs a{};
  a.turn = r ? r->turn : nullptr;
  a.rot_dim = r ? r->rot_dim : 0;
  a.magnitude = r ? r->magnitude : 1.0f;
  a.pos = b.pos, a.kv_len = b.kv_len, a.slot = b.slot;
  a.q = (const uint16_t*)q.ptr, a.k = (const uint16_t*)k.ptr, a.v = (const uint16_t*)v.ptr;
  a.q_out = (uint16_t*)q_out.ptr;
  a.qt = q.token_stride, a.qh = q.head_stride, a.ot = q_out.token_stride, a.oh = q_out.head_stride;
  a.kt = k.token_stride, a.kh = k.head_stride, a.vt = v.token_stride, a.vh = v.head_stride;
  a.kc = (uint8_t*)c.k, a.vc = (uint8_t*)c.v;
  a.k_block = c.k_block_stride, a.v_block = c.v_block_stride;
  // written here and nowhere else: caches of this kind have their scales in memory that may be
  a.k_scale = const_cast<float*>(c.k_scale), a.v_scale = const_cast<float*>(c.v_scale);
  a.slots = (uint64_t)c.n_blocks * b.block_size;
  a.max_tokens = b.max_tokens;
  a.q_heads = q.ptr ? b.q_heads : 0, a.kv_heads = b.kv_heads;
  a.dim_shift = (uint32_t)__builtin_ctz(b.head_dim), a.units = b.head_dim / 16;
  a.heads_each = heads_each_for((uint64_t)b.max_tokens * a.q_heads * a.units);
  a.q_groups = (a.q_heads + a.heads_each - 1) / a.heads_each;
  const uint32_t numbers = b.block_size * b.head_dim;
  a.waves = std::min(std::max(numbers / 2048, 1u), 16u);
  const bool more = numbers > 32768;  // 4,096 of a block's numbers to a wavefront
  const uint32_t threads = a.waves == 1 ? 256 : a.waves * 64;
  const uint64_t qs = ((uint64_t)b.max_tokens * a.q_groups * a.units + threads - 1) / threads;
  const uint64_t tasks = plan_runs(a.runs, b.q_start, b.n_req, b.block_size, b.max_tokens,
                                   b.max_new ? std::min(b.max_new, b.max_tokens) : b.max_tokens) * b.kv_heads * 2;
  const uint64_t groups = a.waves == 1 ? (tasks + 3) / 4 : tasks;
  if (tasks > 0x7fffffffull || qs + groups > 0x7fffffffull || (qs + groups) * threads > 0xffffffffull)
    return fail(KV_ERR_UNSUPPORTED, "kv_paged_append: too many heads for one call");
  a.tasks = (uint32_t)tasks;
  a.run_share = ((groups << 32) + qs + groups - 1) / (qs + groups);  // all of them are `groups` in the end
  const uint32_t grid = (uint32_t)(qs + groups);
  const bool half = !r || r->layout == KV_ROPE_HALF, i8 = c.dtype == KV_DT_I8_BLOCK;
  if (dtype == KV_DT_BF16)
    i8 ? launch_append<bf16x8, I8>(a, half, more, grid, threads, s) : launch_append<bf16x8, Fp8>(a, half, more, grid, threads, s);
  else
    i8 ? launch_append<f16x8, I8>(a, half, more, grid, threads, s) : launch_append<f16x8, Fp8>(a, half, more, grid, threads, s);
  KV_HIP(hipGetLastError());
  return KV_OK;
}

kv_status paged_read(const kv_paged_batch& b, const kv_paged_cache& c, uint32_t dtype, const int32_t* row_start,
                     const int32_t* first, uint32_t max_rows, const kv_heads_view& k, const kv_heads_view& v,
                     hipStream_t s) {
  const int bytes = eight_bits(c.dtype) ? 1 : 2;
  ReadArgs a{};
  a.first = first, a.table = b.table, a.kv_len = b.kv_len;
  a.k = (uint16_t*)k.ptr, a.v = (uint16_t*)v.ptr;
  a.kt = k.token_stride, a.kh = k.head_stride, a.vt = v.token_stride, a.vh = v.head_stride;
  a.kc = (const uint8_t*)c.k, a.vc = (const uint8_t*)c.v;
  a.k_block = c.k_block_stride * bytes, a.v_block = c.v_block_stride * bytes;
  a.k_scale = c.k_scale, a.v_scale = c.v_scale;
  a.by_block = by_block(c.dtype);
  a.max_rows = max_rows, a.max_blocks = b.max_blocks, a.n_blocks = c.n_blocks;
  a.kv_heads = b.kv_heads, a.dim_shift = (uint32_t)__builtin_ctz(b.head_dim);
  const uint64_t runs = plan_runs(a.runs, row_start, b.n_req, b.block_size, max_rows, max_rows) * 2;
  const uint64_t numbers = (uint64_t)b.kv_heads * b.block_size * b.head_dim * bytes;
  a.each = (uint32_t)((numbers + 8191) / 8192);
  const bool few = runs * a.each < kFewTasks;
  if (few) a.each = (uint32_t)((numbers + 2047) / 2048);
  const uint64_t tasks = runs * a.each;
  if (tasks * 64 > 0xffffffffull) return fail(KV_ERR_UNSUPPORTED, "kv_paged_read: too many rows for one call");
  a.tasks = (uint32_t)tasks;
  const uint32_t grid = (uint32_t)((tasks + 3) / 4);
  if (dtype == KV_DT_BF16)
    launch_read<bf16x8>(a, c.dtype, few, grid, s);
  else
    launch_read<f16x8>(a, c.dtype, few, grid, s);
  KV_HIP(hipGetLastError());
  return KV_OK;
}

}  // namespace kv
