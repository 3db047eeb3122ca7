// k_plan.hip - block tables, cache slots, positions and the attention's work
// list of a step, from the requests' lengths.
//
// One launch: every workgroup works out the requests' first tokens and first
// new blocks for itself (two prefix sums over at most 4,096 requests, kept in
// LDS), so none waits for another.  Workgroup 0 writes the per-request arrays
// and the work list, the others four tokens a thread; a token finds its request
// by binary search, and the token at the start of a new block enters the block
// in the table.  Whole numbers throughout; bound by latency (the chain of
// loads, sums and stores of one workgroup) up to some 10^5 tokens: a step of 64
// single tokens takes 5.9 us a call, one of 1,000 prompts of up to 800 tokens
// 9.9 us, where an empty launch takes 4.
#include "kv_device.h"
#include "kv_paged.h"

namespace kv {
namespace {


constexpr uint32_t kClasses = 64;  // of piece lengths: one for each lane of a wavefront

struct PlanArgs {
  kv_paged_batch b;
  uint32_t shift;  // log2 of block_size
  uint32_t group, rows, pieces, few_pieces, max_items, max_parts, max_split;
  uint64_t sizes;
  WorkHeader* head;
  PieceItem* items;
  SplitTile* split;
  uint32_t* done;
};

// Tiles are numbered request by request, a request's last rows first.
struct Tile {
  int32_t req, row0, row_end, key_begin, key_end, units;
};

// A tile, its first piece's place among those of its batch, and where its partial
// results go.
struct Cut {
  Tile x;
  uint32_t at, cut, split_at, part_at;
};

__device__ __forceinline__ Tile tile_of(const PlanArgs& a, const int32_t* first_tile, const int32_t* start,
                                        const int32_t* ctx, int32_t t) {
  // the request: the last one whose first tile is not after t, among those with tiles
  int lo = 0, hi = (int)a.b.n_req;  // first_tile[lo] <= t < first_tile[hi]
  while (hi - lo > 1) {
    const int mid = (lo + hi) / 2;
    if (first_tile[mid] <= t)
      lo = mid;
    else
      hi = mid;
  }
  Tile x;
  x.req = lo;
  const int32_t tiles = first_tile[lo + 1] - first_tile[lo];
  x.row_end = (start[lo + 1] - start[lo]) * (int32_t)a.group;
  x.row0 = (tiles - 1 - (t - first_tile[lo])) * (int32_t)a.rows;
  const int32_t t0 = x.row0 / (int32_t)a.group;
  const int32_t t1 = (min(x.row0 + (int32_t)a.rows, x.row_end) - 1) / (int32_t)a.group;
  x.key_end = ctx[lo] + t1 + 1;
  x.key_begin = a.b.window ? max(0, ctx[lo] + t0 + 1 - (int32_t)a.b.window) / (int32_t)kKeyUnit * (int32_t)kKeyUnit : 0;
  x.units = (x.key_end - x.key_begin + (int32_t)kKeyUnit - 1) / (int32_t)kKeyUnit;
  return x;
}

template <int kNT>
__global__ __launch_bounds__(kNT) void k_paged_plan(PlanArgs a) {
  constexpr uint32_t kTokensEach = 4 * kNT;
  // start: first token of each request; ctx: its cached tokens (0 where its
  // lengths are refused); fresh: its first new block's place in the free list
  // (workgroup 0: then its first tile)
  extern __shared__ int32_t lds[];
  __shared__ uint32_t sh[2][2 * kNT / 64];  // taken in turn by the sums, which then need one barrier each
  const uint32_t R = a.b.n_req, T = a.b.max_tokens, bs = a.b.block_size;
  int32_t* start = lds;
  int32_t* ctx = start + R + 1;
  int32_t* fresh = ctx + R;
  const int tid = threadIdx.x;
  const int32_t most_new = (int32_t)(a.b.max_new ? min(a.b.max_new, T) : T);
  const int64_t most_len = (int64_t)a.b.max_blocks * bs;

  uint32_t tokens = 0, blocks = 0, flags = 0;  // tokens: at most 2^12 * 2^19
  uint32_t last_start = 0;                     // of the first request past max_tokens
  for (uint32_t r0 = 0; r0 < R; r0 += kNT) {
    const uint32_t r = r0 + tid;
    int32_t c = 0, n = 0;
    if (r < R) {
      c = a.b.ctx_len[r];
      n = a.b.new_len[r];
      if (c < 0 || n < 0 || n > most_new || (int64_t)c + n > most_len) {
        c = n = 0;
        flags |= KV_PLAN_BAD_LENGTH;
      }
    }
    uint32_t sum;
    const uint32_t before = block_excl_scan_u32<kNT, false>((uint32_t)n, sh[0], sum);
    const uint32_t at = tokens + before;
    if (at + n > T) {
      flags |= KV_PLAN_TOKENS;
      if (at <= T) last_start = max(last_start, at);
      n = 0;
    }
    if (r < R) {
      start[r] = at > T ? -1 : (int32_t)at;  // -1: set below
      ctx[r] = c;
    }
    const uint32_t need = r < R ? (uint32_t)((c + n + bs - 1) >> a.shift) - (uint32_t)((c + bs - 1) >> a.shift) : 0u;
    uint32_t total;
    const uint32_t place = block_excl_scan_u32<kNT, false>(need, sh[1], total);
    if (r < R) fresh[r] = (int32_t)(blocks + place);
    tokens += sum;
    blocks += total;
  }
  // the step's number of tokens, and the flags of all threads
  __shared__ uint32_t all[2];
  if (tid < 2) all[tid] = 0;
  __syncthreads();
  if (flags) atomicOr(&all[0], flags);
  if (last_start) atomicMax(&all[1], last_start);
  __syncthreads();
  flags = all[0];
  const int32_t n_tokens = flags & KV_PLAN_TOKENS ? (int32_t)all[1] : (int32_t)tokens;
  if (tid == 0) start[R] = n_tokens;
  for (uint32_t r = tid; r < R; r += kNT)
    if (start[r] < 0 || start[r] > n_tokens) start[r] = n_tokens;
  __syncthreads();
  const bool take = a.b.free_list != nullptr;

  if (blockIdx.x > 0) {
    const uint32_t base = (blockIdx.x - 1) * kTokensEach;
    for (uint32_t i = tid; i < kTokensEach; i += kNT) {
      const uint32_t t = base + i;
      if (t >= T) return;
      if ((int32_t)t >= n_tokens) {
        a.b.slot[t] = -1;
        a.b.pos[t] = 0;
        continue;
      }
      int lo = 0, hi = (int)R;  // start[lo] <= t < start[hi]
      while (hi - lo > 1) {
        const int mid = (lo + hi) / 2;
        if (start[mid] <= (int32_t)t)
          lo = mid;
        else
          hi = mid;
      }
      const int32_t p = ctx[lo] + (int32_t)t - start[lo];
      const int32_t col = p >> a.shift, have = (int32_t)((ctx[lo] + bs - 1) >> a.shift);
      int32_t* row = a.b.table + (uint64_t)lo * a.b.max_blocks;
      int32_t page;
      if (take && col >= have) {
        const uint32_t place = (uint32_t)(fresh[lo] + col - have);
        page = place < a.b.n_free ? a.b.free_list[place] : -1;
        if ((p & (int32_t)(bs - 1)) == 0) row[col] = page;
      } else {
        page = row[col];
      }
      a.b.pos[t] = p;
      a.b.slot[t] = page < 0 ? -1 : (int64_t)page * bs + (p & (int32_t)(bs - 1));
    }
    return;
  }

  for (uint32_t r = tid; r <= R; r += kNT) {
    a.b.q_start[r] = start[r];
    if (r < R) a.b.kv_len[r] = ctx[r] + start[r + 1] - start[r];
  }
  if (tid == 0) {
    const uint32_t needed = take ? blocks : 0u, taken = min(needed, a.b.n_free);
    a.b.result[0] = n_tokens;
    a.b.result[1] = (int32_t)needed;
    a.b.result[2] = (int32_t)taken;
    a.b.result[3] = (int32_t)(flags | (taken < needed ? (uint32_t)KV_PLAN_BLOCKS : 0u));
  }
  // tiles
  __syncthreads();
  int32_t* first_tile = fresh;  // [R + 1]: the launch leaves room for one more
  uint32_t n_tiles = 0;
  for (uint32_t r0 = 0; r0 < R; r0 += kNT) {
    const uint32_t r = r0 + tid;
    const uint32_t rows = r < R ? (uint32_t)(start[r + 1] - start[r]) * a.group : 0u;
    uint32_t sum;
    const uint32_t before = block_excl_scan_u32<kNT, false>((rows + a.rows - 1) / a.rows, sh[(r0 / kNT) & 1], sum);
    if (r < R) first_tile[r] = (int32_t)(n_tiles + before);
    n_tiles += sum;
  }
  if (tid == 0) first_tile[R] = (int32_t)n_tiles;
  __syncthreads();
  // how long a piece may be
  __shared__ unsigned long long total_units;
  __shared__ uint32_t most_units, in_class[kClasses];
  if (tid == 0) total_units = 0, most_units = 0;
  if (tid < kClasses) in_class[tid] = 0;
  __syncthreads();
  // each thread keeps its first tiles: finding one is a search
  constexpr uint32_t kKeep = 2;
  Tile kept[kKeep]{};
  auto tile_at = [&](uint32_t t) { return tile_of(a, first_tile, start, ctx, (int32_t)t); };
  auto each_tile = [&](auto&& f) {
#pragma unroll
    for (uint32_t i = 0; i < kKeep; ++i)
      if (tid + i * kNT < n_tiles) f(kept[i]);
    for (uint32_t t = tid + kKeep * kNT; t < n_tiles; t += kNT) f(tile_at(t));
  };
#pragma unroll
  for (uint32_t i = 0; i < kKeep; ++i)
    if (tid + i * kNT < n_tiles) kept[i] = tile_at(tid + i * kNT);
  unsigned long long mine = 0;
  uint32_t most = 0;
  each_tile([&](const Tile& y) {
    mine += (uint32_t)y.units;
    most = max(most, (uint32_t)y.units);
  });
  mine = wave_sum(mine);
#pragma unroll
  for (int d = 1; d < 64; d <<= 1) most = max(most, (uint32_t)__shfl_xor((int)most, d, 64));
  if (lane_id() == 0 && mine) atomicAdd(&total_units, mine), atomicMax(&most_units, most);
  __syncthreads();
  const uint32_t least = a.rows < 128 && total_units * a.b.kv_heads <= 256 ? kMinUnitsFew : kMinUnits;
  uint32_t longest = (uint32_t)((total_units + a.few_pieces - 1) / a.few_pieces);
  if (longest >= kLongUnits) longest = (uint32_t)((total_units + a.pieces - 1) / a.pieces);
  longest = max(longest, least);
  auto cut_of = [&](const Tile& y) { return min(((uint32_t)y.units + longest - 1) / longest, (uint32_t)kMaxParts); };
  // Long pieces go first, so that the last ones to end are short: the list is ordered
  // by classes of length (within one, in any order: results do not depend on it).
  uint32_t shift = 0;
  while ((max(longest, most_units / kMaxParts + 1) >> shift) >= kClasses) ++shift;
  auto class_of = [&](uint32_t units) { return kClasses - 1 - min(units >> shift, kClasses - 1); };
  each_tile([&](const Tile& y) {
    const uint32_t cut = cut_of(y), each = (uint32_t)y.units / cut, more = (uint32_t)y.units % cut;
    if (more) atomicAdd(&in_class[class_of(each + 1)], more);
    atomicAdd(&in_class[class_of(each)], cut - more);
  });
  __syncthreads();
  uint32_t n_items = 0;
  if (tid < 64) {
    const uint32_t n = in_class[tid], upto = wave_incl_scan_u32(n);
    in_class[tid] = upto - n;  // then: where the class's next piece goes
    n_items = (uint32_t)__shfl((int)upto, 63, 64);
  }
  __syncthreads();
  // kNT tiles at a time: a thread writes its tile where it is one piece; the pieces of
  // those that are cut are shared out among all threads
  __shared__ Cut cuts[kNT];
  auto put = [&](const Cut& c, uint32_t i) {
    // equal pieces: the first `more` are one unit longer
    const uint32_t each = (uint32_t)c.x.units / c.cut, more = (uint32_t)c.x.units % c.cut;
    const uint32_t from = i * each + min(i, more), last = from + each + (i < more ? 1u : 0u);
    PieceItem it;
    it.req = c.x.req;
    it.q_start = start[c.x.req];
    it.ctx = ctx[c.x.req];
    it.row_end = c.x.row_end;
    it.row0 = c.x.row0;
    it.key_begin = c.x.key_begin + (int32_t)(from * kKeyUnit);
    it.key_end = min(c.x.key_end, c.x.key_begin + (int32_t)(last * kKeyUnit));
    it.part = c.cut > 1 ? (int32_t)min(c.part_at + i, a.max_parts - 1) : -1;
    it.split = (int32_t)min(c.split_at, a.max_split - 1);
    it.first_part = (int32_t)c.part_at;
    it.n_parts = (int32_t)c.cut;
    it.pad = 0;
    const uint32_t to = atomicAdd(&in_class[class_of(last - from)], 1u);
    if (to < a.max_items) a.items[to] = it;
  };
  uint32_t n_split = 0, n_parts = 0;
  auto batch = [&](uint32_t t0, const Tile& y) {
    const uint32_t cut = t0 + tid < n_tiles ? cut_of(y) : 0u;
    uint32_t at, split_at, parts, splits;
    block_excl_scan2_u32<kNT, false>(cut > 1 ? cut : 0u, cut > 1 ? 1u : 0u, sh[(t0 / kNT) & 1], at, split_at, parts, splits);
    const Cut c{y, at, cut, n_split + split_at, n_parts + at};
    if (cut == 1) put(c, 0);
    if (parts) {
      cuts[tid] = c;
      if (cut > 1 && c.split_at < a.max_split) {
        SplitTile z{};
        z.q_start = start[y.req];
        z.row_end = y.row_end;
        z.row0 = y.row0;
        z.first_part = (int32_t)c.part_at;
        z.n_parts = (int32_t)cut;
        a.split[c.split_at] = z;
      }
      __syncthreads();
      for (uint32_t k = tid; k < parts; k += kNT) {
        int lo = 0, hi = kNT;  // the last cut tile whose first piece is not after k
        while (hi - lo > 1) {
          const int mid = (lo + hi) / 2;
          if (cuts[mid].at <= k)
            lo = mid;
          else
            hi = mid;
        }
        put(cuts[lo], k - cuts[lo].at);
      }
      __syncthreads();  // cuts
    }
    n_split += splits, n_parts += parts;
  };
#pragma unroll
  for (uint32_t i = 0; i < kKeep; ++i)
    if (i * kNT < n_tiles) batch(i * kNT, kept[i]);
  for (uint32_t t0 = kKeep * kNT; t0 < n_tiles; t0 += kNT) batch(t0, t0 + tid < n_tiles ? tile_at(t0 + tid) : Tile{});
  const uint32_t counters = min(n_split, a.max_split) * a.b.kv_heads;
  for (uint32_t i = tid; i < counters; i += kNT) a.done[i] = 0;
  if (tid == 0) {
    a.head->n_items = (int32_t)min(n_items, a.max_items);
    a.head->n_split = (int32_t)min(n_split, a.max_split);
    a.head->sizes = a.sizes;
  }
}

}  // namespace

kv_status paged_plan(const kv_paged_batch& b, const WorkLayout& w, hipStream_t s) {
  PlanArgs a{};
  a.b = b;
  a.shift = (uint32_t)__builtin_ctz(b.block_size);
  a.group = w.group, a.rows = w.rows, a.pieces = w.pieces, a.few_pieces = w.few_pieces;
  a.max_items = w.max_items, a.max_parts = w.max_parts, a.max_split = w.max_split;
  a.sizes = work_sizes(b);
  uint8_t* at = (uint8_t*)b.work;
  a.head = (WorkHeader*)at;
  a.items = (PieceItem*)(at + w.items);
  a.split = (SplitTile*)(at + w.split);
  a.done = (uint32_t*)(at + w.done);
  // Threads of a workgroup: few requests and tiles are done in one round of 256, whose
  // barriers are the cheaper ones (a step of 64 chats: 6.0 us a call, 7.0 with 1,024
  // threads); more of them need the threads (1,000 ragged prompts: 10.0 us, 22.9 with 256).
  const uint32_t threads = b.n_req <= 256 && w.max_tiles <= 512 ? 256 : 1024;
  const uint32_t grid = 1 + (b.max_tokens + 4 * threads - 1) / (4 * threads);
  // three arrays of n_req and two ends: at most 49 KB
  const size_t lds = (3 * b.n_req + 2) * sizeof(int32_t);
  if (threads == 256)
    hipLaunchKernelGGL(k_paged_plan<256>, dim3(grid), dim3(256), lds, s, a);
  else
    hipLaunchKernelGGL(k_paged_plan<1024>, dim3(grid), dim3(1024), lds, s, a);
  KV_HIP(hipGetLastError());
  return KV_OK;
}

}  // namespace kv
