// k_plan.hip - block tables, cache slots, positions and the attention's work
// list of a step, from the requests' lengths.
//
// One launch: every workgroup works out the requests' first tokens and first
// new blocks for itself (two prefix sums over at most 4,096 requests, kept in
// LDS), so none waits for another.  Workgroup 0 writes the per-request arrays
// and the work list, the others four tokens a thread; a token finds its request
// by binary search, and the token at the start of a new block enters the block
// in the table.  Whole numbers throughout; bound by latency (the chain of
// loads, sums and stores of one workgroup) up to some 10^5 tokens.
#include "kv_device.h"
#include "kv_paged.h"

namespace kv {
namespace {


struct PlanArgs {
  kv_paged_batch b;
  uint32_t shift;  // log2 of block_size
  uint32_t group, rows, pieces, max_items, max_parts, max_split;
  WorkHeader* head;
  PieceItem* items;
  SplitTile* split;
  uint32_t* done;
};

// Tiles are numbered request by request, a request's last rows first: they see
// the most keys, and the longest pieces should start first.
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
  if (tid == 0) total_units = 0;
  __syncthreads();
  unsigned long long mine = 0;
  Tile x{};
  for (uint32_t t = tid; t < n_tiles; t += kNT) {
    x = tile_of(a, first_tile, start, ctx, (int32_t)t);
    mine += (uint32_t)x.units;
  }
  if (mine) atomicAdd(&total_units, mine);
  __syncthreads();
  const uint32_t longest = max(kMinUnits, (uint32_t)((total_units + a.pieces - 1) / a.pieces));
  // kNT tiles at a time; their pieces are shared out among all threads
  __shared__ Cut cuts[kNT];
  uint32_t n_items = 0, n_split = 0, n_parts = 0;
  for (uint32_t t0 = 0; t0 < n_tiles; t0 += kNT) {
    const uint32_t t = t0 + tid;
    uint32_t cut = 0;
    if (t < n_tiles) {
      if (n_tiles > (uint32_t)kNT) x = tile_of(a, first_tile, start, ctx, (int32_t)t);
      cut = min(((uint32_t)x.units + longest - 1) / longest, (uint32_t)kMaxParts);
    }
    uint32_t at, split_at, s0, s1, s2;
    block_excl_scan2_u32<kNT, false>(cut, cut > 1 ? 1u : 0u, sh[0], at, split_at, s0, s1);
    const uint32_t part_at = n_parts + block_excl_scan_u32<kNT, false>(cut > 1 ? cut : 0u, sh[1], s2);
    split_at += n_split;
    cuts[tid] = Cut{x, at, cut, split_at, part_at};
    if (cut > 1 && split_at < a.max_split) {
      SplitTile y{};
      y.q_start = start[x.req];
      y.row_end = x.row_end;
      y.row0 = x.row0;
      y.first_part = (int32_t)part_at;
      y.n_parts = (int32_t)cut;
      a.split[split_at] = y;
    }
    __syncthreads();
    for (uint32_t k = tid; k < s0 && n_items + k < a.max_items; k += kNT) {
      int lo = 0, hi = kNT;  // cuts[lo].at <= k, and the first of those after it is beyond k
      while (hi - lo > 1) {
        const int mid = (lo + hi) / 2;
        if (cuts[mid].at <= k)
          lo = mid;
        else
          hi = mid;
      }
      const Cut c = cuts[lo];
      // equal pieces: the first `more` are one unit longer
      const uint32_t i = k - c.at, each = (uint32_t)c.x.units / c.cut, more = (uint32_t)c.x.units % c.cut;
      const uint32_t from = i * each + min(i, more), to = from + each + (i < more ? 1u : 0u);
      PieceItem it;
      it.req = c.x.req;
      it.q_start = start[c.x.req];
      it.ctx = ctx[c.x.req];
      it.row_end = c.x.row_end;
      it.row0 = c.x.row0;
      it.key_begin = c.x.key_begin + (int32_t)(from * kKeyUnit);
      it.key_end = min(c.x.key_end, c.x.key_begin + (int32_t)(to * kKeyUnit));
      it.part = c.cut > 1 ? (int32_t)min(c.part_at + i, a.max_parts - 1) : -1;
      it.split = (int32_t)min(c.split_at, a.max_split - 1);
      it.first_part = (int32_t)c.part_at;
      it.n_parts = (int32_t)c.cut;
      it.pad = 0;
      a.items[n_items + k] = it;
    }
    n_items += s0, n_split += s1, n_parts += s2;
    __syncthreads();  // cuts
  }
  const uint32_t counters = min(n_split, a.max_split) * a.b.kv_heads;
  for (uint32_t i = tid; i < counters; i += kNT) a.done[i] = 0;
  if (tid == 0) {
    a.head->n_items = (int32_t)min(n_items, a.max_items);
    a.head->n_split = (int32_t)min(n_split, a.max_split);
  }
}

}  // namespace

kv_status paged_plan(const kv_paged_batch& b, const WorkLayout& w, hipStream_t s) {
  PlanArgs a{};
  a.b = b;
  a.shift = (uint32_t)__builtin_ctz(b.block_size);
  a.group = w.group, a.rows = w.rows, a.pieces = w.pieces;
  a.max_items = w.max_items, a.max_parts = w.max_parts, a.max_split = w.max_split;
  uint8_t* at = (uint8_t*)b.work;
  a.head = (WorkHeader*)at;
  a.items = (PieceItem*)(at + w.items);
  a.split = (SplitTile*)(at + w.split);
  a.done = (uint32_t*)(at + w.done);
  // Threads of a workgroup: few requests and tiles are done in one round of 256, whose
  // barriers are the cheaper ones (a step of 64 chats: 7.4 us a call, 8.8 with 1,024
  // threads); more of them need the threads (1,000 ragged prompts: 15.6 us, 26.7 with 256).
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
