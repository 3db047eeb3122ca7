// kv_paged.h - internal declarations of the paged-cache operators (the public
// contract is include/kvpaged.h).
#pragma once

#include "../../include/kvpaged.h"
#include "kv_internal.h"

namespace kv {

// ---------------------------------------------------------------------------
// work list of the attention (kv_paged_plan writes it, kv_paged_attention
// walks it)
// ---------------------------------------------------------------------------
// The query rows of a request under one key/value head are its new tokens times
// the G query heads that read the head, token by token (row = token * G +
// head).  A tile is up to `rows` of them; a piece is a tile over a range of
// keys.  Long tiles are cut into pieces so that the chip is filled and no
// workgroup runs much longer than the others.  The pieces of a tile of few rows are
// joined by the workgroup that finishes last (`done` counts them per tile and
// head, and is 0 between calls), those of 128 rows by a second kernel.
constexpr uint32_t kKeyUnit = 64;  // key ranges of pieces are cut at multiples of this

struct PieceItem {
  int32_t req;        // table row
  int32_t q_start;    // the request's first token
  int32_t ctx;        // tokens cached before them
  int32_t row_end;    // rows of the request: new tokens * G
  int32_t row0;       // the tile's first row
  int32_t key_begin;  // multiple of kKeyUnit
  int32_t key_end;
  int32_t part;       // partial result to write, or -1: the tile's only piece
  int32_t split;      // the tile's place among the cut ones
  int32_t first_part, n_parts;
  int32_t pad;
};

struct SplitTile {
  int32_t q_start, row_end, row0;
  int32_t first_part, n_parts;
  int32_t pad[3];
};

struct WorkHeader {
  int32_t n_items, n_split;
  uint64_t sizes;  // work_sizes of the batch that was planned
  int32_t pad[60];
};

// Tells the sizes a work list is for: the attention does nothing with a list made
// for others (or with memory that holds none), rather than follow it out of bounds.
inline uint64_t work_sizes(const kv_paged_batch& b) {
  uint64_t h = 0x6b767061676564ull;
  for (uint64_t x : {(uint64_t)b.n_req, (uint64_t)b.max_tokens, (uint64_t)b.max_new, (uint64_t)b.block_size,
                     (uint64_t)b.max_blocks, (uint64_t)b.q_heads, (uint64_t)b.kv_heads, (uint64_t)b.head_dim,
                     (uint64_t)b.window}) {
    h = (h ^ x) * 0x9e3779b97f4a7c15ull;
    h ^= h >> 29;
  }
  return h;
}

struct WorkLayout {
  uint32_t rows;       // rows of a tile: 16, 32 or 64 (one tile a request) or 128
  uint32_t group;      // G
  uint32_t max_tiles;
  uint32_t pieces;     // pieces wanted per key/value head,
  uint32_t few_pieces; // and where they would otherwise be short
  uint32_t max_items, max_parts, max_split;
  uint64_t items, split, done, acc, ml, bytes;  // offsets from work; bytes in all
};

// A piece is no shorter than this many units: below it, the joining of partial
// results costs more than the shorter walk saves (16 contexts of 1,000 tokens: 16 us,
// with 2 units 21).  Only where two units a piece leave compute units idle all the same,
// a step of few tokens and short contexts, they are the faster ones (one context of
// 501 tokens: 7.3 us a call, with 4 units 8.3).
constexpr uint32_t kMinUnits = 4, kMinUnitsFew = 2;
// Tiles of 128 rows of heads of 64: 1,024 pieces instead of 512 where those would still be
// at least this long, as joining twice as many costs 2 to 7 us more (300 tokens over
// 60,000 cached ones, 24 / 4 heads: 156 us, with 512 pieces 199; 8 chunks of 128 tokens over
// 8,192: 105 and 111; 4 of 512 over 4,096, pieces of 51 units: 98 and 89; 16 of 100 over
// 1,000: 42 and 35).
constexpr uint32_t kLongUnits = 64;
// A tile is cut into no more pieces than this: one workgroup reads them all.  (One
// context of 131,072 tokens, 8 key/value heads of 128: 101 us with 32 pieces a head,
// 105 with 64, 130 with 192.)
constexpr int kMaxParts = 32;

inline WorkLayout work_layout(const kv_paged_batch& b) {
  WorkLayout w{};
  w.group = b.q_heads / b.kv_heads;
  const uint64_t most = (uint64_t)(b.max_new ? std::min(b.max_new, b.max_tokens) : b.max_tokens) * w.group;
  const uint32_t busy = std::min(b.n_req, b.max_tokens);
  // rows * head_dim is at most 4,096 in the kernel for few rows: a wavefront holds
  // the whole tile's results, and more would not leave room for its loads
  const uint32_t few = most <= 16 ? 16 : most <= 32 ? 32 : 64;
  w.rows = most <= 64 && few * b.head_dim <= 4096 ? few : 128;
  w.max_tiles = w.rows < 128 ? busy : (uint32_t)((uint64_t)b.max_tokens * w.group / 128) + busy;
  // Few rows: 1,024 pieces, twice what the chip holds at a time, so that ragged ones fill
  // it evenly (64 chats of up to 16,000 tokens: 115 us, with 512 pieces 127, with three
  // times as many 119).  128 rows: 512, what the chip holds of heads of 128, as the pieces' partial
  // results are large (8 chunks of 128 tokens over 8,192 cached ones: 203 us, with 1,024
  // pieces 217; ragged chunks with a window: the same with either).
  // Of heads of 64 the chip holds 1,024; so many where kLongUnits says.
  w.pieces = ((w.rows < 128 || b.head_dim == 64 ? 1024 : 512) + b.kv_heads - 1) / b.kv_heads;
  w.few_pieces = w.rows < 128 ? w.pieces : (512 + b.kv_heads - 1) / b.kv_heads;
  w.max_items = w.max_tiles + w.pieces;
  w.max_parts = 2 * w.pieces;
  w.max_split = w.pieces;
  auto up = [](uint64_t x) { return (x + 255) / 256 * 256; };
  w.items = sizeof(WorkHeader);
  w.split = up(w.items + (uint64_t)w.max_items * sizeof(PieceItem));
  w.done = up(w.split + (uint64_t)w.max_split * sizeof(SplitTile));
  w.acc = up(w.done + (uint64_t)w.max_split * b.kv_heads * sizeof(uint32_t));
  const uint64_t rows = (uint64_t)w.max_parts * b.kv_heads * w.rows;
  w.ml = up(w.acc + rows * b.head_dim * sizeof(float));
  w.bytes = up(w.ml + rows * 2 * sizeof(float));
  return w;
}

// Scales by block of tokens and head, written with what they scale.
inline bool by_block(uint32_t kept) { return kept == KV_DT_FP8_BLOCK || kept == KV_DT_I8_BLOCK; }
inline bool eight_bits(uint32_t kept) { return kept == KV_DT_FP8 || by_block(kept); }

// The frequencies of a rotation, in 2^-64 turns a token.
struct RopeTable {
  const uint64_t* turn = nullptr;  // device [rot_dim / 2]
  float magnitude = 1.0f;
  uint32_t rot_dim = 0, layout = KV_ROPE_HALF;
};

kv_status rope_apply(const RopeTable& r, uint32_t dtype, const kv_heads_view& x,
                     const kv_heads_view& y, const int32_t* pos, uint32_t n_tokens,
                     uint32_t n_heads, uint32_t head_dim, bool backward, hipStream_t s);
kv_status paged_plan(const kv_paged_batch& b, const WorkLayout& w, hipStream_t s);
// r NULL: no rotation
kv_status paged_append(const kv_paged_batch& b, const kv_paged_cache& c, const RopeTable* r,
                       uint32_t dtype, const kv_heads_view& q, const kv_heads_view& q_out,
                       const kv_heads_view& k, const kv_heads_view& v, hipStream_t s);
// c of KV_DT_FP8_BLOCK or KV_DT_I8_BLOCK
kv_status paged_append_block(const kv_paged_batch& b, const kv_paged_cache& c, const RopeTable* r,
                             uint32_t dtype, const kv_heads_view& q, const kv_heads_view& q_out,
                             const kv_heads_view& k, const kv_heads_view& v, hipStream_t s);
kv_status paged_read(const kv_paged_batch& b, const kv_paged_cache& c, uint32_t dtype,
                     const int32_t* row_start, const int32_t* first, uint32_t max_rows,
                     const kv_heads_view& k, const kv_heads_view& v, hipStream_t s);
kv_status paged_attention(const kv_paged_batch& b, const WorkLayout& w, const kv_paged_cache& c,
                          uint32_t dtype, const kv_heads_view& q, const kv_heads_view& out,
                          float* lse, float scale, hipStream_t s);

}  // namespace kv
