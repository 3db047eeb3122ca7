// k_attn.hip - attention of a step's new tokens over a paged KV cache of 16 bits, or of 8
// with a scale for each head, and the launches of every kind (kernels: attn_kernels.h).
#include "attn_kernels.h"

namespace kv {
namespace attn {

template kv_status launch_dim<BF16, kSixteen>(const AttnArgs&, uint32_t, uint32_t, uint32_t, hipStream_t);
template kv_status launch_dim<F16, kSixteen>(const AttnArgs&, uint32_t, uint32_t, uint32_t, hipStream_t);
template kv_status launch_dim<BF16, kFp8Head>(const AttnArgs&, uint32_t, uint32_t, uint32_t, hipStream_t);
template kv_status launch_dim<F16, kFp8Head>(const AttnArgs&, uint32_t, uint32_t, uint32_t, hipStream_t);
// built by k_attn_block.hip
extern template kv_status launch_dim<BF16, kFp8Block>(const AttnArgs&, uint32_t, uint32_t, uint32_t, hipStream_t);
extern template kv_status launch_dim<F16, kFp8Block>(const AttnArgs&, uint32_t, uint32_t, uint32_t, hipStream_t);
extern template kv_status launch_dim<BF16, kI8Block>(const AttnArgs&, uint32_t, uint32_t, uint32_t, hipStream_t);
extern template kv_status launch_dim<F16, kI8Block>(const AttnArgs&, uint32_t, uint32_t, uint32_t, hipStream_t);

template <class T>
kv_status launch_kind(uint32_t kept, const AttnArgs& a, uint32_t dim, uint32_t rows, uint32_t grid, hipStream_t s) {
  switch (kept) {
    case KV_DT_FP8: return launch_dim<T, kFp8Head>(a, dim, rows, grid, s);
    case KV_DT_FP8_BLOCK: return launch_dim<T, kFp8Block>(a, dim, rows, grid, s);
    case KV_DT_I8_BLOCK: return launch_dim<T, kI8Block>(a, dim, rows, grid, s);
    default: return launch_dim<T, kSixteen>(a, dim, rows, grid, s);
  }
}

}  // namespace attn

using namespace attn;

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
  const kv_status st = dtype == KV_DT_BF16 ? launch_kind<BF16>(c.dtype, a, b.head_dim, w.rows, (uint32_t)grid, s)
                                           : launch_kind<F16>(c.dtype, a, b.head_dim, w.rows, (uint32_t)grid, s);
  if (st != KV_OK) return st;
  // tiles of few rows are joined already, and none is cut when the whole table is
  // at most one piece long
  if (w.rows < 128) return KV_OK;
  if ((uint64_t)b.max_blocks * b.block_size <= kMinUnits * kKeyUnit) return KV_OK;
  const bool by_head = c.dtype == KV_DT_FP8;
  const dim3 join(std::min<uint32_t>(w.max_split * b.kv_heads * 4, 4096));
  if (dtype == KV_DT_BF16)
    hipLaunchKernelGGL((k_attn_join<BF16, false>), join, dim3(256), 0, s, a, b.head_dim, (uint32_t)by_head);
  else if (by_block(c.dtype))
    hipLaunchKernelGGL((k_attn_join<F16, true>), join, dim3(256), 0, s, a, b.head_dim, 0u);
  else
    hipLaunchKernelGGL((k_attn_join<F16, false>), join, dim3(256), 0, s, a, b.head_dim, (uint32_t)by_head);
  KV_HIP(hipGetLastError());
  return KV_OK;
}

}  // namespace kv
