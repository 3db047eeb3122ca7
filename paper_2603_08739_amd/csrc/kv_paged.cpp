// kv_paged.cpp - the C entry points of the paged-cache operators: argument
// checks, the rotation handle and launch order (include/kvpaged.h).
#include "kv_paged.h"

#include <cmath>
#include <mutex>
#include <new>
#include <set>

struct kv_rope {
  kv::RopeTable table;
  void* mem = nullptr;
  int device = 0;
};

namespace kv {
namespace {

std::mutex g_rope_mu;
std::set<const void*> g_ropes;  // live rotations

bool rope_is_live(const kv_rope* r) {
  std::lock_guard<std::mutex> lk(g_rope_mu);
  return g_ropes.count(r) != 0;
}

// The table lies on the device it was made on.
bool rope_is_elsewhere(const kv_rope* r) {
  int dev = -1;
  return hipGetDevice(&dev) != hipSuccess || dev != r->device;
}

kv_status invalid(const char* who, const char* what) {
  return fail(KV_ERR_INVALID, std::string(who) + ": " + what);
}

// C++ exceptions (allocation of host memory) end here.
template <class F>
kv_status guarded(const char* who, F&& f) {
  try {
    return f();
  } catch (const std::bad_alloc&) {
    return fail(KV_ERR_NOMEM, std::string(who) + ": out of host memory");
  } catch (...) {
    return fail(KV_ERR_DEVICE, std::string(who) + ": unexpected failure");
  }
}

bool aligned(const void* p, uintptr_t to) { return ((uintptr_t)p & (to - 1)) == 0; }

const char* check_view(const kv_heads_view& v) {
  if (!v.ptr) return "a view's pointer is NULL";
  if (!aligned(v.ptr, 16)) return "a view's pointer is not 16-byte aligned";
  if (v.token_stride % 8 || v.head_stride % 8) return "a view's strides must be multiples of 8 elements";
  return nullptr;
}

const char* check_sizes(const kv_paged_batch& b) {
  if (b.n_req < 1 || b.n_req > KV_PAGED_MAX_REQ) return "n_req out of range";
  if (b.max_tokens < 1 || b.max_tokens > KV_PAGED_MAX_TOKENS) return "max_tokens out of range";
  if (b.block_size != 16 && b.block_size != 32 && b.block_size != 64 && b.block_size != 128 && b.block_size != 256)
    return "block_size must be 16, 32, 64, 128 or 256";
  if (b.max_blocks < 1 || (uint64_t)b.max_blocks * b.block_size > (1ull << 30)) return "max_blocks out of range";
  if (b.kv_heads < 1 || b.kv_heads > 1024) return "kv_heads out of range";
  if (b.q_heads < 1 || b.q_heads % b.kv_heads || b.q_heads > 65536) return "q_heads must be a multiple of kv_heads, at most 65536";
  if ((uint64_t)b.max_tokens * (b.q_heads / b.kv_heads) > 0x7fffffffull) return "max_tokens * (q_heads / kv_heads) out of range";
  if (b.head_dim != 64 && b.head_dim != 128 && b.head_dim != 256) return "head_dim must be 64, 128 or 256";
  if (b.window > (1u << 30)) return "window out of range";
  return nullptr;
}

const char* check_batch(const kv_paged_batch& b) {
  if (const char* e = check_sizes(b)) return e;
  if (!b.ctx_len || !b.new_len || !b.table || !b.q_start || !b.kv_len || !b.slot || !b.pos || !b.result || !b.work)
    return "a pointer of the batch is NULL";
  for (const void* p : {(const void*)b.ctx_len, (const void*)b.new_len, (const void*)b.table, (const void*)b.free_list,
                        (const void*)b.q_start, (const void*)b.kv_len, (const void*)b.pos, (const void*)b.result})
    if (!aligned(p, 4)) return "an int32 array of the batch is misaligned";
  if (!aligned(b.slot, 8)) return "slot is misaligned";
  if (!aligned(b.work, 256)) return "work is not 256-byte aligned";
  if (b.work_bytes < work_layout(b).bytes) return "work_bytes is less than kv_paged_work_bytes";
  return nullptr;
}

const char* check_cache(const kv_paged_cache& c, const kv_paged_batch& b, uint32_t dtype) {
  if (!c.k || !c.v) return "a cache pointer is NULL";
  if (!aligned(c.k, 16) || !aligned(c.v, 16)) return "a cache pointer is not 16-byte aligned";
  const int64_t block = (int64_t)b.kv_heads * b.block_size * b.head_dim;
  for (int64_t st : {c.k_block_stride, c.v_block_stride})
    if (st < block || st % 16) return "a block stride is below a block's elements or no multiple of 16";
  if (c.n_blocks < 1 || c.n_blocks > (1u << 30)) return "n_blocks out of range";
  if (dtype != KV_DT_BF16 && dtype != KV_DT_F16) return "dtype must be KV_DT_BF16 or KV_DT_F16";
  if (!eight_bits(c.dtype) && c.dtype != dtype) return "the cache's dtype must be one of 8 bits or that of the heads";
  if (!eight_bits(c.dtype) && (c.k_scale || c.v_scale)) return "scales belong to a cache of 8 bits";
  if (by_block(c.dtype) && (!c.k_scale || !c.v_scale)) return "a cache with scales by block needs both scale arrays";
  if (!aligned(c.k_scale, 4) || !aligned(c.v_scale, 4)) return "a scale array is misaligned";
  return nullptr;
}

}  // namespace
}  // namespace kv

using kv::fail;
using kv::guarded;
using kv::invalid;

extern "C" kv_status kv_rope_create(const kv_rope_desc* d, kv_rope** out) {
  const char* who = "kv_rope_create";
  return guarded(who, [&]() -> kv_status {
    if (!out) return invalid(who, "out is NULL");
    *out = nullptr;
    if (!d) return invalid(who, "desc is NULL");
    if (d->rot_dim < 16 || d->rot_dim > 256 || d->rot_dim % 16) return invalid(who, "rot_dim must be a multiple of 16 in 16..256");
    if (d->layout > KV_ROPE_INTERLEAVED) return invalid(who, "unknown layout");
    if (d->scaling > KV_ROPE_BY_PARTS) return invalid(who, "unknown scaling");
    if (!(d->base > 1) || !std::isfinite(d->base)) return invalid(who, "base must be > 1 and finite");
    // as the kernels hold it
    if (!std::isfinite((float)d->magnitude) || (float)d->magnitude == 0) return invalid(who, "magnitude must be finite and not 0 in 32 bits");
    if (d->scaling != KV_ROPE_PLAIN && (!(d->factor >= 1) || !std::isfinite(d->factor))) return invalid(who, "factor must be >= 1 and finite");
    if (d->scaling == KV_ROPE_BY_PARTS && (!d->original_len || !(d->slow >= 0) || !(d->fast > d->slow) || !std::isfinite(d->fast)))
      return invalid(who, "BY_PARTS needs original_len > 0 and fast > slow >= 0");
    const double kTurn = 6.283185307179586476925;
    std::vector<uint64_t> turn(d->rot_dim / 2);
    for (uint32_t i = 0; i < turn.size(); ++i) {
      double f = std::pow(d->base, -2.0 * i / d->rot_dim);
      if (d->scaling == KV_ROPE_LINEAR) f /= d->factor;
      if (d->scaling == KV_ROPE_BY_PARTS) {
        const double g = std::min(1.0, std::max(0.0, (d->original_len * f / kTurn - d->slow) / (d->fast - d->slow)));
        f = g * f + (1 - g) * f / d->factor;
      }
      turn[i] = (uint64_t)std::ldexp(f / kTurn, 64);  // f <= 1: below 2^62
    }
    auto r = new kv_rope();
    r->table.magnitude = (float)d->magnitude;
    r->table.rot_dim = d->rot_dim;
    r->table.layout = d->layout;
    const size_t bytes = turn.size() * sizeof(uint64_t);
    hipError_t e = hipGetDevice(&r->device);
    if (e == hipSuccess) e = hipMalloc(&r->mem, bytes);
    if (e == hipSuccess) e = hipMemcpy(r->mem, turn.data(), bytes, hipMemcpyHostToDevice);
    // the copy of pageable memory may return before it has reached the device
    if (e == hipSuccess) e = hipStreamSynchronize(nullptr);
    if (e != hipSuccess) {
      (void)hipGetLastError();
      if (r->mem) (void)hipFree(r->mem);
      delete r;
      return kv::hip_fail(e, "the rotation's table");
    }
    r->table.turn = (const uint64_t*)r->mem;
    try {
      std::lock_guard<std::mutex> lk(kv::g_rope_mu);
      kv::g_ropes.insert(r);
    } catch (...) {
      (void)hipFree(r->mem);
      delete r;
      throw;
    }
    *out = r;
    return KV_OK;
  });
}

extern "C" kv_status kv_rope_free(kv_rope* r) {
  if (!r) return KV_OK;
  return guarded("kv_rope_free", [&]() -> kv_status {
    {
      std::lock_guard<std::mutex> lk(kv::g_rope_mu);
      if (!kv::g_ropes.erase(r)) return invalid("kv_rope_free", "not a live rotation");
    }
    const hipError_t e = hipFree(r->mem);  // waits for the device
    delete r;
    if (e != hipSuccess) {
      (void)hipGetLastError();
      return kv::hip_fail(e, "hipFree");
    }
    return KV_OK;
  });
}

extern "C" kv_status kv_rope_apply(const kv_rope* r, uint32_t dtype, kv_heads_view x, kv_heads_view y,
                                   const int32_t* pos, uint32_t n_tokens, uint32_t n_heads, uint32_t head_dim,
                                   int backward, void* stream) {
  const char* who = "kv_rope_apply";
  return guarded(who, [&]() -> kv_status {
    if (!r || !kv::rope_is_live(r)) return invalid(who, "not a live rotation");
    if (dtype != KV_DT_BF16 && dtype != KV_DT_F16) return invalid(who, "dtype must be KV_DT_BF16 or KV_DT_F16");
    if (head_dim < r->table.rot_dim || head_dim > 256 || head_dim % 16)
      return invalid(who, "head_dim must be a multiple of 16 in rot_dim..256");
    if (n_heads > 65536) return invalid(who, "n_heads out of range");
    if (n_tokens == 0 || n_heads == 0) return KV_OK;
    if (kv::rope_is_elsewhere(r)) return invalid(who, "the rotation is on another device");
    if (!pos || !kv::aligned(pos, 4)) return invalid(who, "pos is NULL or misaligned");
    if (const char* e = kv::check_view(x)) return invalid(who, e);
    if (const char* e = kv::check_view(y)) return invalid(who, e);
    return kv::rope_apply(r->table, dtype, x, y, pos, n_tokens, n_heads, head_dim, backward != 0, (hipStream_t)stream);
  });
}

extern "C" kv_status kv_paged_work_bytes(const kv_paged_batch* b, uint64_t* bytes) {
  const char* who = "kv_paged_work_bytes";
  return guarded(who, [&]() -> kv_status {
    if (!b || !bytes) return invalid(who, "NULL argument");
    if (const char* e = kv::check_sizes(*b)) return invalid(who, e);
    *bytes = kv::work_layout(*b).bytes;
    return KV_OK;
  });
}

extern "C" kv_status kv_paged_plan(const kv_paged_batch* b, void* stream) {
  const char* who = "kv_paged_plan";
  return guarded(who, [&]() -> kv_status {
    if (!b) return invalid(who, "batch is NULL");
    if (const char* e = kv::check_batch(*b)) return invalid(who, e);
    return kv::paged_plan(*b, kv::work_layout(*b), (hipStream_t)stream);
  });
}

extern "C" kv_status kv_paged_append(const kv_paged_batch* b, const kv_paged_cache* c, const kv_rope* rope, uint32_t dtype,
                                     kv_heads_view q, kv_heads_view q_out, kv_heads_view k, kv_heads_view v, void* stream) {
  const char* who = "kv_paged_append";
  return guarded(who, [&]() -> kv_status {
    if (!b || !c) return invalid(who, "batch or cache is NULL");
    if (const char* e = kv::check_batch(*b)) return invalid(who, e);
    if (const char* e = kv::check_cache(*c, *b, dtype)) return invalid(who, e);
    if (kv::by_block(c->dtype)) {  // keys and values are written by different workgroups, each with its scale
      const uintptr_t ks = (uintptr_t)c->k_scale, vs = (uintptr_t)c->v_scale;
      if ((ks > vs ? ks - vs : vs - ks) < (uint64_t)c->n_blocks * b->kv_heads * sizeof(float))
        return invalid(who, "k_scale and v_scale must not be the same or overlap");
    }
    if (rope && !kv::rope_is_live(rope)) return invalid(who, "not a live rotation");
    if (rope && rope->table.rot_dim > b->head_dim) return invalid(who, "the rotation is wider than a head");
    if (rope && kv::rope_is_elsewhere(rope)) return invalid(who, "the rotation is on another device");
    if (const char* e = kv::check_view(k)) return invalid(who, e);
    if (const char* e = kv::check_view(v)) return invalid(who, e);
    if (q.ptr) {
      if (const char* e = kv::check_view(q)) return invalid(who, e);
      if (const char* e = kv::check_view(q_out)) return invalid(who, e);
    }
    if (kv::by_block(c->dtype))
      return kv::paged_append_block(*b, *c, rope ? &rope->table : nullptr, dtype, q, q_out, k, v, (hipStream_t)stream);
    return kv::paged_append(*b, *c, rope ? &rope->table : nullptr, dtype, q, q_out, k, v, (hipStream_t)stream);
  });
}

extern "C" kv_status kv_paged_read(const kv_paged_batch* b, const kv_paged_cache* c, uint32_t dtype, const int32_t* row_start,
                                   const int32_t* first, uint32_t max_rows, kv_heads_view k, kv_heads_view v, void* stream) {
  const char* who = "kv_paged_read";
  return guarded(who, [&]() -> kv_status {
    if (!b || !c) return invalid(who, "batch or cache is NULL");
    if (const char* e = kv::check_batch(*b)) return invalid(who, e);
    if (const char* e = kv::check_cache(*c, *b, dtype)) return invalid(who, e);
    if (!row_start || !kv::aligned(row_start, 4)) return invalid(who, "row_start is NULL or misaligned");
    if (!kv::aligned(first, 4)) return invalid(who, "first is misaligned");
    if (max_rows > 0x7fffffffu) return invalid(who, "max_rows out of range");
    if (max_rows == 0) return KV_OK;
    if (const char* e = kv::check_view(k)) return invalid(who, e);
    if (const char* e = kv::check_view(v)) return invalid(who, e);
    if (k.ptr == v.ptr) return invalid(who, "k and v must not be the same");
    return kv::paged_read(*b, *c, dtype, row_start, first, max_rows, k, v, (hipStream_t)stream);
  });
}

extern "C" kv_status kv_paged_attention(const kv_paged_batch* b, const kv_paged_cache* c, uint32_t dtype, kv_heads_view q,
                                        kv_heads_view out, float* lse, float scale, void* stream) {
  const char* who = "kv_paged_attention";
  return guarded(who, [&]() -> kv_status {
    if (!b || !c) return invalid(who, "batch or cache is NULL");
    if (const char* e = kv::check_batch(*b)) return invalid(who, e);
    if (const char* e = kv::check_cache(*c, *b, dtype)) return invalid(who, e);
    if (const char* e = kv::check_view(q)) return invalid(who, e);
    if (const char* e = kv::check_view(out)) return invalid(who, e);
    if (!(scale > 0) || !std::isfinite(scale)) return invalid(who, "scale must be > 0 and finite");
    if (!kv::aligned(lse, 4)) return invalid(who, "lse is misaligned");
    // workgroups read queries after others have written their outputs
    if (out.ptr == q.ptr) return invalid(who, "out must not be q");
    return kv::paged_attention(*b, kv::work_layout(*b), *c, dtype, q, out, lse, scale, (hipStream_t)stream);
  });
}
