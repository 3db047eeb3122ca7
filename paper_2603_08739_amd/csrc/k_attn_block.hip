// k_attn_block.hip - attention over a paged KV cache of 8 bits with a scale for each block
// of tokens and head (kernels: attn_kernels.h).
#include "attn_kernels.h"

namespace kv {
namespace attn {

template kv_status launch_dim<BF16, kFp8Block>(const AttnArgs&, uint32_t, uint32_t, uint32_t, hipStream_t);
template kv_status launch_dim<F16, kFp8Block>(const AttnArgs&, uint32_t, uint32_t, uint32_t, hipStream_t);
template kv_status launch_dim<BF16, kI8Block>(const AttnArgs&, uint32_t, uint32_t, uint32_t, hipStream_t);
template kv_status launch_dim<F16, kI8Block>(const AttnArgs&, uint32_t, uint32_t, uint32_t, hipStream_t);

}  // namespace attn
}  // namespace kv
