// Attention of new tokens over a quantised paged KV cache.
#include "paged_attn_impl.hpp"

namespace spa {

hipError_t launch_paged_attn_q8(const PagedDims& d, const PagedParts& parts, const void* q, const void* k_pages, const void* vt_pages,
                                const PagedExps& exps, const int32_t* block_table, const int32_t* q_starts, const int32_t* kv_lens,
                                const float* slopes_or_null, void* out, float* lse_or_null, hipStream_t st) {
    const PagedArgs a = paged_args(d, q, k_pages, vt_pages, exps, block_table, q_starts, kv_lens, nullptr, nullptr, slopes_or_null, out, lse_or_null);
    return d.D == 128 ? launch_parts<128, true>(a, d, parts, st) : launch_parts<64, true>(a, d, parts, st);
}

}  // namespace spa
