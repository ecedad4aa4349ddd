// Attention of new tokens over a paged KV cache: the kernels for pages of bf16 values, and what the calls share on the host.
#include "paged_attn_impl.hpp"

namespace spa {

PagedParts paged_parts(const PagedDims& d, void* ws_or_null) {
    PagedParts p{};
    const int most_new = d.max_new > 0 && d.max_new < d.T ? d.max_new : d.T;
    const int64_t most_rows = (int64_t)most_new * d.G;
    // Few rows are bound by the loads of keys and values, many by the matrix products: up to 32 rows go to the one kernel,
    // more to the other.  Both are launched where a call may have requests of both kinds.
    const int few_rows = most_rows <= 16 || (most_rows > 32 && d.G <= 16) ? 16 : 32;
    if (most_rows <= few_rows || (d.B > 1 && d.G <= few_rows)) {
        p.few.m = few_rows;
        p.few.log_m = few_rows == 16 ? 4 : 5;
        p.few.span = (p.few.m + d.G - 1) / d.G + 1;
        p.few.log_most = 11;
        p.few.min_tiles = 4;
        p.few.whole_tiles = 8;
        p.few.row_lo = 0;
        p.few.row_hi = most_rows <= few_rows ? 0x7fffffff : few_rows;
    }
    if (most_rows > few_rows) {
        p.many.m = kManyRows;
        p.many.log_m = 7;
        p.many.span = (p.many.m + d.G - 1) / d.G + 1;
        p.many.log_most = 10;
        p.many.min_tiles = 2;
        p.many.whole_tiles = 8;
        p.many.row_lo = p.few.m ? few_rows : 0;
        p.many.row_hi = 0x7fffffff;
    }
    size_t off = 0;
    for (PagedPart* part : {&p.few, &p.many}) {
        if (part->m == 0) continue;
        part->n_slots = (int)most_slots(d, *part);
        char* base = (char*)ws_or_null;
        part->o = (float*)(base + off);
        off += (size_t)part->n_slots * part->m * d.D * sizeof(float);
        part->lse = (float*)(base + off);
        off += ((size_t)part->n_slots * part->m * sizeof(float) + 255) / 256 * 256;
        part->piece = (int32_t*)(base + off);
        if (part->n_slots > 0 && part == &p.many) off += 256;
    }
    p.ws_bytes = off;
    return p;
}

hipError_t launch_paged_attn(const PagedDims& d, const PagedParts& parts, const void* q, const void* k_pages, const void* vt_pages,
                             const int32_t* block_table, const int32_t* q_starts, const int32_t* kv_lens, const float* slopes_or_null,
                             void* out, float* lse_or_null, hipStream_t st) {
    const PagedArgs a = paged_args(d, q, k_pages, vt_pages, PagedExps{}, block_table, q_starts, kv_lens, nullptr, nullptr, slopes_or_null, out, lse_or_null);
    return d.D == 128 ? launch_parts<128, false>(a, d, parts, st) : launch_parts<64, false>(a, d, parts, st);
}

}  // namespace spa
