// Paged KV cache: sizes of a call and how its attention is cut into workgroups.
#pragma once
#include "common.hpp"

namespace spa {

constexpr int kMaxRequests = 4096;
constexpr int kPagedTile = 64;        // keys of a tile, the unit in which the key axis is cut

struct PagedDims {
    int B, Hq, Hkv, G, D, P, log_p;
    int n_pages, C, T, max_new;       // C: columns of the table; T: packed tokens
    float scale, cap;
    int sink, window;                 // tokens; window 0: every causal key
    int64_t table_stride;
    int64_t q_t, q_h, o_t, o_h, kp_p, kp_h, vp_p, vp_h;
};

// One of the two attention kernels.  It serves the requests with row_lo < rows <= row_hi, rows = new tokens * query heads of a
// KV head, m = 2^log_m rows a workgroup (0: no such kernel in the call), which span at most `span` tokens, and cuts the key axis
// into pieces: of at least `min_tiles` key tiles, and so that at most 2^log_most of them come about beyond one for every row tile.
struct PagedPart {
    int m, log_m, span;
    int log_most, min_tiles;
    int whole_tiles;                  // key axes of at most so many tiles are not cut (no workspace, no merge)
    int row_lo, row_hi;
    int n_slots;                      // partial results that the workspace has room for; 0: nothing is cut
    float *o, *lse;                   // partial results: [n_slots][m][D], [n_slots][m]; lse in base 2
    int32_t* piece;                   // many rows: key tiles of a piece, as the attention kernel leaves them for the merge
};

// A request's share of a part: row tiles, key tiles (of its longest row tile), pieces of the key axis
struct PagedShare {
    int tiles, keys, splits;
};

__host__ __device__ __forceinline__ int clamp_int(int v, int lo, int hi) { return v < lo ? lo : (v > hi ? hi : v); }

// The key tiles that a row tile with positions pos_lo .. pos_hi looks at, in order: `sinks` tiles from the first on, then
// those from `from` to the one of pos_hi; `n` in all.
struct KeyTiles {
    int sinks, from, n;
    __host__ __device__ __forceinline__ int at(int e) const { return e < sinks ? e : e - sinks + from; }
};
__host__ __device__ __forceinline__ KeyTiles key_tiles(int pos_lo, int pos_hi, int sink, int window) {
    KeyTiles t{0, 0, 0};
    if (pos_hi < 0) return t;
    const int end = pos_hi / kPagedTile + 1;
    if (window > 0) {
        const int first = pos_lo - window + 1;          // first key that the window of the first row reaches
        t.from = first > 0 ? first / kPagedTile : 0;
        const int s = (sink + kPagedTile - 1) / kPagedTile;
        t.sinks = s < t.from ? s : t.from;
    }
    t.n = t.sinks + end - t.from;
    return t;
}
// at least the key tiles of any row tile of a request: q_len new tokens, of which a row tile spans at most `span`
__host__ __device__ __forceinline__ int most_key_tiles(int q_len, int kv_len, int span, int sink, int window) {
    const int all = (kv_len + kPagedTile - 1) / kPagedTile;
    if (window == 0) return all;
    const int64_t some = (int64_t)(sink + kPagedTile - 1) / kPagedTile + ((int64_t)window + (span < q_len ? span : q_len) + kPagedTile - 2) / kPagedTile + 1;
    return some < all ? (int)some : all;
}

constexpr int kWholeAxis = 1 << 24;   // key tiles: more than any key axis has
__host__ __device__ __forceinline__ int piece_within(int64_t tiles, const PagedPart& part) {
    return tiles < part.min_tiles ? part.min_tiles : (tiles > kWholeAxis ? kWholeAxis : (int)tiles);
}
// Key tiles of a piece, for `work` (row tile, key tile, KV head) triples in all.
// The shortest that the workspace has room for:
__host__ __device__ __forceinline__ int shortest_piece(int64_t work, const PagedPart& part) {
    return piece_within((work + (1ll << part.log_most) - 1) >> part.log_most, part);
}
// The kernel for few rows: short enough for 512 workgroups, then not below 16 tiles (a workgroup that starts costs about as much as
// two tiles) until these are more than the workspace's.  Measured with 2^11 = log_most always, or 16 tiles at least: 32 requests with a window of
// 4096 tokens 61.9 / 59.4 us, drafted tokens of 32 requests 65.9 / 64.6, 16 requests of 2400 tokens 24.0 with 4 tiles / 27.4.
__host__ __device__ __forceinline__ int few_rows_piece(int64_t work, const PagedPart& part) {
    const int64_t even = (work + 511) >> 9;
    const int p = piece_within(even < 16 ? even : 16, part), least = shortest_piece(work, part);
    return p > least ? p : least;
}
__host__ __device__ __forceinline__ PagedShare paged_share(const PagedPart& part, int G, int q_len, int kv_len, int sink, int window, int piece) {
    PagedShare s{0, 0, 0};
    const int rows = q_len * G;
    if (rows > part.row_lo && rows <= part.row_hi) {
        s.tiles = (rows + part.m - 1) >> part.log_m;
        s.keys = most_key_tiles(q_len, kv_len, part.span, sink, window);
        s.splits = s.keys <= piece ? 1 : (int)(((uint32_t)s.keys + (uint32_t)piece - 1u) / (uint32_t)piece);
    }
    return s;
}

hipError_t launch_paged_plan(const PagedDims& d, const int32_t* ctx_lens, const int32_t* new_lens, const int32_t* free_pages, int n_free,
                             const int32_t* free_range, int32_t* block_table, int32_t* q_starts, int32_t* kv_lens, int32_t* slots,
                             int32_t* positions_or_null, int32_t* taken, hipStream_t st);
hipError_t launch_paged_append(const PagedDims& d, const void* k, int64_t k_t, int64_t k_h, const void* v, int64_t v_t, int64_t v_h,
                               const int32_t* slots, void* k_pages, void* vt_pages, hipStream_t st);

// The parts of a call (rows_few: for requests of few rows; rows_many), with m = 0 where a part is not needed, and
// their scratch in bytes.  o and lse are set from ws, which may be null.
struct PagedParts {
    PagedPart few, many;
    size_t ws_bytes;
};
PagedParts paged_parts(const PagedDims& d, void* ws_or_null);
hipError_t launch_paged_attn(const PagedDims& d, const PagedParts& parts, const void* q, const void* k_pages, const void* vt_pages,
                             const int32_t* block_table, const int32_t* q_starts, const int32_t* kv_lens, const float* slopes_or_null,
                             void* out, float* lse_or_null, hipStream_t st);

}  // namespace spa
