// Attention of new tokens over a paged KV cache: single tokens, a few of them, chunks of prompts.
//
// The rows of a workgroup are (new token, query head) pairs of one KV head, so that a group's heads take every key and value
// from one load.  The key axis of a row tile is cut into pieces so that few rows fill the chip, too; pieces leave a normalised
// partial result and its log-sum-exp, merged by a second kernel.  How a call is cut depends on lengths that only the device
// knows: every wavefront derives its share from them by itself (part_piece, share_of), without a plan, a host copy or a barrier.
//
// Softmax in base 2: x = (scaled logit) * log2 e, weights 2^(x - m) against a reference m that is set by the first tile and
// moved only when a query's running denominator passes 2^40; the normalisation makes the result independent of m.  Logits,
// weights' sums and outputs are held in fp32.  The second matrix product takes weights in bf16.  The kernel for few rows waits for
// the memory and gives it two bf16 parts of each, 16 bits in all: an error of 2^-16 of a term, lost in the output's rounding (against 64 bits
// 0.0016 to 0.0017 of the norm, as from that rounding alone; 0.0019 to 0.0024 with one part; the same time).  The kernel for many rows
// is bound by its matrix products, of which a second part would make half as many again, and rounds the weights to bf16 once, as the
// sparse prefill does: 2^-8 of a term, about that of the bf16 output (0.0019 to 0.0023 of the norm in all).
#include "attn_parts.hpp"
#include "paged.hpp"

namespace spa {
namespace {

constexpr float kLog2e = 1.44269504088896340736f, kLn2 = 0.69314718055994530942f;
constexpr float kRescaleAt = 1.099511627776e12f;      // 2^40
// Base-2 log-sum-exp of a piece whose keys, if a row sees any, all have a logit of -infinity; -infinity itself where a piece has written no
// values.  A row whose pieces all have it, or that has no pieces and found no finite logit, comes from a query that sees no key if its
// position is below 0 (every other one sees its own key): zeros then, NaN otherwise, as 0 / 0 has it.
constexpr float kNoLogit = -0x1.fffffep127f;      // the lowest finite value
__device__ __forceinline__ float without_logits(int pos) { return pos < 0 ? 0.f : NAN; }

struct PagedArgs {
    const uint16_t *q, *k, *vt;
    const int32_t *table, *q_starts, *kv_lens;
    const float* slopes;                              // nullptr: no bias by distance
    uint16_t* out;
    float* lse;                                       // nullptr: not wanted
    int B, Hq, Hkv, G, T, log_p, n_pages, C, sink, window;
    float scale, cap;                                 // cap 0: none
    int64_t table_stride, q_t, q_h, o_t, o_h, kp_p, kp_h, vp_p, vp_h;
};

// ---------------------------------------------------------------------------------------------------------------
// How a call is cut

__device__ __forceinline__ uint32_t wave_scan(uint32_t v) {                             // inclusive, over the lanes
    v += __builtin_amdgcn_update_dpp(0, (int)v, 0x111, 0xF, 0xF, true);   // row_shr:1, lanes shifted out read 0
    v += __builtin_amdgcn_update_dpp(0, (int)v, 0x112, 0xF, 0xF, true);   // row_shr:2
    v += __builtin_amdgcn_update_dpp(0, (int)v, 0x114, 0xF, 0xF, true);   // row_shr:4
    v += __builtin_amdgcn_update_dpp(0, (int)v, 0x118, 0xF, 0xF, true);   // row_shr:8
    v += __builtin_amdgcn_update_dpp(0, (int)v, 0x142, 0xA, 0xF, true);   // row_bcast15 into rows 1 and 3
    v += __builtin_amdgcn_update_dpp(0, (int)v, 0x143, 0xC, 0xF, true);   // row_bcast31 into rows 2 and 3
    return v;
}
__device__ __forceinline__ uint32_t last_lane(uint32_t v) { return (uint32_t)__builtin_amdgcn_readlane((int)v, 63); }

struct Request {
    int first, len, kv;               // first row and number of its new tokens, cached tokens
};
__device__ __forceinline__ Request request_at(const PagedArgs& a, int b) {
    Request r{0, 0, 0};
    if (b < a.B) {
        r.first = clamp_int(a.q_starts[b], 0, a.T);
        r.len = clamp_int(a.q_starts[b + 1], r.first, a.T) - r.first;
        r.kv = clamp_int(a.kv_lens[b], 0, a.C << a.log_p);
    }
    return r;
}
__device__ __forceinline__ PagedShare share_at(const PagedArgs& a, const PagedPart& part, const Request& r, int piece) {
    return paged_share(part, a.G, r.len, r.kv, a.sink, a.window, piece);
}
// sum and maximum over the 16 lanes of a row, in its last lane
__device__ __forceinline__ uint32_t row_sum(uint32_t v) {
    v += __builtin_amdgcn_update_dpp(0, (int)v, 0x111, 0xF, 0xF, true);
    v += __builtin_amdgcn_update_dpp(0, (int)v, 0x112, 0xF, 0xF, true);
    v += __builtin_amdgcn_update_dpp(0, (int)v, 0x114, 0xF, 0xF, true);
    v += __builtin_amdgcn_update_dpp(0, (int)v, 0x118, 0xF, 0xF, true);
    return v;
}
__device__ __forceinline__ uint32_t row_max(uint32_t v) {
    v = max(v, (uint32_t)__builtin_amdgcn_update_dpp(0, (int)v, 0x111, 0xF, 0xF, true));
    v = max(v, (uint32_t)__builtin_amdgcn_update_dpp(0, (int)v, 0x112, 0xF, 0xF, true));
    v = max(v, (uint32_t)__builtin_amdgcn_update_dpp(0, (int)v, 0x114, 0xF, 0xF, true));
    v = max(v, (uint32_t)__builtin_amdgcn_update_dpp(0, (int)v, 0x118, 0xF, 0xF, true));
    return v;
}
// The kernel for many rows, up to 64 requests: of four lengths of a piece the one with the least time, by a model.  512 workgroups that run
// at once and take about 1.6 us a key tile (fitted with head_dim 128 without a cap, used for all: with head_dim 64 and a key tile in one page
// 768 run at once): the longest piece, or the rounds of average ones, whichever is more; then the merge, 5 us and
// 0.03 for each piece.  The lengths: no cut; as many pieces as run at once (each of the `tiles` row tiles and KV heads may end in a
// short one); twice or four times as long, for short calls; or two rounds of pieces.  With 2^9 pieces always, or 2^10: chunk of
// 2048 tokens 3040 / 3105 us, mixed step 493 / 455 (now 396); 180 tokens over 22000, 48 row tiles, in 528 pieces: 130 us, in 480: 98;
// 87 tokens over 800, 12 row tiles of 14 key tiles, in pieces of 7: 27 us, of 2: 19.
// A row of 16 lanes tries one length.
__device__ __forceinline__ int many_rows_piece(const PagedArgs& a, const PagedPart& part, int64_t work, int64_t tiles, int lane) {
    const int least = shortest_piece(work, part);
    auto pieces_of = [&](int64_t n) { return n > tiles ? piece_within((work + n - tiles - 1) / (n - tiles), part) : kWholeAxis; };
    const int fit = pieces_of(512), turn = lane >> 4;
    int p = turn == 0 ? kWholeAxis : turn == 1 ? fit : turn == 2 ? (fit < 8 ? 4 * fit : pieces_of(1024)) : 2 * fit;
    if (p < least) p = least;
    if (p > kWholeAxis) p = kWholeAxis;
    uint32_t units = 0, cut = 0, longest = 0;
    for (int b0 = 0; b0 < a.B; b0 += 16) {
        const PagedShare s = share_at(a, part, request_at(a, b0 + (lane & 15)), p);
        const uint32_t mine = (uint32_t)(s.tiles * s.splits) * (uint32_t)a.Hkv;
        units += mine;
        cut += s.splits > 1 ? mine : 0u;
        longest = max(longest, (uint32_t)min(s.keys, p));
    }
    units = row_sum(units);
    cut = row_sum(cut);
    const float rounds = ceilf((float)units * (1.f / 512.f)) * (float)work / (float)max(units, 1u);
    const float us = 1.6f * fmaxf((float)row_max(longest), rounds) + (cut > 0 ? 5.f + 0.03f * (float)cut : 0.f);
    auto time_of = [&](int t) { return __uint_as_float((uint32_t)__builtin_amdgcn_readlane(__float_as_int(us), 16 * t + 15)); };
    int best = 0;
#pragma unroll
    for (int t = 1; t < 4; ++t)
        if (time_of(t) < time_of(best)) best = t;
    return __builtin_amdgcn_readlane(p, 16 * best + 15);
}
// key tiles of a part's pieces, the same in every lane
template <bool MANY>
__device__ __forceinline__ int part_piece(const PagedArgs& a, const PagedPart& part, const Request& first, int lane) {
    if (part.n_slots == 0) return kWholeAxis;
    int64_t work = 0;
    uint32_t tiles = 0;
    for (int b0 = 0; b0 < a.B; b0 += 64) {
        const PagedShare s = share_at(a, part, b0 == 0 ? first : request_at(a, b0 + lane), kWholeAxis);
        work += (int64_t)s.tiles * s.keys;
        tiles += (uint32_t)s.tiles;
    }
    // the lanes' sum in two halves of 24 bits; a lane's work of 2^48 and more makes the piece as long as any key axis either way
    const uint32_t lo = last_lane(wave_scan((uint32_t)(work & 0xffffff)));
    const uint32_t hi = last_lane(wave_scan((uint32_t)(work >> 24 > 0xffffff ? 0xffffff : work >> 24)));
    work = (((int64_t)hi << 24) + lo) * a.Hkv;
    if constexpr (!MANY) return few_rows_piece(work, part);
    else return a.B <= 64 ? many_rows_piece(a, part, work, (int64_t)last_lane(wave_scan(tiles)) * a.Hkv, lane) : shortest_piece(work, part);
}

// What a workgroup of a part serves: unit `unit` of request b, counted from the longest row tiles, KV heads next to each
// other (they go to different XCDs, each of which then keeps its heads' keys in its L2).
struct Share {
    int b, unit;                      // b < 0: nothing
    int slot;                         // first partial result of the request (its units' results follow each other)
    PagedShare s;
    Request r;
};
// MERGE: units are the rows of requests whose keys are cut, KV heads next to each other
// first: request_at(a, lane), which a caller has at hand or has in flight together with other loads
template <bool MERGE>
__device__ __forceinline__ Share share_of(const PagedArgs& a, const PagedPart& part, int piece, const Request& first, uint32_t item) {
    const int lane = threadIdx.x & 63;
    uint32_t items_before = 0, slots_before = 0;
    Share found;
    found.b = -1;
    for (int b0 = 0; b0 < a.B; b0 += 64) {
        const Request r = b0 == 0 ? first : request_at(a, b0 + lane);
        const PagedShare s = share_at(a, part, r, piece);
        const uint32_t units = (uint32_t)s.tiles * (uint32_t)s.splits * (uint32_t)a.Hkv;
        const uint32_t slots = s.splits > 1 ? units : 0u;
        const uint32_t items = !MERGE ? units : (s.splits > 1 ? (uint32_t)(r.len * a.Hq) : 0u);
        const uint32_t items_upto = items_before + wave_scan(items), slots_upto = slots_before + wave_scan(slots);
        const uint64_t here = __ballot(item >= items_upto - items && item < items_upto);
        if (here != 0) {
            const int at = __builtin_ctzll(here);
            auto pick = [&](int v) { return __builtin_amdgcn_readlane(v, at); };
            found.b = b0 + at;
            found.unit = (int)(item - (uint32_t)pick((int)(items_upto - items)));
            found.slot = pick((int)(slots_upto - slots));
            found.s = PagedShare{pick(s.tiles), pick(s.keys), pick(s.splits)};
            found.r = Request{pick(r.first), pick(r.len), pick(r.kv)};
            return found;
        }
        items_before = last_lane(items_upto);
        slots_before = last_lane(slots_upto);
    }
    return found;
}
// a request's key tiles are dealt to its pieces evenly
__device__ __forceinline__ int tiles_of_piece(const PagedShare& s) { return (int)((uint32_t)(s.keys + s.splits - 1) / (uint32_t)s.splits); }

// ---------------------------------------------------------------------------------------------------------------
// Masks and logits

// A pair of bf16 values: whether either is infinite or NaN (its exponent is all ones); the pair with such a one as 0.
__device__ __forceinline__ bool not_finite(uint32_t pair) { return (((pair & 0x7f807f80u) + 0x00800080u) & 0x80008000u) != 0; }
__device__ __forceinline__ uint32_t finite_part(uint32_t pair) {
    return pair & (((pair & 0x7f80u) == 0x7f80u ? 0u : 0xffffu) | ((pair & 0x7f800000u) == 0x7f800000u ? 0u : 0xffff0000u));
}
// Which keys the query at position pos sees, and whether one of 32 or 64 keys from key0 on is hidden from one of the positions
// lo .. hi
__device__ __forceinline__ bool sees(const PagedArgs& a, int pos, int key) { return key <= pos && (a.window == 0 || pos - key < a.window || key < a.sink); }
__device__ __forceinline__ bool hides(const PagedArgs& a, int lo, int hi, int key0, int n) {
    return key0 + n - 1 > lo || (a.window > 0 && key0 + n - 1 >= a.sink && key0 <= hi - a.window);
}

// base-2 logits of a lane: what the options make of scaled products
struct Logits {
    float c;                          // scale * log2 e
    float cap, cap_inv2, cap2;        // cap > 0: 2 * scale * log2 e / cap, cap * log2 e
    float slope2;                     // slope * log2 e
};
__device__ __forceinline__ Logits logits_of(const PagedArgs& a, int head) {
    Logits l;
    l.c = a.scale * kLog2e;
    l.cap = a.cap;
    l.cap_inv2 = a.cap > 0.f ? fminf(2.f * l.c / a.cap, 3e38f) : 0.f;     // finite, so that a product of 0 stays 0
    l.cap2 = a.cap * kLog2e;
    l.slope2 = a.slopes != nullptr ? a.slopes[head] * kLog2e : 0.f;
    return l;
}
// back: position of the query less that of the key
template <bool MOD>
__device__ __forceinline__ float logit(const Logits& l, float s, int back) {
    if constexpr (!MOD) {
        return s * l.c;
    } else {
        float x = s * l.c;
        // tanh |y| = (1 - t) / (1 + t), t = e^(-2 |y|) <= 1: nothing overflows, absolute error about 2^-25 near 0
        if (l.cap > 0.f) {
            const float t = __builtin_amdgcn_exp2f(-fabsf(s * l.cap_inv2));
            x = __builtin_copysignf(l.cap2 * (1.f - t) * __builtin_amdgcn_rcpf(1.f + t), s);
        }
        return fmaf(-l.slope2, (float)back, x);
    }
}

__device__ __forceinline__ float max_over_groups(float v) { v = fmaxf(v, __shfl_xor(v, 16)); return fmaxf(v, __shfl_xor(v, 32)); }
__device__ __forceinline__ float sum_over_groups(float v) { v += __shfl_xor(v, 16); return v + __shfl_xor(v, 32); }

// ---------------------------------------------------------------------------------------------------------------
// Few rows: MF * 16 rows, NW wavefronts that each take every NW-th 32 keys, straight from memory into the operands of
// v_mfma_f32_16x16x32_bf16 (S^T = K Q^T, O^T += V^T P^T).  A lane holds keys 8 (lane / 16) .. + 7 of a chunk of one row:
// K rows are assigned to the first product's rows such that the weights are the second one's operand as they are.  Bound
// by HBM: nothing is shared between the wavefronts, so there is no LDS in the loop and no barrier.
// 64 requests of up to 8192 keys: 205 to 207 us for 1.14 GB of keys and values, 5.5 TB/s (a plain sum of 2 GiB: 6.07).
//
// NV > 1: a workgroup makes the outputs of D / NV dims only, from all of K and its share of V.  A CU takes in about 12 bytes a
// clock however many loads it has in flight (256 KB of a head: 22000 cycles of a call of 501 keys), so a call of few workgroups
// is faster on NV times as many, although they read K NV times: 11.8 -> 9.2 us.  The host tells few workgroups from the table's width: the same
// call in a table of 2048 pages takes 15.8.

// LDS of a workgroup: the wavefronts' outputs, references and denominators
template <int D, int MF, int NW, int NV>
constexpr int kFewLds = NW * 16 * (D / NV + 4) * 4 + 2 * NW * MF * 16 * 4;
template <int D, int MF, bool MOD, bool SMALL, int NW, int NV>
__device__ __forceinline__ void few_rows(const PagedArgs& a, const PagedPart& part, unsigned wg, unsigned units, char* lds) {
    constexpr int DS = D / 32;        // MFMAs of a logits tile
    constexpr int DV = D / NV;        // dims of the outputs
    constexpr int DT = DV / 16;       // 16-row tiles of O^T
    constexpr int PAD = DV + 4;
    float (*const s_o)[16][PAD] = reinterpret_cast<float (*)[16][PAD]>(lds);
    float (*const s_m)[MF * 16] = reinterpret_cast<float (*)[MF * 16]>(lds + NW * 16 * PAD * 4);
    float (*const s_l)[MF * 16] = s_m + NW;

    const int dv0 = NV > 1 ? (int)(wg / units) * DV : 0;     // parts of a unit on one XCD where units are a multiple of 8
    const Request first = request_at(a, threadIdx.x & 63);
    const int piece = part_piece<false>(a, part, first, threadIdx.x & 63);
    const Share sh = share_of<false>(a, part, piece, first, NV > 1 ? wg % units : wg);
    if (sh.b < 0) return;
    const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6);
    const int n16 = lane & 15, g = lane >> 4;
    const int kvh = sh.unit % a.Hkv, cut = sh.unit / a.Hkv % sh.s.splits, tile = sh.s.tiles - 1 - sh.unit / a.Hkv / sh.s.splits;
    const int rows = sh.r.len * a.G, row0 = tile * part.m;
    const int last_row = min(row0 + part.m, rows) - 1;
    const int pos0 = sh.r.kv - sh.r.len;                        // position of the request's first new token
    const int pos_lo = pos0 + row0 / a.G, pos_hi = pos0 + last_row / a.G;
    const KeyTiles kt = key_tiles(pos_lo, pos_hi, a.sink, a.window);
    const int per = tiles_of_piece(sh.s);
    const int e_end = min((cut + 1) * per, kt.n);               // of the row tile's key tiles
    const int last_col = pos_hi >= 0 ? pos_hi >> a.log_p : 0;
    const int page = 1 << a.log_p;

    bf16x8 qf[MF][DS];
    int pos[MF], head[MF], token[MF];
    Logits lg[MF];
#pragma unroll
    for (int f = 0; f < MF; ++f) {
        const int row = min(row0 + 16 * f + n16, last_row);      // rows past the last repeat it; they are not stored
        token[f] = row / a.G;
        head[f] = kvh * a.G + row % a.G;
        pos[f] = pos0 + token[f];
        const uint16_t* qrow = a.q + (int64_t)(sh.r.first + token[f]) * a.q_t + head[f] * a.q_h + 8 * g;
#pragma unroll
        for (int s = 0; s < DS; ++s) qf[f][s] = *reinterpret_cast<const bf16x8*>(qrow + 32 * s);
        lg[f] = logits_of(a, head[f]);
    }
    f32x4 o[MF][DT];
    float m[MF], l[MF];
#pragma unroll
    for (int f = 0; f < MF; ++f) {
        m[f] = -INFINITY;
        l[f] = 0.f;
#pragma unroll
        for (int t = 0; t < DT; ++t) o[f][t] = f32x4{0.f, 0.f, 0.f, 0.f};
    }
    const int32_t* const trow = a.table + (int64_t)sh.b * a.table_stride;
    auto page_of = [&](int key) { return clamp_int(trow[min(key >> a.log_p, last_col)], 0, a.n_pages - 1); };
    const int k_row = 8 * (n16 >> 2) + (n16 & 3);               // key of a chunk that this lane loads, and + 4
    // chunks of this workgroup: the last tile's second half only if a row sees it
    const int c_end = e_end == kt.n && (pos_hi & (kPagedTile - 1)) < 32 ? 2 * e_end - 1 : 2 * e_end;
    auto key_of = [&](int c) { return kt.at(c >> 1) * kPagedTile + 32 * (c & 1); };
    struct Pages {                                              // pages of 16 tokens: a chunk lies in two
        int id[SMALL ? 2 : 1];
    };
    auto pages_of = [&](int c) {
        Pages p;
        const int key0 = key_of(min(c, c_end - 1));
        p.id[0] = page_of(key0);
        if constexpr (SMALL) p.id[1] = page_of(key0 + 16);
        return p;
    };
    struct Chunk {
        bf16x8 k0[DS], k1[DS];
        u32x4 v[DT];
    };
    auto v_of = [&](int c, const Pages& pg) __attribute__((always_inline)) {       // a lane's 8 keys of dim dv0 + n16; other tiles 16 page further
        const int in_page = SMALL ? 0 : key_of(c) & (page - 1);
        const int id = SMALL && g >= 2 ? pg.id[SMALL ? 1 : 0] : pg.id[0];
        return a.vt + id * a.vp_p + kvh * a.vp_h + in_page + 8 * (SMALL ? g & 1 : g) + (int64_t)(dv0 + n16) * page;
    };
    auto load = [&](int c, const Pages& pg, Chunk& ch) __attribute__((always_inline)) {
        const int in_page = SMALL ? 0 : key_of(c) & (page - 1);
        const int id_k = SMALL && n16 >= 8 ? pg.id[SMALL ? 1 : 0] : pg.id[0];
        const uint16_t* kp = a.k + id_k * a.kp_p + kvh * a.kp_h + (in_page + (SMALL ? k_row & 15 : k_row)) * D + 8 * g;
        const uint16_t* vp = v_of(c, pg);
#pragma unroll
        for (int s = 0; s < DS; ++s) {
            ch.k0[s] = *reinterpret_cast<const bf16x8*>(kp + 32 * s);
            ch.k1[s] = *reinterpret_cast<const bf16x8*>(kp + 4 * D + 32 * s);
        }
#pragma unroll
        for (int t = 0; t < DT; ++t) ch.v[t] = *reinterpret_cast<const u32x4*>(vp + 16 * t * page);
    };
    bool put_back = false;                                      // of this wavefront
    auto attend = [&](int c, Chunk& ch) __attribute__((always_inline)) {
        const int key0 = key_of(c);
        // Values of keys that no row of the tile sees (behind its last position, or between the sinks and its first window) may be
        // anything, NaN too, and a weight of 0 would not hide them: they become 0.
        const int gone_lo = a.sink, gone_hi = a.window > 0 ? pos_lo - a.window + 1 : 0;       // [gone_lo, gone_hi)
        if (key0 + 31 > pos_hi || (key0 + 31 >= gone_lo && key0 < gone_hi)) {
            const int key = key0 + 8 * g;
            u32x4 keep;
#pragma unroll
            for (int x = 0; x < 4; ++x) {
                const int ka = key + 2 * x, kb = ka + 1;
                keep[x] = (ka <= pos_hi && !(ka >= gone_lo && ka < gone_hi) ? 0xffffu : 0u) |
                          (kb <= pos_hi && !(kb >= gone_lo && kb < gone_hi) ? 0xffff0000u : 0u);
            }
#pragma unroll
            for (int t = 0; t < DT; ++t) ch.v[t] &= keep;
        }
        const bool masked = hides(a, pos_lo, pos_hi, key0, 32);
        // Where some rows see a key and others do not, its infinite and NaN values are taken out and come back at the end.
        if (masked && pos_lo != pos_hi) {
            bool odd = false;
#pragma unroll
            for (int t = 0; t < DT; ++t)
#pragma unroll
                for (int x = 0; x < 4; ++x) odd |= not_finite(ch.v[t][x]);
            if (__any(odd)) {
                put_back = true;
#pragma unroll
                for (int t = 0; t < DT; ++t)
#pragma unroll
                    for (int x = 0; x < 4; ++x) ch.v[t][x] = finite_part(ch.v[t][x]);
            }
        }
#pragma unroll
        for (int f = 0; f < MF; ++f) {
            f32x4 s0 = {0.f, 0.f, 0.f, 0.f}, s1 = s0;
#pragma unroll
            for (int s = 0; s < DS; ++s) {
                s0 = __builtin_amdgcn_mfma_f32_16x16x32_bf16(ch.k0[s], qf[f][s], s0, 0, 0, 0);
                s1 = __builtin_amdgcn_mfma_f32_16x16x32_bf16(ch.k1[s], qf[f][s], s1, 0, 0, 0);
            }
            f32x8 x;
            const int back = pos[f] - key0 - 8 * g;
#pragma unroll
            for (int r = 0; r < 4; ++r) {
                x[r] = logit<MOD>(lg[f], s0[r], back - r);
                x[4 + r] = logit<MOD>(lg[f], s1[r], back - 4 - r);
            }
            if (masked) {
#pragma unroll
                for (int r = 0; r < 8; ++r) {
                    if (!sees(a, pos[f], pos[f] - back + r)) x[r] = -INFINITY;
                }
            }
            const float mr = m[f] == -INFINITY ? 0.f : m[f];
            f32x8 w;
            float sum = 0.f;
#pragma unroll
            for (int r = 0; r < 8; ++r) {
                w[r] = __builtin_amdgcn_exp2f(x[r] - mr);
                sum += w[r];
            }
            if (__any(m[f] == -INFINITY || !(l[f] + sum < kRescaleAt))) {
                float mx = x[0];
#pragma unroll
                for (int r = 1; r < 8; ++r) mx = fmaxf(mx, x[r]);
                mx = max_over_groups(mx);
                const float lq = sum_over_groups(l[f]);
                const float m_new = fmaxf(m[f] == -INFINITY ? m[f] : m[f] + (lq > 1.f ? __log2f(lq) : 0.f), mx);
                const float alpha = m[f] == -INFINITY ? 1.f : __builtin_amdgcn_exp2f(m[f] - m_new);
                m[f] = m_new;
                l[f] *= alpha;
#pragma unroll
                for (int t = 0; t < DT; ++t)
#pragma unroll
                    for (int r = 0; r < 4; ++r) o[f][t][r] *= alpha;
                const float mn = m_new == -INFINITY ? 0.f : m_new;
                sum = 0.f;
#pragma unroll
                for (int r = 0; r < 8; ++r) {
                    w[r] = __builtin_amdgcn_exp2f(x[r] - mn);
                    sum += w[r];
                }
            }
            l[f] += sum;
            const bf16x8 p = __builtin_convertvector(w, bf16x8);
            const bf16x8 rest = __builtin_convertvector(w - __builtin_convertvector(p, f32x8), bf16x8);
#pragma unroll
            for (int t = 0; t < DT; ++t)
                o[f][t] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(__builtin_bit_cast(bf16x8, ch.v[t]), p, o[f][t], 0, 0, 0);
#pragma unroll
            for (int t = 0; t < DT; ++t)
                o[f][t] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(__builtin_bit_cast(bf16x8, ch.v[t]), rest, o[f][t], 0, 0, 0);
        }
    };
    int c = 2 * cut * per + wave;
    if (c < c_end) {
        Pages pg = pages_of(c);
        for (; c < c_end; c += NW) {
            Chunk one;
            load(c, pg, one);
            pg = pages_of(c + NW);                              // one chunk ahead
            attend(c, one);
        }
    }

    // Infinite and NaN values, for the rows that see them: rare.  Those of masked chunks have been taken out, others have met a weight in two
    // parts, the second of which may be 0 or negative.  What a row has of them in a dim is counted, by products of 0 and 1: those that make it
    // +infinite or NaN, and -infinite or NaN.  Finite terms do not matter where there is one.
    bool left = put_back;
#pragma unroll
    for (int f = 0; f < MF; ++f)
#pragma unroll
        for (int t = 0; t < DT; ++t)
#pragma unroll
            for (int r = 0; r < 4; ++r) left |= !(fabsf(o[f][t][r]) < INFINITY);
    if (__any(left)) {
#pragma unroll 1
        for (int tt = 0; tt < DT; ++tt) {
            f32x4 up[MF], down[MF];
#pragma unroll
            for (int f = 0; f < MF; ++f) up[f] = down[f] = f32x4{0.f, 0.f, 0.f, 0.f};
#pragma unroll 1
            for (int cc = 2 * cut * per + wave; cc < c_end; cc += NW) {
                const u32x4 v = *reinterpret_cast<const u32x4*>(v_of(cc, pages_of(cc)) + 16 * tt * page);
                u32x4 ups = {0u, 0u, 0u, 0u}, downs = ups;
#pragma unroll
                for (int x = 0; x < 8; ++x) {
                    const uint32_t u = v[x >> 1] >> (16 * (x & 1)) & 0xffffu, one = 0x3f80u << (16 * (x & 1));
                    const bool nan = (u & 0x7fffu) > 0x7f80u;
                    ups[x >> 1] |= nan || u == 0x7f80u ? one : 0u;
                    downs[x >> 1] |= nan || u == 0xff80u ? one : 0u;
                }
                if (!__any((ups[0] | ups[1] | ups[2] | ups[3] | downs[0] | downs[1] | downs[2] | downs[3]) != 0)) continue;
#pragma unroll
                for (int f = 0; f < MF; ++f) {
                    f32x8 seen;
#pragma unroll
                    for (int r = 0; r < 8; ++r) seen[r] = sees(a, pos[f], key_of(cc) + 8 * g + r) ? 1.f : 0.f;
                    const bf16x8 s = __builtin_convertvector(seen, bf16x8);
                    up[f] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(__builtin_bit_cast(bf16x8, ups), s, up[f], 0, 0, 0);
                    down[f] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(__builtin_bit_cast(bf16x8, downs), s, down[f], 0, 0, 0);
                }
            }
#pragma unroll
            for (int f = 0; f < MF; ++f)
#pragma unroll
                for (int r = 0; r < 4; ++r) {
                    const float value = up[f][r] > 0.f ? (down[f][r] > 0.f ? NAN : INFINITY) : -INFINITY;
                    const bool some = up[f][r] + down[f][r] > 0.f;
#pragma unroll
                    for (int t = 0; t < DT; ++t) o[f][t][r] = some && t == tt ? value : o[f][t][r];
                }
        }
    }

    // The wavefronts' results of a row become one: every wavefront leaves its sums, relative to its own reference
#pragma unroll
    for (int f = 0; f < MF; ++f) {
        const float lq = sum_over_groups(l[f]);
        if (g == 0) { s_m[wave][16 * f + n16] = m[f]; s_l[wave][16 * f + n16] = lq; }
    }
    const bool partial = sh.s.splits > 1;
    const int slot = sh.slot + sh.unit;
    if (partial && (unsigned)slot >= (unsigned)part.n_slots) return;                // starts that are not ascending: more units than there is room for
#pragma unroll
    for (int f = 0; f < MF; ++f) {
        if (f > 0) __syncthreads();
#pragma unroll
        for (int t = 0; t < DT; ++t) *reinterpret_cast<f32x4*>(&s_o[wave][n16][16 * t + 4 * g]) = o[f][t];
        __syncthreads();
        constexpr int VPT = DV == 128 ? 8 : 4, TPR = DV / VPT;   // values of a thread, threads of a row
        const int r16 = tid / TPR, d0 = tid % TPR * VPT;
        const int row = row0 + 16 * f + r16;
        if (r16 < 16 && row <= last_row) {
            float mx = -INFINITY;
#pragma unroll
            for (int w = 0; w < NW; ++w) mx = fmaxf(mx, s_m[w][16 * f + r16]);
            float lsum = 0.f, acc[VPT];
#pragma unroll
            for (int x = 0; x < VPT; ++x) acc[x] = 0.f;
#pragma unroll
            for (int w = 0; w < NW; ++w) {
                const float mw = s_m[w][16 * f + r16];
                const float scale = mw == -INFINITY ? 0.f : __builtin_amdgcn_exp2f(mw - mx);
                lsum = fmaf(s_l[w][16 * f + r16], scale, lsum);
#pragma unroll
                for (int x = 0; x < VPT; ++x) acc[x] = fmaf(s_o[w][r16][d0 + x], scale, acc[x]);
            }
            const bool none = mx == -INFINITY && lsum == 0.f;    // no finite logit (in this piece); NaN is not none
            const float inv = none ? (partial ? 0.f : without_logits(pos0 + row / a.G)) : 1.f / lsum;
            const float lse2 = none ? (partial ? kNoLogit : -INFINITY) : mx + __log2f(lsum);
            if (partial) {
                float* po = part.o + ((int64_t)slot * part.m + 16 * f + r16) * D + dv0 + d0;
#pragma unroll
                for (int x = 0; x < VPT; ++x) po[x] = acc[x] * inv;
                if (tid % TPR == 0 && dv0 == 0) part.lse[(int64_t)slot * part.m + 16 * f + r16] = lse2;
            } else {
                const int tok = sh.r.first + row / a.G, hd = kvh * a.G + row % a.G;
                uint16_t* orow = a.out + (int64_t)tok * a.o_t + hd * a.o_h + dv0 + d0;
#pragma unroll
                for (int x = 0; x < VPT; x += 4) {
                    const f32x4 v = {acc[x] * inv, acc[x + 1] * inv, acc[x + 2] * inv, acc[x + 3] * inv};
                    *reinterpret_cast<bf16x4*>(orow + x) = __builtin_convertvector(v, bf16x4);
                }
                if (a.lse != nullptr && tid % TPR == 0 && dv0 == 0) a.lse[(int64_t)tok * a.Hq + hd] = lse2 * kLn2;
            }
        }
    }
}

template <int D, int MF, bool MOD, bool SMALL, int NW, int NV>
__global__ __launch_bounds__(64 * NW, MF > 1 ? 2 : D == 64 ? 5 : 3) void paged_few_kernel(PagedArgs a, PagedPart part, unsigned units) {
    __shared__ __attribute__((aligned(16))) char lds[kFewLds<D, MF, NW, NV>];
    few_rows<D, MF, MOD, SMALL, NW, NV>(a, part, blockIdx.x, units, lds);
}

// ---------------------------------------------------------------------------------------------------------------
// Many rows: 128 of them, 32 to a wavefront, S^T = K Q^T and O^T += V^T P^T with v_mfma_f32_32x32x16_bf16 on key tiles that all
// four share through LDS: the pipeline step of the sparse prefill's attention kernel (attn.hip: direct loads into a double
// buffer, logits two 32-key chunks ahead of the second product, one barrier a tile), with pages in place of blocks, masks
// where a tile needs them instead of in the last block, and logits that may be capped or biased.  2048 tokens over 98304 of 32 / 8
// heads: 2.97 to 3.2 ms by card, 1.03 to 1.12 PFLOP/s (a plain product of 8192^3: 1.33), matrix cores busy 56 % at 1.8 GHz; with
// head_dim 64, where the exponentials weigh twice as much, 0.78 to 0.84, capped 0.88 to 0.91 and 0.56.
// The keys are taken from the last tile to the first: with a bias that falls with the distance a row then meets its largest
// logits first and its reference hardly moves.
constexpr int kManyRows = 128;

enum Mode { kPlain, kSlopes, kCapped, kCappedSlopes };   // scaled products; with a bias by distance; capped; both

// What the running softmax of a wavefront needs of its row for a chunk: the weight of the product s in register r (key key0 +
// 16 (r / 8) + 8 half + r % 8) is 2^(s c + bias(r)), or with a cap 2^(bias(r) - 2 cap2 / (1 + 2^(s k))), the same as
// cap2 tanh(...) since tanh y = 1 - 2 / (1 + e^2y).  bias holds - m, the cap and the slope's share.
template <int MODE>
struct ChunkWeights {
    static constexpr bool kCap = MODE == kCapped || MODE == kCappedSlopes, kBias = MODE == kSlopes || MODE == kCappedSlopes;
    float c, k, cap2, slope2, base;
    static __device__ __forceinline__ constexpr int key_of(int r) { return 16 * (r >> 3) + (r & 7); }
    // ahead: position of register 0's key less the row's own.  The biases are counted from the lane's last key (r = 15): for keys
    // that all lie at or before the row the two parts have one sign, so no precision is lost where a bias is small.
    __device__ __forceinline__ void at(float m, int ahead) {
        const float less_m = kCap ? cap2 - m : -m;
        base = kBias ? fmaf(slope2, (float)(ahead + key_of(15)), less_m) : less_m;
    }
    __device__ __forceinline__ float bias(int r) const { return kBias ? fmaf(slope2, (float)(key_of(r) - key_of(15)), base) : base; }
    __device__ __forceinline__ float growth(float s) const { return __builtin_amdgcn_exp2f(s * k); }
    // the exponent as a masked chunk needs it, where keys lie on both sides of the row
    __device__ __forceinline__ float exponent(float s, int r, float m, int ahead) const {
        const float less_m = kCap ? cap2 - m : -m;
        const float b = kBias ? fmaf(slope2, (float)(ahead + key_of(r)), less_m) : less_m;
        if constexpr (kCap) return fmaf(-2.f * cap2, __builtin_amdgcn_rcpf(1.f + growth(s)), b);
        else return fmaf(s, c, b);
    }
};

// Instruction group g of a step, its share of the softmax arithmetic: as group_weights (attn_parts.hpp), for all modes; the
// denominator takes the weights in fp32, so that the log-sum-exp is as exact as the logits.
template <int g, int D, int MODE>
__device__ __forceinline__ void group_mode_weights(const f32x16& s, const ChunkWeights<MODE>& cw, f32x8& e, bf16x8& pn0, bf16x8& pn1, float& l_new) {
    constexpr int NG = D / 8, HG = NG / 2;
    constexpr int hb = (g / HG) * 8, gg = g % HG;
    constexpr bool first_half = g < HG, kCap = ChunkWeights<MODE>::kCap;
    auto linear = [&](int x0, int n) {
#pragma unroll
        for (int x = x0; x < x0 + n; ++x) e[x] = fmaf(s[hb + x], cw.c, cw.bias(hb + x));
    };
    auto grow = [&](int x0, int n) {
#pragma unroll
        for (int x = x0; x < x0 + n; ++x) e[x] = cw.growth(s[hb + x]);
    };
    auto turn = [&](int x0, int n) {
#pragma unroll
        for (int x = x0; x < x0 + n; ++x) e[x] = __builtin_amdgcn_rcpf(1.f + e[x]);
    };
    auto capped = [&](int x0, int n) {
#pragma unroll
        for (int x = x0; x < x0 + n; ++x) e[x] = fmaf(-2.f * cw.cap2, e[x], cw.bias(hb + x));
    };
    auto exps = [&](int x0, int n) {
#pragma unroll
        for (int x = x0; x < x0 + n; ++x) e[x] = __builtin_amdgcn_exp2f(e[x]);
    };
    auto finish = [&]() {
#pragma unroll
        for (int x = 0; x < 8; ++x) l_new += e[x];
        if constexpr (first_half) pn0 = __builtin_convertvector(e, bf16x8);
        else pn1 = __builtin_convertvector(e, bf16x8);
        if constexpr (g == NG - 1) asm volatile("" : "+v"(l_new));   // keep the sums inside their groups
    };
    if constexpr (HG == 8 && !kCap) {
        if constexpr (gg < 2) linear(4 * gg, 4);
        else if constexpr (gg < 6) exps(2 * (gg - 2), 2);
        else if constexpr (gg == 7) finish();
    } else if constexpr (HG == 8) {
        if constexpr (gg < 2) grow(4 * gg, 4);
        else if constexpr (gg < 4) turn(4 * (gg - 2), 4);
        else if constexpr (gg == 4) { capped(0, 8); exps(0, 1); }
        else if constexpr (gg == 5) exps(1, 4);
        else if constexpr (gg == 6) exps(5, 3);
        else finish();
    } else if constexpr (!kCap) {
        if constexpr (gg == 0) linear(0, 8);
        else if constexpr (gg < 3) exps(4 * (gg - 1), 4);
        else finish();
    } else {
        if constexpr (gg == 0) grow(0, 8);
        else if constexpr (gg == 1) turn(0, 8);
        else if constexpr (gg == 2) { capped(0, 8); exps(0, 4); }
        else { exps(4, 4); finish(); }
    }
}

// 16 bytes per lane straight into LDS, each lane from an address of its own
template <int IMM>
__device__ __forceinline__ void lds_dma16_from(uint32_t lds_addr, const void* lane_addr) {
    asm volatile("s_add_u32 m0, %0, %2\n\ts_nop 0\n\tglobal_load_lds_dwordx4 %1, off"
                 :
                 : "s"(lds_addr), "v"(lane_addr), "i"(IMM)
                 : "memory", "m0", "scc");
}
// this wavefront's direct loads have landed
__device__ __forceinline__ void wait_for_loads() { asm volatile("s_waitcnt vmcnt(0)" ::: "memory"); }

template <int D, int MODE, bool SMALL>
__device__ __forceinline__ void many_rows(const PagedArgs& a, const PagedPart& part, unsigned wg, char* lds) {
    constexpr int NW = 4;
    constexpr int KT = kPagedTile;
    constexpr int DS = D / 16;          // MFMAs of one logits tile
    constexpr int DT = D / 32;          // 32-row tiles of O^T
    constexpr int NG = 2 * DS;          // instruction groups of a step
    constexpr int TILE = KT * D;
    constexpr int CPR = D / 8;          // 16-byte chunks of a K row
    constexpr int RPI = 64 / CPR;       // K rows filled by one 1-KB load instruction
    constexpr int LPW = TILE / 512 / NW;  // 1-KB load instructions per wave per operand per tile
    constexpr int TILE_B = TILE * 2;
    constexpr int CHUNK_B = 32 * D * 2;
    constexpr int DTILE_B = 32 * KT * 2;
    static_assert(RPI * LPW == 16, "a wavefront loads 16 keys' rows, which lie in one page");
    uint16_t (*const smemK)[TILE] = reinterpret_cast<uint16_t (*)[TILE]>(lds);      // K tile t in buffer t % 2
    uint16_t (*const smemV)[TILE] = smemK + 2;                                      // V^T likewise

    const Request first = request_at(a, threadIdx.x & 63);
    const int piece = part_piece<true>(a, part, first, threadIdx.x & 63);
    if (part.n_slots > 0 && wg == 0 && threadIdx.x == 0) *part.piece = piece;
    const Share sh = share_of<false>(a, part, piece, first, wg);
    if (sh.b < 0) return;
    const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6);
    const int half = lane >> 5, l32 = lane & 31;
    const int kvh = sh.unit % a.Hkv, cut = sh.unit / a.Hkv % sh.s.splits, tile = sh.s.tiles - 1 - sh.unit / a.Hkv / sh.s.splits;
    const int rows = sh.r.len * a.G, row0 = tile * kManyRows;
    const int last_row = min(row0 + kManyRows, rows) - 1;
    const int pos0 = sh.r.kv - sh.r.len;
    const int pos_lo = pos0 + row0 / a.G, pos_hi = pos0 + last_row / a.G;      // of the workgroup's rows
    const KeyTiles kt = key_tiles(pos_lo, pos_hi, a.sink, a.window);
    const int per = tiles_of_piece(sh.s);
    const int e0 = cut * per;
    const int n_st = min((cut + 1) * per, kt.n) - e0;                         // key tiles of this workgroup
    const bool partial = sh.s.splits > 1;
    const int slot = sh.slot + sh.unit;
    if (partial && (unsigned)slot >= (unsigned)part.n_slots) return;

    const int row = min(row0 + 32 * wave + l32, last_row);                    // rows past the last repeat it; they are not stored
    const bool valid = row0 + 32 * wave + l32 <= last_row;
    const int token = row / a.G, head = kvh * a.G + row % a.G, pos = pos0 + token;
    auto store_lse = [&](int at, float lse2) {                                // at: the row, counted from the workgroup's first
        if (partial) {
            part.lse[(int64_t)slot * kManyRows + at] = lse2;
        } else if (a.lse != nullptr) {
            const int r = row0 + at;
            a.lse[(int64_t)(sh.r.first + r / a.G) * a.Hq + kvh * a.G + r % a.G] = lse2 * kLn2;
        }
    };
    auto out_row = [&](int at) {
        const int r = row0 + at;
        return a.out + (int64_t)(sh.r.first + r / a.G) * a.o_t + (kvh * a.G + r % a.G) * a.o_h;
    };
    if (n_st <= 0) {                                                          // no key in sight (of this piece)
        if (valid && half == 0) {
            store_lse(32 * wave + l32, -INFINITY);
            if (!partial) {
                uint16_t* const orow = out_row(32 * wave + l32);
#pragma unroll
                for (int x = 0; x < D / 8; ++x) *reinterpret_cast<u32x4*>(orow + 8 * x) = u32x4{0u, 0u, 0u, 0u};
            }
        }
        return;
    }

    const int last_col = pos_hi >> a.log_p;
    const int page = 1 << a.log_p;
    const int32_t* const trow = a.table + (int64_t)sh.b * a.table_stride;
    const char* const kbase = reinterpret_cast<const char*>(a.k + kvh * a.kp_h);
    const char* const vbase0 = reinterpret_cast<const char*>(a.vt + kvh * a.vp_h);
    auto key_of = [&](int t) { return kt.at(kt.n - 1 - e0 - t) * KT; };       // first key of tile t: the last tiles first
    auto page_of = [&](int key) { return clamp_int(trow[min(key >> a.log_p, last_col)], 0, a.n_pages - 1); };
    struct Pages {                                                            // of a tile's 16-key pieces (one page without SMALL)
        int id[SMALL ? 4 : 1];
    };
    auto pages_of = [&](int t) {
        Pages p;
        const int key0 = key_of(min(t, n_st - 1));
#pragma unroll
        for (int x = 0; x < (SMALL ? 4 : 1); ++x) p.id[x] = page_of(key0 + 16 * x);
        return p;
    };

    uint32_t k_offb[LPW], v_offb[LPW];
    int v_chunk[2];                                                           // 8-key chunk of the tile, for even and odd instructions
#pragma unroll
    for (int x = 0; x < LPW; ++x) {
        const int inst = wave * LPW + x;
        const int krow = RPI * inst + lane / CPR, vrow = 8 * inst + (lane >> 3);
        k_offb[x] = 2u * (uint32_t)((RPI * x + lane / CPR) * D + (((lane % CPR) ^ swz_k<D>(krow)) << 3));
        const int chunk = (lane & 7) ^ swz_v(vrow);
        if (x < 2) v_chunk[x] = chunk;
        v_offb[x] = 2u * (uint32_t)(vrow * page + (SMALL ? (chunk & 1) : chunk) * 8);
    }
    const uint32_t k_dst = lds_address(&smemK[0][0]) + wave * LPW * 1024;
    const uint32_t v_dst = lds_address(&smemV[0][0]) + wave * LPW * 1024;
    // With head_dim 64 (two loads of a wavefront) the second offset follows from the first, 8 rows on with bit 2 of the chunk turned:
    // one register less for each operand
    auto second = [&](const uint32_t (&off)[LPW], auto x_tag, int rows_b) {
        constexpr int X = decltype(x_tag)::value;
        if constexpr (D == 64 && X == 1) {
            uint32_t first = off[0];
            asm volatile("" : "+v"(first));
            return (first ^ 64u) + (uint32_t)rows_b;
        } else {
            return off[X];
        }
    };
    auto issue_k = [&](auto buf_tag, int t, const Pages& pg) {
        constexpr int BUF = decltype(buf_tag)::value;
        const int key = key_of(t) + 16 * wave;                                // this wavefront's 16 keys
        int id = pg.id[0];
        if constexpr (SMALL) id = __builtin_amdgcn_readfirstlane(wave == 0 ? pg.id[0] : wave == 1 ? pg.id[1] : wave == 2 ? pg.id[2] : pg.id[3]);
        const char* const src = kbase + 2 * ((int64_t)id * a.kp_p + (key & (page - 1)) * D);
        static_for<LPW>([&](auto x_tag) {
            constexpr int X = decltype(x_tag)::value;
            lds_dma16<BUF * TILE_B + X * 1024>(k_dst, second(k_offb, x_tag, RPI * D * 2), src);
        });
    };
    auto issue_v = [&](auto buf_tag, int t, const Pages& pg) {
        constexpr int BUF = decltype(buf_tag)::value;
        const int key0 = key_of(t);
        if constexpr (!SMALL) {
            const char* const src = vbase0 + 2 * ((int64_t)pg.id[0] * a.vp_p + (key0 & (page - 1)));
            static_for<LPW>([&](auto x_tag) {
                constexpr int X = decltype(x_tag)::value;
                lds_dma16<BUF * TILE_B + X * 1024>(v_dst, second(v_offb, x_tag, 16 * page), src);
            });
        } else {
            const char* src[2];
#pragma unroll
            for (int x = 0; x < 2; ++x) {
                const int piece = v_chunk[x] >> 1;
                const int id = piece == 0 ? pg.id[0] : piece == 1 ? pg.id[1] : piece == 2 ? pg.id[2] : pg.id[3];
                src[x] = vbase0 + 2 * ((int64_t)id * a.vp_p + ((key0 + 16 * piece) & (page - 1)));
            }
            static_for<LPW>([&](auto x_tag) {
                constexpr int X = decltype(x_tag)::value;
                lds_dma16_from<BUF * TILE_B + X * 1024>(v_dst, src[X % 2] + v_offb[X]);
            });
        }
    };
    // Values of keys that no row of the workgroup sees may be anything, NaN too, and a weight of 0 would not hide them: they
    // become 0 in LDS.  Where some rows see a key and others do not, its infinite and NaN values are taken out and come back at the
    // end.  A wavefront does so for what it has loaded itself, before the barrier that publishes the tile.
    const int gone_hi = a.window > 0 ? pos_lo - a.window + 1 : 0;             // keys sink .. gone_hi - 1 are out of sight
    uint32_t put_back = 0;
    auto clear_unseen = [&](auto buf_tag, int t) {
        constexpr int BUF = decltype(buf_tag)::value;
        const int key0 = key_of(t);
        if (!hides(a, pos_lo, pos_hi, key0, KT)) return;
        const bool unseen = key0 + KT - 1 > pos_hi || (key0 + KT - 1 >= a.sink && key0 < gone_hi);
        u32x4* const at = reinterpret_cast<u32x4*>(reinterpret_cast<char*>(&smemV[BUF][0]) + wave * LPW * 1024 + lane * 16);
        int of = lane;                                      // the chunks found anew, not kept in registers
        asm volatile("" : "+v"(of));
#pragma unroll
        for (int x = 0; x < LPW; ++x) {
            const int chunk = (of & 7) ^ swz_v(8 * (wave * LPW + x) + (of >> 3));
            u32x4 v = at[64 * x];
            bool odd = false;
#pragma unroll
            for (int y = 0; y < 4; ++y) {
                const int ka = key0 + 8 * chunk + 2 * y, kb = ka + 1;
                v[y] &= (ka <= pos_hi && !(ka >= a.sink && ka < gone_hi) ? 0xffffu : 0u) |
                        (kb <= pos_hi && !(kb >= a.sink && kb < gone_hi) ? 0xffff0000u : 0u);
                odd |= not_finite(v[y]);
            }
            const bool some = __any(odd);
            if (some) {
                put_back = 1;
#pragma unroll
                for (int y = 0; y < 4; ++y) v[y] = finite_part(v[y]);
            }
            if (unseen || some) at[64 * x] = v;
        }
    };

    Pages pg1 = pages_of(1);
    {
        const Pages pg0 = pages_of(0);
        issue_k(IC<0>{}, 0, pg0);
        issue_v(IC<0>{}, 0, pg0);
        if (n_st > 1) issue_k(IC<1>{}, 1, pg1);
    }

    bf16x8 qf[DS];
    {
        const uint16_t* const qrow = a.q + (int64_t)(sh.r.first + token) * a.q_t + head * a.q_h + 8 * half;
#pragma unroll
        for (int s = 0; s < DS; ++s) qf[s] = *reinterpret_cast<const bf16x8*>(qrow + 16 * s);
    }
    int kofs[DS], vofs[4];
    {
        const int krow = swap_bits23(l32);
#pragma unroll
        for (int s = 0; s < DS; ++s) kofs[s] = 2 * (krow * D + (((2 * s + half) ^ swz_k<D>(krow)) << 3));
#pragma unroll
        for (int x = 0; x < 4; ++x) vofs[x] = 2 * (l32 * KT + (((2 * x + half) ^ swz_v(l32)) << 3));
    }
    const char* const ldsK = reinterpret_cast<const char*>(&smemK[0][0]);
    const char* const ldsV = reinterpret_cast<const char*>(&smemV[0][0]);
    auto lds16 = [](const char* p) { return *reinterpret_cast<const bf16x8*>(p); };

    // Running softmax, in base 2.  m: the reference; l: the lane's share of the denominator, infinite (which sends the row to the slow path)
    // until the row has seen a key.
    f32x16 oacc[DT];
#pragma unroll
    for (int dc = 0; dc < DT; ++dc)
#pragma unroll
        for (int r = 0; r < 16; ++r) oacc[dc][r] = 0.f;
    ChunkWeights<MODE> cw;
    cw.c = a.scale * kLog2e;
    cw.cap2 = a.cap * kLog2e;
    cw.k = ChunkWeights<MODE>::kCap ? fminf(2.f * cw.c / a.cap, 3e38f) : 0.f;     // finite, so that a product of 0 stays 0
    cw.slope2 = ChunkWeights<MODE>::kBias ? a.slopes[head] * kLog2e : 0.f;
    float m = 0.f, l = INFINITY;
    const int wave_row = row0 + 32 * wave;                                    // wave-uniform bounds of this wavefront's rows
    const int wave_lo = pos0 + min(wave_row, last_row) / a.G, wave_hi = pos0 + min(wave_row + 31, last_row) / a.G;
    auto needs_mask = [&](int key0) { return hides(a, wave_lo, wave_hi, key0, 32); };
    // Slow path of a chunk: masks, and a reference that makes its weights at most 1 and the denominator so far about 1 or less.
    // For the first chunk, masked ones, and where the denominator passed the limit.
    auto slow_weights = [&](const f32x16& s, int key0, bf16x8& p0, bf16x8& p1) __attribute__((always_inline)) {
        const int back = pos - key0 - 8 * half;
        f32x16 x;
#pragma unroll
        for (int r = 0; r < 16; ++r) x[r] = cw.exponent(s[r], r, 0.f, -back);
        uint32_t hidden = 0;
        if (needs_mask(key0)) {
#pragma unroll
            for (int r = 0; r < 16; ++r) {
                if (!sees(a, pos, pos - back + ChunkWeights<MODE>::key_of(r))) {
                    hidden |= 1u << r;
                    x[r] = -INFINITY;
                }
            }
        }
        float mx = x[0];
#pragma unroll
        for (int r = 1; r < 16; ++r) mx = fmaxf(mx, x[r]);
        mx = fmaxf(mx, other_half(mx));
        const float lq = l + other_half(l);
        const bool first = l == INFINITY;
        const float m_new = fmaxf(first ? -INFINITY : m + (lq > 1.f ? __log2f(lq) : 0.f), mx);
        const float alpha = first ? 1.f : __builtin_amdgcn_exp2f(m - m_new);
        m = m_new == -INFINITY ? 0.f : m_new;
        l = m_new == -INFINITY ? INFINITY : first ? 0.f : l * alpha;
#pragma unroll
        for (int dc = 0; dc < DT; ++dc)
#pragma unroll
            for (int r = 0; r < 16; ++r) oacc[dc][r] *= alpha;
        f32x8 w0, w1;
#pragma unroll
        for (int r = 0; r < 8; ++r) {
            w0[r] = (hidden >> r) & 1 ? 0.f : __builtin_amdgcn_exp2f(cw.exponent(s[r], r, m, -back));
            w1[r] = (hidden >> (8 + r)) & 1 ? 0.f : __builtin_amdgcn_exp2f(cw.exponent(s[8 + r], 8 + r, m, -back));
        }
#pragma unroll
        for (int r = 0; r < 8; ++r) l += w0[r] + w1[r];
        p0 = __builtin_convertvector(w0, bf16x8);
        p1 = __builtin_convertvector(w1, bf16x8);
    };
    // first tile with a key in sight of this wavefront; two tiles and more before it, its steps would do nothing.  n_st + 1: no rows
    int first_tile = n_st + 1;
    if (wave_row <= last_row && wave_hi >= 0) {
        first_tile = 0;
        while (first_tile < n_st && key_of(first_tile) > wave_hi) ++first_tile;
    }

    // key0: of the chunk whose products s_cur become weights
    auto step = [&](auto kb_tag, auto vb_tag, auto kc_tag, int key0, const f32x16& s_cur, f32x16& s_nxt, const bf16x8& pc0, const bf16x8& pc1,
                    bf16x8& pn0, bf16x8& pn1, bf16x8 (&f)[4]) __attribute__((always_inline)) {
        constexpr int KB = decltype(kb_tag)::value, VB = decltype(vb_tag)::value, KC = decltype(kc_tag)::value;
        cw.at(m, key0 + 8 * half - pos);
        const char* const vbase = ldsV + VB * TILE_B;
        int vslice[2] = {vofs[2 * KC], vofs[2 * KC + 1]};      // the second chunk's 8-key slices have bit 2 turned: found from the first's
        if constexpr (D == 64 && KC == 1) {
            vslice[0] = vofs[0];
            vslice[1] = vofs[1];
            asm volatile("" : "+v"(vslice[0]), "+v"(vslice[1]));
            vslice[0] ^= 64;
            vslice[1] ^= 64;
        }
        auto operand = [&](auto j_tag) {            // operand j of this step (j < NG) or of the next one
            constexpr int J = decltype(j_tag)::value;
            constexpr int j = J % NG;
            constexpr int kc = KC + J / NG;
            const char* const kb2 = ldsK + KB * TILE_B + kc * CHUNK_B;
            if constexpr (j % 2 == 0) return lds16(kb2 + kofs[j / 2]);
            else return lds16(vbase + (kc == KC ? vslice[(j / 2) / DT] : vofs[2 * kc + (j / 2) / DT]) + ((j / 2) % DT) * DTILE_B);
        };
        f32x8 e;
        float l_new = l;
        auto group = [&](auto g_tag) {
            constexpr int g = decltype(g_tag)::value;
            group_mfma<g, D>(f[g % 4], qf, s_nxt, oacc, pc0, pc1);
            if constexpr (g + 3 < NG || KC == 0) f[(g + 3) % 4] = operand(IC<g + 3>{});
            group_mode_weights<g, D, MODE>(s_cur, cw, e, pn0, pn1, l_new);
            SPA_FENCE();
        };
        SPA_FENCE();
        static_for<NG>([&](auto g_tag) { group(g_tag); });
        if (needs_mask(key0) || __any(!(l_new < kRescaleAt))) slow_weights(s_cur, key0, pn0, pn1);
        else l = l_new;
    };

    // ---- logits of the two chunks of tile 0, weights of chunk 0
    wait_for_loads();
    clear_unseen(IC<0>{}, 0);
    __syncthreads();
    f32x16 sA, sB;                                 // logits of even / odd chunks
#pragma unroll
    for (int r = 0; r < 16; ++r) { sA[r] = 0.f; sB[r] = 0.f; }
#pragma unroll
    for (int s = 0; s < DS; ++s) {
        sA = __builtin_amdgcn_mfma_f32_32x32x16_bf16(lds16(ldsK + kofs[s]), qf[s], sA, 0, 0, 0);
        sB = __builtin_amdgcn_mfma_f32_32x32x16_bf16(lds16(ldsK + CHUNK_B + kofs[s]), qf[s], sB, 0, 0, 0);
    }
    bf16x8 pA0, pA1, pB0, pB1;                     // weights of even / odd chunks
    slow_weights(sA, key_of(0), pA0, pA1);

    Pages pg2 = pages_of(2);
    // tile t = steps 2t and 2t + 1: reads K(t + 1) (logits ahead) and V^T(t)
    auto one_tile = [&](auto par_tag, int t) __attribute__((always_inline)) {
        constexpr int PAR = decltype(par_tag)::value;      // t % 2
        using KB = IC<1 - PAR>;
        using VB = IC<PAR>;
        if (t > 0) {                                       // K(t + 1) and V^T(t) have been requested
            wait_for_loads();
            clear_unseen(VB{}, t);
        }
        __syncthreads();                                   // they are there, and the buffers refilled below have been read
        bf16x8 f[4];
        f[0] = lds16(ldsK + KB::value * TILE_B + kofs[0]);
        f[1] = lds16(ldsV + VB::value * TILE_B + vofs[0]);
        f[2] = lds16(ldsK + KB::value * TILE_B + kofs[1]);
        if (t + 2 < n_st) issue_k(IC<PAR>{}, t + 2, pg2);
        if (t + 1 < n_st) issue_v(IC<1 - PAR>{}, t + 1, pg1);
        pg1 = pg2;
        pg2 = pages_of(t + 3);
        if (t + 1 < first_tile) return;
        step(KB{}, VB{}, IC<0>{}, key_of(t) + 32, sB, sA, pA0, pA1, pB0, pB1, f);
        // past the end: products of a stale buffer, masked like keys behind every position
        step(KB{}, VB{}, IC<1>{}, t + 1 < n_st ? key_of(t + 1) : 1 << 30, sA, sB, pB0, pB1, pA0, pA1, f);
    };
    for (int t = 0;;) {
        one_tile(IC<0>{}, t);
        if (++t == n_st) break;
        one_tile(IC<1>{}, t);
        if (++t == n_st) break;
    }

    // Infinite and NaN values that were taken out, for the rows that see them: rare, so it looks through all the tiles again
    __syncthreads();
    uint32_t* const flags = reinterpret_cast<uint32_t*>(lds);
    if (lane == 0) flags[wave] = put_back;
    __syncthreads();
    if (__builtin_amdgcn_readfirstlane(flags[0] | flags[1] | flags[2] | flags[3])) {
        for (int t = 0; t < n_st; ++t) {
            const int key0 = key_of(t);
            if (!hides(a, pos_lo, pos_hi, key0, KT)) continue;
            for (int key = key0; key < key0 + KT && key <= pos_hi; ++key) {
                const uint16_t* const src = a.vt + page_of(key) * a.vp_p + kvh * a.vp_h + (key & (page - 1));
                int step = page;                                // unknown to the compiler, which would keep all the offsets in registers
                asm volatile("" : "+s"(step));
                if (!sees(a, pos, key)) continue;
#pragma unroll
                for (int dc = 0; dc < DT; ++dc)
#pragma unroll
                    for (int r = 0; r < 16; ++r) {
                        const uint32_t u = src[(32 * dc + 8 * (r >> 2) + 4 * half + (r & 3)) * step];
                        if (not_finite(u)) oacc[dc][r] += __uint_as_float(u << 16);
                        if (r % 4 == 3) asm volatile("" ::: "memory");   // four loads at a time: the registers are for the usual case
                    }
            }
        }
    }

    const float lt = l + other_half(l);
    const bool none = l == INFINITY;         // no finite logit (in this piece); NaN is not none
    const float inv = none ? (partial ? 0.f : without_logits(pos)) : 1.f / lt;
    const float lse2 = none ? (partial ? kNoLogit : -INFINITY) : m + __log2f(lt);
    int at = 32 * wave + l32;
    asm volatile("" : "+v"(at));                           // found anew, not kept in registers all the way
    if (row0 + at > last_row) return;
    if (half == 0) store_lse(at, lse2);
    uint16_t* const orow = out_row(at);
    float* const po = part.o + ((int64_t)slot * kManyRows + at) * D;
#pragma unroll
    for (int dc = 0; dc < DT; ++dc)
#pragma unroll
        for (int rq = 0; rq < 4; ++rq) {
            f32x4 o4;
#pragma unroll
            for (int x = 0; x < 4; ++x) o4[x] = oacc[dc][4 * rq + x] * inv;
            const int d = 32 * dc + 8 * rq + 4 * half;
            if (partial) *reinterpret_cast<f32x4*>(po + d) = o4;
            else *reinterpret_cast<bf16x4*>(orow + d) = __builtin_convertvector(o4, bf16x4);
        }
}

// PAGES: 2, pages of 16 tokens; 1, of 32; 0, a key tile lies in one page.  With head_dim 64 and a key tile in one page three wavefronts share
// a SIMD (prompts of 4000 tokens with slopes 228 -> 197 us); cap and slopes together do not leave the registers for it.
template <int D, int MODE, int PAGES>
__global__ __launch_bounds__(256, D == 64 && PAGES == 0 && MODE != kCappedSlopes ? 3 : 2) void paged_attn_kernel(PagedArgs a, PagedPart many, unsigned many_grid, PagedPart few) {
    __shared__ __attribute__((aligned(1024))) char lds[4 * kPagedTile * D * 2];
    static_assert(kFewLds<D, 1, 4, 1> <= 4 * kPagedTile * D * 2, "few rows fit the tile buffers");
    if (blockIdx.x < many_grid) many_rows<D, MODE, PAGES != 0>(a, many, blockIdx.x, lds);
    else few_rows<D, 1, MODE != kPlain, PAGES == 2, 4, 1>(a, few, blockIdx.x - many_grid, 0, lds);
}

// ---------------------------------------------------------------------------------------------------------------
// Merge of the pieces' results: out = sum_s w_s out_s / sum_s w_s, w_s = 2^(lse_s - max).  A wavefront makes D / NV dims of a row, 64 pieces
// at a time: a lane has the weight of one, then DV / 4 lanes read a piece's values, 64 / (DV / 4) pieces side by side.  NV = 4 for few
// rows: what a CU takes in bounds them (4 requests behind 128K tokens, 128 rows of 64 pieces: 11.7 -> 7.6 us).
template <int D, int NV, bool MANY>
__device__ __forceinline__ void merge_rows(const PagedArgs& a, const PagedPart& part) {
    constexpr int DV = D / NV, LPR = DV / 4, NG = 64 / LPR;       // dims of a wavefront, lanes of a piece, pieces side by side
    const int lane = threadIdx.x & 63;
    const int grp = lane / LPR;
    const Request first = request_at(a, lane);
    // found anew, or, where that takes longer than a load, as the attention kernel has left it
    const int piece = MANY ? __builtin_amdgcn_readfirstlane(*part.piece) : part_piece<false>(a, part, first, lane);
    for (uint32_t item = blockIdx.x * 4 + (threadIdx.x >> 6);; item += gridDim.x * 4) {
        const uint32_t i = (uint32_t)__builtin_amdgcn_readfirstlane((int)item);
        const Share sh = share_of<true>(a, part, piece, first, i / NV);
        if (sh.b < 0) return;
        const int d0 = (int)(i % NV) * DV + 4 * (lane % LPR);
        const int kvh = sh.unit % a.Hkv, row = sh.unit / a.Hkv, splits = sh.s.splits;
        const int tile = row >> part.log_m, rt = row & (part.m - 1);
        const int slot0 = sh.slot + (sh.s.tiles - 1 - tile) * splits * a.Hkv + kvh;
        if (slot0 < 0 || slot0 + (splits - 1) * a.Hkv >= part.n_slots) continue;
        auto at = [&](int s) { return (int64_t)(slot0 + s * a.Hkv) * part.m + rt; };
        float mx = -INFINITY, total = 0.f;
        f32x4 acc = {0.f, 0.f, 0.f, 0.f};
        for (int s0 = 0; s0 < splits; s0 += 64) {
            const float v = s0 + lane < splits ? part.lse[at(s0 + lane)] : -INFINITY;
            float top = v;
#pragma unroll
            for (int x = 32; x > 0; x >>= 1) top = fmaxf(top, __shfl_xor(top, x));     // NaN is dropped here and comes back with the weights
            const float mx_new = fmaxf(mx, top);
            const float old = mx == -INFINITY ? 0.f : __builtin_amdgcn_exp2f(mx - mx_new);
            mx = mx_new;
            const float w = v == -INFINITY ? 0.f : __builtin_amdgcn_exp2f(v - mx);
            const uint64_t with_keys = __ballot(v != -INFINITY);    // of weight 0, too: the piece may hold an infinite or NaN value
            total = fmaf(total, old, w);
            acc *= old;
            const int n = min(64, splits - s0);
            for (int s = 0; s < n; s += 4 * NG) {           // four loads of a lane in flight
                float ws[4];
                bool some[4];
                f32x4 p[4];
#pragma unroll
                for (int y = 0; y < 4; ++y) {
                    const int mine = s + NG * y + grp, there = min(mine, n - 1);
                    ws[y] = __shfl(w, there);
                    some[y] = mine < n && (with_keys >> there & 1) != 0;
                    p[y] = *reinterpret_cast<const f32x4*>(part.o + at(s0 + there) * D + d0);
                }
#pragma unroll
                for (int y = 0; y < 4; ++y)
#pragma unroll
                    for (int x = 0; x < 4; ++x)             // a piece without a key in sight may not have written its values
                        acc[x] = some[y] ? fmaf(p[y][x], ws[y], acc[x]) : acc[x];
            }
        }
#pragma unroll
        for (int x = 1; x < 64; x <<= 1) total += __shfl_xor(total, x);
#pragma unroll
        for (int x = LPR; x < 64; x <<= 1)
#pragma unroll
            for (int y = 0; y < 4; ++y) acc[y] += __shfl_xor(acc[y], x);
        const bool none = total == 0.f || (mx <= kNoLogit && total == total);       // NaN is not none
        const float inv = none ? without_logits(sh.r.kv - sh.r.len + row / a.G) : 1.f / total;
        if (lane < LPR) {
            const int tok = sh.r.first + row / a.G, hd = kvh * a.G + row % a.G;
            *reinterpret_cast<bf16x4*>(a.out + (int64_t)tok * a.o_t + hd * a.o_h + d0) = __builtin_convertvector(acc * inv, bf16x4);
            if (a.lse != nullptr && lane == 0 && d0 == 0) a.lse[(int64_t)tok * a.Hq + hd] = none ? -INFINITY : (mx + __log2f(total)) * kLn2;
        }
    }
}
template <int D, int NV>
__global__ __launch_bounds__(256) void paged_merge_kernel(PagedArgs a, PagedPart few, PagedPart many) {
    if (few.n_slots > 0) merge_rows<D, NV, false>(a, few);
    if (many.n_slots > 0) merge_rows<D, NV, true>(a, many);
}

// Most key tiles of a row tile, by the table's width and the window.  Where they are few, the merge's 5 us are more than pieces save
// (4 tokens behind 1498 keys, window 76: 13.8 -> 9.4 us; 39 behind 1183, window 3: 15.4 -> 11.1).  Few is 8; with 4 a request of 500 keys takes 13.0
// instead of 9.2 us, 180 tokens over 500 22.9 instead of 19.3; with 16 a request of 750 keys 11.4 instead of 13.1, but of 1500 14.1 instead of
// 13.0, and 180 tokens over 1000 30.5 instead of 28.1.
int most_key_tiles_of(const PagedDims& d, const PagedPart& part) { return most_key_tiles(d.T, d.C << d.log_p, part.span, d.sink, d.window); }
// Most workgroups of a part that a call can need, whatever its lengths (2^log_most more than without cuts, and none cut into pieces
// of less than min_tiles)
int64_t most_units(const PagedDims& d, const PagedPart& part) {
    const int64_t requests = d.B < d.T ? d.B : d.T;
    const int64_t tiles = (part.row_hi <= part.m ? requests : (int64_t)d.T * d.G / part.m + requests) * d.Hkv;
    if (most_key_tiles_of(d, part) <= part.whole_tiles) return tiles;
    const int64_t most = 1ll << part.log_most, cuts = (most_key_tiles_of(d, part) + part.min_tiles - 1) / part.min_tiles;
    return tiles * cuts < tiles + most ? tiles * cuts : tiles + most;
}
// Most partial results: requests that are cut have at most twice as many pieces as their work fills
int64_t most_slots(const PagedDims& d, const PagedPart& part) {
    if (most_key_tiles_of(d, part) <= part.whole_tiles) return 0;
    const int64_t units = most_units(d, part), most = 2ll << part.log_most;
    return units < most ? units : most;
}

template <int D, int MF, int NW, int NV>
void launch_few(const PagedArgs& a, const PagedPart& part, unsigned units, hipStream_t st) {
    const bool mod = a.cap > 0.f || a.slopes != nullptr;
    const auto go = [&](auto kernel) { hipLaunchKernelGGL(kernel, dim3(units * NV), dim3(64 * NW), 0, st, a, part, units); };
    if (a.log_p == 4) {
        if (mod) go(paged_few_kernel<D, MF, true, true, NW, NV>);
        else go(paged_few_kernel<D, MF, false, true, NW, NV>);
    } else {
        if (mod) go(paged_few_kernel<D, MF, true, false, NW, NV>);
        else go(paged_few_kernel<D, MF, false, false, NW, NV>);
    }
}

template <int D>
hipError_t launch_parts(const PagedArgs& a, const PagedDims& d, const PagedParts& parts, hipStream_t st) {
    // A call with requests of both kinds runs them side by side, the many-row workgroups first: the ones wait for the matrix cores, the
    // others for the memory (mixed step 431 -> 399 us, 10 short prompts and single tokens 24.8 -> 19.3).  With 17 to 32 query heads of a KV head, one after the other.
    const bool both = parts.many.m && parts.few.m == 16;
    const int64_t few_grid = parts.few.m ? most_units(d, parts.few) : 0, many_grid = parts.many.m ? most_units(d, parts.many) : 0;
    if (few_grid + many_grid > 0x7fffffffll) return hipErrorInvalidValue;
    if (parts.few.m && !both) {
        if (parts.few.m == 32) launch_few<D, 2, 4, 1>(a, parts.few, (unsigned)few_grid, st);
        else if (few_grid <= 64) launch_few<D, 1, 8, 4>(a, parts.few, (unsigned)few_grid, st);
        else launch_few<D, 1, 4, 1>(a, parts.few, (unsigned)few_grid, st);
        const hipError_t e = hipGetLastError();
        if (e != hipSuccess) return e;
    }
    if (parts.many.m) {
        const auto go = [&](auto kernel) {
            hipLaunchKernelGGL(kernel, dim3((unsigned)(many_grid + (both ? few_grid : 0))), dim3(256), 0, st, a, parts.many, (unsigned)many_grid, parts.few);
        };
        const auto with_pages = [&](auto mode) {
            constexpr int MODE = decltype(mode)::value;
            if (a.log_p == 4) go(paged_attn_kernel<D, MODE, 2>);
            else if (a.log_p == 5) go(paged_attn_kernel<D, MODE, 1>);
            else go(paged_attn_kernel<D, MODE, 0>);
        };
        if (a.cap > 0.f && a.slopes != nullptr) with_pages(IC<kCappedSlopes>{});
        else if (a.cap > 0.f) with_pages(IC<kCapped>{});
        else if (a.slopes != nullptr) with_pages(IC<kSlopes>{});
        else with_pages(IC<kPlain>{});
        const hipError_t e = hipGetLastError();
        if (e != hipSuccess) return e;
    }
    if (parts.few.n_slots + parts.many.n_slots == 0) return hipSuccess;
    const int64_t rows = (int64_t)d.T * d.Hq;
    if (rows <= 1024) hipLaunchKernelGGL((paged_merge_kernel<D, 4>), dim3((unsigned)rows), dim3(256), 0, st, a, parts.few, parts.many);
    else hipLaunchKernelGGL((paged_merge_kernel<D, 1>), dim3(1024), dim3(256), 0, st, a, parts.few, parts.many);
    return hipGetLastError();
}

}  // namespace

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
    const PagedArgs a{(const uint16_t*)q, (const uint16_t*)k_pages, (const uint16_t*)vt_pages, block_table, q_starts, kv_lens, slopes_or_null,
                      (uint16_t*)out, lse_or_null, d.B, d.Hq, d.Hkv, d.G, d.T, d.log_p, d.n_pages, d.C, d.sink, d.window, d.scale, d.cap,
                      d.table_stride, d.q_t, d.q_h, d.o_t, d.o_h, d.kp_p, d.kp_h, d.vp_p, d.vp_h};
    return d.D == 128 ? launch_parts<128>(a, d, parts, st) : launch_parts<64>(a, d, parts, st);
}

}  // namespace spa
