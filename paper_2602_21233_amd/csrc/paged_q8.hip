// The quantised paged cache: keys and values to e4m3 on their way into the pages, cached tokens back out of them.
#include "e4m3.hpp"
#include "paged.hpp"

namespace spa {
namespace {

__device__ __forceinline__ int64_t place_of(int slot, int log_p, int64_t page_stride, int in_page) {
    return (slot >> log_p) * page_stride + (int64_t)(slot & ((1 << log_p) - 1)) * in_page;
}

// 8 bf16 values as floats
__device__ __forceinline__ void floats_of(const uint4& r, float (&x)[8]) {
    const uint32_t w[4] = {r.x, r.y, r.z, r.w};
#pragma unroll
    for (int y = 0; y < 4; ++y) {
        x[2 * y] = bf16_lo(w[y]);
        x[2 * y + 1] = bf16_hi(w[y]);
    }
}
// a lane's share of a row's largest finite magnitude, over the N lanes of the row
template <int N>
__device__ __forceinline__ float row_amax(const float (&x)[8]) {
    float m = 0.f;
#pragma unroll
    for (int y = 0; y < 8; ++y) m = fmaxf(m, fabsf(finite_or_zero(x[y])));
#pragma unroll
    for (int n = 1; n < N; n <<= 1) m = fmaxf(m, __shfl_xor(m, n));
    return m;
}
__device__ __forceinline__ uint2 quantise8(const float (&x)[8], uint32_t e) {
    const float inv = two_to(254 - e);
    float y[8];
#pragma unroll
    for (int i = 0; i < 8; ++i) y[i] = finite_or_nan(x[i]) * inv;
    return make_uint2(to_e4m3(y[0], y[1], y[2], y[3]), to_e4m3(y[4], y[5], y[6], y[7]));
}

// Few tokens: a thread quantises 8 dims of a token's key and value; D / 8 lanes share their row's maximum.  Bound by latency and the single-byte stores of V
// (256 scattered tokens of 8 heads of 128: 6.8 us).
template <int D>
__global__ __launch_bounds__(256) void paged_append_q8_kernel(const uint16_t* __restrict__ k, int64_t k_t, int64_t k_h, const uint16_t* __restrict__ v,
                                                              int64_t v_t, int64_t v_h, const int32_t* __restrict__ slots, uint8_t* __restrict__ k_pages,
                                                              int64_t kp_p, int64_t kp_h, uint8_t* __restrict__ vt_pages, int64_t vp_p, int64_t vp_h,
                                                              PagedExps exps, int T, int log_p, int n_slots, int Hkv) {
    constexpr int CPR = D / 8;
    const int64_t u = (int64_t)blockIdx.x * 256 + threadIdx.x;
    const int c = (int)(u % CPR), h = (int)(u / CPR % Hkv);
    const int64_t t = u / CPR / Hkv;
    if (t >= T) return;                                            // whole rows of lanes
    float kx[8], vx[8];
    floats_of(*reinterpret_cast<const uint4*>(k + t * k_t + h * k_h + 8 * c), kx);
    floats_of(*reinterpret_cast<const uint4*>(v + t * v_t + h * v_h + 8 * c), vx);
    const int s = slots[t];
    const uint32_t ke = row_exponent(row_amax<CPR>(kx)), ve = row_exponent(row_amax<CPR>(vx));
    if (s < 0 || s >= n_slots) return;
    *reinterpret_cast<uint2*>(k_pages + place_of(s, log_p, kp_p, D) + h * kp_h + 8 * c) = quantise8(kx, ke);
    uint8_t* const at = vt_pages + place_of(s, log_p, vp_p, 1) + h * vp_h + ((int64_t)(8 * c) << log_p);
    const uint2 w = quantise8(vx, ve);
#pragma unroll
    for (int x = 0; x < 8; ++x) at[x << log_p] = (uint8_t)((x < 4 ? w.x : w.y) >> (8 * (x & 3)));
    if (c == 0) {
        exps.k[place_of(s, log_p, exps.k_p, 1) + h * exps.k_h] = (uint8_t)ke;
        exps.v[place_of(s, log_p, exps.v_p, 1) + h * exps.v_h] = (uint8_t)ve;
    }
}

struct ReadArgs {
    const void *k_pages, *vt_pages;
    PagedExps exps;
    const int32_t *table, *starts, *kv_lens;
    uint16_t *k, *v;
    int64_t table_stride, kp_p, kp_h, vp_p, vp_h, k_t, k_h, v_t, v_h;
    int B, Hkv, T, C, log_p, n_pages;
};
// A wavefront reads 64 positions (a tile) x 64 dims of a head, a lane 8 positions x 8 dims: K rows as they are, V^T pieces of 8 positions transposed
// in registers, both to whole 128-byte lines.  The tiles of the requests follow each other; every wavefront finds its own.  Bound by HBM: 98304 quantised
// tokens 121 us, 605 MB at 5.0 TB/s; 28000 tokens of bf16 pages of 16, head_dim 64, 30 us, 4.9 TB/s (a plain copy of 2 GiB: 4.9).
template <bool Q8>
__global__ __launch_bounds__(256) void paged_read_kernel(ReadArgs a, int dim_parts) {
    const int lane = threadIdx.x & 63;
    const uint32_t unit = blockIdx.x * 4 + __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const int D = 64 * dim_parts, part = (int)(unit % (uint32_t)dim_parts), h = (int)(unit / (uint32_t)dim_parts % (uint32_t)a.Hkv);
    const uint32_t want = unit / (uint32_t)dim_parts / (uint32_t)a.Hkv;

    // the request of the want-th tile: rows end - n .. end - 1 are positions kv - n .. kv - 1, of tiles floor((kv - n) / 64) .. floor((kv - 1) / 64)
    uint32_t before = 0;
    int b = -1, end = 0, n = 0, kv = 0, tile = 0;
    for (int b0 = 0; b0 < a.B; b0 += 64) {
        const int mine = b0 + lane;
        int last = 0, rows = 0, have = 0, tiles = 0;
        if (mine < a.B) {
            const int start = clamp_int(a.starts[mine], 0, a.T);
            last = clamp_int(a.starts[mine + 1], start, a.T);
            rows = last - start;
            have = clamp_int(a.kv_lens[mine], 0, a.C << a.log_p);
            tiles = rows > 0 ? ((have - 1) >> 6) - ((have - rows) >> 6) + 1 : 0;
        }
        uint32_t upto = (uint32_t)tiles;
#pragma unroll
        for (int x = 1; x < 64; x <<= 1) {
            const uint32_t v = __shfl_up(upto, x);
            if (lane >= x) upto += v;
        }
        upto += before;
        const uint64_t here = __ballot(want < upto && want >= upto - (uint32_t)tiles);
        if (here != 0) {
            const int at = __builtin_ctzll(here);
            auto pick = [&](int v) { return __builtin_amdgcn_readlane(v, at); };
            b = b0 + at;
            end = pick(last);
            n = pick(rows);
            kv = pick(have);
            tile = ((kv - n) >> 6) + (int)(want - (uint32_t)pick((int)(upto - (uint32_t)tiles)));
            break;
        }
        before = (uint32_t)__builtin_amdgcn_readlane((int)upto, 63);
    }
    if (b < 0) return;

    const int pos0 = 64 * tile + 8 * (lane >> 3), d0 = 64 * part + 8 * (lane & 7);      // of this lane's positions and dims
    if (pos0 + 7 < kv - n || pos0 >= kv) return;
    uint4 kr[8], vr[8];                                            // [position]
#pragma unroll
    for (int x = 0; x < 8; ++x) kr[x] = vr[x] = make_uint4(0, 0, 0, 0);
    if (pos0 >= 0) {                                               // 8 positions are on one side of 0, and in one page
        const int id = clamp_int(a.table[b * a.table_stride + (pos0 >> a.log_p)], 0, a.n_pages - 1), in_page = pos0 & ((1 << a.log_p) - 1);
        const int64_t kp = id * a.kp_p + h * a.kp_h + in_page * D + d0, vp = id * a.vp_p + h * a.vp_h + ((int64_t)d0 << a.log_p) + in_page;
        if constexpr (Q8) {
            uint2 kb[8], vd[8], vb[8];
#pragma unroll
            for (int x = 0; x < 8; ++x) {
                kb[x] = *reinterpret_cast<const uint2*>((const uint8_t*)a.k_pages + kp + x * D);
                vd[x] = *reinterpret_cast<const uint2*>((const uint8_t*)a.vt_pages + vp + (x << a.log_p));
            }
            const uint2 ke = *reinterpret_cast<const uint2*>(a.exps.k + id * a.exps.k_p + h * a.exps.k_h + in_page);
            const uint2 ve = *reinterpret_cast<const uint2*>(a.exps.v + id * a.exps.v_p + h * a.exps.v_h + in_page);
            transpose8(vd, vb);
#pragma unroll
            for (int x = 0; x < 8; ++x) {
                const float ks = two_to((x < 4 ? ke.x : ke.y) >> (8 * (x & 3)) & 0xffu), vs = two_to((x < 4 ? ve.x : ve.y) >> (8 * (x & 3)) & 0xffu);
                kr[x] = make_uint4(to_bf16_pair<false>(kb[x].x, ks), to_bf16_pair<true>(kb[x].x, ks), to_bf16_pair<false>(kb[x].y, ks), to_bf16_pair<true>(kb[x].y, ks));
                vr[x] = make_uint4(to_bf16_pair<false>(vb[x].x, vs), to_bf16_pair<true>(vb[x].x, vs), to_bf16_pair<false>(vb[x].y, vs), to_bf16_pair<true>(vb[x].y, vs));
            }
        } else {
            uint4 vd[8];                                           // [dim]
#pragma unroll
            for (int x = 0; x < 8; ++x) {
                kr[x] = *reinterpret_cast<const uint4*>((const uint16_t*)a.k_pages + kp + x * D);
                vd[x] = *reinterpret_cast<const uint4*>((const uint16_t*)a.vt_pages + vp + (x << a.log_p));
            }
#pragma unroll
            for (int p = 0; p < 4; ++p) {                          // positions 2p and 2p + 1
                uint32_t in[8];
#pragma unroll
                for (int x = 0; x < 8; ++x) in[x] = p == 0 ? vd[x].x : p == 1 ? vd[x].y : p == 2 ? vd[x].z : vd[x].w;
                uint32_t lo[4], hi[4];
#pragma unroll
                for (int x = 0; x < 4; ++x) {
                    lo[x] = __builtin_amdgcn_perm(in[2 * x + 1], in[2 * x], 0x05040100u);
                    hi[x] = __builtin_amdgcn_perm(in[2 * x + 1], in[2 * x], 0x07060302u);
                }
                vr[2 * p] = make_uint4(lo[0], lo[1], lo[2], lo[3]);
                vr[2 * p + 1] = make_uint4(hi[0], hi[1], hi[2], hi[3]);
            }
        }
    }
#pragma unroll
    for (int x = 0; x < 8; ++x) {
        const int pos = pos0 + x;
        if (pos < kv - n || pos >= kv) continue;
        const int64_t t = end - kv + pos;
        *reinterpret_cast<uint4*>(a.k + t * a.k_t + h * a.k_h + d0) = kr[x];
        *reinterpret_cast<uint4*>(a.v + t * a.v_t + h * a.v_h + d0) = vr[x];
    }
}

// Many tokens: a wavefront moves 32 tokens x 128 dims (with head_dim 64, of two heads), a lane 8 tokens (a window) x 8 dims.  Where 8 tokens that follow
// each other fill an aligned 8-byte piece of a page's V rows (those of a prompt do, wherever its chunk starts), the lanes that have the first of
// them in their window load all 8, quantise and transpose them in registers and store the pieces whole; the others are stored value by value.  Bound by HBM: 16384 tokens of 8
// prompts, 121 MB, 30 us, 4.0 TB/s (value by value: 183 us).
template <int D>
__global__ __launch_bounds__(256) void paged_append_q8_runs_kernel(const uint16_t* __restrict__ k, int64_t k_t, int64_t k_h, const uint16_t* __restrict__ v,
                                                                   int64_t v_t, int64_t v_h, const int32_t* __restrict__ slots,
                                                                   uint8_t* __restrict__ k_pages, int64_t kp_p, int64_t kp_h,
                                                                   uint8_t* __restrict__ vt_pages, int64_t vp_p, int64_t vp_h, PagedExps exps, int T,
                                                                   int log_p, int n_slots, int Hkv, int64_t n_units) {
    constexpr int CPR = D / 8, HW = 128 / D;                          // lanes of a row, heads of a wavefront
    const int lane = threadIdx.x & 63;
    // XCDs (workgroups go round them) take consecutive tokens, so that a V row's cache line is written whole by one L2
    const unsigned per = gridDim.x / 8;
    const int64_t unit = ((int64_t)(blockIdx.x % 8) * per + blockIdx.x / 8) * 4 + (threadIdx.x >> 6);
    if (unit >= n_units) return;
    const int heads = (Hkv + HW - 1) / HW;
    const int c = 8 * (lane % CPR), group = lane / CPR;               // first of the lane's 8 dims; windows 0 .. 3 of a head each
    const int wanted = (int)(unit % heads) * HW + group / 4, h = min(wanted, Hkv - 1), t0 = (int)(unit / heads) * 32;
    const bool real = wanted < Hkv;
    const int window = 8 * (group % 4);

    auto slot_at = [&](int t) {
        const int s = t >= 0 && t < T ? slots[t] : -1;
        return s >= 0 && s < n_slots ? s : -1;
    };
    const int near = slot_at(t0 - 8 + lane);                          // tokens t0 - 8 .. t0 + 55
    auto slot_of = [&](int i) { return __shfl(near, i + 8); };        // of token t0 + i, -8 <= i < 56
    // bit i: 8 tokens from token t0 - 8 + i on make a whole piece; i < 40 matter
    bool whole = near >= 0 && (near & 7) == 0 && lane < 40;
#pragma unroll
    for (int x = 1; x < 8; ++x) whole &= __shfl(near, (lane + x) & 63) == near + x;
    const uint64_t before = __ballot(whole);
    const uint32_t starts = (uint32_t)(before >> 8);                  // of tokens t0 .. t0 + 31
    uint64_t covered = 0;
#pragma unroll
    for (int x = 0; x < 8; ++x) covered |= before << x;               // bit i + 8: token t0 + i lies in a piece

    const int mine = (int)(starts >> window) & 0xff;                  // pieces are disjoint, so at most one starts in a window
    const int first = window + (mine != 0 ? __builtin_ctz(mine) : 0);
    const uint16_t* const vh = v + h * v_h + c;
    const uint16_t* const kh = k + h * k_h + c;
    uint4 kr[8], vr[8];
#pragma unroll
    for (int x = 0; x < 8; ++x) {
        kr[x] = stream_load16(kh + (int64_t)min(t0 + window + x, T - 1) * k_t);
        vr[x] = stream_load16(vh + (int64_t)min(t0 + first + x, T - 1) * v_t);
    }
    auto quantise = [&](const uint4& r, uint32_t& e) {
        float x[8];
        floats_of(r, x);
        e = row_exponent(row_amax<CPR>(x));
        return quantise8(x, e);
    };
#pragma unroll
    for (int x = 0; x < 8; ++x) {
        uint32_t e;
        const uint2 w = quantise(kr[x], e);
        const int s = slot_of(window + x);
        if (s >= 0 && real) {
            *reinterpret_cast<uint2*>(k_pages + place_of(s, log_p, kp_p, D) + h * kp_h + c) = w;
            if (c == 0) exps.k[place_of(s, log_p, exps.k_p, 1) + h * exps.k_h] = (uint8_t)e;
        }
    }
    uint8_t* const vth = vt_pages + h * vp_h + ((int64_t)c << log_p);
    auto store_one = [&](int s, const uint2& w, uint32_t e) {
        uint8_t* const at = vth + place_of(s, log_p, vp_p, 1);
#pragma unroll
        for (int y = 0; y < 8; ++y) at[y << log_p] = (uint8_t)((y < 4 ? w.x : w.y) >> (8 * (y & 3)));
        if (c == 0) exps.v[place_of(s, log_p, exps.v_p, 1) + h * exps.v_h] = (uint8_t)e;
    };
    uint2 vb[8];
    uint32_t ve[8];
#pragma unroll
    for (int x = 0; x < 8; ++x) vb[x] = quantise(vr[x], ve[x]);
    const int s0 = slot_of(first);                                    // before the branch: every lane's slots are asked for
    if (mine != 0) {
        uint2 piece[8];
        transpose8(vb, piece);
        if (real) {
            uint8_t* const at = vth + place_of(s0, log_p, vp_p, 1);
#pragma unroll
            for (int y = 0; y < 8; ++y) *reinterpret_cast<uint2*>(at + (y << log_p)) = piece[y];
            if (c == 0)
                *reinterpret_cast<uint2*>(exps.v + place_of(s0, log_p, exps.v_p, 1) + h * exps.v_h) =
                    make_uint2(ve[0] | ve[1] << 8 | ve[2] << 16 | ve[3] << 24, ve[4] | ve[5] << 8 | ve[6] << 16 | ve[7] << 24);
        }
    }
    // tokens of the window that no piece has: those before its piece, or any of them
#pragma unroll
    for (int x = 0; x < 8; ++x) {
        const int s = slot_of(window + x);
        const bool single = s >= 0 && !(covered >> (window + x + 8) & 1);
        if (mine == 0) {
            if (single && real) store_one(s, vb[x], ve[x]);
        } else if (single) {                                          // the same in all lanes of a row
            uint32_t e;
            const uint2 w = quantise(*reinterpret_cast<const uint4*>(vh + (int64_t)(t0 + window + x) * v_t), e);
            if (real) store_one(s, w, e);
        }
    }
}

// Tokens up to which paged_append_q8_kernel moves them, the other kernel more: 1024 single tokens 15.0 us with the one, 1025 21.1 with the other, of a prompt
// 8.6 and 8.5.
constexpr int kFewAppended = 1024;
template <int D>
hipError_t launch_append(const PagedDims& d, const void* k, int64_t k_t, int64_t k_h, const void* v, int64_t v_t, int64_t v_h,
                         const int32_t* slots, void* k_pages, void* vt_pages, const PagedExps& exps, hipStream_t st) {
    if (d.T > kFewAppended) {
        const int64_t units = ((int64_t)d.T + 31) / 32 * ((d.Hkv + 128 / D - 1) / (128 / D));
        const int64_t nwg = (units + 31) / 32 * 8;       // the same number for each of the 8 XCDs
        if (nwg > 0x7fffffffll) return hipErrorInvalidValue;
        hipLaunchKernelGGL((paged_append_q8_runs_kernel<D>), dim3((unsigned)nwg), dim3(256), 0, st, (const uint16_t*)k, k_t, k_h, (const uint16_t*)v, v_t,
                           v_h, slots, (uint8_t*)k_pages, d.kp_p, d.kp_h, (uint8_t*)vt_pages, d.vp_p, d.vp_h, exps, d.T, d.log_p, d.n_pages << d.log_p,
                           d.Hkv, units);
        return hipGetLastError();
    }
    const int64_t nwg = ((int64_t)d.T * d.Hkv * (D / 8) + 255) / 256;
    if (nwg > 0x7fffffffll) return hipErrorInvalidValue;
    hipLaunchKernelGGL((paged_append_q8_kernel<D>), dim3((unsigned)nwg), dim3(256), 0, st, (const uint16_t*)k, k_t, k_h, (const uint16_t*)v, v_t, v_h, slots,
                       (uint8_t*)k_pages, d.kp_p, d.kp_h, (uint8_t*)vt_pages, d.vp_p, d.vp_h, exps, d.T, d.log_p, d.n_pages << d.log_p, d.Hkv);
    return hipGetLastError();
}

}  // namespace

hipError_t launch_paged_append_q8(const PagedDims& d, const void* k, int64_t k_t, int64_t k_h, const void* v, int64_t v_t, int64_t v_h,
                                  const int32_t* slots, void* k_pages, void* vt_pages, const PagedExps& exps, hipStream_t st) {
    return d.D == 128 ? launch_append<128>(d, k, k_t, k_h, v, v_t, v_h, slots, k_pages, vt_pages, exps, st)
                      : launch_append<64>(d, k, k_t, k_h, v, v_t, v_h, slots, k_pages, vt_pages, exps, st);
}

hipError_t launch_paged_read(const PagedDims& d, const void* k_pages, const void* vt_pages, const PagedExps& exps, const int32_t* block_table,
                             const int32_t* starts, const int32_t* kv_lens, void* k, int64_t k_t, int64_t k_h, void* v, int64_t v_t, int64_t v_h,
                             hipStream_t st) {
    const int64_t tiles = (int64_t)d.T / 64 + 2 * (int64_t)(d.B < d.T ? d.B : d.T);          // a request's rows may start and end inside one
    const int64_t nwg = (tiles * d.Hkv * (d.D / 64) + 3) / 4;
    if (nwg > (1 << 30) / 4) return hipErrorInvalidValue;
    const ReadArgs a{k_pages, vt_pages, exps, block_table, starts, kv_lens, (uint16_t*)k, (uint16_t*)v, d.table_stride, d.kp_p, d.kp_h, d.vp_p, d.vp_h,
                     k_t, k_h, v_t, v_h, d.B, d.Hkv, d.T, d.C, d.log_p, d.n_pages};
    if (exps.k != nullptr) hipLaunchKernelGGL((paged_read_kernel<true>), dim3((unsigned)nwg), dim3(256), 0, st, a, d.D / 64);
    else hipLaunchKernelGGL((paged_read_kernel<false>), dim3((unsigned)nwg), dim3(256), 0, st, a, d.D / 64);
    return hipGetLastError();
}

}  // namespace spa
