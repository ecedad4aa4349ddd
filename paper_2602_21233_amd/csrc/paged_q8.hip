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

// A thread quantises 8 dims of a token's key and value; D / 8 lanes share their row's maximum.
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
// A thread reads 8 dims of a row's key and value.
template <int D, bool Q8>
__global__ __launch_bounds__(256) void paged_read_kernel(ReadArgs a) {
    constexpr int CPR = D / 8;
    const int64_t u = (int64_t)blockIdx.x * 256 + threadIdx.x;
    const int c = (int)(u % CPR), h = (int)(u / CPR % a.Hkv);
    const int64_t t = u / CPR / a.Hkv;
    if (t >= a.T) return;
    int lo = 0, hi = a.B;                          // the last request that starts at or before t
    while (hi - lo > 1) {
        const int mid = (lo + hi) >> 1;
        if (a.starts[mid] <= t) lo = mid;
        else hi = mid;
    }
    const int first = a.starts[lo], end = a.starts[lo + 1];
    if (t < first || t >= end) return;
    const int64_t pos = (int64_t)clamp_int(a.kv_lens[lo], 0, a.C << a.log_p) - end + t;
    uint4 kr = make_uint4(0, 0, 0, 0), vr = kr;
    if (pos >= 0) {
        const int id = clamp_int(a.table[lo * a.table_stride + (pos >> a.log_p)], 0, a.n_pages - 1);
        const int in_page = (int)pos & ((1 << a.log_p) - 1);
        const int64_t kp = id * a.kp_p + h * a.kp_h + in_page * D + 8 * c, vp = id * a.vp_p + h * a.vp_h + ((8 * c) << a.log_p) + in_page;
        uint32_t kw[4], vw[4];
        if constexpr (Q8) {
            const float ks = two_to(a.exps.k[id * a.exps.k_p + h * a.exps.k_h + in_page]), vs = two_to(a.exps.v[id * a.exps.v_p + h * a.exps.v_h + in_page]);
            const uint2 kb = *reinterpret_cast<const uint2*>((const uint8_t*)a.k_pages + kp);
            uint32_t vb[2] = {0, 0};
#pragma unroll
            for (int x = 0; x < 8; ++x) vb[x >> 2] |= (uint32_t)((const uint8_t*)a.vt_pages)[vp + (x << a.log_p)] << (8 * (x & 3));
            kw[0] = to_bf16_pair<false>(kb.x, ks); kw[1] = to_bf16_pair<true>(kb.x, ks);
            kw[2] = to_bf16_pair<false>(kb.y, ks); kw[3] = to_bf16_pair<true>(kb.y, ks);
            vw[0] = to_bf16_pair<false>(vb[0], vs); vw[1] = to_bf16_pair<true>(vb[0], vs);
            vw[2] = to_bf16_pair<false>(vb[1], vs); vw[3] = to_bf16_pair<true>(vb[1], vs);
        } else {
            const uint4 r = *reinterpret_cast<const uint4*>((const uint16_t*)a.k_pages + kp);
            kw[0] = r.x; kw[1] = r.y; kw[2] = r.z; kw[3] = r.w;
#pragma unroll
            for (int x = 0; x < 4; ++x)
                vw[x] = (uint32_t)((const uint16_t*)a.vt_pages)[vp + ((2 * x) << a.log_p)] | (uint32_t)((const uint16_t*)a.vt_pages)[vp + ((2 * x + 1) << a.log_p)] << 16;
        }
        kr = make_uint4(kw[0], kw[1], kw[2], kw[3]);
        vr = make_uint4(vw[0], vw[1], vw[2], vw[3]);
    }
    *reinterpret_cast<uint4*>(a.k + t * a.k_t + h * a.k_h + 8 * c) = kr;
    *reinterpret_cast<uint4*>(a.v + t * a.v_t + h * a.v_h + 8 * c) = vr;
}

template <int D>
hipError_t launch_append(const PagedDims& d, const void* k, int64_t k_t, int64_t k_h, const void* v, int64_t v_t, int64_t v_h,
                         const int32_t* slots, void* k_pages, void* vt_pages, const PagedExps& exps, hipStream_t st) {
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
    const int64_t nwg = ((int64_t)d.T * d.Hkv * (d.D / 8) + 255) / 256;
    if (nwg > 0x7fffffffll) return hipErrorInvalidValue;
    const ReadArgs a{k_pages, vt_pages, exps, block_table, starts, kv_lens, (uint16_t*)k, (uint16_t*)v, d.table_stride, d.kp_p, d.kp_h, d.vp_p, d.vp_h,
                     k_t, k_h, v_t, v_h, d.B, d.Hkv, d.T, d.C, d.log_p, d.n_pages};
    const auto go = [&](auto kernel) { hipLaunchKernelGGL(kernel, dim3((unsigned)nwg), dim3(256), 0, st, a); };
    if (exps.k != nullptr) d.D == 128 ? go(paged_read_kernel<128, true>) : go(paged_read_kernel<64, true>);
    else d.D == 128 ? go(paged_read_kernel<128, false>) : go(paged_read_kernel<64, false>);
    return hipGetLastError();
}

}  // namespace spa
