// The paged KV cache's own kernels: block tables and slot maps of a step, and the new tokens' keys and values into their
// pages.
#include "paged.hpp"

namespace spa {
namespace {

constexpr uint32_t kMany = 0x7fffffffu;
// Sums of lengths stop at 2^31 - 1: an absurd length makes its request (and those behind it) be left out, not wrap around.
// min(a + b, limit) is associative for non-negative values, so a scan may use it.
__device__ __forceinline__ uint32_t add_capped(uint32_t a, uint32_t b) { return min(a + b, kMany); }

// inclusive scan over the lanes of a wavefront
__device__ __forceinline__ uint32_t scan_capped(uint32_t v) {
    v = add_capped(v, __builtin_amdgcn_update_dpp(0, (int)v, 0x111, 0xF, 0xF, true));   // row_shr:1, lanes shifted out read 0
    v = add_capped(v, __builtin_amdgcn_update_dpp(0, (int)v, 0x112, 0xF, 0xF, true));   // row_shr:2
    v = add_capped(v, __builtin_amdgcn_update_dpp(0, (int)v, 0x114, 0xF, 0xF, true));   // row_shr:4
    v = add_capped(v, __builtin_amdgcn_update_dpp(0, (int)v, 0x118, 0xF, 0xF, true));   // row_shr:8
    v = add_capped(v, __builtin_amdgcn_update_dpp(0, (int)v, 0x142, 0xA, 0xF, true));   // row_bcast15 into rows 1 and 3
    v = add_capped(v, __builtin_amdgcn_update_dpp(0, (int)v, 0x143, 0xC, 0xF, true));   // row_bcast31 into rows 2 and 3
    return v;
}

// Every workgroup scans the requests for itself (at most 4096 pairs of lengths, out of the L2) and then serves the
// tokens of its own: one launch, nothing handed from one workgroup to another.  A page that the step takes starts at one of
// its new tokens, so the token at a page's start also writes the table entry.  Bound by latency at every size that occurs.
constexpr int kPlanThreads = 256;
constexpr int kPlanTokens = 4 * kPlanThreads;      // tokens of a workgroup
__global__ __launch_bounds__(kPlanThreads) void paged_plan_kernel(
    const int32_t* __restrict__ ctx_lens, const int32_t* __restrict__ new_lens, const int32_t* __restrict__ free_pages, int n_free,
    const int32_t* __restrict__ free_range, int32_t* __restrict__ table, int64_t table_stride, int32_t* __restrict__ q_starts,
    int32_t* __restrict__ kv_lens, int32_t* __restrict__ slots, int32_t* __restrict__ positions, int32_t* __restrict__ taken, int B, int C,
    int T, int log_p, int n_pages) {
    __shared__ int32_t s_start[kMaxRequests + 1];
    __shared__ int32_t s_before[kMaxRequests];     // pages taken by the requests before; -1: left out
    __shared__ uint32_t s_sum[2][2][kPlanThreads / 64];
    __shared__ int32_t s_taken, s_left_out;

    const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6;
    const bool first_wg = blockIdx.x == 0;
    const int page = 1 << log_p;
    const int first = clamp_int(free_range[0], 0, n_free);
    const int room = clamp_int(free_range[1], first, n_free) - first;
    if (tid == 0) { s_taken = 0; s_left_out = 0; }
    __syncthreads();

    uint32_t tokens_before = 0, pages_before = 0;
    for (int b0 = 0, turn = 0; b0 < B; b0 += kPlanThreads, turn ^= 1) {
        const int b = b0 + tid;
        const int ctx = b < B ? ctx_lens[b] : 0, more = b < B ? new_lens[b] : 0;
        const uint32_t tokens = more > 0 ? (uint32_t)more : 0u;
        // starts first: whether a request fits the packed tokens decides whether it needs pages
        const uint32_t token_scan = scan_capped(tokens);
        if (lane == 63) s_sum[turn][0][wave] = token_scan;
        __syncthreads();
        const uint32_t lane_before = __shfl_up(token_scan, 1);
        uint32_t start = tokens_before;
        for (int w = 0; w < wave; ++w) start = add_capped(start, s_sum[turn][0][w]);
        const uint32_t end = add_capped(start, token_scan);
        start = add_capped(start, lane > 0 ? lane_before : 0u);
        for (int w = 0; w < kPlanThreads / 64; ++w) tokens_before = add_capped(tokens_before, s_sum[turn][0][w]);

        const bool sound = b < B && ctx >= 0 && more >= 0 && (int64_t)ctx + more <= (int64_t)C * page && end <= (uint32_t)T;
        const uint32_t need = sound ? (uint32_t)(((int64_t)ctx + more + page - 1) >> log_p) - (uint32_t)(((int64_t)ctx + page - 1) >> log_p) : 0u;
        const uint32_t need_scan = scan_capped(need);
        if (lane == 63) s_sum[turn][1][wave] = need_scan;
        __syncthreads();
        uint32_t upto = add_capped(pages_before, need_scan);
        for (int w = 0; w < wave; ++w) upto = add_capped(upto, s_sum[turn][1][w]);
        for (int w = 0; w < kPlanThreads / 64; ++w) pages_before = add_capped(pages_before, s_sum[turn][1][w]);
        const bool goes = sound && (need == 0 || upto <= (uint32_t)room);
        if (b < B) {
            s_start[b] = (int)min(start, (uint32_t)T);
            s_before[b] = goes ? (int)(upto - need) : -1;
            if (b == B - 1) s_start[B] = (int)min(end, (uint32_t)T);
            if (first_wg) {
                q_starts[b] = (int)min(start, (uint32_t)T);
                if (b == B - 1) q_starts[B] = (int)min(end, (uint32_t)T);
                kv_lens[b] = goes ? ctx + more : 0;
                if (goes && need) atomicMax(&s_taken, (int)upto);
                if (!goes) atomicAdd(&s_left_out, 1);
            }
        }
    }
    __syncthreads();
    if (first_wg && tid == 0) {
        taken[0] = s_taken;
        taken[1] = s_left_out;
    }

    for (int t = blockIdx.x * kPlanTokens + tid; t < min(T, (int)(blockIdx.x + 1) * kPlanTokens); t += kPlanThreads) {
        int slot = -1, pos = 0;
        if (t < s_start[B]) {
            int lo = 0, hi = B;                    // the last request that starts at or before t: s_start[lo] <= t < s_start[hi]
            while (hi - lo > 1) {
                const int mid = (lo + hi) >> 1;
                if (s_start[mid] <= t) lo = mid;
                else hi = mid;
            }
            const int ctx = ctx_lens[lo], before = s_before[lo];
            pos = (int)((uint32_t)ctx + (uint32_t)(t - s_start[lo]));
            if (before >= 0) {
                const int col = pos >> log_p, have = (ctx + page - 1) >> log_p;
                int id;
                if (col < have) {
                    id = table[(int64_t)lo * table_stride + col];
                } else {
                    id = free_pages[first + before + (col - have)];      // before + need <= room
                    if ((pos & (page - 1)) == 0) table[(int64_t)lo * table_stride + col] = id;
                }
                if (id >= 0 && id < n_pages) slot = (id << log_p) + (pos & (page - 1));
            }
        }
        slots[t] = slot;
        if (positions != nullptr) positions[t] = pos;
    }
}

// K and V of TT tokens of one head into their pages.  K rows are copied in 16-byte pieces.  V goes through LDS: where 8 tokens
// that follow each other fill an aligned 16-byte piece of a page's rows (a prompt's tokens do, wherever its chunk starts), the
// piece is stored whole, other tokens value by value.  HBM-bound: every value is read and written once.
template <int D, int TT>
__global__ __launch_bounds__(256) void paged_append_kernel(const uint16_t* __restrict__ k, int64_t k_t, int64_t k_h, const uint16_t* __restrict__ v,
                                                           int64_t v_t, int64_t v_h, const int32_t* __restrict__ slots, uint16_t* __restrict__ k_pages,
                                                           int64_t kp_p, int64_t kp_h, uint16_t* __restrict__ vt_pages, int64_t vp_p, int64_t vp_h,
                                                           int T, int log_p, int n_slots, int Hkv) {
    constexpr int CPR = D / 8;                     // 16-byte pieces of a row
    constexpr int PAD = D + 8;
    __shared__ __attribute__((aligned(16))) uint16_t s_v[TT][PAD];
    __shared__ int32_t s_slot[TT];
    __shared__ int32_t s_run[TT / 8 + 1], s_one[TT];   // first tokens of whole pieces; tokens stored one by one
    __shared__ int32_t s_runs, s_ones;

    const int tid = threadIdx.x;
    const int h = blockIdx.x % Hkv, t0 = blockIdx.x / Hkv * TT;
    const int n = min(TT, T - t0), page = 1 << log_p;
    if (tid < TT) {
        const int s = tid < n ? slots[t0 + tid] : -1;
        s_slot[tid] = s >= 0 && s < n_slots ? s : -1;
    }
    if (tid == 0) { s_runs = 0; s_ones = 0; }
    // the loads need no slot
    constexpr int PT = TT * CPR / 256 > 0 ? TT * CPR / 256 : 1;   // pieces of a thread
    uint4 kr[PT], vr[PT];
#pragma unroll
    for (int x = 0; x < PT; ++x) {
        const int u = tid + 256 * x, row = u / CPR, c = u % CPR;
        if (row < n) {
            kr[x] = *reinterpret_cast<const uint4*>(k + (t0 + row) * k_t + h * k_h + 8 * c);
            vr[x] = *reinterpret_cast<const uint4*>(v + (t0 + row) * v_t + h * v_h + 8 * c);
        }
    }
    __syncthreads();
    if (tid < TT && s_slot[tid] >= 0) {
        const int lead = tid - (s_slot[tid] & 7);  // the token that would start this one's piece
        bool whole = lead >= 0 && lead + 7 < n;
        if (whole) {
            const int s = s_slot[tid] & ~7;
#pragma unroll
            for (int x = 0; x < 8; ++x) whole &= s_slot[lead + x] == s + x;
        }
        if (whole && lead == tid) s_run[atomicAdd(&s_runs, 1)] = tid;
        if (!whole) s_one[atomicAdd(&s_ones, 1)] = tid;
    }
#pragma unroll
    for (int x = 0; x < PT; ++x) {
        const int u = tid + 256 * x, row = u / CPR, c = u % CPR;
        if (row < n) {
            *reinterpret_cast<uint4*>(&s_v[row][8 * c]) = vr[x];
            const int s = s_slot[row];
            if (s >= 0) *reinterpret_cast<uint4*>(k_pages + (s >> log_p) * kp_p + h * kp_h + (s & (page - 1)) * D + 8 * c) = kr[x];
        }
    }
    __syncthreads();
    const int runs = s_runs, ones = s_ones;
    for (int u = tid; u < runs * D; u += 256) {
        const int d = u / runs, i = s_run[u % runs], s = s_slot[i];
        uint16_t w[8];
#pragma unroll
        for (int x = 0; x < 8; ++x) w[x] = s_v[i + x][d];
        *reinterpret_cast<uint4*>(vt_pages + (s >> log_p) * vp_p + h * vp_h + (int64_t)d * page + (s & (page - 1))) = *reinterpret_cast<const uint4*>(w);
    }
    for (int u = tid; u < ones * D; u += 256) {
        const int d = u / ones, i = s_one[u % ones], s = s_slot[i];
        vt_pages[(s >> log_p) * vp_p + h * vp_h + (int64_t)d * page + (s & (page - 1))] = s_v[i][d];
    }
}

template <int D, int TT>
hipError_t launch_append(const PagedDims& d, const void* k, int64_t k_t, int64_t k_h, const void* v, int64_t v_t, int64_t v_h,
                         const int32_t* slots, void* k_pages, void* vt_pages, hipStream_t st) {
    const int64_t nwg = (int64_t)((d.T + TT - 1) / TT) * d.Hkv;
    if (nwg > 0x7fffffffll) return hipErrorInvalidValue;
    hipLaunchKernelGGL((paged_append_kernel<D, TT>), dim3((unsigned)nwg), dim3(256), 0, st, (const uint16_t*)k, k_t, k_h, (const uint16_t*)v,
                       v_t, v_h, slots, (uint16_t*)k_pages, d.kp_p, d.kp_h, (uint16_t*)vt_pages, d.vp_p, d.vp_h, d.T, d.log_p,
                       d.n_pages << d.log_p, d.Hkv);
    return hipGetLastError();
}

}  // namespace

hipError_t launch_paged_plan(const PagedDims& d, const int32_t* ctx_lens, const int32_t* new_lens, const int32_t* free_pages, int n_free,
                             const int32_t* free_range, int32_t* block_table, int32_t* q_starts, int32_t* kv_lens, int32_t* slots,
                             int32_t* positions_or_null, int32_t* taken, hipStream_t st) {
    const unsigned nwg = (unsigned)(((int64_t)d.T + kPlanTokens - 1) / kPlanTokens);
    hipLaunchKernelGGL(paged_plan_kernel, dim3(nwg), dim3(kPlanThreads), 0, st, ctx_lens, new_lens, free_pages, n_free, free_range,
                       block_table, d.table_stride, q_starts, kv_lens, slots, positions_or_null, taken, d.B, d.C, d.T, d.log_p, d.n_pages);
    return hipGetLastError();
}

hipError_t launch_paged_append(const PagedDims& d, const void* k, int64_t k_t, int64_t k_h, const void* v, int64_t v_t, int64_t v_h,
                               const int32_t* slots, void* k_pages, void* vt_pages, hipStream_t st) {
    return d.D == 128 ? launch_append<128, 64>(d, k, k_t, k_h, v, v_t, v_h, slots, k_pages, vt_pages, st)
                      : launch_append<64, 64>(d, k, k_t, k_h, v, v_t, v_h, slots, k_pages, vt_pages, st);
}

}  // namespace spa
