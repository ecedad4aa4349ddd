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
// its new tokens, so the token at a page's start also writes the table entry.  Bound by latency at every size that occurs: 64 requests of one token 3.0 us, 512
// requests of 103000 tokens 8.2 (two turns of two scans that wait for each other, then nine steps of search a token).
constexpr int kPlanThreads = 256;
// Tokens up to which paged_append_kernel moves them, the other kernel more.  8 heads of 128, us with the one / the other: 512 scattered tokens
// 7.6 / 15.5, 512 of a prompt 6.4 / 7.0; 1024 14.1 / 17.9 and 9.6 / 7.1; 2048 27.3 / 30.3 and 15.4 / 7.5.
constexpr int kFewAppended = 1024;
__global__ __launch_bounds__(kPlanThreads) void paged_plan_kernel(
    const int32_t* __restrict__ ctx_lens, const int32_t* __restrict__ new_lens, const int32_t* __restrict__ free_pages, int n_free,
    const int32_t* __restrict__ free_range, int32_t* __restrict__ table, int64_t table_stride, int32_t* __restrict__ q_starts,
    int32_t* __restrict__ kv_lens, int32_t* __restrict__ slots, int32_t* __restrict__ positions, int32_t* __restrict__ taken, int B, int C,
    int T, int log_p, int n_pages) {
    extern __shared__ int32_t s_requests[];        // 3 B + 1
    int32_t* const s_start = s_requests;
    int32_t* const s_before = s_start + B + 1;     // pages taken by the requests before; -1: left out
    int32_t* const s_ctx = s_before + B;
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
            s_ctx[b] = ctx;
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

    for (int t = blockIdx.x * kPlanThreads + tid; t < T; t += gridDim.x * kPlanThreads) {
        int slot = -1, pos = 0;
        if (t < s_start[B]) {
            int lo = 0, hi = B;                    // the last request that starts at or before t: s_start[lo] <= t < s_start[hi]
            while (hi - lo > 1) {
                const int mid = (lo + hi) >> 1;
                if (s_start[mid] <= t) lo = mid;
                else hi = mid;
            }
            const int ctx = s_ctx[lo], before = s_before[lo];
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

__device__ __forceinline__ int64_t place_of(int slot, int log_p, int64_t page_stride, int in_page) {
    return (slot >> log_p) * page_stride + (int64_t)(slot & ((1 << log_p) - 1)) * in_page;
}

// Few tokens: a thread moves 8 dims of one token, V in single values.  Bound by latency (256 scattered tokens, 8 heads of 128: 5.9 us).
template <int D>
__global__ __launch_bounds__(256) void paged_append_kernel(const uint16_t* __restrict__ k, int64_t k_t, int64_t k_h, const uint16_t* __restrict__ v,
                                                           int64_t v_t, int64_t v_h, const int32_t* __restrict__ slots, uint16_t* __restrict__ k_pages,
                                                           int64_t kp_p, int64_t kp_h, uint16_t* __restrict__ vt_pages, int64_t vp_p, int64_t vp_h,
                                                           int T, int log_p, int n_slots, int Hkv) {
    constexpr int CPR = D / 8;
    const int64_t u = (int64_t)blockIdx.x * 256 + threadIdx.x;
    const int c = (int)(u % CPR), h = (int)(u / CPR % Hkv);
    const int64_t t = u / CPR / Hkv;
    if (t >= T) return;
    const uint4 kr = *reinterpret_cast<const uint4*>(k + t * k_t + h * k_h + 8 * c);
    const uint4 vr = *reinterpret_cast<const uint4*>(v + t * v_t + h * v_h + 8 * c);
    const int s = slots[t];
    if (s < 0 || s >= n_slots) return;
    *reinterpret_cast<uint4*>(k_pages + place_of(s, log_p, kp_p, D) + h * kp_h + 8 * c) = kr;
    uint16_t* const at = vt_pages + place_of(s, log_p, vp_p, 1) + h * vp_h + ((int64_t)(8 * c) << log_p);
    const uint32_t w[4] = {vr.x, vr.y, vr.z, vr.w};
#pragma unroll
    for (int x = 0; x < 8; ++x) at[x << log_p] = (uint16_t)(w[x >> 1] >> (16 * (x & 1)));
}

// Many tokens: a wavefront moves 64 tokens x 64 dims of a head, a lane 8 tokens (a window) x 8 dims.  Where 8 tokens that follow
// each other fill an aligned 16-byte piece of a page's V rows (those of a prompt do, wherever its chunk starts), the lane that has
// the first of them in its window loads all 8, transposes them in registers and stores the pieces whole; the tokens before the
// first piece of a prompt and behind its last one are stored value by value.  All loads of a lane are in flight at once.
// HBM-bound: every value is read and written once (16384 tokens of 8 prompts, 161 MB: 31 us, 5.1 TB/s; a plain copy of 2 GiB: 4.9).
template <int D>
__global__ __launch_bounds__(256) void paged_append_runs_kernel(const uint16_t* __restrict__ k, int64_t k_t, int64_t k_h, const uint16_t* __restrict__ v,
                                                                int64_t v_t, int64_t v_h, const int32_t* __restrict__ slots,
                                                                uint16_t* __restrict__ k_pages, int64_t kp_p, int64_t kp_h,
                                                                uint16_t* __restrict__ vt_pages, int64_t vp_p, int64_t vp_h, int T, int log_p, int n_slots,
                                                                int Hkv, int64_t n_units) {
    const int lane = threadIdx.x & 63;
    // XCDs (workgroups go round them) take consecutive tokens: a V row's cache line then is written whole by one L2, also where the
    // tokens of two wavefronts meet in it, and the inputs are not kept (16384 tokens 48.6 -> 31.7 us, 37.1 without this order)
    const unsigned per = gridDim.x / 8;
    const int64_t unit = ((int64_t)(blockIdx.x % 8) * per + blockIdx.x / 8) * 4 + (threadIdx.x >> 6);
    if (unit >= n_units) return;
    const int c = 8 * (lane & 7) + 64 * (int)(unit % (D / 64));      // first of the lane's 8 dims
    const int h = (int)(unit / (D / 64) % Hkv), t0 = (int)(unit / (D / 64) / Hkv) * 64;
    const int window = 8 * (lane >> 3);

    // The slots of tokens t0 - 8 .. t0 + 71: token t0 - 8 + lane in `early`, t0 + 56 + lane in `late`; -1 where there is none.
    auto slot_at = [&](int t) {
        const int s = t >= 0 && t < T ? slots[t] : -1;
        return s >= 0 && s < n_slots ? s : -1;
    };
    const int early = slot_at(t0 - 8 + lane), late = slot_at(t0 + 56 + lane);
    auto slot_of = [&](int i) {                                      // of token t0 + i, -8 <= i < 72
        const int x = __shfl(early, (i + 8) & 63), y = __shfl(late, (i - 56) & 63);
        return i < 56 ? x : y;
    };
    // bit i: 8 tokens from token t0 - 8 + i on (i < 64), or from t0 + i - 8 on for the last ones, make a whole piece
    bool whole = true, whole_end = true;
    const int head = early, tail = slot_of(56 + (lane & 7));
    whole &= head >= 0 && (head & 7) == 0;
    whole_end &= tail >= 0 && (tail & 7) == 0;
#pragma unroll
    for (int x = 1; x < 8; ++x) {
        whole &= slot_of(lane - 8 + x) == head + x;
        whole_end &= slot_of(56 + (lane & 7) + x) == tail + x;
    }
    const uint64_t before = __ballot(whole);                         // starts t0 - 8 .. t0 + 55
    const uint64_t last8 = __ballot(whole_end) & 0xff;               // starts t0 + 56 .. t0 + 63
    const uint64_t starts = (before >> 8) | (last8 << 56);           // starts t0 .. t0 + 63
    uint64_t covered = 0;
#pragma unroll
    for (int x = 0; x < 8; ++x) covered |= (starts << x) | ((before & 0xff) << x >> 8);

    const int mine = (int)(starts >> window) & 0xff;                 // pieces are disjoint, so at most one starts in a window
    const int first = window + (mine != 0 ? __builtin_ctz(mine) : 0);
    const uint16_t* const vh = v + h * v_h + c;
    const uint16_t* const kh = k + h * k_h + c;
    uint4 kr[8], vr[8];
#pragma unroll
    for (int x = 0; x < 8; ++x) {
        kr[x] = stream_load16(kh + (int64_t)min(t0 + window + x, T - 1) * k_t);
        vr[x] = stream_load16(vh + (int64_t)min(t0 + first + x, T - 1) * v_t);
    }
#pragma unroll
    for (int x = 0; x < 8; ++x) {
        const int s = slot_of(window + x);
        if (s >= 0) *reinterpret_cast<uint4*>(k_pages + place_of(s, log_p, kp_p, D) + h * kp_h + c) = kr[x];
    }
    const int s0 = slot_of(first);
    uint16_t* const vth = vt_pages + h * vp_h + ((int64_t)c << log_p);
    auto store_one = [&](int s, const uint4& r) {
        uint16_t* const at = vth + place_of(s, log_p, vp_p, 1);
        const uint32_t w[4] = {r.x, r.y, r.z, r.w};
#pragma unroll
        for (int y = 0; y < 8; ++y) at[y << log_p] = (uint16_t)(w[y >> 1] >> (16 * (y & 1)));
    };
    // -1 for tokens of a whole piece
    int single[8];
#pragma unroll
    for (int x = 0; x < 8; ++x) {
        const int s = slot_of(window + x);
        single[x] = (covered >> (window + x)) & 1 ? -1 : s;
    }
    if (mine != 0) {
        uint16_t* const at = vth + place_of(s0, log_p, vp_p, 1);
#pragma unroll
        for (int p = 0; p < 4; ++p) {                                // dims c + 2p and c + 2p + 1
            uint32_t in[8];
#pragma unroll
            for (int x = 0; x < 8; ++x) in[x] = p == 0 ? vr[x].x : p == 1 ? vr[x].y : p == 2 ? vr[x].z : vr[x].w;
            uint32_t lo[4], hi[4];
#pragma unroll
            for (int x = 0; x < 4; ++x) {
                lo[x] = __builtin_amdgcn_perm(in[2 * x + 1], in[2 * x], 0x05040100u);
                hi[x] = __builtin_amdgcn_perm(in[2 * x + 1], in[2 * x], 0x07060302u);
            }
            *reinterpret_cast<uint4*>(at + ((int64_t)(2 * p) << log_p)) = make_uint4(lo[0], lo[1], lo[2], lo[3]);
            *reinterpret_cast<uint4*>(at + ((int64_t)(2 * p + 1) << log_p)) = make_uint4(hi[0], hi[1], hi[2], hi[3]);
        }
        for (int x = 0; window + x < first; ++x) {                   // tokens of the window before its piece
            int s = -1;
#pragma unroll
            for (int y = 0; y < 8; ++y) s = y == x ? single[y] : s;
            if (s >= 0) store_one(s, *reinterpret_cast<const uint4*>(vh + (int64_t)(t0 + window + x) * v_t));
        }
    } else {
#pragma unroll
        for (int x = 0; x < 8; ++x)
            if (single[x] >= 0) store_one(single[x], vr[x]);
    }
}

template <int D>
hipError_t launch_append(const PagedDims& d, const void* k, int64_t k_t, int64_t k_h, const void* v, int64_t v_t, int64_t v_h,
                         const int32_t* slots, void* k_pages, void* vt_pages, hipStream_t st) {
    if (d.T <= kFewAppended) {
        const int64_t nwg = ((int64_t)d.T * d.Hkv * (D / 8) + 255) / 256;
        if (nwg > 0x7fffffffll) return hipErrorInvalidValue;
        hipLaunchKernelGGL((paged_append_kernel<D>), dim3((unsigned)nwg), dim3(256), 0, st, (const uint16_t*)k, k_t, k_h, (const uint16_t*)v, v_t,
                           v_h, slots, (uint16_t*)k_pages, d.kp_p, d.kp_h, (uint16_t*)vt_pages, d.vp_p, d.vp_h, d.T, d.log_p, d.n_pages << d.log_p,
                           d.Hkv);
    } else {
        const int64_t units = ((int64_t)d.T + 63) / 64 * d.Hkv * (D / 64);
        const int64_t nwg = (units + 31) / 32 * 8;       // the same number for each of the 8 XCDs
        if (nwg > 0x7fffffffll) return hipErrorInvalidValue;
        hipLaunchKernelGGL((paged_append_runs_kernel<D>), dim3((unsigned)nwg), dim3(256), 0, st, (const uint16_t*)k, k_t, k_h, (const uint16_t*)v,
                           v_t, v_h, slots, (uint16_t*)k_pages, d.kp_p, d.kp_h, (uint16_t*)vt_pages, d.vp_p, d.vp_h, d.T, d.log_p,
                           d.n_pages << d.log_p, d.Hkv, units);
    }
    return hipGetLastError();
}

}  // namespace

hipError_t launch_paged_plan(const PagedDims& d, const int32_t* ctx_lens, const int32_t* new_lens, const int32_t* free_pages, int n_free,
                             const int32_t* free_range, int32_t* block_table, int32_t* q_starts, int32_t* kv_lens, int32_t* slots,
                             int32_t* positions_or_null, int32_t* taken, hipStream_t st) {
    const int wgs = (d.T + kPlanThreads - 1) / kPlanThreads;       // 1024 at most: enough to fill the chip, and none scans for little
    hipLaunchKernelGGL(paged_plan_kernel, dim3(wgs < 1024 ? wgs : 1024), dim3(kPlanThreads), (3 * d.B + 1) * sizeof(int32_t), st, ctx_lens, new_lens, free_pages, n_free, free_range,
                       block_table, d.table_stride, q_starts, kv_lens, slots, positions_or_null, taken, d.B, d.C, d.T, d.log_p, d.n_pages);
    return hipGetLastError();
}

hipError_t launch_paged_append(const PagedDims& d, const void* k, int64_t k_t, int64_t k_h, const void* v, int64_t v_t, int64_t v_h,
                               const int32_t* slots, void* k_pages, void* vt_pages, hipStream_t st) {
    return d.D == 128 ? launch_append<128>(d, k, k_t, k_h, v, v_t, v_h, slots, k_pages, vt_pages, st)
                      : launch_append<64>(d, k, k_t, k_h, v, v_t, v_h, slots, k_pages, vt_pages, st);
}

}  // namespace spa
