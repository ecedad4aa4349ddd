// Which requests share prompts: groups of consecutive requests with the same leading pages, from the block tables of a step.
#include "paged.hpp"

namespace spa {
namespace {

struct SharesArgs {
    const int32_t *table, *q_starts, *kv_lens;
    int32_t* shares;
    int64_t table_stride;
    int B, C, T, log_p, min_tokens;
};

// Tokens in common with the request before, for requests b0 .. b0 + N - 1: a wavefront compares the two rows of each, 256 columns at a time, up to the first that
// differs.  All loads of a turn are in flight at once.
template <int N>
__device__ __forceinline__ void common_tokens(const SharesArgs& a, int b0, int (&tokens)[N]) {
    const int lane = threadIdx.x & 63;
    auto whole = [&](int r) {                      // columns that a request's cached tokens fill
        const int first = clamp_int(a.q_starts[r], 0, a.T), len = clamp_int(a.q_starts[r + 1], first, a.T) - first;
        const int cached = clamp_int(a.kv_lens[r], 0, a.C << a.log_p) - len;
        return cached > 0 ? cached >> a.log_p : 0;
    };
    int columns[N], differs[N], most = 0;
#pragma unroll
    for (int n = 0; n < N; ++n) {
        const int b = b0 + n;
        columns[n] = b > 0 && b < a.B ? min(whole(b), whole(b - 1)) : 0;
        differs[n] = columns[n];
        most = max(most, columns[n]);
    }
    for (int c0 = 0; c0 < most; c0 += 256) {
        int x[N][4], y[N][4];
#pragma unroll
        for (int n = 0; n < N; ++n) {
            const int b = min(b0 + n, a.B - 1), last = max(columns[n] - 1, 0);
            const int32_t* const mine = a.table + b * a.table_stride;
            const int32_t* const other = a.table + max(b - 1, 0) * a.table_stride;
#pragma unroll
            for (int u = 0; u < 4; ++u) {
                const int c = min(c0 + 64 * u + lane, last);
                x[n][u] = mine[c];
                y[n][u] = other[c];
            }
        }
        most = 0;                                  // columns of those that have not differed yet
#pragma unroll
        for (int n = 0; n < N; ++n) {
            int here = columns[n];
#pragma unroll
            for (int u = 3; u >= 0; --u) {
                const uint64_t odd = __ballot(x[n][u] != y[n][u]);
                if (odd != 0) here = c0 + 64 * u + __builtin_ctzll(odd);
            }
            if (differs[n] == columns[n] && here < columns[n]) differs[n] = here;
            if (differs[n] == columns[n]) most = max(most, columns[n]);
        }
    }
#pragma unroll
    for (int n = 0; n < N; ++n) tokens[n] = differs[n] << a.log_p;
}
__global__ __launch_bounds__(256) void paged_common_kernel(SharesArgs a) {
    const int b = blockIdx.x * 4 + (threadIdx.x >> 6);
    if (b >= a.B) return;
    int tokens[1];
    common_tokens(a, b, tokens);
    if ((threadIdx.x & 63) == 0) a.shares[2 * a.B + b] = tokens[0];
}

// Groups from the tokens in common: one workgroup, four consecutive requests a thread.  ALONE: it finds the tokens in common, too; else
// shares[2] holds what the kernel before has found.
constexpr int kThreads = 1024, kEach = kMaxRequests / kThreads;
// What takes a workgroup longer than another launch, 3.5 us of the host's time: turns of 64 requests x 256 columns, about 1.2 us each.  64 requests with 512 of 575
// columns in common: 11.2 us a call with two launches, 7.7 with one.
constexpr int kTurnsAlone = 4;
template <bool ALONE>
__global__ __launch_bounds__(kThreads) void paged_groups_kernel(SharesArgs a) {
    __shared__ int32_t s_common[kMaxRequests + 2], s_members[kMaxRequests], s_least[kMaxRequests], s_first[kThreads / 64];
    const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6, B = a.B;
    int32_t* const shares = a.shares;
    if constexpr (ALONE) {
        for (int b0 = 4 * wave; b0 < B; b0 += 4 * (kThreads / 64)) {
            int tokens[4];
            common_tokens(a, b0, tokens);
#pragma unroll
            for (int n = 0; n < 4; ++n)
                if (lane == 0 && b0 + n < B) s_common[b0 + n] = tokens[n];
        }
    }
    for (int b = tid; b < B; b += kThreads) {
        if constexpr (!ALONE) s_common[b] = shares[2 * B + b];
        s_members[b] = 0;
        s_least[b] = 0x7fffffff;
    }
    if (tid == 0) s_common[B] = 0;
    __syncthreads();
    auto joins = [&](int b) {
        if (b == 0) return false;
        const int64_t beside = max(s_common[b - 1], s_common[b + 1]);
        return s_common[b] >= max(a.min_tokens, 1) && 2 * (int64_t)s_common[b] >= beside;
    };
    int first[kEach];                              // of the groups that start at this thread's requests, 0 where none does
    int last = 0;
#pragma unroll
    for (int x = 0; x < kEach; ++x) {
        const int b = kEach * tid + x;
        if (b < B && !joins(b)) last = b;
        first[x] = last;
    }
    int upto = last;                               // running maximum over the threads
#pragma unroll
    for (int n = 1; n < 64; n <<= 1) {
        const int v = __shfl_up(upto, n);
        if (lane >= n) upto = max(upto, v);
    }
    if (lane == 63) s_first[wave] = upto;
    int before = __shfl_up(upto, 1);
    if (lane == 0) before = 0;
    __syncthreads();
    for (int w = 0; w < wave; ++w) before = max(before, s_first[w]);
#pragma unroll
    for (int x = 0; x < kEach; ++x) {
        const int b = kEach * tid + x;
        first[x] = max(first[x], before);
        if (b < B) {
            atomicAdd(&s_members[first[x]], 1);
            if (first[x] != b) atomicMin(&s_least[first[x]], s_common[b]);
        }
    }
    __syncthreads();
#pragma unroll
    for (int x = 0; x < kEach; ++x) {
        const int b = kEach * tid + x;
        if (b < B) {
            const int n = s_members[first[x]];
            shares[b] = first[x];
            shares[B + b] = n;
            shares[2 * B + b] = n > 1 ? s_least[first[x]] : 0;
        }
    }
}

}  // namespace

hipError_t launch_paged_shares(const PagedDims& d, const int32_t* block_table, const int32_t* q_starts, const int32_t* kv_lens, int min_tokens,
                               int32_t* shares, hipStream_t st) {
    const SharesArgs a{block_table, q_starts, kv_lens, shares, d.table_stride, d.B, d.C, d.T, d.log_p, min_tokens};
    if (((int64_t)d.B + 63) / 64 * (((int64_t)d.C + 255) / 256) <= kTurnsAlone) {
        hipLaunchKernelGGL(paged_groups_kernel<true>, dim3(1), dim3(kThreads), 0, st, a);
        return hipGetLastError();
    }
    hipLaunchKernelGGL(paged_common_kernel, dim3((unsigned)(d.B + 3) / 4), dim3(256), 0, st, a);
    const hipError_t e = hipGetLastError();
    if (e != hipSuccess) return e;
    hipLaunchKernelGGL(paged_groups_kernel<false>, dim3(1), dim3(kThreads), 0, st, a);
    return hipGetLastError();
}

}  // namespace spa
