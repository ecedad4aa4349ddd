// Which requests share prompts: groups of consecutive requests with the same leading pages, from the block tables of a step.
#include "paged.hpp"

namespace spa {
namespace {

// Tokens in common with the request before: a wavefront compares the two rows of a request, 256 columns at a time, up to the first that differs.  Bound by the
// latency of its loads.
__global__ __launch_bounds__(256) void paged_common_kernel(const int32_t* __restrict__ table, int64_t table_stride, const int32_t* __restrict__ q_starts,
                                                           const int32_t* __restrict__ kv_lens, int32_t* __restrict__ common, int B, int C, int T, int log_p) {
    const int lane = threadIdx.x & 63, b = blockIdx.x * 4 + (threadIdx.x >> 6);
    if (b >= B) return;
    auto whole = [&](int r) {                      // columns that a request's cached tokens fill
        const int first = clamp_int(q_starts[r], 0, T), len = clamp_int(q_starts[r + 1], first, T) - first;
        const int cached = clamp_int(kv_lens[r], 0, C << log_p) - len;
        return cached > 0 ? cached >> log_p : 0;
    };
    int n = 0;
    if (b > 0) {
        const int columns = min(whole(b), whole(b - 1));
        const int32_t* const mine = table + b * table_stride;
        const int32_t* const other = mine - table_stride;
        n = columns;
        for (int c0 = 0; c0 < columns; c0 += 256) {
            int x[4], y[4];
#pragma unroll
            for (int u = 0; u < 4; ++u) {
                const int c = min(c0 + 64 * u + lane, columns - 1);
                x[u] = mine[c];
                y[u] = other[c];
            }
            int differs = columns;
#pragma unroll
            for (int u = 3; u >= 0; --u) {
                const uint64_t here = __ballot(x[u] != y[u]);
                if (here != 0) differs = c0 + 64 * u + __builtin_ctzll(here);
            }
            if (differs < columns) {
                n = differs;
                break;
            }
        }
    }
    if (lane == 0) common[b] = n << log_p;
}

// Groups from the tokens in common: one workgroup, four consecutive requests a thread.  shares[2] holds what the kernel before has found.
constexpr int kThreads = 1024, kEach = kMaxRequests / kThreads;
__global__ __launch_bounds__(kThreads) void paged_groups_kernel(int32_t* __restrict__ shares, int B, int min_tokens) {
    __shared__ int32_t s_common[kMaxRequests + 2], s_members[kMaxRequests], s_least[kMaxRequests], s_first[kThreads / 64];
    const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6;
    for (int b = tid; b < B; b += kThreads) {
        s_common[b] = shares[2 * B + b];
        s_members[b] = 0;
        s_least[b] = 0x7fffffff;
    }
    if (tid == 0) s_common[B] = 0;
    __syncthreads();
    auto joins = [&](int b) {
        if (b == 0) return false;
        const int64_t beside = max(s_common[b - 1], s_common[b + 1]);
        return s_common[b] >= max(min_tokens, 1) && 2 * (int64_t)s_common[b] >= beside;
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
    hipLaunchKernelGGL(paged_common_kernel, dim3((unsigned)(d.B + 3) / 4), dim3(256), 0, st, block_table, d.table_stride, q_starts, kv_lens,
                       shares + 2 * (int64_t)d.B, d.B, d.C, d.T, d.log_p);
    const hipError_t e = hipGetLastError();
    if (e != hipSuccess) return e;
    hipLaunchKernelGGL(paged_groups_kernel, dim3(1), dim3(kThreads), 0, st, shares, d.B, min_tokens);
    return hipGetLastError();
}

}  // namespace spa
