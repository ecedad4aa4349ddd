// What the attention kernels share: operand types, tile staging (direct loads into LDS, the swizzles against bank conflicts) and
// the instruction groups of their pipeline step.  gfx950.
#pragma once
#include <hip/hip_runtime.h>
#include <stdint.h>

#include <type_traits>

namespace spa {

typedef __attribute__((ext_vector_type(8))) __bf16 bf16x8;
typedef __attribute__((ext_vector_type(4))) __bf16 bf16x4;
typedef __attribute__((ext_vector_type(2))) __bf16 bf16x2;
typedef __attribute__((ext_vector_type(4))) uint32_t u32x4;
typedef __attribute__((ext_vector_type(16))) float f32x16;
typedef __attribute__((ext_vector_type(8))) float f32x8;
typedef __attribute__((ext_vector_type(4))) float f32x4;
typedef __attribute__((address_space(3))) void lds_void;
typedef __attribute__((address_space(1))) const void gbl_void;

__device__ __forceinline__ int swz_v(int row) { return (row >> 1) & 7; }                        // 128-B rows
// K rows are 2 * head_dim bytes: 256 B (16 chunks of 16 B) or 128 B (8 chunks, same rule as V^T rows)
template <int HD>
__device__ __forceinline__ int swz_k(int row) {
    if constexpr (HD == 128) return ((row & 3) << 2) | ((row >> 2) & 3);
    else return (row >> 1) & 7;
}
// value held by lane ^ 32, via v_permlane32_swap (no LDS round trip)
__device__ __forceinline__ float other_half(float x) {
    typedef __attribute__((ext_vector_type(2))) unsigned u32x2;
    u32x2 r = __builtin_amdgcn_permlane32_swap(__float_as_uint(x), __float_as_uint(x), false, false);
    // r[0]: lanes 32..63 now hold lanes 0..31's value; r[1]: lanes 0..31 hold lanes 32..63's value
    return __uint_as_float((threadIdx.x & 32) ? r[0] : r[1]);
}
// 16 bytes per lane straight from global memory into LDS (global_load_lds_dwordx4): the wave's 64
// lanes fill 1 KB starting at LDS byte address lds_addr + IMM, lane l from sbase + voff(l).  Written as
// inline assembly on purpose: the compiler models the builtin form as an access whose completion
// order is unknown, and from then on turns every wait for an LDS read into a wait for all of
// them, which defeats the read-ahead in the pipeline step.  The kernel waits for these loads
// itself (s_waitcnt vmcnt(0) before the barrier that publishes a sub-tile).
#pragma clang diagnostic ignored "-Winline-asm"
template <int IMM>
__device__ __forceinline__ void lds_dma16(uint32_t lds_addr, uint32_t voff, const void* sbase) {
    asm volatile("s_add_u32 m0, %0, %3\n\ts_nop 0\n\tglobal_load_lds_dwordx4 %1, %2"
                 :
                 : "s"(lds_addr), "v"(voff), "s"(sbase), "i"(IMM)
                 : "memory", "m0", "scc");
}
__device__ __forceinline__ uint32_t lds_address(const void* p) { return (uint32_t)(size_t)(lds_void*)p; }
__device__ __forceinline__ int swap_bits23(int x) { return (x & ~12) | ((x & 4) << 1) | ((x & 8) >> 1); }

// ---------------------------------------------------------------------------
// Instruction order inside a pipeline step is written out by hand: every group between two
// fences holds one MFMA, the LDS read of an operand needed three MFMAs later and a few softmax
// VALU instructions, and the scheduler may not move anything across a fence.  Left to itself the
// compiler (register pressure is high) sinks each LDS read to just before the MFMA that uses it
// and clusters the VALU work, so the wave stalls on the LDS latency once per MFMA.
#define SPA_FENCE() __builtin_amdgcn_sched_barrier(0)

template <int N>
using IC = std::integral_constant<int, N>;
// f(IC<0>{}), ..., f(IC<N-1>{})
template <int N, typename F>
__device__ __forceinline__ void static_for(F&& f) {
    if constexpr (N > 0) {
        static_for<N - 1>(f);
        f(IC<N - 1>{});
    }
}

// Instruction group g of a pipeline step (a step = one 32-key chunk = NG = D / 8 groups, one MFMA each).
// The MFMA: even groups add slice g / 2 of the logits of chunk n + 2 (A operand `a` = 32 K rows x 16
// dims), odd groups add V^T (32 d rows x 16 keys) times the weights pc of chunk n into O^T.
template <int g, int D>
__device__ __forceinline__ void group_mfma(const bf16x8& a, const bf16x8 (&qf)[D / 16], f32x16& s_nxt,
                                           f32x16 (&oacc)[D / 32], const bf16x8& pc0, const bf16x8& pc1) {
    constexpr int NG = D / 8, DT = D / 32;
    if constexpr (g % 2 == 0) {
        if constexpr (g == 0) {
            f32x16 zero;
#pragma unroll
            for (int r = 0; r < 16; ++r) zero[r] = 0.f;
            s_nxt = __builtin_amdgcn_mfma_f32_32x32x16_bf16(a, qf[g / 2], zero, 0, 0, 0);
        } else {
            s_nxt = __builtin_amdgcn_mfma_f32_32x32x16_bf16(a, qf[g / 2], s_nxt, 0, 0, 0);
        }
    } else {
        constexpr int dc = (g / 2) % DT;
        if constexpr (g < NG / 2) oacc[dc] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(a, pc0, oacc[dc], 0, 0, 0);
        else oacc[dc] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(a, pc1, oacc[dc], 0, 0, 0);
    }
}
// The group's share of the softmax arithmetic of chunk n + 1: its 16 logits s_cur form two halves of
// 8 (keys 0-15 / 16-31), each turned into weights pn over NG / 2 consecutive groups: scaled
// differences (8 fma), powers of two (8 exp2), conversion to bf16, denominator.
template <int g, int D>
__device__ __forceinline__ void group_weights(const f32x16& s_cur, float c, float mcb, f32x8& e, bf16x8& pn0, bf16x8& pn1,
                                              float& l_new) {
    constexpr int NG = D / 8;
    constexpr int HG = NG / 2;               // groups per half of the chunk's 16 logits
    constexpr int hb = (g / HG) * 8;         // which half
    constexpr int gg = g % HG;
    constexpr bool first_half = g < HG;
    auto scale_sub = [&](int x0, int n) {
#pragma unroll
        for (int x = x0; x < x0 + n; ++x) e[x] = fmaf(s_cur[hb + x], c, -mcb);
    };
    auto exps = [&](int x0, int n) {
#pragma unroll
        for (int x = x0; x < x0 + n; ++x) e[x] = __builtin_amdgcn_exp2f(e[x]);
    };
    auto convert = [&]() {
        if constexpr (first_half) pn0 = __builtin_convertvector(e, bf16x8);
        else pn1 = __builtin_convertvector(e, bf16x8);
    };
    auto sum_and_test = [&]() {
        const bf16x2 ones = {(__bf16)1.0f, (__bf16)1.0f};
        const bf16x8 pw = first_half ? pn0 : pn1;
#pragma unroll
        for (int x = 0; x < 4; ++x)
            l_new = __builtin_amdgcn_fdot2_f32_bf16(bf16x2{pw[2 * x], pw[2 * x + 1]}, ones, l_new, false);
        if constexpr (g == NG - 1) asm volatile("" : "+v"(l_new));   // keep the sums inside their groups
    };
    if constexpr (HG == 8) {                 // head_dim 128: 8 groups per half
        if constexpr (gg < 2) scale_sub(4 * gg, 4);
        else if constexpr (gg < 6) exps(2 * (gg - 2), 2);
        else if constexpr (gg == 6) convert();
        else sum_and_test();
    } else {                                 // head_dim 64: 4 groups per half
        static_assert(HG == 4 || HG == 8, "head_dim 64 or 128");
        if constexpr (gg == 0) scale_sub(0, 8);
        else if constexpr (gg == 1) exps(0, 4);
        else if constexpr (gg == 2) exps(4, 4);
        else { convert(); sum_and_test(); }
    }
}

}  // namespace spa
