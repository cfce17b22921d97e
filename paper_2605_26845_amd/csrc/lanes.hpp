// Reductions over the lanes of a wavefront and over the wavefronts of a workgroup.  The order of the additions is fixed.
#pragma once
#include "common.hpp"

namespace moe {

// x of the lane that differs in bit 0, bit 1, and of the mirrored lane of 8 and of 16: four steps leave every lane of 16 with the same result
template <int CTRL> __device__ __forceinline__ float dpp_f32(float x) {
    return __builtin_bit_cast(float, __builtin_amdgcn_update_dpp(0, __builtin_bit_cast(int, x), CTRL, 0xF, 0xF, true));
}
template <int CTRL> __device__ __forceinline__ unsigned int dpp_u32(unsigned int x) {
    return (unsigned int)__builtin_amdgcn_update_dpp(0, (int)x, CTRL, 0xF, 0xF, true);
}
constexpr int DPP_XOR1 = 0xB1, DPP_XOR2 = 0x4E, DPP_HALF_MIRROR = 0x141, DPP_MIRROR = 0x140;

// the two rows of 16 (halves of 32 lanes, of the wavefront) next to each other: what both hold, in the same order in every lane
__device__ __forceinline__ void rows16(unsigned int x, unsigned int& a, unsigned int& b) {
    const auto r = __builtin_amdgcn_permlane16_swap(x, x, false, false);
    a = r[0]; b = r[1];
}
__device__ __forceinline__ void rows32(unsigned int x, unsigned int& a, unsigned int& b) {
    const auto r = __builtin_amdgcn_permlane32_swap(x, x, false, false);
    a = r[0]; b = r[1];
}

// sum over the LANES (a power of two) neighbouring lanes, in all of them
template <int LANES> __device__ __forceinline__ float lanes_sum(float x) {
    if (LANES >= 2) x += dpp_f32<DPP_XOR1>(x);
    if (LANES >= 4) x += dpp_f32<DPP_XOR2>(x);
    if (LANES >= 8) x += dpp_f32<DPP_HALF_MIRROR>(x);
    if (LANES >= 16) x += dpp_f32<DPP_MIRROR>(x);
    unsigned int a, b;
    if (LANES >= 32) { rows16(__builtin_bit_cast(unsigned int, x), a, b); x = __builtin_bit_cast(float, a) + __builtin_bit_cast(float, b); }
    if (LANES >= 64) { rows32(__builtin_bit_cast(unsigned int, x), a, b); x = __builtin_bit_cast(float, a) + __builtin_bit_cast(float, b); }
    return x;
}
template <int LANES> __device__ __forceinline__ unsigned int lanes_max(unsigned int x) {
    if (LANES >= 2) x = max(x, dpp_u32<DPP_XOR1>(x));
    if (LANES >= 4) x = max(x, dpp_u32<DPP_XOR2>(x));
    if (LANES >= 8) x = max(x, dpp_u32<DPP_HALF_MIRROR>(x));
    if (LANES >= 16) x = max(x, dpp_u32<DPP_MIRROR>(x));
    unsigned int a, b;
    if (LANES >= 32) { rows16(x, a, b); x = max(a, b); }
    if (LANES >= 64) { rows32(x, a, b); x = max(a, b); }
    return x;
}
template <int LANES> __device__ __forceinline__ unsigned int lanes_min(unsigned int x) { return ~lanes_max<LANES>(~x); }

// Workgroup barrier that orders LDS traffic only: stores to memory stay in flight across it.
__device__ __forceinline__ void lds_only_barrier() {
    asm volatile("s_waitcnt lgkmcnt(0)" ::: "memory");
    __builtin_amdgcn_s_barrier();
    asm volatile("" ::: "memory");
}

// N sums over the THREADS threads of a workgroup, in all of them; s: 2 * N * THREADS / 64 floats, of which `half` picks the half that is
// written (the other one may still be read by wavefronts that are behind)
template <int THREADS, int N> __device__ __forceinline__ void workgroup_sums(float (&v)[N], float* s, int& half) {
#pragma unroll
    for (int n = 0; n < N; ++n) v[n] = lanes_sum<64>(v[n]);
    if constexpr (THREADS > 64) {
        constexpr int W = THREADS / 64;
        float* const at = s + half * (N * W);
        const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
        if (lane == 0) {
#pragma unroll
            for (int n = 0; n < N; ++n) at[n * W + wave] = v[n];
        }
        lds_only_barrier();
#pragma unroll
        for (int n = 0; n < N; ++n) {
            float t = at[n * W];
#pragma unroll
            for (int w = 1; w < W; ++w) t += at[n * W + w];
            v[n] = t;
        }
        half ^= 1;
    }
}

}  // namespace moe
