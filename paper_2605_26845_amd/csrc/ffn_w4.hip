// moe_expert_ffn_w4_sliced: the experts' SwiGLU FFN over the row groups of a schedule with weights of 4 bits and one scale (and zero
// point) per group of 32, 64 or 128 inputs:   W[n][k] = (q[n][k] - zero[k / G][n]) * scale[k / G][n].
//
// A code becomes a bf16 value with two instructions per pair: its four bits are the upper four of a mantissa whose exponent makes the number
// (16 + q) 2^-12, exactly.  The matrix cores add products of these with x in fp32 over one group; what the 16 and the zero point added is a multiple
// of the group's sum of x, which one more product with a constant gives; and the scale multiplies the fp32 sum.  So no weight is ever
// rounded.  (2^-12: the sums of 128 products with the largest finite x stay finite.)
#include "common.hpp"
#include "rows.hpp"
#include <algorithm>
#include <type_traits>

namespace {

typedef __attribute__((ext_vector_type(8))) __bf16 bf16x8;
typedef __attribute__((ext_vector_type(4))) float f32x4;
typedef __attribute__((ext_vector_type(4))) unsigned int u32x4;

constexpr int W4_STEP = 128;                    // values of K per step: 16 bytes of codes per lane, 16 weight rows
constexpr unsigned int CODE_BASE = 0x3B803B80u; // 16 * 2^-12 twice; the code goes to bits 3 .. 6 of either half
constexpr unsigned int ONES = 0x39803980u;      // 2^-12 twice
constexpr unsigned int MINUS_24 = 0xBBC0BBC0u;  // -24 * 2^-12 twice: symmetric codes have the zero point 8
constexpr float CODE_UNIT = 0x1p12f;

struct W4Args {
    const __bf16* x; __bf16* h; __bf16* y;      // h: K-major, [f / 8][M][8]
    const unsigned char *qg, *qu, *qd;
    const unsigned short *sg, *su, *sd;
    const unsigned char *zg, *zu, *zd;
    const int32_t* offsets;
    const int32_t* row_map; const float* row_gate;
    int M, S, E, d, f;
};

__device__ __forceinline__ float silu(float g) { return g * __builtin_amdgcn_rcpf(1.0f + __expf(-g)); }

__device__ __forceinline__ int w4_mapped(const W4Args& a, int m) {
    if (!a.row_map) return m;
    const int r = a.row_map[m];
    return (unsigned)r < (unsigned)a.M ? r : 0;
}

// Positions first .. first + ROWS - 1 of expert e's rows (of all slices, in schedule order) -> s_row; returns how many rows the expert has.
// All THREADS threads take part.
template <int THREADS, int ROWS>
__device__ __forceinline__ int expert_rows(const W4Args& a, int e, int first, int* s_row, int* s_scan) {
    constexpr int W = THREADS / 64;
    const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6;
    int total = 0;
    for (int s0 = 0; s0 < a.S; s0 += THREADS) {
        const int s = s0 + tid;
        int lo = 0, rows = 0;
        if (s < a.S) rows = group_rows(a.offsets, s * a.E + e, a.M, lo);
        int incl = rows;
#pragma unroll
        for (int off = 1; off < 64; off <<= 1) {
            const int o = __shfl_up(incl, off);
            if (lane >= off) incl = add_rows(incl, o, a.M);
        }
        if (lane == 63) s_scan[wave] = incl;
        __syncthreads();
        int base = total;
#pragma unroll
        for (int w = 0; w < W; ++w) {
            const int t = s_scan[w];
            if (w < wave) base = add_rows(base, t, a.M);
            total = add_rows(total, t, a.M);
        }
        const int p0 = add_rows(base, incl, a.M) - rows;
        for (int p = max(p0, first); p < min(p0 + rows, first + ROWS); ++p) s_row[p - first] = lo + (p - p0);
        __syncthreads();
    }
    return total;
}

// 16 bytes of codes per lane: lane (r16, g4) has k = 32 g4 .. 32 g4 + 31 of its weight row.  Afterwards dword i holds k = 32 i + 8 g4 .. + 7,
// so that a matrix instruction over dword i stays inside 32 consecutive values of K, as the order of x in memory and groups of 32 want it.
__device__ __forceinline__ void across_lanes(u32x4& c) {
    auto a = __builtin_amdgcn_permlane32_swap(c[0], c[2], false, false);
    auto b = __builtin_amdgcn_permlane32_swap(c[1], c[3], false, false);
    auto p = __builtin_amdgcn_permlane16_swap(a[0], b[0], false, false);
    auto q = __builtin_amdgcn_permlane16_swap(a[1], b[1], false, false);
    c = u32x4{p[0], p[1], q[0], q[1]};
}

// 8 codes -> (16 + q) 2^-12 in the order 0 4 1 5 2 6 3 7
__device__ __forceinline__ bf16x8 code_values(unsigned int c) {
    constexpr unsigned int MASK = 0x00780078u;
    const u32x4 v = {((c << 3) & MASK) | CODE_BASE, ((c >> 1) & MASK) | CODE_BASE, ((c >> 5) & MASK) | CODE_BASE, ((c >> 9) & MASK) | CODE_BASE};
    return __builtin_bit_cast(bf16x8, v);
}
// 8 values of x in that order
__device__ __forceinline__ bf16x8 in_code_order(u32x4 x) {
    const u32x4 v = {__builtin_amdgcn_perm(x[2], x[0], 0x05040100u), __builtin_amdgcn_perm(x[2], x[0], 0x07060302u),
                     __builtin_amdgcn_perm(x[3], x[1], 0x05040100u), __builtin_amdgcn_perm(x[3], x[1], 0x07060302u)};
    return __builtin_bit_cast(bf16x8, v);
}
__device__ __forceinline__ bf16x8 splat(unsigned int two) { return __builtin_bit_cast(bf16x8, (u32x4{two, two, two, two})); }

// The NG groups of a step: lane (r16, g4) was given group g4 % NG of its weight row, as scale << 16 | zero; all lanes get all of them.
template <int NG> __device__ __forceinline__ void all_groups(unsigned int v, unsigned int (&out)[NG]) {
    if constexpr (NG == 1) out[0] = v;
    if constexpr (NG == 2) {
        const auto r = __builtin_amdgcn_permlane16_swap(v, v, false, false);
        out[0] = r[0]; out[1] = r[1];
    }
    if constexpr (NG == 4) {
        const auto r = __builtin_amdgcn_permlane32_swap(v, v, false, false);
        const auto p = __builtin_amdgcn_permlane16_swap(r[0], r[0], false, false), q = __builtin_amdgcn_permlane16_swap(r[1], r[1], false, false);
        out[0] = p[0]; out[1] = p[1]; out[2] = q[0]; out[3] = q[1];
    }
}

// ---------------------------------------------------------------------------------- few rows per expert (decoding)
// Bound by the weights' way from HBM.  A workgroup takes 16 output columns of one expert (phase 1: the gate and the up rows of 16 hidden units) and up to
// 16 * MT of its rows; its W wavefronts share the contraction, 128 values of K each in turn, codes and activations straight from memory into the
// fragments of the matrix instruction, D - 1 steps in flight.  The W partial sums meet in LDS and are added in a fixed order.
template <int PHASE, int W, int MT, int D, int G, bool ZERO>
__global__ __launch_bounds__(W * 64)
void ffn_w4_stream_kernel(W4Args a) {
    constexpr int NC = PHASE == 1 ? 2 : 1, NG = W4_STEP / G, PER = G / 32;
    constexpr int ROWS = 16 * MT;
    __shared__ int s_row[ROWS];
    __shared__ int s_scan[W];
    __shared__ f32x4 s_red[NC * W * 64];
    const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6);
    const int r16 = lane & 15, g4 = lane >> 4;
    const int e = blockIdx.y, col0 = blockIdx.x * 16;
    const int K = PHASE == 1 ? a.d : a.f, NO = PHASE == 1 ? a.f : a.d;
    const int KT = K / W4_STEP, n = (KT - wave + W - 1) / W;               // steps in all, and of this wavefront
    const int rot = (int)((blockIdx.x * 3u + e * 3u) % (unsigned)KT);      // the strips start at different steps: neighbouring strips' rows lie in the same memory channels

    for (int first = (int)blockIdx.z * ROWS;; first += (int)gridDim.z * ROWS) {
        const int rows = min(expert_rows<W * 64, ROWS>(a, e, first, s_row, s_scan) - first, ROWS);
        if (rows <= 0) return;
        auto work = [&](auto tag) __attribute__((always_inline)) {
            constexpr int T = decltype(tag)::value;                        // 16-row tiles of x
            f32x4 acc[NC][T];
#pragma unroll
            for (int c = 0; c < NC; ++c)
#pragma unroll
                for (int t = 0; t < T; ++t) acc[c][t] = f32x4{0.f, 0.f, 0.f, 0.f};
            unsigned int xoff[T];                                          // (M * K * 2 < 2^32 is a condition of this kernel)
#pragma unroll
            for (int t = 0; t < T; ++t) {
                const int m = s_row[min(t * 16 + r16, rows - 1)];          // rows past the end repeat the last one and are not stored
                xoff[t] = PHASE == 1 ? ((unsigned int)w4_mapped(a, m) * (unsigned int)K + (unsigned int)g4 * 8u) * 2u : ((unsigned int)g4 * (unsigned int)a.M + (unsigned int)m) * 16u;
            }
            const void* const xbase = PHASE == 1 ? (const void*)a.x : (const void*)a.h;
            const unsigned int xbytes = (unsigned int)a.M * (unsigned int)K * 2u;
            const unsigned int xk = PHASE == 1 ? 2u : 2u * (unsigned int)a.M;              // bytes per value of K
            const unsigned char* qbase[NC];
            const unsigned short* sbase[NC];
            const unsigned char* zbase[NC];
#pragma unroll
            for (int c = 0; c < NC; ++c) {
                const size_t row = (size_t)e * NO + col0, group = (size_t)e * (K / G) * NO + col0;
                qbase[c] = (PHASE == 2 ? a.qd : c ? a.qu : a.qg) + row * (size_t)(K / 2);
                sbase[c] = (PHASE == 2 ? a.sd : c ? a.su : a.sg) + group;
                zbase[c] = ZERO ? (PHASE == 2 ? a.zd : c ? a.zu : a.zg) + group : nullptr;
            }
            const unsigned int qoff = (unsigned int)r16 * (unsigned int)(K / 2) + (unsigned int)g4 * 16u, qbytes = 16u * (unsigned int)(K / 2);
            const unsigned int soff = (unsigned int)(g4 % NG) * (unsigned int)NO + (unsigned int)r16, selems = (unsigned int)(K / G) * (unsigned int)NO - (unsigned int)col0;
            struct Buf { u32x4 q[NC], x[T][4]; unsigned int s[NC], z[NC]; };
            Buf buf[D];
            // steps past the last one read through an empty descriptor: zeros, and no memory traffic
            auto load = [&](Buf& b, int i) __attribute__((always_inline)) {
                const bool live = i < n;
                int kc = wave + W * (live ? i : 0) + rot;
                kc = kc >= KT ? kc - KT : kc;
                const __amdgpu_buffer_rsrc_t rx = __builtin_amdgcn_make_buffer_rsrc((void*)xbase, 0, live ? xbytes : 0u, 0x00020000);
#pragma unroll
                for (int c = 0; c < NC; ++c) {
                    const __amdgpu_buffer_rsrc_t rq = __builtin_amdgcn_make_buffer_rsrc((void*)qbase[c], 0, live ? qbytes : 0u, 0x00020000);
                    b.q[c] = __builtin_amdgcn_raw_buffer_load_b128(rq, qoff + (unsigned int)kc * (W4_STEP / 2), 0, 0);
                    const __amdgpu_buffer_rsrc_t rs = __builtin_amdgcn_make_buffer_rsrc((void*)sbase[c], 0, live ? selems * 2u : 0u, 0x00020000);
                    const unsigned int so = soff + (unsigned int)kc * NG * (unsigned int)NO;
                    b.s[c] = __builtin_amdgcn_raw_buffer_load_b16(rs, so * 2u, 0, 0);
                    if (ZERO) {
                        const __amdgpu_buffer_rsrc_t rz = __builtin_amdgcn_make_buffer_rsrc((void*)zbase[c], 0, live ? selems : 0u, 0x00020000);
                        b.z[c] = __builtin_amdgcn_raw_buffer_load_b8(rz, so, 0, 0);
                    }
                }
#pragma unroll
                for (int t = 0; t < T; ++t)
#pragma unroll
                    for (int i4 = 0; i4 < 4; ++i4) b.x[t][i4] = __builtin_amdgcn_raw_buffer_load_b128(rx, xoff[t] + ((unsigned int)kc * W4_STEP + i4 * 32u) * xk, 0, 0);
            };
            auto multiply = [&](Buf& b) __attribute__((always_inline)) {
                const f32x4 none = {0.f, 0.f, 0.f, 0.f};
                const bf16x8 constant = splat(ZERO ? ONES : MINUS_24);
                bf16x8 xv[T][4];
                f32x4 part[T][NG];                                         // the group's sum of x, times 2^-12 (with zero points) or -24 * 2^-12
#pragma unroll
                for (int t = 0; t < T; ++t)
#pragma unroll
                    for (int i = 0; i < 4; ++i) {
                        xv[t][i] = in_code_order(b.x[t][i]);
                        part[t][i / PER] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(xv[t][i], constant, i % PER == 0 ? none : part[t][i / PER], 0, 0, 0);
                    }
#pragma unroll
                for (int c = 0; c < NC; ++c) {
                    across_lanes(b.q[c]);
                    unsigned int sz[NG];
                    all_groups<NG>(b.s[c] << 16 | (ZERO ? b.z[c] & 15u : 0u), sz);
#pragma unroll
                    for (int gr = 0; gr < NG; ++gr) {
                        f32x4 sum[T];
#pragma unroll
                        for (int i = gr * PER; i < (gr + 1) * PER; ++i) {
                            const bf16x8 wv = code_values(b.q[c][i]);
#pragma unroll
                            for (int t = 0; t < T; ++t) sum[t] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(xv[t][i], wv, i % PER != 0 ? sum[t] : ZERO ? none : part[t][gr], 0, 0, 0);
                        }
                        const float scale = __builtin_bit_cast(float, sz[gr] & 0xFFFF0000u) * CODE_UNIT;
                        const float off = -(16.0f + (float)(sz[gr] & 15u));
#pragma unroll
                        for (int t = 0; t < T; ++t)
#pragma unroll
                            for (int v = 0; v < 4; ++v) {
                                const float w = ZERO ? __builtin_fmaf(off, part[t][gr][v], sum[t][v]) : sum[t][v];
                                acc[c][t][v] = __builtin_fmaf(scale, w, acc[c][t][v]);
                            }
                    }
                }
            };
#pragma unroll
            for (int i = 0; i < D - 1; ++i) load(buf[i], i);
            for (int i = 0; i < n; i += D) {
#pragma unroll
                for (int u = 0; u < D; ++u) {
                    load(buf[(u + D - 1) % D], i + u + D - 1);
                    __builtin_amdgcn_sched_barrier(0);
                    multiply(buf[u]);
                    __builtin_amdgcn_sched_barrier(0);
                }
            }
            // ---- acc[c][t][v]: row 4 * g4 + v of row tile t, column r16
#pragma unroll
            for (int t = 0; t < T; ++t) {
                if (t > 0) __syncthreads();
#pragma unroll
                for (int c = 0; c < NC; ++c) s_red[(c * W + wave) * 64 + lane] = acc[c][t];
                __syncthreads();
                const float* const red = (const float*)s_red;
                for (int it = tid; it < 256; it += W * 64) {
                    const int col = it & 15, m16 = it >> 4, at = ((m16 >> 2) * 16 + col) * 4 + (m16 & 3);
                    float s0 = red[at], s1 = 0.f;
#pragma unroll
                    for (int w = 1; w < W; ++w) s0 += red[w * 256 + at];
                    if (PHASE == 1) {
#pragma unroll
                        for (int w = 0; w < W; ++w) s1 += red[(W + w) * 256 + at];
                    }
                    if (t * 16 + m16 < rows) {
                        const int m = s_row[t * 16 + m16], o = col0 + col;
                        // the hidden activation is rounded to bf16 once, as the operand of the second product
                        if (PHASE == 1) a.h[((size_t)(o >> 3) * a.M + m) * 8 + (o & 7)] = (__bf16)(silu(s0) * s1);
                        else a.y[(size_t)w4_mapped(a, m) * a.d + o] = (__bf16)(a.row_gate ? a.row_gate[m] * s0 : s0);
                    }
                }
            }
        };
        const int tiles = (rows + 15) / 16;
        if (MT == 1 || tiles == 1) work(std::integral_constant<int, 1>{});
        else if (MT == 2 || tiles == 2) work(std::integral_constant<int, (MT < 2 ? MT : 2)>{});
        else work(std::integral_constant<int, MT>{});
        __syncthreads();                                                   // s_row and s_red are used again
    }
}

template <int PHASE, int W, int MT, int D, int G, bool ZERO> moe_status launch_stream(const W4Args& a, hipStream_t s) {
    const int blocks = std::min((a.M - 1) / (16 * MT) + 1, 8);
    moe::LaunchScope k(PHASE == 1 ? "ffn_w4_stream1_kernel" : "ffn_w4_stream2_kernel", s);
    hipLaunchKernelGGL((ffn_w4_stream_kernel<PHASE, W, MT, D, G, ZERO>), dim3((PHASE == 1 ? a.f : a.d) / 16, a.E, blocks), dim3(W * 64), 0, s, a);
    return k.done();
}
template <int G, bool ZERO> moe_status stream_both(const W4Args& a, hipStream_t s) {
    moe_status st;
    if (a.M <= 16) {
        if ((st = launch_stream<1, 8, 1, 4, G, ZERO>(a, s))) return st;
        return launch_stream<2, 8, 1, 4, G, ZERO>(a, s);
    }
    if ((st = launch_stream<1, 8, 2, 2, G, ZERO>(a, s))) return st;
    return launch_stream<2, 8, 2, 2, G, ZERO>(a, s);
}
template <int G> moe_status stream_of(const W4Args& a, hipStream_t s) { return a.zg ? stream_both<G, true>(a, s) : stream_both<G, false>(a, s); }

size_t h_bytes(int M, int f) { return (((size_t)M * f * 2) + 255) & ~(size_t)255; }

constexpr int W4_MAX_GROUPS = 65536;

}  // namespace

extern "C" size_t moe_ffn_w4_workspace_bytes(int M, int d, int f) {
    if (M < 0 || d < 1 || f < 1) return 0;
    return h_bytes(M, f);
}

extern "C" moe_status moe_expert_ffn_w4_sliced(const void* x, const int32_t* offsets, int M, int S, int E_loc, int d, int f, int group,
                                               const void* q_gate, const void* q_up, const void* q_down, const void* s_gate, const void* s_up, const void* s_down,
                                               const void* z_gate, const void* z_up, const void* z_down, const int32_t* row_map, const float* row_gate,
                                               void* y, void* workspace, size_t workspace_bytes, void* hip_stream) {
    if (M < 0 || S < 0 || E_loc < 1 || d < 1 || f < 1 || !offsets || !q_gate || !q_up || !q_down || !s_gate || !s_up || !s_down) return MOE_ERR_INVALID_ARG;
    if ((z_gate == nullptr) != (z_up == nullptr) || (z_gate == nullptr) != (z_down == nullptr)) return MOE_ERR_INVALID_ARG;
    if ((group != 32 && group != 64 && group != 128) || d % 256 != 0 || f % 128 != 0) return MOE_ERR_UNSUPPORTED_SHAPE;
    const long long groups = (long long)S * E_loc;
    if (groups > W4_MAX_GROUPS || d > (1 << 22) || f > (1 << 22) || (long long)d * f >= (1LL << 31)) return MOE_ERR_UNSUPPORTED_SHAPE;
    if ((unsigned long long)M * std::max(d, f) * 2 >= 0xFFFFFF00ull) return MOE_ERR_UNSUPPORTED_SHAPE;
    if (M == 0 || groups == 0) return MOE_OK;
    if (!x || !y) return MOE_ERR_INVALID_ARG;
    if ((((uintptr_t)x | (uintptr_t)y | (uintptr_t)q_gate | (uintptr_t)q_up | (uintptr_t)q_down | (uintptr_t)workspace) & 15) != 0) return MOE_ERR_INVALID_ARG;
    if ((((uintptr_t)s_gate | (uintptr_t)s_up | (uintptr_t)s_down) & 1) != 0 || (((uintptr_t)row_map | (uintptr_t)row_gate | (uintptr_t)offsets) & 3) != 0) return MOE_ERR_INVALID_ARG;
    if (!workspace || workspace_bytes < moe_ffn_w4_workspace_bytes(M, d, f)) return MOE_ERR_WORKSPACE;
    const W4Args a = {(const __bf16*)x, (__bf16*)workspace, (__bf16*)y, (const unsigned char*)q_gate, (const unsigned char*)q_up, (const unsigned char*)q_down,
                      (const unsigned short*)s_gate, (const unsigned short*)s_up, (const unsigned short*)s_down, (const unsigned char*)z_gate,
                      (const unsigned char*)z_up, (const unsigned char*)z_down, offsets, row_map, row_gate, M, S, E_loc, d, f};
    hipStream_t s = (hipStream_t)hip_stream;
    return group == 32 ? stream_of<32>(a, s) : group == 64 ? stream_of<64>(a, s) : stream_of<128>(a, s);
}
