// moe_block_norm, moe_block_join and their backward passes: the norms before and after a MoE block, its token gate and residual scale
// (Section 2.1: a MoE block replaces the feed-forward block between two residual connections).
//
//   join:  u = z rsqrt(mean z^2 + eps) w1 (or z),  out = scale stream + gate u,  next = out rsqrt(mean out^2 + eps) w2
//
// All of it is one pass over the rows: a row stays in registers between the two sums over its columns, so z and the stream are read once and
// out and next written once.  HBM bound; a thread owns 8 consecutive columns per step (16 bytes of bf16).  A row of up to 1024 columns belongs to
// one wavefront (no barriers, four rows per workgroup), a longer one to a workgroup.  16381 rows of 7168 in bf16: 168 us, 5.6 TB/s (with 256 threads and four steps a row 184), the
// first dozens of passes after a pause 183; 4096 rows of 16384, two steps of 1024 threads: 101 us, 5.3 TB/s; one row of 4096: 2.6 us, a launch and two trips to memory.
#include "lanes.hpp"
#include <algorithm>

namespace {

typedef __attribute__((ext_vector_type(8))) __bf16 b_bf16x8;
typedef __attribute__((ext_vector_type(4))) unsigned int b_u32x4;
typedef __attribute__((ext_vector_type(4))) float b_f32x4;

constexpr int BLOCK_MAX_COLUMNS = 16384;       // a row's columns live in registers
constexpr int BLOCK_MAX_PARTS = 1024;          // sums over tokens that are added up by a second kernel

struct Raw8 { b_u32x4 a, b; };                 // 8 values as they lie in memory: bf16 (a) or float (a, b)

template <bool F32> __device__ __forceinline__ Raw8 load8(const void* p, size_t i) {
    Raw8 r;
    if constexpr (F32) {
        r.a = *reinterpret_cast<const b_u32x4*>((const float*)p + i);
        r.b = *reinterpret_cast<const b_u32x4*>((const float*)p + i + 4);
    } else {
        r.a = *reinterpret_cast<const b_u32x4*>((const __bf16*)p + i);
        r.b = b_u32x4{0u, 0u, 0u, 0u};
    }
    return r;
}
template <bool F32> __device__ __forceinline__ void widen8(const Raw8& r, float (&v)[8]) {
    if constexpr (F32) {
        const b_f32x4 a = __builtin_bit_cast(b_f32x4, r.a), b = __builtin_bit_cast(b_f32x4, r.b);
#pragma unroll
        for (int c = 0; c < 4; ++c) { v[c] = a[c]; v[4 + c] = b[c]; }
    } else {
        const b_bf16x8 x = __builtin_bit_cast(b_bf16x8, r.a);
#pragma unroll
        for (int c = 0; c < 8; ++c) v[c] = (float)x[c];
    }
}
template <bool F32> __device__ __forceinline__ void store8(void* p, size_t i, const float (&v)[8]) {
    if constexpr (F32) {
        *reinterpret_cast<b_f32x4*>((float*)p + i) = b_f32x4{v[0], v[1], v[2], v[3]};
        *reinterpret_cast<b_f32x4*>((float*)p + i + 4) = b_f32x4{v[4], v[5], v[6], v[7]};
    } else {
        b_bf16x8 o;
#pragma unroll
        for (int c = 0; c < 8; ++c) o[c] = (__bf16)v[c];
        *reinterpret_cast<b_u32x4*>((__bf16*)p + i) = __builtin_bit_cast(b_u32x4, o);
    }
}
__device__ __forceinline__ void weights8(const float* w, int col, float (&v)[8]) {
    Raw8 r = load8<true>(w, (size_t)col);
    widen8<true>(r, v);
}
__device__ __forceinline__ float inverse_rms(float sum_of_squares, int d, float eps) { return 1.0f / sqrtf(sum_of_squares / (float)d + eps); }

// out may be the stream and next may be z: a thread reads its columns of a row before it writes any of them
struct ForwardArgs {
    const void* z;                             // join only
    const void* stream;
    const float *w1, *gate, *w2;
    void *out, *next;                          // out: join only
    float scale, eps;
    int T, d;
    int first;                                 // row of the first workgroup
};

// NT threads and NV steps of NT * 8 columns per row
template <int NT, int NV, bool F32, bool JOIN>
__global__ __launch_bounds__(NT == 64 ? 256 : NT)
void block_forward_kernel(ForwardArgs a) {
    constexpr int PER = NT == 64 ? 4 : 1;                                  // rows per workgroup
    __shared__ float s_sum[2 * (NT / 64)];
    int half = 0;
    const int tid = threadIdx.x % NT;
    const long long row = a.first + (long long)blockIdx.x * PER + (int)threadIdx.x / NT;
    if (row >= a.T) return;                                               // (a whole wavefront, which meets no barrier if NT is 64)
    const size_t base = (size_t)row * a.d;
    Raw8 rz[NV], rx[NV];
#pragma unroll
    for (int v = 0; v < NV; ++v) {
        const int col = (v * NT + tid) * 8;
        rz[v] = rx[v] = Raw8{b_u32x4{0u, 0u, 0u, 0u}, b_u32x4{0u, 0u, 0u, 0u}};
        if (col < a.d) {
            if (JOIN) rz[v] = load8<false>(a.z, base + col);
            rx[v] = load8<F32>(a.stream, base + col);
        }
    }
    float x[NV][8];
#pragma unroll
    for (int v = 0; v < NV; ++v) widen8<F32>(rx[v], x[v]);
    if constexpr (JOIN) {
        const float g = a.gate ? a.gate[row] : 1.0f;
        float r1 = 1.0f;
        if (a.w1) {
            float sum[1] = {0.f};
#pragma unroll
            for (int v = 0; v < NV; ++v) {
                float z[8];
                widen8<false>(rz[v], z);
#pragma unroll
                for (int c = 0; c < 8; ++c) sum[0] = __builtin_fmaf(z[c], z[c], sum[0]);
            }
            moe::workgroup_sums<NT>(sum, s_sum, half);
            r1 = inverse_rms(sum[0], a.d, a.eps);
        }
#pragma unroll
        for (int v = 0; v < NV; ++v) {
            const int col = (v * NT + tid) * 8;
            float z[8], w[8];
            widen8<false>(rz[v], z);
#pragma unroll
            for (int c = 0; c < 8; ++c) w[c] = 1.0f;
            if (a.w1 && col < a.d) weights8(a.w1, col, w);
#pragma unroll
            for (int c = 0; c < 8; ++c) x[v][c] = __builtin_fmaf(a.scale, x[v][c], g * (z[c] * r1 * w[c]));
            if (col < a.d) store8<F32>(a.out, base + col, x[v]);
        }
        if (!a.w2) return;
    }
    // the norm of out is taken of the values before they are rounded to the stream's type
    float sum[1] = {0.f};
#pragma unroll
    for (int v = 0; v < NV; ++v)
#pragma unroll
        for (int c = 0; c < 8; ++c) sum[0] = __builtin_fmaf(x[v][c], x[v][c], sum[0]);
    moe::workgroup_sums<NT>(sum, s_sum, half);
    const float r2 = inverse_rms(sum[0], a.d, a.eps);
#pragma unroll
    for (int v = 0; v < NV; ++v) {
        const int col = (v * NT + tid) * 8;
        if (col < a.d) {
            float w[8], o[8];
            weights8(a.w2, col, w);
#pragma unroll
            for (int c = 0; c < 8; ++c) o[c] = x[v][c] * r2 * w[c];
            store8<false>(a.next, base + col, o);
        }
    }
}

struct BackwardArgs {
    const void *d_out, *d_next;                // gradients that arrive at the stream (NULL = zero) and at the normalised rows (NULL = zero)
    const void *z, *out;                       // z: join only
    const float *w1, *gate, *w2;
    void *d_z, *d_stream;
    float* d_gate;
    float *part1, *part2;                      // sums over a workgroup's rows for w1 and w2, [workgroups][d]
    float scale, eps;
    int T, d;
};

// With n2 = out r2, n1 = z r1 (r = 1 / rms) and D the gradient of out:
//   D = d_out + r2 (d_next w2 - n2 mean(d_next w2 n2)),  d_stream = scale D,  d_w2 = sum_t d_next n2
//   d_gate = sum_c D n1 w1,  d_z = r1 gate (D w1 - n1 mean(D w1 n1)),  d_w1 = sum_t gate D n1
// Three sums over the columns of a row meet in one reduction (out^2, d_next w2 out, z^2), the fourth (D w1 z) in a second one.
// The sums over the tokens stay in registers while a workgroup walks its rows; four wavefronts per SIMD (without the bound on registers a workgroup of 256 had two or three: 137
// against 127 us).  8192 rows of 4096 with a float32 stream: 119 us, 5.1 TB/s, and 5 for the sums over the workgroups.
// Above 8192 columns two steps of 1024 threads do not fit the 128 registers that such a workgroup leaves each: the join's kernel spills 19 of them with a bf16 stream and 58 with float32
// (4096 rows of 16384: 202 us, 3.9 TB/s, and 326 us, 3.6 TB/s; the norm's does not spill: 94 and 138 us). Two steps of a wavefront with a float32 stream spill 9.
template <int NT, int NV, bool F32, bool JOIN>
__global__ __attribute__((amdgpu_waves_per_eu(4))) __launch_bounds__(NT == 64 ? 256 : NT)
void block_backward_kernel(BackwardArgs a) {
    constexpr int PER = NT == 64 ? 4 : 1;
    __shared__ float s_sum3[2 * 3 * (NT / 64)], s_sum1[2 * (NT / 64)];
    int half3 = 0, half1 = 0;
    const int tid = threadIdx.x % NT;
    float dw1[NV][8], dw2[NV][8];
#pragma unroll
    for (int v = 0; v < NV; ++v)
#pragma unroll
        for (int c = 0; c < 8; ++c) dw1[v][c] = dw2[v][c] = 0.f;
    const float by_d = 1.0f / (float)a.d;
    for (long long row = (long long)blockIdx.x * PER + (int)threadIdx.x / NT; row < a.T; row += (long long)gridDim.x * PER) {
        const size_t base = (size_t)row * a.d;
        Raw8 ro[NV], rn[NV], rg[NV], rz[NV];
#pragma unroll
        for (int v = 0; v < NV; ++v) {
            const int col = (v * NT + tid) * 8;
            ro[v] = rn[v] = rg[v] = rz[v] = Raw8{b_u32x4{0u, 0u, 0u, 0u}, b_u32x4{0u, 0u, 0u, 0u}};
            if (col < a.d) {
                if (a.w2) ro[v] = load8<F32>(a.out, base + col);
                if (a.w2) rn[v] = load8<false>(a.d_next, base + col);
                if (JOIN) rz[v] = load8<false>(a.z, base + col);
                if (a.d_out) rg[v] = load8<F32>(a.d_out, base + col);
            }
        }
        const float g = JOIN && a.gate ? a.gate[row] : 1.0f;
        float sum[3] = {0.f, 0.f, 0.f};
#pragma unroll
        for (int v = 0; v < NV; ++v) {
            const int col = (v * NT + tid) * 8;
            if (a.w2 && col < a.d) {
                float o[8], n[8], w[8];
                widen8<F32>(ro[v], o);
                widen8<false>(rn[v], n);
                weights8(a.w2, col, w);
#pragma unroll
                for (int c = 0; c < 8; ++c) {
                    sum[0] = __builtin_fmaf(o[c], o[c], sum[0]);
                    sum[1] = __builtin_fmaf(n[c] * w[c], o[c], sum[1]);
                }
            }
            if (JOIN) {
                float z[8];
                widen8<false>(rz[v], z);
#pragma unroll
                for (int c = 0; c < 8; ++c) sum[2] = __builtin_fmaf(z[c], z[c], sum[2]);
            }
        }
        moe::workgroup_sums<NT>(sum, s_sum3, half3);
        const float r2 = inverse_rms(sum[0], a.d, a.eps), r1 = JOIN && a.w1 ? inverse_rms(sum[2], a.d, a.eps) : 1.0f;
        // (an infinitely long row, r = 0, has no gradient through its norm, whatever its product with the gradient came to: that may have passed fp32 as well)
        const float back2 = r2 == 0.0f ? 0.0f : sum[1] * by_d * r2 * r2;
        float D[NV][8], q[1] = {0.f};
#pragma unroll
        for (int v = 0; v < NV; ++v) {
            const int col = (v * NT + tid) * 8;
            widen8<F32>(rg[v], D[v]);
            if (col < a.d) {
                if (a.w2) {
                    float o[8], n[8], w[8];
                    widen8<F32>(ro[v], o);
                    widen8<false>(rn[v], n);
                    weights8(a.w2, col, w);
#pragma unroll
                    for (int c = 0; c < 8; ++c) {
                        D[v][c] = __builtin_fmaf(r2, n[c] * w[c] - o[c] * back2, D[v][c]);
                        dw2[v][c] = __builtin_fmaf(n[c], o[c] * r2, dw2[v][c]);
                    }
                }
                float ds[8];
#pragma unroll
                for (int c = 0; c < 8; ++c) ds[c] = a.scale * D[v][c];
                store8<F32>(a.d_stream, base + col, ds);
                if (JOIN) {
                    float z[8], w[8];
                    widen8<false>(rz[v], z);
#pragma unroll
                    for (int c = 0; c < 8; ++c) w[c] = 1.0f;
                    if (a.w1) weights8(a.w1, col, w);
#pragma unroll
                    for (int c = 0; c < 8; ++c) {
                        dw1[v][c] = __builtin_fmaf(g * D[v][c], z[c] * r1, dw1[v][c]);
                        D[v][c] *= w[c];
                        q[0] = __builtin_fmaf(D[v][c], z[c], q[0]);
                    }
                }
            }
        }
        if constexpr (JOIN) {
            if (a.w1 || a.d_gate) moe::workgroup_sums<NT>(q, s_sum1, half1);
            if (r1 == 0.0f) q[0] = 0.0f;
            if (a.d_gate && tid == 0) a.d_gate[row] = q[0] * r1;
            const float back1 = a.w1 ? q[0] * by_d * r1 * r1 : 0.0f, rg1 = r1 * g;
#pragma unroll
            for (int v = 0; v < NV; ++v) {
                const int col = (v * NT + tid) * 8;
                if (col < a.d) {
                    float z[8], o[8];
                    widen8<false>(rz[v], z);
#pragma unroll
                    for (int c = 0; c < 8; ++c) o[c] = rg1 * (D[v][c] - z[c] * back1);
                    store8<false>(a.d_z, base + col, o);
                }
            }
        }
    }
    auto keep = [&](float (&dw)[NV][8], float* part) __attribute__((always_inline)) {
        if constexpr (PER == 1) {
#pragma unroll
            for (int v = 0; v < NV; ++v) {
                const int col = (v * NT + tid) * 8;
                if (col < a.d) store8<true>(part, (size_t)blockIdx.x * a.d + col, dw[v]);
            }
        } else {
            __shared__ float s_dw[PER][NV * NT * 8];
            __syncthreads();
#pragma unroll
            for (int v = 0; v < NV; ++v)
#pragma unroll
                for (int c = 0; c < 8; ++c) s_dw[threadIdx.x / NT][(v * 8 + c) * NT + tid] = dw[v][c];
            __syncthreads();
            for (int i = threadIdx.x; i < NV * NT * 8; i += PER * NT) {
                const int t = i % NT, vc = i / NT, col = (vc / 8 * NT + t) * 8 + vc % 8;
                if (col < a.d) part[(size_t)blockIdx.x * a.d + col] = (s_dw[0][i] + s_dw[1][i]) + (s_dw[2][i] + s_dw[3][i]);
            }
        }
    };
    if (a.w2) keep(dw2, a.part2);
    if (JOIN && a.w1) keep(dw1, a.part1);
}

// out[c] = sum of part[0 .. parts - 1][c] in that order within 16 strides; blockIdx.y picks the vector
__global__ __launch_bounds__(1024)
void block_columns_kernel(const float* part_a, float* out_a, const float* part_b, float* out_b, int parts, int d) {
    __shared__ float s[16][64];
    const float* const part = blockIdx.y ? part_b : part_a;
    float* const out = blockIdx.y ? out_b : out_a;
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6, col = blockIdx.x * 64 + lane;
    float t = 0.f;
    if (col < d) {
#pragma unroll 8
        for (int p = wave; p < parts; p += 16) t += part[(size_t)p * d + col];
    }
    s[wave][lane] = t;
    __syncthreads();
    if (wave == 0 && col < d) {
        float sum = s[0][lane];
#pragma unroll
        for (int w = 1; w < 16; ++w) sum += s[w][lane];
        out[col] = sum;
    }
}

constexpr int MOST_ROWS = 1 << 21;               // per launch, whose threads are counted in 32 bits
template <int NT, int NV, bool F32, bool JOIN> moe_status forward(ForwardArgs a, hipStream_t s) {
    constexpr int PER = NT == 64 ? 4 : 1;
    moe::LaunchScope k(JOIN ? "block_join_kernel" : "block_norm_kernel", s);
    for (long long first = 0; first < a.T; first += MOST_ROWS) {
        a.first = (int)first;
        const int rows = (int)std::min<long long>(a.T - first, MOST_ROWS);
        hipLaunchKernelGGL((block_forward_kernel<NT, NV, F32, JOIN>), dim3((unsigned)((rows - 1) / PER + 1)), dim3(NT == 64 ? 256 : NT), 0, s, a);
    }
    return k.done();
}
template <bool F32, bool JOIN> moe_status forward_of(const ForwardArgs& a, hipStream_t s) {
    // 8 columns per thread; two steps of 256 threads where more than a third of 512 would have none (T 8192: d 2304 30 us against 34, d 4096 48 against 47, its float32 stream 80
    // against 74; T 64, d 4096: 8.6 against 6.5; d 8192: 512 threads 104, 1024 threads 100)
    if (a.d <= 512) return forward<64, 1, F32, JOIN>(a, s);
    if (a.d <= 1024) return forward<64, 2, F32, JOIN>(a, s);
    if (a.d <= 2048) return forward<256, 1, F32, JOIN>(a, s);
    if (a.d <= 2736) return forward<256, 2, F32, JOIN>(a, s);
    if (a.d <= 4096) return forward<512, 1, F32, JOIN>(a, s);
    if (a.d <= 8192) return forward<1024, 1, F32, JOIN>(a, s);
    return forward<1024, 2, F32, JOIN>(a, s);
}

template <int NT, int NV, bool F32, bool JOIN> moe_status backward(BackwardArgs a, float* d_w1, float* d_w2, float* work, hipStream_t s) {
    constexpr int PER = NT == 64 ? 4 : 1;
    // the workgroups that the chip holds at 1024 threads per compute unit, each walking its share of the rows
    const int parts = a.T == 0 ? 0 : std::min({(a.T - 1) / PER + 1, BLOCK_MAX_PARTS, moe::compute_units() * (1024 / (NT == 64 ? 256 : NT))});
    a.part2 = work;
    a.part1 = work + (size_t)(a.w2 ? parts : 0) * a.d;
    if (parts > 0) {
        moe::LaunchScope k(JOIN ? "block_join_backward_kernel" : "block_norm_backward_kernel", s);
        hipLaunchKernelGGL((block_backward_kernel<NT, NV, F32, JOIN>), dim3(parts), dim3(NT == 64 ? 256 : NT), 0, s, a);
        if (const moe_status st = k.done()) return st;
    }
    const int vectors = (a.w2 ? 1 : 0) + (a.w1 ? 1 : 0);
    if (vectors == 0) return MOE_OK;
    moe::LaunchScope k("block_columns_kernel", s);
    hipLaunchKernelGGL(block_columns_kernel, dim3((a.d + 63) / 64, vectors), dim3(1024), 0, s, a.w2 ? a.part2 : a.part1, a.w2 ? d_w2 : d_w1, a.part1, d_w1, parts, a.d);
    return k.done();
}
template <bool F32, bool JOIN> moe_status backward_of(const BackwardArgs& a, float* d_w1, float* d_w2, float* work, hipStream_t s) {
    // as in the forward pass; a bf16 stream leaves enough registers for two steps of half the threads, which many rows fill better (T 8192, d 7168: 155 us against 165, in float32
    // 224 against 216; T 64: 17 against 11)
    if (a.d <= 512) return backward<64, 1, F32, JOIN>(a, d_w1, d_w2, work, s);
    if (a.d <= 1024) return backward<64, 2, F32, JOIN>(a, d_w1, d_w2, work, s);
    if (a.d <= 2048) return backward<256, 1, F32, JOIN>(a, d_w1, d_w2, work, s);
    if (a.d <= 2736) return backward<256, 2, F32, JOIN>(a, d_w1, d_w2, work, s);
    if (a.d <= 4096) return backward<512, 1, F32, JOIN>(a, d_w1, d_w2, work, s);
    if constexpr (!F32) {
        if (a.d <= 8192 && a.T > 1024) return backward<512, 2, F32, JOIN>(a, d_w1, d_w2, work, s);
    }
    if (a.d <= 8192) return backward<1024, 1, F32, JOIN>(a, d_w1, d_w2, work, s);
    return backward<1024, 2, F32, JOIN>(a, d_w1, d_w2, work, s);
}

bool misaligned(std::initializer_list<const void*> ps) {
    uintptr_t all = 0;
    for (const void* p : ps) all |= (uintptr_t)p;
    return (all & 15) != 0;
}
// sizes, the type and the numbers that every call here has
moe_status checked(int T, int d, int stream_type, float scale, float eps) {
    if (T < 0 || d < 1 || (stream_type != MOE_T_BF16 && stream_type != MOE_T_F32)) return MOE_ERR_INVALID_ARG;
    if (!(eps > 0.0f) || !(eps < __builtin_inff()) || !(__builtin_fabsf(scale) < __builtin_inff())) return MOE_ERR_INVALID_ARG;
    if (d % 8 != 0 || d > BLOCK_MAX_COLUMNS) return MOE_ERR_UNSUPPORTED_SHAPE;
    return MOE_OK;
}

}  // namespace

extern "C" size_t moe_block_backward_workspace_bytes(int T, int d) {
    if (T < 0 || d < 1) return 0;
    return (size_t)2 * std::max(1, std::min(T, BLOCK_MAX_PARTS)) * d * sizeof(float);
}

extern "C" moe_status moe_block_norm(const void* x, int stream_type, const float* weight, float eps, int T, int d, void* out, void* hip_stream) {
    if (const moe_status st = checked(T, d, stream_type, 1.0f, eps)) return st;
    if (T == 0) return MOE_OK;
    if (!x || !weight || !out || misaligned({x, weight, out})) return MOE_ERR_INVALID_ARG;
    const ForwardArgs a = {nullptr, x, nullptr, nullptr, weight, nullptr, out, 1.0f, eps, T, d, 0};
    return stream_type == MOE_T_F32 ? forward_of<true, false>(a, (hipStream_t)hip_stream) : forward_of<false, false>(a, (hipStream_t)hip_stream);
}

extern "C" moe_status moe_block_join(const void* z, const void* stream, int stream_type, const float* post_weight, const float* gate,
                                     const float* next_weight, float scale, float eps, int T, int d, void* out, void* next, void* hip_stream) {
    if (const moe_status st = checked(T, d, stream_type, scale, eps)) return st;
    if ((next_weight == nullptr) != (next == nullptr) && T > 0) return MOE_ERR_INVALID_ARG;
    if (T == 0) return MOE_OK;
    if (!z || !stream || !out || misaligned({z, stream, post_weight, next_weight, out, next})) return MOE_ERR_INVALID_ARG;
    const ForwardArgs a = {z, stream, post_weight, gate, next_weight, out, next, scale, eps, T, d, 0};
    return stream_type == MOE_T_F32 ? forward_of<true, true>(a, (hipStream_t)hip_stream) : forward_of<false, true>(a, (hipStream_t)hip_stream);
}

extern "C" moe_status moe_block_norm_backward(const void* d_out, const void* x, int stream_type, const float* weight, const void* d_stream, float eps,
                                              int T, int d, void* d_x, float* d_weight, void* workspace, size_t workspace_bytes, void* hip_stream) {
    if (const moe_status st = checked(T, d, stream_type, 1.0f, eps)) return st;
    if (!weight || !d_weight || (T > 0 && (!d_out || !x || !d_x))) return MOE_ERR_INVALID_ARG;
    if (misaligned({d_out, x, weight, d_stream, d_x, d_weight, workspace})) return MOE_ERR_INVALID_ARG;
    if (!workspace || workspace_bytes < moe_block_backward_workspace_bytes(T, d)) return MOE_ERR_WORKSPACE;
    const BackwardArgs a = {d_stream, d_out, nullptr, x, nullptr, nullptr, weight, nullptr, d_x, nullptr, nullptr, nullptr, 1.0f, eps, T, d};
    hipStream_t s = (hipStream_t)hip_stream;
    return stream_type == MOE_T_F32 ? backward_of<true, false>(a, nullptr, d_weight, (float*)workspace, s)
                                    : backward_of<false, false>(a, nullptr, d_weight, (float*)workspace, s);
}

extern "C" moe_status moe_block_join_backward(const void* d_out, const void* d_next, const void* z, const void* out, int stream_type,
                                              const float* post_weight, const float* gate, const float* next_weight, float scale, float eps, int T, int d,
                                              void* d_z, void* d_stream, float* d_gate, float* d_post_weight, float* d_next_weight,
                                              void* workspace, size_t workspace_bytes, void* hip_stream) {
    if (const moe_status st = checked(T, d, stream_type, scale, eps)) return st;
    // a gradient is written for each input that is there, and for no other
    if ((post_weight == nullptr) != (d_post_weight == nullptr) || (next_weight == nullptr) != (d_next_weight == nullptr)) return MOE_ERR_INVALID_ARG;
    if (T > 0 && ((gate == nullptr) != (d_gate == nullptr) || !z || !d_z || !d_stream)) return MOE_ERR_INVALID_ARG;
    if (T > 0 && ((next_weight == nullptr) != (d_next == nullptr) || (next_weight && !out) || (!d_out && !d_next))) return MOE_ERR_INVALID_ARG;
    if (misaligned({d_out, d_next, z, out, post_weight, next_weight, d_z, d_stream, d_post_weight, d_next_weight, workspace})) return MOE_ERR_INVALID_ARG;
    if (!workspace || workspace_bytes < moe_block_backward_workspace_bytes(T, d)) return MOE_ERR_WORKSPACE;
    const BackwardArgs a = {d_out, d_next, z, out, post_weight, gate, next_weight, d_z, d_stream, d_gate, nullptr, nullptr, scale, eps, T, d};
    hipStream_t s = (hipStream_t)hip_stream;
    return stream_type == MOE_T_F32 ? backward_of<true, true>(a, d_post_weight, d_next_weight, (float*)workspace, s)
                                    : backward_of<false, true>(a, d_post_weight, d_next_weight, (float*)workspace, s);
}
