// moe_combine_topk_sum: the last step of dispatch -> compute -> combine (Section 2.1): once the expert results are
// back at the rank that owns the tokens, every token's output is the router-weighted sum of the results of its topk
// experts.  HBM bound: topk rows of d bf16 values are read per token and one is written, each exactly once.
// Workgroups of 256 threads each walk a share of the tokens for one 2048-column stretch; a thread owns 8 consecutive
// columns (16 bytes), issues the loads of all its slots before it adds (the bytes in flight per thread are what fills
// the memory pipeline) and accumulates in fp32 in slot order.  Result rows are read once by the whole grid, so the loads
// are non-temporal.
#include "lanes.hpp"
#include <algorithm>

namespace {

typedef __attribute__((ext_vector_type(8))) __bf16 cb_bf16x8;
typedef __attribute__((ext_vector_type(4))) unsigned int cb_u32x4;
constexpr int CB_THREADS = 256;
constexpr int CB_COLS = CB_THREADS * 8;        // columns one workgroup covers

template <int TOPK>                            // 0 = any topk (a loop), else unrolled
__global__ __launch_bounds__(CB_THREADS)
void combine_kernel(const __bf16* __restrict__ y, const int32_t* __restrict__ row_of, const float* __restrict__ gate,
                    int T, int topk, int d, int R, __bf16* __restrict__ out) {
    const int col = blockIdx.y * CB_COLS + threadIdx.x * 8;
    if (col >= d) return;
    if constexpr (TOPK != 0) {
        // A workgroup walks tokens blockIdx.x, blockIdx.x + gridDim.x, ...; the row numbers and weights of the next token
        // are fetched while the rows of the current one are in flight (otherwise every token costs two dependent
        // round trips to memory).
        int rows[TOPK], nrows[TOPK];
        float w[TOPK], nw[TOPK];
        auto fetch_index = [&](int t, int (&r)[TOPK], float (&g)[TOPK]) __attribute__((always_inline)) {
#pragma unroll
            for (int j = 0; j < TOPK; ++j) {
                r[j] = row_of[(size_t)t * TOPK + j];
                g[j] = gate ? gate[(size_t)t * TOPK + j] : 1.0f;
            }
        };
        int t = blockIdx.x;
        if (t < T) fetch_index(t, rows, w);
        while (t < T) {
            cb_u32x4 v[TOPK];
#pragma unroll
            for (int j = 0; j < TOPK; ++j) {
                const bool live = rows[j] >= 0 && rows[j] < R;                // a dropped assignment contributes nothing
                if (!live) w[j] = 0.0f;
                v[j] = cb_u32x4{0u, 0u, 0u, 0u};
                if (live) v[j] = __builtin_nontemporal_load(reinterpret_cast<const cb_u32x4*>(y + (size_t)rows[j] * d + col));
            }
            const int tn = t + gridDim.x;
            if (tn < T) fetch_index(tn, nrows, nw);
            float acc[8];
#pragma unroll
            for (int c = 0; c < 8; ++c) acc[c] = 0.f;
#pragma unroll
            for (int j = 0; j < TOPK; ++j) {
                const cb_bf16x8 b = __builtin_bit_cast(cb_bf16x8, v[j]);
#pragma unroll
                for (int c = 0; c < 8; ++c) acc[c] = __builtin_fmaf(w[j], (float)b[c], acc[c]);
            }
            cb_bf16x8 o;
#pragma unroll
            for (int c = 0; c < 8; ++c) o[c] = (__bf16)acc[c];
            __builtin_nontemporal_store(__builtin_bit_cast(cb_u32x4, o), reinterpret_cast<cb_u32x4*>(out + (size_t)t * d + col));
            t = tn;
#pragma unroll
            for (int j = 0; j < TOPK; ++j) { rows[j] = nrows[j]; w[j] = nw[j]; }
        }
    } else {
        for (int t = blockIdx.x; t < T; t += gridDim.x) {
            const int32_t* rows = row_of + (size_t)t * topk;
            const float* g = gate ? gate + (size_t)t * topk : nullptr;
            float acc[8];
#pragma unroll
            for (int c = 0; c < 8; ++c) acc[c] = 0.f;
            for (int j = 0; j < topk; ++j) {
                const int r = rows[j];
                if (r < 0 || r >= R) continue;
                const float w = g ? g[j] : 1.0f;
                const cb_bf16x8 b = __builtin_bit_cast(cb_bf16x8, __builtin_nontemporal_load(reinterpret_cast<const cb_u32x4*>(y + (size_t)r * d + col)));
#pragma unroll
                for (int c = 0; c < 8; ++c) acc[c] = __builtin_fmaf(w, (float)b[c], acc[c]);
            }
            cb_bf16x8 o;
#pragma unroll
            for (int c = 0; c < 8; ++c) o[c] = (__bf16)acc[c];
            __builtin_nontemporal_store(__builtin_bit_cast(cb_u32x4, o), reinterpret_cast<cb_u32x4*>(out + (size_t)t * d + col));
        }
    }
}

}  // namespace

extern "C" moe_status moe_combine_topk_sum(const void* y, const int32_t* row_of, const float* gate, int T, int topk, int d, int R,
                                           void* out, void* hip_stream) {
    if (T < 0 || topk < 1 || d < 1 || R < 0) return MOE_ERR_INVALID_ARG;
    if (d % 8 != 0 || T > 0x7FFFFFFF / topk) return MOE_ERR_UNSUPPORTED_SHAPE;
    if (T == 0) return MOE_OK;
    if (!row_of || !out || (R > 0 && !y)) return MOE_ERR_INVALID_ARG;
    if ((((uintptr_t)y | (uintptr_t)out) & 15) != 0) return MOE_ERR_INVALID_ARG;         // rows are moved in 16-byte pieces
    hipStream_t s = (hipStream_t)hip_stream;
    const unsigned ycols = (unsigned)((d + CB_COLS - 1) / CB_COLS);
    if (ycols > 65535u) return MOE_ERR_UNSUPPORTED_SHAPE;
    int cus = 256;
    {
        int dev = 0;
        if (hipGetDevice(&dev) != hipSuccess || hipDeviceGetAttribute(&cus, hipDeviceAttributeMultiprocessorCount, dev) != hipSuccess || cus <= 0) cus = 256;
    }
    // about eight workgroups per compute unit, each walking its share of the tokens
    const unsigned per_col = (unsigned)std::max(1, cus * 8 / (int)ycols);
    const dim3 grid(std::min<unsigned>((unsigned)T, per_col), ycols);
    moe::LaunchScope k("combine_kernel", s);
    const __bf16* yy = (const __bf16*)y;
    __bf16* oo = (__bf16*)out;
    switch (topk) {
        case 1: hipLaunchKernelGGL(combine_kernel<1>, grid, dim3(CB_THREADS), 0, s, yy, row_of, gate, T, topk, d, R, oo); break;
        case 2: hipLaunchKernelGGL(combine_kernel<2>, grid, dim3(CB_THREADS), 0, s, yy, row_of, gate, T, topk, d, R, oo); break;
        case 4: hipLaunchKernelGGL(combine_kernel<4>, grid, dim3(CB_THREADS), 0, s, yy, row_of, gate, T, topk, d, R, oo); break;
        case 6: hipLaunchKernelGGL(combine_kernel<6>, grid, dim3(CB_THREADS), 0, s, yy, row_of, gate, T, topk, d, R, oo); break;
        case 8: hipLaunchKernelGGL(combine_kernel<8>, grid, dim3(CB_THREADS), 0, s, yy, row_of, gate, T, topk, d, R, oo); break;
        default: hipLaunchKernelGGL(combine_kernel<0>, grid, dim3(CB_THREADS), 0, s, yy, row_of, gate, T, topk, d, R, oo); break;
    }
    return k.done();
}

// ---------------------------------------------------------------------------------- gradients of the combine
// moe_combine_topk_sum_backward: d_y[row_of[t][j]] += gate[t][j] d_out[t], d_gate[t][j] = d_out[t] . y[row_of[t][j]].
// HBM bound: d_out is read once, y read and d_y written once.  A workgroup takes a token: its threads hold d_out[t] (8 columns a
// step) and walk the token's rows, whose loads go out together.  Nearly always a row belongs to one assignment and is written right here.  A row that
// several assignments name (counted beforehand, in small calls by every workgroup for itself) is left to the workgroups behind the tokens', which add them up in the order of the assignments, and so
// is a row that none names, whose gradient is zero.  8192 tokens to 8 rows of 4096: 228 us, 5.0 TB/s, and 9 for the counts; two steps of 256 threads per row (512 threads of one
// step: 235; 4 rows in flight per token, 8: 229; d 7168: 217 with 512 threads, 228 with 1024).
namespace {

constexpr int CBB_MAX_COLUMNS = 16384;

// uses[r] = number of assignments that name row r
__global__ __launch_bounds__(256)
void combine_clear_kernel(int32_t* __restrict__ uses, int R) {
    for (long long i = (long long)blockIdx.x * 256 + threadIdx.x; i < R; i += (long long)gridDim.x * 256) uses[i] = 0;
}
__global__ __launch_bounds__(256)
void combine_count_kernel(const int32_t* __restrict__ row_of, int n, int R, int32_t* __restrict__ uses) {
    for (long long i = (long long)blockIdx.x * 256 + threadIdx.x; i < n; i += (long long)gridDim.x * 256) {
        const int r = row_of[i];
        if ((unsigned)r < (unsigned)R) atomicAdd(uses + r, 1);
    }
}

// by one workgroup, in its LDS
template <int THREADS>
__device__ __forceinline__ void count_rows(const int32_t* __restrict__ row_of, int n, int R, int32_t* s_uses) {
    for (int i = threadIdx.x; i < n; i += THREADS) {
        const int r = row_of[i];
        if ((unsigned)r < (unsigned)R) atomicAdd(s_uses + r, 1);
    }
}
// Few rows and assignments: every workgroup counts for itself, so that the call is one launch (777 tokens to 2 rows: 10.5 us a call, with a launch for the counts 14.4).
constexpr int COUNT_ROWS = 4096;

struct CombineBackwardArgs {
    const __bf16 *d_out, *y;
    const int32_t* row_of;
    const float* gate;
    const int32_t* uses;
    __bf16* d_y;
    float* d_gate;
    int T, topk, d, R;
    int first, tokens;                         // of this launch
};

__device__ __forceinline__ void cb_widen(cb_u32x4 r, float (&v)[8]) {
    const cb_bf16x8 b = __builtin_bit_cast(cb_bf16x8, r);
#pragma unroll
    for (int c = 0; c < 8; ++c) v[c] = (float)b[c];
}
__device__ __forceinline__ cb_u32x4 cb_scaled(const float (&v)[8], float w) {
    cb_bf16x8 o;
#pragma unroll
    for (int c = 0; c < 8; ++c) o[c] = (__bf16)(w * v[c]);
    return __builtin_bit_cast(cb_u32x4, o);
}

// Rows that no assignment names, or several do, by workgroup `first` of `step`: it looks at its share of the rows, a row per thread (at most), and does those
// it finds one after the other (777 tokens to 2 rows of 2048, 1 % unnamed: 10 us, with 256 rows per workgroup 21 us; 65536 rows of 4096 looked at one by one: 28 us more).
// The several are found by going through all assignments, a workgroup's width at a time, and added in their order.
template <int THREADS>
__device__ __forceinline__ void combine_backward_rest(const CombineBackwardArgs& a, const int32_t* uses_of, int first, int step) {
    constexpr int W = THREADS / 64;
    __shared__ unsigned long long s_hit[W], s_odd[W];
    const int wave = threadIdx.x >> 6;
    const long long n = (long long)a.T * a.topk;
    const int share = min(THREADS, (a.R - 1) / step + 1);
    for (long long r0 = (long long)first * share; r0 < a.R; r0 += (long long)step * share) {
        const unsigned long long odd = __ballot((int)threadIdx.x < share && r0 + threadIdx.x < a.R && uses_of[r0 + threadIdx.x] != 1);
        __syncthreads();
        if ((threadIdx.x & 63) == 0) s_odd[wave] = odd;
        __syncthreads();
        for (int q = 0; q < THREADS; ++q) {
            if (s_odd[q >> 6] == 0) { q |= 63; continue; }
            if (!((s_odd[q >> 6] >> (q & 63)) & 1)) continue;
            const long long r = r0 + q;
            const int uses = uses_of[r];                                        // (the same for the whole workgroup)
            if (uses == 0) {
                for (int col = threadIdx.x * 8; col < a.d; col += THREADS * 8) *reinterpret_cast<cb_u32x4*>(a.d_y + (size_t)r * a.d + col) = cb_u32x4{0u, 0u, 0u, 0u};
                continue;
            }
            for (int c0 = 0; c0 < a.d; c0 += THREADS * 8) {
                const int col = c0 + threadIdx.x * 8;
                float sum[8];
#pragma unroll
                for (int c = 0; c < 8; ++c) sum[c] = 0.0f;
                int left = uses;
                for (long long i0 = 0; i0 < n && left > 0; i0 += THREADS) {
                    const long long i = i0 + threadIdx.x;
                    const unsigned long long hit = __ballot(i < n && a.row_of[i < n ? i : 0] == r);
                    if ((threadIdx.x & 63) == 0) s_hit[wave] = hit;
                    __syncthreads();
                    for (int w = 0; w < W; ++w) {
                        unsigned long long h = s_hit[w];
                        while (h) {
                            const int at = (int)i0 + w * 64 + __builtin_ctzll(h);
                            h &= h - 1;
                            --left;
                            if (col < a.d) {
                                const float g = a.gate ? a.gate[at] : 1.0f;
                                float v[8];
                                cb_widen(*reinterpret_cast<const cb_u32x4*>(a.d_out + (size_t)(at / a.topk) * a.d + col), v);
#pragma unroll
                                for (int c = 0; c < 8; ++c) sum[c] = __builtin_fmaf(g, v[c], sum[c]);
                            }
                        }
                    }
                    __syncthreads();
                }
                if (col < a.d) *reinterpret_cast<cb_u32x4*>(a.d_y + (size_t)r * a.d + col) = cb_scaled(sum, 1.0f);
            }
        }
    }
}

// NT threads per token, NV steps of NT * 8 columns, J rows of y in flight at once; COUNT: the rows' counts are made here, in LDS (R integers)
template <int NT, int NV, int J, bool COUNT>
__global__ __launch_bounds__(NT == 64 ? 256 : NT)
void combine_backward_kernel(CombineBackwardArgs a) {
    constexpr int PER = NT == 64 ? 4 : 1;
    __shared__ float s_sum[2 * J * (NT / 64)];
    extern __shared__ int32_t s_uses[];
    const int32_t* uses = a.uses;
    if constexpr (COUNT) {
        constexpr int THREADS = NT == 64 ? 256 : NT;
        for (int r = threadIdx.x; r < a.R; r += THREADS) s_uses[r] = 0;
        __syncthreads();
        count_rows<THREADS>(a.row_of, a.T * a.topk, a.R, s_uses);
        __syncthreads();
        uses = s_uses;
    }
    int half = 0;
    const int tid = threadIdx.x % NT;
    const int token_blocks = a.tokens == 0 ? 0 : (a.tokens - 1) / PER + 1;
    if ((int)blockIdx.x >= token_blocks) {                                // the workgroups behind the tokens'
        combine_backward_rest<(NT == 64 ? 256 : NT)>(a, uses, (int)blockIdx.x - token_blocks, (int)gridDim.x - token_blocks);
        return;
    }
    const long long t = a.first + (long long)blockIdx.x * PER + (int)threadIdx.x / NT;
    if (t >= a.T) return;                                                 // (a whole wavefront, which meets no barrier if NT is 64)
    cb_u32x4 raw[NV];
#pragma unroll
    for (int v = 0; v < NV; ++v) {
        const int col = (v * NT + tid) * 8;
        raw[v] = cb_u32x4{0u, 0u, 0u, 0u};
        if (col < a.d) raw[v] = *reinterpret_cast<const cb_u32x4*>(a.d_out + (size_t)t * a.d + col);
    }
    for (int j0 = 0; j0 < a.topk; j0 += J) {
        int row[J];
        bool alone[J];
        float w[J], dot[J];
        cb_u32x4 y[J][NV];
#pragma unroll
        for (int j = 0; j < J; ++j) {
            const size_t at = (size_t)t * a.topk + min(j0 + j, a.topk - 1);
            row[j] = j0 + j < a.topk ? a.row_of[at] : -1;
            if ((unsigned)row[j] >= (unsigned)a.R) row[j] = -1;
            w[j] = a.gate && row[j] >= 0 ? a.gate[at] : 1.0f;
            alone[j] = row[j] >= 0 && uses[row[j]] == 1;
            dot[j] = 0.0f;
#pragma unroll
            for (int v = 0; v < NV; ++v) {
                const int col = (v * NT + tid) * 8;
                y[j][v] = cb_u32x4{0u, 0u, 0u, 0u};
                if (a.d_gate && row[j] >= 0 && col < a.d) y[j][v] = __builtin_nontemporal_load(reinterpret_cast<const cb_u32x4*>(a.y + (size_t)row[j] * a.d + col));
            }
        }
#pragma unroll
        for (int v = 0; v < NV; ++v) {
            const int col = (v * NT + tid) * 8;
            float g[8];
            cb_widen(raw[v], g);
#pragma unroll
            for (int j = 0; j < J; ++j) {
                float b[8];
                cb_widen(y[j][v], b);
#pragma unroll
                for (int c = 0; c < 8; ++c) dot[j] = __builtin_fmaf(g[c], b[c], dot[j]);
                if (alone[j] && col < a.d)
                    __builtin_nontemporal_store(cb_scaled(g, w[j]), reinterpret_cast<cb_u32x4*>(a.d_y + (size_t)row[j] * a.d + col));
            }
        }
        if (a.d_gate) {
            moe::workgroup_sums<NT>(dot, s_sum, half);
            if (tid < J && j0 + tid < a.topk) {
                float mine = 0.0f;
#pragma unroll
                for (int j = 0; j < J; ++j) mine = tid == j && row[j] >= 0 ? dot[j] : mine;      // a dropped assignment's weight has no effect
                a.d_gate[(size_t)t * a.topk + j0 + tid] = mine;
            }
        }
    }
}

constexpr int MOST_TOKENS = 1 << 21;              // per launch, whose threads are counted in 32 bits
template <int NT, int NV, int J> void launch_combine_backward(CombineBackwardArgs a, bool count, hipStream_t s) {
    constexpr int PER = NT == 64 ? 4 : 1;
    long long first = 0;
    do {
        a.first = (int)first;
        a.tokens = (int)std::min<long long>(a.T - first, MOST_TOKENS);
        const int token_blocks = a.tokens == 0 ? 0 : (a.tokens - 1) / PER + 1, rest_blocks = first + a.tokens == a.T ? std::min(a.R, moe::compute_units()) : 0;
        const dim3 grid((unsigned)token_blocks + (unsigned)rest_blocks), block(NT == 64 ? 256 : NT);
        if (count) hipLaunchKernelGGL((combine_backward_kernel<NT, NV, J, true>), grid, block, a.R * (int)sizeof(int32_t), s, a);
        else hipLaunchKernelGGL((combine_backward_kernel<NT, NV, J, false>), grid, block, 0, s, a);
        first += MOST_TOKENS;
    } while (first < a.T);
}
template <int NT, int NV> void launch_combine_backward(const CombineBackwardArgs& a, bool count, hipStream_t s) {
    if (a.topk == 1) launch_combine_backward<NT, NV, 1>(a, count, s);
    else if (a.topk == 2) launch_combine_backward<NT, NV, 2>(a, count, s);
    else launch_combine_backward<NT, NV, 4>(a, count, s);
}

}  // namespace

extern "C" size_t moe_combine_backward_workspace_bytes(int R) { return R < 0 ? 0 : (((size_t)R * sizeof(int32_t)) + 255) & ~(size_t)255; }

extern "C" moe_status moe_combine_topk_sum_backward(const void* d_out, const void* y, const int32_t* row_of, const float* gate, int T, int topk, int d, int R,
                                                    void* d_y, float* d_gate, void* workspace, size_t workspace_bytes, void* hip_stream) {
    if (T < 0 || topk < 1 || d < 1 || R < 0) return MOE_ERR_INVALID_ARG;
    if (d % 8 != 0 || d > CBB_MAX_COLUMNS || T > 0x7FFFFFFF / topk) return MOE_ERR_UNSUPPORTED_SHAPE;
    if ((T > 0 && (!d_out || !row_of || (gate && !d_gate))) || (R > 0 && (!y || !d_y)) || (!gate && d_gate)) return MOE_ERR_INVALID_ARG;
    if ((((uintptr_t)d_out | (uintptr_t)y | (uintptr_t)d_y | (uintptr_t)workspace) & 15) != 0) return MOE_ERR_INVALID_ARG;
    if (R > 0 && (!workspace || workspace_bytes < moe_combine_backward_workspace_bytes(R))) return MOE_ERR_WORKSPACE;
    hipStream_t s = (hipStream_t)hip_stream;
    const int cus = moe::compute_units(), n = T * topk;
    CombineBackwardArgs a = {(const __bf16*)d_out, (const __bf16*)y, row_of, gate, (const int32_t*)workspace, (__bf16*)d_y, d_gate, T, topk, d, R, 0, 0};
    const auto blocks = [&](int items) { return dim3((unsigned)std::min((items - 1) / 256 + 1, cus * 8)); };
    const bool count_here = R <= COUNT_ROWS && n <= COUNT_ROWS;
    if (R > 0 && !count_here) {
        moe::LaunchScope k("combine_count_kernel", s);
        hipLaunchKernelGGL(combine_clear_kernel, blocks(R), dim3(256), 0, s, (int32_t*)workspace, R);
        if (n > 0) hipLaunchKernelGGL(combine_count_kernel, blocks(n), dim3(256), 0, s, row_of, n, R, (int32_t*)workspace);
        if (const moe_status st = k.done()) return st;
    }
    if (T > 0 || R > 0) {
        moe::LaunchScope k("combine_backward_kernel", s);
        if (d <= 512) launch_combine_backward<64, 1>(a, count_here, s);
        else if (d <= 1024) launch_combine_backward<64, 2>(a, count_here, s);
        else if (d <= 2048) launch_combine_backward<256, 1>(a, count_here, s);
        else if (d <= 4096) launch_combine_backward<256, 2>(a, count_here, s);
        else if (d <= 8192) launch_combine_backward<512, 2>(a, count_here, s);
        else launch_combine_backward<1024, 2>(a, count_here, s);
        if (const moe_status st = k.done()) return st;
    }
    return MOE_OK;
}
